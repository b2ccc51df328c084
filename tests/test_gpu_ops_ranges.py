"""The attention and KV-cache operators at the ends of the ranges they accept,
against the definitions in float64 (tolerances: ops_reference.attention)."""
import pytest
import torch

import ops_reference as ref
from paper_2509_16248_amd import ops
from paper_2509_16248_amd.ops import KvCache

pytestmark = pytest.mark.gpu


def rows(shape, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * size).to(ref.DT[dtype])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("exponent", [-119, -123, -127, -131])
def test_cached_values_of_the_smallest_scales(bits, hd, exponent):
    """Value scales down to the smallest subnormals: alone, next to groups of zeros,
    next to hidden positions, and before tiles of ordinary values.

    A weight is p s 16 / b in fp16, b a power of two that is at most twice the largest
    scale met or, for scales as small as these, 2^-123.  Half a step of fp16's subnormals,
    2^-25, then stands for 2^-25 2^-123 / 16 = 2^-152, times a code of at most 2^7 for each
    of n keys: n 2^-145 on top of the tolerance."""
    B, n, H = 1, 600, 2
    q, k = rows((B, 1, H, hd), "bf16", 1), rows((B, n, H, hd), "bf16", 2)
    tiny = rows((B, n, H, hd), "f32", 3) * 2.0 ** exponent
    zeros, later = tiny.clone(), tiny.clone()
    zeros[:, 1::3] = 0
    later[:, 256:] *= 2.0 ** (-exponent)          # every wavefront's first tile is tiny
    mask = torch.ones(B, n, dtype=torch.int32)
    mask[:, 2::5] = 0
    for what, v, m in (("alone", tiny, None), ("zeros", zeros, None), ("hidden", tiny, mask),
                       ("later", later, None), ("later, hidden", later, mask)):
        v = v.to(torch.bfloat16)
        for cap in (n, 40000):                    # one chunk, and several with a merge
            c = KvCache(B, H, cap, hd, bits=bits, masked=m is not None)
            c.write(k.cuda(), v.cuda(), mask=None if m is None else m.cuda())
            for length in (n, 100):
                got = ops.cached_attention(q.cuda(), c, torch.tensor([length], dtype=torch.int32).cuda())
                tol = torch.zeros(q.shape, dtype=torch.float64)
                want = ref.cached(q, k, v, [length], bits, valid=m, tol=tol)
                tol += n * 2.0 ** -145
                ref.check(got, want, tol, f"2^{exponent} q{bits} hd{hd} {what} cap {cap} length {length}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_finite_groups_up_to_the_largest_number_read_back(bits, dtype):
    """Groups whose largest element is near the end of the type's range, with zeros and
    both signs: every stored value is code * scale, Inf only where that product is."""
    tops = [2.9e38, 3.0e38, 3.2e38, 3.38e38, 3.3895e38]
    x = torch.linspace(-1, 1, 32, dtype=torch.float64).repeat(len(tops), 1)
    x *= torch.tensor(tops, dtype=torch.float64)[:, None]
    x[:, 5], x[:, 9], x[:, 20] = 0, 1e30, -1e36
    x = x.to(ref.DT[dtype])[None, :, None]
    assert torch.isfinite(x).all()
    c = KvCache(1, 1, 64, 32, bits=bits)
    c.write(x.cuda(), (-x).cuda())
    k, v = c.read(len(tops), dtype=ref.DT[dtype])
    want = ref.stored(x, bits).to(ref.DT[dtype])
    # (Q * scale may round to Inf, scale having been rounded up; no smaller code's value does)
    smaller = ref.quantise(x, bits)[0].abs() < (127 if bits == 8 else 7)
    assert smaller.any() and torch.isfinite(want[smaller]).all()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)


@pytest.mark.parametrize("softcap", [0.0, 30.0])
@pytest.mark.parametrize("dtype,scale", [("bf16", 1e-37), ("f16", 1e-37), ("f32", 1e-37), ("bf16", 1e-30),
                                         ("f16", 1e-3), ("bf16", 1e30), ("f32", 1e30)])
def test_prompt_biases_under_any_scale(dtype, softcap, scale):
    """A distance bias next to products that a tiny scale makes vanish (or a large one
    lets dominate), where only far keys are visible."""
    B, S, H, hd = 1, 150, 2, 64
    size = 1e-16 if scale > 1 else 1.0            # scores of a size that a softmax tells apart
    q, k, v = rows((B, S, H, hd), dtype, 1, size), rows((B, S, H, hd), dtype, 2, size), rows((B, S, H, hd), dtype, 3)
    slopes = torch.tensor([1.0, 0.25])
    mask = (torch.arange(S) < 8).int()[None]
    kw = dict(causal=True, softcap=softcap, scale=scale)
    got = ops.attention(q.cuda(), k.cuda(), v.cuda(), slopes=slopes.cuda(), key_mask=mask.cuda(), **kw)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.prompt(q, k, v, slopes=slopes, key_mask=mask, tol=tol, **kw)
    assert want.abs().amax(-1).gt(0).all()
    ref.check(got, want, tol, f"{dtype} cap {softcap} scale {scale:g}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("softcap", [20.0, 50.0, 51.0])
@pytest.mark.parametrize("side", [-1, 1])
@pytest.mark.parametrize("exponent", [-100, 0, 100])
def test_capped_prompts_whose_scores_all_lie_at_one_end(dtype, softcap, side, exponent):
    """Every visible score near -cap or +cap, with small and large values: a softmax
    does not depend on what its scores have in common."""
    B, S, H, hd = 1, 140, 2, 64
    # scores near 1.2 times the cap before it
    size = (1.2 * softcap / hd ** 0.5) ** 0.5
    q = (size + rows((B, S, H, hd), "f32", 1) * 0.05).to(ref.DT[dtype])
    k = (side * size + rows((B, S, H, hd), "f32", 2) * 0.5).to(ref.DT[dtype])
    v = rows((B, S, H, hd), dtype, 3, 2.0 ** exponent)
    for causal in (True, False):
        got = ops.attention(q.cuda(), k.cuda(), v.cuda(), causal=causal, softcap=softcap)
        tol = torch.zeros(q.shape, dtype=torch.float64)
        want = ref.prompt(q, k, v, causal=causal, softcap=softcap, tol=tol)
        ref.check(got, want, tol, f"{dtype} cap {softcap} side {side} 2^{exponent} causal {causal}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_operator_on_another_stream_gives_the_same_bits(dtype):
    B, H, hd, n = 2, 4, 64, 500
    k, v = rows((B, n, H, hd), dtype, 2).cuda(), rows((B, n, H, hd), dtype, 4).cuda()
    q = rows((B, n, H, hd), dtype, 3).cuda()
    lengths = torch.tensor([n, 77], dtype=torch.int32, device="cuda")
    here, there = (KvCache(B, H, n, hd, bits=8) for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    there.write(k, v, stream=s)
    a = [*there.read(n, dtype=ref.DT[dtype], stream=s),
         ops.cached_attention(q[:, :1], there, lengths, stream=s),
         ops.attention(q, k, v, causal=True, softcap=30.0, stream=s)]
    here.write(k, v)
    b = [*here.read(n, dtype=ref.DT[dtype]), ops.cached_attention(q[:, :1], here, lengths),
         ops.attention(q, k, v, causal=True, softcap=30.0)]
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype,hd,H,Hkv", [("bf16", 128, 8, 2), ("f16", 64, 4, 4), ("f32", 32, 4, 1)])
@pytest.mark.parametrize("Sq,lengths", [(64, [300, 64, 70]), (129, [299, 129, 40]), (256, [256, 300, 0])])
def test_cached_chunks_of_tokens(bits, dtype, hd, H, Hkv, Sq, lengths):
    """A chunk of a prompt over what is stored, up to the whole cache: lengths equal to
    the chunk, one more, and short of it."""
    B, n = 3, 300
    q = rows((B, Sq, H, hd), dtype, 1)
    k, v = rows((B, n, Hkv, hd), dtype, 2), rows((B, n, Hkv, hd), dtype, 3)
    c = KvCache(B, Hkv, n, hd, bits=bits)
    c.write(k.cuda(), v.cuda())
    got = ops.cached_attention(q.cuda(), c, torch.tensor(lengths, dtype=torch.int32).cuda(), softcap=20.0)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.cached(q, k, v, lengths, bits, 20.0, tol=tol)
    ref.check(got, want, tol, f"{dtype} q{bits} hd{hd} {Sq}x{H}/{Hkv}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype,hd,ratio", [("bf16", 128, 2.0 ** 30), ("bf16", 32, 2.0 ** 60), ("f16", 64, 2.0 ** 22)])
@pytest.mark.parametrize("at", [0, 45, 301, 599])
def test_cached_large_values_of_no_weight(bits, dtype, hd, ratio, at):
    """A key whose values are far larger than the others', and whose weight is nothing:
    the others' values come out with all of their bits.

    A weight p s is held in fp16 in units of b / 16, b a power of two at most twice the
    largest weight: half a step of fp16's subnormals, 2^-25, is 2^-28 of that weight, times
    a code of at most Q, for each of n keys."""
    B, n, H = 1, 600, 2
    # scores: 0.8 |q| |k| cos with one key at -90 or so, against a spread of a few units
    q, k = rows((B, 1, H, hd), "f32", 1).abs() + 0.5, rows((B, n, H, hd), "f32", 2, 0.2)
    v = rows((B, n, H, hd), "f32", 3)
    if dtype == "f16":
        v = v * 2.0 ** -8
    # exp(-90) 2^60 of an ordinary value is 2^-69 of it
    k[:, at] = -90 / hd ** 0.5 * (q / (q * q).sum(-1, keepdim=True) * hd)[:, 0]
    v[:, at] *= ratio
    q, k, v = (x.to(ref.DT[dtype]) for x in (q, k, v))
    assert torch.isfinite(v).all()
    ks, vs = ref.stored(k, bits), ref.stored(v, bits)
    scores = torch.einsum("hc,nhc->hn", q[0, 0].double(), ks[0]) / hd ** 0.5
    assert (scores.amax(1) - scores[:, at]).min() > 80
    for cap in (n, 40000):                            # one chunk, and several with a merge
        c = KvCache(B, H, cap, hd, bits=bits)
        c.write(k.cuda(), v.cuda())
        got = ops.cached_attention(q.cuda(), c, torch.tensor([n], dtype=torch.int32).cuda())
        tol = torch.zeros((1, H, hd), dtype=torch.float64)
        want = ref.attention(q[0], ks[0], vs[0], torch.ones(1, n, dtype=torch.bool),
                             torch.zeros(1, n), hd ** -0.5, tol=tol)
        others = torch.arange(n) != at
        tol += n * 2.0 ** -28 * (1 + 2.0 ** -7) * vs[0, others].abs().max()
        ref.check(got[0], want, tol, f"{dtype} q{bits} hd{hd} at {at} cap {cap}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [32, 128])
@pytest.mark.parametrize("fq,fk,fv", [(120, -120, 0), (124, -120, -100), (-120, 120, 120), (60, -60, 0)])
def test_cached_fp32_sizes_far_from_one(bits, hd, fq, fk, fv):
    """Queries whose products with a code alone would pass fp32, and sizes at the other
    end, whose scores are ordinary."""
    B, n, H = 1, 70, 2
    q = rows((B, 2, H, hd), "f32", 1, 2.0 ** fq)
    k, v = rows((B, n, H, hd), "f32", 2, 2.0 ** fk), rows((B, n, H, hd), "f32", 3, 2.0 ** fv)
    q[:, 1] *= 2.0 ** -130 if fq > 100 else 1.0       # one row huge, one small
    assert torch.isfinite(q).all()
    for cap in (n, 40000):
        c = KvCache(B, H, cap, hd, bits=bits)
        c.write(k.cuda(), v.cuda())
        for softcap in (0.0, 3.0):
            got = ops.cached_attention(q.cuda(), c, torch.tensor([n], dtype=torch.int32).cuda(), softcap=softcap)
            tol = torch.zeros(q.shape, dtype=torch.float64)
            want = ref.cached(q, k, v, [n], bits, softcap, tol=tol)
            ref.check(got, want, tol, f"q{bits} hd{hd} 2^{fq} 2^{fk} 2^{fv} cap {cap} softcap {softcap}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("signs", [False, True])
def test_cached_values_near_the_largest_number(bits, hd, signs):
    """bf16 values near the end of the range, whose averages are finite, under scores
    that rise by less than a move of the running maximum and by more."""
    B, n, H = 1, 600, 2
    q = torch.full((B, 1, H, hd), hd ** -0.5).bfloat16()
    v = 3.2e38 - 1e37 * rows((B, n, H, hd), "f32", 3).abs().clamp(max=3.0)
    if signs:
        v = v * torch.sign(rows((B, n, H, hd), "f32", 4))
    v = v.bfloat16()
    for rise in (0.0, 5.0, 40.0):
        # a score is k's average times scale hd = hd ** 0.5 times it: from 0 to `rise`
        k = (torch.linspace(0, rise, n)[None, :, None, None] + rows((B, n, H, hd), "f32", 2, 0.1)).bfloat16()
        for cap in (n, 40000):                    # one chunk, and several with a merge
            c = KvCache(B, H, cap, hd, bits=bits)
            c.write(k.cuda(), v.cuda())
            got = ops.cached_attention(q.cuda(), c, torch.tensor([n], dtype=torch.int32).cuda(), scale=hd ** -0.5)
            tol = torch.zeros(q.shape, dtype=torch.float64)
            want = ref.cached(q, k, v, [n], bits, scale=hd ** -0.5, tol=tol)
            assert torch.isfinite(want.bfloat16()).all()
            ref.check(got, want, tol, f"q{bits} hd{hd} rise {rise} cap {cap}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_prompt_values_near_the_largest_number(dtype, hd, softcap):
    """Values whose sum passes fp32 and whose average does not, next to queries that see
    nothing and under masks."""
    B, S, H = 2, 150, 2
    q, k = rows((B, S, H, hd), dtype, 1), rows((B, S, H, hd), dtype, 2)
    v = (3.2e38 - 1e37 * rows((B, S, H, hd), "f32", 3).abs().clamp(max=3.0)).to(ref.DT[dtype])
    v[1] = (v[1].float() * torch.sign(rows((S, H, hd), "f32", 4))).to(ref.DT[dtype])
    mask = torch.ones(B, S, dtype=torch.int32)
    mask[0, :20], mask[1, 90:] = 0, 0
    v[1, 100, :, 3] = float("nan")                    # hidden
    got = ops.attention(q.cuda(), k.cuda(), v.cuda(), causal=True, softcap=softcap, key_mask=mask.cuda())
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.prompt(q, k, v, causal=True, softcap=softcap, key_mask=mask, tol=tol)
    assert torch.isfinite(want.to(ref.DT[dtype])).all() and not want[0, :20].any()
    ref.check(got, want, tol, f"{dtype} hd{hd} cap {softcap}")


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("signs", [False, True])
def test_cached_fp32_values_near_the_largest_number(bits, hd, signs):
    """As the bf16 test above, and where only some sequences, groups or keys are so large."""
    B, n, H = 2, 300, 2
    q, k = rows((B, 2, H, hd), "f32", 1), rows((B, n, H, hd), "f32", 2)
    v = 3.2e38 - 1e37 * rows((B, n, H, hd), "f32", 3).abs().clamp(max=3.0)
    if signs:
        v = v * torch.sign(rows((B, n, H, hd), "f32", 4))
    v[1, :150] *= 1e-30                               # later keys large
    v[1, :, :, hd - 32:] *= 2.0 ** -100               # a group of ordinary size
    for cap in (n, 40000):                            # one chunk, and several with a merge
        c = KvCache(B, H, cap, hd, bits=bits)
        c.write(k.cuda(), v.cuda())
        got = ops.cached_attention(q.cuda(), c, torch.tensor([n, 290], dtype=torch.int32).cuda())
        tol = torch.zeros(q.shape, dtype=torch.float64)
        want = ref.cached(q, k, v, [n, 290], bits, tol=tol)
        assert torch.isfinite(want.float()).all()
        ref.check(got, want, tol, f"q{bits} hd{hd} cap {cap}")
