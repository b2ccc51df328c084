"""Attention over a quantised cache and attention with modified scores on the GPU,
against the definitions in float64 (tolerances: ops_reference.attention)."""
import pytest
import torch

import ops_reference as ref
from paper_2509_16248_amd import gm, ops
from paper_2509_16248_amd.ops import KvCache

pytestmark = pytest.mark.gpu


def rows(shape, dtype, seed, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * size).to(ref.DT[dtype])


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def slopes_of(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)])


# ------------------------------------------------------------ over the cache
def cached_case(dtype, bits, hd, B, Sq, H, Hkv, n, lengths, seed=0, softcap=0.0, alibi=False,
                mask=None, cap=None, size=1.0):
    q = rows((B, Sq, H, hd), dtype, seed + 1, size)
    k, v = rows((B, n, Hkv, hd), dtype, seed + 2, size), rows((B, n, Hkv, hd), dtype, seed + 3)
    c = KvCache(B, Hkv, cap or n, hd, bits=bits, masked=mask is not None)
    c.write(k.cuda(), v.cuda(), mask=None if mask is None else mask.cuda())
    sl = slopes_of(H) if alibi else None
    got = ops.cached_attention(q.cuda(), c, ints(lengths), softcap=softcap,
                               slopes=None if sl is None else sl.cuda())
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.cached(q, k, v, lengths, bits, softcap, sl, mask, tol=tol)
    ref.check(got, want, tol, f"{dtype} q{bits} hd{hd} {B}x{Sq}x{H}/{Hkv} n{n}")
    return got


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Sq,H,Hkv", [(1, 3, 3), (1, 8, 2), (1, 16, 1), (3, 4, 2), (5, 8, 8)])
def test_cached_heads_and_new_tokens(bits, dtype, hd, Sq, H, Hkv):
    cached_case(dtype, bits, hd, 2, Sq, H, Hkv, 150, [150, 67])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257])
def test_cached_lengths_at_the_edges(bits, dtype, length):
    cached_case(dtype, bits, 64, 2, 1, 4, 4, 260, [length, 260 - length], seed=length)


@pytest.mark.parametrize("bits,dtype", [(8, "bf16"), (4, "f16"), (4, "bf16"), (8, "f32")])
@pytest.mark.parametrize("softcap,alibi", [(30.0, False), (0.0, True), (5.0, True)])
def test_cached_scores(bits, dtype, softcap, alibi):
    cached_case(dtype, bits, 128, 2, 2, 8, 4, 200, [200, 111], softcap=softcap, alibi=alibi, size=3.0)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_cached_long_sequences_are_split(bits, dtype, hd):
    cached_case(dtype, bits, hd, 2, 1, 2, 1, 3000, [3000, 1411], cap=9000)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("bits,dtype", [(8, "bf16"), (4, "f16"), (4, "bf16"), (8, "f16")])
def test_cached_one_chunk_of_eight_wavefronts(bits, dtype, hd):
    # a capacity over 256 that one chunk holds; lengths that leave wavefronts without a
    # tile, end inside one and fill two rounds
    cached_case(dtype, bits, hd, 5, 3, 6, 2, 500, [500, 257, 33, 1, 0], cap=510, softcap=4.0)
    cached_case(dtype, bits, hd, 2, 1, 2, 2, 290, [289, 255], cap=290, alibi=True)


@pytest.mark.parametrize("heads", [4, 5])
@pytest.mark.parametrize("bits", [8, 4])
def test_cached_row_blocks_on_either_side_of_one_a_cu(bits, heads):
    # 64 sequences of 4 key heads are 256 row blocks (one chunk), of 5 are 320 (two)
    cached_case("bf16", bits, 128, 64, 1, 2 * heads, heads, 700, [700 - 11 * b for b in range(64)])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_cached_hidden_positions(bits, dtype):
    """Padded keys, a sequence with every key hidden, and Inf and NaN stored where
    the mask or the length hides them."""
    B, n, H, hd = 3, 140, 4, 64
    q = rows((B, 2, H, hd), dtype, 1)
    k, v = rows((B, n, H, hd), dtype, 2), rows((B, n, H, hd), dtype, 3)
    mask = torch.ones(B, n, dtype=torch.int32)
    mask[0, 10:30] = 0
    mask[1] = 0
    lengths = [100, 120, 137]
    for x in (k, v):
        x[0, 12, 0, 3] = float("nan")
        x[0, 13, 1, 40] = float("inf")
        x[0, 100:, 2] = float("nan")       # past the length
        x[1, :, 3] = float("-inf")
        x[2, 136, :, 9] = float("nan")     # the last token: the one before must not see it
    c = KvCache(B, H, n, hd, bits=bits, masked=True)
    c.write(k.cuda(), v.cuda(), mask=mask.cuda())
    got = ops.cached_attention(q.cuda(), c, ints(lengths))
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.cached(q, k, v, lengths, bits, valid=mask, tol=tol)
    assert torch.isfinite(want[:2]).all() and torch.isfinite(want[2, 0]).all()
    assert not got[1].any()
    ref.check(got[:2], want[:2], tol[:2])
    ref.check(got[2, 0], want[2, 0], tol[2, 0])
    assert torch.isnan(got[2, 1]).all()


def test_cached_lengths_past_the_cache_and_short_of_the_queries():
    B, n, H, hd = 3, 64, 2, 32
    q, k = rows((B, 4, H, hd), "bf16", 1), rows((B, n, H, hd), "bf16", 2)
    c = KvCache(B, H, n, hd, bits=8)
    c.write(k.cuda(), k.cuda())
    got = ops.cached_attention(q.cuda(), c, ints([1000, 2, -3]))
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.cached(q, k, k, [64, 2, 0], 8, tol=tol)      # 1000 counts as max_seq
    ref.check(got, want, tol)
    assert not got[1, :2].any() and not got[2].any()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_cached_sizes_far_from_one(dtype):
    """Queries, keys and values of magnitudes near the ends of the type's range."""
    B, n, H, hd = 1, 70, 2, 64
    big = 2.0 ** 14 if dtype == "f16" else 2.0 ** 60
    q = rows((B, 1, H, hd), "f32", 1)
    k, v = rows((B, n, H, hd), "f32", 2), rows((B, n, H, hd), "f32", 3)
    for fq, fk, fv in ((big, 1 / big, 1.0), (1 / big, big, big), (1.0, 1.0, 1 / big)):
        qq, kk, vv = ((x * f).to(ref.DT[dtype]) for x, f in ((q, fq), (k, fk), (v, fv)))
        vv[0, ::7] *= 2.0 ** -9                      # keys of very different value scales
        c = KvCache(B, H, n, hd, bits=8)
        c.write(kk.cuda(), vv.cuda())
        got = ops.cached_attention(qq.cuda(), c, ints([n]))
        tol = torch.zeros(qq.shape, dtype=torch.float64)
        want = ref.cached(qq, kk, vv, [n], 8, tol=tol)
        ref.check(got, want, tol, f"{dtype} {fq:g} {fk:g} {fv:g}")


def test_cached_strided_queries_and_outputs():
    B, Sq, H, hd, n = 2, 3, 4, 64, 50
    qkv = rows((B, Sq, 3 * H, hd), "bf16", 1).cuda()
    k = rows((B, n, H, hd), "bf16", 2)
    c = KvCache(B, H, n, hd, bits=4)
    c.write(k.cuda(), k.cuda())
    out = torch.zeros(B, H, Sq, hd, dtype=torch.bfloat16, device="cuda").transpose(1, 2)
    got = ops.cached_attention(qkv[:, :, :H], c, ints([n, 9]), out=out)
    assert got is out
    plain = ops.cached_attention(qkv[:, :, :H].contiguous(), c, ints([n, 9]))
    assert torch.equal(out, plain)
    assert ops.cached_attention(qkv[:0, :, :H], c, ints([])).shape == (0, Sq, H, hd)


def test_cached_graph_follows_the_lengths_and_two_graphs_do_not_share():
    B, H, hd, n = 2, 4, 128, 1500
    c = KvCache(B, H, n, hd, bits=4)
    k = rows((B, n, H, hd), "bf16", 2)
    c.write(k.cuda(), k.cuda())
    assert gm.gm_attention_cached_workspace(c.c, gm.GM_DTYPE_BF16, B, 1, H) > 0
    qs = [rows((B, 1, H, hd), "bf16", s).cuda() for s in (5, 6)]
    lengths = ints([1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for q in qs:
            ops.cached_attention(q, c, lengths)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ops.cached_attention(q, c, lengths))
        graphs.append(g)
    for L in ([700, 3], [1500, 1499], [0, 64]):
        lengths.copy_(torch.tensor(L))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for q, o in zip(qs, outs):
            assert torch.equal(o, ops.cached_attention(q, c, lengths)), L


def test_on_another_stream_repeats_bit_for_bit():
    B, H, hd, n = 2, 8, 128, 2000
    c = KvCache(B, H, n, hd, bits=8)
    k = rows((B, n, H, hd), "bf16", 2).cuda()
    q = rows((B, 1, H, hd), "bf16", 3).cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.write(k, k, stream=s)
    a = ops.cached_attention(q, c, ints([n, 777]), stream=s)
    b = ops.cached_attention(q, c, ints([n, 777]), stream=s)
    p = ops.attention(q, k, k, stream=s)
    s.synchronize()
    assert torch.equal(a, b) and p.shape == q.shape


# ------------------------------------------------------------ whole prompts
def prompt_case(dtype, hd, B, Sq, Sk, H, Hkv, seed=0, what="", size=1.0, device_only=(), **kw):
    q = rows((B, Sq, H, hd), dtype, seed + 1, size)
    k, v = rows((B, Sk, Hkv, hd), dtype, seed + 2, size), rows((B, Sk, Hkv, hd), dtype, seed + 3)
    dev = {n: x.cuda() if torch.is_tensor(x) else x for n, x in kw.items()}
    got = ops.attention(q.cuda(), k.cuda(), v.cuda(), **dev)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.prompt(q, k, v, tol=tol, **kw)
    ref.check(got, want, tol, f"{dtype} hd{hd} {B}x{Sq}/{Sk}x{H}/{Hkv} {what}")
    return got, want


SIZES = [(1, 1), (1, 7), (16, 16), (33, 33), (64, 64), (65, 129), (130, 130), (200, 300), (300, 200)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Sq,Sk", SIZES)
def test_prompt_lengths(dtype, hd, Sq, Sk):
    prompt_case(dtype, hd, 2, Sq, Sk, 4, 2, causal=True, softcap=20.0, what="causal cap")
    prompt_case(dtype, hd, 1, Sq, Sk, 2, 2, causal=False, slopes=slopes_of(2), what="open alibi")


def masks(name, B, Sq, Sk):
    g = torch.Generator().manual_seed(Sq * 1000 + Sk)
    kw = {"causal": "causal" in name or "prefix" in name}
    if "prefix" in name:
        kw["prefix"] = torch.tensor([(b * 41 + 17) % (Sk + 20) for b in range(B)], dtype=torch.int32)
    if "pads" in name:
        kw["key_mask"] = (torch.arange(Sk)[None] < torch.tensor([Sk - (b * 37) % Sk for b in range(B)])[:, None]).int()
    if "holes" in name:
        kw["key_mask"] = (torch.rand((B, Sk), generator=g) < 0.5).int()
        kw["key_mask"][0] = 0
    if "docs" in name:
        ids = torch.cumsum((torch.rand((B, Sk), generator=g) < 0.02).int(), 1).int()
        kw["k_doc"], kw["q_doc"] = ids, ids[:, Sk - Sq:].contiguous()
    if "mixed" in name:
        kw["k_doc"] = torch.randint(-2, 3, (B, Sk), generator=g, dtype=torch.int32)
        kw["q_doc"] = torch.randint(-2, 4, (B, Sq), generator=g, dtype=torch.int32)
    return kw


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 64), ("f16", 64), ("f16", 32), ("f32", 64)])
@pytest.mark.parametrize("name", ["prefix", "causal pads", "holes", "causal docs", "docs pads",
                                  "causal mixed", "prefix docs", "prefix pads", "mixed holes"])
def test_prompt_masks(dtype, hd, name):
    B, Sq, Sk = 3, 290, 290
    prompt_case(dtype, hd, B, Sq, Sk, 4, 4, what=name, softcap=10.0, slopes=slopes_of(4),
                **masks(name, B, Sq, Sk))


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("f16", 32), ("f32", 32)])
@pytest.mark.parametrize("S", [1, 2, 3, 4, 5, 62, 63, 64, 65, 67])
def test_prompt_masks_of_short_rows(dtype, hd, S):
    for name in ("pads", "mixed holes", "causal docs", "prefix pads"):
        prompt_case(dtype, hd, 2, S, S, 2, 1, what=name, **masks(name, 2, S, S))


@pytest.mark.parametrize("softcap", [1e-6, 0.5, 50.0, 50.5, 1024.0])
def test_caps_from_the_smallest_to_the_largest(softcap):
    for dtype in ("bf16", "f16"):
        prompt_case(dtype, 64, 1, 100, 100, 2, 2, what=f"cap {softcap}", softcap=softcap, size=4.0)
        cached_case(dtype, 8, 64, 1, 1, 2, 2, 100, [100], softcap=softcap, size=4.0)


def test_prompt_keys_past_the_tile_marks():
    """More keys than a workgroup keeps marks for (131072), masked and of several
    documents on both sides of that."""
    Sq, Sk = 130, 131072 + 5000
    g = torch.Generator().manual_seed(3)
    ids = (torch.arange(Sk) // 9000).int()[None]
    q_doc = torch.randint(0, 16, (1, Sq), generator=g, dtype=torch.int32)
    mask = (torch.rand((1, Sk), generator=g) < 0.9).int()
    prompt_case("bf16", 64, 1, Sq, Sk, 1, 1, what="long", k_doc=ids, q_doc=q_doc, key_mask=mask)
    prompt_case("bf16", 64, 1, Sq, Sk, 1, 1, what="long, causal", causal=True, key_mask=mask)


def test_cached_very_long_sequences():
    cached_case("bf16", 4, 64, 1, 2, 2, 1, 70001, [70001], alibi=True)
    cached_case("f32", 8, 32, 1, 1, 1, 1, 70001, [69999])


def test_capture_on_a_stream_given_to_the_call():
    B, H, hd, n = 2, 4, 64, 3000
    c = KvCache(B, H, n, hd, bits=8)
    k = rows((B, n, H, hd), "bf16", 2).cuda()
    q = rows((B, 1, H, hd), "bf16", 3).cuda()
    lengths = ints([n, 500])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.write(k, k)
        ops.cached_attention(q, c, lengths)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = ops.cached_attention(q, c, lengths, stream=s)
        full = ops.attention(q, k, k, stream=s)
    for L in ([1, 2], [3000, 2999]):
        lengths.copy_(torch.tensor(L))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.cached_attention(q, c, lengths))
        assert torch.equal(full, ops.attention(q, k, k))


def test_prompt_many_documents_over_many_tiles():
    B, Sq, Sk = 1, 700, 1100
    prompt_case("bf16", 64, B, Sq, Sk, 4, 1, what="docs", causal=True, **{
        k: v for k, v in masks("docs", B, Sq, Sk).items() if k != "causal"})
    # documents out of order: every tile range overlaps, few pairs match
    ids = torch.randperm(Sk, generator=torch.Generator().manual_seed(1)).int()[None] % 50
    prompt_case("bf16", 64, B, Sq, Sk, 4, 1, what="shuffled docs",
                k_doc=ids, q_doc=ids[:, -Sq:].contiguous())


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 64), ("f16", 32), ("f32", 128)])
def test_prompt_hidden_inf_and_nan(dtype, hd):
    """Inf and NaN in keys and values reach exactly the queries that see them."""
    B, S, H = 2, 150, 2
    q, k, v = (rows((B, S, H, hd), dtype, s) for s in (1, 2, 3))
    mask = torch.ones(B, S, dtype=torch.int32)
    mask[0, 20:25] = 0
    for x in (k, v):
        x[0, 20:25, :, 1] = torch.tensor([float("nan"), float("inf"), float("-inf"), 65504.0, float("nan")])[:, None].to(x.dtype)
    v[1, 100, 0, 3] = float("inf")
    v[1, 140, 1, 0] = float("nan")
    got = ops.attention(q.cuda(), k.cuda(), v.cuda(), causal=True, softcap=15.0, key_mask=mask.cuda())
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.prompt(q, k, v, causal=True, softcap=15.0, key_mask=mask, tol=tol)
    assert torch.isfinite(want[0]).all() and not torch.isfinite(want[1, 120, 0, 3])
    assert torch.isfinite(want[1, :100]).all()
    ref.check(got, want, tol, f"{dtype} hd{hd} Inf and NaN")


def test_prompt_rows_that_see_nothing():
    B, S, H, hd = 2, 140, 2, 64
    for dtype in ("bf16", "f32"):
        q, k, v = (rows((B, S, H, hd), dtype, s).cuda() for s in (1, 2, 3))
        # queries before the first key
        got = ops.attention(q, k, v, causal=True, q_offset=-70)
        assert not got[:, :70].any() and got[:, 70:].abs().sum(-1).ne(0).all()
        # no key at all, a mask of zeros, a document nobody has
        assert not ops.attention(q, k[:, :0], v[:, :0]).any()
        assert not ops.attention(q, k, v, key_mask=ints([[0] * S] * B)).any()
        assert not ops.attention(q, k, v, q_doc=ints([[1] * S] * B), k_doc=ints([[2] * S] * B)).any()
        assert ops.attention(q[:, :0], k, v).shape == (B, 0, H, hd)


def test_prompt_offsets():
    for dtype, hd in (("bf16", 64), ("f32", 32)):
        for off in (-5, 0, 7, 200):
            prompt_case(dtype, hd, 1, 90, 150, 2, 2, what=f"offset {off}", causal=True,
                        slopes=slopes_of(2), q_offset=off)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f16", 32), ("f32", 64)])
def test_prompt_views_and_orders(dtype, hd):
    B, S, H = 2, 70, 3
    qkv = rows((B, S, 3 * H, hd), dtype, 1).cuda()
    q, k, v = qkv[:, :, :H], qkv[:, :, H:2 * H], qkv[:, :, 2 * H:]
    out = torch.zeros(B, H, S, hd, dtype=ref.DT[dtype], device="cuda").transpose(1, 2)
    ops.attention(q, k, v, causal=True, softcap=9.0, out=out)
    assert torch.equal(out, ops.attention(q.contiguous(), k.contiguous(), v.contiguous(), causal=True,
                                          softcap=9.0))
    # one head and one sequence broadcast
    kb = k[:1, :, :1].expand(B, S, H, hd)
    a = ops.attention(q, kb, kb)
    assert torch.equal(a, ops.attention(q, kb.contiguous(), kb.contiguous()))
    # sequence-major memory
    qs = q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(ops.attention(qs, kb, kb), a)


def test_prompt_capture_replays():
    B, S, H, hd = 2, 200, 4, 64
    q, k, v = (rows((B, S, H, hd), "bf16", s).cuda() for s in (1, 2, 3))
    pre = ints([0, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.attention(q, k, v, causal=True, prefix=pre)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = ops.attention(q, k, v, causal=True, prefix=pre)
    for p in ([3, 150], [200, 0], [64, 65]):
        pre.copy_(torch.tensor(p))
        q.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ops.attention(q, k, v, causal=True, prefix=pre))


# ------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,bits,H,Hkv,hd", [("bf16", 4, 8, 2, 128), ("f16", 8, 4, 4, 64),
                                                 ("f32", 8, 4, 2, 32)])
def test_prompt_then_tokens(dtype, bits, H, Hkv, hd):
    """A ragged prompt stored and attended to, then tokens one by one and a few at
    once: every step's output is the definition's over everything stored so far."""
    B, S, cap = 3, 90, 128
    g = dict(softcap=25.0, slopes=slopes_of(H))
    dev = dict(softcap=25.0, slopes=slopes_of(H).cuda())
    lens = [90, 41, 1]
    q, k, v = rows((B, S, H, hd), dtype, 1), rows((B, S, Hkv, hd), dtype, 2), rows((B, S, Hkv, hd), dtype, 3)
    c = KvCache(B, Hkv, cap, hd, bits=bits)
    c.write(k.cuda(), v.cuda(), count=ints(lens))
    # the prompt attends to the keys as the cache holds them
    kr, vr = c.read(S, count=ints(lens), dtype=ref.DT[dtype])
    mask = (torch.arange(S)[None] < torch.tensor(lens)[:, None]).int()
    got = ops.attention(q.cuda(), kr, vr, causal=True, key_mask=mask.cuda(), **dev)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    want = ref.prompt(q, kr.cpu(), vr.cpu(), causal=True, key_mask=mask, tol=tol, **g)
    ref.check(got, want, tol, "prompt")
    seq = [[k[b, :lens[b]], v[b, :lens[b]]] for b in range(B)]
    pos = ints(lens)
    for step, n in enumerate((1, 1, 4, 1)):
        qn, kn, vn = (rows((B, n, h, hd), dtype, 10 * step + s) for s, h in ((4, H), (5, Hkv), (6, Hkv)))
        c.write(kn.cuda(), vn.cuda(), pos)
        pos = pos + n
        got = ops.cached_attention(qn.cuda(), c, pos, **dev)
        for b in range(B):
            seq[b] = [torch.cat((seq[b][0], kn[b])), torch.cat((seq[b][1], vn[b]))]
            tol = torch.zeros((1, n, H, hd), dtype=torch.float64)
            want = ref.cached(qn[b:b + 1], seq[b][0][None], seq[b][1][None], [int(pos[b])], bits,
                              tol=tol, **g)
            ref.check(got[b:b + 1], want, tol, f"step {step} sequence {b}")


def test_wrapper_refusals_on_the_device():
    q = rows((1, 4, 4, 64), "bf16", 1).cuda()
    c = KvCache(1, 4, 64, 64)
    with pytest.raises(ValueError, match="shape"):
        ops.attention(q, q, q[:, :3])
    with pytest.raises(ValueError, match="must be torch.bfloat16"):
        ops.attention(q, q, q.half())
    with pytest.raises(ValueError, match="channels"):
        ops.attention(q.transpose(1, 3).contiguous().transpose(1, 3), q, q)
    with pytest.raises(ValueError, match="key_mask"):
        ops.attention(q, q, q, key_mask=ints([[1] * 3]))
    with pytest.raises(ValueError, match="slopes"):
        ops.attention(q, q, q, slopes=torch.ones(4, device="cuda").double())
    with pytest.raises(gm.GmError, match="16-byte"):
        ops.attention(torch.zeros(1 * 4 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(1, 4, 4, 64), q, q)
    with pytest.raises(gm.GmError, match="overlap"):
        ops.attention(q, q, q, out=q.new_zeros(1, 1, 4, 64).expand(1, 4, 4, 64))
    with pytest.raises(ValueError, match="head_dim"):
        ops.cached_attention(q[..., :32], c, ints([3]))
    with pytest.raises(ValueError, match="lengths"):
        ops.cached_attention(q, c, ints([3, 4]))
    with pytest.raises(ValueError, match="batch"):
        c.write(q.expand(2, 4, 4, 64), q.expand(2, 4, 4, 64))
    with pytest.raises(gm.GmError, match="valid bytes"):
        c.write(q, q, mask=ints([[1] * 4]))
