"""PagedCache.append on the GPU against the definition in float64: keys turned by their
positions, values as they are, nothing else touched."""
import pytest
import torch

import ops_reference as ref
import paged_reference as pr
from paper_2509_16248_amd import ops
from paper_2509_16248_amd.ops import PagedCache

pytestmark = pytest.mark.gpu


def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(pr.DT[dtype])


def tables(positions, rot):
    return ops.rotary_table(positions, rot, device="cpu")


def check_append(call, dtype, hd, H, Hkv, rot=None, extra=0, in_place=False, seed=0, place=lambda x: x.cuda()):
    rot = hd if rot is None else rot
    shape = call.tokens(extra)
    k, v = rand((*shape, Hkv, hd), dtype, seed + 1), rand((*shape, Hkv, hd), dtype, seed + 2)
    kp, vp = (rand((call.pages, Hkv, call.ps, hd), dtype, seed + s) for s in (3, 4))
    q = rand((*shape, H, hd), dtype, seed + 5) if H else None
    q_out = None if q is None else q if in_place else rand((*shape, H, hd), dtype, seed + 6)
    rotary = tables(call.cap, rot) if rot else None
    cache = PagedCache.of(kp.cuda(), vp.cuda())
    args, kw = call.device_args()
    if rotary:
        kw["rotary"] = tuple(t.cuda() for t in rotary)
    if H:
        kw["q"] = place(q)
        kw["q_out"] = kw["q"] if in_place else q_out.cuda()
    got = cache.append(place(k), place(v), *args, **kw)
    want, tol = pr.append(call, k, v, kp, vp, rotary, q, q_out)
    for name, g, w, t in zip(("k", "v", "q"), (cache.k, cache.v, got), want, tol):
        ref.check(g, w, t, f"{name} {dtype} hd{hd}")
    return cache


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("packed", [False, True])
def test_types_and_heads(dtype, hd, packed):
    for H, Hkv, ps in ((3, 3, 16), (8, 2, 32), (1, 1, 256), (0, 5, 64)):
        new = [7, 1, 12] if packed else [7, 7, 7]
        check_append(pr.Call([40, 9, 300], new, ps, packed, seed=H), dtype, hd, H, Hkv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,rot", [(32, 0), (32, 16), (64, 16), (64, 48), (128, 64), (128, 96), (128, 112)])
def test_part_of_a_head_turns(dtype, hd, rot):
    check_append(pr.Call([90, 50], [20, 20], 16, False), dtype, hd, 4, 2, rot)


@pytest.mark.parametrize("heads", [(32, 8), (64, 64), (33, 1), (5, 40)])
def test_many_heads_go_round(heads):
    check_append(pr.Call([9, 30], [2, 3], 16, True), "bf16", 128, *heads)


@pytest.mark.parametrize("packed", [False, True])
def test_rows_of_no_place(packed):
    """Positions before the first (left padding, an idle sequence), past the table, and in
    holes; pages that are no pages."""
    holes = [(2, 1, -1), (2, 2, 10 ** 6), (2, 0, -2 ** 31)]
    call = pr.Call([3, 0, 60, 100, -5], [8] * 5, 16, packed, width=5, holes=holes)
    check_append(call, "bf16", 64, 4, 2)
    check_append(call, "f32", 32, 2, 2, in_place=True)


@pytest.mark.parametrize("packed", [False, True])
def test_lengths_of_any_size(packed):
    check_append(pr.Call([2 ** 31 - 1, -2 ** 31, 2 ** 30, 30], [8] * 4, 16, packed, width=5), "bf16", 64, 4, 2)


def test_empty_and_many_packed_sequences():
    new = [(b * 7) % 4 for b in range(150)]              # many of them without a token
    check_append(pr.Call([20 + b % 13 for b in range(150)], new, 16, True), "bf16", 64, 2, 1)
    check_append(pr.Call([5] * 64, [1] * 64, 16, True), "f16", 32, 1, 1)
    check_append(pr.Call([5] * 65, [0] * 64 + [5], 16, True), "f16", 32, 1, 1)


def test_packed_rows_before_the_first_sequence():
    call = pr.Call([20, 9], [5, 2], 16, True)
    k = rand((10, 2, 64), "bf16", 1).cuda()
    a, b = PagedCache(call.pages, 16, 2, 64), PagedCache(call.pages, 16, 2, 64)
    (table, lengths), kw = call.device_args()
    rotary = ops.rotary_table(call.cap, 64)
    want = a.append(k[3:], k[3:], table, lengths, q=k[3:], rotary=rotary, **kw)
    out = torch.full_like(k, 7.0)
    b.append(k, k, table, lengths, offsets=kw["offsets"] + 3, q=k, q_out=out, rotary=rotary)
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(out[3:], want) and (out[:3] == 7).all()


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_behind_the_last_sequence_are_left(in_place):
    check_append(pr.Call([30, 8], [5, 3], 16, True), "bf16", 64, 4, 2, extra=6, in_place=in_place)


def test_nothing_to_do():
    cache = PagedCache(4, 16, 2, 64)
    t = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    x = torch.zeros((0, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert cache.append(x, x, t, t[:, 0].contiguous(), q=x).shape == x.shape
    t = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    x = x.reshape(2, 0, 2, 64)
    cache.append(x, x, t, t[:, 0].contiguous())
    assert not cache.k.any()


def test_views_of_a_fused_projection():
    """q, k and v as slices of one [batch, tokens, (H + 2 Hkv) * hd] buffer, a strided table."""
    H, Hkv, hd, call = 8, 2, 64, pr.Call([40, 33, 12], [9, 9, 9], 16, False)
    fused = rand((3, 9, (H + 2 * Hkv), hd), "bf16", 1)
    kp, vp = (rand((call.pages, Hkv, 16, hd), "bf16", s) for s in (2, 3))
    dev = fused.cuda()
    cache = PagedCache.of(kp.cuda(), vp.cuda())
    (_, lengths), _ = call.device_args()
    wide = torch.full((3, call.width + 5), 77, dtype=torch.int32)
    wide[:, 2:2 + call.width] = call.table
    rotary = tables(call.cap, hd)
    q, k, v = fused[:, :, :H], fused[:, :, H:H + Hkv], fused[:, :, H + Hkv:]
    dq, dk, dv = dev[:, :, :H], dev[:, :, H:H + Hkv], dev[:, :, H + Hkv:]
    got = cache.append(dk, dv, wide.cuda()[:, 2:2 + call.width], lengths, q=dq, q_out=dq,
                       rotary=tuple(t.cuda() for t in rotary))
    want, tol = pr.append(call, k, v, kp, vp, rotary, q, q)
    for g, w, t in zip((cache.k, cache.v, got), want, tol):
        ref.check(g, w, t)
    assert torch.equal(dev[:, :, H:].cpu(), fused[:, :, H:])


def test_inf_nan_and_the_ends_of_the_range_pass():
    call = pr.Call([6], [6], 16, False)
    k = torch.zeros(1, 6, 1, 32, dtype=torch.bfloat16)
    k[0, 0, 0, 3], k[0, 1, 0, 20], k[0, 2, 0, 5] = float("nan"), float("inf"), 3e38
    k[0, 3, 0, 7] = 1e-39
    cache = PagedCache(call.pages, 16, 1, 32)
    args, _ = call.device_args()
    cache.append(k.cuda(), k.cuda(), *args)
    got = [t[int(call.table[0, 0]), 0, :6].cpu() for t in (cache.k, cache.v)]
    for g in got:
        assert torch.equal(g.view(torch.int16), k[0, :, 0].view(torch.int16))


def test_offsets_past_32_bits():
    pages, ps, Hkv, hd = 4200, 256, 32, 128            # 2^32 elements lie before page 4096
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    cache = PagedCache.of(*(torch.zeros((pages, Hkv, ps, hd), dtype=torch.bfloat16, device="cuda")
                            for _ in range(2)))
    k, v = rand((1, 3, Hkv, hd), "bf16", 1), rand((1, 3, Hkv, hd), "bf16", 2)
    table = torch.tensor([[7, 4190]], dtype=torch.int32, device="cuda")
    cache.append(k.cuda(), v.cuda(), table, torch.tensor([258], dtype=torch.int32, device="cuda"))
    for pool, x in ((cache.k, k), (cache.v, v)):
        assert torch.equal(pool[7, :, 255].cpu(), x[0, 0])
        assert torch.equal(pool[4190, :, :2].transpose(0, 1).cpu(), x[0, 1:])
        assert int((pool != 0).sum()) == int((x != 0).sum())


def test_a_captured_append_follows_its_inputs():
    """Replays store the tokens, lengths and pages that the buffers then hold."""
    B, Hkv, hd, ps = 3, 2, 64, 16
    cache, eager = PagedCache(20, ps, Hkv, hd), PagedCache(20, ps, Hkv, hd)
    rotary = ops.rotary_table(64, hd)
    k, v, q = (rand((B, 1, Hkv, hd), "bf16", s).cuda() for s in (1, 2, 3))
    table = torch.full((B, 4), -1, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    cache.append(k, v, table, lengths, rotary=rotary, q=q, q_out=out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cache.append(k, v, table, lengths, rotary=rotary, q=q, q_out=out)
    for step in range(20):
        lengths += 1
        if step % ps == 0:
            table[:, step // ps] = torch.tensor([3, 9, 14], dtype=torch.int32, device="cuda") + step // ps
        for t, s in ((k, 10), (v, 11), (q, 12)):
            t.copy_(rand(t.shape, "bf16", s + 3 * step))
        g.replay()
        want = eager.append(k, v, table, lengths, rotary=rotary, q=q)
        assert torch.equal(out, want) and torch.equal(cache.k, eager.k) and torch.equal(cache.v, eager.v)
        torch.cuda.synchronize()


def test_another_stream():
    call, s = pr.Call([40, 9], [7, 7], 16, False), torch.cuda.Stream()
    k, v = (rand((2, 7, 2, 64), "bf16", x).cuda() for x in (1, 2))
    args, _ = call.device_args()
    a, b = PagedCache(call.pages, 16, 2, 64), PagedCache(call.pages, 16, 2, 64)
    q0 = a.append(k, v, *args, q=k, rotary=ops.rotary_table(call.cap, 64))
    rotary = ops.rotary_table(call.cap, 64)
    torch.cuda.synchronize()
    q1 = b.append(k, v, *args, q=k, rotary=rotary, stream=s)
    s.synchronize()
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(q0, q1)
