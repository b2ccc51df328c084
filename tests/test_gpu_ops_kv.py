"""KV cache in 8 and 4 bits on the GPU: stored rows, codes and scales against the
definition in float64, exactly (a code is the nearest integer of an exact
quotient, ties to even; a value is one product, rounded once)."""
import pytest
import torch

import ops_reference as ref
from paper_2509_16248_amd.ops import KvCache

pytestmark = pytest.mark.gpu


def rows(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g) * torch.exp(torch.randn(shape[:-1] + (1,), generator=g))
    return x.to(ref.DT[dtype])


def cache_codes(t, bits):
    """Codes [batch, positions, heads, hd] as the cache's own bytes hold them."""
    t = t.cpu()
    if bits == 4:
        t = torch.stack((t & 15, t >> 4), -1).flatten(-2)
    return (t.int() - (1 << (bits - 1))).permute(0, 2, 1, 3)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("B,n,H", [(1, 1, 1), (3, 1, 12), (2, 77, 3), (1, 130, 8)])
def test_rows_read_back_as_the_definition(bits, dtype, hd, B, n, H):
    k, v = rows((B, n, H, hd), dtype, 1), rows((B, n, H, hd), dtype, 2)
    c = KvCache(B, H, n + 5, hd, bits=bits)
    start = torch.arange(B, dtype=torch.int32, device="cuda") % 6
    c.write(k.cuda(), v.cuda(), start)
    for out_dtype in ("f32", dtype):
        got = c.read(n, start, dtype=ref.DT[out_dtype])
        for g, x in zip(got, (k, v)):
            assert torch.equal(g.cpu(), ref.stored(x, bits).to(ref.DT[out_dtype]))
    for held, scale, x in ((c.k, c.k_scale, k), (c.v, c.v_scale, v)):
        q, s = ref.quantise(x, bits)
        codes = cache_codes(held, bits)
        for b in range(B):
            p = int(start[b])
            assert torch.equal(codes[b, p:p + n].double(), q[b])
            assert torch.equal(scale[b, :, :, p:p + n].cpu().double().permute(2, 0, 1), s[b])


@pytest.mark.parametrize("bits", [8, 4])
def test_ties_subnormals_and_groups_of_zeros(bits):
    Q = 127 if bits == 8 else 7
    x = torch.zeros(1, 7, 1, 32)
    x[0, 0, 0, :8] = torch.tensor([Q, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, -Q])     # ties, scale 1
    x[0, 1] = x[0, 0] * 2.0 ** 100
    x[0, 2] = x[0, 0] * 2.0 ** -100
    x[0, 3] = x[0, 0] * 2.0 ** -132                                  # the scale is subnormal
    x[0, 4, 0, 3] = 1e-45                                            # the scale rounds to 0
    x[0, 5] = torch.randn(32, generator=torch.Generator().manual_seed(5)) * 3e38 / 4
    x[0, 6] = torch.randn(32, generator=torch.Generator().manual_seed(6)) * 2.0 ** -120
    c = KvCache(1, 1, 64, 32, bits=bits)
    c.write(x.cuda(), (-x).cuda())
    k, v = c.read(7, dtype=torch.float32)
    want = ref.stored(x, bits).float()
    # (row 5 holds an Inf, 3e38 times a normal, and reads as NaN)
    torch.testing.assert_close(k.cpu(), want, rtol=0, atol=0, equal_nan=True)
    torch.testing.assert_close(v.cpu(), -want, rtol=0, atol=0, equal_nan=True)
    # the largest scale is 1 up to its rounding, and ties went to the even code
    assert cache_codes(c.k, bits)[0, 0, 0, :8].tolist() == [Q, 0, 2, 2, 0, -2, -2, -Q]


@pytest.mark.parametrize("bits", [8, 4])
def test_a_group_with_inf_or_nan_reads_as_nan_and_only_that_group(bits):
    x = rows((1, 3, 2, 64), "bf16", 7)
    x[0, 0, 0, 5] = float("inf")
    x[0, 1, 1, 40] = float("nan")
    x[0, 2, 0, 63] = float("-inf")
    c = KvCache(1, 2, 64, 64, bits=bits)
    c.write(x.cuda(), x.cuda())
    k, _ = c.read(3, dtype=torch.float32)
    bad = torch.zeros(3, 2, 2, dtype=torch.bool)
    bad[0, 0, 0] = bad[1, 1, 1] = bad[2, 0, 1] = True
    groups = k.cpu()[0].unflatten(-1, (2, 32))
    assert torch.isnan(groups[bad]).all() and torch.isfinite(groups[~bad]).all()
    want = ref.stored(x, bits)[0].unflatten(-1, (2, 32))
    assert torch.equal(groups[~bad], want[~bad].float())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("hd", [32, 128])
def test_only_the_named_rows_change(bits, hd):
    B, n, H, cap = 3, 9, 2, 20
    c = KvCache(B, H, cap, hd, bits=bits, masked=True)
    full = rows((B, cap, H, hd), "bf16", 8).cuda()
    c.write(full, full)
    before = [t.clone() for t in c._tensors()]
    k, v = rows((B, n, H, hd), "bf16", 9).cuda(), rows((B, n, H, hd), "bf16", 10).cuda()
    # sequence 0: rows before 0 are dropped; 1: none; 2: rows past the capacity
    # (which the cache rounds up to 64) are dropped
    start = torch.tensor([-4, 3, 60], dtype=torch.int32, device="cuda")
    count = torch.tensor([7, 0, 9], dtype=torch.int32, device="cuda")
    mask = (torch.arange(B * n, device="cuda").view(B, n) % 3 != 0).int()
    c.write(k, v, start, count=count, mask=mask)
    stored = {0: range(4, 7), 1: range(0), 2: range(0, 4)}
    changed = torch.zeros(B, 64, dtype=torch.bool)
    for b in range(B):
        for i in stored[b]:
            changed[b, int(start[b]) + i] = True
    for t, old in zip(c._tensors(), before):
        if t is c.valid:
            assert torch.equal(t.cpu()[~changed], old.cpu()[~changed])
        elif t.dtype == torch.uint8:
            assert torch.equal(t.cpu().transpose(1, 2)[~changed], old.cpu().transpose(1, 2)[~changed])
        else:
            a, o = (u.cpu().view(torch.int16).permute(0, 3, 1, 2) for u in (t, old))
            assert torch.equal(a[~changed], o[~changed])
    gk, gv = c.read(n, start, count=count, dtype=torch.float32)
    for got, x in ((gk, k), (gv, v)):
        want = ref.stored(x, bits).float()
        for b in range(B):
            for i in range(n):
                if i in stored[b]:
                    assert torch.equal(got[b, i].cpu(), want[b, i])
                    assert int(c.valid[b, int(start[b]) + i]) == int(mask[b, i])
                else:
                    assert not got[b, i].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_of_a_fused_projection_and_other_orders(dtype):
    B, n, H, hd = 2, 19, 3, 64
    qkv = rows((B, n, 3 * H, hd), dtype, 11).cuda()
    k, v = qkv[:, :, H:2 * H], qkv[:, :, 2 * H:]
    c = KvCache(B, H, n, hd, bits=8)
    c.write(k, v)
    # read into tensors stored head-major, and into a slice of a wider one
    ok = torch.zeros(B, H, n, hd, dtype=ref.DT[dtype], device="cuda").transpose(1, 2)
    wide = torch.full((B, n, 2 * H, hd), 7.0, dtype=ref.DT[dtype], device="cuda")
    c.read(n, out=(ok, wide[:, :, :H]))
    assert torch.equal(ok.cpu(), ref.stored(k, 8).to(ref.DT[dtype]))
    assert torch.equal(wide[:, :, :H].cpu(), ref.stored(v, 8).to(ref.DT[dtype]))
    assert (wide[:, :, H:] == 7).all()
    # one head's rows given to every head
    c.write(k[:, :, :1].expand(B, n, H, hd), v)
    assert torch.equal(c.read(n, dtype=torch.float32)[0].cpu(),
                       ref.stored(k[:, :, :1], 8).float().expand(B, n, H, hd))


def test_fewer_sequences_than_the_cache_and_empty_calls():
    c = KvCache(4, 2, 64, 32, bits=4)
    x = rows((2, 5, 2, 32), "f16", 12).cuda()
    c.write(x, x)
    c.write(x[:0], x[:0])
    c.write(x[:, :0], x[:, :0])
    k, _ = c.read(5, batch=2, dtype=torch.float16)
    assert torch.equal(k.cpu(), ref.stored(x, 4).half())
    k, _ = c.read(5, dtype=torch.float16)
    assert not k[2:].any()
    assert c.read(0)[0].shape == (4, 0, 2, 32)


def test_offsets_past_32_bits():
    """A cache of 4.3 GB per operand: the last head's rows lie past 2^32 bytes."""
    H, cap, hd = 528, 64 * 1000, 128
    c = KvCache(1, H, cap, hd, bits=8)
    assert c.k.numel() > 1 << 32
    x = rows((1, 3, H, hd), "bf16", 13).cuda()
    start = torch.tensor([cap - 3], dtype=torch.int32, device="cuda")
    c.write(x, -x, start)
    k, v = c.read(3, start)
    want = ref.stored(x, 8).bfloat16()
    assert torch.equal(k.cpu(), want) and torch.equal(v.cpu(), -want)
    assert not c.read(1)[0].any()


def test_captured_append_replays_at_the_current_positions():
    B, H, hd = 2, 3, 64
    c = KvCache(B, H, 64, hd, bits=4)
    x = rows((B, 1, H, hd), "bf16", 14).cuda()
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = tuple(torch.empty(B, 4, H, hd, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.write(x, x, pos)
        c.read(4, out=out)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.write(x, x, pos)
        c.read(4, out=out)
    for t in range(4):
        new = rows((B, 1, H, hd), "bf16", 20 + t)
        x.copy_(new)
        pos.fill_(t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0][:, t].cpu(), ref.stored(new, 4).bfloat16()[:, 0])
    assert out[0].abs().sum(-1).ne(0).all()
