"""Attention over a paged cache on the GPU, against the definition in float64
(tolerances: ops_reference.attention)."""
import pytest
import torch

import ops_reference as ref
import paged_reference as pr
from paper_2509_16248_amd import gm, ops
from paper_2509_16248_amd.ops import PagedCache, paged_attention

pytestmark = pytest.mark.gpu
NAN = float("nan")


def rand(shape, dtype, seed, size=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * size).to(pr.DT[dtype])


def slopes_of(H):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)])


def check_attention(call, dtype, hd, H, Hkv, seed=0, window=0, softcap=0.0, alibi=False, size=1.0,
                    extra=0, spoil=True, change=None, scale=None):
    """``spoil``: every place that no sequence holds is NaN."""
    q = rand((*call.tokens(extra), H, hd), dtype, seed + 1, size)
    kp = rand((call.pages, Hkv, call.ps, hd), dtype, seed + 2, size)
    vp = rand((call.pages, Hkv, call.ps, hd), dtype, seed + 3)
    if spoil:
        held = torch.zeros(call.pages, call.ps, dtype=torch.bool)
        for b, length in enumerate(call.lengths):
            for p in range(max(0, min(length, call.cap))):
                at = call.place(b, p)
                if at is not None:
                    held[at] = True
        for x in (kp, vp):
            x.masked_fill_(~held[:, None, :, None], NAN)
    if change is not None:
        change(call, q, kp, vp)
    sl = slopes_of(H) if alibi else None
    args, kw = call.device_args()
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    got = paged_attention(q.cuda(), PagedCache.of(kp.cuda(), vp.cuda()), *args, **kw, window=window,
                          softcap=softcap, slopes=None if sl is None else sl.cuda(), out=out, scale=scale)
    want, tol = pr.attention(call, q, kp, vp, window, softcap, sl, scale=scale, out=out.new_full(q.shape, 7.0, device="cpu"))
    ref.check(got, want, tol, f"{dtype} hd{hd} {H}/{Hkv} ps{call.ps}")
    return got


TYPES = ["bf16", "f16", "f32"]


# ------------------------------------------------------------ a few tokens
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("n,H,Hkv", [(1, 3, 3), (1, 8, 2), (1, 16, 1), (1, 32, 1), (3, 4, 2), (5, 24, 4), (2, 34, 2)])
def test_heads_and_new_tokens(dtype, hd, n, H, Hkv):
    check_attention(pr.Call([150, 67], [n, n], 16, False), dtype, hd, H, Hkv)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_pages_and_lengths_at_their_edges(dtype, ps):
    for length in (0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257):
        check_attention(pr.Call([length, 260 - length], [1, 1], ps, False, width=-(-260 // ps), seed=length),
                        dtype, 64, 4, 2, seed=length)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
def test_long_sequences_are_cut_up(dtype, hd):
    check_attention(pr.Call([3000, 1411, 1], [1] * 3, 16, False), dtype, hd, 2, 1)
    check_attention(pr.Call([9000], [2], 64, False), dtype, hd, 4, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_long_sequence_among_short_ones(dtype):
    lengths = [30 + 11 * b for b in range(30)]
    lengths[13] = 7000
    check_attention(pr.Call(lengths, [1] * 30, 32, False), dtype, 64, 4, 2)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("B", [63, 64, 65, 130, 300])
def test_many_sequences(dtype, B):
    check_attention(pr.Call([(b * 37) % 400 for b in range(B)], [1] * B, 16, False, width=40), dtype, 32, 2, 2)


def test_a_table_much_wider_than_the_sequences():
    check_attention(pr.Call([5, 700], [1, 1], 16, False, width=4000), "bf16", 64, 2, 2)
    check_attention(pr.Call([5, 700], [1, 1], 16, False, width=4000), "f32", 64, 2, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("softcap,alibi", [(30.0, False), (0.0, True), (5.0, True)])
def test_scores_of_a_few_tokens(dtype, softcap, alibi):
    check_attention(pr.Call([200, 111], [2, 2], 16, False), dtype, 128, 8, 2, softcap=softcap, alibi=alibi, size=3.0)


# ------------------------------------------------------------ prompts and chunks
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (6, 2), (8, 1)])
def test_whole_prompts(dtype, hd, H, Hkv):
    for n in (33, 64, 130, 257):
        check_attention(pr.Call([n, n], [n, n], 16, False, seed=n), dtype, hd, H, Hkv)


@pytest.mark.parametrize("B,n,H,Hkv", [(1, 2700, 12, 12), (1, 1700, 24, 24), (3, 400, 40, 20), (1, 100, 257, 257),
                                       (257, 70, 1, 1), (100, 200, 2, 2), (2, 1000, 32, 32), (5, 180, 68, 17),
                                       (2, 1040, 32, 32)])
def test_prompts_of_one_round_of_blocks(B, n, H, Hkv):
    """More than one block of 128 rows for each of 256 workgroups, and at most two (and some more): the order
    they come in still has every row of every sequence."""
    check_attention(pr.Call([n + 7 * (b % 3) for b in range(B)], [n] * B, 16, False), "bf16", 32, H, Hkv)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ps", [16, 64, 256])
def test_chunks_behind_what_is_stored(dtype, ps):
    check_attention(pr.Call([700, 333], [100, 100], ps, False), dtype, 128, 4, 2)
    check_attention(pr.Call([700, 333, 65], [100, 333, 1], ps, True), dtype, 64, 4, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("softcap,alibi", [(30.0, False), (0.0, True), (5.0, True)])
def test_scores_of_prompts(dtype, softcap, alibi):
    check_attention(pr.Call([300, 222], [150, 150], 32, False), dtype, 128, 4, 4, softcap=softcap, alibi=alibi, size=2.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_rows_of_every_kind(dtype):
    """Single tokens over long caches, chunks, whole prompts, idle sequences, and rows
    behind the last one, which keep what they hold."""
    new = [1, 200, 0, 33, 1, 7, 90, 0, 16, 17]
    lengths = [2500, 200, 900, 500, 1, 7, 1600, 0, 40, 41]
    got = check_attention(pr.Call(lengths, new, 16, True), dtype, 64, 4, 2, extra=9)
    assert (got[sum(new):] == 7.0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B", [64, 65, 130])
def test_many_packed_sequences(dtype, B):
    check_attention(pr.Call([(b * 37) % 90 + 40 for b in range(B)], [(b * 13) % 37 for b in range(B)], 16, True),
                    dtype, 32, 4, 2)
    check_attention(pr.Call([(b * 37) % 90 + 40 for b in range(B)], [b % 2 for b in range(B)], 16, True), dtype, 32, 2, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n", [9, 16, 17, 24, 25, 32, 33, 41])
def test_blocks_with_rows_for_some_wavefronts(dtype, n):
    """36 to 164 rows of a key head: the last block has them for one to four wavefronts of 32."""
    check_attention(pr.Call([700, n, n + 70], [n] * 3, 16, False), dtype, 64, 8, 2)
    check_attention(pr.Call([1500, 90], [n, n], 32, False), dtype, 128, 4, 1, window=100)
    check_attention(pr.Call([1500, 90], [n, 8], 32, True), dtype, 32, 4, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunks_of_few_blocks_are_cut_up(dtype):
    check_attention(pr.Call([5000], [40], 64, False), dtype, 128, 2, 2)
    check_attention(pr.Call([5000, 1100, 300], [40, 90, 100], 64, True), dtype, 64, 2, 1)


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_single_tokens_and_a_chunk_among_them(dtype):
    new = [1] * 200
    check_attention(pr.Call([(b * 37) % 300 + 1 for b in range(200)], new, 16, True), dtype, 64, 4, 2)
    new[77] = 150
    check_attention(pr.Call([(b * 37) % 300 + n for b, n in enumerate(new)], new, 16, True), dtype, 64, 4, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 50])
def test_packed_rows_before_the_first_sequence(dtype, n):
    """offsets may begin behind row 0: rows before it are no sequence's."""
    call = pr.Call([150, 99], [n, n], 16, False)
    cache, q = pools(call, dtype, 2, 64), rand((4 + 2 * n, 4, 64), dtype, 9).cuda()
    (table, lengths), _ = call.device_args()
    out = torch.full_like(q, 7.0)
    paged_attention(q, cache, table, lengths, offsets=torch.tensor([4, 4 + n, 4 + 2 * n], dtype=torch.int32, device="cuda"), out=out)
    want = paged_attention(q[4:], cache, table, lengths, offsets=torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"))
    assert (out[:4] == 7.0).all() and torch.equal(out[4:], want)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("n", [1, 60])
def test_a_scale_of_its_own(dtype, n):
    check_attention(pr.Call([200, 77], [n, n], 16, False), dtype, 64, 4, 2, scale=0.5)
    check_attention(pr.Call([200, 77], [n, n], 16, False), dtype, 64, 4, 2, scale=1e-3, softcap=2.0)


# ------------------------------------------------------------ windows and holes
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 64, 100, 1000])
def test_windows(dtype, window):
    check_attention(pr.Call([400, 93], [1, 1], 16, False), dtype, 64, 4, 2, window=window)
    check_attention(pr.Call([400, 93], [6, 6], 16, False), dtype, 64, 4, 2, window=window)
    check_attention(pr.Call([400, 333], [170, 170], 32, False), dtype, 64, 4, 2, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_window_over_a_long_cache(dtype):
    check_attention(pr.Call([9000, 2500], [5, 5], 32, False), dtype, 128, 8, 2, window=1024)
    check_attention(pr.Call([9000, 2500], [1, 77], 32, True), dtype, 128, 8, 2, window=700, alibi=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 4, 60])
def test_holes(dtype, n):
    """Pages given back before the window, in the middle, entries that are no page, and a
    sequence of nothing but holes."""
    width = 13
    holes = [(0, i, -1) for i in range(3)] + [(0, 7, 10 ** 9), (0, 11, -7)] + [(1, i, -1) for i in range(width)]
    holes += [(2, i, -2 ** 31) for i in range(5, width)]       # past its length
    call = pr.Call([200, 190, 75], [n] * 3, 16, False, width=width, holes=holes)
    got = check_attention(call, dtype, 64, 4, 2)
    assert not got[1].any()
    check_attention(call, dtype, 128, 4, 4, window=64)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 50])
def test_rows_that_see_nothing(dtype, n):
    """Lengths of zero, below zero and below the new tokens."""
    got = check_attention(pr.Call([0, -3, 2, 90], [n] * 4, 16, False), dtype, 64, 4, 2)
    assert not got[:2].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 50])
def test_lengths_past_the_table(dtype, n):
    check_attention(pr.Call([70, 64 + n, 30 + n], [n] * 3, 16, False, width=4), dtype, 64, 2, 2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 4, 50])
@pytest.mark.parametrize("packed", [False, True])
def test_lengths_of_any_size(dtype, n, packed):
    """Past the table by far: without a window such tokens see all of it, with the weights of
    those right behind it, and with one nothing."""
    lengths = [2 ** 31 - 1, 2 ** 30 + 64 + n, 2 ** 25, 64 + n]
    check_attention(pr.Call(lengths, [n] * 4, 16, packed, width=4), dtype, 64, 4, 2)
    for width in (4, 200):                                     # (whole items, and cut ones)
        call = pr.Call(lengths[:3], [n] * 3, 16, packed, width=width)
        cache, q = pools(call, dtype, 2, 64), rand((*call.tokens(), 4, 64), dtype, 9).cuda()
        (table, far), kw = call.device_args()
        near = torch.full_like(far, call.cap + n)
        biased = dict(slopes=slopes_of(4).cuda(), **kw)
        want = paged_attention(q, cache, table, near, **biased)
        assert want.any() and torch.equal(paged_attention(q, cache, table, far, **biased), want)
        for window in (1, 16, 1000, 1 << 24):
            out = paged_attention(q, cache, table, far, window=window, out=torch.full_like(q, 7.0), **biased)
            assert not out.any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [4, 60])
def test_inf_and_nan_reach_only_who_sees_them(dtype, n):
    """The last token's key and value are seen by its own query alone, a window's first
    by the first query alone."""
    def change(call, q, kp, vp):
        for b, p, x, value in ((0, 149, vp, NAN), (1, 119, kp, NAN), (2, 99, vp, float("inf"))):
            at = call.place(b, p)
            x[at[0], 0, at[1], 5] = value

    call = pr.Call([150, 120, 100], [n] * 3, 16, False)
    got = check_attention(call, dtype, 64, 4, 2, change=change).cpu()
    assert torch.isfinite(got[:, :-1].float()).all()
    assert torch.isnan(got[0, -1, 0, 5]) and torch.isfinite(got[0, -1, 2:].float()).all()

    def first(call, q, kp, vp):
        at = call.place(0, 150 - n - 19)                       # the last one that query 0 sees
        vp[at[0], 1, at[1], 7] = NAN

    got = check_attention(call, dtype, 64, 4, 2, change=first, window=20).cpu()
    assert torch.isnan(got[0, 0, 2:, 7]).all() and torch.isfinite(got[0, 1:].float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 4, 60])
@pytest.mark.parametrize("where", ["last token", "before the window", "seen by all", "hole"])
def test_inf_and_nan_in_a_part_of_a_cut_row(dtype, n, where):
    """Long rows are cut along the keys; one of the parts holds the value that is not finite."""
    length, window = 5200, 4001 if where == "before the window" else 0
    call = pr.Call([length], [n], 16, False)
    call.table, call.pages = call.table + 1, call.pages + 1    # page 0 is nobody's: all of it NaN
    if where == "hole":
        call.table[0, 150:153] = torch.tensor([-1, 10 ** 6, -1], dtype=torch.int32)
        call.table[0, 290] = -1

    def change(call, q, kp, vp):
        p = {"last token": length - 1, "before the window": length - n - window, "seen by all": 2000}.get(where)
        if p is not None:
            at = call.place(0, p)
            vp[at[0], 0, at[1], 5] = float("inf")

    got = check_attention(call, dtype, 64, 4, 2, change=change, window=window).cpu()[0].float()
    rows = {"last token": slice(n - 1, n), "seen by all": slice(0, n)}.get(where, slice(0, 0))
    assert torch.isinf(got[rows, :2, 5]).all()
    assert int((~torch.isfinite(got)).sum()) == 2 * got[rows].shape[0]


@pytest.mark.parametrize("dtype,top", [("bf16", 3.3e38), ("f16", 65504.0), ("f32", 3.3e38)])
@pytest.mark.parametrize("n,length", [(1, 90), (40, 90), (1, 2600), (40, 2600)])
def test_averages_of_the_largest_values_are_finite(dtype, top, n, length):
    def change(call, q, kp, vp):
        vp.fill_(top)
        vp[:, :, ::2, ::3] *= -1

    got = check_attention(pr.Call([length], [n], 16, False), dtype, 64, 2, 2, change=change, spoil=False)
    assert torch.isfinite(got.float()).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_large_scores_move_the_maximum(dtype, n):
    def change(call, q, kp, vp):
        for p in range(0, call.lengths[0], 7):                 # scores that climb along the keys
            at = call.place(0, p)
            kp[at[0], :, at[1]] *= 1.0 + p / 20.0

    check_attention(pr.Call([300], [n], 16, False), dtype, 64, 2, 2, change=change, size=2.0)


# ------------------------------------------------------------ how it is called
def pools(call, dtype, Hkv, hd, seed=0):
    return PagedCache.of(*(rand((call.pages, Hkv, call.ps, hd), dtype, seed + s).cuda() for s in (2, 3)))


@pytest.mark.parametrize("n", [1, 50])
def test_strided_queries_outputs_and_tables(n):
    H, Hkv, hd, call = 8, 2, 64, pr.Call([120, 77], [n, n], 16, False)
    cache = pools(call, "bf16", Hkv, hd)
    wide = rand((2, n, H + 4, hd + 8), "bf16", 1).cuda()
    q = wide[:, :, 2:2 + H, 8:]
    (table, lengths), _ = call.device_args()
    want = paged_attention(q.contiguous(), cache, table, lengths)
    buf = torch.full((n, 2, H + 3, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    big = torch.full((2, call.width + 3), -1, dtype=torch.int32, device="cuda")
    big[:, 1:1 + call.width] = table
    out = buf.transpose(0, 1)[:, :, 1:1 + H]
    got = paged_attention(q, cache, big[:, 1:1 + call.width], lengths, out=out)
    assert torch.equal(got, want) and (buf[:, :, 0] == 7).all() and (buf[:, :, 1 + H:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_and_padded_calls_agree(dtype):
    """The same tokens in rows of one length and packed."""
    for n in (1, 6, 70):
        call = pr.Call([150, 99, 70], [n] * 3, 16, False)
        cache, q = pools(call, dtype, 2, 64), rand((3, n, 4, 64), dtype, 9).cuda()
        (table, lengths), _ = call.device_args()
        offsets = torch.arange(0, 3 * n + 1, n, dtype=torch.int32, device="cuda")
        a = paged_attention(q, cache, table, lengths)
        b = paged_attention(q.reshape(3 * n, 4, 64), cache, table, lengths, offsets=offsets)
        torch.testing.assert_close(a.reshape(3 * n, 4, 64), b, rtol=2.0 ** -6, atol=2.0 ** -7)


@pytest.mark.parametrize("n,length", [(1, 5000), (5, 700), (80, 3000)])
def test_results_are_the_same_bits_every_time(n, length):
    call = pr.Call([length, length // 3], [n, n], 16, False)
    cache, q = pools(call, "bf16", 2, 128), rand((2, n, 8, 128), "bf16", 9).cuda()
    (table, lengths), _ = call.device_args()
    first = paged_attention(q, cache, table, lengths)
    for _ in range(5):
        assert torch.equal(first, paged_attention(q, cache, table, lengths))


def test_another_stream():
    call, s = pr.Call([3000, 700], [1, 1], 16, False), torch.cuda.Stream()
    cache, q = pools(call, "bf16", 2, 128), rand((2, 1, 8, 128), "bf16", 9).cuda()
    (table, lengths), _ = call.device_args()
    want = paged_attention(q, cache, table, lengths)
    torch.cuda.synchronize()
    got = paged_attention(q, cache, table, lengths, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own."""
    calls = [pr.Call([4000, 700], [1, 1], 16, False, seed=i) for i in range(2)]
    caches = [pools(c, "bf16", 2, 128, seed=10 * i) for i, c in enumerate(calls)]
    q = rand((2, 1, 8, 128), "bf16", 9).cuda()
    args = [c.device_args()[0] for c in calls]
    want = [paged_attention(q, c, *a) for c, a in zip(caches, args)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(paged_attention(q, caches[i], *args[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_offsets_past_32_bits():
    pages, ps, Hkv, hd = 4200, 256, 32, 128            # 2^32 elements lie before page 4096
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    k, v = (torch.zeros((pages, Hkv, ps, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = [rand((3, Hkv, ps, hd), "bf16", s).cuda() for s in (1, 2)]
    at = torch.tensor([5, 4150, 4199], device="cuda")
    k[at], v[at] = small
    cache, few = PagedCache.of(k, v), PagedCache.of(*small)
    lengths = torch.tensor([700], dtype=torch.int32, device="cuda")
    for n in (1, 50):
        q = rand((1, n, 32, hd), "bf16", 4).cuda()
        a = paged_attention(q, cache, at.int()[None], lengths)
        b = paged_attention(q, few, torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda"), lengths)
        assert torch.equal(a, b)


def test_wrong_calls_raise():
    cache = PagedCache(4, 16, 2, 64)
    t, n = torch.zeros((1, 3), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 1, 3, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(gm.GmError, match="multiple of the cache's heads"):
        paged_attention(q, cache, t, n)
    k = q[:, :, :2].contiguous()
    with pytest.raises(gm.GmError, match="every position"):
        cache.append(k, k, t, n, rotary=ops.rotary_table(40, 64))
    with pytest.raises(gm.GmError, match="window"):
        paged_attention(k, cache, t, n, window=-3)
    with pytest.raises(gm.GmError, match="overlap"):
        paged_attention(k, cache, t, n, out=k)
    with pytest.raises(ValueError, match="table must"):
        paged_attention(k, cache, t.cpu(), n)
    with pytest.raises(ValueError, match="q must be"):
        paged_attention(k.cpu(), cache, t, n)


def test_a_cache_whose_memory_was_replaced():
    t, n = torch.zeros((1, 3), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    q = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    cache = PagedCache(4, 16, 2, 64)
    cache.append(q, q, t, n)
    cache.v.resize_(400, 2, 16, 64)
    for call in (lambda: cache.append(q, q, t, n), lambda: paged_attention(q, cache, t, n)):
        with pytest.raises(ValueError, match="not where it was"):
            call()


def test_nothing_to_do():
    cache = PagedCache(4, 16, 2, 64)
    t = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    q = torch.zeros((0, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert paged_attention(q, cache, t, t[:, 0].contiguous()).shape == q.shape


def test_a_prompt_then_tokens_as_a_program_runs_them():
    """Prompts packed, then decode steps captured in one graph with their append,
    against attention over the whole sequences, turned, at every step."""
    B, H, Hkv, hd, ps, steps = 3, 8, 2, 64, 16, 20
    prompt, cap = [37, 5, 64], 96
    rotary = ops.rotary_table(cap, hd)
    total = [n + steps for n in prompt]
    x = {n: [rand((t, heads, hd), "bf16", 10 * i + s).cuda() for i, t in enumerate(total)]
         for n, heads, s in (("q", H, 1), ("k", Hkv, 2), ("v", Hkv, 3))}
    cache = PagedCache(B * cap // ps, ps, Hkv, hd)
    order = torch.randperm(B * cap // ps, generator=torch.Generator().manual_seed(0)).int()
    table = order.reshape(B, cap // ps).cuda()
    lengths = torch.tensor(prompt, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 37, 42, 106], dtype=torch.int32, device="cuda")
    q, k, v = (torch.cat([t[:n] for t, n in zip(x[name], prompt)]) for name in "qkv")
    q = cache.append(k, v, table, lengths, offsets=offsets, rotary=rotary, q=q, q_out=q)
    out = paged_attention(q, cache, table, lengths, offsets=offsets)

    def turned(t):
        pos = torch.arange(t.shape[0])
        y = [pr.rotated(row.double(), *(r.cpu() for r in rotary), int(p))[0] for row, p in zip(t.cpu(), pos)]
        return torch.stack(y).to(t.dtype).cuda()

    full = {n: [turned(t) for t in x[n]] for n in "qk"}

    def whole(b, n):
        """Attention of sequence b's first n tokens, in float32, by the operator for prompts."""
        return ops.attention(*(t[None, :n].float() for t in (full["q"][b], full["k"][b], x["v"][b])), causal=True)[0]

    # turned queries and keys are bf16 on both sides, at most a step apart where roundings differ
    for b in range(B):
        torch.testing.assert_close(out[offsets[b]:offsets[b + 1]].float(), whole(b, prompt[b]), rtol=2.0 ** -6, atol=2.0 ** -5)
    q1, k1, v1 = (torch.zeros((B, 1, heads, hd), dtype=torch.bfloat16, device="cuda") for heads in (H, Hkv, Hkv))
    o1 = torch.zeros_like(q1)

    def step():
        paged_attention(cache.append(k1, v1, table, lengths, rotary=rotary, q=q1), cache, table, lengths, out=o1)

    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    lengths.zero_()                                            # (the warm-up and capture store nothing)
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    lengths.copy_(torch.tensor(prompt, dtype=torch.int32))
    for i in range(steps):
        lengths += 1
        for t, name in ((q1, "q"), (k1, "k"), (v1, "v")):
            t.copy_(torch.stack([y[n + i] for y, n in zip(x[name], prompt)])[:, None])
        g.replay()
        for b in range(B):
            want = whole(b, prompt[b] + i + 1)[-1]
            torch.testing.assert_close(o1[b, 0].float(), want, rtol=2.0 ** -6, atol=2.0 ** -5)


def test_graphs_of_two_calls_replayed_in_turn():
    """Captured calls keep workspaces of their own."""
    calls = [pr.Call([6000, 700], [1, 1], 16, False, seed=1), pr.Call([2500, 2000], [60, 60], 32, False, seed=2)]
    caches = [pools(c, "bf16", 2, 128, seed=10 * i) for i, c in enumerate(calls)]
    qs = [rand((2, c.new[0], 8, 128), "bf16", 9).cuda() for c in calls]
    args = [c.device_args()[0] for c in calls]
    outs = [torch.zeros_like(q) for q in qs]
    want = [paged_attention(q, c, *a) for q, c, a in zip(qs, caches, args)]
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            paged_attention(qs[i], caches[i], *args[i], out=outs[i])
    for _ in range(4):
        for i in (0, 1, 1, 0):
            outs[i].zero_()
            graphs[i].replay()
            eager = paged_attention(qs[i], caches[i], *args[i])
            assert torch.equal(outs[i], want[i]) and torch.equal(eager, want[i])
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_a_captured_call_follows_lengths_offsets_and_tables(dtype, packed):
    """What the arrays hold at each replay counts: sequences that grow, move to other pages, take
    other shares of the packed rows, or have none."""
    B, width, ps, H, Hkv, hd, total = 4, 250, 16, 4, 2, 64, 130
    cache = PagedCache.of(*(rand((B * width, Hkv, ps, hd), dtype, s).cuda() for s in (2, 3)))
    q = rand((total, H, hd) if packed else (B, 2, H, hd), dtype, 4).cuda()
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    lengths, offsets = torch.ones(B, dtype=torch.int32, device="cuda"), torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    kw = {"offsets": offsets} if packed else {}
    paged_attention(q, cache, table, lengths, out=out, **kw)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        paged_attention(q, cache, table, lengths, out=out, **kw)
    for i, (length, new) in enumerate([([4000, 3, 900, 60], [100, 1, 0, 29]), ([130, 4000, 4000, 2000], [1, 1, 1, 1]),
                                       ([0, 0, 0, 0], [0, 0, 0, 0]), ([150, 2, 3999, 700], [130, 0, 0, 0]),
                                       ([40, 41, 42, 43], [33, 32, 31, 34])]):
        table.copy_(torch.randperm(B * width, generator=torch.Generator().manual_seed(i)).reshape(B, width).int())
        lengths.copy_(torch.tensor(length, dtype=torch.int32))
        offsets.copy_(torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32))
        out.fill_(7.0)
        want = torch.full_like(q, 7.0)
        g.replay()
        paged_attention(q, cache, table, lengths, out=want, **kw)
        assert torch.equal(out, want), i
        if packed:
            assert (out[sum(new):] == 7.0).all()
        torch.cuda.synchronize()
