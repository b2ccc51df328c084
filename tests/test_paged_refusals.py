"""What the operators over a paged cache refuse, on the host: bad arguments give
GM_E_INVAL (or ValueError from the torch wrappers) before anything is enqueued, so no GPU
is needed and the pointers are never looked at."""
import ctypes

import pytest
import torch

from paper_2509_16248_amd import gm, ops

P = 0x10000          # never dereferenced


def refused(call, message):
    with pytest.raises(gm.GmError) as e:
        call()
    assert e.value.code == gm.GM_E_INVAL
    assert message in str(e.value), str(e.value)


def cache(**kw):
    a = dict(dtype=1, pages=10, page_size=16, heads=4, head_dim=64, k=P, v=P << 1)
    a.update(kw)
    return gm.gm_paged_cache(**a)


def tensor(at=4 * P, **kw):
    a = dict(p=at, batch=8 * 4 * 64, token=4 * 64, head=64)
    a.update(kw)
    return gm.gm_tensor(**a)


def rows(**kw):
    a = dict(B=2, n=8, width=5, table_stride=5, table=P, lengths=P, offsets=None)
    a.update(kw)
    return gm.gm_paged_rows(**a)


def append(**kw):
    c = kw.pop("c", {})
    a = dict(cache=ctypes.pointer(cache(**c)), rows=rows(**kw.pop("r", {})), k=tensor(), v=tensor(8 * P),
             n_q_heads=4, rot=64, q=tensor(16 * P), q_out=tensor(32 * P), cos=P, sin=P, positions=80)
    a.update(kw)
    return gm.gm_paged_append_args(**a)


def attention(**kw):
    c = kw.pop("c", {})
    a = dict(cache=ctypes.pointer(cache(**c)), rows=rows(**kw.pop("r", {})), n_heads=4, window=0,
             q=tensor(16 * P), out=tensor(32 * P), scores=gm.gm_scores(0.125, 0.0, None), workspace=P,
             workspace_bytes=1 << 40)
    a.update(kw)
    return gm.gm_paged_attention_args(**a)


BAD = [
    (dict(c=dict(dtype=3)), "dtype"), (dict(c=dict(head_dim=96)), "head_dim"),
    (dict(c=dict(page_size=8)), "page_size"), (dict(c=dict(page_size=48)), "page_size"),
    (dict(c=dict(page_size=512)), "page_size"), (dict(c=dict(pages=0)), "must be positive"),
    (dict(c=dict(heads=0)), "must be positive"), (dict(c=dict(heads=(1 << 16) + 1)), "must be positive"),
    (dict(c=dict(k=None)), "NULL"), (dict(c=dict(v=P + 8)), "aligned"),
    (dict(r=dict(B=-1)), "B must"), (dict(r=dict(B=(1 << 20) + 1)), "B must"),
    (dict(r=dict(n=-1)), "n must"), (dict(r=dict(n=1 << 24)), "n must"),
    (dict(r=dict(width=0)), "width"), (dict(r=dict(width=(1 << 20) + 1)), "width"),
    (dict(r=dict(B=1 << 13, n=1 << 11)), "below 2^24"),
    (dict(r=dict(table=None)), "NULL"), (dict(r=dict(lengths=None)), "NULL"),
    (dict(r=dict(lengths=P + 2)), "4-byte"), (dict(r=dict(offsets=P + 1)), "4-byte"),
    (dict(r=dict(table_stride=-1)), "table_stride"), (dict(cache=None), "cache is NULL"),
]


@pytest.mark.parametrize("bad,message", BAD)
def test_caches_and_places(bad, message):
    big = dict(batch=1 << 30, token=256, head=64)      # (strides that hold any of these sizes)
    refused(lambda: gm.gm_paged_append(append(**bad, k=tensor(**big), v=tensor(8 * P, **big), q=tensor(16 * P, **big),
                                              q_out=tensor(32 * P, **big)), 0), message)
    refused(lambda: gm.gm_paged_attention(attention(**bad, q=tensor(16 * P, **big), out=tensor(32 * P, **big)), 0),
            message)


@pytest.mark.parametrize("kw,message", [
    (dict(k=tensor(p=None)), "NULL"), (dict(v=tensor(p=P + 8)), "16-byte"),
    (dict(k=tensor(token=250)), "multiples of 16 bytes"), (dict(v=tensor(head=-64)), "negative"),
    (dict(n_q_heads=-1), "n_q_heads"), (dict(q=tensor(p=None)), "NULL"), (dict(q_out=tensor(head=32)), "overlap"),
    (dict(q_out=tensor(token=0)), "overlap"), (dict(rot=8), "rot must"), (dict(rot=-16), "rot must"),
    (dict(rot=80), "rot must"), (dict(cos=None), "cos and sin"), (dict(sin=P + 4), "cos and sin"),
    (dict(positions=79), "every position"), (dict(k=tensor(P)), "the cache overlap"),
    (dict(v=tensor(P << 1)), "the cache overlap"), (dict(q_out=tensor()), "another tensor overlap"),
    (dict(q_out=tensor(P)), "another tensor overlap"),
    (dict(q_out=tensor(16 * P, batch=64 * 64, token=512)), "not another view"),
])
def test_append_refusals(kw, message):
    refused(lambda: gm.gm_paged_append(append(**kw), 0), message)


@pytest.mark.parametrize("kw,message", [
    (dict(n_heads=6), "multiple of the cache's heads"), (dict(n_heads=0), "multiple"),
    (dict(window=-1), "window"), (dict(window=(1 << 24) + 1), "window"), (dict(q=tensor(p=P + 2)), "16-byte"),
    (dict(out=tensor(32 * P, token=64)), "overlap"), (dict(out=tensor(16 * P)), "overlap"), (dict(out=tensor(P)), "overlap"),
    (dict(scores=gm.gm_scores(0.0, 0.0, None)), "scale"), (dict(scores=gm.gm_scores(float("inf"), 0.0, None)), "scale"),
    (dict(scores=gm.gm_scores(1.0, 2000.0, None)), "softcap"), (dict(scores=gm.gm_scores(1.0, 0.0, P + 1)), "slopes"),
])
def test_attention_refusals(kw, message):
    refused(lambda: gm.gm_paged_attention(attention(**kw), 0), message)


def test_query_rows_fit_a_launch():
    wide = dict(batch=1 << 40, token=1 << 20, head=64)
    for r, n_heads in ((dict(B=1 << 12, n=1 << 6), 64), (dict(B=1 << 18, n=100, offsets=P), 64)):
        refused(lambda: gm.gm_paged_attention(attention(r=r, n_heads=n_heads, q=tensor(16 * P, **wide),
                                                        out=tensor(32 * P, **wide)), 0), "below 2^24")
        assert gm.gm_paged_attention_workspace(cache(), r["B"], r["n"], 5, n_heads, 0, "offsets" in r) == 0


@pytest.mark.parametrize("n,packed", [(1, False), (200, False), (200, True), (8, True)])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_attention_needs_its_workspace(n, packed, dtype):
    c, width = dict(dtype=dtype, heads=1), 4096
    need = gm.gm_paged_attention_workspace(cache(**c), 1, n, width, 1, 0, packed)
    assert need > 0
    r = dict(B=1, n=n, width=width, offsets=P if packed else None)
    for workspace, size in ((None, need), (P + 8, need), (P, need - 1)):
        refused(lambda: gm.gm_paged_attention(attention(c=c, r=r, n_heads=1, workspace=workspace, workspace_bytes=size), 0),
                "workspace")


@pytest.mark.parametrize("B,n,width,H", [(0, 1, 5, 4), (1, 0, 5, 4), (1, 1, 0, 4), (1, 1, 5, 3), (1, 1, 5, 0),
                                         (-1, 1, 5, 4), (2147483647, 2147483647, 2147483647, 2147483647)])
def test_workspace_of_sizes_that_the_call_refuses(B, n, width, H):
    for packed in (False, True):
        assert gm.gm_paged_attention_workspace(cache(), B, n, width, H, 0, packed) == 0


def test_null_arguments_and_nothing_to_do():
    L = gm.lib()
    assert L.gm_paged_append(None, None) == gm.GM_E_INVAL
    assert L.gm_paged_attention(None, None) == gm.GM_E_INVAL
    assert L.gm_paged_attention_workspace(None, 1, 1, 1, 1, 0, 0) == 0
    none = tensor(p=None)
    for r in (dict(B=0, table=None, lengths=None), dict(n=0, table=None, lengths=None)):
        gm.gm_paged_append(append(r=r, k=none, v=none, q=none, q_out=none, cos=None), 0)
        gm.gm_paged_attention(attention(r=r, q=none, out=none), 0)


def test_wrappers_refuse_bad_caches():
    for bad in (dict(pages=0), dict(page_size=8), dict(page_size=24), dict(heads=0), dict(head_dim=80),
                dict(dtype=torch.int8), dict(dtype=torch.float64)):
        with pytest.raises(ValueError):
            ops.PagedCache(**{**dict(pages=4, page_size=16, heads=2, head_dim=64, device="cpu"), **bad})
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    for a, b in ((k, k[:3]), (k, k.half()), (k.transpose(1, 2), k.transpose(1, 2)), (k[0], k[0])):
        with pytest.raises(ValueError):
            ops.PagedCache.of(a, b)
    c = ops.PagedCache.of(k, k.clone())
    assert c.k is k and (c.pages, c.heads, c.page_size, c.head_dim) == (4, 2, 16, 64)
    with pytest.raises(ValueError, match="even"):
        ops.rotary_table(4, 3, device="cpu")


def test_wrappers_refuse_bad_calls():
    c = ops.PagedCache(4, 16, 2, 64, device="cpu")
    x, t, n = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="HIP device"):
        c.append(x, x, t, n)
    with pytest.raises(ValueError, match="HIP device"):
        ops.paged_attention(x, c, t, n)
    # what the compiled module refuses before any launch, here of a cache on the host
    M = gm.torch_lib()

    def attend(q=x, table=t, lengths=n, offsets=None, slopes=None, out=None, window=0, scale=0.1):
        return M.attention(c._address, c.k, q, table, lengths, offsets, window, 0.0, slopes, scale, out, 0)

    def append(q=x, table=t, lengths=n, offsets=None, v=None, cos=None, sin=None, queries=None, q_out=None):
        return M.append(c._address, c.k, q, q if v is None else v, table, lengths, offsets, cos, sin, queries, q_out, 0)

    for kw, message in [
        (dict(q=x[:, 0]), "without"), (dict(offsets=torch.zeros(3, dtype=torch.int32)), "with offsets"),
        (dict(table=t.long()), "int32"), (dict(table=t[0]), "table must"),
        (dict(table=torch.zeros(3, 2, dtype=torch.int32).t()), "table must"), (dict(table=t[:1]), "sequences"),
        (dict(lengths=n.long()), "lengths must"), (dict(lengths=n[:1]), "lengths must"),
        (dict(lengths=torch.zeros(4, dtype=torch.int32)[::2]), "lengths must"), (dict(lengths=None), "lengths is missing"),
        (dict(q=x[0], offsets=n), "offsets must"), (dict(q=x.half()), "must be BFloat16"),
        (dict(q=x[..., :32]), "must be BFloat16 of shape"), (dict(q=torch.zeros(2, 1, 64, 2, dtype=torch.bfloat16).transpose(2, 3)), "channels"),
    ]:
        for call in (attend, append):
            with pytest.raises(ValueError, match=message):
                call(**kw)
    with pytest.raises(ValueError, match="12 arguments"):
        M.append(1)
    with pytest.raises(TypeError, match="must be a tensor"):
        attend(q=[1.0])
    with pytest.raises(TypeError):
        attend(window=1.5)
    with pytest.raises(TypeError):
        attend(scale="x")
    for kw, message in [(dict(out=x.half()), "out must"), (dict(out=x[0]), "out must"), (dict(slopes=n), "slopes must"),
                        (dict(slopes=torch.zeros(3)), "slopes must")]:
        with pytest.raises(ValueError, match=message):
            attend(**kw)
    r = torch.zeros(48, 32)
    for kw, message in [
        (dict(v=x.half()), "v must"), (dict(v=x[..., :1, :]), "v must"), (dict(cos=r[0], sin=r), "cos must be"),
        (dict(cos=r, sin=r[1:]), "sin must"), (dict(cos=r.double(), sin=r), "cos must"), (dict(cos=r.t(), sin=r), "cos must"),
        (dict(queries=x[0]), "dimensions"), (dict(queries=x.half()), "q must"), (dict(queries=x[:1]), "q must"),
        (dict(q_out=x), "q_out needs q"), (dict(queries=x, q_out=x[:, :0]), "q_out must"),
    ]:
        with pytest.raises(ValueError, match=message):
            append(**kw)
    # codes of the C entry come back as numbers: a window below 0 and one past an int
    assert attend(window=-1) == gm.GM_E_INVAL and attend(window=1 << 40) == gm.GM_E_INVAL
    assert append(cos=r[:40], sin=r[:40]) == gm.GM_E_INVAL and b"every position" in gm.lib().gm_last_error()


def test_half_a_rotary_table():
    """cos and sin go together: neither is left out in silence."""
    M, c, r = gm.torch_lib(), ops.PagedCache(4, 16, 2, 64, device="cpu"), torch.zeros(48, 32)
    x, t, n = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="sin needs cos"):
        M.append(c._address, c._pools, x, x, t, n, None, None, r, None, None, 0)
    assert M.append(c._address, c._pools, x, x, t, n, None, r, None, None, None, 0) == gm.GM_E_INVAL


def test_a_cache_whose_memory_was_replaced():
    """Calls go by the addresses that k and v had when the cache was made."""
    M = gm.torch_lib()
    x, t, n = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)

    def made():
        k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
        return ops.PagedCache.of(k, k.clone())

    c = made()
    for name in ("k", "v"):
        with pytest.raises(AttributeError):
            setattr(c, name, torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16))
    other = torch.ones(9, 2, 16, 64, dtype=torch.bfloat16)
    for which in ("k", "v"):
        for replace in (lambda p: p.resize_(4000, 2, 16, 64), lambda p: p.set_(other), lambda p: setattr(p, "data", other)):
            c = made()
            # (a window below 0 is refused by the C entry, behind the check of the memory)
            assert M.attention(c._address, c._pools, x, t, n, None, -1, 0.0, None, 0.1, None, 0) == gm.GM_E_INVAL
            replace(getattr(c, which))
            with pytest.raises(ValueError, match="not where it was"):
                M.attention(c._address, c._pools, x, t, n, None, -1, 0.0, None, 0.1, None, 0)
            with pytest.raises(ValueError, match="not where it was"):
                M.append(c._address, c._pools, x, x, t, n, None, None, None, None, None, 0)


def test_rotary_tables():
    """Against the angles by Python's own arithmetic, rounded once: half a step of float32 of the
    value, and what an angle of up to 5000 loses in float64, 5000 * 2^-52."""
    import math
    cos, sin = ops.rotary_table(5000, 64, base=500.0, device="cpu")
    assert cos.shape == sin.shape == (5000, 32) and cos.dtype == sin.dtype == torch.float32
    assert (cos[0] == 1).all() and (sin[0] == 0).all()
    for p in (1, 77, 4999):
        for c in (0, 1, 17, 31):
            angle = p * 500.0 ** (-2 * c / 64)
            for got, want in ((cos, math.cos(angle)), (sin, math.sin(angle))):
                assert abs(float(got[p, c]) - want) <= 2.0 ** -24 * abs(want) + 4 * 5000 * 2.0 ** -52
    assert ops.rotary_table(0, 64, device="cpu")[0].shape == (0, 32)
    assert ops.rotary_table(8, 0, device="cpu")[1].shape == (8, 0)
