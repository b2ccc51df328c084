"""What the attention and KV-cache operators refuse, on the host: bad arguments
give GM_E_INVAL (or ValueError from the torch wrappers) before anything is
enqueued, so no GPU is needed and the pointers are never looked at."""
import ctypes

import pytest
import torch

from paper_2509_16248_amd import gm, ops

P = 0x10000          # never dereferenced


def cache(**kw):
    a = dict(bits=8, batch=2, heads=4, max_seq=128, head_dim=64, k=P, v=P, k_scale=P, v_scale=P,
             valid=None)
    a.update(kw)
    return gm.gm_kv_cache(**a)


def tensor(**kw):
    a = dict(p=P, batch=8 * 4 * 64, token=4 * 64, head=64)
    a.update(kw)
    return gm.gm_tensor(**a)


def refused(call, message):
    with pytest.raises(gm.GmError) as e:
        call()
    assert e.value.code == gm.GM_E_INVAL
    assert message in str(e.value), str(e.value)


BAD_CACHE = [
    (dict(bits=5), "bits must be 8 or 4"), (dict(head_dim=48), "head_dim"),
    (dict(max_seq=100), "multiple of 64"), (dict(max_seq=0), "multiple of 64"),
    (dict(max_seq=1 << 24), "below 2^24"), (dict(batch=0), "must be positive"),
    (dict(heads=-1), "must be positive"), (dict(k=None), "NULL"), (dict(v_scale=P + 2), "aligned"),
    (dict(valid=P + 4), "aligned"),
]


@pytest.mark.parametrize("bad,message", BAD_CACHE)
def test_bad_caches(bad, message):
    c = cache(**bad)
    refused(lambda: gm.gm_kv_write(c, 1, 2, 8, tensor(), tensor(), None, None, None, 0), message)
    refused(lambda: gm.gm_kv_read(c, 1, 2, 8, None, None, tensor(), tensor(), 0), message)
    refused(lambda: gm.gm_attention_cached(cached(cache=ctypes.pointer(c)), 0), message)
    assert gm.gm_attention_cached_workspace(c, 1, 2, 1, 4) == 0


@pytest.mark.parametrize("kw,message", [
    (dict(dtype=7), "dtype"), (dict(B=3), "batch"), (dict(B=-1), "batch"), (dict(n=-1), "n must"),
    (dict(n=1 << 24), "n must"), (dict(k=tensor(p=None)), "NULL"), (dict(k=tensor(p=P + 8)), "16-byte"),
    (dict(v=tensor(head=66)), "multiples of 16 bytes"), (dict(v=tensor(token=-256)), "negative"),
    (dict(k=tensor(batch=1 << 48)), "out of range"), (dict(start=P + 2), "4-byte"),
    (dict(mask=P), "valid bytes"),
])
def test_kv_write_refusals(kw, message):
    a = dict(dtype=1, B=2, n=8, k=tensor(), v=tensor(), start=None, count=None, mask=None)
    a.update(kw)
    refused(lambda: gm.gm_kv_write(cache(), a["dtype"], a["B"], a["n"], a["k"], a["v"], a["start"],
                                   a["count"], a["mask"], 0), message)


@pytest.mark.parametrize("k,message", [
    (tensor(token=0), "overlap"), (tensor(head=32), "overlap"), (tensor(batch=64), "overlap"),
    (tensor(token=128), "overlap"),
])
def test_kv_read_outputs_may_not_overlap(k, message):
    refused(lambda: gm.gm_kv_read(cache(), 1, 2, 8, None, None, k, tensor(), 0), message)
    refused(lambda: gm.gm_kv_read(cache(), 1, 2, 8, None, None, tensor(), k, 0), message)


def test_too_many_rows():
    c = cache(batch=1 << 20, heads=1 << 16, max_seq=64, head_dim=128)
    t = tensor(batch=1 << 40, token=1 << 24, head=128)
    refused(lambda: gm.gm_kv_write(c, 1, 1 << 20, 60, t, t, None, None, None, 0), "below 2^32")


def cached(**kw):
    a = dict(cache=ctypes.pointer(cache()), dtype=1, B=2, Sq=8, n_heads=4, q=tensor(), out=tensor(),
             lengths=P, scores=gm.gm_scores(0.125, 0.0, None), workspace=P,
             workspace_bytes=1 << 40)
    a.update(kw)
    return gm.gm_cached_attention(**a)


@pytest.mark.parametrize("kw,message", [
    (dict(cache=None), "NULL"), (dict(dtype=-1), "dtype"), (dict(B=3), "batch"), (dict(Sq=129), "Sq"),
    (dict(n_heads=6), "multiple of the cache's heads"), (dict(n_heads=0), "multiple"),
    (dict(q=tensor(p=P + 2)), "16-byte"), (dict(out=tensor(token=64)), "overlap"),
    (dict(lengths=None), "lengths"), (dict(scores=gm.gm_scores(float("nan"), 0.0, None)), "scale"),
    (dict(scores=gm.gm_scores(1.0, -1.0, None)), "softcap"),
    (dict(scores=gm.gm_scores(1.0, float("inf"), None)), "softcap"),
    (dict(scores=gm.gm_scores(1.0, 1025.0, None)), "softcap"),
    (dict(scores=gm.gm_scores(1.0, 1e-7, None)), "softcap"),
    (dict(scores=gm.gm_scores(0.0, 0.0, None)), "scale"),
    (dict(scores=gm.gm_scores(-1.0, 0.0, None)), "scale"),
    (dict(scores=gm.gm_scores(1.0, 0.0, P + 1)), "slopes"),
])
def test_cached_attention_refusals(kw, message):
    refused(lambda: gm.gm_attention_cached(cached(**kw), 0), message)


@pytest.mark.parametrize("workspace,less", [(None, 0), (P + 8, 0), (P, 1)])
def test_cached_attention_needs_its_workspace(workspace, less):
    c = cache(max_seq=1 << 16, batch=1)
    need = gm.gm_attention_cached_workspace(c, 1, 1, 1, 4)
    assert need > 0
    refused(lambda: gm.gm_attention_cached(
        cached(cache=ctypes.pointer(c), B=1, Sq=1, workspace=workspace, workspace_bytes=need - less), 0),
        "workspace")


def prompt(**kw):
    a = dict(dtype=1, B=2, Sq=8, Sk=8, n_heads=4, kv_heads=4, head_dim=64, q=tensor(), k=tensor(),
             v=tensor(), out=tensor(), causal=1, q_offset=0,
             scores=gm.gm_scores(0.125, 0.0, None), key_mask=None, q_doc=None, k_doc=None,
             prefix=None)
    a.update(kw)
    return gm.gm_prompt_attention(**a)


@pytest.mark.parametrize("kw,message", [
    (dict(dtype=3), "dtype"), (dict(head_dim=96), "head_dim"), (dict(B=-1), "negative"),
    (dict(Sk=-1), "negative"), (dict(n_heads=5), "multiple of kv_heads"), (dict(kv_heads=0), "multiple"),
    (dict(Sk=1 << 24), "2^24"), (dict(q_offset=-(1 << 24)), "2^24"), (dict(q=tensor(p=None)), "NULL"),
    (dict(k=tensor(token=250)), "multiples of 16 bytes"), (dict(v=tensor(p=P + 4)), "16-byte"),
    (dict(out=tensor(head=0)), "overlap"), (dict(q_doc=P), "go together"), (dict(k_doc=P), "go together"),
    (dict(prefix=P, causal=0), "prefix needs causal"), (dict(key_mask=P + 2), "4-byte"),
    (dict(scores=gm.gm_scores(0.1, float("nan"), None)), "softcap"),
])
def test_prompt_attention_refusals(kw, message):
    refused(lambda: gm.gm_attention(prompt(**kw), 0), message)


def test_outputs_may_not_start_where_another_tensor_does():
    refused(lambda: gm.gm_kv_read(cache(), 1, 2, 8, None, None, tensor(), tensor(), 0), "overlap")
    refused(lambda: gm.gm_attention_cached(cached(), 0), "overlap")
    far = dict(q=tensor(p=P + 4096), k=tensor(p=P + 8192), v=tensor(p=P + 16384))
    for name in far:
        refused(lambda: gm.gm_attention(prompt(**{**far, name: tensor()}), 0), "overlap")


def test_null_arguments():
    L = gm.lib()
    assert L.gm_attention(None, None) == gm.GM_E_INVAL
    assert L.gm_attention_cached(None, None) == gm.GM_E_INVAL
    assert L.gm_kv_write(None, 0, 1, 1, tensor(), tensor(), None, None, None, None) == gm.GM_E_INVAL
    assert L.gm_attention_cached_workspace(None, 0, 1, 1, 1) == 0


def test_nothing_to_do_is_ok_without_a_device():
    gm.gm_kv_write(cache(), 1, 0, 8, tensor(p=None), tensor(p=None), None, None, None, 0)
    gm.gm_kv_write(cache(), 1, 2, 0, tensor(p=None), tensor(p=None), None, None, None, 0)
    gm.gm_attention_cached(cached(B=0, lengths=None), 0)
    gm.gm_attention(prompt(Sq=0), 0)


def test_wrappers_refuse_host_tensors_and_bad_arguments():
    q = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="HIP device"):
        ops.attention(q, q, q)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        ops.attention(q.double(), q, q)
    for bad in (dict(bits=3), dict(head_dim=80), dict(max_seq=0), dict(batch=0)):
        with pytest.raises(ValueError):
            ops.KvCache(**{**dict(batch=1, heads=1, max_seq=64, head_dim=64, bits=8, device="cpu"), **bad})
    c = ops.KvCache(2, 4, 100, 64, bits=4, device="cpu")
    assert c.c.max_seq == 128 and c.k.shape == (2, 4, 128, 32) and c.k_scale.shape == (2, 4, 2, 128)
    with pytest.raises(ValueError, match="HIP device"):
        c.write(q, q)
    with pytest.raises(ValueError, match="HIP device"):
        ops.cached_attention(q, c, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError, match="dtype"):
        c.read(4, dtype=torch.int8)
    with pytest.raises(ValueError, match="batch"):
        c.read(4, batch=3)


@pytest.mark.parametrize("name,over,opts,message", [
    ("causal_lm_768", dict(kv_cache=1), dict(kv_bits=3), "kv_bits must be"),
    ("causal_lm_768", {}, dict(kv_bits=8), "needs kv_cache"),
    ("causal_lm_768", {}, dict(softcap=-1.0), "softcap"),
    ("causal_lm_768", {}, dict(softcap=float("inf")), "softcap"),
    ("seq2seq_768", {}, dict(softcap=5.0), "encoder-decoder"),
    ("seq2seq_768", {}, dict(slopes=P), "encoder-decoder"),
    ("decoder_4096", dict(kv_cache=1, max_batch=512, max_seq=32000), dict(kv_bits=4), "2^32"),
])
def test_model_option_refusals(name, over, opts, message):
    import synth
    from paper_2509_16248_amd.model import make_config
    c = make_config(synth.preset(name))
    for k, v in over.items():
        setattr(c, k, v)
    refused(lambda: gm.gm_model_create_ex(c, gm.gm_weights(), gm.gm_attn_options(**opts)), message)


def test_segment_and_cache_entries_refuse_null():
    L = gm.lib()
    assert L.gm_set_segments(None, None, None, 1, 1) == gm.GM_E_INVAL
    assert L.gm_model_kv_cache(None, 0, None) == gm.GM_E_INVAL
    out = ctypes.c_void_p()
    assert L.gm_model_create_ex(None, None, None, ctypes.byref(out)) == gm.GM_E_INVAL
