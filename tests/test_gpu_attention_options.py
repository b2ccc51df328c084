"""Models with attention options (gm_model_create_ex, gm_set_segments) against the
oracle: capped and distance-biased scores, documents and prefixes in forwards and
decode steps, and decoding over a cache in 8 and 4 bits.

The oracle here is the float64 model of ``oracle`` with its attention step
replaced by the modified one.  A quantised cache cannot be compared from the
inputs alone (a key that differs in its last bit may round to another code), so
its content is checked exactly against the quantisation of the GPU's own stored
k and v, and each decode step's logits against the oracle's step over the
content of the GPU's cache.
"""
import numpy as np
import pytest
import torch

import ops_reference as ref
import synth
from oracle import OracleDecoder, OracleModel
from oracle import numerics as nx
from paper_2509_16248_amd import gm

from test_gpu_parity import TOL, check_logits, f64, gpu_model, run

pytestmark = pytest.mark.gpu


def slopes_of(H):
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


class Oracle(OracleModel):
    """OracleModel with capped, biased, document- and prefix-masked attention."""

    def __init__(self, cfg, w, softcap=0.0, slopes=None, docs=None, prefix=None):
        super().__init__(cfg, w)
        self.softcap, self.slopes, self.docs, self.prefixes = softcap, slopes, docs, prefix

    def begin(self, ids, mask, *a, **kw):
        st = super().begin(ids, mask, *a, **kw)
        S = st.S
        if self.prefixes is not None:
            j = np.arange(S)
            causal = np.tril(np.ones((S, S), dtype=bool))[None]
            seen = causal | (j[None, None] < np.asarray(self.prefixes)[:, None, None])
            if st.pad_any:
                seen = seen & (np.asarray(mask)[:, None, :] == 1)
            st.allowed = seen[:, None]
        if self.docs is not None:
            d = np.asarray(self.docs)[:, :S]
            st.allowed = st.allowed & (d[:, None, :, None] == d[:, None, None, :])
        return st

    def scores(self, q, k, distance):
        """[B, H, Sq, Sk] of q [B, H, Sq, hd] and k [B, H, Sk, hd]."""
        s = (q @ k.transpose(0, 1, 3, 2)) / np.sqrt(q.shape[-1])
        if self.softcap:
            s = self.softcap * np.tanh(s / self.softcap)
        if self.slopes is not None:
            s = s - np.asarray(self.slopes)[None, :, None, None] * np.abs(distance)
        return s

    def step_attention(self, q, k, v, allowed):
        B, H, S, hd = q.shape
        i = np.arange(S)
        p = nx.masked_softmax(self.scores(q, k, (i[:, None] - i[None])[None, None]), allowed)
        return self.R(p @ v).transpose(0, 2, 1, 3).reshape(B, S, H * hd)


CASES = [
    ("tiny_decoder", dict(softcap=0.005)), ("tiny_decoder", dict(slopes=True)),
    ("causal_lm_768", dict(softcap=20.0, slopes=True)), ("encoder_1024", dict(slopes=True)),
    ("encoder_clamp_1024", dict(softcap=30.0)), ("decoder_4096", dict(softcap=0.1)),
]


def setup(name, opts, seed, **kw):
    cfg = synth.preset(name, batch=2) if name == "tiny_decoder" else synth.reduced(name)
    cfg = cfg.replace(**kw)
    w = synth.make_weights(cfg, seed)
    o = {k: slopes_of(cfg.n_heads) if k == "slopes" else v for k, v in opts.items()}
    return cfg, w, o


@pytest.mark.parametrize("name,opts", CASES)
def test_forward_with_modified_scores(name, opts):
    cfg, w, o = setup(name, opts, 51)
    ids, mask = synth.make_inputs(cfg, 3)
    res = Oracle(cfg, w, **o).forward(ids, mask)
    plain = OracleModel(cfg, w).forward(ids, mask)
    m = gpu_model(cfg, w, **o)
    out = run(m, ids, mask)
    check_logits(f64(out), res.logits_f64, cfg.dtype, f"{name} {sorted(o)}")
    # the options matter: the plain model's logits are further away than the tolerance allows
    moved = np.abs(res.logits_f64 - plain.logits_f64).max() / np.abs(plain.logits_f64).max()
    print(f"{name}: the options move the logits by {moved:.3g}", flush=True)
    assert moved > TOL[cfg.dtype]
    assert m.check_error() == (0, 0) and m.stats()["host_syncs_in_forward"] == 0
    # the eager, fragmented and no-allocation forwards run the same kernels
    for mode in ("eager", "fragmented"):
        m.set_exec_mode(mode)
        assert torch.equal(run(m, ids, mask).view(torch.uint8), out.view(torch.uint8)), mode
    t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (ids, mask)]
    other = m.forward_noalloc(*t, m.new_logits(*ids.shape))
    assert torch.equal(other.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("name", ["tiny_decoder", "causal_lm_768", "decoder_4096"])
def test_documents_and_prefixes(name):
    cfg, w, o = setup(name, dict(softcap=15.0), 52, batch=2)
    ids, mask = synth.make_inputs(cfg, 4)
    B, S = ids.shape
    docs = np.sort(np.random.default_rng(1).integers(0, 4, (B, S)), axis=1).astype(np.int32)
    prefix = np.array([S // 3, S], dtype=np.int32)
    m = gpu_model(cfg, w, **o)
    d, p = torch.from_numpy(docs).cuda(), torch.from_numpy(prefix).cuda()
    for dd, pp in ((docs, None), (None, prefix), (docs, prefix)):
        m.set_segments(d if dd is not None else None, p if pp is not None else None, shape=(B, S))
        res = Oracle(cfg, w, docs=dd, prefix=pp, **o).forward(ids, mask)
        check_logits(f64(run(m, ids, mask)), res.logits_f64, cfg.dtype,
                     f"{name} docs {dd is not None} prefix {pp is not None}")
    # the arrays are read when a forward runs, so a cached graph follows them
    captures = m.stats()["captures"]
    d.copy_(torch.from_numpy(docs[::-1].copy()))
    p.copy_(torch.tensor([0, 5], dtype=torch.int32))
    res = Oracle(cfg, w, docs=docs[::-1], prefix=[0, 5], **o).forward(ids, mask)
    out = m.new_logits(B, S)
    t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (ids, mask)]
    for _ in range(3):
        m.forward(*t, out)
        check_logits(f64(out), res.logits_f64, cfg.dtype, f"{name} changed segments")
    assert m.stats()["captures"] <= captures + 1      # (one if the buffers are not run()'s)
    # another shape is refused, on the host; without segments it runs again
    with pytest.raises(gm.GmError, match="another B and S"):
        m.forward(t[0][:1].contiguous(), t[1][:1].contiguous(), m.new_logits(1, S))
    m.set_segments()
    res = Oracle(cfg, w, **o).forward(ids, mask)
    check_logits(f64(run(m, ids, mask)), res.logits_f64, cfg.dtype, f"{name} segments removed")


def decode(m, toks):
    t = torch.tensor(toks, dtype=torch.int32, device="cuda")
    out = m.new_decode_logits(len(toks))
    m.decode(t, out)
    torch.cuda.synchronize()
    return f64(out)


@pytest.mark.parametrize("name,opts", [("tiny_decoder", dict(softcap=0.005, slopes=True)),
                                       ("causal_lm_768", dict(slopes=True)),
                                       ("decoder_4096", dict(softcap=0.1))])
def test_decode_with_modified_scores_over_the_plain_cache(name, opts):
    cfg, w, o = setup(name, opts, 53)
    ids, mask = synth.make_inputs(cfg, 5, seq=12 if name == "tiny_decoder" else 100)
    dec = OracleDecoder(Oracle(cfg, w, **o), cfg.seq)
    dec.prefill(ids, mask)
    m = gpu_model(cfg, w, max_seq=cfg.seq, kv_cache=True, **o)
    run(m, ids, mask)
    rng = np.random.default_rng(2)
    for k in range(4):
        toks = rng.integers(0, cfg.vocab, ids.shape[0]).tolist()
        check_logits(decode(m, toks), dec.step(toks).logits_f64, cfg.dtype, f"{name} step {k}")


def test_decode_continues_the_last_document():
    cfg, w, o = setup("causal_lm_768", dict(softcap=15.0), 54)
    ids, mask = synth.make_inputs(cfg, 6, seq=100, max_pad=20)
    B, S = ids.shape
    docs = np.sort(np.random.default_rng(3).integers(0, 3, (B, S)), axis=1).astype(np.int32)
    lens = [int(np.nonzero(r)[0][-1]) + 1 for r in mask]
    longer = np.zeros((B, cfg.seq), dtype=np.int32)
    for b, L in enumerate(lens):
        longer[b, :L], longer[b, L:] = docs[b, :L], docs[b, L - 1]
    dec = OracleDecoder(Oracle(cfg, w, docs=longer, **o), cfg.seq)
    dec.prefill(ids, mask)
    for bits in (0, 8):
        m = gpu_model(cfg, w, max_seq=cfg.seq, kv_cache=True, kv_bits=bits, **o)
        m.set_segments(torch.from_numpy(docs).cuda())
        run(m, ids, mask)
        if bits == 0:
            for k in range(3):
                toks = [7 * k + b for b in range(B)]
                check_logits(decode(m, toks), dec.step(toks).logits_f64, cfg.dtype, f"step {k}")
        else:
            c = gm.gm_model_kv_cache(m.handle, 0)
            quantised_step(m, Oracle(cfg, w, **o), [3, 4, 5], lens,
                           [(docs[b, :L] == docs[b, L - 1]) & (mask[b, :L] == 1)
                            for b, L in enumerate(lens)], "documents, 8 bits")
            assert c.bits == 8 and c.heads == cfg.n_heads


def quantised_step(m, orc, toks, lens, valid, what):
    """One decode step of a quantised model, its logits against the oracle's step
    over the content of the GPU's cache; lens and valid describe the keys before."""
    c = orc.cfg
    B = len(toks)
    got = decode(m, toks)
    if c.pos == "rotary":
        orc._rope_build(max(lens) + 1)
    n = max(lens) + 1
    caches = [[t.double().cpu().numpy() for t in m.read_cache(l, n)] for l in range(c.n_layers)]
    rows = []
    for b in range(B):
        L = lens[b]
        h = orc._g("tok_emb")[[toks[b]]][None]
        if c.pos == "learned":
            h = h + orc._g("pos_emb")[L][None, None]
        h = orc.R(h)
        for l in range(c.n_layers):
            W = orc.layer_weights(l)
            q, _, _ = orc.step_qkv(orc.step_norm(h, W, 1), W, 1, positions=[L])
            k, v = (x[b:b + 1, :L + 1].transpose(0, 2, 1, 3) for x in caches[l])
            s = orc.scores(q, k, (L - np.arange(L + 1))[None, None, None])
            ok = np.append(valid[b], True)[None, None, None]
            ctx = orc.R(nx.masked_softmax(s, ok) @ v).transpose(0, 2, 1, 3).reshape(1, 1, -1)
            h, _ = orc.step_residual(h, ctx, W["wo"], W.get("bo"))
            h, _ = orc.step_residual(h, orc.step_ffn(orc.step_norm(h, W, 2), W), W["w2"], W.get("b2"))
        rows.append(orc.step_head(h)[0, 0])
    check_logits(got, np.stack(rows), c.dtype, what)
    for b in range(B):
        lens[b] += 1
        valid[b] = np.append(valid[b], True)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name,opts", [("tiny_decoder", {}), ("tiny_decoder", dict(slopes=True)),
                                       ("causal_lm_768", dict(softcap=20.0)), ("decoder_4096", {})])
def test_decode_over_the_quantised_cache(name, opts, bits):
    cfg, w, o = setup(name, opts, 55)
    ids, mask = synth.make_inputs(cfg, 7, seq=12 if name == "tiny_decoder" else 130)
    B, S = ids.shape
    orc = Oracle(cfg, w, **o)
    res = orc.forward(ids, mask)
    m = gpu_model(cfg, w, max_seq=cfg.seq, kv_cache=True, kv_bits=bits, **o)
    t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (ids, mask)]
    out = m.new_logits(B, S)
    points = m.forward_layers(*t, out)               # the prefill, with its stored q | k | v
    check_logits(f64(out), res.logits_f64, cfg.dtype, f"{name} prefill")
    d, H, hd = cfg.d_model, cfg.n_heads, cfg.head_dim
    for l in range(cfg.n_layers):
        qkv = points["qkv"][l].view(B, S, 3, H, hd)
        for got, i in zip(m.read_cache(l, S, batch=B), (1, 2)):
            assert torch.equal(got.cpu(), ref.stored(qkv[:, :, i], bits).to(got.dtype)), (l, i)
    lens = [int(np.nonzero(r)[0][-1]) + 1 for r in mask]
    valid = [mask[b, :L] == 1 for b, L in enumerate(lens)]
    rng = np.random.default_rng(4)
    for k in range(3):
        toks = rng.integers(0, cfg.vocab, B).tolist()
        quantised_step(m, orc, toks, lens, valid, f"{name} {bits} bits step {k}")
    # a step with a bad token stores nothing and leaves the lengths
    before = [x.clone() for x in m.read_cache(0, cfg.seq)]
    decode(m, [cfg.vocab] + [0] * (B - 1))
    assert m.check_error() == (1, 0)
    for a, b in zip(before, m.read_cache(0, cfg.seq)):
        assert torch.equal(a, b)
    quantised_step(m, orc, rng.integers(0, cfg.vocab, B).tolist(), lens, valid, f"{name} after the trap")


def test_quantised_decode_graph_replays_and_fills_the_cache():
    cfg, w, o = setup("tiny_decoder", {}, 56)
    ids, mask = synth.make_inputs(cfg, 8, seq=4, max_pad=0)
    outs = {}
    for mode in ("graph", "eager"):
        m = gpu_model(cfg, w, max_seq=16, kv_cache=True, kv_bits=8)
        m.set_exec_mode(mode)
        run(m, ids, mask)
        cur = torch.zeros(2, dtype=torch.int32, device="cuda")
        logits, hist = m.new_decode_logits(2), []
        for _ in range(12):                           # up to the capacity
            m.decode(cur, logits, cur)
            hist.append(logits.clone())
        torch.cuda.synchronize()
        assert m.check_error() == (0, 0)
        m.decode(cur, logits, cur)                    # one more: the cache is full
        assert m.check_error() == (4, 0)
        outs[mode] = torch.stack(hist)
        if mode == "graph":
            assert m.stats()["host_syncs_in_forward"] == 0
    assert torch.equal(outs["graph"], outs["eager"])


def test_refusals():
    cfg, w, _ = setup("tiny_decoder", {}, 57)
    m = gpu_model(cfg, w, kv_cache=True)
    with pytest.raises(gm.GmError, match="without kv_bits"):
        m.read_cache(0, 1)
    with pytest.raises(gm.GmError, match="out of range"):
        m.set_segments(torch.zeros(1000, 16, dtype=torch.int32, device="cuda"))
    enc = synth.reduced("encoder_1024")
    e = gpu_model(enc, synth.make_weights(enc, 1))
    with pytest.raises(gm.GmError, match="causal"):
        e.set_segments(prefix=torch.zeros(1, dtype=torch.int32, device="cuda"), shape=(1, 8))
    q = gpu_model(cfg, w, kv_cache=True, kv_bits=4)
    with pytest.raises(gm.GmError, match="layer out of range"):
        q.read_cache(1, 1)
