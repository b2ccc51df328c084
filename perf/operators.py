"""Measured cases of the attention and KV-cache operators.

Three operators that a program serving a language model calls one after the
other: storing keys and values into a cache held in 8 or 4 bits and reading
them back (:class:`KvCache`), attention of new tokens over that cache
(:func:`cached_attention`), and attention over a whole prompt whose scores are
capped by a tanh, biased by distance, or limited to a document or a prefix
(:func:`attention`).

``run`` computes each in plain torch operations, or, with ``own`` set, with the
library's operators; ``exact`` computes the same in float64 from the
definitions.

Definitions.  A cache group is 32 consecutive channels of one token and head;
Q is 127 (8 bits) or 7 (4 bits); a the largest magnitude of the group; the scale
s is the fp32 product a * fp32(1/Q) rounded to bfloat16; a code is x / s rounded
to the nearest integer (ties to even) and limited to [-Q, Q]; the stored value
is code * s.  Scores are scale * q.k, then cap * tanh(score / cap), then
- slope * |query position - key position|; the output is the softmax-weighted
sum of the values over the visible keys, zero where there is none.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_GROUP = 32


def listed():
    return [
        # ---- cache: store and read back
        # one decode step's append of the 12-head model over a batch of 8: latency only
        {"name": "kv_append_8x12x64_q8", "op": "kv", "dtype": "bf16", "bits": 8, "batch": 8,
         "heads": 12, "hd": 64, "n": 1, "cap": 512, "store": True},
        # the 4096-wide decoder's prompt at its benchmark length, one layer
        {"name": "kv_prompt_1x2048x32x128_q4", "op": "kv", "dtype": "bf16", "bits": 4, "batch": 1,
         "heads": 32, "hd": 128, "n": 2048, "cap": 4096, "store": True},
        # a ragged fp32 batch of odd lengths, stored behind what is there
        {"name": "kv_prompt_3x777x12x64_q4_f32", "op": "kv", "dtype": "f32", "bits": 4, "batch": 3,
         "heads": 12, "hd": 64, "n": 777, "cap": 1000, "store": True},
        # a long cache of grouped heads handed over whole (prefix reuse, moving a sequence)
        {"name": "kv_read_4x8192x8x128_q8", "op": "kv", "dtype": "f16", "bits": 8, "batch": 4,
         "heads": 8, "hd": 128, "n": 8192, "cap": 8192, "store": False},
        # ---- new tokens over the cache
        # the smallest: fp32, four tokens appended at once to two short sequences
        {"name": "cached_2x4x32_q8_f32", "op": "cached", "dtype": "f32", "bits": 8, "batch": 2,
         "heads": 4, "kv_heads": 4, "hd": 32, "sq": 4, "len": 37, "cap": 64, "softcap": 0.0,
         "alibi": False},
        # a decode step of the 12-head model, 8 ragged sequences
        {"name": "cached_8x12x64_q8", "op": "cached", "dtype": "bf16", "bits": 8, "batch": 8,
         "heads": 12, "kv_heads": 12, "hd": 64, "sq": 1, "len": 640, "cap": 1024, "softcap": 0.0,
         "alibi": False},
        # one long conversation of a 32-head model with distance biases
        {"name": "cached_1x32x128_q4_long", "op": "cached", "dtype": "bf16", "bits": 4, "batch": 1,
         "heads": 32, "kv_heads": 32, "hd": 128, "sq": 1, "len": 32000, "cap": 32768,
         "softcap": 0.0, "alibi": True},
        # a full serving batch of grouped heads with capped scores
        {"name": "cached_32x32g8x128_q4_cap", "op": "cached", "dtype": "f16", "bits": 4,
         "batch": 32, "heads": 32, "kv_heads": 8, "hd": 128, "sq": 1, "len": 8190, "cap": 8192,
         "softcap": 30.0, "alibi": False},
        # ---- whole prompts
        # the smallest: fp32, one short prompt with capped scores
        {"name": "attn_1x16x2x32_f32_cap", "op": "attn", "dtype": "f32", "batch": 1, "heads": 2,
         "kv_heads": 2, "hd": 32, "sq": 16, "sk": 16, "causal": True, "softcap": 20.0,
         "alibi": False, "docs": 0, "prefix": False, "pads": False},
        # the 4096-wide decoder's prompt with capped scores
        {"name": "attn_1x2048x32x128_cap", "op": "attn", "dtype": "bf16", "batch": 1, "heads": 32,
         "kv_heads": 32, "hd": 128, "sq": 2048, "sk": 2048, "causal": True, "softcap": 50.0,
         "alibi": False, "docs": 0, "prefix": False, "pads": False},
        # a padded fp16 batch of odd length: bidirectional prefixes and distance biases
        {"name": "attn_4x1000x16x64_prefix", "op": "attn", "dtype": "f16", "batch": 4, "heads": 16,
         "kv_heads": 16, "hd": 64, "sq": 1000, "sk": 1000, "causal": True, "softcap": 0.0,
         "alibi": True, "docs": 0, "prefix": True, "pads": True},
        # documents packed into one long row, grouped heads
        {"name": "attn_1x8192x32g8x128_docs", "op": "attn", "dtype": "bf16", "batch": 1,
         "heads": 32, "kv_heads": 8, "hd": 128, "sq": 8192, "sk": 8192, "causal": True,
         "softcap": 0.0, "alibi": False, "docs": 7, "prefix": False, "pads": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["kv", "cached", "attn"])
    dtype = rng.choice(["bf16", "f16", "bf16", "f32"])
    hd = rng.choice([32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 12, 32])
    if op == "kv":
        heads = kv_heads
        batch = _log_uniform(rng, 1, 16)
        n = _log_uniform(rng, 1, max(2, min(8192, 33_000_000 // (batch * heads * hd))))
        return {"op": op, "dtype": dtype, "bits": rng.choice([8, 4]), "batch": batch,
                "heads": heads, "hd": hd, "n": n, "cap": n + rng.randrange(0, 300),
                "store": rng.random() < 0.7}
    group = rng.choice([1, 1, 2, 4, 8])
    heads = min(64, kv_heads * group) // kv_heads * kv_heads
    if op == "cached":
        batch = _log_uniform(rng, 1, 32)
        top = 134_000_000 // (batch * kv_heads * hd)
        if dtype == "f32":
            top //= 8
        length = _log_uniform(rng, 1, max(2, min(60000, top)))
        sq = min(length, rng.choice([1, 1, 1, 2, 5]))
        return {"op": op, "dtype": dtype, "bits": rng.choice([8, 4]), "batch": batch,
                "heads": heads, "kv_heads": kv_heads, "hd": hd, "sq": sq, "len": length,
                "cap": length + rng.randrange(0, 300),
                "softcap": rng.choice([0.0, 0.0, 30.0]), "alibi": rng.random() < 0.4}
    batch = _log_uniform(rng, 1, 8)
    heads = min(heads, 32) // kv_heads * kv_heads
    work = 32 * 8192 * 8192 * 128 // (16 if dtype == "f32" or hd == 32 else 2)
    top = int(math.sqrt(work / (batch * heads * hd)))
    sk = _log_uniform(rng, 1, max(2, min(8192, top)))
    sq = sk if rng.random() < 0.7 else max(1, sk - rng.randrange(0, sk))
    causal = rng.random() < 0.7
    return {"op": op, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads,
            "hd": hd, "sq": sq, "sk": sk, "causal": causal,
            "softcap": rng.choice([0.0, 30.0, 50.0]), "alibi": rng.random() < 0.3,
            "docs": rng.choice([0, 0, min(sk, 5)]), "prefix": causal and rng.random() < 0.3,
            "pads": rng.random() < 0.4}


# ------------------------------------------------------------ inputs
def _slopes(heads):
    """The geometric slopes 2^(-8 (h + 1) / heads) of distance-biased models."""
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


def _lengths(case):
    """Ragged lengths in (len / 2, len], never below the new tokens'."""
    L = case["len"]
    return [max(case["sq"], L - (b * 97) % (L // 2 + 1)) for b in range(case["batch"])]


def _counts(case):
    """Rows each sequence stores: the first all, the others fewer."""
    n = case["n"]
    return [n - (b * 53) % (n // 2 + 1) for b in range(case["batch"])]


def _starts(case):
    room = case["cap"] - case["n"]
    return [(b * 31) % (room + 1) for b in range(case["batch"])]


def _doc_ids(n, docs):
    """Ids of ``docs`` documents of uneven lengths packed into n positions."""
    ends = [n * (i + 1) * (i + 2) // (docs * (docs + 1)) for i in range(docs)]
    ids, d = [], 0
    for p in range(n):
        while p >= ends[d]:
            d += 1
        ids.append(d)
    return ids


def _prefixes(case):
    return [(b + 1) * case["sk"] // (case["batch"] + 2) for b in range(case["batch"])]


def _visible_lengths(case):
    """Unpadded keys of each sequence."""
    sk = case["sk"]
    if not case["pads"]:
        return [sk] * case["batch"]
    return [max(1, sk - (b * 61) % (sk // 2 + 1)) for b in range(case["batch"])]


def _inputs(case, seed):
    """Tensors a program holds before the call, [batch, tokens, heads, head_dim]."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPE[case["dtype"]]
    hd, B = case["hd"], case["batch"]

    def normal(tokens, heads, outliers=False):
        x = torch.randn((B, tokens, heads, hd), generator=g, device="cuda")
        if outliers:
            # a few channels of every key head carry most of the magnitude
            x *= 1.0 + 4.0 * (torch.rand((heads, hd), generator=g, device="cuda") < 0.05)
        return x.to(dt)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    if case["op"] == "kv":
        return {"k": normal(case["n"], case["heads"], True), "v": normal(case["n"], case["heads"]),
                "start": ints(_starts(case)), "count": ints(_counts(case))}
    if case["op"] == "cached":
        out = {"q": normal(case["sq"], case["heads"]),
               "k": normal(case["len"], case["kv_heads"], True),
               "v": normal(case["len"], case["kv_heads"]), "lengths": ints(_lengths(case))}
    else:
        out = {"q": normal(case["sq"], case["heads"]),
               "k": normal(case["sk"], case["kv_heads"], True),
               "v": normal(case["sk"], case["kv_heads"])}
        if case["pads"]:
            lens = ints(_visible_lengths(case))
            out["mask"] = (torch.arange(case["sk"], device="cuda")[None] < lens[:, None]).int()
        if case["docs"]:
            ids = ints(_doc_ids(case["sk"], case["docs"])).expand(B, -1).contiguous()
            out["k_doc"] = ids
            out["q_doc"] = ids[:, case["sk"] - case["sq"]:].contiguous()
        if case["prefix"]:
            out["prefix"] = ints(_prefixes(case))
    if case["alibi"]:
        out["slopes"] = torch.tensor(_slopes(case["heads"]), dtype=torch.float32, device="cuda")
    return out


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if case["op"] == "kv" or case["op"] == "cached":
        heads = case["heads"] if case["op"] == "kv" else case["kv_heads"]
        B, cap, hd = case["batch"], case["cap"], case["hd"]
        filled = case["op"] == "cached" or not case["store"]
        start = state["start"] if case["op"] == "kv" else torch.zeros(B, dtype=torch.int32,
                                                                       device="cuda")
        if own:
            from paper_2509_16248_amd.ops import KvCache
            state["cache"] = KvCache(B, heads, cap, hd, bits=case["bits"], device="cuda")
            if filled:
                state["cache"].write(state["k"], state["v"], start)
        else:
            cache = {}
            for name in ("k", "v"):
                cache[name] = torch.zeros((B, cap, heads, hd), dtype=torch.int8, device="cuda")
                cache[name + "_scale"] = torch.zeros((B, cap, heads, hd // _GROUP),
                                                     dtype=torch.bfloat16, device="cuda")
            state["cache"] = cache
            if filled:
                _plain_write(cache, state["k"], state["v"], start, None, case["bits"])
        if filled:
            del state["k"], state["v"]
    return state


# ------------------------------------------------------------ plain forms
def _plain_quantise(x, bits):
    """[..., hd] -> codes int8 [..., hd], scales bfloat16 [..., hd / 32]."""
    top = 127 if bits == 8 else 7
    g = x.float().unflatten(-1, (-1, _GROUP))
    inv = torch.tensor(1.0 / top, dtype=torch.float32, device=x.device)
    scale = (g.abs().amax(-1) * inv).bfloat16()
    # quotients in float64: one next to a half must not be rounded twice
    q = g.double() / scale.double().unsqueeze(-1)
    q = torch.where(scale.unsqueeze(-1) == 0, 0.0, q)
    return q.round().clamp(-top, top).to(torch.int8).flatten(-2), scale


def _plain_values(codes, scale):
    return (codes.float().unflatten(-1, (-1, _GROUP)) * scale.float().unsqueeze(-1)).flatten(-2)


def _plain_write(cache, k, v, start, count, bits):
    B, n = k.shape[:2]
    i = torch.arange(n, device=k.device)[None]
    pos = start[:, None].long() + i
    for name, x in (("k", k), ("v", v)):
        codes, scale = _plain_quantise(x, bits)
        if count is None:
            b = torch.arange(B, device=k.device)[:, None].expand(B, n)
            cache[name][b, pos] = codes
            cache[name + "_scale"][b, pos] = scale
        else:
            # rows past the count keep what the cache holds there
            b = torch.arange(B, device=k.device)[:, None].expand(B, n)
            keep = (i < count[:, None])[..., None, None]
            cache[name][b, pos] = torch.where(keep, codes, cache[name][b, pos])
            old = cache[name + "_scale"][b, pos]
            cache[name + "_scale"][b, pos] = torch.where(keep, scale, old)


def _plain_read(cache, start, count, n, dtype):
    B = start.shape[0]
    i = torch.arange(n, device=start.device)[None]
    pos = start[:, None].long() + i
    b = torch.arange(B, device=start.device)[:, None].expand(B, n)
    keep = (i < count[:, None])[..., None, None]
    out = []
    for name in ("k", "v"):
        x = _plain_values(cache[name][b, pos], cache[name + "_scale"][b, pos])
        out.append(torch.where(keep, x, 0.0).to(dtype))
    return out


def _plain_attention(q, k, v, visible, qpos, kpos, scale, softcap, slopes):
    """q [Sq, H, hd], k and v [Sk, Hkv, hd] in float32, visible [Sq, Sk]."""
    Sq, H, hd = q.shape
    G = H // k.shape[1]
    kh = k.transpose(0, 1).repeat_interleave(G, 0)
    vh = v.transpose(0, 1).repeat_interleave(G, 0)
    s = torch.bmm(q.transpose(0, 1).contiguous(), kh.transpose(1, 2).contiguous()) * scale
    if softcap > 0.0:
        s = softcap * torch.tanh(s / softcap)
    if slopes is not None:
        s = s - slopes[:, None, None] * (qpos[:, None] - kpos[None]).abs().float()
    s = s.masked_fill(~visible, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0.0, 1.0, total)
    return torch.bmm(p, vh.contiguous()).transpose(0, 1)


def _plain_cached(state, case):
    cache, q = state["cache"], state["q"]
    B, Sq = q.shape[:2]
    L = case["len"]
    i = torch.arange(Sq, device=q.device)
    j = torch.arange(L, device=q.device)
    out = torch.empty_like(q)
    for b in range(B):
        k = _plain_values(cache["k"][b, :L], cache["k_scale"][b, :L])
        v = _plain_values(cache["v"][b, :L], cache["v_scale"][b, :L])
        qpos = state["lengths"][b] - Sq + i
        out[b] = _plain_attention(q[b].float(), k, v, j[None] <= qpos[:, None], qpos, j,
                                  1.0 / math.sqrt(case["hd"]), case["softcap"],
                                  state.get("slopes")).to(q.dtype)
    return out


def _plain_prompt(state, case):
    q, k, v = state["q"], state["k"], state["v"]
    B, Sq = q.shape[:2]
    Sk = k.shape[1]
    out = torch.empty_like(q)
    j = torch.arange(Sk, device=q.device)
    # queries in parts, so that the float32 scores stay a few GB
    step = max(1, min(Sq, 1_000_000_000 // (Sk * case["heads"])))
    for b in range(B):
        kb, vb = k[b].float(), v[b].float()
        for i0 in range(0, Sq, step):
            i = torch.arange(i0, min(Sq, i0 + step), device=q.device)
            qpos = i + Sk - Sq
            visible = torch.ones((len(i), Sk), dtype=torch.bool, device=q.device)
            if case["causal"]:
                visible = j[None] <= qpos[:, None]
                if "prefix" in state:
                    visible = visible | (j < state["prefix"][b])[None]
            if "mask" in state:
                visible = visible & (state["mask"][b] != 0)[None]
            if "k_doc" in state:
                visible = visible & (state["q_doc"][b][i][:, None] == state["k_doc"][b][None])
            out[b, i0:i0 + len(i)] = _plain_attention(
                q[b, i0:i0 + len(i)].float(), kb, vb, visible, qpos, j,
                1.0 / math.sqrt(case["hd"]), case["softcap"], state.get("slopes")).to(q.dtype)
    return out


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        from paper_2509_16248_amd import ops
        if op == "kv":
            cache = state["cache"]
            if case["store"]:
                cache.write(state["k"], state["v"], state["start"], count=state["count"])
            return cache.read(case["n"], start=state["start"], count=state["count"],
                              dtype=_DTYPE[case["dtype"]])
        if op == "cached":
            return ops.cached_attention(state["q"], state["cache"], state["lengths"],
                                        softcap=case["softcap"], slopes=state.get("slopes"))
        return ops.attention(state["q"], state["k"], state["v"], causal=case["causal"],
                             softcap=case["softcap"], slopes=state.get("slopes"),
                             key_mask=state.get("mask"), q_doc=state.get("q_doc"),
                             k_doc=state.get("k_doc"), prefix=state.get("prefix"))
    if op == "kv":
        if case["store"]:
            _plain_write(state["cache"], state["k"], state["v"], state["start"], state["count"],
                         case["bits"])
        return _plain_read(state["cache"], state["start"], state["count"], case["n"],
                           _DTYPE[case["dtype"]])
    if op == "cached":
        return _plain_cached(state, case)
    return _plain_prompt(state, case)


# ------------------------------------------------------------ work
def _visible_pairs(case):
    """(query, key) pairs that the masks leave, over the batch, of one head."""
    Sq, Sk = case["sq"], case["sk"]
    docs = torch.tensor(_doc_ids(Sk, case["docs"])) if case["docs"] else None
    total = 0
    for b in range(case["batch"]):
        n = _visible_lengths(case)[b]
        pre = _prefixes(case)[b] if case["prefix"] else 0
        # keys of query position p: [lo, hi), from its document's start on
        p = torch.arange(Sk - Sq, Sk)
        hi = torch.clamp(torch.full_like(p, Sk) if not case["causal"] else
                         torch.maximum(p + 1, torch.tensor(pre)), max=n)
        lo = torch.zeros_like(p)
        if docs is not None:
            first = torch.searchsorted(docs, docs[p])
            last = torch.searchsorted(docs, docs[p], right=True)
            lo, hi = first, torch.minimum(hi, last)
        total += int(torch.clamp(hi - lo, min=0).sum())
    return total


def work(case):
    e, hd = _BYTES[case["dtype"]], case["hd"]
    if case["op"] == "kv":
        rows = sum(_counts(case)) * case["heads"] * 2
        held = rows * (hd * case["bits"] // 8 + hd // _GROUP * 2)
        plain = rows * hd * e
        return {"bytes": (held + plain) * (2 if case["store"] else 1), "flops": 0}
    q = case["batch"] * case["sq"] * case["heads"] * hd * e
    if case["op"] == "cached":
        keys = sum(_lengths(case))
        held = keys * case["kv_heads"] * 2 * (hd * case["bits"] // 8 + hd // _GROUP * 2)
        pairs = sum(case["sq"] * n - case["sq"] * (case["sq"] - 1) // 2 for n in _lengths(case))
        return {"bytes": held + 2 * q, "flops": 4 * hd * pairs * case["heads"]}
    kv = 2 * case["batch"] * case["sk"] * case["kv_heads"] * hd * e
    return {"bytes": kv + 2 * q, "flops": 4 * hd * case["heads"] * _visible_pairs(case)}


# ------------------------------------------------------------ exact
def _exact_stored(x, bits):
    """Values that the cache stands for, float64, [..., hd]."""
    top = 127.0 if bits == 8 else 7.0
    x64 = x.double().reshape(*x.shape[:-1], x.shape[-1] // _GROUP, _GROUP)
    largest = torch.max(torch.abs(x64), dim=-1, keepdim=True).values
    reciprocal = torch.tensor(1.0 / top, dtype=torch.float32).double().item()
    scale = (largest * reciprocal).to(torch.float32).to(torch.bfloat16).double()
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    codes = torch.minimum(torch.maximum(torch.round(x64 / safe), torch.tensor(-top, device=x.device)),
                          torch.tensor(top, device=x.device))
    return (codes * scale).reshape(x.shape)


def _exact_head(q, k, v, bias, hidden, cap, scale):
    """One head: q [Sq, hd], k and v [Sk, hd], bias and hidden [Sq, Sk]."""
    logits = (q @ k.t().contiguous()) * scale
    if cap:
        logits = cap * torch.tanh(logits / cap)
    if bias is not None:
        logits = logits + bias
    logits[hidden] = -math.inf
    lse = torch.logsumexp(logits, dim=1, keepdim=True)
    weights = torch.exp(logits - lse)
    weights[torch.isinf(lse).expand_as(weights)] = 0.0
    return weights @ v


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "kv":
        count = x["count"]
        result = []
        for t in (x["k"], x["v"]):
            vals = _exact_stored(t, case["bits"])
            for b in range(case["batch"]):
                vals[b, int(count[b]):] = 0.0
            result.append(vals)
        return result
    q = x["q"].double()
    B, Sq, H, hd = q.shape
    G = H // case["kv_heads"]
    if case["op"] == "cached":
        k, v = _exact_stored(x["k"], case["bits"]), _exact_stored(x["v"], case["bits"])
    else:
        k, v = x["k"].double(), x["v"].double()
    Sk = k.shape[1]
    out = torch.zeros_like(q)
    keys = torch.arange(Sk, device=q.device).view(1, -1)
    for b in range(B):
        n = int(x["lengths"][b]) if case["op"] == "cached" else Sk
        for i0 in range(0, Sq, 2048):
            rows = torch.arange(i0, min(Sq, i0 + 2048), device=q.device).view(-1, 1)
            at = rows + (n - Sq)
            if case["op"] == "cached":
                hidden = keys > at
            else:
                hidden = torch.zeros((rows.shape[0], Sk), dtype=torch.bool, device=q.device)
                if case["causal"]:
                    hidden |= keys > at
                if case["prefix"]:
                    hidden &= keys >= int(x["prefix"][b])
                if case["pads"]:
                    hidden |= (x["mask"][b] == 0).view(1, -1)
                if case["docs"]:
                    hidden |= x["q_doc"][b].view(-1, 1)[i0:i0 + 2048] != x["k_doc"][b].view(1, -1)
            for h in range(H):
                bias = None
                if case["alibi"]:
                    bias = -float(x["slopes"][h]) * torch.abs(at - keys).double()
                out[b, i0:i0 + 2048, h] = _exact_head(
                    q[b, i0:i0 + 2048, h], k[b, :, h // G], v[b, :, h // G], bias, hidden,
                    case["softcap"], 1.0 / math.sqrt(hd))
    return out
