"""Plain float64 definitions of the operators over a paged cache, and the random
calls that the tests make of them."""
import math

import torch

import ops_reference as ref

DT = ref.DT


class Call:
    """Sequences with pages handed out in a shuffled order: their table, lengths and new
    tokens (uniform: n each; packed: new[b] each), on the host."""

    def __init__(self, lengths, new, page_size, packed, seed=0, width=None, spare=2, holes=()):
        g = torch.Generator().manual_seed(seed)
        self.lengths, self.new, self.ps, self.packed = list(lengths), list(new), page_size, packed
        B = len(self.lengths)
        self.width = width or max(1, -(-max([1, *self.lengths]) // page_size))
        self.pages = B * self.width + spare
        order = torch.randperm(self.pages, generator=g)[:B * self.width]
        self.table = order.reshape(B, self.width).int()
        for b, i, value in holes:
            self.table[b, i] = value
        self.cap = self.width * page_size
        self.offsets = [sum(self.new[:b]) for b in range(B + 1)]

    def tokens(self, extra=0):
        if self.packed:
            return (self.offsets[-1] + extra,)
        assert len(set(self.new)) == 1
        return (len(self.lengths), self.new[0])

    def device_args(self, device="cuda"):
        t = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
        return (self.table.to(device), t(self.lengths)), (
            {"offsets": t(self.offsets)} if self.packed else {})

    def rows(self, x):
        """[(sequence, position of its first new token, its rows [n, heads, hd])]."""
        out = []
        for b, (n, length) in enumerate(zip(self.new, self.lengths)):
            r = x[self.offsets[b]:self.offsets[b + 1]] if self.packed else x[b]
            out.append((b, length - n, r))
        return out

    def place(self, b, pos):
        """(page, slot) of a position, or None."""
        if not 0 <= pos < self.cap:
            return None
        page = int(self.table[b, pos // self.ps])
        return (page, pos % self.ps) if 0 <= page < self.pages else None


def rotated(x, cos, sin, pos):
    """x [heads, hd] float64 at a position, and the size of the products in each channel."""
    h = cos.shape[1]
    c, s = cos[pos].double(), sin[pos].double()
    lo, hi = x[:, :h], x[:, h:2 * h]
    y, size = x.clone(), torch.zeros_like(x)
    y[:, :h], y[:, h:2 * h] = lo * c - hi * s, hi * c + lo * s
    size[:, :h], size[:, h:2 * h] = (lo * c).abs() + (hi * s).abs(), (hi * c).abs() + (lo * s).abs()
    return y, size


def append(call, k, v, k_pages, v_pages, rotary=None, q=None, q_out=None):
    """Float64 (k_pages, v_pages, q_out) after the call, each with how far a kernel may be
    off: half a step of the type for its rounding, and one rounding of a product and one of
    the sum in fp32, 2^-23 of their size in all; what is copied, and what is not
    written, exactly."""
    u = torch.finfo(k.dtype).eps / 2
    tiny = torch.finfo(k.dtype).tiny * u
    out = [t.double().clone() for t in (k_pages, v_pages)]
    tol = [torch.zeros_like(t) for t in out]
    if q is not None:
        out.append(q_out.double().clone())
        tol.append(torch.zeros_like(out[2]))

    def turn(x, pos):
        x = x.double()
        if rotary is None:
            return x, torch.zeros_like(x)
        y, size = rotated(x, *rotary, pos)
        t = u * y.abs() + 2.0 ** -23 * (1 + u) * size + tiny * (size > 0)
        return y, torch.where(size > 0, t, 0.0)

    for which, x in (("k", k), ("v", v)):
        for b, p0, rows in call.rows(x):
            for i in range(rows.shape[0]):
                at = call.place(b, p0 + i)
                if at is None:
                    continue
                n = 0 if which == "k" else 1
                y, t = turn(rows[i], p0 + i) if which == "k" else (rows[i].double(), 0.0)
                out[n][at[0], :, at[1]] = y
                tol[n][at[0], :, at[1]] = t
    if q is not None:
        for (b, p0, rows), (_, _, dst), (_, _, t) in zip(call.rows(q), call.rows(out[2]),
                                                         call.rows(tol[2])):
            for i in range(rows.shape[0]):
                if 0 <= p0 + i < call.cap:
                    dst[i], t[i] = turn(rows[i], p0 + i)
                else:
                    dst[i] = 0.0
    return out, tol


def attention(call, q, k_pages, v_pages, window=0, softcap=0.0, slopes=None, scale=None, out=None):
    """(float64 result shaped as q, tolerance); rows of no sequence keep what `out` has."""
    hd = q.shape[-1]
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    res = torch.zeros(q.shape, dtype=torch.float64) if out is None else out.double().clone()
    tol = torch.zeros(q.shape, dtype=torch.float64)
    for (b, p0, rows), (_, _, r), (_, _, t) in zip(call.rows(q), call.rows(res), call.rows(tol)):
        n = rows.shape[0]
        S = max(0, min(call.lengths[b], call.cap))
        if n == 0:
            continue
        if S == 0:
            r.zero_()
            continue
        pos = torch.arange(S)
        page = call.table[b].long()[pos // call.ps]
        ok = (page >= 0) & (page < call.pages)
        pg = torch.where(ok, page, 0)
        k, v = (x[pg, :, pos % call.ps] for x in (k_pages, v_pages))
        i = torch.arange(n)[:, None] + p0
        seen = (pos[None] <= i) & ok[None]
        if window:
            seen &= pos[None] > i - window
        # what nobody sees may hold anything
        dark = ~seen.any(0)
        k, v = (torch.where(dark[:, None, None], 0.0, x.double()).to(x.dtype) for x in (k, v))
        part = torch.zeros_like(t)
        # fp16 probabilities are held times 2^7: half a step of the subnormals is 2^-32
        r[:] = ref.attention(rows, k, v, seen, i - pos[None], scale, softcap, slopes, part,
                             2.0 ** -32 if q.dtype == torch.float16 else 0.0)
        t[:] = part
    return res, tol
