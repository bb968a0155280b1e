"""Plain NumPy definitions of the operators declared in include/fluxbin_quant.h: 4-bit linears, and the
paged 8-bit key/value cache with its attention. What a kernel computes in
32 bits and stores (scales, codes) is computed here with the same 32-bit operations, products and sums in 64 bits."""
from __future__ import annotations

import numpy as np

F32 = np.float32


def _groups(W, g):
    """W fp32 [M, N] padded with zeros to [M, G, width]; NaN as 0, values past fp16's range as its largest."""
    M, N = W.shape
    g = min(g, N)
    G = -(-N // g)
    w = np.clip(np.nan_to_num(W.astype(F32), nan=0.0, posinf=65504.0, neginf=-65504.0), F32(-65504), F32(65504))
    out = np.zeros((M, G * g), F32)
    out[:, :N] = w
    return out.reshape(M, G, g)


def w4_quantize(W, g, asym):
    """(codes uint8 [M, N], scales fp16 [M, G], zeros uint8 [M, G]); zeros are 8 without zero points."""
    M, N = W.shape
    w = _groups(W, g)
    lo, hi = np.minimum(w.min(-1), F32(0)), np.maximum(w.max(-1), F32(0))
    scales = np.abs(((hi - lo) * (F32(1) / F32(15)) if asym else np.maximum(hi, -lo) * (F32(1) / F32(7))).astype(np.float16))
    s = scales.astype(F32)
    inv = np.zeros_like(s)
    inv[s > 0] = F32(1) / s[s > 0]
    r = np.rint(w * inv[..., None])
    if asym:
        z = np.clip(np.rint(-lo * inv), 0, 15)
        q = np.clip(r + z[..., None], 0, 15)
    else:
        z = np.full_like(s, 8)
        q = np.clip(r, -8, 7) + 8
    return q.reshape(M, -1)[:, :N].astype(np.uint8), scales, z.astype(np.uint8)


def w4_words(codes):
    """uint32 [M, ceil(N/8)]: column 8 w + t in bits 4 t of word w."""
    M, N = codes.shape
    c = np.zeros((M, -(-N // 8) * 8), np.uint32)
    c[:, :N] = codes
    return (c.reshape(M, -1, 8) << (4 * np.arange(8, dtype=np.uint32))).sum(-1, dtype=np.uint32)


def w4_dense(codes, scales, zeros, g):
    """(q - z) s in fp64 [M, N]."""
    at = np.arange(codes.shape[1]) // g
    return (codes.astype(np.int64) - zeros.astype(np.int64)[:, at]) * scales.astype(np.float64)[:, at]


def w4_depth(N):
    """Additions on the longest path of a product's sum: 128 in a group, then one per group, and 32 for the parts of the
    columns."""
    return 128 + -(-N // 32) + 32


def w4_bound(W, x, half):
    """How far a product may be from W x (fp64 [B, M]): per row one rounding of 2^-23 of the sum of magnitudes for each
    addition on the longest path; an fp16 result half a step more."""
    bound = w4_depth(W.shape[1]) * 2.0 ** -23 * (np.abs(x) @ np.abs(W).T)
    if half:
        bound = bound * (1 + 2.0 ** -11) + np.abs(x @ W.T) * 2.0 ** -11 + 2.0 ** -25
    return bound


# ---------------------------------------------------------------------------------------------- 8-bit cache

class Kv8:
    """A paged cache: codes int32 [2, pages, P, H, D] and scales fp32 [2, pages, H], keys first."""

    def __init__(self, pages, P, H, D):
        self.P, self.pages = P, pages
        self.codes = np.zeros((2, pages, P, H, D), np.int32)
        self.scales = np.zeros((2, pages, H), F32)

    def page(self, table, b, pos):
        p = pos // self.P
        if pos < 0 or p >= table.shape[1]:
            return -1
        page = int(table[b, p])
        return page if 0 <= page < self.pages else -1

    def append(self, k, v, offsets, context, table):
        """k, v fp16 [T, H, D]."""
        T = k.shape[0]
        for b in range(len(context)):
            o0, o1 = int(offsets[b]), int(offsets[b + 1])
            if not (0 <= o0 <= o1 <= T):
                continue
            i = o0
            while i < o1:
                pos = int(context[b]) - (o1 - i)
                n = 1 if pos < 0 else min(o1 - i, self.P - pos % self.P)
                page = self.page(table, b, pos)
                if page >= 0:
                    for side, x in ((0, k), (1, v)):
                        self._store(side, page, pos % self.P, x[i:i + n])
                i += n

    def _store(self, side, page, first, x):
        x = np.clip(np.nan_to_num(x.astype(F32), nan=0.0, posinf=65504.0, neginf=-65504.0), F32(-65504), F32(65504))
        old = self.scales[side, page] if first > 0 else np.zeros_like(self.scales[side, page])
        s = np.maximum(old, np.abs(x).max((0, 2)) * (F32(1) / F32(127)))
        inv = np.where(s > 0, F32(1) / np.where(s > 0, s, F32(1)), F32(0)).astype(F32)
        ratio = np.where(s > old, old / np.where(s > 0, s, F32(1)), F32(1)).astype(F32)
        c = self.codes[side, page]
        c[:first] = np.rint(c[:first].astype(F32) * ratio[None, :, None]).astype(np.int32)
        c[first:first + x.shape[0]] = np.clip(np.rint(x * inv[None, :, None]), -127, 127).astype(np.int32)
        self.scales[side, page] = s

    def values(self, side, b, count, table):
        """fp64 [count, H, D] of positions 0 .. count - 1, and which of them have a page."""
        out = np.zeros((count,) + self.codes.shape[3:])
        ok = np.zeros(count, bool)
        for p0 in range(0, count, self.P):
            page, n = self.page(table, b, p0), min(self.P, count - p0)
            if page >= 0:
                out[p0:p0 + n] = self.codes[side, page, :n] * self.scales[side, page].astype(np.float64)[None, :, None]
                ok[p0:p0 + n] = True
        return out, ok

    def read(self, offsets, context, table, T):
        """(k, v) fp16 [T, H, D] and the rows that are written."""
        out = np.zeros((2, T) + self.codes.shape[3:], np.float16)
        written = np.zeros(T, bool)
        for b in range(len(context)):
            o0, o1 = int(offsets[b]), int(offsets[b + 1])
            if not (0 <= o0 <= o1 <= T):
                continue
            written[o0:o1] = True
            c = max(0, int(context[b]))
            for side in (0, 1):
                x, _ = self.values(side, b, c, table)
                for i in range(o0, o1):
                    pos = c - (o1 - i)
                    if pos >= 0:
                        out[side, i] = x[pos].astype(F32).astype(np.float16)
        return out[0], out[1], written

    def attention(self, q, offsets, context, table, scale, causal=True, window=0):
        """out fp64 [T, Hq, D] and, for bounds, sum_j p_j |v_j|, and per row and head the largest score's magnitude and the
        largest p_j times 127 scales of its page's values."""
        T, Hq, D = q.shape
        H = self.codes.shape[3]
        out, mag, big, peak = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq))
        written = np.zeros(T, bool)
        for b in range(len(context)):
            o0, o1 = int(offsets[b]), int(offsets[b + 1])
            if not (0 <= o0 <= o1 <= T):
                continue
            written[o0:o1] = True
            c = max(0, int(context[b]))
            n = min(c, table.shape[1] * self.P)
            k, ok = self.values(0, b, n, table)
            v, _ = self.values(1, b, n, table)
            scale_at = np.stack([self.scales[1, max(0, self.page(table, b, i))] for i in range(n)] or [np.zeros(H)])
            pos = c - np.arange(o1 - o0, 0, -1)[:, None]
            j = np.arange(n)[None]
            seen = np.broadcast_to(ok[None], (o1 - o0, n)).copy()
            if causal:
                seen &= j <= pos
            if window > 0:
                seen &= j > pos - window
            some = seen.any(1)
            for h in range(Hq):
                kk, vv, qq = k[:, h // (Hq // H)], v[:, h // (Hq // H)], q[o0:o1, h].astype(np.float64)
                s = np.where(seen, qq @ kk.T * scale, -np.inf)
                e = np.exp(s - np.where(some, s.max(1, initial=-np.inf), 0.0)[:, None])
                e /= np.where(some, e.sum(1), 1.0)[:, None]
                out[o0:o1, h], mag[o0:o1, h] = e @ vv, e @ np.abs(vv)
                big[o0:o1, h] = np.where(seen, np.abs(qq) @ np.abs(kk).T, 0.0).max(1, initial=0.0) * abs(scale)
                peak[o0:o1, h] = (e * 127 * scale_at[:n, h // (Hq // H)]).max(1, initial=0.0)
        return out, mag, big, peak, written


def attention_bound(out, mag, big, peak, keys, chunk=False, log2_scale=64):
    """How far fp32 attention may be from `out`. A score is a sum of D <= 256 exact products: off by at most 300 * 2^-23 of
    its terms' magnitudes (`big`), and after conversion to base 2 with the logarithm of a scale (up to 2^6, or what the
    caller knows: `log2_scale`) by 8 * 2^-23 of big + 64 more; so every weight by that factor, and 2^-20 for exponentials,
    reciprocals and its 21 bits; sums over keys by (keys / 4 + 64) * 2^-23. Numerator and denominator both: twice. Weights
    are fed as fp16 numbers of which the largest (with its page's value scale in it) is at least 2^8, and those are
    multiples of 2^-24: each may be off by 2^-25, 2^-33 of the largest, times a code of up to 127, which is 2^-33 of `peak`
    for each key. The result is rounded to fp16. chunk: room for weights of one fp16 number (half a step: 2^-11), which no
    form has; attention_apart tells them."""
    eps = 2 * ((300 * big + 8 * (big + log2_scale)) * 2.0 ** -23 + 2.0 ** -20 + (keys / 4 + 64) * 2.0 ** -23)
    if chunk:
        eps = eps + 2.0 ** -11
    off = eps[..., None] * mag + (keys * 2.0 ** -33 * peak)[..., None]
    return off * (1 + 2.0 ** -11) + np.abs(out) * 2.0 ** -11 + 2.0 ** -25


# Norm of the difference to the fp16-rounded reference, relative to the reference's norm, that attention in fp32 with weights
# of two fp16 numbers may have on ordinary data (attention_apart).
APART = 2.0 ** -13


def attention_apart(got, ref):
    """How far fp16 results are from the 64-bit reference rounded to fp16, relative to the reference's norm: what is left
    when the final rounding, which would cover errors of its own size, is taken out.

    An element whose value before that rounding is off by e differs by a step u where a border between two fp16 numbers
    lies between it and the reference, which over many elements happens to |e| / u of them. The sum of the squares is then
    about the sum of |e| u, at most |e| |u| <= t 2^-10 of the reference's square where t is the error's norm relative to the
    reference's. fp32 arithmetic whose roundings are independent has t below 2^-17: scores of magnitude up to 16 are rounded
    a few times (2^-21 each time), their sums over D <= 256 products add sqrt(D) 2^-24 of the largest, sums over keys less,
    a weight of two fp16 numbers 2^-21. So the result is below 2^-13.5, and APART is one and a half times that. One fp16
    number for a weight (t = 2^-12.3) gives 2^-11.2; scores in fp16 (2^-11 of magnitudes above 1) or weights in bf16 more."""
    ref = np.asarray(ref, np.float64)
    return float(np.linalg.norm(np.asarray(got, np.float64) - ref.astype(np.float16).astype(np.float64)) / np.linalg.norm(ref))
