"""Plain definitions of the operators around the paged 8-bit cache (include/fluxbin_serve.h): rotations, drafted trees, kept
rows and pages. Test infrastructure: loops and fp64 where a result is rounded, the format's fp32 steps where it is exact."""
import numpy as np

from oracle import quant_oracle as qo

F32 = np.float32


# ---------------------------------------------------------------------------------------------- norm and rotation

def rotate(x, positions, frequencies, weight=None, eps=1e-6, magnitude=1.0, interleaved=False):
    """(y, size) fp64 of x fp16 [T, H, D]: the result, and of every element the sum of the magnitudes that it is made of."""
    x = x.astype(np.float64)
    D, R = x.shape[-1], 2 * len(frequencies)
    if weight is not None:
        x = x / np.sqrt((x * x).sum(-1, keepdims=True) / D + eps) * weight.astype(np.float64)
    y, size = x.copy(), np.abs(x)
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        angle = positions.astype(np.float64) * float(frequencies[i])
        c, s = (magnitude * f(angle)[:, None] for f in (np.cos, np.sin))
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(magnitude)
    return y, size


def rotate_bound(y, size):
    """How far fp32 arithmetic and one rounding to fp16 may be from y. The mean of squares: 16 fused steps and up to 4 sums
    over lanes, 20 * 2^-24 of it, and so half as much of the root, whose function adds 2 * 2^-24; two products 2 * 2^-24. The
    angle, at most half a turn, is rounded to 2^-25 turns, 2^-22.3 radians; the functions add 2 ulp, 2^-22, with the magnitude
    2^-24. The turn's two products and sum 2 * 2^-24. In units of 2^-24: 10 + 2 + 2 + 3.3 + 4 + 1 + 2 < 32, of the magnitudes
    that an element is made of. Then half a step of fp16, 2^-11 of the value or 2^-25 among its smallest."""
    off = size * 2.0 ** -19
    return off + (np.abs(y) + off) * 2.0 ** -11 + 2.0 ** -25


# ---------------------------------------------------------------------------------------------- drafted trees

def tree_masks(parents, offsets, context, words, T):
    """masks bool [T, 64 words], positions [T], and which rows are written."""
    masks, positions, written = np.zeros((T, 64 * words), bool), np.zeros(T, np.int64), np.zeros(T, bool)
    for b in range(len(context)):
        o0, o1 = int(offsets[b]), int(offsets[b + 1])
        if not (0 <= o0 <= o1 <= T) or o1 - o0 > 64 * words:
            continue
        written[o0:o1] = True
        for i in range(o1 - o0):
            p = int(parents[o0 + i])
            if 0 <= p < i:
                masks[o0 + i] = masks[o0 + p]
            positions[o0 + i] = min(max(0, int(context[b])), 1 << 30) - (o1 - o0) + masks[o0 + i].sum()
            masks[o0 + i, i] = True
    return masks, positions, written


def packed(masks):
    """int64 words of bool [T, 64 words]."""
    return np.packbits(masks, axis=1, bitorder="little").view(np.int64)


class Kv8(qo.Kv8):
    """The paged cache of quant_oracle with trees and kept rows."""

    def tree_attention(self, q, masks, offsets, context, table, scale, window=0):
        """As attention() of a cache, with masks bool [T, 64 words]."""
        T, Hq, D = q.shape
        H = self.codes.shape[3]
        out, mag, big, peak = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq)), np.zeros((T, Hq))
        written = np.zeros(T, bool)
        for b in range(len(context)):
            o0, o1 = int(offsets[b]), int(offsets[b + 1])
            if not (0 <= o0 <= o1 <= T) or o1 - o0 > masks.shape[1]:
                continue
            written[o0:o1] = True
            n, c = o1 - o0, max(0, int(context[b]))
            seen = np.zeros((n, max(c, n)), bool)
            for i in range(n):
                for j in range(max(0, c - n)):
                    seen[i, j] = True
                for j in range(n):
                    if masks[o0 + i, j] and c - n + j >= 0:
                        seen[i, c - n + j] = True
                if window > 0:
                    at = np.flatnonzero(seen[i])
                    seen[i, at[:max(0, len(at) - window)]] = False
            keys = min(c, table.shape[1] * self.P)
            k, ok = self.values(0, b, keys, table)
            v, _ = self.values(1, b, keys, table)
            scale_at = np.stack([self.scales[1, max(0, self.page(table, b, i))] for i in range(keys)] or [np.zeros(H)])
            seen = seen[:, :keys] & ok[None]
            some = seen.any(1)
            for h in range(Hq):
                kk, vv, qq = k[:, h // (Hq // H)], v[:, h // (Hq // H)], q[o0:o1, h].astype(np.float64)
                s = np.where(seen, qq @ kk.T * scale, -np.inf)
                e = np.exp(s - np.where(some, s.max(1, initial=-np.inf), 0.0)[:, None])
                e /= np.where(some, e.sum(1), 1.0)[:, None]
                out[o0:o1, h], mag[o0:o1, h] = e @ vv, e @ np.abs(vv)
                big[o0:o1, h] = np.where(seen, np.abs(qq) @ np.abs(kk).T, 0.0).max(1, initial=0.0) * abs(scale)
                peak[o0:o1, h] = (e * 127 * scale_at[:keys, h // (Hq // H)]).max(1, initial=0.0)
        return out, mag, big, peak, written

    def keep(self, keep, kept, offsets, context, table, T):
        for b in range(len(context)):
            o0, o1 = int(offsets[b]), int(offsets[b + 1])
            if not (0 <= o0 <= o1 <= T):
                continue
            n = o1 - o0
            base, m = max(0, int(context[b])) - n, min(max(0, int(kept[b])), n)
            pages = {}
            for k in range(m):
                if base + k >= 0:
                    pages.setdefault((base + k) // self.P, []).append((base + int(keep[o0 + k]), base + k))
            for moves in pages.values():
                page, first = self.page(table, b, moves[0][1]), moves[0][1] % self.P
                if page < 0 or all(of == to for of, to in moves):
                    continue
                source = [(self.page(table, b, of), of % self.P) for of, _ in moves]
                for side in (0, 1):
                    zero = np.zeros_like(self.scales[side, 0])
                    of = [self.scales[side, p].copy() if p >= 0 else zero for p, _ in source]
                    rows = [self.codes[side, p, i].copy() if p >= 0 else np.zeros_like(self.codes[side, 0, 0]) for p, i in source]
                    own = self.scales[side, page].copy() if first > 0 else zero
                    s = np.max(of + [own], axis=0).astype(F32)
                    some = np.where(s > 0, s, F32(1))
                    brought = lambda c, was: np.rint(c.astype(F32) * np.where(was < s, was / some, F32(1)).astype(F32)[:, None]).astype(np.int32)
                    for i in range(first):
                        self.codes[side, page, i] = brought(self.codes[side, page, i], own)
                    for (_, to), row, was in zip(moves, rows, of):
                        self.codes[side, page, to % self.P] = brought(row, was)
                    self.scales[side, page] = s


# ---------------------------------------------------------------------------------------------- pages

class Pool:
    """References of pages; tables are numpy arrays that the calls change."""

    def __init__(self, pages, P):
        self.refs, self.P, self.missing = np.zeros(pages, np.int64), P, 0

    def held(self, row):
        n = 0
        while n < len(row) and 0 <= row[n] < len(self.refs):
            n += 1
        return n

    def take(self):
        free = np.flatnonzero(self.refs <= 0)
        if len(free) == 0:
            self.missing += 1
            return -1
        self.refs[free[0]] = 1
        return int(free[0])

    def resize(self, table, tokens):
        self.missing = 0
        need = [-1 if t < 0 else min(-(-int(t) // self.P), table.shape[1]) for t in tokens]
        for row, n in zip(table, need):
            if n >= 0:
                h = self.held(row)
                for p in range(n, h):
                    self.refs[row[p]] -= 1
                    row[p] = -1
        for row, n in zip(table, need):
            for p in range(self.held(row), max(0, n)):
                row[p] = self.take()

    def fork(self, table, context, source, children):
        """Changes children; returns copies [C, 2]."""
        self.missing = 0
        copies = np.full((len(source), 2), -1, np.int32)
        children[:] = -1
        fresh = []
        for c, b in enumerate(source):
            if not 0 <= b < len(table):
                continue
            tokens, row = max(0, int(context[b])), table[b]
            cap = min(table.shape[1], children.shape[1])
            for p in range(min(tokens // self.P, cap, self.held(row))):
                children[c, p] = row[p]
                self.refs[row[p]] += 1
            p = tokens // self.P
            if tokens % self.P and p < cap and 0 <= row[p] < len(self.refs):
                fresh.append((c, p, int(row[p])))
        for c, p, old in fresh:
            new = self.take()
            children[c, p] = new
            if new >= 0:
                copies[c] = old, new
        return copies
