"""Plain NumPy definitions of the operators declared in include/fluxbin_quant.h: 4-bit linears. What a kernel computes in
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


def w4_bound(W, x, half):
    """How far a product may be from W x (fp64 [B, M]): per row one rounding of 2^-23 of the sum of magnitudes for each
    addition on the longest path (128 in a group, then one per group, and 32 for the parts of the columns); an fp16 result
    half a step more."""
    depth = 128 + -(-W.shape[1] // 32) + 32
    bound = depth * 2.0 ** -23 * (np.abs(x) @ np.abs(W).T)
    if half:
        bound = bound * (1 + 2.0 ** -11) + np.abs(x @ W.T) * 2.0 ** -11 + 2.0 ** -25
    return bound
