"""Plain 64-bit NumPy forms of the operators around the prefill: norm of each
head and rotation by position, 4-bit storage, and attention over a paged cache.
Written from the formulas in include/proxyattn.h; shares no code with the HIP
path."""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def round_to(x, dtype: str):
    """x (64 bits) rounded to fp32, then for "bf16" to its nearest bf16 (ties to
    even), as 64-bit values."""
    f = np.asarray(x, np.float64).astype(np.float32)
    if dtype == "bf16":
        u = f.view(np.uint32).astype(np.uint64)
        u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
        f = u.astype(np.uint32).view(np.float32)
    return f.astype(np.float64)


def norm_rotate(x, positions, rot=0, interleaved=False, cos=None, sin=None, weight=None, eps=1e-6):
    """x [T][H][d] of tokens at `positions`, normed with a weight and rotated; not rounded."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if not rot:
        return x
    y = x.copy()
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c = cos[positions, j].astype(np.float64)[:, None]
        s = sin[positions, j].astype(np.float64)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def quantise(x):
    """Values [..., d] as codes [..., d / 2] uint8 and scales [..., d / 32] uint8."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(g).max(axis=-1)
    e = np.full(top.shape, -110)
    while True:   # the smallest power of two that no value is over 7 of
        low = (top > 7 * 2.0 ** e) & (e < 125)
        if not low.any():
            break
        e = e + low
    a = np.abs(g) / 2.0 ** e[..., None]
    dist = np.abs(a[..., None] - GRID)
    best = dist.min(axis=-1, keepdims=True)
    tie = dist == best   # one, or two neighbours: the even code of these
    code = np.where(tie, np.arange(8) + 100 * (np.arange(8) % 2), 1000).argmin(axis=-1)
    code = code + 8 * np.signbit(g)
    code = code.reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).astype(np.uint8), (e + 127).astype(np.uint8)


def dequantise(codes, scales):
    nib = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], codes.shape[-1] // 16, 32)
    v = np.where(nib & 8, -1.0, 1.0) * GRID[nib & 7]
    return (v * 2.0 ** (scales.astype(np.float64) - 127)[..., None]).reshape(
        *codes.shape[:-1], 2 * codes.shape[-1])


def batch(seq_lens, new_start, num_seqs):
    """(sequence, position) of each of the batch's tokens."""
    if new_start is None:
        new_start = list(range(num_seqs + 1))
    out = []
    for b in range(num_seqs):
        n = new_start[b + 1] - new_start[b]
        out += [(new_start[b] + j, b, seq_lens[b] - n + j) for j in range(n)]
    return out


def attention(q, keys, values, tokens, scale):
    """q [T][Hq][d]; keys, values: [n][Hkv][d] of each sequence; tokens as from
    batch().  Returns out, lse, and for the error bounds the probabilities'
    sum of |v| and the largest sum of |c q k|."""
    t, hq, d = q.shape
    out, lse = np.zeros((t, hq, d)), np.full((hq, t), -np.inf)
    absv, big = np.zeros((t, hq, d)), np.zeros((t, hq))
    for row, b, pos in tokens:
        if pos < 0:
            continue
        k, v = keys[b][:pos + 1], values[b][:pos + 1]
        rep = hq // k.shape[1]
        for i in range(hq):
            s = scale * (k[:, i // rep] @ q[row, i])
            top = s.max()
            p = np.exp(s - top)
            lse[i, row] = top + np.log(p.sum())
            p /= p.sum()
            out[row, i] = p @ v[:, i // rep]
            absv[row, i] = p @ np.abs(v[:, i // rep])
            big[row, i] = scale * (np.abs(k[:, i // rep]) @ np.abs(q[row, i])).max()
    return out, lse, absv, big
