"""What lies between a model's scans and after its last layer, in 64 bits -- TEST INFRASTRUCTURE ONLY.

Plain numpy from the definitions: the norm with the residual's addition and its gradients, 8-bit floats (e4m3) with scales
and their products, and the choice of the next token.  No code is shared with the library.  Only ``tests/`` may import
this module.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128


def rms_norm(h, weight=None, eps=1e-5):
    """y and 1 / sqrt(mean(h^2) + eps) of the rows of h."""
    h = np.asarray(h, dtype=np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(-1) + eps)
    y = h * rstd[..., None]
    return (y if weight is None else y * np.asarray(weight, np.float64)), rstd


def rms_norm_grad(dy, h, rstd, weight=None, dh=None):
    """d (dx and dresidual) and dweight, row after row."""
    dy, h, rstd = (np.asarray(a, dtype=np.float64) for a in (dy, h, rstd))
    w = np.ones(h.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    d, dw = np.zeros_like(h), np.zeros(h.shape[-1])
    for i in range(h.shape[0]):
        u, g = h[i] * rstd[i], dy[i] * w
        d[i] = rstd[i] * (g - u * (g * u).mean())
        dw += dy[i] * u
    return (d if dh is None else d + np.asarray(dh, np.float64)), dw


def _e4m3():
    """The 256 values: sign, 4 bits of exponent (bias 7), 3 of mantissa; all ones is NaN, and there is no infinity."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = -v if c & 128 else v
    return out


E4M3 = _e4m3()


def to_e4m3(v):
    """The nearest codes, ties to the even one.  |v| up to 448 and a half step."""
    v = np.asarray(v, dtype=np.float64)
    high = E4M3[:127]                                   # 0 to 448, rising
    at = np.searchsorted(high, np.abs(v)).clip(1, 126)
    below, above = high[at - 1], high[at]
    gap_low, gap_high = np.abs(v) - below, above - np.abs(v)
    up = (gap_high < gap_low) | ((gap_high == gap_low) & (at % 2 == 0))
    code = np.where(up, at, at - 1).astype(np.int64)
    code = np.where(np.isnan(v), 127, code)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def block_tops(x, tile):
    """The largest magnitude of each block of 128 columns of a row, or of each tile; a NaN is passed over."""
    x = np.abs(np.asarray(x))
    rows, cols = x.shape
    x = np.where(np.isnan(x), 0, x)
    out = np.zeros((-(-rows // BLOCK) if tile else rows, -(-cols // BLOCK)), x.dtype)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            r = slice(i * BLOCK, (i + 1) * BLOCK) if tile else slice(i, i + 1)
            out[i, j] = x[r, j * BLOCK:(j + 1) * BLOCK].max()
    return out


def widen(scales, rows, cols, tile):
    """Each value's scale."""
    out = np.repeat(scales, BLOCK, 1)[:, :cols]
    return np.repeat(out, BLOCK, 0)[:rows] if tile else out


def quantize(x, tile=False):
    """Codes and scales of a matrix of fp32 values, in the definition's fp32 steps."""
    x = np.asarray(x, dtype=np.float32)
    scales = np.maximum(block_tops(x, tile) / np.float32(448), np.float32(2.0 ** -126))
    with np.errstate(invalid="ignore", over="ignore"):
        v = x * widen(np.float32(1) / scales, *x.shape, tile)
    return to_e4m3(v), scales


def sample(logits, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One sequence: the token, its probability, and the relative distance of the race's second from its winner."""
    l, noise = np.asarray(logits, dtype=np.float64), np.asarray(noise, dtype=np.float64)
    if np.isnan(l).any() or (l == np.inf).any() or not (l > -np.inf).any():
        return -1, 0.0, 1.0
    order = np.lexsort((np.arange(len(l)), -l))
    if temperature == 0:
        return int(order[0]), 1.0, 1.0
    if top_k > 0:
        order = order[:top_k]
    e = np.exp((l[order] - l[order[0]]) / temperature)
    if top_p < 1:
        upto = np.cumsum(e)
        kept = upto - e < top_p * upto[-1]
        kept[0] = True
        order, e = order[kept], e[kept]
    order, e = order[e >= min_p], e[e >= min_p]
    with np.errstate(divide="ignore", invalid="ignore"):
        score = np.where(e > 0, e / noise[order], 0.0)
    score = np.where(np.isnan(score), 0.0, score)
    if not score.max() > 0:
        return -1, 0.0, 1.0
    first = order[score == score.max()].min()
    second = max(score[score < score.max()], default=0.0)
    return int(first), float(e[order == first][0] / e.sum()), float(1.0 - second / score.max())
