"""What surrounds a model's layers, in 64 bits -- TEST INFRASTRUCTURE ONLY.

Plain numpy from the definitions, element after element where that is short: the embedding and its
gradient, the causal convolution and its gradient, the norm of a list of tensors and the clipping by
it, and the verification of drafted tokens from given random numbers.  No code is shared with the
library.  Only ``tests/`` may import this module.
"""
from __future__ import annotations

import numpy as np


def embedding(tokens, weight, scale=1.0):
    tokens, weight = np.asarray(tokens, dtype=np.int64), np.asarray(weight, dtype=np.float64)
    out = np.full(tokens.shape + (weight.shape[1],), np.nan)
    for at in np.ndindex(*tokens.shape):
        t = tokens[at]
        if t < 0:
            out[at] = 0.0
        elif t < weight.shape[0]:
            out[at] = scale * weight[t]
    return out


def embedding_grad(tokens, dy, vocab, scale=1.0):
    tokens, dy = np.asarray(tokens, dtype=np.int64).ravel(), np.asarray(dy, dtype=np.float64)
    dy = dy.reshape(tokens.size, dy.shape[-1])
    out = np.zeros((vocab, dy.shape[1]))
    for t, row in zip(tokens, dy):
        if 0 <= t < vocab:
            out[t] += scale * row
    return out


def conv(x, w, bias=None, state=None, silu=True):
    """(batch, dim, L) -> y and the last k - 1 inputs."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    B, D, L = x.shape
    H = w.shape[1] - 1
    ext = np.concatenate([np.zeros((B, D, H)) if state is None else np.asarray(state, dtype=np.float64), x], 2)
    pre = np.zeros((B, D, L))
    for t in range(L):
        pre[:, :, t] = (ext[:, :, t:t + H + 1] * w).sum(2) + (0.0 if bias is None else np.asarray(bias, np.float64))
    return (pre / (1.0 + np.exp(-pre)) if silu else pre), ext[:, :, L:]


def conv_grad(x, w, dy, bias=None, state=None, dstate_out=None, silu=True):
    """dx, dw, dbias, dstate: every product of the forward, and what flows back through it."""
    x, w, dy = (np.asarray(a, dtype=np.float64) for a in (x, w, dy))
    B, D, L = x.shape
    K = w.shape[1]
    H = K - 1
    ext = np.concatenate([np.zeros((B, D, H)) if state is None else np.asarray(state, dtype=np.float64), x], 2)
    dext, dw, dbias = np.zeros_like(ext), np.zeros((D, K)), np.zeros(D)
    if dstate_out is not None:
        dext[:, :, L:] += np.asarray(dstate_out, dtype=np.float64)
    for t in range(L):
        pre = (ext[:, :, t:t + K] * w).sum(2) + (0.0 if bias is None else np.asarray(bias, np.float64))
        s = 1.0 / (1.0 + np.exp(-pre))
        g = dy[:, :, t] * ((s + pre * s * (1.0 - s)) if silu else 1.0)
        dext[:, :, t:t + K] += g[:, :, None] * w
        dw += (g[:, :, None] * ext[:, :, t:t + K]).sum(0)
        dbias += g.sum(0)
    return {"dx": dext[:, :, H:], "dw": dw, "dbias": dbias, "dstate": dext[:, :, :H]}


def norm(tensors):
    return float(np.sqrt(sum(float((np.asarray(t, dtype=np.float64) ** 2).sum()) for t in tensors)))


def clip(tensors, max_norm, eps=1e-6):
    n = norm(tensors)
    f = 1.0 if n + eps <= max_norm else max_norm / (n + eps)
    return n, [np.asarray(t, dtype=np.float64) * f for t in tensors]


def softmax(logits, temperature=1.0):
    """A row's probabilities, or None where it is no distribution."""
    lg = np.asarray(logits, dtype=np.float64)
    if np.isnan(lg).any() or (lg == np.inf).any() or not (lg > -np.inf).any():
        return None
    e = np.exp((lg - lg.max()) / temperature)
    return e / e.sum()


def verify_sample(logits, draft, uniform, noise, draft_logits=None, lengths=None, temperature=1.0):
    """accepted, next_token (batch,), probs (batch, ndraft), and `margin` (batch,): how far, relatively, the nearest
    decision on the way was from falling otherwise."""
    B, n = np.asarray(draft).shape
    V = logits.shape[2]
    acc, nxt = np.zeros(B, np.int64), np.zeros(B, np.int64)
    probs, margin = np.zeros((B, n)), np.full(B, np.inf)
    for b in range(B):
        length = n if lengths is None else min(max(int(lengths[b]), 0), n)
        c = None
        q_c = None
        for i in range(length):
            p, x = softmax(logits[b, i], temperature), int(draft[b, i])
            if draft_logits is None:
                q = np.zeros(V)
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                q = softmax(draft_logits[b, i], temperature)
            there = 0 <= x < V and p is not None
            probs[b, i] = p[x] if there else 0.0
            if c is None:
                passes = False
                if there and q is not None:
                    lhs = float(uniform[b, i]) * q[x]
                    passes = lhs < p[x]
                    if max(lhs, p[x]) > 0:
                        margin[b] = min(margin[b], abs(lhs - p[x]) / max(lhs, p[x]))
                if not passes:
                    c, q_c = i, q
        if c is None:
            c, q_c = length, None
        acc[b] = c
        p = softmax(logits[b, c], temperature)
        if p is None:
            nxt[b] = -1
            continue
        r = p if q_c is None else np.maximum(p - q_c, 0.0)
        if not (r > 0).any():
            r = p
        score = r / np.asarray(noise[b], dtype=np.float64)
        nxt[b] = int(np.argmax(score))
        two = np.sort(score)[-2:]
        if V > 1:
            margin[b] = min(margin[b], (two[1] - two[0]) / two[1])
    return acc, nxt, probs, margin
