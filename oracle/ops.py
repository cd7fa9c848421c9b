"""The operators of a residual block in float64 numpy: decayed attention token by
token, Philox dropout on Python-sized integers, the norm behind the residual.

Written from the definitions (include/ambptt_ops.h states them); shares no code
with the library.
"""
from __future__ import annotations

import numpy as np


def attention(q, k, v, log_decay, s0=None, lengths=None, scale=1.0):
    """q [B, T, H G, a], k [B, T, H, a], v [B, T, H, e] -> (o [B, T, H G, e], sn [B, H, a, e])."""
    B, T, HG, a = q.shape
    H, e = k.shape[2], v.shape[3]
    G = HG // H
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((B, H, a, e)) if s0 is None else np.array(s0, np.float64)
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    o = np.zeros((B, T, HG, e))
    for b in range(B):
        for t in range(n[b]):
            S[b] = lam * S[b] + k[b, t][:, :, None] * v[b, t][:, None, :]
            o[b, t] = scale * np.einsum("hga,hae->hge", q[b, t].reshape(H, G, a), S[b]).reshape(HG, e)
    return o, S


def attention_backward(q, k, v, log_decay, do, s0=None, dsn=None, lengths=None, scale=1.0):
    """-> (dq, dk, dv, ds0)."""
    B, T, HG, a = q.shape
    H, e = k.shape[2], v.shape[3]
    G = HG // H
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    n = np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)
    D = np.zeros((B, H, a, e)) if dsn is None else np.array(dsn, np.float64)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        S = np.zeros((H, a, e)) if s0 is None else np.array(s0[b], np.float64)
        for t in range(n[b]):
            S = lam * S + k[b, t][:, :, None] * v[b, t][:, None, :]
            dq[b, t] = scale * np.einsum("hge,hae->hga", do[b, t].reshape(H, G, e), S).reshape(HG, a)
        for t in reversed(range(n[b])):
            A = D[b] + scale * np.einsum("hga,hge->hae", q[b, t].reshape(H, G, a), do[b, t].reshape(H, G, e))
            dk[b, t] = np.einsum("hae,he->ha", A, v[b, t])
            dv[b, t] = np.einsum("hae,ha->he", A, k[b, t])
            D[b] = lam * A
    return dq, dk, dv, D


def philox(counter, key):
    """Philox-4x32-10 of one 128-bit counter (four 32-bit words) under two key words."""
    x, k, m = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & m, (a >> 32) ^ x[3] ^ k[1], a & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return x


def dropout_factors(rows, cols, p, seed, offset):
    """What each element is multiplied by, float64 [rows, cols] (zero: dropped)."""
    t = int(np.rint(65536 * p))
    up = 65536 / (65536 - t) if t < 65536 else 0.0
    wide = -(-cols // 8)
    f = np.zeros((rows, wide * 8))
    for r in range(rows):
        for c in range(wide):
            n = (offset + r * wide + c) % (1 << 64)
            w = philox((n & 0xFFFFFFFF, n >> 32, 0, 0), (seed & 0xFFFFFFFF, seed >> 32))
            for j in range(8):
                f[r, 8 * c + j] = up if (w[j // 2] >> (16 * (j % 2))) & 0xFFFF >= t else 0.0
    return f[:, :cols]


def dropped(x, f):
    """x times the factors; zero where dropped, whatever x holds."""
    return np.where(f > 0, x * np.where(f > 0, f, 1.0), 0.0)


def norm(h, w, eps):
    return w * h / np.sqrt((h * h).mean(-1, keepdims=True) + eps)


def norm_backward(dy, h, w, dh, eps):
    """-> (dr, dw)."""
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    a = w * dy
    return dh + r * (a - h * r * r * (a * h).mean(-1, keepdims=True)), (dy * h * r).sum(0)
