"""Plain float64 forms of the language-model operators, from their definitions."""

from __future__ import annotations

import numpy as np


def linear_attention(q, k, v, decay, scale, lengths=None, state=None):
    """Token by token: S = a S + k v^T, o = scale S^T q.  [B, T, H, d] float64."""
    B, T, H, d = q.shape
    a = decay.reshape(1, H, 1, 1)
    S = np.zeros((B, H, d, d)) if state is None else state.copy()
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    o = np.zeros((B, T, H, d))
    for t in range(T):
        on = t < n
        new = a * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        S = np.where(on[:, None, None, None], new, S)
        o[:, t] = np.where(on[:, None, None], scale * np.einsum("bhij,bhi->bhj", S, q[:, t]), 0.0)
    return o, S


def linear_attention_grads(do, q, k, v, decay, scale, lengths=None, state=None, dstate=None):
    """dq, dk, dv, d(first state) by reverse accumulation through the same steps."""
    B, T, H, d = q.shape
    a = decay.reshape(1, H, 1, 1)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    S = np.zeros((B, H, d, d)) if state is None else state.copy()
    states = []
    for t in range(T):
        on = (t < n)[:, None, None, None]
        S = np.where(on, a * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        states.append(S)
    G = np.zeros((B, H, d, d)) if dstate is None else dstate.copy()   # dL/dS_t
    dq, dk, dv = (np.zeros((B, T, H, d)) for _ in range(3))
    for t in range(T - 1, -1, -1):
        on = t < n
        o3, o4 = on[:, None, None], on[:, None, None, None]
        g = scale * do[:, t]
        dq[:, t] = np.where(o3, np.einsum("bhij,bhj->bhi", states[t], g), 0.0)
        G1 = np.where(o4, G + q[:, t, :, :, None] * g[:, :, None, :], G)
        dk[:, t] = np.where(o3, np.einsum("bhij,bhj->bhi", G1, v[:, t]), 0.0)
        dv[:, t] = np.where(o3, np.einsum("bhij,bhi->bhj", G1, k[:, t]), 0.0)
        G = np.where(o4, a * G1, G)
    return dq, dk, dv, G


def embedding_grad(ids, dy, V, scale):
    """(gradient, sum of magnitudes, counts) per table row; ids outside [0, V) count nowhere."""
    dw = np.zeros((V, dy.shape[1]))
    mag = np.zeros_like(dw)
    ok = (ids >= 0) & (ids < V)
    np.add.at(dw, ids[ok], scale * dy[ok])
    np.add.at(mag, ids[ok], np.abs(scale * dy[ok]))
    return dw, mag, np.bincount(ids[ok], minlength=V)


def philox4x32(counter, key, rounds=10):
    """Philox4x32: counter [n, 4], key (k0, k1) as Python or numpy integers -> [n, 4] words."""
    M = np.uint64(0xFFFFFFFF)
    c = [np.asarray(counter[:, i], dtype=np.uint64) for i in range(4)]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & M,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & M]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, axis=1)


def dropout_keep(n, p, seed, offset):
    """Which of n elements dropout keeps: draw i % 8 of counter (i / 8, offset)."""
    j = np.arange((n + 7) // 8, dtype=np.uint64)
    M = np.uint64(0xFFFFFFFF)
    ctr = np.stack([j & M, j >> np.uint64(32), np.full_like(j, offset & 0xFFFFFFFF),
                    np.full_like(j, offset >> 32)], axis=1)
    w = philox4x32(ctr, (seed & 0xFFFFFFFF, seed >> 32))
    draws = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=2).reshape(len(j), 8)
    return (draws >= np.uint64(round(p * 65536))).reshape(-1)[:n]
