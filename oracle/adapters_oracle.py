"""Plain numpy evaluation in 64 bits of dropout from a counter-based generator and of low-rank adapters of many requests beside a
shared projection, with their gradients.  Test infrastructure: written from the formulas, no code shared with the GPU path.

    drop(x)[i, j] = x[i, j] * 65536 / (65536 - q) where its 16 random bits are at least q = rint(65536 p), else 0
    T = drop(X) U_a^T       Y = base + s_a T V_a^T                            a = adapter of the token
    S = s_a E V_a           E_X = base + drop'(S U_a)      G_U[a] = sum S_t^T drop(X)_t      G_V[a] = s_a sum E_t^T T_t
"""
from __future__ import annotations

import numpy as np


def philox4x32_10(counter, key):
    """Philox4x32 with ten rounds on arrays of 32-bit words (Salmon et al., 2011).  counter: four, key: two; returns four."""
    word = 0xFFFFFFFF
    c = [np.asarray(x, dtype=object) if np.ndim(x) == 0 else np.asarray(x, dtype=np.uint64) for x in counter]
    c = [np.uint64(int(x)) if x.ndim == 0 else x for x in c]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(10):
        p0 = c[0] * np.uint64(0xD2511F53)
        p1 = c[2] * np.uint64(0xCD9E8D57)
        hi0, lo0, hi1, lo1 = p0 >> np.uint64(32), p0 & np.uint64(word), p1 >> np.uint64(32), p1 & np.uint64(word)
        c = [hi1 ^ c[1] ^ np.uint64(k0), lo1, hi0 ^ c[3] ^ np.uint64(k1), lo0]
        k0, k1 = (k0 + 0x9E3779B9) & word, (k1 + 0xBB67AE85) & word
    return c


def keep_mask(rows, cols, p, seed, offset):
    """Truth values [rows, cols]: which elements dropout keeps."""
    groups = -(-cols // 8)
    g, r = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(rows, dtype=np.uint64))
    const = lambda v: np.full((rows, groups), v & 0xFFFFFFFF, dtype=np.uint64)
    words = philox4x32_10([g, r, const(offset), const(offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    halves = [h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return np.stack(halves, axis=-1).reshape(rows, groups * 8)[:, :cols] >= np.uint64(threshold(p))


def threshold(p):
    return int(np.rint(65536.0 * p))


def drop(x, p, seed, offset):
    """drop(x) in 64 bits; an element that is dropped is 0 whatever it was."""
    x = np.asarray(x, dtype=np.float64)
    q = threshold(p)
    if q == 0:
        return x
    keep = keep_mask(x.shape[0], x.shape[1], p, seed, offset)
    return np.where(keep, x * (65536.0 / (65536 - q) if q < 65536 else 0.0), 0.0)


def _tokens(adapter_of, ranks, slots, max_rank):
    for a in range(slots):
        r = max_rank if ranks is None else min(max(int(ranks[a]), 0), max_rank)
        t = np.flatnonzero(np.asarray(adapter_of) == a)
        if len(t) and r:
            yield a, r, t


def forward(X, U, V, adapter_of, ranks=None, scale=None, base=None, p=0.0, seed=0, offset=0):
    """(Y, T); U [slots, max_rank, m], V [slots, n, max_rank]."""
    slots, max_rank, _ = U.shape
    b, n = len(adapter_of), V.shape[1]
    Y = np.zeros((b, n)) if base is None else np.array(base, dtype=np.float64)
    T = np.zeros((b, max_rank))
    x = drop(X, p, seed, offset)
    for a, r, t in _tokens(adapter_of, ranks, slots, max_rank):
        T[t, :r] = x[t] @ U[a, :r].astype(np.float64).T
        Y[t] += (1.0 if scale is None else float(scale[a])) * (T[t, :r] @ V[a, :, :r].astype(np.float64).T)
    return Y, T


def backward(E, X, T, U, V, adapter_of, ranks=None, scale=None, base=None, p=0.0, seed=0, offset=0):
    """(E_X, G_U, G_V, S)."""
    slots, max_rank, m = U.shape
    b, n = len(adapter_of), V.shape[1]
    S = np.zeros((b, max_rank))
    low = np.zeros((b, m))
    GU, GV = np.zeros((slots, max_rank, m)), np.zeros((slots, n, max_rank))
    x = drop(X, p, seed, offset)
    E, T = np.asarray(E, dtype=np.float64), np.asarray(T, dtype=np.float64)
    for a, r, t in _tokens(adapter_of, ranks, slots, max_rank):
        s = 1.0 if scale is None else float(scale[a])
        S[t, :r] = s * (E[t] @ V[a, :, :r].astype(np.float64))
        low[t] = S[t, :r] @ U[a, :r].astype(np.float64)
        GU[a, :r] = S[t, :r].T @ x[t]
        GV[a, :, :r] = s * (E[t].T @ T[t, :r])
    EX = drop(low, p, seed, offset)
    return (EX if base is None else EX + np.asarray(base, dtype=np.float64)), GU, GV, S
