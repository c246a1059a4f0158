"""CPU oracle of the scored attention, the drafted-token attention and the cache's
keep (float64 NumPy). TEST INFRASTRUCTURE ONLY; shares no code with the library.

For query row i and value row j, with z = scale <q~_i, v_j> (Eq. 4):
    x_ij = cap tanh(z / cap) - slope_h |pos_i - pos_j|      (cap 0: z itself)
and row i sees the rows that its mask lets it. Every function works head by head
(query head h reads value group h // (H // G)) from the definition.
"""

from __future__ import annotations

import numpy as np

from .keyless import _f64, cache_rows, default_scale


def row_ranges(B: int, N: int, first=None, last=None, causal: bool = True):
    """What each row sees: boolean [B, N, N], row i the columns first_i <= j < last_i."""
    i = np.arange(N)
    lo = np.zeros((B, N), int) if first is None else np.asarray(first).astype(int)
    if last is None:
        hi = np.broadcast_to(i + 1 if causal else np.full(N, N), (B, N))
    else:
        hi = np.asarray(last).astype(int)
    return (i >= lo[:, :, None]) & (i < hi[:, :, None])


def scores(q, V, scale: float, cap: float, slope: float, distance):
    """(x, d x / d z) of the rows q [n, d] against V [L, d]."""
    z = scale * (_f64(q) @ _f64(V).T)
    bend = np.ones_like(z)
    if cap > 0:
        t = np.tanh(z / cap)
        z, bend = cap * t, 1.0 - t * t
    return z - slope * distance, bend


def masked_softmax(x, seen):
    """(P, log-sum-exp) over the seen columns; a row that sees none: zeros, -inf."""
    x = np.where(seen, x, -np.inf)
    m = np.max(x, axis=1, keepdims=True, initial=-np.inf)
    e = np.exp(x - np.where(np.isinf(m), 0.0, m))
    total = np.sum(e, axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + m)[:, 0]
    return e / np.where(total > 0, total, 1.0), lse


def scored_attention(Qr, V, cap: float = 0.0, slopes=None, seen=None, scale: float | None = None):
    """Qr [B, N, H, d], V [B, N, G, d], seen [B, N, N]; returns (out, lse [B, H, N])."""
    Qr, V = _f64(Qr), _f64(V)
    B, N, H, d = Qr.shape
    rep = H // V.shape[2]
    tau = default_scale(d) if scale is None else float(scale)
    dist = np.abs(np.arange(N)[:, None] - np.arange(N)[None])
    out, lse = np.zeros(Qr.shape), np.zeros((B, H, N))
    for b in range(B):
        for h in range(H):
            x, _ = scores(Qr[b, :, h], V[b, :, h // rep], tau, cap, 0.0 if slopes is None else slopes[h], dist)
            P, lse[b, h] = masked_softmax(x, seen[b])
            out[b, :, h] = P @ V[b, :, h // rep]
    return out, lse


def scored_attention_backward(Qr, V, dO, cap: float = 0.0, slopes=None, seen=None,
                              scale: float | None = None):
    """(dQ~, dV) of scored_attention given dL/dO: the softmax backward
    dx = P * (dP - rowsum(P * dP)) with dP = dO V^T, through the cap
    dz = dx (1 - tanh^2), then dQ~ = tau dz V and dV = P^T dO + tau dz^T Q~ (both
    roles of the values, Section 2.3, Eq. 6), summed over a group's heads."""
    Qr, V, dO = _f64(Qr), _f64(V), _f64(dO)
    B, N, H, d = Qr.shape
    rep = H // V.shape[2]
    tau = default_scale(d) if scale is None else float(scale)
    dist = np.abs(np.arange(N)[:, None] - np.arange(N)[None])
    dQ, dV = np.zeros(Qr.shape), np.zeros(V.shape)
    for b in range(B):
        for h in range(H):
            q, v, g = Qr[b, :, h], V[b, :, h // rep], dO[b, :, h]
            x, bend = scores(q, v, tau, cap, 0.0 if slopes is None else slopes[h], dist)
            P, _ = masked_softmax(x, seen[b])
            dP = g @ v.T
            dz = P * (dP - np.sum(P * dP, axis=1, keepdims=True)) * bend
            dQ[b, :, h] = tau * (dz @ v)
            dV[b, :, h // rep] += P.T @ g + tau * (dz.T @ q)
    return dQ, dV


def tree_words(parents):
    """Words of a tree from its parents [B, T] (-1 for a root): a token sees its
    ancestors and itself. Returns uint64 [B, T]."""
    parents = np.asarray(parents)
    words = np.zeros(parents.shape, np.uint64)
    for b in range(parents.shape[0]):
        for t in range(parents.shape[1]):
            above = words[b, parents[b, t]] if parents[b, t] >= 0 else np.uint64(0)
            words[b, t] = above | (np.uint64(1) << np.uint64(t))
    return words


def tree_decode(q, cache, lengths_before, tree, H: int, G: int, cap: float = 0.0, slopes=None,
                block_table=None, block_size: int = 16, scale: float | None = None,
                capacity: int | None = None):
    """Drafted tokens q [B, T, H, d] over rows 0 .. n - 1 and the drafted rows u (cache
    row n + u) whose bit the token's word has (None: a chain). A token's depth is the
    number of bits beside its own; positions are n + depth."""
    q = _f64(q)
    B, T, _, d = q.shape
    tau = default_scale(d) if scale is None else float(scale)
    out = np.zeros(q.shape)
    for b in range(B):
        n = int(lengths_before[b])
        words = [(2 << t) - 1 if tree is None else int(tree[b][t]) & ((1 << T) - 1) for t in range(T)]
        sees = np.array([[bool(w >> u & 1) for u in range(T)] for w in words])
        depth = np.array([int(sees[t].sum()) - int(sees[t, t]) for t in range(T)])
        rows = n + T if capacity is None else min(n + T, capacity)
        pos = np.concatenate([np.arange(n), n + depth])[:rows]
        seen = np.concatenate([np.ones((T, n), bool), sees], axis=1)[:, :rows]
        dist = np.abs((n + depth)[:, None] - pos[None])
        for g in range(G):
            V = cache_rows(cache, b, g, rows, block_table, block_size)
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x, _ = scores(q[b, :, h], V, tau, cap, 0.0 if slopes is None else slopes[h], dist)
                out[b, :, h] = masked_softmax(x, seen)[0] @ V
    return out


def value_cache_keep(cache, lengths_before, path, kept, block_table=None, block_size: int = 16):
    """A copy of the cache with row n + k set to what row n + path[b, k] was, k < kept[b]."""
    old = np.asarray(cache)
    new = np.array(old, copy=True)
    for b in range(len(lengths_before)):
        n = int(lengths_before[b])
        for k in range(int(kept[b])):
            to, at = n + k, n + int(path[b][k])
            if block_table is None:
                new[b, :, to] = old[b, :, at]
            else:
                t = block_table[b]
                new[int(t[to // block_size]), :, to % block_size] = \
                    old[int(t[at // block_size]), :, at % block_size]
    return new
