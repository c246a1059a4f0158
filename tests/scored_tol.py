"""How far the scored kernels may be from the 64-bit oracle, element by element, from
the roundings they make. Written down before the kernels were first run.

u is half a step of the result's type (2^-8 relative for bf16, 2^-24 for fp32), e =
2^-24 half a step of fp32, in which every sum is held. For head rows i, j:
  S_ij = scale sum_c |q_ic v_jc| bounds the products of a score; their sum in any order
    is off by (2 D + 8) e S. The tanh (an exponential and a reciprocal of 2^-22 each)
    is off by 2^-21, the score by cap times that; the bias, the shift by the row's
    maximum and the change to base 2 round terms of the size of the score a few times.
    d_ij = e ((2 D + 8) S + 8 (|x| + |bias| + |lse|)) + 2^-21 cap.
  A weight is then off by a factor within h_i = 2 max_j d_ij + 2^-20 (its own error, the
    normaliser's, and the exponential's), plus u for bf16, whose weights are rounded for
    the products. A sum of L terms adds L e of its absolute sum.
  out:  u |out| + (u_p + h + L e) sum_j p |v|
  lse:  max_j d + L e + 2^-20 + 2 e |lse|
  Dd = sum_j p dP: (u_p + h + (L + 2 D) e) sum_j p C, C_ij = sum_c |dO_ic v_jc|
  dz = p bend (dP - Dd): p (|bend| (err Dd + 2 D e C) + (h |bend| + 2^-19) |dP - Dd|) + u_p |dz|
  dq:   u |dq| + scale sum_j |v_j| (err dz + L e |dz|)
  dv:   u |dv| + sum over heads and i of (u_p + h + L' e) p |dO| + scale |q| (err dz + L' e |dz|)
"""

import numpy as np

from oracle import scored as S
from oracle.keyless import default_scale

E = 2.0 ** -24


def bounds(q, v, dO, cap, slopes, seen, bf16: bool, scale=None):
    """dict(out, lse, dq, dv) of absolute bounds; dq and dv only with dO."""
    B, N, H, d = q.shape
    G, rep = v.shape[2], H // v.shape[2]
    tau = default_scale(d) if scale is None else scale
    u, up = (2.0 ** -8, 2.0 ** -8) if bf16 else (E, 0.0)
    dist = np.abs(np.arange(N)[:, None] - np.arange(N)[None])
    got = dict(out=np.zeros(q.shape), lse=np.zeros((B, H, N)))
    if dO is not None:
        got.update(dq=np.zeros(q.shape), dv=np.zeros(v.shape))
        exact_dv = S.scored_attention_backward(q, v, dO, cap, slopes, seen, scale)[1]
        got["dv"] += u * np.abs(exact_dv)
    for b in range(B):
        for h in range(H):
            Q, V = q[b, :, h], v[b, :, h // rep]
            slope = 0.0 if slopes is None else slopes[h]
            x, bend = S.scores(Q, V, tau, cap, slope, dist)
            P, lse = S.masked_softmax(x, seen[b])
            lse = np.where(np.isinf(lse), 0.0, lse)
            sizes = tau * (np.abs(Q) @ np.abs(V).T)
            dl = E * ((2 * d + 8) * sizes + 8 * (np.abs(x) + np.abs(slope) * dist + np.abs(lse)[:, None])) \
                + 2.0 ** -21 * cap
            dl = np.max(np.where(seen[b], dl, 0.0), axis=1, initial=0.0)
            L = N
            hh = (2 * dl + 2.0 ** -20)[:, None]
            out = P @ V
            got["out"][b, :, h] = u * np.abs(out) + (up + hh + L * E) * (P @ np.abs(V))
            got["lse"][b, h] = dl + L * E + 2.0 ** -20 + 2 * E * np.abs(lse)
            if dO is None:
                continue
            g = dO[b, :, h]
            dP, C = g @ V.T, np.abs(g) @ np.abs(V).T
            Dd = np.sum(P * dP, axis=1, keepdims=True)
            eD = (up + hh + (L + 2 * d) * E) * np.sum(P * C, axis=1, keepdims=True)
            dz = P * bend * (dP - Dd)
            ez = P * (np.abs(bend) * (eD + 2 * d * E * C)
                      + (hh * np.abs(bend) + 2.0 ** -19) * np.abs(dP - Dd)) + up * np.abs(dz)
            dq = tau * (dz @ V)
            got["dq"][b, :, h] = u * np.abs(dq) + tau * ((ez + L * E * np.abs(dz)) @ np.abs(V))
            LL = N * rep
            got["dv"][b, :, h // rep] += ((up + hh + LL * E) * P).T @ np.abs(g) \
                + tau * ((ez + LL * E * np.abs(dz)).T @ np.abs(Q))
    return got


def check(what, got, ref, bound):
    """Every element within its bound; equal where the reference is not finite."""
    got = np.asarray(got, np.float64)
    fin = np.isfinite(ref)
    assert np.array_equal(got[~fin], ref[~fin]), f"{what}: not the reference's infinities"
    over = np.abs(got[fin] - ref[fin]) - (bound[fin] + 1e-30)
    worst = float(over.max()) if over.size else 0.0
    assert np.isfinite(got[fin]).all() and worst <= 0, \
        f"{what}: {int((over > 0).sum())} of {over.size} past their bound, worst by {worst:.3e}"
