"""Output-head oracle: 4-bit weights, sampling and distillation in binary64 numpy, entry by entry from the definitions.

Shares no code with the GPU library.  Stored values (codes, scales, binary32 parameters) are taken as given; every
sum and function value is binary64."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1_nearest(a):
    """Codes 0..7 nearest to magnitudes a >= 0, ties to the even code, above 6 the code of 6."""
    a = np.minimum(np.asarray(a, np.float64), 6.0)
    d = np.abs(a[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    pick = np.where(even.any(-1, keepdims=True), even, near)
    return pick.argmax(-1)


def quantize(W, group, scale_cast, quotient):
    """(codes m x n in 0..15, scales m x G) of W in its own values; scale_cast rounds a binary32 value to the scale's
    type (returned as binary64), quotient is np.float32 or np.float64: the type that max * (1/6) and w / scale round to."""
    W = np.asarray(W)
    m, n = W.shape
    G = -(-n // group)
    codes = np.zeros((m, n), np.int64)
    scales = np.zeros((m, G))
    for g in range(G):
        w = W[:, g * group:(g + 1) * group].astype(quotient)
        amax = np.abs(w).max(1)
        with np.errstate(all="ignore"):
            s = scale_cast((amax * (quotient(1) / quotient(6))).astype(np.float32))
        bad = ~np.isfinite(w).all(1) | ~np.isfinite(s)
        s = np.where(bad, np.nan, s)
        scales[:, g] = s
        with np.errstate(all="ignore"):
            a = np.where((s > 0)[:, None], np.abs(w) / s[:, None].astype(quotient), 0).astype(quotient)
        c = e2m1_nearest(np.where(np.isfinite(a), a, 0)) + 8 * (np.signbit(w) & ~bad[:, None])
        codes[:, g * group:(g + 1) * group] = c
    return codes, scales


def pack(codes):
    """Packed rows (uint8, 16 ceil(n / 32) bytes) of codes m x n."""
    m, n = codes.shape
    full = np.zeros((m, -(-n // 32) * 32), np.uint8)
    full[:, :n] = codes
    return full[:, 0::2] | (full[:, 1::2] << 4)


def weights(codes, scales, group):
    """The m x n binary64 weights of codes 0..15."""
    n = codes.shape[1]
    v = np.where(codes >= 8, -1.0, 1.0) * E2M1[codes % 8]
    return v * np.repeat(np.asarray(scales, np.float64), group, axis=1)[:, :n]


def q4_apply(W, X, U=None, s=None, V=None):
    Y = X @ W.T
    if U is not None:
        Y = Y + ((X @ V) * s) @ U.T
    return Y


def sample_kept(l, T=1.0, k=0, p=1.0, mp=0.0):
    """(order of the tokens by logit, kept weights in vocabulary order) of one row of binary64 logits."""
    l = np.where(np.isnan(l), -np.inf, l)
    M = l.max()
    with np.errstate(invalid="ignore"):
        z = np.where(l == M, 0.0, (l - M) / T)
    w = np.floor(np.exp(z) * 2.0 ** 31)
    order = np.lexsort((np.arange(len(l)), -l))
    keep = np.ones(len(l), bool)
    if 0 < k < len(l):
        keep[k:] = False
    ws = w[order]
    if p < 1.0:
        before = np.cumsum(ws) - ws
        keep &= before < max(p * ws[keep].sum(), 1.0)
    if mp > 0.0:
        keep &= np.exp(z)[order] >= min(mp, 1.0)
    kept = np.zeros(len(l))
    kept[order[keep]] = ws[keep]
    return order, kept


def distill(z, ids, top, T=1.0, lse=None, weight=None):
    """(loss, gradient of the sum of the losses) of binary64 logits z."""
    N, V = z.shape
    loss, grad = np.zeros(N), np.zeros((N, V))
    for i in range(N):
        w = 1.0 if weight is None else weight[i]
        if w == 0.0:
            continue
        ok = (ids[i] >= 0) & (ids[i] < V)
        named, t = ids[i][ok], top[i][ok] / T
        if lse is None and (len(t) == 0 or t.max() == -np.inf):
            continue
        with np.errstate(all="ignore"):
            x = z[i] / T
            logq = x - x.max() - np.log(np.exp(x - x.max()).sum())
            logp = t - (lse[i] if lse is not None else t.max() + np.log(np.exp(t - t.max()).sum()))
            p = np.exp(logp)
            kl = np.where(p == 0, 0.0, p * (logp - logq[named])).sum()
            q = np.exp(logq)
            g = q.copy()
            if lse is not None:
                other = np.ones(V, bool)
                other[named] = False
                r, Q = max(1.0 - p.sum(), 0.0), q[other].sum()
                g *= p.sum() + r                          # the teacher's whole mass: above 1 where the named ones are
                if r > 0:
                    kl += r * (np.log(r) - np.log(Q))
                    g[other] -= r * q[other] / Q
                g[other & (q == 0)] = 0.0
        np.add.at(g, named, -p)
        loss[i] = w * T * T * kl
        grad[i] = w * T * g
    return loss, grad
