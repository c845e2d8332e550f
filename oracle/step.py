"""Oracle of the operators around the compressed projections in binary64 numpy: norm, adapters and their gradients, e4m3,
and the verification of drafted tokens.  Shares no code with the GPU library."""
from __future__ import annotations

import numpy as np

# the 127 magnitudes of e4m3 (sign, 4 exponent bits of bias 7, 3 of significand; 0x7F is NaN)
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def e4m3_nearest(a):
    """Values of e4m3 nearest to the numbers a, ties to the even code, magnitudes above 448 become 448."""
    a = np.asarray(a, np.float64)
    m = np.minimum(np.abs(a), 448.0)
    hi = np.clip(np.searchsorted(E4M3, m), 1, 126)
    lo = hi - 1
    down, up = m - E4M3[lo], E4M3[hi] - m
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.copysign(E4M3[pick], a)


def rms_norm(h, w=None, eps=1e-6):
    """(y, rstd) of binary64 rows h."""
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    y = h * rstd[:, None]
    return (y if w is None else y * w), rstd


def rms_norm_backward(dy, h, w=None, eps=1e-6, dsum=None):
    """(dx, dw) of y = rms_norm(h, w): dx also of dsum, which reaches h by other ways."""
    rstd = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    g = dy if w is None else dy * w
    dx = rstd * g - h * rstd ** 3 * (g * h).mean(1, keepdims=True)
    if dsum is not None:
        dx = dx + dsum
    return dx, (dy * h * rstd).sum(0)


def adapters(X, A, B, ids, scale=None, base=None):
    """(Y, hidden)"""
    Y = np.zeros((X.shape[0], B.shape[1])) if base is None else np.array(base, np.float64)
    hidden = np.zeros((X.shape[0], A.shape[1]))
    for i, a in enumerate(ids):
        if 0 <= a < len(A):
            hidden[i] = A[a] @ X[i]
            Y[i] += (1.0 if scale is None else scale[a]) * (B[a] @ hidden[i])
    return Y, hidden


def adapters_backward(dY, X, A, B, ids, scale=None, base=None):
    """(dX, dA, dB)"""
    dX = np.zeros(X.shape) if base is None else np.array(base, np.float64)
    dA, dB = np.zeros(A.shape), np.zeros(B.shape)
    for i, a in enumerate(ids):
        if 0 <= a < len(A):
            c = 1.0 if scale is None else scale[a]
            dh = c * (dY[i] @ B[a])
            dX[i] += dh @ A[a]
            dA[a] += np.outer(dh, X[i])
            dB[a] += c * np.outer(dY[i], A[a] @ X[i])
    return dX, dA, dB


def verify(P, drafts, u, Q=None):
    """(tokens, accepted) of one request from whole-number weights: P (D + 1) x V of the target, Q D x V of the draft model
    or None (certain drafts), u D + 1 numbers.  Every comparison is made in exact integers, u as the binary64 value
    that it is; the units of the residual are those of 2^52 over the sum, rounded down."""
    D, V = len(drafts), P.shape[1]
    P = [[int(x) for x in row] for row in P]
    Q = None if Q is None else [[int(x) for x in row] for row in Q]
    out = [-1] * (D + 1)

    def draw(weights, x):
        S = sum(weights)
        if S == 0:
            return -1
        num, den = (float(x) if x > 0 else 0.0).as_integer_ratio()
        t = min(num * S // den, S - 1)
        run = 0
        for i, w in enumerate(weights):
            run += w
            if run > t:
                return i

    for j in range(D + 1):
        if j == D or not 0 <= drafts[j] < V:
            out[j] = draw(P[j], u[D])
            return out, j
        t = int(drafts[j])
        q = [int(i == t) for i in range(V)] if Q is None else Q[j]
        Sp, Sq = sum(P[j]), sum(q)
        num, den = float(min(max(u[j], 0.0), 1.0 - 2.0 ** -24)).as_integer_ratio()
        if num * q[t] * Sp < den * P[j][t] * Sq:
            out[j] = t
            continue
        rest = [max((a << 52) // max(Sp, 1) - ((b << 52) // Sq if Sq else 0), 0) for a, b in zip(P[j], q)]
        out[j] = draw(rest if sum(rest) else P[j], u[D])
        return out, j
