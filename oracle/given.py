"""What sbw_sample_given gives, from its definition: numpy and Python's whole numbers, one row at a time."""
from __future__ import annotations

import math

import numpy as np

# (ln 2)^k / k!, highest power first, rounded to fp32
_EXP2 = [np.float32(math.log(2.0) ** k / math.factorial(k)) for k in range(7, -1, -1)]


def weights(x: np.ndarray, m: np.float32, c: np.float32) -> np.ndarray:
    """The integer weights (int64) of fp32 values x under the maximum m, with c = log2(e) / temperature."""
    x = np.asarray(x, np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        y = np.where(x == m, np.float32(0), (x - m) * np.float32(c)).astype(np.float32)
    real = y >= -41.0
    y = np.where(real, y, np.float32(0))
    n = np.rint(y)
    f = (y - n).astype(np.float64)
    p = np.zeros_like(y)
    for a in _EXP2:                                # fused: the product of two fp32 numbers is exact in fp64
        p = (p.astype(np.float64) * f + np.float64(a)).astype(np.float32)
    w = np.floor(np.ldexp(p.astype(np.float64), (n + 40).astype(np.int32))).astype(np.int64)
    return np.where(real, w, 0)


def sample_row(x: np.ndarray, u: float, tau: float, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0):
    """(token, its weight, the kept weights' sum, number kept) of one row of biased logits, widened to fp32."""
    x = np.where(np.isnan(x), np.float32(-np.inf), np.asarray(x, np.float32)) + np.float32(0)
    m = x.max()
    if m == -np.inf:
        return 0, 0, 0, 0
    if m == np.inf:
        x = np.where(x == np.inf, np.float32(0), np.float32(-np.inf))
        m = np.float32(0)
    tau, top_p, min_p = (float(np.float32(v)) for v in (tau, top_p, min_p))
    greedy = not np.float32(tau) >= np.float32(1e-6)
    c = np.float32(1.0 if greedy else 1.4426950408889634 / tau)
    w = weights(x, m, c)
    if greedy:
        top_k, top_p, min_p = 1, 1.0, 0.0
    if min_p > 0:
        with np.errstate(over="ignore", invalid="ignore"):
            y = np.where(x == m, np.float32(0), (x - m) * c)
        w = np.where(y >= np.float32(min(0.0, math.log2(min_p))), w, 0)
    cols = np.flatnonzero(w)
    cols = cols[np.argsort(-x[cols], kind="stable")]
    if top_k > 0:
        cols = cols[:top_k]
    run = [int(v) for v in np.cumsum(w[cols])]     # below 2^58: exact
    if top_p < 1:
        p32 = max(1, math.floor(top_p * 2 ** 32))
        keep = sum(1 for i, v in enumerate(run) if (v - int(w[cols[i]])) << 32 < p32 * run[-1])
        run, cols = run[:keep], cols[:keep]
    u32 = 0 if not u > 0 else min(2 ** 32 - 1, math.floor(float(np.float32(u)) * 2 ** 32)) if u < 1 else 2 ** 32 - 1
    target = u32 * run[-1] >> 32
    at = next(i for i, v in enumerate(run) if v > target)
    return int(cols[at]), int(w[cols[at]]), run[-1], len(run)


def sample(x: np.ndarray, u, tau, top_k=None, top_p=None, min_p=None):
    """Tokens, probabilities (fp64) and numbers kept of the rows of x (fp32 values of the biased logits)."""
    B = x.shape[0]
    out = [sample_row(x[b], u[b], tau[b], 0 if top_k is None else int(top_k[b]), 1.0 if top_p is None else top_p[b],
                      0.0 if min_p is None else min_p[b]) for b in range(B)]
    return (np.array([o[0] for o in out], np.int32), np.array([o[1] / o[2] if o[2] else 0.0 for o in out]),
            np.array([o[3] for o in out], np.int32))
