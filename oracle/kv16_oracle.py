"""fp64 oracle of the operators on a bf16 cache (test infrastructure): causal attention behind a prefix, the weight that
entries accumulate, and the scores made of it.  Written from the definitions of the operators; it shares no code with the
library."""
from __future__ import annotations

import numpy as np


def visible(m: int, n: int) -> np.ndarray:
    """[m][n]: query i stands at entry n - m + i and sees the entries up to its own."""
    return np.arange(n)[None] <= (np.arange(m) + n - m)[:, None]


def attention(q, k, v, kp=None, vp=None, scale=None):
    """(o [m][d], lse [m]) of rows q [m][d] over a prefix kp, vp (all of it) and own entries k, v [n][d]."""
    m, d = q.shape
    see = visible(m, len(k))
    if kp is not None:
        k, v = np.concatenate([kp, k]), np.concatenate([vp, v])
        see = np.concatenate([np.ones((m, len(kp)), bool), see], 1)
    tau = d ** -0.5 if scale is None else scale
    o, lse = np.zeros((m, d)), np.full(m, -np.inf)
    for i in range(m):
        js = np.flatnonzero(see[i])
        if len(js) == 0:
            continue
        with np.errstate(invalid="ignore"):
            z = tau * (k[js] @ q[i])
            top = z.max()
            w = np.exp(z - top)
            o[i] = (w / w.sum()) @ v[js]
            lse[i] = top + np.log(w.sum())
    return o, lse


def weights(q, k, lse, scale=None):
    """[n]: what entries k [n][d] receive of one head's queries q [m][d] with log-sum-exps lse [m]."""
    m, d = q.shape
    if m == 0 or len(k) == 0:
        return np.zeros(len(k))
    tau = d ** -0.5 if scale is None else scale
    return np.where(visible(m, len(k)), np.exp(np.where(visible(m, len(k)), tau * (q @ k.T) - lse[:, None], 0.0)), 0.0).sum(0)


def scores(w, first: int, recent: int):
    """Selection scores of one segment's weights w [n]."""
    s = np.array(w, dtype=np.float64)
    s[:first] = np.inf
    if recent:
        s[max(0, len(s) - recent):] = np.inf
    return s
