"""Plain 64-bit attention under any mask, and which keys a sliding window with first tokens lets a query see."""
import numpy as np


def seen(first_query, n, m, window=None, sinks=0):
    """bool [n, m]: queries at positions first_query, first_query + 1, ... over m keys."""
    p, j = first_query + np.arange(n)[:, None], np.arange(m)[None, :]
    ok = j <= p
    if window is not None:
        ok &= (j > p - window) | (j < sinks)
    return ok


def attend(q, k, v, ok, scale):
    """q [n, D], k, v [m, D] float64: out, lse, p, p @ |v|; 0 and -inf for a query without a key.  Keys that a query does
    not see have no part in it, whatever they hold."""
    n, m = ok.shape
    out, mag = np.zeros((n, v.shape[1])), np.zeros((n, v.shape[1]))
    lse, p = np.full(n, -np.inf), np.zeros((n, m))
    for i in range(n):
        at = np.flatnonzero(ok[i])
        if len(at) == 0:
            continue
        s = (k[at] @ q[i]) * scale
        t = s.max()
        x = np.exp(s - t)
        lse[i] = t + np.log(x.sum())
        p[i, at] = x / x.sum()
        out[i], mag[i] = p[i, at] @ v[at], p[i, at] @ np.abs(v[at])
    return out, lse, p, mag
