"""Plain implementations of the operators on logits rows, for the tests: the
draw in whole numbers as include/epic.h defines it, the same draw in 64 bits,
and the divergence from a teacher's top logits in 64 bits (numpy, row by row)."""
from __future__ import annotations

import numpy as np

ONE = 2 ** 31


def share(mass: int, part: int) -> int:
    return mass * part // 2 ** 24


def scale_of(T: float) -> np.float32:
    """log2(e) / T in float32; greedy rows have T = 1."""
    if T <= 0:
        return np.float32(1.4426950408889634)
    return np.float32(min(np.float32(np.float64(1.4426950408889634) / np.float64(T)), np.float32(1e30)))


def exponents(l: np.ndarray, T: float) -> np.ndarray:
    """x of every logit: two float32 roundings."""
    with np.errstate(all="ignore"):
        return ((l - np.float32(np.nanmax(l))) * scale_of(T)).astype(np.float32)


def draw(l: np.ndarray, e: np.ndarray, u: float, T: float, k: int, p: float, q: float):
    """Token and confidence of one row: l float32 logits, e float32 = 2^x."""
    top = np.nanmax(l) if not np.all(np.isnan(l)) else -np.inf
    if not np.isfinite(top) or np.isnan(T):
        return -1, 0.0
    e = np.where(np.isnan(e) | np.isnan(l), 0, e).astype(np.float32)
    # the sum with 1/2 is rounded to float32 before it is cut off
    w = np.floor((e * np.float32(ONE) + np.float32(0.5)).astype(np.float64)).astype(np.int64)
    W = int(w.sum())
    key = np.where(np.isnan(l), -np.inf, l) + np.float32(0)
    order = np.lexsort((np.arange(len(l)), -key.astype(np.float64)))
    if T <= 0:
        tok = int(order[0])
        return tok, float(e[tok]) * ONE / W
    ws = w[order]
    n = len(l) if k <= 0 else min(k, len(l))
    S = int(ws[:n].sum())
    P = 2 ** 24 if not p < 1 else int(np.float32(max(p, 0.0)) * np.float32(2 ** 24))
    need = max(1, share(S, P))
    least = 0 if not q > 0 else int(np.float32(min(q, 1.0)) * np.float32(ONE) + np.float32(0.5))
    before = np.cumsum(ws) - ws
    keep = (np.arange(len(l)) < n) & (before < need) & (ws >= least)
    kept = np.zeros_like(w)
    kept[order] = ws * keep
    uu = 0.0 if np.isnan(u) else min(max(u, 0.0), 1.0)
    U = min(int(np.float32(uu) * np.float32(2 ** 24)), 2 ** 24 - 1)
    upto = np.cumsum(kept)
    tok = int(np.searchsorted(upto, share(int(upto[-1]), U), side="right"))
    return tok, float(e[tok]) * ONE / W


def probabilities(l: np.ndarray, T: float) -> np.ndarray:
    z = np.where(np.isnan(l), -np.inf, l).astype(np.float64) / (T if T > 0 else 1.0)
    p = np.exp(z - z.max())
    return p / p.sum()


def kept_range(p: np.ndarray, u: float, k: int, top_p: float, q: float, slack: float):
    """The tokens that a draw in 64 bits can give when every probability may be
    off by the share `slack`: those whose interval of the kept mass comes within
    slack of u, and the filters' borders within slack too."""
    order = np.lexsort((np.arange(len(p)), -p))
    n = len(p) if k <= 0 else min(k, len(p))
    mass = np.cumsum(p[order])
    S = mass[n - 1]
    P = 1.0 if not top_p < 1 else np.floor(max(top_p, 0.0) * 2 ** 24) / 2 ** 24
    sure = np.zeros(len(p), bool)
    maybe = np.zeros(len(p), bool)
    r = np.arange(len(p))
    before = mass - p[order]
    for out, s in ((sure, -slack), (maybe, slack)):
        ok = (r < n) & (before < S * P + s * max(S, 1e-300)) & (p[order] >= p[order[0]] * q * (1 - s) - 1e-300)
        ok[0] = True
        out[order] = ok
    if k > 0 and n < len(p):  # equal at the border: ids decide, in both
        edge = p[order[n - 1]]
        maybe |= np.abs(p - edge) <= slack * edge
    return sure, maybe


def distill(l: np.ndarray, ids, t, tau: float, lse_T):
    """loss, dloss/dlogits, lse, lse_rest of one row in 64 bits."""
    V = len(l)
    ids, t = np.asarray(ids), np.asarray(t, np.float64) / tau
    zero = np.zeros(V)
    if np.any(ids >= V):
        return np.nan, zero, 0.0, 0.0
    z = l.astype(np.float64) / tau
    there = ids >= 0
    fine = there.any() and (lse_T is not None or np.max(t[there], initial=-np.inf) > -np.inf)

    def lse_of(a):
        m = np.max(a, initial=-np.inf)
        return m if not np.isfinite(m) else m + np.log(np.sum(np.exp(a - m)))

    member = np.zeros(V, bool)
    member[ids[there]] = True
    lse, lse_rest = lse_of(z), lse_of(z[~member])
    if not fine or lse == -np.inf:
        return 0.0, zero, lse, lse_rest
    logq = t[there] - (lse_T if lse_T is not None else lse_of(t[there]))
    q = np.exp(logq)
    rest = max(0.0, 1.0 - q.sum()) if lse_T is not None and lse_rest > -np.inf else 0.0
    on = q > 0
    loss = np.sum(q[on] * (logq[on] - z[ids[there]][on] + lse))
    if rest > 0:
        loss += rest * (np.log(rest) - lse_rest + lse)
    want = np.zeros(V)
    np.add.at(want, ids[there], q)
    p = np.exp(z - lse)
    grad = p - want
    if lse_rest > -np.inf:
        out = np.exp(z - lse_rest) * (np.exp(lse_rest - lse) - rest)
        grad[~member] = out[~member]
    return tau * tau * loss, tau * grad, lse, lse_rest
