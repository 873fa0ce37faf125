"""Plain implementations of the operators between hidden states and logits, for
the tests: row by row from the definitions in include/epic.h, on the CPU.  The
cross entropy and its gradients in 64 bits, the 8-bit rows and logits in the
float32 roundings that the header names (whole sums in 64 bits)."""
from __future__ import annotations

import numpy as np
import torch


def counted(B, m, seqs=None, start=None, target=None) -> np.ndarray:
    """Which rows count [B, m]."""
    on = np.ones((B, m), bool)
    for b in range(B):
        for i in range(m):
            if seqs is not None:
                at = (0 if start is None else int(start[b])) + i
                on[b, i] = 0 <= at < seqs.shape[1] and seqs[b, at] == -1
            if target is not None and target[b, i] < 0:
                on[b, i] = False
    return on


def loss(hidden, head, target, on, weight=None, lse=None):
    """loss, lse [B, m], grad_hidden [B, m, d], grad_head [V, d] in 64 bits, and
    for each gradient the sums of its terms' magnitudes (what roundings are
    relative to).  With lse the gradients go by it."""
    h, w = hidden.double(), head.double()
    B, m, d = h.shape
    V = w.shape[0]
    out = torch.zeros((B, m), dtype=torch.float64), torch.zeros((B, m), dtype=torch.float64)
    gh, gw = torch.zeros_like(h), torch.zeros_like(w)
    gh_size, gw_size = torch.zeros_like(h), torch.zeros_like(w)
    for b, i in zip(*np.nonzero(on)):
        y = int(target[b, i])
        l = w @ h[b, i]
        own = torch.logsumexp(l, 0)
        out[1][b, i] = own
        if y >= V:
            out[0][b, i] = float("nan")
            continue
        out[0][b, i] = own - l[y]
        p = torch.exp(l - (own if lse is None else lse[b, i].double()))
        g = p.clone()
        g[y] -= 1
        g *= 1.0 if weight is None else float(weight[b, i])
        gh[b, i] = g @ w
        gh_size[b, i] = g.abs() @ w.abs()
        gw += g[:, None] * h[b, i]
        gw_size += g.abs()[:, None] * h[b, i].abs()
    return out[0], out[1], gh, gw, gh_size, gw_size


def quantize(x):
    """q (float32 whole numbers) and scale of the rows of x [R, d]."""
    x = x.float()
    if x.shape[1] == 0 or x.shape[0] == 0:
        return x, x.new_zeros(x.shape[0])
    odd = ~torch.isfinite(x).all(1)
    top = x.abs().amax(1)
    none = top < 1e-30
    safe = torch.where(odd | none, torch.ones_like(top), top)
    q = torch.round(x * (torch.full_like(safe, 127.0) / safe)[:, None])
    q = torch.where((odd | none)[:, None], torch.zeros_like(q), q)
    scale = torch.where(none, torch.zeros_like(top), top / torch.full_like(top, 127.0))
    return q, torch.where(odd, torch.full_like(top, float("nan")), scale)


def logits_q8(hidden, q_head, scale_head, on, dtype):
    """Logits [rows that count, V] in dtype, in the order of the rows."""
    q, scale = quantize(hidden[torch.from_numpy(on)])
    sums = q.to(torch.int64) @ q_head.to(torch.int64).t()
    return ((sums.to(torch.float32) * scale[:, None]) * scale_head[None, :]).to(dtype)
