"""A small denoiser trained on a teacher's top logits, then decoding under the
grammar: the operators on logits rows together with the check.

    python -m paper_2606_00722_amd.denoise [--preset 1] [--train 60] [--seed 42]

The denoiser is one linear layer over fixed random features of every position,
in the place of a network's last hidden states; the teacher's likeliest token is
the hidden answer's.  A training step is two products around distill_forward,
which gives losses and the logits' gradient in one call.  A decoding step is
sample, propose, validate, select and fallback (one commit where the selection
is empty), all on the device; the host reads the number of candidates and
whether masks are left.
"""
from __future__ import annotations

import argparse
import math
from typing import Callable, List, Optional

import numpy as np

from . import epic
from . import workloads as W


class Denoiser:
    """Features [B, n, d], weights [d, V] in float32; logits [B, n, V] in
    bfloat16, in one buffer that the gradient overwrites."""

    def __init__(self, B: int, n: int, V: int, device, gen):
        import torch

        d = max(64, B * n)
        self.torch = torch
        self.x = torch.randn((B * n, d), generator=gen, device=device) / math.sqrt(d)
        self.w = torch.zeros((d, V), device=device)
        self.out = torch.empty((B, n, V), dtype=torch.bfloat16, device=device)
        self.loss = torch.empty((B, n), device=device)
        self.stats = torch.empty((B, n, 2), device=device)

    def logits(self):
        self.out.view(-1, self.out.shape[2]).copy_(self.x @ self.w)
        return self.out

    def train_step(self, seqs, top_idx, top_logit, teacher_lse, lr: float, tau: float = 1.0):
        """Mean loss over the masked positions (a device scalar)."""
        out = self.logits()
        masked = seqs == W.MASK
        weight = masked.to(self.torch.float32)
        epic.distill_forward(out, seqs, top_idx, top_logit, self.loss, self.stats, teacher_lse=teacher_lse, tau=tau,
                             weight=weight, grad=out)
        self.w -= lr * (self.x.t() @ out.view(-1, out.shape[2]).float())
        return self.loss.sum() / masked.sum()


def teacher(hidden: np.ndarray, V: int, K: int, rng: np.random.Generator, device):
    """Top logits per position: the answer's token and K - 1 others, and their
    logsumexp with 5 % left to the tokens that are not listed."""
    import torch

    B, n = hidden.shape
    idx = rng.integers(0, V, size=(B, n, K)).astype(np.int32)
    idx[:, :, 0] = hidden
    logit = rng.standard_normal((B, n, K)).astype(np.float32)
    logit[:, :, 0] += 6.0
    for k in range(1, K):  # no token twice
        idx[:, :, k][(idx[:, :, k, None] == idx[:, :, :k]).any(-1)] = -1
    lse = np.log(np.sum(np.where(idx >= 0, np.exp(logit), 0.0), axis=-1) / 0.95).astype(np.float32)
    return tuple(torch.from_numpy(a).to(device) for a in (idx, logit, lse))


def decode(ctx, model: Denoiser, seqs, gen, per_seq: int = 8, temperature: float = 0.8, top_k: int = 0, top_p: float = 0.95,
           max_steps: int = 500) -> int:
    """Fills the masks of seqs (int32 [B, n] on the GPU) in place; steps taken."""
    torch = model.torch
    dev, (B, n) = seqs.device, seqs.shape
    i32 = dict(dtype=torch.int32, device=dev)
    C = B * per_seq
    tok, conf = torch.empty((B, n), **i32), torch.empty((B, n), device=dev)
    cand = [torch.empty(C, **i32) for _ in range(3)]
    cand_conf, offsets = torch.empty(C, device=dev), torch.empty(B + 1, **i32)
    verdict, selected, accepted = (torch.zeros(C, dtype=torch.uint8, device=dev) for _ in range(3))
    T, p = torch.full((B,), temperature, device=dev), torch.full((B,), top_p, device=dev)
    k, one = torch.full((B,), top_k, **i32), torch.ones(B, **i32)
    ws = ctx.alloc_workspace(dev)
    logits = model.logits()  # of this denoiser they do not depend on what is committed
    for step in range(max_steps):
        if not bool((seqs == W.MASK).any()):
            return step
        u = torch.rand((B, n), generator=gen, device=dev)
        epic.sample(logits, seqs, u, tok, conf, temperature=T, top_k=k, top_p=p)
        epic.propose(tok, conf, per_seq, *cand, cand_conf, offsets)
        C = int(offsets[-1])
        s, at, t = (c[:C] for c in cand)
        ctx.validate(seqs, s, at, t, verdict[:C], ws)
        ctx.select(seqs, s, at, t, cand_conf[:C], verdict[:C], selected[:C], ws)
        ctx.fallback(seqs, s, at, t, cand_conf[:C], verdict[:C], selected[:C], one, accepted[:C], ws)
        take = (selected[:C] | accepted[:C]).bool()
        seqs[s[take].long(), at[take].long()] = t[take]
    return max_steps


def run(preset: int = 1, train: int = 60, seed: int = 42, lr: float = 4.0, log: Optional[Callable] = None) -> dict:
    import torch

    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    inst = W.make_instance(preset, seed)
    ctx = epic.Context.from_problem(W.arrays(inst.lang, inst.vocab), inst.B, inst.n, 8 * inst.B)
    ctx.lexmemo_build()
    model = Denoiser(inst.B, inst.n, inst.vocab.size, dev, gen)
    seqs = torch.from_numpy(inst.seqs).to(dev)
    top = teacher(inst.hidden, inst.vocab.size, 16, np.random.default_rng(seed), dev)
    losses: List[float] = []
    for i in range(train):
        loss = model.train_step(seqs, *top, lr=lr)
        if i % 10 == 0 or i == train - 1:
            losses.append(float(loss))
            if log:
                log(f"training step {i}: divergence {losses[-1]:.4f}")
    steps = decode(ctx, model, seqs, gen)
    filled = seqs.cpu().numpy()
    masked = inst.seqs == W.MASK
    res = {"losses": losses, "steps": steps, "seqs": filled, "left": int((filled == W.MASK).sum()),
           "as_answer": float((filled == inst.hidden)[masked].mean()), "errors": ctx.device_error()}
    if log:
        log(f"decoded {int(masked.sum())} masked tokens in {steps} steps, {res['left']} left, "
            f"{100 * res['as_answer']:.1f} % as in the answer")
    return res


if __name__ == "__main__":
    a = argparse.ArgumentParser(description="distill a small denoiser and decode with it under a grammar")
    a.add_argument("--preset", type=int, default=1, choices=sorted(W.PRESETS))
    a.add_argument("--train", type=int, default=60)
    a.add_argument("--seed", type=int, default=42)
    args = a.parse_args()
    run(args.preset, args.train, args.seed, log=lambda text: print(text, flush=True))
