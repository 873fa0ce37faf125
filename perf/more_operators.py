"""The operators between a denoiser's hidden states and its logits (the head),
as cases to be timed.

A case names its operator in `op`:

* "loss":   softmax cross entropy of the masked rows' tokens over the whole
            vocabulary, from hidden states and the head's weights, without
            keeping the logits.  `pass`: "forward" (losses), "backward" (the
            gradients of hidden states and head from what the forward pass
            kept) or "both" (a training step: one after the other);
* "logits": the masked rows' logits from hidden states and a head laid out in
            8-bit integers: a scale for each row of hidden states (found in the
            call) and for each token of the vocabulary.

Where `own` is false, run() computes the same in elementary torch operations;
where it is true, it calls the library.  Hidden states are [B, m, d]: row i of
sequence b is its position start[b] + i (a window of m positions; a case whose
m equals n has no window), and only rows whose position is masked (token -1)
count.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
BYTES = {"float32": 4, "float16": 2, "bfloat16": 2}


def _loss(name, direction, B, n, m, V, d, dtype, mask, pad=0):
    c = {"op": "loss", "pass": direction, "B": B, "n": n, "m": m, "V": V, "d": d, "dtype": dtype, "mask": mask, "pad": pad}
    return {"name": name, **c} if name else c


def _logits(name, B, n, m, V, d, dtype, mask, pad=0):
    c = {"op": "logits", "B": B, "n": n, "m": m, "V": V, "d": d, "dtype": dtype, "mask": mask, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the arithmetic workload's training step, a small denoiser in 32 bits: latency counts
        _loss("loss_4x32_v512_d128", "both", 4, 32, 32, 512, 128, "float32", 0.5),
        # how likely one answer's window is under a model of a large vocabulary: few rows, the head read once
        _loss("loss_forward_1x16_v131072_d4096", "forward", 1, 256, 16, 131072, 4096, "bfloat16", 1.0),
        # an evaluation pass over odd sizes, rows at odd addresses
        _loss("loss_forward_12x130_v50021_d1000", "forward", 12, 130, 130, 50021, 1000, "float16", 0.6, 3),
        # the JSON workload's training step in 32 bits
        _loss("loss_8x128_v4096_d1024", "both", 8, 128, 128, 4096, 1024, "float32", 0.5),
        # the code workload's training step
        _loss("loss_16x256_v32768_d2048", "both", 16, 256, 256, 32768, 2048, "bfloat16", 0.7),
        # the backward pass alone of a large training batch, every position counts
        _loss("loss_backward_32x256_v32768_d4096", "backward", 32, 256, 256, 32768, 4096, "bfloat16", 1.0),
        # one masked position of one user: the head read once, latency
        _logits("logits_1x1_v32768_d2048", 1, 1, 1, 32768, 2048, "bfloat16", 1.0),
        # the JSON workload, a small model
        _logits("logits_8x128_v4096_d1024", 8, 128, 128, 4096, 1024, "float16", 0.5),
        # the code workload at scale: a block of 32 positions of 1024
        _logits("logits_64x32_v32768_d4096", 64, 1024, 32, 32768, 4096, "bfloat16", 0.8),
        # odd sizes in 32 bits, rows at odd addresses, late in decoding
        _logits("logits_5x211_v100003_d1000", 5, 211, 211, 100003, 1000, "float32", 0.15, 3),
        # whole canvases of the code workload
        _logits("logits_16x256_v32768_d4096", 16, 256, 256, 32768, 4096, "bfloat16", 0.7),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case of the same ranges: either operator, batch, window,
    vocabulary from 512 to 131072, width from 64 to 4096, type, share of masks
    and row stride."""
    op = rng.choice(["loss", "loss", "logits"])
    mask = round(rng.uniform(0.1, 1.0), 3)
    dtype = rng.choice(["float32", "float16", "bfloat16", "bfloat16"])
    V, d = _log_int(rng, 512, 131072), _log_int(rng, 64, 4096)
    if rng.random() < 0.5:
        V = max(512, V // 64 * 64)
    if rng.random() < 0.7:
        d = d // 64 * 64
    pad = rng.choice([0, 0, 0, 1, 8, 64])
    n = _log_int(rng, 1, 1024)
    m = n if rng.random() < 0.5 else min(n, rng.choice([16, 32, 33, 64]))
    # products of one pass over the head, and logits, at most
    rows = min(2 ** 39 // (V * d), 2 ** 28 // V) if op == "loss" else min(2 ** 39 // (V * d), 2 ** 27 // V)
    m = min(m, max(1, rows))
    B = _log_int(rng, 1, max(1, min(64, rows // m)))
    if op == "loss":
        return _loss(None, rng.choice(["both", "both", "forward", "backward"]), B, n, m, V, d, dtype, mask, pad)
    return _logits(None, B, n, m, V, d, dtype, mask, pad)


def _masked_rows(case):
    """How many rows of a sequence's window are masked."""
    return min(case["m"], max(1, round(case["mask"] * case["m"])))


def _canvas(case, rng):
    """Sequences int32 [B, n] with the window's share of masks (and nothing but
    masks behind it), and the windows' first positions."""
    B, n, m = case["B"], case["n"], case["m"]
    seqs = rng.integers(0, 500, size=(B, n)).astype(np.int32)
    start = rng.integers(0, n - m + 1, size=B).astype(np.int32)
    for b in range(B):
        seqs[b, start[b] + m:] = -1
        seqs[b, start[b] + rng.choice(m, _masked_rows(case), replace=False)] = -1
    return seqs, start


def _normal(shape, pad, scale, dtype, gen, dev):
    """Rows of normal numbers whose strides are the width and `pad`."""
    full = torch.empty((*shape[:-1], shape[-1] + pad), dtype=dtype, device=dev)
    full.normal_(0.0, scale, generator=gen)
    return full[..., : shape[-1]]


def _quantized(x):
    """Whole numbers from -127 to 127 (as float32) and the scale of each row:
    the scale is a 127th of the row's largest magnitude.  The quotients are
    float32, ties go to the even number."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    some = top > 0
    # tensors on both sides: of a number over a tensor, torch takes the reciprocal
    ratio = torch.where(some, torch.full_like(top, 127.0) / torch.where(some, top, 1.0), 0.0)
    return torch.round(x * ratio), (top / torch.full_like(top, 127.0))[..., 0]


def prepare(case, seed):
    """What the program around the operator holds: the network's hidden states,
    the head, the sequences, the answers' tokens, and the output tensors."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng([int(seed), 723])
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 7919 + 29)
    B, n, m, V, d = (case[k] for k in ("B", "n", "m", "V", "d"))
    dtype = DTYPES[case["dtype"]]
    seqs, start = _canvas(case, rng)
    s = {"op": case["op"], "rows": B * _masked_rows(case), "B": B, "n": n, "m": m,
         "seqs": torch.from_numpy(seqs).to(dev), "start": None if m == n else torch.from_numpy(start).to(dev)}
    # normed states, a bulk of logits that spreads by 2, and the answers' tokens up to 12 above it
    head = _normal((V, d), case["pad"], 2.0 / math.sqrt(d), dtype, gen, dev)
    hidden = _normal((B, m, d), case["pad"], 1.0, dtype, gen, dev)
    target = torch.randint(0, V, (B, m), generator=gen, device=dev)
    target = torch.where(torch.rand((B, m), generator=gen, device=dev) < 0.3, target % 97, target)  # some tokens are common
    step = max(1, (1 << 26) // (m * d))
    for b in range(0, B, step):
        lead = 3.0 * torch.rand((min(step, B - b), m, 1), generator=gen, device=dev)
        hidden[b:b + step] += (lead * head[target[b:b + step]].float()).to(dtype)
    s["hidden"] = hidden
    if case["op"] == "logits":
        stride = (d + 127) // 128 * 128  # how the library lays such a head out, once
        q = torch.zeros((V, stride), dtype=torch.int8, device=dev)
        scale = torch.empty(V, dtype=torch.float32, device=dev)
        step = max(1, (1 << 26) // d)
        for v in range(0, V, step):
            part, scale[v:v + step] = _quantized(head[v:v + step])
            q[v:v + step, :d] = part.to(torch.int8)
        s["q"], s["scale"] = q, scale
        s["logits"] = torch.zeros((B, m, V), dtype=dtype, device=dev)
    else:
        s["pass"], s["head"], s["target"] = case["pass"], head, target.to(torch.int32)
        # each position's weight in the batch's mean; gradients in float16 come with a loss scale
        up = (4096.0 if case["dtype"] == "float16" else 1.0) / s["rows"]
        s["weight"] = up * (0.5 + torch.rand((B, m), generator=gen, device=dev))
        s["loss"] = torch.empty((B, m), dtype=torch.float32, device=dev)
        s["lse"] = torch.empty((B, m), dtype=torch.float32, device=dev)
        if case["pass"] == "backward":
            s["lse"] = _plain_forward(s)["lse"]
        if case["pass"] != "forward":
            s["grad_hidden"] = torch.empty((B, m, d), dtype=dtype, device=dev)
            s["grad_head"] = torch.empty((V, d), dtype=dtype, device=dev)
    if own:
        from paper_2606_00722_amd import epic

        if case["op"] == "logits":
            s["workspace"] = epic.alloc_logits_q8_workspace(hidden)
        else:
            s["workspace"] = epic.alloc_head_loss_workspace(hidden, head, backward=case["pass"] != "forward")
    return s


def _counted(s):
    """Which rows count: the masked positions of the windows."""
    at = torch.arange(s["m"], device=s["seqs"].device)[None, :]
    if s["start"] is not None:
        at = at + s["start"][:, None]
    inside = (at >= 0) & (at < s["n"])
    there = s["seqs"].gather(1, at.clamp(0, s["n"] - 1).expand(s["seqs"].shape[0], -1).long())
    return inside & (there == -1)


def _rows_that_count(s):
    """Their numbers; how many they are, the program knows that masked them."""
    return (~_counted(s)).reshape(-1).to(torch.int32).sort(stable=True).indices[: s["rows"]]


def _spread(s, rows, values):
    """float32 [B, m, ...] of the rows' values, 0 for the others."""
    out = torch.zeros((s["B"] * s["m"], *values.shape[1:]), dtype=values.dtype, device=values.device)
    out[rows] = values
    return out.view(s["B"], s["m"], *values.shape[1:])


def _plain_products(s):
    rows = _rows_that_count(s)
    h, w = s["hidden"].reshape(-1, s["hidden"].shape[-1])[rows].float(), s["head"].float()
    return rows, h, w, h @ w.t()


def _plain_forward(s, products=None):
    rows, _, _, l = products or _plain_products(s)
    top = l.amax(-1, keepdim=True)
    lse = (top + torch.log(torch.exp(l - top).sum(-1, keepdim=True)))[:, 0]
    loss = lse - l.gather(1, s["target"].view(-1)[rows, None].long())[:, 0]
    return {"loss": _spread(s, rows, loss), "lse": _spread(s, rows, lse)}


def _plain_backward(s, lse, products=None):
    rows, h, w, l = products or _plain_products(s)
    p = torch.exp(l - lse.view(-1)[rows, None])
    one = torch.ones((), device=p.device)
    p.scatter_add_(1, s["target"].view(-1)[rows, None].long(), -one.expand(len(rows), 1))
    p *= s["weight"].view(-1)[rows, None]
    return {"grad_hidden": _spread(s, rows, p @ w).to(s["hidden"].dtype), "grad_head": (p.t() @ h).to(s["head"].dtype)}


def _plain_loss(s):
    if s["pass"] == "forward":
        return _plain_forward(s)
    if s["pass"] == "backward":
        return _plain_backward(s, s["lse"])
    products = _plain_products(s)
    out = _plain_forward(s, products)
    return {**out, **_plain_backward(s, out["lse"], products)}


def _plain_logits(s):
    d = s["hidden"].shape[-1]
    rows = _rows_that_count(s)
    q, scale = _quantized(s["hidden"].reshape(-1, d)[rows])
    l = (q @ s["q"][:, :d].float().t()) * scale[:, None] * s["scale"]
    return {"logits": _spread(s, rows, l.to(s["logits"].dtype))}


def run(state):
    s = state
    if not own:
        return _plain_logits(s) if s["op"] == "logits" else _plain_loss(s)
    from paper_2606_00722_amd import epic

    if s["op"] == "logits":  # rows that do not count stay as they are
        epic.logits_q8(s["hidden"], s["seqs"], s["q"], s["scale"], s["logits"], s["workspace"], start=s["start"])
        return {"logits": s["logits"]}
    out = {}
    if s["pass"] != "backward":
        epic.head_loss_forward(s["hidden"], s["seqs"], s["head"], s["target"], s["loss"], s["lse"], s["workspace"], start=s["start"])
        out = {"loss": s["loss"], "lse": s["lse"]}
    if s["pass"] != "forward":
        epic.head_loss_backward(s["hidden"], s["seqs"], s["head"], s["target"], s["lse"], s["weight"], s["grad_hidden"],
                                s["grad_head"], s["workspace"], start=s["start"])
        out.update(grad_hidden=s["grad_hidden"], grad_head=s["grad_head"])
    return out


def work(case):
    """Bytes: the hidden states of rows that count and the head read once, every
    output written once (a gradient of hidden states has a row for every
    position, logits only those that count).  Operations: 2 V d for each row
    and product: one for losses or logits, three for gradients (of which a pass
    that also gives losses shares the first)."""
    B, m, V, d = (case[k] for k in ("B", "m", "V", "d"))
    size, rows = BYTES[case["dtype"]], B * _masked_rows(case)
    other = 4 * B * m + (0 if m == case["n"] else 4 * B)  # the window's tokens, starts
    if case["op"] == "logits":
        return {"bytes": rows * d * size + V * d + 4 * V + rows * V * size + other, "flops": 2 * rows * V * d}
    read, grad = (rows + V) * d * size + other + 4 * rows, (B * m + V) * d * size
    if case["pass"] == "forward":
        return {"bytes": read + 8 * B * m, "flops": 2 * rows * V * d}
    if case["pass"] == "backward":
        return {"bytes": read + grad + 8 * rows, "flops": 6 * rows * V * d}
    return {"bytes": read + grad + 8 * B * m + 4 * rows, "flops": 6 * rows * V * d}


def _exact_loss(case, s):
    """Sequence by sequence, in 64 bits: log probabilities, and the gradient
    as what the softmax gives too much or too little to every token."""
    B, m, V, d = (case[k] for k in ("B", "m", "V", "d"))
    dev, counted, w = s["seqs"].device, _counted(s), s["head"].double()
    loss = torch.zeros((B, m), dtype=torch.float64, device=dev)
    lse = torch.zeros((B, m), dtype=torch.float64, device=dev)
    grad_hidden = torch.zeros((B, m, d), dtype=torch.float64, device=dev)
    grad_head = torch.zeros((V, d), dtype=torch.float64, device=dev)
    for b in range(B):
        at = counted[b].nonzero()[:, 0]
        h, y = s["hidden"][b, at].double(), s["target"][b, at].long()
        l = torch.mm(h, w.t())
        lse[b, at] = torch.logsumexp(l, dim=-1)
        loss[b, at] = lse[b, at] - (h * w[y]).sum(-1)
        if case["pass"] != "forward":
            u = s["weight"][b, at].double()
            known = s["lse"][b, at].double() if case["pass"] == "backward" else lse[b, at]
            excess = torch.exp(l - known[:, None]) * u[:, None]
            grad_hidden[b, at] = torch.mm(excess, w) - u[:, None] * w[y]
            grad_head.addmm_(excess.t(), h)
            grad_head.index_add_(0, y, -u[:, None] * h)
    if case["pass"] == "forward":
        return {"loss": loss, "lse": lse}
    if case["pass"] == "backward":
        return {"grad_hidden": grad_hidden, "grad_head": grad_head}
    return {"loss": loss, "lse": lse, "grad_hidden": grad_hidden, "grad_head": grad_head}


def _exact_logits(case, s):
    """The sums of whole numbers and the two scales in 64 bits; which whole
    numbers they are, the definition says in 32: a 127th of the largest
    magnitude is 1, the quotient rounded to float32."""
    B, m, V, d = (case[k] for k in ("B", "m", "V", "d"))
    counted = _counted(s)
    out = torch.zeros((B, m, V), dtype=torch.float64, device=counted.device)
    q_head = s["q"][:, :d].double() * s["scale"].double()[:, None]
    for b in range(B):
        at = counted[b].nonzero()[:, 0]
        x = s["hidden"][b, at].float()
        top = x.abs().amax(-1, keepdim=True)
        q = torch.round((x * (torch.full_like(top, 127.0) / top)).double())
        out[b, at] = torch.mm(q * (top.double() / 127.0), q_head.t())
    return {"logits": out}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_logits(case, s) if case["op"] == "logits" else _exact_loss(case, s)
