"""The operators around the validity check, as cases to be timed: what turns a
denoiser's logits into proposals, and what trains the denoiser.

A case names its operator in `op`:

* "sample":   one token and its confidence for every masked position, from
              logits rows and given uniform numbers (temperature, top-k, top-p,
              min-p per sequence);
* "propose":  the most confident sampled tokens of every sequence as the
              candidate arrays that the validity check reads;
* "distill":  the divergence of a student's rows from a teacher's top logits.
              `pass`: "both" (losses and the logits' gradient in one call),
              "forward" (losses) or "backward" (the gradient from what the
              forward pass kept).

Where `own` is false, run() computes the same in elementary torch operations;
where it is true, it calls the library.  Logits are [B, m, V]: row i of
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
LOG2E = 1.4426950408889634
ONE = 2147483648.0  # the weight of the likeliest token, 2**31


def _sample(name, B, n, m, V, dtype, mask, temperature, top_k=0, top_p=1.0, min_p=0.0, mixed=False, pad=0):
    c = {"op": "sample", "B": B, "n": n, "m": m, "V": V, "dtype": dtype, "mask": mask, "temperature": temperature,
         "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed, "pad": pad}
    return {"name": name, **c} if name else c


def _propose(name, B, n, m, per_seq, mask, coarse):
    c = {"op": "propose", "B": B, "n": n, "m": m, "per_seq": per_seq, "mask": mask, "coarse": coarse}
    return {"name": name, **c} if name else c


def _distill(name, direction, B, n, m, V, dtype, mask, K, tau, rest, pad=0):
    c = {"op": "distill", "pass": direction, "B": B, "n": n, "m": m, "V": V, "dtype": dtype, "mask": mask, "K": K,
         "tau": tau, "rest": rest, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the arithmetic workload: four short expressions, half masked, no filter
        _sample("sample_4x32_v512", 4, 32, 32, 512, "float32", 0.5, 1.0),
        # one masked position of one user, every filter: latency only
        _sample("sample_1x1_v32768", 1, 1, 1, 32768, "bfloat16", 1.0, 0.8, 50, 0.95, 0.02),
        # the JSON workload, nucleus sampling
        _sample("sample_8x128_v4096", 8, 128, 128, 4096, "float16", 0.5, 0.7, 0, 0.9),
        # the code workload, every request with settings of its own (some greedy)
        _sample("sample_16x256_v32768", 16, 256, 256, 32768, "bfloat16", 0.7, 1.0, 0, 1.0, 0.0, True),
        # the code workload at scale: a block of 32 positions of 1024, the plain softmax
        _sample("sample_64x32_v32768", 64, 1024, 32, 32768, "bfloat16", 0.8, 1.0),
        # a large odd vocabulary in 32 bits, rows at odd addresses, late in decoding
        _sample("sample_5x211_v100003", 5, 211, 211, 100003, "float32", 0.15, 0.9, 0, 0.95, 0.01, False, 2),
        # the JSON workload's candidates
        _propose("propose_8x128", 8, 128, 128, 8, 0.5, False),
        # whole canvases of a serving batch, confidences with many ties
        _propose("propose_64x1024", 64, 1024, 1024, 16, 0.8, True),
        # a small student in 32 bits: losses and gradient
        _distill("distill_4x32_v512", "both", 4, 32, 32, 512, "float32", 0.5, 8, 1.0, True),
        # an evaluation pass over odd sizes: losses alone, the teacher's top renormalised
        _distill("distill_forward_12x130_v50021", "forward", 12, 130, 130, 50021, "float16", 0.6, 32, 2.0, False, 1),
        # a training step of the code workload: losses and gradient in one call
        _distill("distill_16x256_v32768", "both", 16, 256, 256, 32768, "bfloat16", 0.7, 64, 1.0, True),
        # the backward pass alone of a large training batch, every position counts
        _distill("distill_backward_32x256_v32768", "backward", 32, 256, 256, 32768, "bfloat16", 1.0, 64, 2.0, True),
    ]


def _log_int(rng, lo, hi):
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case of the same ranges: any operator, batch, window,
    vocabulary from 512 to 131072, type, settings and row stride."""
    op = rng.choice(["sample", "sample", "sample", "propose", "distill", "distill", "distill"])
    mask = round(rng.uniform(0.1, 1.0), 3)
    if op == "propose":
        n = _log_int(rng, 1, 1024)
        m = n if rng.random() < 0.5 else rng.randint(1, n)
        return _propose(None, _log_int(rng, 1, 64), n, m, rng.randint(1, 64), mask, rng.random() < 0.5)
    dtype = rng.choice(["float32", "float16", "bfloat16", "bfloat16"])
    V = _log_int(rng, 512, 131072)
    if rng.random() < 0.4:
        V = max(512, V // 64 * 64)
    pad = rng.choice([0, 0, 1, 5, 8, 64])
    n = _log_int(rng, 1, 1024)
    m = n if rng.random() < 0.5 else min(n, rng.choice([16, 32, 33, 64]))
    rows = 4096 * 32768 if op == "sample" else 4096 * 16384  # elements, at most
    m = min(m, max(1, rows // (V + pad)))
    B = _log_int(rng, 1, max(1, min(64, rows // ((V + pad) * m))))
    if op == "sample":
        return _sample(None, B, n, m, V, dtype, mask, rng.choice([0.0, 0.3, 0.7, 1.0, 1.3]), rng.choice([0, 0, 1, 40, 300, 5000]),
                       rng.choice([1.0, 1.0, 0.99, 0.9, 0.5]), rng.choice([0.0, 0.0, 0.02, 0.1]), rng.random() < 0.4, pad)
    return _distill(None, rng.choice(["both", "both", "forward", "backward"]), B, n, m, V, dtype, mask, rng.randint(1, 128),
                    rng.choice([1.0, 1.0, 2.0, 0.5]), rng.random() < 0.6, pad)


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


def _logits(case, gen, dev):
    """Rows as a language model has them: a spread-out bulk, a few likely
    tokens that stand out by 3 to 14, and ids that may not be written (-inf).
    Row strides are V + pad."""
    B, m, V = case["B"], case["m"], case["V"]
    full = torch.empty((B, m, V + case["pad"]), dtype=DTYPES[case["dtype"]], device=dev)
    full.normal_(0.0, 2.0, generator=gen)
    l = full[:, :, :V]
    allowed = V - max(1, V // 100)
    apart = allowed // 6  # six different ids
    hot = torch.randint(0, apart, (B, m, 6), generator=gen, device=dev) + torch.arange(6, device=dev) * apart
    hot = (hot + torch.randint(0, allowed, (B, m, 1), generator=gen, device=dev)) % allowed
    up = 3.0 + 11.0 * torch.rand((B, m, 6), generator=gen, device=dev)
    up[:, :, 1:] -= 3.0
    l.scatter_(2, hot, up.to(l.dtype))
    l[:, :, allowed:] = -math.inf
    return l, hot, allowed


def prepare(case, seed):
    """What the program around the operator holds: the model's logits, the
    sequences, the requests' settings, the random numbers, the teacher's top
    logits, and the output tensors."""
    dev = torch.device("cuda:0")
    rng = np.random.default_rng([int(seed), 722])
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 7919 + 17)
    B, n, m = case["B"], case["n"], case["m"]
    seqs, start = _canvas(case, rng)
    s = {"op": case["op"], "seqs": torch.from_numpy(seqs).to(dev),
         "start": None if m == n else torch.from_numpy(start).to(dev), "B": B, "n": n, "m": m}
    if case["op"] == "propose":
        masked = _counted(s)
        conf = torch.rand((B, m), generator=gen, device=dev)
        if case["coarse"]:  # confidences of a model in 16 bits
            conf = (conf * 64).floor() / 64
        s["tok"] = torch.where(masked, torch.randint(0, 32768, (B, m), generator=gen, device=dev), -1).to(torch.int32)
        s["conf"] = torch.where(masked, conf, 0.0)
        s["per_seq"] = case["per_seq"]
        C = B * case["per_seq"]
        s["cand"] = [torch.empty(C, dtype=torch.int32, device=dev) for _ in range(3)]
        s["cand"].append(torch.empty(C, dtype=torch.float32, device=dev))
        s["offsets"] = torch.empty(B + 1, dtype=torch.int32, device=dev)
        return s
    s["logits"], hot, allowed = _logits(case, gen, dev)
    V = case["V"]
    if case["op"] == "sample":
        t, k, p, q = (np.full(B, case[x]) for x in ("temperature", "top_k", "top_p", "min_p"))
        if case["mixed"]:
            t = np.where(rng.random(B) < 0.125, 0.0, rng.uniform(0.5, 1.5, B))
            k = rng.choice([0, 20, 50, 200], B)
            p = np.where(rng.random(B) < 0.3, 1.0, rng.uniform(0.5, 1.0, B))
            q = rng.choice([0.0, 0.05, 0.1], B)
        on = lambda a, d: torch.from_numpy(np.ascontiguousarray(a.astype(d))).to(dev)  # noqa: E731
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = on(t, np.float32), on(k, np.int32), on(p, np.float32), on(q, np.float32)
        s["uniform"] = torch.rand((B, m), generator=gen, device=dev)
        s["tok"] = torch.empty((B, m), dtype=torch.int32, device=dev)
        s["conf"] = torch.empty((B, m), dtype=torch.float32, device=dev)
        return s
    K, tau = min(case["K"], V // 2), case["tau"]
    s["pass"], s["tau"] = case["pass"], tau
    # the teacher's likeliest token is one that the student likes too
    s["top_idx"] = ((hot[:, :, :1] + torch.arange(K, device=dev) * (allowed // K)) % allowed).to(torch.int32)
    lead = 3.0 * torch.randn((B, m, K), generator=gen, device=dev) + 2.0
    lead[:, :, :1] += 6.0
    s["top_logit"] = lead.sort(dim=-1, descending=True).values
    share = 0.02 + 0.2 * torch.rand((B, m, 1), generator=gen, device=dev)  # the teacher's mass outside its top
    lse = torch.logsumexp(s["top_logit"] / tau, dim=-1, keepdim=True) - torch.log(1 - share)
    s["teacher_lse"] = lse[:, :, 0].contiguous() if case["rest"] else None
    counted = _counted(s)
    # each position's weight in the batch's mean; gradients in float16 come with a loss scale
    scale = (4096.0 if case["dtype"] == "float16" else 1.0) / (B * _masked_rows(case))
    s["weight"] = scale * (0.5 + torch.rand((B, m), generator=gen, device=dev))
    s["loss"] = torch.empty((B, m), dtype=torch.float32, device=dev)
    s["stats"] = torch.empty((B, m, 2), dtype=torch.float32, device=dev)
    if case["pass"] != "forward":
        s["grad"] = torch.empty((B, m, V), dtype=s["logits"].dtype, device=dev)
    if case["pass"] == "backward":
        step = max(1, (1 << 26) // (m * V))
        for b in range(0, B, step):
            part = {k: v[b:b + step] if isinstance(v, torch.Tensor) else v for k, v in s.items()}
            s["stats"][b:b + step] = _distill_rows(part, counted[b:b + step])[4]
    return s


def _counted(s):
    """Which rows count: the masked positions of the windows."""
    at = torch.arange(s["m"], device=s["seqs"].device)[None, :]
    if s["start"] is not None:
        at = at + s["start"][:, None]
    inside = (at >= 0) & (at < s["n"])
    there = s["seqs"].gather(1, at.clamp(0, s["n"] - 1).expand(s["seqs"].shape[0], -1).long())
    return inside & (there == -1)


def _share(mass, part):
    """floor(mass * part / 2**24) of whole numbers, part <= 2**24."""
    return (mass >> 24) * part + (((mass & 16777215) * part) >> 24)


def _plain_sample(s):
    l = s["logits"].float()
    l = torch.where(torch.isnan(l), -math.inf, l) + 0.0
    top = l.amax(-1, keepdim=True)
    T = s["temperature"][:, None, None]
    greedy = T <= 0
    c = (LOG2E / torch.where(greedy, 1.0, T).double()).float().clamp(max=1e30)
    e = torch.exp2((l - top) * c)
    e = torch.where(torch.isnan(e), 0.0, e)
    w = (e * ONE + 0.5).to(torch.int64)
    all_mass = w.sum(-1, keepdim=True)
    ids = l.sort(dim=-1, descending=True, stable=True).indices
    ws = w.gather(-1, ids)
    rank = torch.arange(l.shape[-1], device=l.device)
    k = s["top_k"][:, None, None]
    in_k = (k <= 0) | (rank < k)
    part = (s["top_p"][:, None, None] * 16777216.0).clamp(0, 16777216).to(torch.int64)
    need = _share((ws * in_k).sum(-1, keepdim=True), part).clamp(min=1)
    least = (s["min_p"][:, None, None].clamp(0, 1) * ONE + 0.5).to(torch.int64)
    keep = torch.where(greedy, rank == 0, in_k & (ws.cumsum(-1) - ws < need) & (ws >= least))
    kept = torch.zeros_like(w).scatter_(-1, ids, ws * keep)
    upto = kept.cumsum(-1)
    u = (s["uniform"].clamp(0, 1)[:, :, None] * 16777216.0).to(torch.int64).clamp(max=16777215)
    tok = (upto <= _share(upto[:, :, -1:], u)).sum(-1, keepdim=True).clamp(max=l.shape[-1] - 1)
    conf = e.gather(-1, tok) * (ONE / all_mass.float())
    ok = _counted(s)[:, :, None] & torch.isfinite(top) & (all_mass > 0)
    return {"tok": torch.where(ok, tok, -1)[:, :, 0].to(torch.int32), "conf": torch.where(ok, conf, 0.0)[:, :, 0]}


def _plain_propose(s):
    tok, conf, B, m, P = s["tok"], s["conf"], s["B"], s["m"], s["per_seq"]
    fine = (tok >= 0) & ~torch.isnan(conf)
    key = torch.where(fine, conf, -math.inf)
    order = key.sort(dim=-1, descending=True, stable=True).indices
    # rows that count come first, the most confident before the others
    order = order.gather(1, (~fine.gather(1, order)).to(torch.int32).sort(dim=-1, stable=True).indices)
    count = fine.sum(-1).clamp(max=P)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=tok.device), count.cumsum(0)])
    rank = torch.arange(m, device=tok.device)[None, :]
    slot = torch.where(rank < count[:, None], offsets[:-1, None] + rank, B * P).reshape(-1)
    pos = order if s["start"] is None else order + s["start"][:, None]
    seq = torch.arange(B, device=tok.device)[:, None].expand(-1, m)

    def put(values, nothing, dtype):
        out = torch.full((B * P + 1,), nothing, dtype=dtype, device=tok.device)
        out[slot] = values.reshape(-1).to(dtype)
        return out[:-1]

    return {"seq": put(seq, -1, torch.int32), "pos": put(pos, -1, torch.int32), "tok": put(tok.gather(1, order), -1, torch.int32),
            "conf": put(conf.gather(1, order), 0.0, torch.float32), "offsets": offsets.to(torch.int32)}


def _lse(z):
    top = z.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    return top + torch.log(torch.exp(z - top).sum(-1, keepdim=True))


def _teacher(s):
    """The shares of the teacher's entries [B, m, K], what is left to the rest
    [B, m, 1], and which entries there are."""
    there = s["top_idx"] >= 0
    t = torch.where(there, s["top_logit"].float() / s["tau"], -math.inf)
    if s["teacher_lse"] is None:
        q = torch.exp(t - _lse(t))
        return torch.where(there, q, 0.0), torch.zeros_like(q[:, :, :1]), there
    q = torch.exp(t - s["teacher_lse"][:, :, None])
    return q, (1.0 - q.sum(-1, keepdim=True)).clamp(min=0.0), there


def _distill_rows(s, counted):
    """The losses, the student's scaled rows, the teacher's shares by token,
    what is left to the rest, and lse and lse_rest."""
    z = s["logits"].float() / s["tau"]
    q, rest, there = _teacher(s)
    at = torch.where(there, s["top_idx"], 0).long()
    member = torch.zeros_like(z).scatter_add_(-1, at, there.float()) > 0
    lse_rest = _lse(torch.where(member, -math.inf, z))
    lse = _lse(z)
    rest = torch.where(torch.isfinite(lse_rest), rest, 0.0)
    own_q = torch.where(q > 0, q, 1.0)
    each = torch.where(q > 0, q * (torch.log(own_q) - z.gather(-1, at) + lse), 0.0)
    left = torch.where(rest > 0, rest * (torch.log(torch.where(rest > 0, rest, 1.0)) - lse_rest + lse), 0.0)
    loss = (each.sum(-1, keepdim=True) + left) * (s["tau"] * s["tau"])
    counts = counted[:, :, None] & torch.isfinite(lse) & there.any(-1, keepdim=True)
    shares = torch.zeros_like(z).scatter_add_(-1, at, q)
    return (torch.where(counts, loss, 0.0)[:, :, 0], z, (member, shares, rest), counts,
            torch.where(counts, torch.cat([lse, lse_rest], -1), 0.0))


def _distill_grad(s, z, member, shares, rest, counts, stats):
    lse, lse_rest = stats[:, :, :1], stats[:, :, 1:]
    outside = torch.exp(z - lse_rest) * (torch.exp(lse_rest - lse) - rest)
    grad = torch.where(member, torch.exp(z - lse) - shares, outside)
    return torch.where(counts, grad * (s["tau"] * s["weight"][:, :, None]), 0.0).to(s["logits"].dtype)


def _plain_distill(s):
    counted = _counted(s)
    loss, z, (member, shares, rest), counts, stats = _distill_rows(s, counted)
    if s["pass"] == "forward":
        return {"loss": loss, "stats": stats}
    if s["pass"] == "backward":
        return {"grad": _distill_grad(s, z, member, shares, rest, counts, s["stats"])}
    return {"loss": loss, "stats": stats, "grad": _distill_grad(s, z, member, shares, rest, counts, stats)}


def run(state):
    s = state
    if not own:
        return {"sample": _plain_sample, "propose": _plain_propose, "distill": _plain_distill}[s["op"]](s)
    from paper_2606_00722_amd import epic

    if s["op"] == "sample":
        epic.sample(s["logits"], s["seqs"], s["uniform"], s["tok"], s["conf"], start=s["start"],
                    temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"tok": s["tok"], "conf": s["conf"]}
    if s["op"] == "propose":
        seq, pos, tok, conf = s["cand"]
        epic.propose(s["tok"], s["conf"], s["per_seq"], seq, pos, tok, conf, s["offsets"], start=s["start"])
        return {"seq": seq, "pos": pos, "tok": tok, "conf": conf, "offsets": s["offsets"]}
    teacher = {"start": s["start"], "teacher_lse": s["teacher_lse"], "tau": s["tau"]}
    if s["pass"] == "backward":
        epic.distill_backward(s["logits"], s["seqs"], s["top_idx"], s["top_logit"], s["stats"], s["weight"], s["grad"], **teacher)
        return {"grad": s["grad"]}
    if s["pass"] == "forward":
        epic.distill_forward(s["logits"], s["seqs"], s["top_idx"], s["top_logit"], s["loss"], s["stats"], **teacher)
        return {"loss": s["loss"], "stats": s["stats"]}
    epic.distill_forward(s["logits"], s["seqs"], s["top_idx"], s["top_logit"], s["loss"], s["stats"],
                         weight=s["weight"], grad=s["grad"], **teacher)
    return {"loss": s["loss"], "stats": s["stats"], "grad": s["grad"]}


def work(case):
    """Bytes: every row that counts read once, every output written once (a
    gradient has a row for every position).  Operations: per logit, a
    difference, a product, an exponential and a sum, and for a gradient an
    exponential and two products more."""
    B, m = case["B"], case["m"]
    other = 4 * B * m + (0 if m == case["n"] else 4 * B)  # the window's tokens, starts
    if case["op"] == "propose":
        return {"bytes": 8 * B * m + (0 if m == case["n"] else 4 * B) + 16 * B * case["per_seq"] + 4 * (B + 1), "flops": 0}
    V, size = case["V"], BYTES[case["dtype"]]
    rows = B * _masked_rows(case)
    if case["op"] == "sample":
        return {"bytes": rows * V * size + other + 16 * B + 4 * rows + 8 * B * m, "flops": 4 * rows * V}
    K = min(case["K"], V // 2)
    other += rows * (8 * K + (4 if case["rest"] else 0))
    read, grad = rows * V * size, B * m * V * size
    if case["pass"] == "forward":
        return {"bytes": read + other + 12 * B * m, "flops": 4 * rows * V}
    if case["pass"] == "backward":
        return {"bytes": read + grad + other + 12 * rows, "flops": 4 * rows * V}
    return {"bytes": read + grad + other + 12 * B * m + 4 * rows, "flops": 7 * rows * V}


def _exact_sample(case, s):
    """One sequence after another: probabilities in 64 bits, the prefix of the
    sorted tokens that the filters leave, and the draw from it in the order of
    the ids."""
    B, m, V = case["B"], case["m"], case["V"]
    counted = _counted(s)
    conf = torch.zeros((B, m), dtype=torch.float64, device=counted.device)
    for b in range(B):
        rows = counted[b].nonzero()[:, 0]
        z = s["logits"][b, rows].double()
        T = float(s["temperature"][b])
        p = torch.softmax(z / (T if T > 0 else 1.0), dim=-1)
        if T <= 0:
            conf[b, rows] = p.max(dim=-1).values
            continue
        likely, ids = p.sort(dim=-1, descending=True, stable=True)
        k = int(s["top_k"][b])
        count = torch.full((len(rows), 1), V if k <= 0 else min(k, V), device=p.device)
        mass = likely.cumsum(-1)
        P = math.floor(min(1.0, float(s["top_p"][b])) * 2 ** 24) / 2 ** 24
        if P < 1.0:
            goal = mass.gather(-1, count - 1) * P
            count = torch.minimum(count, 1 + (mass < goal).sum(-1, keepdim=True))
        count = torch.minimum(count, (likely >= likely[:, :1] * float(s["min_p"][b])).sum(-1, keepdim=True))
        left = torch.where(torch.arange(V, device=p.device) < count, likely, 0.0)
        upto = torch.zeros_like(p).scatter_(-1, ids, left).cumsum(-1)
        u = (s["uniform"][b, rows].double() * 2 ** 24).floor() / 2 ** 24
        at = torch.searchsorted(upto, (upto[:, -1] * u)[:, None], right=True).clamp(max=V - 1)
        conf[b, rows] = p.gather(-1, at)[:, 0]
    return {"tok": None, "conf": conf}


def _exact_propose(case, s):
    B, m, P = case["B"], case["m"], case["per_seq"]
    tok, conf = s["tok"].cpu().numpy(), s["conf"].cpu().numpy().astype(np.float64)
    out = []
    for b in range(B):
        at = np.flatnonzero(tok[b] >= 0)
        out += conf[b, at[np.lexsort((at, -conf[b, at]))[:P]]].tolist()
    return {"seq": None, "pos": None, "tok": None, "conf": np.array(out + [0.0] * (B * P - len(out))), "offsets": None}


def _exact_distill(case, s):
    """Row by row from the divergence of the two distributions over the
    teacher's tokens and the rest; the gradient through the softmax of it."""
    B, m, V, tau = case["B"], case["m"], case["V"], case["tau"]
    dev = s["seqs"].device
    counted = _counted(s)
    loss = torch.zeros((B, m), dtype=torch.float64, device=dev)
    stats = torch.zeros((B, m, 2), dtype=torch.float64, device=dev)
    grad = None if case["pass"] == "forward" else torch.zeros((B, m, V), dtype=torch.float64, device=dev)
    for b in range(B):
        rows = counted[b].nonzero()[:, 0]
        ids, t = s["top_idx"][b, rows].long(), s["top_logit"][b, rows].double() / tau
        logp = torch.log_softmax(s["logits"][b, rows].double() / tau, dim=-1)
        z = s["logits"][b, rows].double() / tau
        others = torch.ones_like(z, dtype=torch.bool).scatter_(-1, ids, False)
        lse_rest = torch.logsumexp(z.masked_fill(~others, -math.inf), dim=-1)
        lse = torch.logsumexp(z, dim=-1)
        if s["teacher_lse"] is None:
            logq = torch.log_softmax(t, dim=-1)
            rest = torch.zeros_like(lse)
        else:
            logq = t - s["teacher_lse"][b, rows, None].double()
            rest = 1 - logq.exp().sum(-1)
        kl = (logq.exp() * (logq - logp.gather(-1, ids))).sum(-1)
        kl = kl + torch.where(rest > 0, rest * (torch.log(rest.clamp(min=1e-300)) - (lse_rest - lse)), 0.0)
        loss[b, rows] = kl * tau * tau
        stats[b, rows] = torch.stack([lse, lse_rest], -1)
        if grad is not None:
            # every token pulls by its share of the teacher: a listed one by its own, the others by what the rest is given
            want = torch.where(others, rest[:, None] * torch.exp(z - lse_rest[:, None]), 0.0).scatter_add_(-1, ids, logq.exp())
            grad[b, rows] = (logp.exp() - want) * (tau * s["weight"][b, rows, None].double())
    if case["pass"] == "forward":
        return {"loss": loss, "stats": stats}
    if case["pass"] == "backward":
        return {"grad": grad}
    return {"loss": loss, "stats": stats, "grad": grad}


def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "propose": _exact_propose, "distill": _exact_distill}[case["op"]](case, s)
