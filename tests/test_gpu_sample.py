"""epic_sample and epic_propose through the binding: every token bit for bit
against the draw in whole numbers (with torch's exp2 as the only shared step),
and against a draw in 64 bits within a bound on the kernel's roundings."""
import math

import numpy as np
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    return epic


DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def on(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dt)


def run(epic, logits, seqs=None, u=None, T=None, k=None, p=None, q=None, start=None, stream=None):
    B, m, _ = logits.shape
    tok = torch.full((B, m), -7, dtype=torch.int32, device=DEV)
    conf = torch.full((B, m), -7.0, device=DEV)
    u = np.full((B, m), 0.5) if u is None else u
    per = lambda a, dt: None if a is None else on(np.broadcast_to(np.asarray(a), (B,)), dt)  # noqa: E731
    epic.sample(logits, seqs, on(u, torch.float32), tok, conf, start=start, temperature=per(T, torch.float32),
                top_k=per(k, torch.int32), top_p=per(p, torch.float32), min_p=per(q, torch.float32), stream=stream)
    return tok, conf


def check_rows(l, u, T, k, p, q, tok, conf, V):
    """Rows of one sequence: float32 logits [R, V] on the GPU, host numbers."""
    rows = l.cpu().numpy()
    for i, row in enumerate(rows):
        with np.errstate(all="ignore"):
            x = R.exponents(row, T) if not np.all(np.isnan(row)) else np.full(V, np.nan, np.float32)
        e = torch.exp2(torch.from_numpy(x).to(DEV)).cpu().numpy()
        want = R.draw(row, e, float(u[i]), T, k, p, q)
        assert (tok[i], ) == (want[0], ), f"row {i}: token {tok[i]}, definition {want}"
        assert abs(conf[i] - want[1]) <= 4e-7 * want[1]  # two roundings of float32 and one of W
        if want[0] < 0:
            continue
        prob = R.probabilities(row, T)
        # x is at most 33 and rounded three times (c, the difference, the product); a weight by 2^-32 of the largest
        slack = 33 * 3 * 2.0 ** -24 + V * 2.0 ** -32 + 2.0 ** -22
        assert abs(conf[i] - prob[tok[i]]) <= slack * prob[tok[i]] + 2.0 ** -32 * prob.max()
        if T <= 0:
            continue
        sure, maybe = R.kept_range(prob, u[i], k, p, q, 8 * slack)
        assert maybe[tok[i]]
        lo = prob[:tok[i]][sure[:tok[i]]].sum() / prob[maybe].sum()
        hi = prob[:tok[i] + 1][maybe[:tok[i] + 1]].sum() / prob[sure].sum()
        uu = min(max(float(u[i]), 0.0), 1.0)
        assert lo - 8 * slack - 2.0 ** -23 <= uu <= hi + 8 * slack + 2.0 ** -23


# vocabularies: one token, around a wavefront's and a workgroup's share, odd, rows too long for registers
SIZES = [1, 2, 63, 64, 65, 513, 1000, 4097, 8192, 32768, 40001, 100003, 131073, 262144]
SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.2, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.1), (0.9, 300, 0.8, 0.02),
            (0.0, 7, 0.3, 0.5), (1.5, 5000, 0.99, 0.0)]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_tokens_bit_exact(epic, dt, V):
    rng = np.random.default_rng(V + len(dt))
    B, m = len(SETTINGS), 2 if V > 50000 else 4
    full = torch.from_numpy((2.5 * rng.standard_normal((B, m, V + 3))).astype(np.float32))
    full[:, 0] *= 3  # a peaked row: few tokens matter
    full[:, 1] *= 0.01  # a flat one: all do
    logits = full.to(DEV, DT[dt])[:, :, 1:V + 1]  # rows at odd addresses
    if V > 64:
        logits[:, :, V // 3:V // 3 + 20] = -math.inf
    u = rng.random((B, m)).astype(np.float32)
    T, k, p, q = zip(*SETTINGS)
    tok, conf = run(epic, logits, u=u, T=T, k=k, p=p, q=q)
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    for b in range(B):
        check_rows(logits[b].float(), u[b], np.float32(T[b]), k[b], np.float32(p[b]), np.float32(q[b]), tok[b], conf[b], V)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kind", ["equal", "two", "few", "near", "signs", "lowest", "wide"])
def test_rows_with_many_equal_logits(epic, dt, kind):
    V, rng = 6007, np.random.default_rng(3)
    lowest = torch.finfo(DT[dt]).min
    row = {"equal": np.full(V, 1.5), "two": np.where(np.arange(V) % 7 == 0, 2.0, 1.0),
           "few": rng.choice([-3.0, 0.5, 0.75, 4.0], V), "near": 1.0 + rng.integers(0, 3, V) * 2.0 ** -7,
           "signs": rng.choice([0.0, -0.0, 1e-7, -1e-7], V), "lowest": np.full(V, lowest),
           "wide": rng.choice([lowest, -40.0, -20.0, 0.0, 12.0], V)}[kind]
    B = len(SETTINGS) + 3
    T, k, p, q = zip(*(SETTINGS + [(1.0, 2000, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (1.0, 1, 1.0, 0.0)]))
    logits = torch.from_numpy(np.broadcast_to(row, (B, 3, V)).astype(np.float32)).to(DEV, DT[dt]).contiguous()
    u = rng.random((B, 3)).astype(np.float32)
    tok, conf = run(epic, logits, u=u, T=T, k=k, p=p, q=q)
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    for b in range(B):
        for i in range(3):
            l = logits[b, i].float().cpu().numpy()
            e = torch.exp2(torch.from_numpy(R.exponents(l, np.float32(T[b]))).to(DEV)).cpu().numpy()
            want = R.draw(l, e, float(u[b, i]), np.float32(T[b]), k[b], np.float32(p[b]), np.float32(q[b]))
            assert tok[b, i] == want[0] and abs(conf[b, i] - want[1]) <= 4e-7 * want[1], (b, i, want)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_lists_with_equal_or_adjacent_tokens(epic, dt):
    """A few hundred tokens in reach of the filters: many of them equal, or
    all of adjacent ids in a long row."""
    rng = np.random.default_rng(17)
    equal = np.full(3000, -30.0)
    at = rng.permutation(3000)[:230]
    equal[at[:50]] = 3.0 + 0.125 * rng.integers(0, 8, 50)
    equal[at[50:200]] = 2.5
    equal[at[200:]] = 2.25
    long = np.full(131072, -40.0)
    long[70000:70300] = 2.0 + 0.25 * rng.integers(0, 9, 300)
    combos = [(1.0, k, p, q) for k, p, q in [(40, 1.0, 0.0), (80, 1.0, 0.0), (120, 0.9, 0.0), (200, 0.5, 0.0), (210, 0.99, 0.0),
                                             (230, 1.0, 0.3), (260, 0.7, 0.0), (0, 0.6, 0.0), (0, 0.97, 0.0), (0, 1.0, 0.2)]]
    T, k, p, q = zip(*combos)
    for l in (equal, long):
        logits = on(l, torch.float32).to(DT[dt]).expand(len(combos), 4, len(l))
        u = rng.random((len(combos), 4)).astype(np.float32)
        tok, conf = run(epic, logits, u=u, T=T, k=k, p=p, q=q)
        tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
        row = logits[0, 0].float().cpu().numpy()
        e = torch.exp2(torch.from_numpy(R.exponents(row, np.float32(1.0))).to(DEV)).cpu().numpy()
        for b, i in np.ndindex(*u.shape):
            want = R.draw(row, e, float(u[b, i]), np.float32(1.0), k[b], np.float32(p[b]), np.float32(q[b]))
            assert tok[b, i] == want[0] and abs(conf[b, i] - want[1]) <= 4e-7 * want[1], (len(l), combos[b], i, want)


def test_rows_without_a_choice(epic):
    V = 300
    logits = torch.zeros((1, 6, V), device=DEV)
    logits[0, 0] = -math.inf
    logits[0, 1] = math.nan
    logits[0, 2, 7] = math.inf
    logits[0, 3] = -math.inf
    logits[0, 3, 211] = -5.0  # one token left
    logits[0, 4, ::2] = math.nan  # not tokens: the others are
    for T, k, p in ((1.0, 0, 1.0), (0.0, 0, 1.0), (1.0, 5, 0.5)):
        tok, conf = run(epic, logits, T=T, k=k, p=p)
        tok, conf = tok.cpu().numpy()[0], conf.cpu().numpy()[0]
        assert list(tok[:4]) == [-1, -1, -1, 211] and list(conf[:3]) == [0, 0, 0]
        assert conf[3] == 1.0 and tok[4] % 2 == 1 and abs(conf[4] - 2 / V) < 1e-6 / V
    tok, conf = run(epic, logits, T=math.nan)
    assert (tok == -1).all() and (conf == 0).all()


def test_settings_at_their_ends(epic):
    """Every combination bit for bit: probabilities of 0 and 1, NaN, temperatures
    from tiny to infinite, numbers at and past the ends of [0, 1)."""
    V, rng = 777, np.random.default_rng(6)
    l = (2 * rng.standard_normal(V)).astype(np.float32)
    us = [0.0, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, math.nan, 2.0 ** -24, 0.25]
    combos = [(T, k, p, q) for T in (1e-30, 0.05, 1.0, 1e4, math.inf, -1.0) for k, p, q in
              [(0, 0.0, 0.0), (0, -1.0, 0.0), (0, math.nan, math.nan), (0, 2.0, -1.0), (V, 1.0, 1.0), (V + 5, 1.0, 3.0),
               (-3, 2.0 ** -24, 0.0), (3, 1 - 2.0 ** -24, 1e-9), (V - 1, 1.0, 0.0), (1, 0.0, 0.0)]]
    logits = on(l, torch.float32).expand(len(combos), len(us), V)  # a broadcast row
    T, k, p, q = zip(*combos)
    tok, conf = run(epic, logits, u=np.broadcast_to(us, (len(combos), len(us))), T=T, k=k, p=p, q=q)
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    for b, (T, k, p, q) in enumerate(combos):
        T, p, q = np.float32(T), np.float32(p), np.float32(q)
        e = torch.exp2(torch.from_numpy(R.exponents(l, T)).to(DEV)).cpu().numpy()
        for i, u in enumerate(us):
            want = R.draw(l, e, u, T, k, p, q)
            assert tok[b, i] == want[0] and abs(conf[b, i] - want[1]) <= 4e-7 * want[1], (T, k, p, q, u, want)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_masks_of_the_lowest_value_at_huge_temperatures(epic, dt):
    """There they weigh as much as the others, and count for every filter."""
    V, rng = 700, np.random.default_rng(12)
    l = np.full(V, torch.finfo(DT[dt]).min)
    l[rng.permutation(V)[:5]] = [0.0, 1.0, 2.0, 3.0, -1.0]
    combos = [(T, k, p, q) for T in (1e38, math.inf) for k, p, q in
              [(0, 1.0, 0.0), (50, 1.0, 0.0), (500, 1.0, 0.0), (0, 0.5, 0.0), (60, 0.9, 0.0), (0, 1.0, 0.01)]]
    us = np.array([0.0, 0.3, 0.7, 1 - 2.0 ** -24])
    logits = on(l, torch.float32).to(DT[dt]).expand(len(combos), len(us), V)
    T, k, p, q = zip(*combos)
    tok, conf = run(epic, logits, u=np.broadcast_to(us, (len(combos), len(us))), T=T, k=k, p=p, q=q)
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    row = logits[0, 0].float().cpu().numpy()
    for b, (T, k, p, q) in enumerate(combos):
        T, p, q = np.float32(T), np.float32(p), np.float32(q)
        e = torch.exp2(torch.from_numpy(R.exponents(row, T)).to(DEV)).cpu().numpy()
        for i, u in enumerate(us):
            want = R.draw(row, e, u, T, k, p, q)
            assert tok[b, i] == want[0] and abs(conf[b, i] - want[1]) <= 4e-7 * want[1], (T, k, p, q, u, want)


def test_windows_and_masks(epic):
    """Only masked positions inside the sequence count; what the others hold is
    not looked at."""
    B, n, m, V = 5, 40, 16, 900
    rng = np.random.default_rng(2)
    seqs = rng.integers(0, 50, (B, n)).astype(np.int32)
    seqs[rng.random((B, n)) < 0.5] = -1
    seqs[2] = 3  # nothing masked
    start = np.array([0, 24, 5, 30, -4], np.int32)  # past the end, before the beginning
    logits = torch.from_numpy(rng.standard_normal((B, m, V)).astype(np.float32)).to(DEV)
    at = start[:, None] + np.arange(m)
    inside = (at >= 0) & (at < n)
    counts = inside & (np.take_along_axis(seqs, at.clip(0, n - 1), 1) == -1)
    assert counts.any() and not counts[2].any()
    logits[on(~counts, torch.bool)] = math.nan
    u = rng.random((B, m)).astype(np.float32)
    tok, conf = run(epic, logits, on(seqs, torch.int32), u=u, T=0.8, k=40, start=on(start, torch.int32))
    tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
    assert (tok[~counts] == -1).all() and (conf[~counts] == 0).all() and (tok[counts] >= 0).all()
    for b, i in zip(*np.nonzero(counts)):
        check_rows(logits[b, i:i + 1], u[b, i:i + 1], np.float32(0.8), 40, 1.0, 0.0, tok[b, i:i + 1], conf[b, i:i + 1], V)


@pytest.mark.parametrize("dt,B,m,V", [("bf16", 3, 100, 40001), ("bf16", 300, 1, 140001), ("f32", 7, 37, 40001), ("f16", 1, 2048, 33001),
                                      ("f16", 1, 2049, 33001), ("f16", 1, 1500, 60001)])
def test_long_rows_of_which_some_count(epic, dt, B, m, V):
    """The same tokens as a call on these rows alone, and no others touched."""
    rng = np.random.default_rng(V + m)
    logits = torch.randn((B, m, V), device=DEV, generator=torch.Generator(DEV).manual_seed(V)).to(DT[dt])
    u = rng.random((B, m)).astype(np.float32)
    for masked in (0.0, 0.07, 0.9, 1.0):
        seqs = np.where(rng.random((B, m + 3)) < masked, -1, 9).astype(np.int32)
        counts = seqs[:, :m] == -1
        tok, conf = run(epic, logits, on(seqs, torch.int32), u=u, T=0.9, k=100, p=0.9)
        tok, conf = tok.cpu().numpy(), conf.cpu().numpy()
        assert (tok[~counts] == -1).all() and (conf[~counts] == 0).all()
        rows = np.flatnonzero(counts.reshape(-1))[:200]  # at most 200: a call whose rows stay where they are
        if len(rows):
            some = logits.view(-1, V)[on(rows, torch.int64)][None]
            one = run(epic, some, u=u.reshape(1, -1)[:, rows], T=0.9, k=100, p=0.9)
            assert (one[0][0].cpu().numpy() == tok.reshape(-1)[rows]).all()
            assert (one[1][0].cpu().numpy() == conf.reshape(-1)[rows]).all()
        assert (tok[counts] >= 0).all()


def test_a_row_draws_the_same_in_any_batch(epic):
    V, rng = 5003, np.random.default_rng(4)
    logits = torch.from_numpy((2 * rng.standard_normal((6, 9, V))).astype(np.float32)).to(DEV, torch.bfloat16)
    u = rng.random((6, 9)).astype(np.float32)
    kw = dict(T=0.9, k=800, p=0.9, q=0.001)
    tok, conf = run(epic, logits, u=u, **kw)
    again = run(epic, logits, u=u, **kw)
    assert torch.equal(tok, again[0]) and torch.equal(conf, again[1])
    for b, i in ((0, 0), (3, 7), (5, 8)):
        one = run(epic, logits[b:b + 1, i:i + 1], u=u[b:b + 1, i:i + 1], **kw)
        assert one[0].item() == tok[b, i].item() and one[1].item() == conf[b, i].item()
    turned = logits.transpose(0, 1).contiguous().transpose(0, 1)  # another order of rows in memory
    other = run(epic, turned, u=u, **kw)
    assert torch.equal(tok, other[0]) and torch.equal(conf, other[1])


def test_rows_past_32_bit_offsets(epic):
    V, far = 1000, 2 ** 32 + 11
    base = torch.empty(far + 2 * V, dtype=torch.bfloat16, device=DEV)
    logits = base.as_strided((2, 1, V), (far, V, 1))
    rows = torch.from_numpy(np.random.default_rng(1).standard_normal((2, 1, V)).astype(np.float32)).to(DEV)
    logits.copy_(rows)
    tok, conf = run(epic, logits, T=1.0, k=20)
    near = run(epic, logits.contiguous(), T=1.0, k=20)
    assert torch.equal(tok, near[0]) and torch.equal(conf, near[1])


def test_other_stream_and_graph(epic):
    V, rng = 3000, np.random.default_rng(9)
    logits = torch.from_numpy(rng.standard_normal((4, 8, V)).astype(np.float32)).to(DEV)
    u = torch.from_numpy(rng.random((4, 8)).astype(np.float32)).to(DEV)
    k = torch.full((4,), 30, dtype=torch.int32, device=DEV)
    outs = [torch.zeros((4, 8), dtype=torch.int32, device=DEV), torch.zeros((4, 8), device=DEV)]
    cand = [torch.zeros(4 * 5, dtype=torch.int32, device=DEV) for _ in range(3)] + [torch.zeros(4 * 5, device=DEV)]
    off = torch.zeros(5, dtype=torch.int32, device=DEV)

    def step():
        epic.sample(logits, None, u, *outs, top_k=k)
        epic.propose(*outs, 5, *cand, off)

    def eager():
        step()
        torch.cuda.synchronize()
        return [t.clone() for t in outs + cand + [off]]

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
    side.synchronize()
    first = [t.clone() for t in outs + cand + [off]]
    assert all(torch.equal(a, b) for a, b in zip(first, eager()))
    with torch.cuda.graph(graph, stream=side):
        step()
    for turn in range(4):
        logits.copy_(torch.from_numpy(np.random.default_rng(turn).standard_normal((4, 8, V)).astype(np.float32)))
        u.copy_(torch.from_numpy(np.random.default_rng(turn + 50).random((4, 8)).astype(np.float32)))
        want = eager()
        for t in outs + cand + [off]:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs + cand + [off])), turn


# ------------------------------------------------------------------ proposals
def plain_propose(tok, conf, start, P):
    rows, off = [], [0]
    for b in range(len(tok)):
        at = [i for i in range(tok.shape[1]) if tok[b, i] >= 0 and not np.isnan(conf[b, i])]
        at.sort(key=lambda i: (-conf[b, i], i))
        rows += [(b, (0 if start is None else start[b]) + i, tok[b, i], conf[b, i]) for i in at[:P]]
        off.append(len(rows))
    return rows + [(-1, -1, -1, 0.0)] * (len(tok) * P - len(rows)), off


@pytest.mark.parametrize("B,m,P", [(1, 1, 1), (3, 7, 64), (4, 64, 3), (2, 65, 16), (5, 1024, 16), (1, 3001, 64),
                                   (256, 33, 2), (257, 70, 5), (1500, 130, 64)])
def test_propose(epic, B, m, P):
    rng = np.random.default_rng(B * m + P)
    tok = np.where(rng.random((B, m)) < 0.6, rng.integers(0, 9999, (B, m)), -1).astype(np.int32)
    conf = (rng.integers(0, 12, (B, m)) / 12).astype(np.float32)  # ties
    conf[rng.random((B, m)) < 0.02] = np.nan
    conf[rng.random((B, m)) < 0.02] = np.inf
    conf[rng.random((B, m)) < 0.02] = -np.inf
    conf[rng.random((B, m)) < 0.02] = -0.0
    if B > 2:
        tok[1] = -1  # a sequence without proposals
    start = rng.integers(0, 500, B).astype(np.int32) if B != 4 else None
    cand = [torch.full((B * P,), 77, dtype=torch.int32, device=DEV) for _ in range(3)]
    cand.append(torch.full((B * P,), 77.0, device=DEV))
    off = torch.full((B + 1,), 77, dtype=torch.int32, device=DEV)
    epic.propose(on(tok, torch.int32), on(conf, torch.float32), P, *cand, off,
                 start=None if start is None else on(start, torch.int32))
    want, woff = plain_propose(tok, conf, start, P)
    assert off.tolist() == woff
    got = list(zip(*(c.tolist() for c in cand)))
    assert got == [(int(a), int(b), int(c), float(d)) for a, b, c, d in want]


def test_propose_feeds_the_check(epic):
    """Sampled tokens as candidates of validate: a verdict of 0 or 1 for each
    candidate, no error flag."""
    from paper_2606_00722_amd import workloads as W
    from tests import gpu_util

    inst = W.make_instance(1, 42)
    V = inst.vocab.size
    g = gpu_util.Gpu(W.arrays(inst.lang, inst.vocab), inst.B, inst.n, 64)
    rng = np.random.default_rng(0)
    l = rng.standard_normal((inst.B, inst.n, V)).astype(np.float32)
    np.put_along_axis(l, inst.hidden[:, :, None], 9.0, 2)
    seqs = on(inst.seqs, torch.int32)
    tok, conf = run(epic, on(l, torch.float32), seqs, u=rng.random((inst.B, inst.n)), T=0.8, p=0.95)
    cand = [torch.empty(inst.B * 8, dtype=torch.int32, device=DEV) for _ in range(3)]
    cand.append(torch.empty(inst.B * 8, device=DEV))
    off = torch.empty(inst.B + 1, dtype=torch.int32, device=DEV)
    epic.propose(tok, conf, 8, *cand, off)
    C = int(off[-1])
    assert C == inst.B * 8
    verdict = g.validate(inst.seqs, *(c[:C].cpu().numpy() for c in cand[:3]))
    assert g.errors() == 0 and set(verdict.tolist()) <= {0, 1} and verdict.sum() > 0


# ------------------------------------------------------------------- refusals
def test_refusals(epic):
    B, m, V = 2, 3, 50
    logits = torch.zeros((B, m, V), device=DEV)
    seqs = torch.full((B, m), -1, dtype=torch.int32, device=DEV)
    u, tok, conf = torch.zeros((B, m), device=DEV), torch.zeros((B, m), dtype=torch.int32, device=DEV), torch.zeros((B, m), device=DEV)

    def bad(f):
        with pytest.raises(ValueError):
            f()

    bad(lambda: epic.sample(logits[0], seqs, u, tok, conf))
    bad(lambda: epic.sample(logits.double(), seqs, u, tok, conf))
    bad(lambda: epic.sample(logits.cpu(), seqs, u, tok, conf))
    bad(lambda: epic.sample(logits.transpose(1, 2), seqs, u, tok, conf))
    bad(lambda: epic.sample(logits, seqs.long(), u, tok, conf))
    bad(lambda: epic.sample(logits, seqs[:1], u, tok, conf))
    bad(lambda: epic.sample(logits, seqs, u.double(), tok, conf))
    bad(lambda: epic.sample(logits, seqs, None, tok, conf))
    bad(lambda: epic.sample(logits, seqs, u, tok.float(), conf))
    bad(lambda: epic.sample(logits, seqs, u, tok, conf.t().contiguous().t()))
    bad(lambda: epic.sample(logits, seqs, u, tok, conf, top_k=torch.zeros(B + 1, dtype=torch.int32, device=DEV)))
    bad(lambda: epic.sample(logits, seqs, u, tok, conf, top_p=torch.zeros(B, device="cpu")))
    c = [torch.zeros(B * 4, dtype=torch.int32, device=DEV) for _ in range(3)] + [torch.zeros(B * 4, device=DEV)]
    off = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    bad(lambda: epic.propose(tok, conf, 4, *c, off[:B]))
    bad(lambda: epic.propose(tok, conf, 5, *c, off))
    bad(lambda: epic.propose(tok.float(), conf, 4, *c, off))
    big = [torch.zeros(B * 65, dtype=torch.int32, device=DEV) for _ in range(3)] + [torch.zeros(B * 65, device=DEV)]
    for P, arrays in ((65, big), (0, [t[:0] for t in c])):
        with pytest.raises(epic.EpicError) as e:
            epic.propose(tok, conf, P, *arrays, off)
        assert e.value.code == -2
    with pytest.raises(epic.EpicError) as e:
        epic.sample(torch.zeros((1, 1, 262145), device=DEV), None, u[:1, :1].contiguous(), tok[:1, :1].contiguous(),
                    conf[:1, :1].contiguous())
    assert e.value.code == -9


def test_empty_batches(epic):
    i32 = dict(dtype=torch.int32, device=DEV)
    for B, m in ((0, 4), (3, 0)):
        epic.sample(torch.zeros((B, m, 9), device=DEV), None, torch.zeros((B, m), device=DEV), torch.zeros((B, m), **i32),
                    torch.zeros((B, m), device=DEV))
        off = torch.full((B + 1,), 5, **i32)
        cand = [torch.zeros(B * 2, **i32) for _ in range(3)] + [torch.ones(B * 2, device=DEV)]
        epic.propose(torch.zeros((B, m), **i32), torch.zeros((B, m), device=DEV), 2, *cand, off)
        assert off.tolist() == [0] * (B + 1) and cand[0].tolist() == [-1] * (2 * B) and cand[3].tolist() == [0.0] * (2 * B)
