"""The operators between hidden states and logits against plain implementations:
cross entropy and its gradients in 64 bits, 8-bit rows and logits bit for bit.

Tolerances (u16: half a step of the 16-bit type, u32 = 2^-24).  A logit is a sum
of d products: with n roundings of at most u32 of the terms' magnitudes A the
error is taken as 8 sqrt(n) u32 A (eight deviations of n independent ones);
float32 inputs add what their two 16-bit parts leave out, 2^-22 A.  exp2's
argument x log2(e) is rounded relative to |x| <= 60 (u32 * 60 * 1.5), exp2 and
log to a few u32, and a sum over the vocabulary adds 100 roundings: 2e-5 in all.
Gradients: every G is off by its logit's error and lse's, and by u16 from its own
rounding (float32: 2^-22); float16 rounds its rows' weights' powers of two
exactly.  The sums of G W and G h over V or N terms as above, the result is
rounded once more."""
import math

import numpy as np
import pytest

from tests import head_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U32 = 2.0 ** -24
DT = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
U = {"float32": 2.0 ** -22, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic as E

    E.lib()
    return E


def strided(shape, pad, dtype, gen, scale=1.0):
    """Random rows with `pad` numbers between them that are NaN."""
    full = torch.full((*shape[:-1], shape[-1] + pad), float("nan"), dtype=dtype)
    full[..., : shape[-1]] = (scale * torch.randn(shape, generator=gen)).to(dtype)
    return full


def cut(t, d, dev="cuda:0"):
    return t.to(dev)[..., :d]


class Case:
    def __init__(self, dtype, B, m, V, d, pad=0, share=0.6, window=False, weights="some", seed=0):
        self.B, self.m, self.V, self.d, self.dtype = B, m, V, d, dtype
        g = torch.Generator().manual_seed(1000 * seed + 7 * V + d)
        rng = np.random.default_rng(seed + V)
        self.n = m + 9 if window else m
        seqs = np.where(rng.random((B, self.n)) < share, -1, 4).astype(np.int32)
        seqs[0, :] = -1
        self.start = rng.integers(-3, self.n - m + 4, size=B).astype(np.int32) if window else None
        self.seqs = seqs
        self.target = torch.randint(0, V, (B, m), generator=g).to(torch.int32)
        self.target[rng.random((B, m)) < 0.2] = -1
        self.target[0, 0] = min(3, V - 1)
        self.on = head_ref.counted(B, m, seqs, self.start, self.target)
        self.full_h = strided((B, m, d), pad, DT[dtype], g)
        self.full_h[~torch.from_numpy(self.on)] = float("nan")  # rows that do not count are not read
        self.full_w = strided((V, d), pad, DT[dtype], g, 2 / math.sqrt(d))
        self.h, self.w = cut(self.full_h, d, "cpu"), cut(self.full_w, d, "cpu")
        w = torch.randn((B, m), generator=g)
        if weights == "far":  # over sixty powers of two, signs, and zeros
            w = w * torch.exp2(torch.randint(-40, 20, (B, m), generator=g).float())
            w[rng.random((B, m)) < 0.2] = 0
        self.weight = None if weights is None else w

    def on_gpu(self):
        to = lambda a: None if a is None else (torch.from_numpy(a) if isinstance(a, np.ndarray) else a).to("cuda:0")  # noqa: E731
        return cut(self.full_h, self.d), to(self.seqs), cut(self.full_w, self.d), to(self.target), to(self.start), to(self.weight)


def forward(epic, c, ws=None):
    h, seqs, w, y, start, _ = c.on_gpu()
    loss, lse = (torch.full((c.B, c.m), 7.0, device="cuda:0") for _ in range(2))
    if ws is None:
        ws = epic.alloc_head_loss_workspace(h, w)
        ws.fill_(255)  # NaN, whatever is read as
    epic.head_loss_forward(h, seqs, w, y, loss, lse, ws, start=start)
    return loss, lse


def backward(epic, c, lse, hidden=True, head=True, pad=0):
    h, seqs, w, y, start, weight = c.on_gpu()
    dt = DT[c.dtype]
    gh = torch.full((c.B, c.m, c.d + pad), 7.0, dtype=dt, device="cuda:0")
    gw = torch.full((c.V, c.d + pad), 7.0, dtype=dt, device="cuda:0")
    ws = epic.alloc_head_loss_workspace(h, w)
    ws.fill_(255)
    epic.head_loss_backward(h, seqs, w, y, lse, weight, gh[..., : c.d] if hidden else None, gw[..., : c.d] if head else None, ws, start=start)
    torch.cuda.synchronize()
    assert bool((gh[..., c.d:] == 7).all()) and bool((gw[..., c.d:] == 7).all())
    return gh[..., : c.d].cpu(), gw[..., : c.d].cpu()


def logit_error(c):
    """Bound of the logits' errors (and of lse's, but for 2e-5)."""
    on = torch.from_numpy(c.on)
    if not bool(on.any()):
        return 0.0
    A = float((c.h[on].double().abs() @ c.w.double().abs().t()).max())
    return (8 * math.sqrt(c.d) * U32 + (2.0 ** -22 if c.dtype == "float32" else 0.0)) * A


def check(epic, c, pad=0):
    loss, lse = forward(epic, c)
    want = head_ref.loss(c.h, c.w, c.target, c.on, c.weight)
    e = logit_error(c) + 2e-5
    assert float((lse.cpu() - want[1]).abs().max()) <= e
    assert float((loss.cpu() - want[0]).abs().max()) <= 2 * e
    assert bool((loss.cpu()[~torch.from_numpy(c.on)] == 0).all()) and bool((lse.cpu()[~torch.from_numpy(c.on)] == 0).all())
    gh, gw = backward(epic, c, lse, pad=pad)
    _, _, want_h, want_w, size_h, size_w = head_ref.loss(c.h, c.w, c.target, c.on, c.weight, lse.cpu())
    u = U[c.dtype]
    tiny = {"float32": 1e-37, "float16": 2.0 ** -25, "bfloat16": 1e-37}[c.dtype]  # half a step of subnormal numbers
    # exp(l - lse) and expm1 are off by their argument's error, of G or (next to p = 1) of 1
    off = 2 * e
    for got, exact, size, terms, extra in (
            (gh, want_h, size_h, c.V, extra_h(c, off)), (gw, want_w, size_w, c.B * c.m, extra_w(c, off))):
        bound = size * (u + 8 * math.sqrt(terms) * U32) + extra + exact.abs() * u + tiny
        # past the type's largest number M the rounded result is infinite: an exact value of at least M + half a
        # step, and with what the sums are off by any within `bound` of M, may be +-inf, and none smaller
        M = torch.finfo(got.dtype).max
        over = torch.isinf(got) & (got.double().sign() == exact.sign()) & (exact.abs() + bound >= M)
        bad = ~over & ~((got.double() - exact).abs() <= bound)
        assert not bool(bad.any()), (float((got.double() - exact).abs().max()), float(bound.max()), int(bad.sum()))
    return loss, lse, gh, gw


def extra_h(c, off):
    """What errors `off` of the logits put on the gradient: G's of p by p, and 1 - p by p."""
    return off * _p_sizes(c)[0]


def extra_w(c, off):
    return off * _p_sizes(c)[1] + weights_left_out(c)


def weights_left_out(c):
    """float16 rows are multiplied with their weights' powers of two relative to
    the largest: subnormal numbers' half steps, 2^-25, times that (float32: two
    parts, 2^-40 of the largest row)."""
    if c.dtype == "bfloat16":
        return 0.0
    w = 1.0 if c.weight is None else float(c.weight.abs().max())
    on = torch.from_numpy(c.on)
    rows = int(on.sum())
    top = float(c.h[on].abs().max()) if rows else 0.0
    return 2 * w * rows * (2.0 ** -25 if c.dtype == "float16" else 2.0 ** -38 * top)


def _p_sizes(c):
    """Sums of |weight| p |W| and |weight| p |h|."""
    h, w = c.h.double(), c.w.double()
    a, b = torch.zeros_like(h), torch.zeros_like(w)
    for x, i in zip(*np.nonzero(c.on)):
        if int(c.target[x, i]) >= c.V:
            continue
        p = torch.softmax(w @ h[x, i], 0) * (1.0 if c.weight is None else abs(float(c.weight[x, i])))
        a[x, i] = p @ w.abs()
        b += p[:, None] * h[x, i].abs()
    return a, b


SIZES = [  # B, m, V, d, pad, window
    (1, 1, 1, 1, 0, False), (1, 1, 2, 3, 1, False), (1, 3, 63, 64, 0, False), (2, 5, 64, 65, 3, True),
    (1, 17, 257, 63, 0, True), (3, 11, 300, 128, 8, False), (2, 64, 256, 64, 0, False), (2, 65, 1025, 127, 1, True),
    (5, 33, 640, 320, 0, True), (2, 40, 257, 72, 0, False), (3, 33, 1003, 136, 8, True), (2, 70, 514, 1000, 0, False), (1, 9, 67, 64, 0, False),
    (2, 33, 130, 120, 8, False)]


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_loss_and_gradients(dtype, size, epic):
    B, m, V, d, pad, window = size
    check(epic, Case(dtype, B, m, V, d, pad, window=window), pad=pad)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("weights", [None, "far"])
def test_weights(dtype, weights, epic):
    check(epic, Case(dtype, 2, 40, 200, 96, weights=weights, seed=1))


@pytest.mark.parametrize("dtype,size", [("bfloat16", (2, 150, 70001, 64, 0)), ("float16", (3, 300, 20032, 192, 0)),
                                        ("float32", (2, 300, 28001, 100, 1)), ("bfloat16", (1, 520, 33000, 320, 2))], ids=str)
def test_large(dtype, size, epic):
    """More than one piece of the vocabulary, and the large tiles."""
    B, m, V, d, pad = size
    c = Case(dtype, B, m, V, d, pad, share=0.15, seed=2)
    c.seqs[0, m // 3:] = 1  # some tens of rows that count, over several tiles' range
    c.on = head_ref.counted(B, m, c.seqs, None, c.target)
    check(epic, c)


MANY = [(8, 150, 1500, 192, 0.8), (4, 250, 20096, 256, 0.9), (6, 1000, 30016, 192, 0.3), (4, 64, 20032, 64, 0.5), (2, 64, 9024, 448, 0.9),
        (9, 700, 26000, 72, 0.95), (3, 100, 4992, 1088, 1.0), (4, 700, 20011, 264, 0.9), (2, 300, 9999, 1032, 0.9), (2, 90, 30001, 200, 0.8)]
MANY = [(dt, size) for size in MANY for dt in sorted(DT)]
# a head that is written out in pieces for the losses too; the largest vocabulary and width; a great many rows
MANY += [("bfloat16", (1, 90, 70001, 1999, 0.5)), ("float32", (1, 70, 40000, 1990, 0.9)), ("bfloat16", (1, 20, 262144, 64, 1.0)),
         ("float32", (1, 20, 262144, 64, 1.0)), ("float16", (1, 5, 100, 65536, 1.0)), ("float32", (1, 5, 100, 65536, 1.0)),
         ("bfloat16", (3, 100000, 40, 16, 0.5)), ("float32", (2, 50000, 70, 24, 0.5))]


@pytest.mark.parametrize("dtype,size", MANY, ids=str)
def test_many_rows(dtype, size, epic):
    """More rows that count than a tile has, every size of tile, several pieces of
    the vocabulary and slices of them, by sums over all rows on the GPU in 64 bits."""
    B, m, V, d, share = size
    c = Case(dtype, B, m, V, d, share=share, seed=3, weights="some")
    loss, lse = forward(epic, c)
    gh, gw = backward(epic, c, lse)
    on = torch.from_numpy(c.on)
    h, w, y = c.h[on].double().cuda(), c.w.double().cuda(), c.target[on].long().cuda()
    l = h @ w.t()
    e = logit_error(c) + 2e-5
    want = torch.logsumexp(l, -1)
    assert float((lse.cuda()[on.cuda()] - want).abs().max()) <= e
    p = torch.exp(l - lse[on.cuda()].double()[:, None]).scatter_add_(1, y[:, None], torch.full((len(y), 1), -1.0, dtype=torch.float64, device="cuda"))
    G = p * c.weight[on].double().cuda()[:, None]
    u = U[c.dtype]
    P = torch.softmax(l, -1) * c.weight[on].double().cuda().abs()[:, None]
    # (2^-25: half a step of float16's smallest numbers)
    bound = (G.abs() @ w.abs()) * (u + 8 * math.sqrt(V) * U32) + 2 * e * (P @ w.abs()) + (G @ w).abs() * u + 2.0 ** -25
    assert bool(((gh[on].cuda().double() - G @ w).abs() <= bound).all())
    bound = (G.abs().t() @ h.abs()) * (u + 8 * math.sqrt(len(y)) * U32) + 2 * e * (P.t() @ h.abs()) + (G.t() @ h).abs() * u
    assert bool(((gw.cuda().double() - G.t() @ h).abs() <= bound + weights_left_out(c) + 2.0 ** -25).all())
    assert not bool(gh[~on].any())


@pytest.mark.parametrize("dtype", sorted(DT))
def test_no_row_counts(dtype, epic):
    c = Case(dtype, 2, 5, 70, 40)
    c.seqs[:] = 3
    c.on[:] = False
    loss, lse = forward(epic, c)
    assert not bool(loss.any()) and not bool(lse.any())
    gh, gw = backward(epic, c, lse)
    assert not bool(gh.any()) and not bool(gw.any())


def test_no_rows_at_all(epic):
    """A batch without sequences has a head's gradient, which is 0."""
    h, w = torch.zeros((0, 4, 64), device="cuda"), torch.ones((70, 64), device="cuda")
    seqs, y = (torch.zeros((0, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    f = torch.zeros((0, 4), device="cuda")
    ws = epic.alloc_head_loss_workspace(h, w)
    epic.head_loss_forward(h, seqs, w, y, f, f, ws)
    gw = torch.ones_like(w)
    epic.head_loss_backward(h, seqs, w, y, f, None, None, gw, ws)
    assert not bool(gw.any())


@pytest.mark.parametrize("dtype", sorted(DT))
def test_tokens_outside_the_vocabulary(dtype, epic):
    c = Case(dtype, 2, 6, 90, 48, share=1.0)
    c.target[0, 1], c.target[1, 2] = c.V, 2 ** 31 - 1
    c.on = head_ref.counted(c.B, c.m, c.seqs, None, c.target)
    loss, lse = forward(epic, c)
    assert torch.isnan(loss.cpu()[0, 1]) and torch.isnan(loss.cpu()[1, 2]) and int(torch.isnan(loss).sum()) == 2
    assert bool(torch.isfinite(lse).all())
    gh, gw = backward(epic, c, lse)
    assert not bool(gh[0, 1].any()) and not bool(gh[1, 2].any()) and bool(torch.isfinite(gw.float()).all())
    part = Case(dtype, 2, 6, 90, 48, share=1.0)
    part.target[0, 1] = part.target[1, 2] = -1
    part.on = head_ref.counted(part.B, part.m, part.seqs, None, part.target)
    _, gw2 = backward(epic, part, forward(epic, part)[1])
    want = head_ref.loss(c.h, c.w, c.target, c.on, c.weight, lse.cpu())
    assert torch.allclose(gw.float(), gw2.float(), rtol=4 * U[dtype], atol=float(want[5].max()) * 2 * U[dtype])


@pytest.mark.parametrize("rows", [90, 1100])
@pytest.mark.parametrize("dtype", sorted(DT))
def test_weight_of_a_row_that_adds_nothing(dtype, rows, epic):
    """However large it is, the others' gradients are those without the row."""
    c = Case(dtype, 1, rows, 70, 40, share=1.0, seed=6)
    c.target[0, rows - 5] = c.V
    c.full_h[0, rows - 5] = 1.0
    c.weight[0, rows - 5] = 1e30
    c.on = head_ref.counted(1, rows, c.seqs, None, c.target)
    _, lse = forward(epic, c)
    gh, gw = backward(epic, c, lse)
    c.weight[0, rows - 5] = 0
    gh2, gw2 = backward(epic, c, lse)
    assert torch.equal(gh, gh2) and torch.equal(gw, gw2) and bool(gw.any())


@pytest.mark.parametrize("dtype", sorted(DT))
def test_not_a_number_stays_in_its_row(dtype, epic):
    c = Case(dtype, 2, 8, 100, 64, share=1.0)
    c.target[:] = c.target.clamp(min=0)
    c.on = head_ref.counted(c.B, c.m, c.seqs, None, c.target)
    c.full_h[0, 2, 5] = float("nan")
    c.full_h[1, 3, 7] = float("inf")
    loss, lse = forward(epic, c)
    # (rows that had no token at first are NaN too, and count now)
    bad = ~torch.isfinite(c.h).all(-1)
    assert bad[0, 2] and bad[1, 3] and 2 <= int(bad.sum()) < 10
    assert torch.equal(torch.isnan(loss.cpu()), bad)
    gh, gw = backward(epic, c, lse)
    assert bool(torch.isnan(gh[bad]).all()) and bool(torch.isfinite(gh[~bad]).all())
    c.full_h[bad] = 0.5
    c.full_w[7, 1] = float("nan")
    loss, _ = forward(epic, c)
    assert bool(torch.isnan(loss).all())


@pytest.mark.parametrize("dtype", sorted(DT))
def test_sure_tokens(dtype, epic):
    """Probabilities next to 1: the gradient keeps what 1 - p has."""
    c = Case(dtype, 1, 8, 50, 64, share=1.0, weights=None)
    c.target[:] = torch.arange(8).to(torch.int32)
    c.on = head_ref.counted(1, 8, c.seqs, None, c.target)
    c.full_w[:, :64] = 0
    c.full_w[torch.arange(50), torch.arange(50)] = 1
    c.full_h[0, :, :64] = 0
    c.full_h[0, torch.arange(8), torch.arange(8)] = torch.tensor([4.0, 8, 10, 12, 14, 20, 30, 60]).to(DT[dtype])
    loss, lse = forward(epic, c)
    want = head_ref.loss(c.h, c.w, c.target, c.on)
    assert torch.allclose(loss.cpu().double(), want[0], rtol=1e-5, atol=60 * 2 * U32)
    gh, _ = backward(epic, c, lse)
    exact = head_ref.loss(c.h, c.w, c.target, c.on, None, lse.cpu())[2]
    # with the lse that it is given: G = expm1(l - lse), exact to float32
    assert torch.allclose(gh.double(), exact, rtol=3 * U[dtype], atol=2.0 ** -38 + (2.0 ** -25 if dtype == "float16" else 0))


@pytest.mark.parametrize("dtype", sorted(DT))
def test_gradient_over_the_hidden_states(dtype, epic):
    c = Case(dtype, 2, 30, 200, 64)
    _, lse = forward(epic, c)
    gh, gw = backward(epic, c, lse)
    h, seqs, w, y, start, weight = c.on_gpu()
    h = h.contiguous()
    gw2 = torch.empty_like(w)
    ws = epic.alloc_head_loss_workspace(h, w)
    epic.head_loss_backward(h, seqs, w, y, lse, weight, h, gw2, ws)
    assert torch.equal(h.cpu(), gh) and torch.equal(gw2.cpu(), gw)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_either_gradient_alone(dtype, epic):
    c = Case(dtype, 2, 30, 300, 80)
    _, lse = forward(epic, c)
    gh, gw = backward(epic, c, lse)
    only_h, untouched = backward(epic, c, lse, head=False)
    assert torch.equal(only_h, gh) and bool((untouched == 7).all())
    untouched, only_w = backward(epic, c, lse, hidden=False)
    assert torch.equal(only_w, gw) and bool((untouched == 7).all())


def test_repeated_rows(epic):
    """One row of hidden states for all (stride 0), and every row counting."""
    d, V, m = 64, 130, 9
    g = torch.Generator().manual_seed(5)
    row, w = torch.randn((1, 1, d), generator=g), torch.randn((V, d), generator=g) / 8
    h = row.cuda().expand(2, m, d)
    y = torch.arange(2 * m, dtype=torch.int32).view(2, m)
    loss, lse = torch.empty((2, m), device="cuda"), torch.empty((2, m), device="cuda")
    ws = epic.alloc_head_loss_workspace(h, w.cuda())
    epic.head_loss_forward(h, None, w.cuda(), y.cuda(), loss, lse, ws)
    l = (w.double() @ row[0, 0].double())
    want = torch.logsumexp(l, 0) - l[y.long()]
    A = float((w.double().abs() @ row[0, 0].double().abs()).max())
    assert float((loss.cpu() - want).abs().max()) <= 2 * ((8 * math.sqrt(d) * U32 + 2.0 ** -22) * A + 2e-5)


def _graph(run, eager, outs):
    """The captured call, replayed among eager work, against eager results."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for k in range(4):
        change = eager(k)
        want = [x.clone() for x in change]
        for o in outs:
            o.fill_(3)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", sorted(DT))
def test_captured(dtype, epic):
    c = Case(dtype, 3, 50, 400, 72)
    h, seqs, w, y, start, weight = c.on_gpu()
    h, w = torch.nan_to_num(h).contiguous(), w.contiguous()
    B, m, V = c.B, c.m, c.V
    loss, lse = torch.empty((B, m), device="cuda"), torch.empty((B, m), device="cuda")
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    q, s = epic.alloc_q8(V, c.d)
    logits = torch.zeros((B, m, V), device="cuda")
    ws, ws2 = epic.alloc_head_loss_workspace(h, w), epic.alloc_logits_q8_workspace(h)
    outs = [loss, lse, gh, gw, s, logits]

    def run():
        epic.head_loss_forward(h, seqs, w, y, loss, lse, ws)
        epic.head_loss_backward(h, seqs, w, y, lse, weight, gh, gw, ws)
        epic.quantize(w, q, s)
        epic.logits_q8(h, seqs, q, s, logits, ws2)

    def eager(k):
        seqs.copy_(torch.where(torch.rand((B, m), device="cuda") < 0.2 * (k + 1), -1, 3))
        h.normal_()
        logits.fill_(3)
        run()
        return outs

    _graph(run, eager, outs)


def test_on_another_stream(epic):
    c = Case("bfloat16", 2, 40, 500, 128)
    want = forward(epic, c)
    h, seqs, w, y, start, _ = c.on_gpu()
    ws = epic.alloc_head_loss_workspace(h, w)
    loss, lse = torch.empty((2, 40), device="cuda"), torch.empty((2, 40), device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    epic.head_loss_forward(h, seqs, w, y, loss, lse, ws, stream=s)
    s.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(lse, want[1])


def test_same_bits_every_time(epic):
    c = Case("bfloat16", 4, 200, 9000, 256, share=0.7)
    first = None
    for _ in range(3):
        loss, lse = forward(epic, c)
        out = [loss.cpu(), lse.cpu(), *backward(epic, c, lse)]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))


# ------------------------------------------------------------------ 8 bits


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("V,d,pad", [(1, 1, 0), (3, 127, 1), (70, 128, 0), (129, 1000, 3), (1000, 65, 0)])
def test_quantize(dtype, V, d, pad, epic):
    g = torch.Generator().manual_seed(d)
    full = strided((V, d), pad, DT[dtype], g, 3.0)
    x = full[:, :d]
    if V > 60:
        x[0] = 0
        x[1, 0] = float("nan")
        x[2, d - 1] = float("-inf")
        x[3] = torch.arange(d).to(x.dtype) % 128 / 2  # ties
        x[4] = x[4] * 2.0 ** -14
        if dtype != "float16":
            x[5] = x[5].clamp(-1, 1) * 1e-31  # below what counts
            x[6] = 1e30 * x[6]
    q, s = epic.alloc_q8(V, d)
    q.fill_(77)
    epic.quantize(full.cuda()[:, :d], q, s)
    want_q, want_s = head_ref.quantize(x)
    assert torch.equal(q.cpu()[:, :d].float(), want_q) and not bool(q[:, d:].any())
    assert torch.equal(s.cpu().nan_to_num(7e7), want_s.nan_to_num(7e7))


Q_SIZES = [(1, 1, 1, 1, 0, False), (1, 1, 200, 64, 0, False), (2, 7, 65, 129, 1, True), (3, 50, 1001, 300, 3, True),
           (2, 65, 640, 128, 0, False), (1, 1, 5000, 2100, 0, False), (4, 33, 257, 1024, 8, False)]


@pytest.mark.parametrize("dtype,out", [("float32", "float32"), ("float16", "float16"), ("bfloat16", "bfloat16"),
                                       ("bfloat16", "float32"), ("float32", "bfloat16"), ("bfloat16", "float16")])
@pytest.mark.parametrize("size", Q_SIZES, ids=str)
def test_logits(dtype, out, size, epic):
    """Bit for bit, and nothing else is written."""
    B, m, V, d, pad, window = size
    c = Case(dtype, B, m, V, d, pad, window=window)
    _logits(epic, c, out, pad)


def _logits(epic, c, out, pad=0):
    h, seqs, w, _, start, _ = c.on_gpu()
    on = head_ref.counted(c.B, c.m, c.seqs, c.start)
    hc = c.h.clone()
    if not np.array_equal(on, c.on):  # rows without a token count here
        c.full_h[torch.from_numpy(on & ~c.on)] = 0.25
        h, hc = cut(c.full_h, c.d), cut(c.full_h, c.d, "cpu")
    q, s = epic.alloc_q8(c.V, c.d)
    epic.quantize(w, q, s)
    full = torch.full((c.B, c.m, c.V + pad), 3.0, dtype=DT[out], device="cuda")
    ws = epic.alloc_logits_q8_workspace(h)
    ws.fill_(255)
    epic.logits_q8(h, seqs, q, s, full[:, :, : c.V], ws, start=start)
    torch.cuda.synchronize()
    got = full.cpu()
    keep = torch.from_numpy(on)
    want = head_ref.logits_q8(hc, q.cpu()[:, : c.d], s.cpu(), on, DT[out])
    assert torch.equal(got[keep][:, : c.V], want)
    assert bool((got[~keep] == 3).all()) and bool((got[:, :, c.V:] == 3).all())


@pytest.mark.parametrize("dtype,size", [("bfloat16", (2, 300, 40000, 64)), ("float16", (1, 520, 50021, 100)), ("float32", (3, 200, 33000, 200))], ids=str)
def test_logits_large(dtype, size, epic):
    c = Case(dtype, *size, pad=1, share=0.1, seed=4)
    c.seqs[0, 40:] = 1
    c.on = head_ref.counted(c.B, c.m, c.seqs, None, c.target)
    _logits(epic, c, dtype, 1)


def test_logits_of_rows_that_are_no_numbers(epic):
    c = Case("bfloat16", 1, 4, 40, 30, share=1.0)
    c.full_h[:] = 1.0
    c.full_h[0, 1, 3] = float("nan")
    c.full_h[0, 2] = 0
    c.full_w[5, 2] = float("inf")
    h, seqs, w, *_ = c.on_gpu()
    q, s = epic.alloc_q8(40, 30)
    epic.quantize(w, q, s)
    logits = torch.zeros((1, 4, 40), device="cuda")
    epic.logits_q8(h, None, q, s, logits, epic.alloc_logits_q8_workspace(h))
    bad = torch.isnan(logits.cpu()[0])
    assert bool(bad[1].all()) and bool(bad[:, 5].all()) and int(bad.sum()) == 40 + 3
    assert not bool(logits[0, 2, :5].any())


def test_logits_stay_whole_at_the_largest_width(epic):
    """65536 products of 127 by 127 are below 2^31."""
    d = 65536
    h, w = torch.ones((1, 2, d), device="cuda"), torch.ones((3, d), device="cuda")
    w[1] = -1
    q, s = epic.alloc_q8(3, d)
    epic.quantize(w, q, s)
    logits = torch.zeros((1, 2, 3), device="cuda")
    epic.logits_q8(h, None, q, s, logits, epic.alloc_logits_q8_workspace(h))
    one = np.float32(1) / np.float32(127)
    want = np.float32(np.float32(127 * 127 * d) * one) * one
    assert logits.cpu().tolist() == [[[float(want), -float(want), float(want)]] * 2]


def test_binding_refusals(epic):
    h, w = torch.zeros((1, 2, 64), device="cuda"), torch.zeros((9, 64), device="cuda")
    y, f = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros((1, 2), device="cuda")
    ws = epic.alloc_head_loss_workspace(h, w)
    with pytest.raises(ValueError, match="target"):
        epic.head_loss_forward(h, None, w, y.long(), f, f, ws)
    with pytest.raises(ValueError, match="head"):
        epic.head_loss_forward(h, None, h, y, f, f, ws)
    with pytest.raises(ValueError, match="workspace"):
        epic.head_loss_forward(h, None, w, y, f, f, ws.float())
    with pytest.raises(ValueError, match="adjacent"):
        epic.head_loss_forward(h, None, w.t().contiguous().t(), y, f, f, ws)
    with pytest.raises(epic.EpicError, match="capacity"):
        epic.head_loss_forward(h, None, w, y, f, f, ws[:512])
    with pytest.raises(epic.EpicError, match="range"):
        epic.head_loss_forward(h, None, w.half(), y, f, f, ws)
    with pytest.raises(epic.EpicError, match="null"):
        epic.head_loss_backward(h, None, w, y, f, None, None, None, ws)
    q, s = epic.alloc_q8(9, 64)
    logits = torch.zeros((1, 2, 9), device="cuda")
    with pytest.raises(ValueError, match="q"):
        epic.logits_q8(h, None, q[:, :64].contiguous(), s, logits, ws)
    with pytest.raises(ValueError, match="scale"):
        epic.logits_q8(h, None, q, s[:8], logits, ws)
    with pytest.raises(epic.EpicError, match="range"):
        epic.logits_q8(h, None, q, s, torch.zeros((1, 1, 9), device="cuda").expand(1, 2, 9), ws)
