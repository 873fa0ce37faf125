"""epic_distill_forward and epic_distill_backward through the binding, against
the divergence and its gradient in 64 bits."""
import math

import numpy as np
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # of rounding a gradient to nearest
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    return epic


def on(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dt)


def inputs(rng, B, m, V, K, tau, dt, pad=0):
    l = torch.from_numpy((3 * rng.standard_normal((B, m, V + pad))).astype(np.float32)).to(DEV, DT[dt])
    ids = np.stack([[rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(m)] for _ in range(B)])
    t = (3 * rng.standard_normal((B, m, K))).astype(np.float32)
    a = t.astype(np.float64) / tau
    lse = (a.max(-1) + np.log(np.exp(a - a.max(-1, keepdims=True)).sum(-1)) + 0.2).astype(np.float32)
    return l[:, :, pad // 2:pad // 2 + V], ids.astype(np.int32), t, lse


def call(epic, logits, seqs, ids, t, lse, tau, weight, start=None, grad=None, backward=True):
    """Losses alone, losses with the gradient, and the backward pass."""
    B, m, _ = logits.shape
    loss, loss2 = (torch.full((B, m), 7.0, device=DEV) for _ in range(2))
    stats, stats2 = (torch.full((B, m, 2), 7.0, device=DEV) for _ in range(2))
    grads = [torch.full(logits.shape, 7.0, dtype=logits.dtype, device=DEV) for _ in range(2)]
    te = {"teacher_lse": None if lse is None else on(lse, torch.float32), "tau": tau,
          "start": None if start is None else on(start, torch.int32)}
    top = (None if seqs is None else on(seqs, torch.int32), on(ids, torch.int32), on(t, torch.float32))
    w = None if weight is None else on(weight, torch.float32)
    epic.distill_forward(logits, *top, loss, stats, **te)
    epic.distill_forward(logits, *top, loss2, stats2, weight=w, grad=grads[0], **te)
    epic.distill_backward(logits, *top, stats, w, grads[1], **te)
    assert torch.equal(loss.nan_to_num(9), loss2.nan_to_num(9)) and torch.equal(stats.nan_to_num(9), stats2.nan_to_num(9))
    return loss.cpu().numpy(), stats.cpu().numpy(), [g.float().cpu().numpy() for g in grads]


def check(logits, ids, t, lse, tau, weight, counts, loss, stats, grads, dt):
    """Bounds: an exponent (z - lse, t - lse_T) is a sum of numbers up to `size`
    with six roundings, so it is off by 6 * 2^-24 * size, and so is a share by
    that much of itself; the loss sums shares times exponents."""
    host = logits.float().cpu().numpy()
    K = ids.shape[2]
    for b, i in np.ndindex(*counts.shape):
        w = 1.0 if weight is None else weight[b, i]
        if not counts[b, i]:
            assert loss[b, i] == 0 and all((g[b, i] == 0).all() for g in grads)
            continue
        l = host[b, i]
        want, grad, z0, z1 = R.distill(l, ids[b, i], t[b, i], tau, None if lse is None else float(lse[b, i]))
        some = t[b, i][ids[b, i] >= 0]
        size = (np.abs(l[np.isfinite(l)]).max(initial=0) + np.abs(some[np.isfinite(some)]).max(initial=0)) / tau + 2 * math.log(len(l) + K) + 2
        off = 6 * 2.0 ** -24 * size
        # the rest's share of the teacher is a difference from 1: off by the shares' own error
        assert abs(loss[b, i] - want) <= tau * tau * off * (3 + size), (b, i, loss[b, i], want)
        for got, right in ((stats[b, i, 0], z0), (stats[b, i, 1], z1)):
            assert got == right or abs(got - right) <= off
        member = np.zeros(len(l), bool)
        member[ids[b, i][ids[b, i] >= 0]] = True
        with np.errstate(all="ignore"):
            p = np.exp(l.astype(np.float64) / tau - z0)
            of_rest = np.where(member, 0, np.exp(l.astype(np.float64) / tau - z1)) if z1 > -np.inf else np.zeros(len(l))
        pulled = p + np.abs(grad) / tau + of_rest  # what was subtracted from what
        bound = abs(w) * tau * (2 * off * pulled + of_rest * off)
        for g in grads:
            err = np.abs(g[b, i] - w * grad)
            assert (err <= bound + EPS[dt] * (np.abs(w * grad) + bound) + TINY[dt]).all(), (b, i, err.max())


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V,K", [(1, 1), (2, 1), (64, 64), (65, 5), (513, 8), (1000, 1000), (4097, 128), (32768, 64), (40001, 33),
                                 (131073, 20), (262144, 1024)])
def test_losses_and_gradients(epic, dt, V, K):
    rng = np.random.default_rng(V + K)
    B, m = (2, 1) if V > 50000 else (2, 3)
    for tau, rest in ((1.0, True), (2.0, False), (0.5, True)):
        logits, ids, t, lse = inputs(rng, B, m, V, K, tau, dt, pad=3)
        lse = lse if rest else None
        weight = (0.5 + rng.random((B, m))).astype(np.float32)
        loss, stats, grads = call(epic, logits, None, ids, t, lse, tau, weight)
        check(logits, ids, t, lse, tau, weight, np.ones((B, m), bool), loss, stats, grads, dt)


@pytest.mark.parametrize("rest", [True, False])
def test_windows_masks_and_odd_entries(epic, rest):
    """Rows that do not count hold NaN; entries absent, listed twice, of logit
    -inf; tokens of -inf; rows without entries or finite logits."""
    rng = np.random.default_rng(11)
    B, n, m, V, K = 4, 30, 12, 700, 9
    logits, ids, t, lse = inputs(rng, B, m, V, K, 1.0, "f32")
    logits = logits.clone()
    seqs = np.where(rng.random((B, n)) < 0.6, -1, 5).astype(np.int32)
    start = np.array([0, 18, 25, -2], np.int32)
    at = start[:, None] + np.arange(m)
    counts = (at >= 0) & (at < n) & (np.take_along_axis(seqs, at.clip(0, n - 1), 1) == -1)
    seqs[0, :6] = -1
    counts[0, :6] = True
    ids[:, :, 3] = -1
    ids[:, :, 5] = ids[:, :, 1]  # listed twice
    t[:, :, 7] = -np.inf
    logits[:, :, 650:] = -math.inf
    ids[ids >= 650] -= 60
    ids[0, 0] = -1  # no entries
    logits[0, 1] = -math.inf  # nothing to choose from
    t[0, 2] = -np.inf
    logits[0, 3, :] = -math.inf  # every finite logit is listed
    for j in ids[0, 3][ids[0, 3] >= 0]:
        logits[0, 3, j] = 1.5
    logits[0, 4] = -3.0e38  # masks of a very low value beside listed tokens
    for j in ids[0, 4][ids[0, 4] >= 0]:
        logits[0, 4, j] = 0.25
    logits[on(~counts, torch.bool)] = math.nan
    lse = lse if rest else None
    if rest:
        lse = lse + 0.5  # the entries listed twice count twice: leave room
    weight = rng.random((B, m)).astype(np.float32)
    loss, stats, grads = call(epic, logits, seqs, ids, t, lse, 1.0, weight, start=start)
    assert loss[0, 0] == 0 and loss[0, 1] == 0
    skip = counts.copy()
    skip[0, 1] = False  # no finite logit: loss and gradient are 0
    if rest:
        # the rest weighs 3e38 less than the listed: its part of the loss is that large, and is not compared closely
        assert loss[0, 4] > 1e37
        skip[0, 4] = False
        grads = [np.where((np.arange(m) == 4)[None, :, None] & (np.arange(B) == 0)[:, None, None], 0, g) for g in grads]
        loss[0, 4] = 0
    check(logits, ids, t, lse, 1.0, weight, skip, loss, stats, grads, "f32")


def test_ids_outside_the_vocabulary_and_nan(epic):
    rng = np.random.default_rng(1)
    logits, ids, t, lse = inputs(rng, 1, 4, 300, 5, 1.0, "f32")
    logits = logits.clone()
    ids[0, 0, 2] = 300
    logits[0, 1, 17] = math.nan
    t[0, 2, 1] = np.nan
    logits[0, 3, 3] = math.inf
    loss, stats, grads = call(epic, logits, None, ids, t, lse, 1.0, None)
    assert np.isnan(loss).all()
    for g in grads:
        assert (g[0, 0] == 0).all() and np.isnan(g[0, 1]).all()


def test_nan_reaches_losses_and_gradients(epic):
    """A NaN among the teacher's logits or the student's is not taken for an
    absent entry or an empty row."""
    rng = np.random.default_rng(2)
    V = 300
    logits, ids, t, lse = inputs(rng, 1, 3, V, 5, 1.0, "f32")
    logits = logits.clone()
    t[0, 0, 1] = np.nan
    t[0, 1] = np.nan
    logits[0, 2] = -math.inf
    left = np.setdiff1d(np.arange(V), ids[0, 2])
    logits[0, 2, int(left[7])] = math.nan  # the only one above -inf, and not listed
    for te in (lse, None):
        loss, stats, grads = call(epic, logits, None, ids, t, te, 1.0, None)
        assert np.isnan(loss).all() and np.isnan(stats[0, 2]).all()
        for g in grads:
            assert all(np.isnan(g[0, i, ids[0, i]]).all() for i in (1, 2))
            if te is not None:  # an entry's own share, and what is left to the rest
                others = np.delete(ids[0, 0], 1)
                assert np.isfinite(g[0, 0, others]).all() and np.isnan(np.delete(g[0, 0], others)).all() and np.isnan(g[0, 1]).all()
            else:  # every share of the softmax
                assert np.isnan(g[0, 0, ids[0, 0]]).all()


def test_gradient_against_differences(epic):
    """Differences of the loss in 64 bits at the kernel's float32 inputs."""
    rng = np.random.default_rng(21)
    V, K, tau = 40, 6, 1.5
    logits, ids, t, lse = inputs(rng, 1, 1, V, K, tau, "f32")
    _, _, grads = call(epic, logits, None, ids, t, lse, tau, None)
    l = logits[0, 0].double().cpu().numpy()
    h = 1e-5
    for j in range(V):
        a, b = l.copy(), l.copy()
        a[j] += h
        b[j] -= h
        d = (R.distill(a, ids[0, 0], t[0, 0], tau, float(lse[0, 0]))[0] - R.distill(b, ids[0, 0], t[0, 0], tau, float(lse[0, 0]))[0]) / (2 * h)
        for g in grads:
            assert abs(g[0, 0, j] - d) <= 2e-5  # 6 roundings of numbers up to 20, and h^2


@pytest.mark.parametrize("V", [600, 40000, 140000])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradient_in_place_and_in_other_strides(epic, dt, V):
    rng = np.random.default_rng(V)
    B, m, K = 2, 3, 7
    logits, ids, t, lse = inputs(rng, B, m, V, K, 1.0, dt, pad=1)
    args = (None, on(ids, torch.int32), on(t, torch.float32))
    te = {"teacher_lse": on(lse, torch.float32)}
    loss, stats = torch.zeros((B, m), device=DEV), torch.zeros((B, m, 2), device=DEV)
    w = torch.ones((B, m), device=DEV)
    want = torch.zeros_like(logits.contiguous())
    epic.distill_forward(logits, *args, loss, stats, weight=w, grad=want, **te)
    back = torch.zeros((m, B, V + 5), dtype=logits.dtype, device=DEV)
    out = back.transpose(0, 1)[:, :, 3:V + 3]  # sequences innermost, rows at odd addresses
    epic.distill_forward(logits, *args, loss, stats, weight=w, grad=out, **te)
    assert torch.equal(out, want) and (back[:, :, :3] == 0).all() and (back[:, :, V + 3:] == 0).all()
    other = torch.zeros_like(want)
    epic.distill_backward(logits, *args, stats, w, other, **te)
    for f in (True, False):
        copy = torch.zeros((B, m, V + 1), dtype=logits.dtype, device=DEV)
        mine = copy[:, :, :V]
        mine.copy_(logits)
        if f:
            epic.distill_forward(mine, *args, loss, stats, weight=w, grad=mine, **te)
        else:
            epic.distill_backward(mine, *args, stats, w, mine, **te)
        assert torch.equal(mine, want if f else other) and (copy[:, :, V] == 0).all()


def test_the_same_bits_in_any_batch(epic):
    rng = np.random.default_rng(3)
    logits, ids, t, lse = inputs(rng, 4, 5, 3001, 20, 1.0, "bf16")
    loss, stats, grads = call(epic, logits, None, ids, t, lse, 1.0, None)
    one = call(epic, logits[2:3, 3:4], None, ids[2:3, 3:4], t[2:3, 3:4], lse[2:3, 3:4], 1.0, None)
    assert one[0][0, 0] == loss[2, 3] and (one[1][0, 0] == stats[2, 3]).all()
    assert all((a[0, 0] == b[2, 3]).all() for a, b in zip(one[2], grads))


def test_refusals(epic):
    rng = np.random.default_rng(3)
    B, m, V, K = 2, 3, 64, 4
    logits, ids, t, lse = inputs(rng, B, m, V, K, 1.0, "f32")
    ids, t = on(ids, torch.int32), on(t, torch.float32)
    loss, stats, grad = torch.zeros((B, m), device=DEV), torch.zeros((B, m, 2), device=DEV), torch.zeros((B, m, V), device=DEV)

    def refused(code, f):
        with pytest.raises(epic.EpicError) as e:
            f()
        assert e.value.code == code

    for tau in (0.0, -1.0, math.inf, math.nan, 1e-44):
        refused(-2, lambda: epic.distill_forward(logits, None, ids, t, loss, stats, tau=tau))
    refused(-2, lambda: epic.distill_forward(logits, None, ids, t, loss, stats, grad=grad.bfloat16()))
    refused(-2, lambda: epic.distill_forward(logits, None, ids, t, loss, stats, grad=grad[:, :, :V - 1]))
    refused(-2, lambda: epic.distill_backward(logits, None, ids, t, stats, None, grad[:, :1].expand(B, m, V)))
    refused(-2, lambda: epic.distill_forward(logits, None, ids[:, :, :0], t[:, :, :0], loss, stats))
    many = torch.zeros((B, m, 1025), device=DEV)
    refused(-2, lambda: epic.distill_forward(logits, None, many.int(), many, loss, stats))
    for f in (lambda: epic.distill_forward(logits, None, ids.long(), t, loss, stats),
              lambda: epic.distill_forward(logits, None, ids, t[:, :, :2], loss, stats),
              lambda: epic.distill_forward(logits, None, ids, t, loss, stats[:, :, 0]),
              lambda: epic.distill_forward(logits, None, ids, t, loss, stats, weight=loss.double()),
              lambda: epic.distill_backward(logits, None, ids, t, stats, None, grad.cpu()),
              lambda: epic.distill_backward(logits, None, ids, t, stats, None, grad.transpose(1, 2))):
        with pytest.raises(ValueError):
            f()
