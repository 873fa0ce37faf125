"""epic_distill_forward and epic_distill_backward where the teacher's numbers
are infinite or the student's are none, and at the least tau."""
import math

import numpy as np
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    return epic


def run(epic, l, ids, t, lse, tau=1.0):
    on = lambda a, dt: torch.from_numpy(np.asarray(a)).to(DEV, dt)  # noqa: E731
    logits, top = on(l, torch.float32), (on(ids, torch.int32), on(t, torch.float32))
    te = {"teacher_lse": None if lse is None else on(lse, torch.float32), "tau": tau}
    B, m, _ = logits.shape
    loss, stats = torch.full((B, m), 7.0, device=DEV), torch.full((B, m, 2), 7.0, device=DEV)
    alone = torch.full((B, m), 7.0, device=DEV)
    grads = [torch.full_like(logits, 7.0) for _ in range(2)]
    epic.distill_forward(logits, None, *top, alone, stats, **te)
    epic.distill_forward(logits, None, *top, loss, stats, grad=grads[0], **te)
    epic.distill_backward(logits, None, *top, stats, None, grads[1], **te)
    assert torch.equal(alone.nan_to_num(9), loss.nan_to_num(9))
    return loss.cpu().numpy(), [g.cpu().numpy() for g in grads]


def test_infinite_teacher_numbers_give_nan(epic):
    """+inf among the entries' logits or as the teacher's logsumexp."""
    rng = np.random.default_rng(4)
    V, K = 90, 4
    l = rng.standard_normal((1, 3, V))
    ids = np.tile(np.array([5, 80, 33, 7]), (1, 3, 1))
    t = rng.standard_normal((1, 3, K))
    t[0, 0, 1] = math.inf
    lse = np.log(np.exp(rng.standard_normal((1, 3, K))).sum(-1)) + 3
    lse[0, 1] = math.inf
    t[0, 2, 2] = lse[0, 2] = math.inf
    loss, grads = run(epic, l, ids, t, lse)
    assert np.isnan(loss).all()
    others = np.setdiff1d(np.arange(V), ids[0, 0])
    for g in grads:
        assert np.isnan(g[0, 0, 80]) and np.isnan(g[0, :, others]).all()  # its share, and what is left to the rest
        assert np.isfinite(g[0, 0, [5, 33, 7]]).all() and np.isnan(g[0, 1:]).all()
    loss, grads = run(epic, l[:, :1], ids[:, :1], t[:, :1], None)
    assert np.isnan(loss).all()
    for g in grads:
        assert np.isnan(g[0, 0, ids[0, 0]]).all()


def test_teacher_of_nothing_but_masks(epic):
    """Entries of -inf have no share, with a logsumexp of -inf too: the rest has
    it all."""
    rng = np.random.default_rng(9)
    l = rng.standard_normal((1, 1, 70)).astype(np.float32)
    ids, t = np.array([[[3, 60, 11]]]), np.full((1, 1, 3), -math.inf)
    loss, grads = run(epic, l, ids, t, np.full((1, 1), -math.inf))
    want, grad, _, _ = R.distill(l[0, 0], ids[0, 0], t[0, 0], 1.0, 0.0)  # as beside any finite logsumexp
    assert abs(loss[0, 0] - want) <= 1e-5  # 6 roundings of numbers up to 10
    for g in grads:
        assert np.abs(g[0, 0] - grad).max() <= 1e-5


def test_nan_of_the_student_beside_no_share(epic):
    """Every token listed, none with a share: the row's NaN is still seen."""
    l = np.zeros((1, 1, 3))
    l[0, 0, 1] = math.nan
    loss, grads = run(epic, l, np.array([[[0, 1, 2]]]), np.full((1, 1, 3), -math.inf), np.zeros((1, 1)))
    assert np.isnan(loss).all() and all(np.isnan(g).all() for g in grads)


def test_tiny_tau(epic):
    """A tau whose log2(e) / tau is past float32 is refused; one a little above
    leaves the largest logit all of the mass."""
    V, K = 50, 2
    l, ids, t = np.zeros((1, 1, V)), np.array([[[7, -1]]]), np.zeros((1, 1, K))
    for tau in (1e-44, 3e-39, 4.2e-39):
        with pytest.raises(epic.EpicError) as e:
            run(epic, l, ids, t, None, tau)
        assert e.value.code == -2
    l[0, 0, 7] = 1.0
    loss, grads = run(epic, l, ids, t, None, 4.3e-39)
    assert loss[0, 0] == 0 and all((g == 0).all() for g in grads)
