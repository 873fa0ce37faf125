"""The plain cross entropy's gradients against differences of its losses (CPU)."""
import numpy as np
import torch

from tests import head_ref


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    B, m, V, d = 2, 3, 11, 5
    h = torch.randn((B, m, d), generator=g, dtype=torch.float64)
    w = torch.randn((V, d), generator=g, dtype=torch.float64)
    target = torch.tensor([[0, 4, -1], [10, 4, 2]], dtype=torch.int32)
    weight = torch.tensor([[0.5, -2.0, 9.0], [1.0, 0.0, 3.0]])
    seqs = np.array([[-1, -1, -1], [-1, -1, 7]], np.int32)
    on = head_ref.counted(B, m, seqs, None, target)
    assert on.tolist() == [[True, True, False], [True, True, False]]
    _, _, gh, gw, _, _ = head_ref.loss(h, w, target, on, weight)

    def total(h, w):
        return float((head_ref.loss(h, w, target, on)[0] * weight).sum())

    step = 1e-5
    for x, grad in ((h, gh), (w, gw)):
        for at in np.ndindex(*x.shape):
            a, b = x.clone(), x.clone()
            a[at] += step
            b[at] -= step
            diff = (total(a, w) - total(b, w) if x is h else total(h, a) - total(h, b)) / (2 * step)
            # the second differences' error: step^2 / 6 times third derivatives of at most a few hundred here
            assert abs(diff - float(grad[at])) < 1e-7 + 1e-6 * abs(diff)


def test_rows_that_count():
    seqs = np.array([[-1, 3, -1, -1]], np.int32)
    assert head_ref.counted(1, 3, seqs, np.array([2])).tolist() == [[True, True, False]]
    assert head_ref.counted(1, 3, seqs, np.array([-1])).tolist() == [[False, True, False]]
    assert head_ref.counted(1, 2).tolist() == [[True, True]]


def test_quantized_rows():
    x = torch.tensor([[127.0, 0.5, 1.5, -2.5, -127.0], [0.0, 0.0, 0.0, 0.0, 0.0], [1e-31, 0.0, 0.0, 0.0, 0.0],
                      [1.0, float("nan"), 0.0, 0.0, 0.0], [1.0, float("-inf"), 0.0, 0.0, 0.0]])
    q, s = head_ref.quantize(x)
    assert q.tolist() == [[127.0, 0.0, 2.0, -2.0, -127.0]] + [[0.0] * 5] * 4
    assert s[:3].tolist() == [1.0, 0.0, 0.0] and torch.isnan(s[3:]).all()
