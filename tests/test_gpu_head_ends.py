"""The operators between hidden states and logits at the ends of what their inputs
may be."""
import pytest

from tests import head_ref
from tests.test_gpu_head import DT, Case, backward, epic, forward  # noqa: F401 (epic: a fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# ------------------------------------------------------------------ 8 bits


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("d,stride", [(1, 4224), (1000, 8192), (1000, 131072), (4095, 4224), (4096, 4224), (4096, 12288), (4097, 4224),
                                      (5000, 5120), (5000, 16384), (9000, 9088), (65536, 65536), (65536, 65664)])
def test_quantize_to_any_stride(dtype, d, stride, epic):  # noqa: F811
    """Zeros behind the width wherever the row ends."""
    g = torch.Generator().manual_seed(d + stride)
    x = (3 * torch.randn((5, d), generator=g)).to(DT[dtype])
    x[3] = 0
    q = torch.full((5, stride), 77, dtype=torch.int8, device="cuda")
    s = torch.empty(5, device="cuda")
    epic.quantize(x.cuda(), q, s)
    want_q, want_s = head_ref.quantize(x)
    assert torch.equal(q.cpu()[:, :d].float(), want_q) and torch.equal(s.cpu(), want_s)
    assert not bool(q[:, d:].any())


# ------------------------------------------------ rows that add nothing


@pytest.mark.parametrize("rows", [90, 1100])
@pytest.mark.parametrize("dtype", sorted(DT))
def test_hidden_states_of_a_row_that_adds_nothing(dtype, rows, epic):  # noqa: F811
    """However large they are, the others' gradients are those without the row."""
    c = Case(dtype, 1, rows, 70, 40, share=1.0, seed=6)
    c.target[0, rows - 5] = c.V
    c.on = head_ref.counted(1, rows, c.seqs, None, c.target)
    c.full_h[0, rows - 5] = 1.0
    _, lse = forward(epic, c)
    want = backward(epic, c, lse)
    c.full_h[0, rows - 5] = 60000.0 if dtype == "float16" else 1e30
    got = backward(epic, c, lse)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool(got[1].any())
