"""The operators on logits rows at the limits of their arguments: more rows
than one launch can have, sequences without positions."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    return epic


MANY = 2 ** 26 + 70  # rows: with 64 lanes each, more than one launch can have


def test_rows_past_one_launch(epic):
    """More rows than a launch has work-items for, of one logits row that is
    repeated: all are written."""
    rng = np.random.default_rng(1)
    V = 40
    logits = torch.from_numpy((2 * rng.standard_normal(V)).astype(np.float32)).to(DEV).expand(1, MANY, V)
    u = torch.arange(MANY, device=DEV, dtype=torch.float32)[None] / MANY
    tok = torch.full((1, MANY), -7, dtype=torch.int32, device=DEV)
    conf = torch.full((1, MANY), -7.0, device=DEV)
    epic.sample(logits, None, u, tok, conf)
    assert int(tok.min()) >= 0 and int(tok.max()) < V
    assert (tok[0, 1:] >= tok[0, :-1]).all()  # the number rises, and so does the token
    for at in (0, 2 ** 26 - 2, MANY - 9):
        some = slice(at, at + 9)
        one = [torch.zeros((1, min(9, MANY - at)), dtype=dt, device=DEV) for dt in (torch.int32, torch.float32)]
        epic.sample(logits[:, some], None, u[:, some].contiguous(), *one)
        assert torch.equal(tok[:, some], one[0]) and torch.equal(conf[:, some], one[1])


def test_losses_and_gradients_past_one_launch(epic):
    V, K = 3, 1
    gen = torch.Generator(DEV).manual_seed(3)
    logits = torch.randn((1, 1, V), device=DEV, generator=gen).to(torch.bfloat16).expand(1, MANY, V)
    ids = torch.zeros((1, MANY, K), dtype=torch.int32, device=DEV)
    ids[0, 1::2] = 2
    t = torch.zeros((1, MANY, K), device=DEV)
    loss, stats = torch.full((1, MANY), 7.0, device=DEV), torch.full((1, MANY, 2), 7.0, device=DEV)
    grads = [torch.full((1, MANY, V), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    epic.distill_forward(logits, None, ids, t, loss, stats, grad=grads[0])
    epic.distill_backward(logits, None, ids, t, stats, None, grads[1])
    for a in (loss, stats, *grads):  # two kinds of rows, alike from the first to the last
        assert (a[:, 2::2] == a[:, :1]).all() and (a[:, 3::2] == a[:, 1:2]).all() and (a[:, :2] != 7).all()
    few = torch.zeros((1, 2), device=DEV)
    epic.distill_forward(logits[:, :2], None, ids[:, :2].contiguous(), t[:, :2].contiguous(), few, stats[:, :2].contiguous())
    assert torch.equal(few, loss[:, :2])


def test_proposals_past_one_launch(epic):
    tok = torch.arange(MANY, dtype=torch.int32, device=DEV)[:, None].contiguous()
    tok[::3] = -1
    conf = torch.full((MANY, 1), 0.5, device=DEV)
    cand = [torch.full((MANY,), 77, dtype=torch.int32, device=DEV) for _ in range(3)] + [torch.full((MANY,), 77.0, device=DEV)]
    off = torch.full((MANY + 1,), 77, dtype=torch.int32, device=DEV)
    epic.propose(tok, conf, 1, *cand, off)
    there = (tok[:, 0] >= 0).nonzero()[:, 0].to(torch.int32)
    C = len(there)
    assert off[0] == 0 and torch.equal(off[1:], (tok[:, 0] >= 0).cumsum(0).to(torch.int32))
    assert torch.equal(cand[0][:C], there) and torch.equal(cand[2][:C], there) and (cand[1][:C] == 0).all() and (cand[3][:C] == 0.5).all()
    assert all((c[C:] == -1).all() for c in cand[:3]) and (cand[3][C:] == 0).all()


def test_sequences_without_positions_are_refused(epic):
    """An empty tensor has no address, which is not the same as no sequences."""
    B, m, V = 2, 3, 64
    logits = torch.zeros((B, m, V), device=DEV)
    seqs = torch.zeros((B, 0), dtype=torch.int32, device=DEV)
    u, tok, conf = torch.zeros((B, m), device=DEV), torch.full((B, m), -7, dtype=torch.int32, device=DEV), torch.zeros((B, m), device=DEV)
    ids, t = torch.zeros((B, m, 2), dtype=torch.int32, device=DEV), torch.zeros((B, m, 2), device=DEV)
    loss, stats = torch.full((B, m), 7.0, device=DEV), torch.zeros((B, m, 2), device=DEV)
    for f in (lambda: epic.sample(logits, seqs, u, tok, conf),
              lambda: epic.distill_forward(logits, seqs, ids, t, loss, stats),
              lambda: epic.distill_backward(logits, seqs, ids, t, stats, None, logits)):
        with pytest.raises(ValueError):
            f()
    assert (tok == -7).all() and (loss == 7).all()
    none = torch.zeros((0, 0), dtype=torch.int32, device=DEV)  # no sequences at all: nothing to do
    epic.sample(logits[:0], none, u[:0], tok[:0], conf[:0])
