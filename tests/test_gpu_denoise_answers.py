"""The example that learns the answers' tokens without logits and decodes with its
weights in 8 bits: the operators between hidden states and logits, sampling,
proposals and the check as they are used together.  Every mask is filled, the
oracle finds every sequence in the grammar's language, and the first training
step's losses and gradient are those of the formula."""
import numpy as np
import pytest

from paper_2606_00722_amd import workloads as W
from tests import head_ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")


def test_denoiser_of_answers_decodes_sentences():
    import oracle
    from paper_2606_00722_amd import denoise

    res = denoise.run(preset=1, train=40, seed=42, answers=True)
    assert np.isfinite(res["losses"]).all()
    assert res["left"] == 0 and res["errors"] == 0
    inst = W.make_instance(1, 42)
    kept = inst.seqs != W.MASK
    assert (res["seqs"][kept] == inst.seqs[kept]).all()
    # each sequence with its last token taken out and proposed again
    last = np.full(inst.B, inst.n - 1, np.int32)
    tok = res["seqs"][:, -1].copy()
    seqs = res["seqs"].copy()
    seqs[:, -1] = W.MASK
    p = oracle.problem_from(inst.lang, inst.vocab)
    assert oracle.validate_batch(p, seqs, np.arange(inst.B, dtype=np.int32), last, tok).tolist() == [1] * inst.B


def test_first_step():
    """Zero weights: every token has probability 1 / V, and the gradient's sums are
    of bfloat16 numbers, G rounded to half a step (2^-8) and the result once more."""
    from paper_2606_00722_amd import denoise

    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    B, n, V = 2, 20, 130
    model = denoise.AnswerDenoiser(B, n, V, dev, gen)
    seqs = torch.where(torch.rand((B, n), generator=gen, device=dev) < 0.6, -1, 3).to(torch.int32)
    target = torch.randint(0, V, (B, n), generator=gen, device=dev).to(torch.int32)
    mean = float(model.train_step(seqs, target, lr=0.0))
    assert abs(mean - np.log(V)) < 1e-5  # log of a sum of V ones, and a mean of 40
    on = head_ref.counted(B, n, seqs.cpu().numpy(), None, target.cpu())
    _, _, _, want, _, size = head_ref.loss(model.hidden.cpu(), model.head.cpu(), target.cpu(), on)
    assert bool(((model.grad.cpu().double() - want).abs() <= size * 2.0 ** -8 + want.abs() * 2.0 ** -8 + 1e-12).all())
    # the weights in 8 bits give the same rows' logits as the plain implementation
    model.head.normal_(generator=gen)
    got = model.logits(seqs)[torch.from_numpy(on).to(dev)]
    want = head_ref.logits_q8(model.hidden.cpu(), model.q.cpu()[:, : model.head.shape[1]], model.scale.cpu(), on, torch.bfloat16)
    assert torch.equal(got.cpu(), want)


def test_step_goes_against_the_gradient():
    from paper_2606_00722_amd import denoise

    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(2)
    B, n, V = 2, 20, 130
    model = denoise.AnswerDenoiser(B, n, V, dev, gen)
    seqs = torch.full((B, n), -1, dtype=torch.int32, device=dev)
    target = torch.randint(0, V, (B, n), generator=gen, device=dev).to(torch.int32)
    model.train_step(seqs, target, lr=0.25)
    on = head_ref.counted(B, n, seqs.cpu().numpy(), None, target.cpu())
    _, _, _, want, _, size = head_ref.loss(model.hidden.cpu(), torch.zeros_like(model.head).cpu(), target.cpu(), on)
    assert bool(((model.w.cpu().double() + 0.25 * want).abs() <= 0.25 * (size * 2.0 ** -8 + want.abs() * 2.0 ** -8 + 1e-12)).all())
    assert bool(model.w.any()) and torch.equal(model.head, model.w.to(torch.bfloat16))
