"""The example that distills a small denoiser and decodes with it: the
divergence falls, every mask is filled, and the oracle finds every sequence in
the grammar's language."""
import numpy as np
import pytest

from paper_2606_00722_amd import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_distilled_denoiser_decodes_sentences():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    import oracle
    from paper_2606_00722_amd import denoise

    res = denoise.run(preset=1, train=60, seed=42)
    assert res["losses"][-1] < 0.25 * res["losses"][0]
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
