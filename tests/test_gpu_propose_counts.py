"""epic_propose where its counting takes another way: batches around those that
one launch counts, windows around 64, 320 and 1088 rows, sequences with few,
enough and no proposals side by side."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.mark.parametrize("m", [1, 63, 64, 65, 129, 320, 321, 1088, 1089, 2500])
@pytest.mark.parametrize("B", [1, 2, 3, 16, 17, 40, 257, 1024, 1030])
def test_counts(B, m):
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    rng = np.random.default_rng(1000 * B + m)
    share = rng.choice([0.0, 0.01, 0.1, 0.9, 1.0], (B, 1))
    tok = np.where(rng.random((B, m)) < share, rng.integers(0, 9999, (B, m)), -1).astype(np.int32)
    conf = rng.random((B, m)).astype(np.float32)
    conf[rng.random((B, m)) < 0.05] = np.nan
    tok[::5, :min(m, 64)] = -1  # their first proposals come late
    tok[::5, m - 1] = 3
    conf[::5, m - 1] = 0.25
    key = np.where((tok >= 0) & ~np.isnan(conf), conf, -1)
    order = np.argsort(-key, axis=1, kind="stable")
    for P in (1, 9, 64):
        cand = [torch.full((B * P,), 77, dtype=torch.int32, device=DEV) for _ in range(3)]
        cand.append(torch.full((B * P,), 77.0, device=DEV))
        off = torch.full((B + 1,), 77, dtype=torch.int32, device=DEV)
        epic.propose(torch.from_numpy(tok).to(DEV), torch.from_numpy(conf).to(DEV), P, *cand, off)
        count = np.minimum((key >= 0).sum(1), P)
        want = np.concatenate([[0], np.cumsum(count)])
        assert off.tolist() == want.tolist()
        pos = np.concatenate([order[b, :count[b]] for b in range(B)])
        seq = np.repeat(np.arange(B), count)
        C = len(seq)
        for got, right in zip(cand, (seq, pos, tok[seq, pos], conf[seq, pos])):
            got = got.cpu().numpy()
            assert (got[:C] == right).all() and (got[C:] == (0 if got.dtype == np.float32 else -1)).all()
