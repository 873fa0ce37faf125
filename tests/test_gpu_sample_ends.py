"""epic_sample where whole-number weights are small: top-p close to 1 and a
min-p close to 0, each without top-k, on rows whose tail lies 20 to 22.5 nats
below the largest logit, where a weight is a handful of units and its rounding
is as large as itself.  Bit for bit against the definition."""
import math

import numpy as np
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = [512, 4096, 32768, 131072, 140000]  # every number of vectors a lane, with rows too long for registers


@pytest.fixture(scope="module")
def epic():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible to the gpu-marked tests")
    from paper_2606_00722_amd import epic

    return epic


def rows_of(kind, V, rng):
    """A peak of 22 and a tail below it."""
    at = int(rng.integers(1, V))
    if kind == "flat":
        l = np.zeros(V)
    elif kind == "spread":
        l = rng.uniform(-0.5, 2.0, V)
    else:  # few: a handful of tokens in the band, the others far below
        l = np.full(V, -40.0)
        l[rng.permutation(V)[:60]] = rng.uniform(-0.5, 2.0, 60)
    l[at] = 22.0
    return l.astype(np.float32)


def check(epic, dt, row, settings, us, T=1.0):
    """Every setting with every number on one row, bit for bit."""
    V, B = len(row), len(settings)
    one = torch.from_numpy(row).to(DEV, DT[dt])
    logits = one.expand(B, len(us), V)
    p, q = (torch.tensor(a, dtype=torch.float32, device=DEV) for a in zip(*settings))
    u = torch.tensor(us, dtype=torch.float32, device=DEV).expand(B, len(us)).contiguous()
    tok = torch.full((B, len(us)), -7, dtype=torch.int32, device=DEV)
    conf = torch.full((B, len(us)), -7.0, device=DEV)
    epic.sample(logits, None, u, tok, conf, temperature=torch.full((B,), T, device=DEV), top_p=p, min_p=q)
    tok, conf, l = tok.cpu().numpy(), conf.cpu().numpy(), one.float().cpu().numpy()
    e = torch.exp2(torch.from_numpy(R.exponents(l, np.float32(T))).to(DEV)).cpu().numpy()
    for b, (p, q) in enumerate(settings):
        for i, x in enumerate(us):
            want = R.draw(l, e, x, np.float32(T), 0, np.float32(p), np.float32(q))
            assert tok[b, i] == want[0] and abs(conf[b, i] - want[1]) <= 4e-7 * want[1], (p, q, x, tok[b, i], want)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_top_p_close_to_one(epic, dt, V):
    """Masses left out of V times half a unit to V units, and a few around."""
    rng = np.random.default_rng(V)
    share = V / 128  # in 2^24ths, what V units are of the likeliest token's 2^31
    parts = sorted({max(1, round(share * x)) for x in (0.4, 0.55, 0.66, 0.75, 0.9, 1.3)} | {1, 168})
    settings = [(1 - n * 2.0 ** -24, 0.0) for n in parts] + [(1 - parts[-2] * 2.0 ** -24, 1e-9)]
    for kind in ("flat", "spread", "few"):
        check(epic, dt, rows_of(kind, V, rng), settings, [0.5, 1 - 2.0 ** -24])


@pytest.mark.parametrize("dt", ["f16", "f32"])
def test_top_p_close_to_one_at_other_temperatures(epic, dt):
    rng = np.random.default_rng(5)
    row = rows_of("flat", 32768, rng)
    check(epic, dt, row / 2, [(0.99999, 0.0), (0.9999, 0.0)], [0.0, 0.5, 1 - 2.0 ** -24], T=0.5)
    check(epic, dt, 2 * row, [(0.99999, 0.0), (0.9999, 0.0)], [0.0, 0.5, 1 - 2.0 ** -24], T=2.0)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_min_p_close_to_zero(epic, dt, V):
    """From half a unit on: a token passes when its weight rounds up to the
    least that passes."""
    rng = np.random.default_rng(V + 1)
    settings = [(1.0, q) for q in (2.0 ** -32, 2.0 ** -31, 1e-9, 3e-9, 1e-8, 3e-8, 1e-7)]
    for kind in ("flat", "spread", "few"):
        check(epic, dt, rows_of(kind, V, rng), settings, [0.0, 1 - 2.0 ** -24])


def test_min_p_keeps_the_half_unit(epic):
    """One token just above, one just below the half unit of every weight."""
    row = np.full(2000, -60.0, np.float32)
    row[1999] = 0.0
    settings = []
    for i, w in enumerate([1, 2, 3, 5, 9, 17, 40, 70, 100]):
        edge = math.log((w - 0.5) / 2 ** 31)
        row[2 * i + 1], row[2 * i] = edge + 2e-5, edge - 2e-5  # x is rounded to within 4e-6
        settings.append((1.0, w / 2 ** 31))
    check(epic, "f32", row, settings, [0.0, 2.0 ** -24, 0.5])
