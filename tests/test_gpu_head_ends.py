"""The operators between hidden states and logits at the ends of what their inputs
may be: strides above the least, rows that add nothing,
logits past 2^31, rows and weights of very unlike size, heads at odd addresses, rows in
another order, losses of many rows.

Tolerances as in test_gpu_head (u32 = 2^-24), by row: a row's logits are off by
(8 sqrt(d) u32 + 2^-22) of its largest sum A of terms' magnitudes, its lse by that, 2e-5 and,
where it is large, the roundings of a float32 number of its size (lse's sum, the loss's
difference: 4 u32 |lse| for both).  In grad_head a float32 row's hidden states are two
float16 numbers whose half step is 2^-25, of rows scaled so that the largest
product of weight and magnitude of a row (powers of two, each below twice its number) is
2^15: with |G| <= 1 times its weight, 2^-38 of the largest such product for every row; G itself,
2^14 at most, is off by 2^-39 of its row's weight where it is small."""
import math

import pytest

from tests import head_ref
from tests.test_gpu_head import DT, U32, Case, backward, epic, forward  # noqa: F401 (epic: a fixture)

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


# ------------------------------------------------------- large logits


def by_row(c, lse):
    """Bounds of every row's logits, and of lse and loss [B, m]."""
    h, w = c.h.double(), c.w.double()
    A = torch.zeros((c.B, c.m), dtype=torch.float64)
    on = torch.from_numpy(c.on)
    A[on] = (h[on].abs() @ w.abs().t()).amax(-1)
    off = (8 * math.sqrt(c.d) * U32 + (2.0 ** -22 if c.dtype == "float32" else 0.0)) * A
    return off, off + 2e-5 + 4 * U32 * lse.abs()


@pytest.mark.parametrize("dtype,m", [("bfloat16", 6), ("float16", 6), ("float32", 6), ("float32", 70)])
def test_logits_past_two_to_the_31(dtype, m, epic):  # noqa: F811
    """One token of 2^35 and more in every row: it has probability 1, the others 0."""
    V, d = 300, 128
    c = Case(dtype, 2, m, V, d, share=1.0, seed=14)
    g = torch.Generator().manual_seed(15)
    c.full_h[..., :d] = (2.0 ** 14 * (1 + torch.rand((2, m, d), generator=g))).to(DT[dtype])
    c.full_w[:, :d] = (torch.randn((V, d), generator=g)).to(DT[dtype])
    c.full_w[5] = (2.0 ** 14 * (1 + torch.rand(d, generator=g))).to(DT[dtype])
    c.target = torch.randint(6, V, (2, m), generator=g).to(torch.int32)
    c.target[:, ::2] = 5
    c.on = head_ref.counted(2, m, c.seqs, None, c.target)
    loss, lse = forward(epic, c)
    want = head_ref.loss(c.h, c.w, c.target, c.on, c.weight)
    off, _ = by_row(c, want[1])
    e = off + 4 * U32 * want[1]
    assert bool((want[1] > 2.0 ** 34).all())
    assert bool(((lse.cpu() - want[1]).abs() <= e).all()) and bool(((loss.cpu() - want[0]).abs() <= 2 * e).all())
    assert not bool(loss[:, ::2].any())
    gh, gw = backward(epic, c, lse)
    # G is the row's weight at token 5 and minus it at the row's own, each rounded to the type, as the result
    w = c.w.double()
    diff, size = w[5] - w[c.target.long()], w[5].abs() + w[c.target.long()].abs()
    u = torch.finfo(DT[dtype]).eps / 2 if dtype != "float32" else 2.0 ** -22
    weight = c.weight.double()[..., None]
    lim = torch.finfo(DT[dtype]).max
    got, want_h = gh.double(), (diff * weight)
    assert bool(((got - want_h).abs() <= 3 * u * size * weight.abs())[want_h.abs() < 0.9 * lim].all())
    assert not bool(gh[:, ::2].any())
    G = torch.zeros((2 * m, V), dtype=torch.float64)
    G[:, 5] += c.weight.double().reshape(-1)
    G[torch.arange(2 * m), c.target.reshape(-1).long()] -= c.weight.double().reshape(-1)
    h = c.h.double().reshape(2 * m, d)
    want_w, size_w = G.t() @ h, G.abs().t() @ h.abs()
    left = 2 * m * float((c.weight.abs().max() * c.h.abs().max())) * (2.0 ** -38 if dtype == "float32" else 0.0) \
        + (2.0 ** -25 + 4 * m * float(c.weight.abs().max()) * 2.0 ** -25 if dtype == "float16" else 0.0)
    bad = ~((gw.double() - want_w).abs() <= 3 * u * size_w + 8 * math.sqrt(2 * m) * U32 * size_w + left) & (want_w.abs() < 0.9 * lim)
    assert not bool(bad.any())


@pytest.mark.parametrize("dtype,m", [("bfloat16", 64), ("float16", 64), ("float32", 64), ("float32", 90)])
def test_rows_beside_large_logits(dtype, m, epic):  # noqa: F811
    """Their losses and gradients are those without the large ones, bit for bit."""
    c = Case(dtype, 1, m, 300, 128, share=1.0, seed=21)
    c.target.clamp_(min=0)
    c.on = head_ref.counted(1, m, c.seqs, None, c.target)
    g = torch.Generator().manual_seed(22)
    c.full_h[..., :128] = torch.randn((1, m, 128), generator=g).to(DT[dtype])
    c.full_h[..., 0] = 0.01
    c.full_w[:, 0] = (4000 * torch.randn(300, generator=g)).to(DT[dtype])
    loss, lse = forward(epic, c)
    gh, _ = backward(epic, c, lse)
    rest = torch.arange(m) % 9 != 4
    for row in (~rest).nonzero()[:, 0].tolist():
        c.full_h[0, row] *= 2.0 ** (9 if dtype == "float16" else 40)
        c.full_h[0, row, 0] = 60000.0 if dtype == "float16" else 2.0 ** 40
    loss2, lse2 = forward(epic, c)
    gh2, _ = backward(epic, c, lse2)
    assert float(lse2[0, ~rest].min()) > 2.0 ** (24 if dtype == "float16" else 31)
    assert torch.equal(loss[0, rest], loss2[0, rest]) and torch.equal(lse[0, rest], lse2[0, rest])
    assert torch.equal(gh[0, rest], gh2[0, rest])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_logit_of_minus_infinity(dtype, epic):  # noqa: F811
    """Out of finite numbers: the token has probability 0, its own loss is infinite."""
    m, V, d = 6, 300, 128
    c = Case(dtype, 2, m, V, d, share=1.0, seed=19)
    g = torch.Generator().manual_seed(20)
    c.full_h[..., :d] = (1e25 * (1 + torch.rand((2, m, d), generator=g))).to(DT[dtype])
    c.full_w[:, :d] = (1e-26 * torch.randn((V, d), generator=g)).to(DT[dtype])
    c.full_w[5] = -1e25
    c.target = torch.randint(6, V, (2, m), generator=g).to(torch.int32)
    c.target[0, 2] = 5
    c.on = head_ref.counted(2, m, c.seqs, None, c.target)
    loss, lse = forward(epic, c)
    want = head_ref.loss(c.h, c.w, c.target, c.on, c.weight)
    c2 = c.w.clone()
    c2[5] = 0  # (the bound is by the other tokens)
    A = (c.h.double().abs() @ c2.double().abs().t()).amax(-1)
    e = 8 * math.sqrt(d) * U32 * A + 2e-5 + 4 * U32 * want[1].abs()
    assert float(loss[0, 2]) == math.inf
    loss[0, 2] = want[0][0, 2] = 0
    assert bool(((lse.cpu() - want[1]).abs() <= e).all()) and bool(((loss.cpu() - want[0]).abs() <= 2 * e).all())
    gh, gw = backward(epic, c, lse)
    assert bool(torch.isfinite(gh).all()) and bool(torch.isfinite(gw).all())
    # its row alone has a gradient at the token
    want_w = -c.weight[0, 2].double() * c.h[0, 2].double()
    assert bool(((gw[5].double() - want_w).abs() <= 3 * torch.finfo(DT[dtype]).eps / 2 * want_w.abs()).all())
    own = c.weight[0, 2].double() * -c.w[5].double()
    assert bool(((gh[0, 2].double() - own).abs() <= 3 * torch.finfo(DT[dtype]).eps / 2 * own.abs()).all())


# ---------------------------------------------- rows of very unlike size


def check_rows(epic, c, loss, lse):  # noqa: F811
    """Every row's loss and gradient of hidden states, and the head's gradient, within
    what is theirs."""
    on = torch.from_numpy(c.on)
    want = head_ref.loss(c.h, c.w, c.target, c.on, c.weight)
    _, e = by_row(c, want[1])
    assert bool(((lse.cpu() - want[1]).abs() <= e).all())
    assert bool(((loss.cpu() - want[0]).abs() <= 2 * e)[on].all())
    gh, gw = backward(epic, c, lse)
    given = lse.cpu().double()
    if c.weight is not None:  # (0 times what a rounded lse would leave)
        given = torch.where(c.weight == 0, want[1], given)
    _, _, want_h, want_w, size_h, size_w = head_ref.loss(c.h, c.w, c.target, c.on, c.weight, given)
    h, w = c.h.double().clone(), c.w.double()
    h[~on] = 0
    weight = torch.ones((c.B, c.m), dtype=torch.float64) if c.weight is None else c.weight.double().abs()
    p = torch.softmax(h @ w.t(), -1) * (weight * on)[..., None]
    terms = c.B * c.m
    bound_h = size_h * (2.0 ** -22 + 8 * math.sqrt(c.V) * U32) + 2 * e[..., None] * (p @ w.abs()) + want_h.abs() * U32 \
        + 2.0 ** -38 * weight[..., None] * w.abs().max() * c.V + 1e-37
    assert bool(((gh.double() - want_h).abs() <= bound_h)[on].all())
    most = weight * h.abs().amax(-1) * on
    flat, rows = p.reshape(terms, -1), h.abs().reshape(terms, -1)
    bound_w = size_w * (2.0 ** -22 + 8 * math.sqrt(terms) * U32) + (2 * e.reshape(-1, 1) * flat).t() @ rows + want_w.abs() * U32 \
        + (2.0 ** -38 * terms * float(most.max()) + 2.0 ** -38 * float(most.sum())) + 1e-37
    bad = ~((gw.double() - want_w).abs() <= bound_w)
    assert not bool(bad.any()), (float((gw.double() - want_w).abs().max()), float(bound_w.max()), int(bad.sum()))


@pytest.mark.parametrize("m,V", [(60, 300), (600, 70)])
def test_a_row_far_larger_than_the_others(m, V, epic):  # noqa: F811
    """Of weight 0, so that the head's gradient is the others' too."""
    c = Case("float32", 2, m, V, 96, share=1.0, seed=7)
    c.target.clamp_(min=0)
    c.on = head_ref.counted(2, m, c.seqs, None, c.target)
    c.full_h[..., :96] = torch.randn((2, m, 96), generator=torch.Generator().manual_seed(8))
    c.full_h[0, 7] *= 2.0 ** 40
    c.full_h[1, 11] *= 2.0 ** -50
    c.weight[0, 7] = 0
    loss, lse = forward(epic, c)
    check_rows(epic, c, loss, lse)


@pytest.mark.parametrize("m", [90, 1100])
def test_products_of_weights_and_rows(m, epic):  # noqa: F811
    """Rows 2^k smaller of weights 2^k larger all count alike in the head's gradient."""
    c = Case("float32", 1, m, 200, 96, share=1.0, seed=9)
    c.target.clamp_(min=0)
    c.on = head_ref.counted(1, m, c.seqs, None, c.target)
    k = (torch.arange(m) % 41).float()
    c.full_h[0, :, :96] = torch.randn((m, 96), generator=torch.Generator().manual_seed(10)) * torch.exp2(-k)[:, None]
    c.weight[0] = torch.exp2(k) * (0.5 + torch.rand(m, generator=torch.Generator().manual_seed(11)))
    loss, lse = forward(epic, c)
    check_rows(epic, c, loss, lse)


def test_scales_whose_product_is_past_float32(epic):  # noqa: F811
    """A head of 2^100, rows of 2^-100, and one of 2^60 whose logits are infinite."""
    c = Case("float32", 1, 90, 120, 96, share=1.0, seed=12)
    c.target.clamp_(min=0)
    c.on = head_ref.counted(1, 90, c.seqs, None, c.target)
    c.full_w *= 2.0 ** 100
    c.full_h[0, :, :96] = torch.randn((90, 96), generator=torch.Generator().manual_seed(13)) * 2.0 ** -100
    small = c.full_h[0, 4].clone()
    c.full_h[0, 4] *= 2.0 ** 80
    c.full_h[0, 4] *= 2.0 ** 80
    loss, lse = forward(epic, c)
    assert bool(torch.isnan(loss[0, 4])) and int(torch.isfinite(loss).sum()) == 89
    c.full_h[0, 4] = small
    loss2, lse2 = forward(epic, c)
    loss[0, 4], lse[0, 4] = loss2[0, 4], lse2[0, 4]
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    check_rows(epic, c, loss, lse)


# ------------------------------------------------------ heads at odd addresses


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows", [20, 90])
def test_workspace_for_a_head_at_any_address(dtype, rows, epic):  # noqa: F811
    """A workspace made for tensors of these shapes, types and strides does for a head that
    lies in the middle of a buffer."""
    c = Case(dtype, 1, rows, 5000, 64, share=1.0, seed=16)
    h, seqs, w, y, _, weight = c.on_gpu()
    ws = epic.alloc_head_loss_workspace(h, w)
    ws1 = epic.alloc_head_loss_workspace(h, w, backward=False)
    flat = torch.zeros(5000 * 64 + 1, dtype=DT[dtype], device="cuda")
    odd = flat[1:].view(5000, 64)
    odd.copy_(w)
    out = []
    for head in (w, odd):
        loss, lse = torch.empty((1, rows), device="cuda"), torch.empty((1, rows), device="cuda")
        gh, gw = torch.empty_like(h), torch.empty_like(w)
        epic.head_loss_forward(h, seqs, head, y, loss, lse, ws1)
        epic.head_loss_backward(h, seqs, head, y, lse, weight, gh, gw, ws)
        out.append((loss, lse, gh, gw))
    if dtype != "float32":
        assert all(torch.equal(a, b) for a, b in zip(*out))
        return
    # few float32 rows take other products
    e = by_row(c, out[0][1].double().cpu())[1]
    assert all(bool(((a - b).abs().cpu() <= 4 * e).all()) for a, b in list(zip(*out))[:2])
    assert all(bool(((a - b).abs() <= 1e-5 * a.abs().max()).all()) for a, b in list(zip(*out))[2:])


# ------------------------------------------------------ orders, many rows


@pytest.mark.parametrize("dtype", sorted(DT))
def test_sequences_closer_than_rows(dtype, epic):  # noqa: F811
    """Tensors of [m, B, d] turned round give what others do."""
    c = Case(dtype, 5, 40, 260, 72, share=0.7, seed=17)
    h, seqs, w, y, _, weight = c.on_gpu()
    B, m, V, d = c.B, c.m, c.V, c.d
    turned = h.transpose(0, 1).contiguous().transpose(0, 1)
    assert turned.stride(0) == d and turned.stride(1) == B * d
    out = []
    for x in (h, turned):
        loss, lse = torch.empty((B, m), device="cuda"), torch.empty((B, m), device="cuda")
        gh = torch.full((m, B, d), 7.0, dtype=DT[dtype], device="cuda").transpose(0, 1) if x is turned else torch.full_like(h, 7.0)
        gw = torch.empty_like(w)
        ws = epic.alloc_head_loss_workspace(x, w)
        epic.head_loss_forward(x, seqs, w, y, loss, lse, ws)
        epic.head_loss_backward(x, seqs, w, y, lse, weight, gh, gw, ws)
        q, s = epic.alloc_q8(V, d)
        epic.quantize(w, q, s)
        logits = torch.full((m, B, V), 3.0, device="cuda").transpose(0, 1) if x is turned else torch.full((B, m, V), 3.0, device="cuda")
        keep = torch.from_numpy(c.on).cuda()
        z = torch.where(keep[..., None], x, torch.zeros((), dtype=x.dtype, device="cuda")) if x is h else \
            torch.where(keep[..., None], x, torch.zeros((), dtype=x.dtype, device="cuda")).transpose(0, 1).contiguous().transpose(0, 1)
        epic.logits_q8(z, seqs, q, s, logits, epic.alloc_logits_q8_workspace(z))
        out.append((loss, lse, gh, gw, logits))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert bool((out[0][4] == 3).any()) and bool((out[0][4] != 3).any())
    # and the gradient over hidden states that lie so
    ws = epic.alloc_head_loss_workspace(turned, w)
    gw = torch.empty_like(w)
    epic.head_loss_backward(turned, seqs, w, y, out[0][1], weight, turned, gw, ws)
    assert torch.equal(turned, out[0][2]) and torch.equal(gw, out[0][3])


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("size", [(4, 250, 20096, 256, 0.9), (4, 700, 20011, 264, 0.9), (9, 700, 26000, 72, 0.95), (3, 100, 4992, 1088, 1.0)], ids=str)
def test_losses_of_many_rows(dtype, size, epic):  # noqa: F811
    """Every size of tile, several pieces of the vocabulary; 0 in rows that do not count."""
    B, m, V, d, share = size
    c = Case(dtype, B, m, V, d, share=share, seed=18)
    loss, lse = forward(epic, c)
    on = torch.from_numpy(c.on).cuda()
    h, w, y = cut_on(c)
    l = h @ w.t()
    want = torch.logsumexp(l, -1)
    A = float((h.abs() @ w.abs().t()).max())
    e = (8 * math.sqrt(d) * U32 + (2.0 ** -22 if dtype == "float32" else 0.0)) * A + 2e-5
    assert float((lse[on] - want).abs().max()) <= e
    assert float((loss[on] - (want - l.gather(1, y[:, None])[:, 0])).abs().max()) <= 2 * e
    assert not bool(loss[~on].any()) and not bool(lse[~on].any())


def cut_on(c):
    on = torch.from_numpy(c.on)
    return c.h[on].double().cuda(), c.w.double().cuda(), c.target[on].long().cuda()
