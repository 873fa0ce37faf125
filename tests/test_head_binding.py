"""What the operators between hidden states and logits refuse (CPU: the checks
come before any device work), through the C ABI and the binding."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2606_00722_amd import epic  # noqa: E402

F32, F16, BF16 = 0, 1, 2
NULL, ARG, CAPACITY, UNSUPPORTED = -1, -2, -3, -9
AT = 1 << 20  # an address that nothing reads


def rows(dtype=BF16, batch=2, rows=3, vocab=64, data=AT, seq=None, row=None):
    row = vocab if row is None else row
    return epic._Rows(data, dtype, batch, rows, vocab, rows * row if seq is None else seq, row)


def ref(x):
    return None if x is None else ctypes.byref(x)


def quantize(x, q=AT, stride=128, scale=AT):
    return epic.lib().epic_quantize_rows(ref(x), q, stride, scale, 0)


def logits(x, out, q=AT, stride=128, scale=AT, n=0, seqs=0, ws=AT, bytes=1 << 30):
    return epic.lib().epic_logits_q8(ref(x), seqs, n, 0, q, stride, scale, ref(out), ws, bytes, 0)


def forward(x, w, target=AT, loss=AT, lse=AT, n=0, seqs=0, ws=AT, bytes=1 << 40):
    return epic.lib().epic_head_loss_forward(ref(x), seqs, n, 0, ref(w), target, loss, lse, ws, bytes, 0)


def backward(x, w, gh, gw, target=AT, lse=AT, ws=AT, bytes=1 << 40):
    return epic.lib().epic_head_loss_backward(ref(x), 0, 0, 0, ref(w), target, lse, 0, ref(gh), ref(gw), ws, bytes, 0)


def head(**kw):
    return rows(**{"batch": 1, "rows": 100, **kw})


def test_quantize_refuses():
    assert quantize(None) == NULL
    assert quantize(rows(dtype=3)) == ARG
    assert quantize(rows(vocab=0)) == ARG
    assert quantize(rows(data=AT + 1)) == ARG
    assert quantize(rows(data=0)) == NULL
    assert quantize(rows(vocab=65537), stride=65664) == UNSUPPORTED
    assert quantize(rows(batch=1 << 13, rows=1 << 12)) == UNSUPPORTED
    assert quantize(rows(vocab=129), stride=128) == ARG
    assert quantize(rows(), stride=192) == ARG
    assert quantize(rows(), stride=1 << 40) == ARG
    assert quantize(rows(), q=AT + 8) == ARG
    assert quantize(rows(), q=0) == NULL
    assert quantize(rows(), scale=0) == NULL
    assert quantize(rows(batch=0), q=0, scale=0) == 0
    assert quantize(rows(rows=0), q=0, scale=0) == 0


def test_logits_refuses():
    x, out = rows(), rows(vocab=1000)
    assert logits(None, out) == NULL and logits(x, None) == NULL
    assert logits(x, rows(vocab=1000, rows=4)) == ARG
    assert logits(x, rows(vocab=1000, batch=3)) == ARG
    assert logits(x, rows(vocab=1000, row=999, seq=5000)) == ARG  # overlapping rows
    assert logits(x, rows(vocab=262145)) == UNSUPPORTED
    assert logits(x, out, stride=256) == ARG
    assert logits(x, out, q=0) == NULL and logits(x, out, scale=0) == NULL and logits(x, out, ws=0) == NULL
    assert logits(x, out, q=AT + 4) == ARG and logits(x, out, ws=AT + 64) == ARG
    assert logits(x, out, seqs=AT, n=0) == ARG
    need = epic.lib().epic_logits_q8_workspace_bytes(ref(x))
    assert need > 0 and logits(x, out, bytes=need - 1) == CAPACITY
    assert epic.lib().epic_logits_q8_workspace_bytes(ref(rows(vocab=65537))) == 0
    assert epic.lib().epic_logits_q8_workspace_bytes(None) == 0
    assert logits(rows(batch=0), rows(batch=0, vocab=9), q=0, scale=0, ws=0) == 0


def test_loss_refuses():
    x, w = rows(), head()
    assert forward(None, w) == NULL and forward(x, None) == NULL
    for bad in (head(dtype=F16), head(vocab=65), head(batch=2), head(rows=0)):
        assert forward(x, bad) == ARG
        assert epic.lib().epic_head_loss_workspace_bytes(ref(x), ref(bad), 1) == 0
    assert forward(x, head(rows=262145)) == UNSUPPORTED
    assert forward(rows(vocab=65537), head(vocab=65537)) == UNSUPPORTED
    assert forward(rows(batch=1 << 12, rows=(1 << 12) + 1), w) == UNSUPPORTED
    assert forward(x, w, target=0) == NULL and forward(x, w, loss=0) == NULL and forward(x, w, lse=0) == NULL
    assert forward(x, w, ws=0) == NULL and forward(x, w, ws=AT + 128) == ARG
    assert forward(x, w, seqs=AT, n=0) == ARG
    need = epic.lib().epic_head_loss_workspace_bytes(ref(x), ref(w), 0)
    assert need > 0 and forward(x, w, bytes=need - 1) == CAPACITY
    assert forward(rows(batch=0), w, target=0, loss=0, lse=0, ws=0) == 0


def test_gradients_refuse():
    x, w = rows(), head()
    gh, gw = rows(), head()
    assert backward(x, w, None, None) == NULL
    assert backward(x, w, rows(dtype=F16), gw) == ARG and backward(x, w, gh, head(dtype=F16)) == ARG
    assert backward(x, w, rows(rows=2), gw) == ARG and backward(x, w, gh, head(rows=99)) == ARG
    assert backward(x, w, rows(row=63, seq=900), gw) == ARG and backward(x, w, gh, head(row=63)) == ARG
    assert backward(x, w, gh, gw, lse=0) == NULL and backward(x, w, gh, gw, target=0) == NULL
    assert backward(x, w, gh, gw, ws=0) == NULL
    need = epic.lib().epic_head_loss_workspace_bytes(ref(x), ref(w), 1)
    assert need >= epic.lib().epic_head_loss_workspace_bytes(ref(x), ref(w), 0)
    # what the forward pass needs may be more than what the gradients do
    assert backward(x, w, gh, gw, bytes=1 << 10) == CAPACITY
    assert backward(rows(batch=0), w, rows(batch=0), None, target=0, lse=0, ws=0) == 0


def test_binding_refuses_tensors():
    h, w = torch.zeros(1, 2, 64), torch.zeros(9, 64)
    y = torch.zeros(1, 2, dtype=torch.int32)
    f = torch.zeros(1, 2)
    ws = torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(ValueError, match="hidden"):
        epic.head_loss_forward(h, None, w, y, f, f, ws)  # not on a GPU
    with pytest.raises(ValueError, match="hidden"):
        epic.head_loss_backward(h[0], None, w, y, f, None, h, w, ws)
    with pytest.raises(ValueError, match="hidden"):
        epic.logits_q8(h.double(), None, None, None, h, ws)
    with pytest.raises(ValueError, match="x"):
        epic.quantize(h, None, None)
    with pytest.raises(ValueError, match="hidden"):
        epic.alloc_head_loss_workspace(h, w)
    with pytest.raises(ValueError, match="hidden"):
        epic.alloc_logits_q8_workspace(h)
    assert [epic.q8_width(d) for d in (1, 128, 129)] == [128, 128, 256]
    q, s = epic.alloc_q8(7, 130, device="cpu")
    assert q.shape == (7, 256) and q.dtype is torch.int8 and s.shape == (7,)
