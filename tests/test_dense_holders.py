"""The holders of the dense operators and the marshalling below them, on the
host: which tensors they refuse before an address reaches the library."""

import gc
import weakref

import pytest

torch = pytest.importorskip("torch")

from paper_2607_02805_gb300 import binding as b  # noqa: E402
from paper_2607_02805_gb300 import dense  # noqa: E402

B = torch.bfloat16


class Reached(Exception):
    """The library would have been called."""


@pytest.fixture
def no_library(monkeypatch):
    def call(name, *args):
        raise Reached(name)

    monkeypatch.setattr(b, "_call", call)
    monkeypatch.setattr(b, "_stream", lambda stream: None)


def _expanded(rows, cols):
    return torch.zeros(1, cols, dtype=B).expand(rows, cols)


def _overlapping(rows, cols):
    return torch.zeros(rows * cols, dtype=B).as_strided((rows, cols), (cols - 1, 1))


def _column(rows, cols):
    """One element for all rows of a tensor of a single column."""
    return torch.zeros(1, 1, dtype=B).expand(rows, 1)


@pytest.mark.parametrize("rows", [4, 64])
@pytest.mark.parametrize("make", [_expanded, _overlapping])
def test_holders_refuse_rows_that_overlap(rows, make, no_library):
    """A row stride of 0 means "the row length" below: the library would read (or write) rows * width elements."""
    op = dense.Linear(rows, 8, 16, "none", B, device="cpu")
    x, w, y = torch.zeros(rows, 8, dtype=B), torch.zeros(16, 8, dtype=B), torch.zeros(rows, 16, dtype=B)
    for kw, name in ((dict(x=make(rows, 8)), "x"), (dict(x=x, residual=make(rows, 16)), "residual"),
                     (dict(x=x, out=make(rows, 16)), "out")):
        with pytest.raises(ValueError, match=f"rows of {name} overlap"):
            op.forward(w=w, **kw)
    for a, dy, name in ((make(rows, 8), y, "x"), (x, make(rows, 16), "dy")):
        with pytest.raises(ValueError, match=f"rows of {name} overlap"):
            op.backward(a, w, dy)
    ls = dense.LmLoss(rows, 8, 16, B, device="cpu")
    t = torch.zeros(rows, dtype=torch.int64)
    for call in (lambda h: ls.forward(h, w, t), lambda h: ls.backward(h, w, t, lse=torch.zeros(rows))):
        with pytest.raises(ValueError, match="rows of h overlap"):
            call(make(rows, 8))


def test_holders_refuse_one_element_for_all_rows(no_library):
    op = dense.Linear(4, 1, 16, "none", B, device="cpu")
    with pytest.raises(ValueError, match="rows of x overlap"):
        op.forward(_column(4, 1), torch.zeros(16, 1, dtype=B))


def test_holders_take_rows_of_their_own(no_library):
    """What a row stride may be: the length, more than that, anything where there is one row."""
    for x in (torch.zeros(4, 8, dtype=B), torch.zeros(4, 24, dtype=B)[:, 8:16], torch.zeros(1, 8, dtype=B).expand(1, 8),
              torch.zeros(8, dtype=B).as_strided((1, 8), (0, 1))):
        with pytest.raises(Reached):
            dense.Linear(x.shape[0], 8, 16, "none", B, device="cpu").forward(x, torch.zeros(16, 8, dtype=B))


def test_binding_refuses_rows_that_overlap():
    for t in (_expanded(4, 8), _overlapping(4, 8), _column(4, 1)):
        with pytest.raises(ValueError, match="overlap"):
            b.row_stride(t)
        with pytest.raises(ValueError, match="overlap"):
            b._ptr2(t)
    assert b.row_stride(torch.zeros(4, 24)[:, :8]) == 24
    assert b.row_stride(torch.zeros(1, 8).expand(1, 8)) == 8 and b.row_stride(torch.zeros(1, 1)) == 1


# ---------------------------------------------------------------------------
# workspaces and streams
# ---------------------------------------------------------------------------
class FakeStream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def fake_streams(monkeypatch):
    """Calls that reach the library are noted with their workspace and stream; a list of (stream, bytes) allocated and
    one of (address, stream) marked."""
    calls, allocated, marked, within = [], [], [], [None]
    empty = torch.empty

    class stream:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            self.before, within[0] = within[0], self.s

        def __exit__(self, *exc):
            within[0] = self.before

    def note_empty(*args, **kw):
        t = empty(*args, **kw)
        allocated.append((within[0], t.data_ptr()))
        return t

    monkeypatch.setattr(b, "_call", lambda name, *args: calls.append((name,) + args[-3:]))
    monkeypatch.setattr(b, "_stream", lambda s: None if s is None else s.cuda_stream)
    monkeypatch.setattr(torch, "empty", note_empty)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: marked.append((t.data_ptr(), s)))
    return calls, allocated, marked


def _step(op, forward, backward, stream=None):
    x, w = torch.zeros(300, 448), torch.zeros(1792, 448)
    if forward:
        op.forward(x, w, save_pre=True, stream=stream)
    if backward:
        op.backward(x, w, torch.zeros(300, 1792), stream=stream)


def test_outgrown_workspaces_are_kept(fake_streams):
    """The backward needs more than the forward; work of the forward, or a graph of it, may still use the first one."""
    calls, _, _ = fake_streams
    op = dense.Linear(300, 448, 1792, "gelu", torch.float32, device="cpu")
    _step(op, True, False)
    first = weakref.ref(op._buf["workspace"])
    _step(op, False, True)
    gc.collect()
    (_, a, n, _), (_, c, m, _) = calls
    assert m > n and a != c
    assert first() is not None and first().data_ptr() == a and first().numel() == n
    _step(op, True, True)  # later calls use the larger one
    assert all(q[1:3] == (c, m) for q in calls[2:])


def test_a_row_stride_that_needs_more_keeps_the_first_workspace(fake_streams):
    calls, _, _ = fake_streams
    op = dense.Linear(200, 64, 128, "none", B, device="cpu")
    w = torch.zeros(128, 64, dtype=B)
    op.forward(torch.zeros(200, 69, dtype=B)[:, :64], w)
    first = weakref.ref(op._buf["workspace"])
    op.backward(torch.zeros(200, 69, dtype=B)[:, :64], w, torch.zeros(200, 133, dtype=B)[:, :128])
    gc.collect()
    assert calls[1][2] > calls[0][2] and first() is not None


def test_buffers_come_from_the_stream_of_the_call(fake_streams):
    calls, allocated, marked = fake_streams
    op = dense.Linear(300, 448, 1792, "gelu", torch.float32, device="cpu")
    _step(op, True, False, FakeStream(5))
    assert allocated and {s for s, _ in allocated if s is not None} == {5} and not marked
    held = {t.data_ptr() for t in op._buf.values()}
    assert held <= {p for s, p in allocated if s == 5}
    before = len(allocated)
    _step(op, True, True, FakeStream(6))  # what the first stream allocated is used on the second
    assert held <= {p for p, s in marked if s == 6}
    grown = {t.data_ptr() for t in op._buf.values()} - held
    assert grown and grown <= {p for s, p in allocated[before:] if s == 6}
    marks = len(marked)
    _step(op, True, True, FakeStream(6))
    assert len(marked) == marks and [c[-1] for c in calls] == [5, 6, 6, 6, 6]


def test_loss_buffers_come_from_the_stream_of_the_call(fake_streams):
    calls, allocated, _ = fake_streams
    op = dense.LmLoss(40, 8, 16, B, device="cpu")
    h, w, t = torch.zeros(40, 8, dtype=B), torch.zeros(16, 8, dtype=B), torch.zeros(40, dtype=torch.int64)
    op.forward(h, w, t, stream=FakeStream(5))
    op.backward(h, w, t, stream=FakeStream(5))
    assert {t.data_ptr() for t in op._buf.values()} <= {p for s, p in allocated if s == 5}
    assert [c[-1] for c in calls] == [5, 5]


def test_holders_refuse_another_current_device(fake_streams, monkeypatch):
    """Kernels are launched on the current device: a holder of another one would hand them that device's addresses."""
    calls, allocated, _ = fake_streams
    op = dense.Linear(4, 8, 16, "none", B, device="cuda:1")
    ls = dense.LmLoss(4, 8, 16, B, device="cuda:1")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(dense, "_rows", lambda name, t, shape, dtype, index: (1 << 20, shape[1]))
    monkeypatch.setattr(dense, "_whole", lambda *args: 1 << 20)
    for call in (lambda: op.forward(None, None), lambda: op.backward(None, None, None),
                 lambda: ls.forward(None, None, None), lambda: ls.backward(None, None, None, lse=1),
                 lambda: op.forward(None, None, stream=FakeStream(5))):
        with pytest.raises(ValueError, match="holder is on cuda:1, the current device is cuda:0"):
            call()
    assert not calls and not allocated


def test_holders_refuse_what_the_call_writes(fake_streams):
    """A result is the holder's buffer: as the next call's input it would be read while it is written."""
    calls, _, _ = fake_streams
    op = dense.Linear(4, 8, 8, "none", B, device="cpu")
    x, w, dy = torch.zeros(4, 8, dtype=B), torch.zeros(8, 8, dtype=B), torch.zeros(4, 8, dtype=B)
    y = op.forward(x, w)
    dx, dw, _ = op.backward(x, w, dy)
    ls = dense.LmLoss(4, 8, 8, B, device="cpu")
    t = torch.zeros(4, dtype=torch.int64)
    ls.forward(x, w, t)
    dh, dhead = ls.backward(x, w, t)
    n = len(calls)
    for call, name in ((lambda: op.forward(y, w), "x"), (lambda: op.forward(x, w, out=x), "x"),
                       (lambda: op.backward(dx, w, dy), "x"), (lambda: op.backward(x, w, dx), "dy"),
                       (lambda: op.backward(x, dw, dy), "w"), (lambda: ls.backward(dh, w, t), "h"),
                       (lambda: ls.backward(x, dhead, t), "w")):
        with pytest.raises(ValueError, match=f"^{name} is a buffer that this call writes"):
            call()
    assert len(calls) == n
    # read before it is written, written by no product of the call, or another holder's
    op.forward(x, w, residual=y)
    op.forward(dx, w)
    op.backward(y, w, dy, need_dx=False)
    op.backward(x, w, dx, need_dx=False)
    dense.Linear(4, 8, 8, "none", B, device="cpu").forward(y, w)
    empty = dense.Linear(0, 8, 8, "none", B, device="cpu")
    empty.forward(torch.zeros(0, 8, dtype=B), w)
    assert len(calls) == n + 6
