"""The holders of the dense operators and the marshalling below them, on the
host: which tensors they refuse before an address reaches the library."""

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
