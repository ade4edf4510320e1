"""The gated linear layer on the host: the C ABI and its mirror, sizes, refusals
before anything touches a GPU, and the oracle's pins."""

import os
import re

import numpy as np
import pytest

from oracle import dense as od
from paper_2607_02805_gb300 import binding as b

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bdscan_dense.h")
FAKE = 1 << 20  # an aligned address that is never dereferenced on the error paths


def test_header_binding_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decls = dict(re.findall(r"\b(bdscan_gated_linear_\w+)\s*\(([^)]*)\)", text))
    assert sorted(decls) == sorted(n for n, _, _ in b.GATED_SIGNATURES)
    for name, _, args in b.GATED_SIGNATURES:
        assert hasattr(b, name) and len(decls[name].split(",")) == len(args), name
    for debug in (False, True):
        assert all(hasattr(b.load(debug=debug), n) for n, _, _ in b.GATED_SIGNATURES)


def _dims(**kw):
    a = dict(rows=100, d_in=64, d_hidden=96, act=b.BDSCAN_ACT_SILU, dtype=b.BDSCAN_BF16)
    a.update(kw)
    return b.make_gated_linear_dims(**a)


def _fwd(d, x=FAKE, w=FAKE, bias=None, y=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_gated_linear_forward(d, x, w, bias, y, ws, n, None)


def _bwd(d, x=FAKE, w=FAKE, bias=None, dy=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_gated_linear_backward(d, x, w, bias, dy, dx, dw, db, ws, n, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), b.BDSCAN_ERR_ARG, "negative rows"),
    (dict(d_in=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(d_hidden=-3), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(dtype=7), b.BDSCAN_ERR_ARG, "bad dtype"),
    (dict(act=9), b.BDSCAN_ERR_ARG, "bad act"),
    (dict(ld_x=63), b.BDSCAN_ERR_ARG, "ld_x is below d_in"),
    (dict(ld_y=95), b.BDSCAN_ERR_ARG, "ld_y is below d_hidden"),
    (dict(rows=1 << 31), b.BDSCAN_ERR_UNSUPPORTED, "rows above"),
    (dict(d_in=1 << 25), b.BDSCAN_ERR_UNSUPPORTED, "above 2^24"),
    (dict(d_hidden=1 << 24), b.BDSCAN_ERR_UNSUPPORTED, "above 2^23"),
    (dict(ld_y=1 << 31), b.BDSCAN_ERR_UNSUPPORTED, "row stride"),
])
def test_refuses_bad_dims(kw, code, msg):
    d = _dims(**kw)
    assert _fwd(d) == code and msg in b.bdscan_last_error()
    assert _bwd(d) == code and msg in b.bdscan_last_error()
    assert b.bdscan_gated_linear_forward_workspace_size(d) == 0
    assert b.bdscan_gated_linear_backward_workspace_size(d) == 0


def test_refuses_bad_pointers():
    d = _dims()
    assert _fwd(None) == b.BDSCAN_ERR_ARG and _bwd(None) == b.BDSCAN_ERR_ARG
    for kw, msg in ((dict(x=None), "x is NULL"), (dict(w=FAKE + 8), "w is not 16-byte aligned"),
                    (dict(bias=FAKE + 2), "bias is not"), (dict(y=None), "y is NULL")):
        assert _fwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    for kw, msg in ((dict(x=None), "x is NULL"), (dict(w=None), "w is NULL"), (dict(bias=FAKE + 4), "bias is not"),
                    (dict(dy=None), "dy is NULL"), (dict(dx=FAKE + 8), "dx is not"), (dict(dw=FAKE + 8), "dw is not"),
                    (dict(db=FAKE + 8), "dbias is not")):
        assert _bwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    need = b.bdscan_gated_linear_backward_workspace_size(d)
    assert need > 0
    assert _bwd(d, n=need - 1) == b.BDSCAN_ERR_ARG and "needed" in b.bdscan_last_error()
    assert _bwd(d, ws=None) == b.BDSCAN_ERR_ARG and "workspace is NULL" in b.bdscan_last_error()


def test_sizes():
    # aligned bf16 reads its operands where they lie; a few rows need nothing, whatever the alignment
    assert b.bdscan_gated_linear_forward_workspace_size(_dims(rows=16384, d_in=832, d_hidden=3328)) == 0
    assert b.bdscan_gated_linear_forward_workspace_size(_dims(rows=8, d_in=451, d_hidden=33)) == 0
    # odd d_in: copies of x and w with rows of whole 16 bytes; fp32: three pieces
    n = b.bdscan_gated_linear_forward_workspace_size(_dims(rows=16384, d_in=451, d_hidden=3328))
    assert n == 16384 * 456 * 2 + 2 * 3328 * 456 * 2
    n = b.bdscan_gated_linear_forward_workspace_size(_dims(rows=16384, d_in=448, d_hidden=512, dtype=b.BDSCAN_F32))
    assert n == 3 * (16384 + 1024) * 448 * 2
    # no rows: nothing to do, and no pointer is looked at
    d = _dims(rows=0)
    assert b.bdscan_gated_linear_forward_workspace_size(d) == 0
    assert _fwd(d, x=None, w=None, y=None, ws=None, n=0) == b.BDSCAN_OK
    # no gradient asked for
    assert _bwd(_dims(), x=None, w=None, dy=None, dx=None, dw=None, db=None, ws=None, n=0) == b.BDSCAN_OK


def test_holder_refuses(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2607_02805_gb300.dense import GatedLinear
    op = GatedLinear(4, 8, 16, device="cpu")
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(32, 8, dtype=torch.bfloat16)
    for bad, msg in ((dict(x=x[:3], w=w), "x has shape"), (dict(x=x.float(), w=w), "x has dtype"),
                     (dict(x=x, w=w[:16]), "w has shape"), (dict(x=x, w=w.t().contiguous().t()), "w is not contiguous"),
                     (dict(x=x[:1].expand(4, 8), w=w), "rows of x overlap"),
                     (dict(x=x, w=w, bias=torch.zeros(32)), "bias has dtype"),
                     (dict(x=x, w=w, out=x), "out has shape")):
        with pytest.raises(ValueError, match=msg):
            op.forward(**bad)
    with pytest.raises(ValueError, match="dy has shape"):
        op.backward(x, w, x)
    with pytest.raises(ValueError, match="unknown activation"):
        GatedLinear(4, 8, 16, "relu", device="cpu")
    with pytest.raises(ValueError, match="unsupported dtype"):
        GatedLinear(4, 8, 16, dtype=torch.float16, device="cpu")
    monkeypatch.setattr(b, "_stream", lambda stream: None)
    square = GatedLinear(4, 8, 8, device="cpu")
    ws = torch.zeros(16, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="x is a buffer that this call writes"):
        square.forward(x, ws, out=x)


def test_waits_of_the_epilogue_are_bounded():
    """By reading: no loop around a poll without a limit, no barrier that would wait for a warp that has given up, and
    every way out of the loop over tiles says whether one has."""
    root = os.path.dirname(os.path.dirname(HEADER))
    code = re.sub(r"//[^\n]*", "", open(os.path.join(root, "paper_2607_02805_gb300", "csrc", "gemm_gate.cuh")).read())
    assert "try_wait" not in code and "bar.sync" not in code and "__syncthreads" not in code
    assert not re.search(r"while\s*\(", code) and not re.search(r"for\s*\(\s*;\s*;", code)
    assert code.count("warp_wait(") == 2 and "if (!ok) break;" in code and "return ok;" in code


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_oracle_against_differences(act):
    rng = np.random.default_rng(0)
    x, w, bias, dy = rng.normal(size=(3, 5)), rng.normal(size=(8, 5)), rng.normal(size=8), rng.normal(size=(3, 4))
    grads = od.gated_linear_backward(x, w, bias, dy, act)
    for place, grad in enumerate(grads):
        for at in np.ndindex(grad.shape):
            lo, hi = [v.copy() for v in (x, w, bias)], [v.copy() for v in (x, w, bias)]
            lo[place][at] -= 1e-6
            hi[place][at] += 1e-6
            diff = ((od.gated_linear_forward(*hi, act) - od.gated_linear_forward(*lo, act)) * dy).sum() / 2e-6
            assert abs(diff - grad[at]) < 1e-6 * max(1.0, np.abs(grad).max()) * 10


def test_oracle_identities():
    rng = np.random.default_rng(1)
    x, w = rng.normal(size=(4, 6)), rng.normal(size=(10, 6))
    # without an activation the two projections may change places
    swapped = np.concatenate((w[5:], w[:5]))
    np.testing.assert_allclose(od.gated_linear_forward(x, w, None, "none"),
                               od.gated_linear_forward(x, swapped, None, "none"), rtol=1e-14)
    # an up projection of zeros but a bias of one leaves the activation
    w[5:] = 0
    bias = np.concatenate((np.zeros(5), np.ones(5)))
    np.testing.assert_allclose(od.gated_linear_forward(x, w, bias, "silu"), od.act("silu", x @ w[:5].T), rtol=1e-14)
