"""The C ABI of the dense operators on the host: every function of
include/bdscan_dense.h is exported and mirrored, sizes are answered, and bad
arguments are refused before anything touches a GPU."""

import os
import re

import pytest

from paper_2607_02805_gb300 import binding as b

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "bdscan_dense.h")
FAKE = 1 << 20  # an aligned address that is never dereferenced on the error paths


def test_header_binding_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    decls = dict(re.findall(r"\b(bdscan_(?:linear|lm_loss)_\w+)\s*\(([^)]*)\)", text))
    decls = {k: v for k, v in decls.items()}
    assert sorted(decls) == sorted(n for n, _, _ in b.DENSE_SIGNATURES)
    for name, _, args in b.DENSE_SIGNATURES:
        assert hasattr(b.load(), name) and hasattr(b, name)
        assert len(decls[name].split(",")) == len(args), name
    for debug in (False, True):
        assert all(hasattr(b.load(debug=debug), n) for n, _, _ in b.DENSE_SIGNATURES)


def _lin(**kw):
    a = dict(rows=100, d_in=64, d_out=96, act=b.BDSCAN_ACT_GELU, dtype=b.BDSCAN_BF16)
    a.update(kw)
    return b.make_linear_dims(**a)


def _fwd(d, x=FAKE, w=FAKE, bias=None, res=None, pre=None, y=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_linear_forward(d, x, w, bias, res, pre, y, ws, n, None)


def _bwd(d, x=FAKE, w=FAKE, pre=FAKE, dy=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_linear_backward(d, x, w, pre, dy, dx, dw, db, ws, n, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), b.BDSCAN_ERR_ARG, "negative rows"),
    (dict(d_in=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(d_out=-3), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(dtype=7), b.BDSCAN_ERR_ARG, "bad dtype"),
    (dict(out_dtype=7), b.BDSCAN_ERR_ARG, "bad out_dtype"),
    (dict(dtype=b.BDSCAN_F32, out_dtype=b.BDSCAN_BF16), b.BDSCAN_ERR_UNSUPPORTED, "f32 inputs"),
    (dict(act=9), b.BDSCAN_ERR_ARG, "bad act"),
    (dict(ld_x=63), b.BDSCAN_ERR_ARG, "ld_x is below d_in"),
    (dict(ld_res=95), b.BDSCAN_ERR_ARG, "ld_res is below d_out"),
    (dict(ld_y=95), b.BDSCAN_ERR_ARG, "ld_y is below d_out"),
    (dict(rows=1 << 31), b.BDSCAN_ERR_UNSUPPORTED, "rows above"),
    (dict(d_in=1 << 25), b.BDSCAN_ERR_UNSUPPORTED, "above 2^24"),
    (dict(ld_x=1 << 31), b.BDSCAN_ERR_UNSUPPORTED, "row stride"),
])
def test_linear_refuses_bad_dims(kw, code, msg):
    d = _lin(**kw)
    assert _fwd(d) == code and msg in b.bdscan_last_error()
    assert _bwd(d) == code and msg in b.bdscan_last_error()
    assert b.bdscan_linear_forward_workspace_size(d) == 0
    assert b.bdscan_linear_backward_workspace_size(d) == 0


def test_linear_refuses_bad_pointers():
    d = _lin()
    assert b.bdscan_linear_forward(None, *[FAKE] * 7, 1 << 40, None) == b.BDSCAN_ERR_ARG
    for kw, msg in ((dict(x=None), "x is NULL"), (dict(w=FAKE + 8), "w is not 16-byte aligned"),
                    (dict(bias=FAKE + 2), "bias is not"), (dict(res=FAKE + 4), "residual is not"),
                    (dict(pre=FAKE + 1), "pre is not"), (dict(y=None), "y is NULL")):
        assert _fwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    for kw, msg in ((dict(x=None), "x is NULL"), (dict(w=None), "w is NULL"), (dict(pre=None), "pre is NULL"),
                    (dict(dy=None), "dy is NULL"), (dict(dx=FAKE + 8), "dx is not"), (dict(dw=FAKE + 8), "dw is not"),
                    (dict(db=FAKE + 8), "dbias is not")):
        assert _bwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    need = b.bdscan_linear_backward_workspace_size(d)
    assert need > 0
    assert _bwd(d, n=need - 1) == b.BDSCAN_ERR_ARG and "needed" in b.bdscan_last_error()
    assert _bwd(d, ws=None) == b.BDSCAN_ERR_ARG and "workspace is NULL" in b.bdscan_last_error()


def test_linear_sizes():
    # aligned bf16 that fills the SMs reads its operands where they lie
    assert b.bdscan_linear_forward_workspace_size(_lin(rows=16384, d_in=832, d_out=3328)) == 0
    # a few rows need nothing, whatever the alignment
    assert b.bdscan_linear_forward_workspace_size(_lin(rows=8, d_in=451, d_out=33)) == 0
    # odd d_in: copies of x and w with rows of whole 16 bytes
    n = b.bdscan_linear_forward_workspace_size(_lin(rows=16384, d_in=451, d_out=3328))
    assert n == 16384 * 456 * 2 + 3328 * 456 * 2
    # fp32: three pieces
    n = b.bdscan_linear_forward_workspace_size(_lin(rows=16384, d_in=448, d_out=3328, dtype=b.BDSCAN_F32))
    assert n == 3 * (16384 + 3328) * 448 * 2
    # no rows: nothing to do, and no pointer is looked at
    d = _lin(rows=0)
    assert b.bdscan_linear_forward_workspace_size(d) == 0
    assert _fwd(d, x=None, w=None, y=None, ws=None, n=0) == b.BDSCAN_OK


def _loss(**kw):
    a = dict(rows=100, d_model=64, vocab=1000, dtype=b.BDSCAN_BF16)
    a.update(kw)
    return b.make_lm_loss_dims(**a)


def _lf(d, h=FAKE, w=FAKE, t=FAKE, wt=None, loss=FAKE, lse=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_lm_loss_forward(d, h, w, t, wt, loss, lse, ws, n, None)


def _lb(d, h=FAKE, w=FAKE, t=FAKE, wt=None, lse=FAKE, dl=None, dh=FAKE, dw=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_lm_loss_backward(d, h, w, t, wt, lse, dl, dh, dw, ws, n, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), b.BDSCAN_ERR_ARG, "negative rows"),
    (dict(d_model=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(vocab=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(dtype=3), b.BDSCAN_ERR_ARG, "bad dtype"),
    (dict(excluded=-2), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(excluded=1000), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(ld_h=63), b.BDSCAN_ERR_ARG, "ld_h is below"),
    (dict(vocab=1 << 25), b.BDSCAN_ERR_UNSUPPORTED, "above 2^24"),
])
def test_loss_refuses_bad_dims(kw, code, msg):
    d = _loss(**kw)
    assert _lf(d) == code and msg in b.bdscan_last_error()
    assert _lb(d) == code and msg in b.bdscan_last_error()
    assert b.bdscan_lm_loss_forward_workspace_size(d) == 0
    assert b.bdscan_lm_loss_backward_workspace_size(d) == 0


def test_loss_refuses_bad_pointers():
    d = _loss()
    for kw, msg in ((dict(h=None), "h is NULL"), (dict(w=FAKE + 8), "w is not"), (dict(t=None), "target is NULL"),
                    (dict(wt=FAKE + 4), "weight is not"), (dict(loss=None), "loss is NULL"),
                    (dict(lse=None), "lse is NULL"), (dict(n=1), "needed"), (dict(ws=None), "workspace is NULL")):
        assert _lf(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    for kw, msg in ((dict(h=None), "h is NULL"), (dict(w=None), "w is NULL"), (dict(t=FAKE + 8), "target is not"),
                    (dict(dl=FAKE + 4), "dloss is not"), (dict(lse=None), "lse is NULL"), (dict(dh=None), "dh is NULL"),
                    (dict(dw=None), "dw is NULL"), (dict(n=1), "needed")):
        assert _lb(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw


def test_loss_workspace_holds_pieces_not_logits():
    d = _loss(rows=16384, d_model=832, vocab=50304)
    logits = 16384 * 50304 * 2
    assert b.bdscan_lm_loss_forward_workspace_size(d) < logits // 10
    assert b.bdscan_lm_loss_backward_workspace_size(d) < logits // 3
    assert _lf(_loss(rows=0), h=None, w=None, t=None, loss=None, lse=None, ws=None, n=0) == b.BDSCAN_OK


def test_holders_refuse():
    torch = pytest.importorskip("torch")
    from paper_2607_02805_gb300.dense import Linear, LmLoss
    op = Linear(4, 8, 16, "silu", torch.bfloat16, device="cpu")
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(16, 8, dtype=torch.bfloat16)
    for bad, msg in ((dict(x=x[:3], w=w), "x has shape"), (dict(x=x.float(), w=w), "x has dtype"),
                     (dict(x=x, w=w.t().contiguous().t()), "w is not contiguous"),
                     (dict(x=x.t().contiguous().t(), w=w), "rows of x"),
                     (dict(x=x, w=w, bias=torch.zeros(16)), "bias has dtype"),
                     (dict(x=x, w=w, residual=x), "residual has shape")):
        with pytest.raises(ValueError, match=msg):
            op.forward(**bad)
    with pytest.raises(ValueError, match="save_pre"):
        op.backward(x, w, torch.zeros(4, 16, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="unknown activation"):
        Linear(4, 8, 16, "relu")
    with pytest.raises(ValueError, match="unsupported dtype"):
        Linear(4, 8, 16, dtype=torch.float16)
    ls = LmLoss(4, 8, 16, torch.bfloat16, device="cpu")
    t = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="target has dtype"):
        ls.forward(x, w, t.int())
    with pytest.raises(ValueError, match="forward or its lse"):
        ls.backward(x, w, t)
