"""The distillation loss on the host: the C ABI and its mirror, sizes, refusals
before anything touches a GPU, and the oracle's pins."""

import math
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
    decls = dict(re.findall(r"\b(bdscan_distill_loss_\w+)\s*\(([^)]*)\)", text))
    assert sorted(decls) == sorted(n for n, _, _ in b.DISTILL_SIGNATURES)
    for name, _, args in b.DISTILL_SIGNATURES:
        assert hasattr(b, name) and len(decls[name].split(",")) == len(args), name
    for debug in (False, True):
        assert all(hasattr(b.load(debug=debug), n) for n, _, _ in b.DISTILL_SIGNATURES)


def _dims(**kw):
    a = dict(rows=100, d_model=64, vocab=1000, top=8, dtype=b.BDSCAN_BF16)
    a.update(kw)
    return b.make_distill_loss_dims(**a)


def _fwd(d, h=FAKE, w=FAKE, ids=FAKE, t=FAKE, wt=None, loss=FAKE, lse=FAKE, z=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_distill_loss_forward(d, h, w, ids, t, wt, loss, lse, z, ws, n, None)


def _bwd(d, h=FAKE, w=FAKE, ids=FAKE, t=FAKE, wt=None, lse=FAKE, z=FAKE, dl=None, dh=FAKE, dw=FAKE, ws=FAKE, n=1 << 40):
    return b.bdscan_distill_loss_backward(d, h, w, ids, t, wt, lse, z, dl, dh, dw, ws, n, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), b.BDSCAN_ERR_ARG, "negative rows"),
    (dict(d_model=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(vocab=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(dtype=3), b.BDSCAN_ERR_ARG, "bad dtype"),
    (dict(excluded=-2), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(excluded=1000), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(ld_h=63), b.BDSCAN_ERR_ARG, "ld_h is below"),
    (dict(vocab=1 << 25), b.BDSCAN_ERR_UNSUPPORTED, "above 2^24"),
    (dict(top=0), b.BDSCAN_ERR_ARG, "top must be positive"),
    (dict(top=65), b.BDSCAN_ERR_UNSUPPORTED, "top above 64"),
    (dict(temperature=0.0), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=-2.0), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=math.nan), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=math.inf), b.BDSCAN_ERR_ARG, "temperature"),
])
def test_refuses_bad_dims(kw, code, msg):
    d = _dims(**kw)
    assert _fwd(d) == code and msg in b.bdscan_last_error()
    assert _bwd(d) == code and msg in b.bdscan_last_error()
    assert b.bdscan_distill_loss_forward_workspace_size(d) == 0
    assert b.bdscan_distill_loss_backward_workspace_size(d) == 0


def test_refuses_bad_pointers():
    d = _dims()
    assert _fwd(None) == b.BDSCAN_ERR_ARG and _bwd(None) == b.BDSCAN_ERR_ARG
    for kw, msg in ((dict(h=None), "h is NULL"), (dict(w=FAKE + 8), "w is not"), (dict(ids=None), "ids is NULL"),
                    (dict(t=FAKE + 4), "teacher is not"), (dict(wt=FAKE + 4), "weight is not"),
                    (dict(loss=None), "loss is NULL"), (dict(lse=None), "lse is NULL"), (dict(z=None), "z is NULL"),
                    (dict(n=1), "needed"), (dict(ws=None), "workspace is NULL")):
        assert _fwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    for kw, msg in ((dict(h=None), "h is NULL"), (dict(w=FAKE + 8), "w is not"), (dict(ids=FAKE + 8), "ids is not"),
                    (dict(t=None), "teacher is NULL"), (dict(dl=FAKE + 4), "dloss is not"),
                    (dict(lse=None), "lse is NULL"), (dict(z=None), "z is NULL"), (dict(dh=None), "dh is NULL"),
                    (dict(dw=None), "dw is NULL"), (dict(n=1), "needed")):
        assert _bwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    need = b.bdscan_distill_loss_forward_workspace_size(d)
    assert _fwd(d, n=need - 1) == b.BDSCAN_ERR_ARG and str(need) in b.bdscan_last_error()
    assert _fwd(_dims(rows=0), *[None] * 4, loss=None, lse=None, z=None, ws=None, n=0) == b.BDSCAN_OK


def test_workspace_holds_pieces_not_logits():
    d = _dims(rows=16384, d_model=832, vocab=50304, top=64)
    logits = 16384 * 50304 * 2
    assert b.bdscan_distill_loss_forward_workspace_size(d) < logits // 10
    assert b.bdscan_distill_loss_backward_workspace_size(d) < logits // 3


def test_holder_refuses(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2607_02805_gb300.dense import DistillLoss
    op = DistillLoss(4, 8, 16, 2, device="cpu")
    h, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(16, 8, dtype=torch.bfloat16)
    ids, t = torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2)
    for bad, msg in ((dict(h=h[:3]), "h has shape"), (dict(h=h.float()), "h has dtype"),
                     (dict(h=h[:1].expand(4, 8)), "rows of h overlap"), (dict(w=w[:8]), "w has shape"),
                     (dict(ids=ids.int()), "ids has dtype"), (dict(ids=ids[:, :1]), "ids has shape"),
                     (dict(ids=ids.t().contiguous().t()), "ids is not contiguous"),
                     (dict(teacher=t.bfloat16()), "teacher has dtype"), (dict(weight=t[0]), "weight has shape")):
        with pytest.raises(ValueError, match=msg):
            op.forward(**{**dict(h=h, w=w, ids=ids, teacher=t), **bad})
    with pytest.raises(ValueError, match="needs a forward"):
        op.backward(h, w, ids, t)
    monkeypatch.setattr(b, "_stream", lambda stream: None)
    op._buf["z"] = t
    with pytest.raises(ValueError, match="teacher is a buffer that this call writes"):
        op.forward(h, w, ids, t)
    op._buf["lse"], op._buf["dh"] = t, h
    with pytest.raises(ValueError, match="h is a buffer that this call writes"):
        op.backward(h, w, ids, torch.zeros(4, 2))


def _rand(rng, t=5, k=4, v=9, n=3):
    ids = np.stack([rng.permutation(v)[:n] for _ in range(t)])
    return (rng.normal(size=(t, k)), rng.normal(size=(v, k)), ids, rng.normal(size=(t, n)),
            rng.random(t) + 0.5, rng.normal(size=t))


def test_oracle_against_differences():
    rng = np.random.default_rng(0)
    h, w, ids, teacher, weight, dloss = _rand(rng)
    ids[0, 1], ids[1, 2], weight[2], ids[3, 1] = -1, 8, 0.0, ids[3, 0]
    grads = od.distill_loss_backward(h, w, ids, teacher, weight, dloss, 8, 1.7)
    for place, grad in enumerate(grads):
        for at in np.ndindex(grad.shape):
            lo, hi = [h.copy(), w.copy()], [h.copy(), w.copy()]
            lo[place][at] -= 1e-6
            hi[place][at] += 1e-6
            a, c = (od.distill_loss_forward(*x, ids, teacher, weight, 8, 1.7)[0] for x in (lo, hi))
            assert abs(((c - a) * dloss).sum() / 2e-6 - grad[at]) < 1e-7


def test_oracle_identities():
    rng = np.random.default_rng(1)
    h, w, ids, teacher, weight, dloss = _rand(rng, n=1)
    # one entry: the vocabulary loss of that target
    a = od.distill_loss_forward(h, w, ids, teacher, weight, 8)
    c = od.lm_loss_forward(h, w, ids[:, 0], np.where(ids[:, 0] == 8, 0, weight), 8)
    np.testing.assert_allclose(a[0], c[0], rtol=1e-13)
    np.testing.assert_allclose(a[1], c[1], rtol=1e-13)
    # everything known and equal: no loss and no gradient, at any temperature
    ids = np.tile(np.arange(9), (5, 1))
    z = h @ w.T
    for temperature in (0.5, 3.0):
        assert np.abs(od.distill_loss_forward(h, w, ids, z, weight, -1, temperature)[0]).max() < 1e-14
        for g in od.distill_loss_backward(h, w, ids, z, weight, dloss, -1, temperature):
            assert np.abs(g).max() < 1e-14
    # a teacher's constant does not matter, and an entry of minus infinity is none
    x = rng.normal(size=(5, 9))
    y = np.concatenate((x + 3.0, np.full((5, 1), -np.inf)), 1)
    more = np.concatenate((ids, np.full((5, 1), 4)), 1)
    np.testing.assert_allclose(od.distill_loss_forward(h, w, ids, x, weight)[0],
                               od.distill_loss_forward(h, w, more, y, weight)[0], rtol=1e-13)
