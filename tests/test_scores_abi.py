"""Token scores on the host: the C ABI and its mirror, refusals before anything
touches a GPU, and the oracle's pins."""

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
    decls = dict(re.findall(r"\b(bdscan_token_scores_\w+)\s*\(([^)]*)\)", text))
    assert sorted(decls) == sorted(n for n, _, _ in b.SCORES_SIGNATURES)
    for name, _, args in b.SCORES_SIGNATURES:
        assert hasattr(b, name) and len(decls[name].split(",")) == len(args), name
    for debug in (False, True):
        assert all(hasattr(b.load(debug=debug), n) for n, _, _ in b.SCORES_SIGNATURES)


def _dims(**kw):
    a = dict(rows=10, vocab=100, top=4, dtype=b.BDSCAN_BF16)
    a.update(kw)
    return b.make_token_scores_dims(**a)


def _fwd(d, z=FAKE, t=FAKE, lp=FAKE, h=FAKE, st=FAKE, ids=FAKE, top=FAKE):
    return b.bdscan_token_scores_forward(d, z, t, lp, h, st, ids, top, None)


def _bwd(d, z=FAKE, t=FAKE, st=FAKE, h=FAKE, dl=FAKE, dh=FAKE, dz=FAKE):
    return b.bdscan_token_scores_backward(d, z, t, st, h, dl, dh, dz, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), b.BDSCAN_ERR_ARG, "negative rows"),
    (dict(vocab=0), b.BDSCAN_ERR_ARG, "must be positive"),
    (dict(dtype=7), b.BDSCAN_ERR_ARG, "bad dtype"),
    (dict(top=-1), b.BDSCAN_ERR_ARG, "negative top"),
    (dict(top=65), b.BDSCAN_ERR_UNSUPPORTED, "top above 64"),
    (dict(excluded=100), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(excluded=-2), b.BDSCAN_ERR_ARG, "excluded"),
    (dict(temperature=0.0), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=-1.0), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=math.nan), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(temperature=math.inf), b.BDSCAN_ERR_ARG, "temperature"),
    (dict(ld_logits=99), b.BDSCAN_ERR_ARG, "ld_logits is below"),
    (dict(ld_dlogits=99), b.BDSCAN_ERR_ARG, "ld_dlogits is below"),
    (dict(rows=1 << 28), b.BDSCAN_ERR_UNSUPPORTED, "rows above"),
    (dict(vocab=1 << 25), b.BDSCAN_ERR_UNSUPPORTED, "vocab above"),
    (dict(ld_logits=1 << 31), b.BDSCAN_ERR_UNSUPPORTED, "row stride"),
])
def test_refuses_bad_dims(kw, code, msg):
    d = _dims(**kw)
    assert _fwd(d) == code and msg in b.bdscan_last_error()
    assert _bwd(d) == code and msg in b.bdscan_last_error()


def test_refuses_bad_pointers():
    d = _dims()
    assert _fwd(None) == b.BDSCAN_ERR_ARG and _bwd(None) == b.BDSCAN_ERR_ARG
    for kw, msg in ((dict(z=None), "logits is NULL"), (dict(z=FAKE + 2), "logits is not 16-byte"),
                    (dict(t=FAKE + 8), "token is not"), (dict(lp=None), "logp is NULL"),
                    (dict(t=None), "logp without token"), (dict(h=FAKE + 4), "entropy is not"),
                    (dict(st=FAKE + 8), "stats is not"), (dict(ids=None), "top_ids is NULL"),
                    (dict(top=None), "top_logp is NULL")):
        assert _fwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    for kw, msg in ((dict(z=None), "logits is NULL"), (dict(t=None), "dlogp without token"),
                    (dict(st=None), "stats is NULL"), (dict(h=None), "entropy is NULL"),
                    (dict(dl=FAKE + 4), "dlogp is not"), (dict(dh=FAKE + 4), "dentropy is not"),
                    (dict(dz=None), "dlogits is NULL")):
        assert _bwd(d, **kw) == b.BDSCAN_ERR_ARG and msg in b.bdscan_last_error(), kw
    # in place, rows that would be written before they are read
    assert _bwd(_dims(ld_dlogits=104)) == b.BDSCAN_ERR_ARG and "another row stride" in b.bdscan_last_error()
    # no rows: no pointer is looked at
    assert _fwd(_dims(rows=0), *[None] * 7) == b.BDSCAN_OK and _bwd(_dims(rows=0), *[None] * 7) == b.BDSCAN_OK


def test_holder_refuses(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2607_02805_gb300.dense import TokenScores
    op = TokenScores(4, 10, 2, device="cpu")
    z, t = torch.zeros(4, 10, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for bad, msg in ((dict(logits=z[:3]), "logits has shape"), (dict(logits=z.float()), "logits has dtype"),
                     (dict(logits=z[:1].expand(4, 10)), "rows of logits overlap"),
                     (dict(logits=z.t().contiguous().t()), "rows of logits are not contiguous"),
                     (dict(logits=z, token=t.int()), "token has dtype")):
        with pytest.raises(ValueError, match=msg):
            op.forward(**bad)
    with pytest.raises(ValueError, match="needs a forward"):
        op.backward(z, t, torch.zeros(4))
    with pytest.raises(ValueError, match="dlogp has dtype"):
        op.backward(z, t, torch.zeros(4).double())
    with pytest.raises(ValueError, match="unsupported dtype"):
        TokenScores(4, 10, dtype=torch.float16, device="cpu")
    monkeypatch.setattr(b, "_stream", lambda stream: None)
    op._buf["stats"] = op._buf["entropy"] = torch.zeros(4, 2)
    wide = torch.zeros(4, 12, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="another row stride"):
        op.backward(wide.flatten()[:40].view(4, 10), out=wide[:, :10])
    one = TokenScores(4, 10, 1, device="cpu")
    one._buf["ids"] = t.view(4, 1)
    with pytest.raises(ValueError, match="token is a buffer that this call writes"):
        one.forward(z, t)
    op._buf["dlogits"] = z
    with pytest.raises(ValueError, match="logits is a buffer that this call writes"):
        op.backward(z)


def test_oracle_closed_forms():
    # equal logits: log vocab; one entry left: zero; ties to the lower index
    z = np.zeros((2, 8))
    z[1, 1:] = -np.inf
    logp, h, ids, best = od.token_scores_forward(z, np.array([3, 0]), 3)
    np.testing.assert_allclose(logp, [-math.log(8), 0], atol=1e-15)
    np.testing.assert_allclose(h, [math.log(8), 0], atol=1e-15)
    assert ids.tolist() == [[0, 1, 2], [0, -1, -1]] and best[1].tolist() == [0, -np.inf, -np.inf]
    # two entries at temperature T: a logistic function
    z = np.array([[1.5, 0.0]])
    logp, _, _, _ = od.token_scores_forward(z, np.array([0]), temperature=0.5)
    np.testing.assert_allclose(logp, -np.log1p(np.exp(-3.0)), rtol=1e-14)
    # an excluded entry is as if it were not there
    rng = np.random.default_rng(0)
    z = rng.normal(size=(3, 9))
    a = od.token_scores_forward(z, np.array([0, 1, 2]), 4, excluded=8)
    c = od.token_scores_forward(z[:, :8], np.array([0, 1, 2]), 4)
    for p, q in zip(a, c):
        np.testing.assert_allclose(p, q, rtol=1e-14)


def test_oracle_against_differences():
    rng = np.random.default_rng(1)
    z, token = rng.normal(size=(3, 7)), np.array([2, 6, -1])
    dl, dh = rng.normal(size=3), rng.normal(size=3)
    grad = od.token_scores_backward(z, token, dl, dh, 5, 0.6)

    def value(y):
        logp, h, _, _ = od.token_scores_forward(y, token, 0, 5, 0.6)
        return (logp * dl).sum() + (h * dh).sum()

    for at in np.ndindex(z.shape):
        lo, hi = z.copy(), z.copy()
        lo[at] -= 1e-6
        hi[at] += 1e-6
        assert abs((value(hi) - value(lo)) / 2e-6 - grad[at]) < 1e-8
