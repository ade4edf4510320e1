"""Token scores on the GPU against the fp64 oracle: vocabularies from one entry
to rows shared by a cluster, ties, masks down to empty rows, values that are not
finite, strides, gradients.

Tolerances, fixed beforehand. With n = vocab / 128 + 64 the additions that a
sum of exponentials goes through at most, each off by 2^-24 of the (positive)
sum, and 2^-21 for the MUFU exponentials, differences and products that make up
an exponent:
  * logp: n 2^-24 + 2^-21 (1 + |logp|)
  * entropy: its two terms, log s and t / s, are at most log vocab each, off by
    that share and by the share of s: 2 (n 2^-24 + 2^-21) (1 + log vocab)
  * a gradient: p (dlogp + dentropy (entropy + log p)) with log p off by the
    same amount again: (n 2^-24 + 2^-21 (2 + log vocab)) (|dlogp| + |dentropy| (2
    + 2 log vocab)) / T at most, since p |log p| < 1 (bf16: and 2^-8 of itself).
Indices are equal.
"""

import math

import numpy as np
import pytest

from oracle import dense as od

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300.dense import Linear, TokenScores  # noqa: E402

B, F = torch.bfloat16, torch.float32


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def within(name, got, want, tol):
    got = got.double().cpu().numpy()
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)  # its range ends there
    assert np.array_equal(np.isnan(got), np.isnan(want)), name
    assert np.array_equal(got == -np.inf, want == -np.inf) and not (got == np.inf).any(), name
    ok = np.isfinite(want)
    bad = np.abs(got[ok] - want[ok]) - (tol[ok] if isinstance(tol, np.ndarray) else tol)
    assert not bad.size or bad.max() <= 0, (name, bad.max())


def check(z, token=None, top=0, excluded=-1, temperature=1.0, dlogp=None, dentropy=None, op=None):
    rows, vocab = z.shape
    op = op or TokenScores(rows, vocab, top, z.dtype, excluded, temperature)
    logp, entropy, ids, best = op.forward(z, token)
    tk = None if token is None else token.cpu().numpy()
    wl, we, wi, wb = od.token_scores_forward(f64(z), tk, top, excluded, temperature)
    e = (vocab / 128 + 64) * 2.0 ** -24 + 2.0 ** -21
    mag = lambda w: e + 2.0 ** -21 * np.abs(np.where(np.isfinite(w), w, 0))  # noqa: E731
    if token is None:
        assert logp is None
    else:
        within("logp", logp, wl, mag(wl))
    within("entropy", entropy, we, 2 * e * (1 + math.log(vocab)))
    if top:
        assert np.array_equal(ids.cpu().numpy(), wi)
        within("top", best, wb, mag(wb))
    else:
        assert ids is None and best is None
    if dlogp is not None or dentropy is not None:
        got = op.backward(z, token, dlogp, dentropy)
        want = od.token_scores_backward(f64(z), tk, f64(dlogp), f64(dentropy), excluded, temperature)
        size = (np.zeros(rows) if dlogp is None else np.abs(f64(dlogp))) + \
            (np.zeros(rows) if dentropy is None else np.abs(f64(dentropy)) * (2 + 2 * math.log(vocab)))
        tol = ((e + 2.0 ** -21 * (1 + math.log(vocab))) * size / temperature)[:, None] + np.zeros(z.shape)
        if z.dtype == B:
            tol = tol + 2.0 ** -8 * np.abs(want)
        within("dlogits", got, want, tol)
    return op


def draw(rows, vocab, dtype, seed=0, ld=0, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(rows, vocab + ld, generator=g, device="cuda") * std).to(dtype)[:, :vocab]
    token = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    dl, dh = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda") * 0.1
    return z, token, dl, dh


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 31, 64, 65, 127, 500, 1023, 2048, 4096, 4097, 8191, 20000, 50021])
@pytest.mark.parametrize("dtype", [B, F])
def test_vocabularies(vocab, dtype):
    z, token, dl, dh = draw(5, vocab, dtype, seed=vocab)
    check(z, token, 8, -1, 1.0, dl, dh)
    check(z, token, 3, vocab - 1, 0.7, dl, dh)


@pytest.mark.parametrize("rows", [1, 2, 17, 40, 80, 151, 153, 400])
@pytest.mark.parametrize("dtype", [B, F])
def test_rows(rows, dtype):
    z, token, dl, dh = draw(rows, 9001, dtype, seed=rows)
    check(z, token, 5, 17, 1.3, dl, dh)


@pytest.mark.parametrize("top", [0, 1, 2, 16, 33, 63, 64])
@pytest.mark.parametrize("vocab", [40, 700, 5000, 40000])
@pytest.mark.parametrize("rows", [2, 200])
def test_tops(top, vocab, rows):
    check(draw(rows, vocab, B, seed=top)[0], None, top)


@pytest.mark.parametrize("ld", [1, 3, 4, 8, 13])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("vocab", [50, 5003])
def test_strided_rows(ld, dtype, vocab):
    z, token, dl, dh = draw(9, vocab, dtype, ld=ld)
    check(z, token, 6, 2, 0.5, dl, dh)
    # the gradient into rows of a third stride, whose other columns stay as they are
    wide = torch.full((9, vocab + 5), 7.0, device="cuda", dtype=dtype)
    op = TokenScores(9, vocab, 0, dtype)
    op.forward(z, token)
    got = op.backward(z, token, dl, dh).clone()
    out = op.backward(z, token, dl, dh, out=wide[:, :vocab])
    assert torch.equal(out, got) and (wide[:, vocab:] == 7).all()


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("vocab", [600, 9000, 50000])
def test_equal_logits_go_to_the_lower_index(dtype, vocab):
    for rows in (3, 160):
        z = torch.zeros(rows, vocab, device="cuda", dtype=dtype)
        check(z, None, 64)
        check(z, None, 7, excluded=0)
        z[:, ::3] = 1.0
        check(z, None, 64)
        z = (torch.arange(vocab, device="cuda") // 40).to(dtype).repeat(rows, 1)  # rising, with runs
        check(z, None, 33)
        check(z.flip(1), None, 33)
        z[:, :100] = -0.0
        z[:, 100:] = 0.0
        check(z, None, 10)


@pytest.mark.parametrize("vocab", [9, 300, 7000])
@pytest.mark.parametrize("dtype", [B, F])
def test_masked_logits(vocab, dtype):
    """Minus infinity and the type's lowest value: few entries left, one, none."""
    z, token, dl, dh = draw(8, vocab, dtype)
    z = z.clone()
    for low in (-math.inf, torch.finfo(dtype).min):
        y = z.clone()
        y[0] = low
        y[1, 1:] = low
        y[2, :-1] = low
        y[3, 2:] = low
        y[4, ::2] = low
        token[:5] = torch.tensor([0, 0, vocab - 1, 1, 1], device="cuda")
        check(y, token, 5, -1, 1.0, dl, dh)
        check(y, token, 5, vocab - 1, 2.0, None, dh)
        check(y, token, 5, 0, 0.3, None, dh)
    token[0] = 2  # a token that the mask has taken
    check(y, token, 5)


def test_excluded_entry_is_never_read_as_a_value():
    z, token, dl, dh = draw(4, 1000, F)
    for bad in (math.nan, math.inf, 1e30):
        z[:, 77] = bad
        token[:] = 5
        check(z, token, 4, 77, 1.0, dl, dh)
    token[:] = 77
    logp = TokenScores(4, 1000, 0, F, 77).forward(z, token)[0]
    assert (logp == -math.inf).all()


@pytest.mark.parametrize("vocab", [100, 9000])
def test_values_that_are_not_finite_stay_visible(vocab):
    for rows in (4, 200):
        for bad in (math.nan, math.inf):
            for dtype in (B, F):
                z, token, dl, dh = draw(rows, vocab, dtype)
                z[1, vocab // 2] = bad
                op = TokenScores(rows, vocab, 4, dtype)
                logp, entropy, ids, best = op.forward(z, token)
                rest = torch.arange(rows, device="cuda") != 1
                for v in (logp, entropy, best):
                    assert torch.isnan(v[1]).all() and torch.isfinite(v[rest]).all()
                assert (ids[1] == -1).all() and (ids[rest] >= 0).all()
                dz = op.backward(z, token, dl, dh)
                assert torch.isnan(dz[1]).all() and torch.isfinite(dz[rest]).all()


@pytest.mark.parametrize("vocab", [100, 9000])
@pytest.mark.parametrize("rows", [6, 200])
def test_rows_that_do_not_count(vocab, rows):
    z, token, dl, dh = draw(rows, vocab, F)
    token[1], token[3], token[4] = -1, vocab, -5
    z[1], z[3] = math.nan, math.inf
    dl[1] = math.nan
    op = TokenScores(rows, vocab, 3, F)
    logp, entropy, ids, best = op.forward(z, token)
    dz = op.backward(z, token, dl, dh)
    for r in (1, 3, 4):
        assert logp[r] == 0 and entropy[r] == 0 and (ids[r] == -1).all() and (best[r] == -math.inf).all()
        assert not dz[r].any()
    # nor have they one where the gradient is of the entropy alone and the tokens are not given again
    alone = op.backward(z, None, None, dh)
    assert not alone[[1, 3, 4]].any() and torch.isfinite(alone).all()
    dz = op.backward(z, token, dl, dh)
    keep = torch.tensor([i for i in range(rows) if i not in (1, 3, 4)], device="cuda")
    part = TokenScores(len(keep), vocab, 3, F)
    want = [t.clone() for t in part.forward(z[keep], token[keep])]
    want.append(part.backward(z[keep], token[keep], dl[keep], dh[keep]))
    for a, b in zip((logp, entropy, ids, best, dz), want):
        torch.testing.assert_close(a[keep], b, rtol=1e-5, atol=1e-6)


def test_no_rows():
    op = TokenScores(0, 50, 3)
    z, token = torch.zeros(0, 50, device="cuda", dtype=B), torch.zeros(0, device="cuda", dtype=torch.int64)
    logp, entropy, ids, best = op.forward(z, token)
    assert logp.shape == entropy.shape == (0,) and ids.shape == best.shape == (0, 3)
    assert op.backward(z, token, logp, entropy).shape == (0, 50)


def test_gradient_in_place_and_alone():
    z, token, dl, dh = draw(20, 3001, B)
    op = TokenScores(20, 3001, 0, B)
    op.forward(z, token)
    both = op.backward(z, token, dl, dh).clone()
    zero = torch.zeros(20, device="cuda")
    assert torch.equal(op.backward(z, token, dl), op.backward(z, token, dl, zero).clone())
    assert torch.equal(op.backward(z, None, None, dh).clone(), op.backward(z, token, zero, dh))
    assert not op.backward(z, token).any()
    out = op.backward(z, token, dl, dh, out=z)
    assert out.data_ptr() == z.data_ptr() and torch.equal(z, both)


def test_offsets_past_32_bits():
    """Logits are columns of a buffer of 60,000 rows of 40,000 elements, the gradient of another."""
    t, v, ld = 60000, 300, 40000
    wide = torch.zeros((t, ld), dtype=B, device="cuda")
    z = wide[:, 64:64 + v]
    z.copy_((torch.randn(t, v, device="cuda") * 3).to(B))
    token = torch.randint(0, v, (t,), device="cuda")
    op = TokenScores(t, v, 3, B)
    got = [x.clone() for x in op.forward(z, token)]
    dl = torch.randn(t, device="cuda")
    dz = op.backward(z, token, dl, out=wide[:, 1024:1024 + v])
    # the copy's rows lie on other boundaries, and sums add up in another order: each side is off by the bounds above
    same = TokenScores(t, v, 3, B)
    close = z.contiguous()
    want = same.forward(close, token)
    e = (v / 128 + 64) * 2.0 ** -24 + 2.0 ** -21
    assert torch.equal(got[2], want[2])
    for i in (0, 3):
        assert ((got[i] - want[i]).abs() <= 2 * (e + 2.0 ** -21 * want[i].abs())).all()
    assert ((got[1] - want[1]).abs() <= 4 * e * (1 + math.log(v))).all()
    grad = same.backward(close, token, dl).float()
    size = (e + 2.0 ** -21 * (2 + math.log(v))) * dl.abs()[:, None]
    assert ((dz.float() - grad).abs() <= 2 * (size + 2.0 ** -8 * grad.abs())).all()
    assert not wide[:, :64].any() and not wide[:, 64 + v:1024].any() and not wide[:, 1024 + v:].any()


def test_two_streams_with_a_holder_each():
    args = [draw(70, 9001, B, seed=i) for i in (1, 2)]
    ops = [TokenScores(70, 9001, 5, B) for _ in args]

    def step(o, a, s=None):
        return (*o.forward(a[0], a[1], stream=s), o.backward(*a, stream=s))

    want = [[t.clone() for t in step(o, a)] for o, a in zip(ops, args)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(8):
        got = [step(o, a, s) for o, a, s in zip(ops, args, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, v in zip(got, want) for p, q in zip(g, v))


@pytest.mark.parametrize("vocab", [100, 5000, 90000])
@pytest.mark.parametrize("rows", [2, 300])
@pytest.mark.parametrize("dtype", [B, F])
def test_same_scores_however_a_row_lies(vocab, rows, dtype):
    """Rows on other boundaries, with neighbours that must not be read: the same entries, and scores to rounding."""
    z, token, dl, dh = draw(rows, vocab, dtype)
    op = TokenScores(rows, vocab, 8, dtype)
    want = [t.clone() for t in op.forward(z, token)]
    grad = op.backward(z, token, dl, dh).clone()
    wide = torch.full((rows, vocab + 11), math.nan, device="cuda", dtype=dtype)
    y = wide[:, :vocab]
    y.copy_(z)
    got = op.forward(y, token)
    assert torch.equal(got[2], want[2])
    for i in (0, 1, 3):
        torch.testing.assert_close(got[i], want[i], rtol=2e-6, atol=2e-6 * math.log(vocab + 1))
    torch.testing.assert_close(op.backward(y, token, dl, dh), grad, rtol=2.0 ** -7 if dtype == B else 1e-5, atol=1e-6)


def test_gradients_against_differences():
    z, token, dl, dh = draw(3, 12, F, std=1.0)
    op = TokenScores(3, 12, 0, F, 4, 0.8)
    op.forward(z, token.fill_(2))
    grad = op.backward(z, token, dl, dh).clone()

    def value(y):
        logp, entropy, _, _ = op.forward(y, token)
        return float((logp.double() * dl.double()).sum() + (entropy.double() * dh.double()).sum())

    step = 2.0 ** -7
    for r, v in ((0, 0), (1, 2), (2, 11), (1, 4)):
        lo, hi = z.clone(), z.clone()
        lo[r, v] -= step
        hi[r, v] += step
        # forward errors of 1e-6 over 2 step, and step^2 times a third derivative below ten
        assert abs((value(hi) - value(lo)) / (2 * step) - float(grad[r, v])) < 1.5e-3


@pytest.mark.parametrize("rows,vocab", [(3, 40000), (200, 3000)])
def test_same_bits_and_captured_replays(rows, vocab):
    z, token, dl, dh = draw(rows, vocab, B)
    op = TokenScores(rows, vocab, 9, B)
    want = [t.clone() for t in (*op.forward(z, token), op.backward(z, token, dl, dh))]
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(want, (*op.forward(z, token), op.backward(z, token, dl, dh))))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = (*op.forward(z, token), op.backward(z, token, dl, dh))
    old = z.clone()
    z.copy_(old.flip(0)), token.copy_(token.flip(0)), dl.copy_(dl.flip(0)), dh.copy_(dh.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q.flip(0)) for p, q in zip(got, want))


def test_scores_of_a_heads_logits():
    """Logits of a block by the linear layer, scored in place; the gradient goes back through the head."""
    rows, k, vocab = 70, 64, 1003
    g = torch.Generator(device="cuda").manual_seed(0)
    h = torch.randn(rows, k, generator=g, device="cuda")
    w = torch.randn(vocab, k, generator=g, device="cuda") / 8
    token = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    dl, dh = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda") * 0.1
    head, sc = Linear(rows, k, vocab, dtype=F), TokenScores(rows, vocab, 4, F, temperature=1.5)
    z = head.forward(h, w)
    logp, entropy, ids, _ = sc.forward(z, token)
    gh, gw, _ = head.backward(h, w, sc.backward(z, token, dl, dh), bias=False)
    hs, ws = h.double().requires_grad_(True), w.double().requires_grad_(True)
    lp = torch.log_softmax(hs @ ws.t() / 1.5, 1)
    wl, we = lp[torch.arange(rows), token], -(lp.exp() * lp).sum(1)
    wh, ww = torch.autograd.grad((wl * dl).sum() + (we * dh).sum(), (hs, ws))
    for a, b in ((logp, wl), (entropy, we), (gh, wh), (gw, ww)):
        torch.testing.assert_close(a.double(), b.detach(), rtol=1e-5, atol=1e-5)
    assert torch.equal(ids[:, 0], lp.argmax(1))
