"""The dense operators on the GPU against the fp64 oracle: sizes from one row
to tiles of pairs of CTAs, odd widths, every activation and type, strides,
rows that do not count, vocabularies in several pieces.

Tolerances (per tensor, tests/parity.py: max |err| - u |oracle| over max
|oracle|), fixed beforehand:
  * bf16 outputs: u = 2^-8, forward 2e-3, gradients 5e-3 (the products read dz
    rounded to bf16, half an ulp 2^-9 per term, adding up like a random walk).
  * fp32 outputs: sums over k terms. The tensor cores add 16 products at a time
    and cut each addition off below 2^-23 of the running sum (fp32 inputs: 24
    additions per 64 terms, then fp32 additions); with the oracle's largest
    value about four standard deviations of a sum, i.e. sqrt(k) / 4 of the
    sum of magnitudes, that is at most 2^-23 (k / 16 + 24) max(1, sqrt(k) / 4),
    plus 2e-6 for the MUFU exponentials and reciprocals of the epilogues.
"""

import math

import numpy as np
import pytest

import parity
from oracle import dense as od

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import Linear, LmLoss  # noqa: E402

B, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    assert binding.bdscan_ssd_wait_flag(1) == 0
    yield
    torch.cuda.synchronize()
    assert binding.bdscan_ssd_wait_flag(1) == 0


def tol32(k):
    return 2.0 ** -23 * (k / 16 + 24) * max(1.0, math.sqrt(k) / 4) + 2e-6


def close(name, t, ora, k, grad=False):
    a = t.detach().double().cpu().numpy()
    if t.dtype == B:
        parity.assert_close(name, a, ora, parity.GRAD_TOL if grad else parity.FWD_TOL, parity.BF16_U)
    else:
        parity.assert_close(name, a, ora, tol32(k))


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def draw(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def linear_case(t, k, n, act, dtype, out=None, bias=True, residual=False, seed=0, ld=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = out or dtype
    x = draw(g, (t, k + ld), 1.0, dtype)[:, :k]
    w = draw(g, (n, k), 1 / math.sqrt(k), dtype)
    b = draw(g, (n,), 0.3, dtype) if bias else None
    r = draw(g, (t, n + ld), 1.0, out)[:, :n] if residual else None
    dy = draw(g, (t, n + ld), 1.0, out)[:, :n]
    return x, w, b, r, dy


def check_linear(t, k, n, act, dtype, out=None, bias=True, residual=False, seed=0, ld=0):
    x, w, b, r, dy = linear_case(t, k, n, act, dtype, out, bias, residual, seed, ld)
    op = Linear(t, k, n, act, dtype, out)
    y = op.forward(x, w, b, r, save_pre=True)
    oy, pre = od.linear_forward(f64(x), f64(w), f64(b), f64(r), act)
    close("y", y, oy, k)
    if act != "none":
        close("pre", op.pre, pre, k)
    dx, dw, db = op.backward(x, w, dy, bias=bias)
    gx, gw, gb = od.linear_backward(f64(x), f64(w), pre, f64(dy), act)
    close("dx", dx, gx, n, True)
    close("dw", dw, gw, t, True)
    if bias:
        close("dbias", db, gb, t, True)


ROWS = [1, 2, 5, 8, 9, 31, 128, 129, 257]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("dtype", [B, F])
def test_linear_rows(rows, dtype):
    check_linear(rows, 72, 136, "gelu", dtype, residual=True, seed=rows)


@pytest.mark.parametrize("k,n", [(1, 1), (1, 40), (7, 3), (8, 8), (15, 33), (64, 32), (65, 200), (451, 95), (200, 449)])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows", [3, 150])
def test_linear_widths(rows, k, n, dtype):
    check_linear(rows, k, n, "silu", dtype, residual=True, seed=k + n)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dtype,out", [(B, B), (B, F), (F, F)])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_linear_options(act, dtype, out, bias, residual):
    check_linear(140, 96, 80, act, dtype, out, bias, residual)
    check_linear(4, 96, 80, act, dtype, out, bias, residual)


@pytest.mark.parametrize("ld", [8, 5])
@pytest.mark.parametrize("dtype,out", [(B, B), (B, F), (F, F)])
def test_linear_strided_rows(ld, dtype, out):
    for t in (6, 140):
        check_linear(t, 64, 72, "gelu", dtype, out, True, True, ld=ld)


@pytest.mark.parametrize("t,k,n", [(2000, 448, 1792), (2000, 1792, 448), (1111, 451, 1789), (33, 3328, 832)])
@pytest.mark.parametrize("dtype", [B, F])
def test_linear_large(t, k, n, dtype):
    check_linear(t, k, n, "gelu", dtype, residual=True)


def test_linear_output_inside_a_wider_buffer():
    """y and the residual are the same columns of a wider buffer; its other columns stay as they are."""
    for n, off in ((72, 8), (73, 8)):
        x, w, b, _, _ = linear_case(140, 64, n, "silu", B)
        wide = torch.randn(140, 160, device="cuda").to(B)
        before = wide.clone()
        y = wide[:, off:off + n]
        Linear(140, 64, n, "silu", B).forward(x, w, b, y, out=y)
        oy, _ = od.linear_forward(f64(x), f64(w), f64(b), f64(before[:, off:off + n]), "silu")
        close("y", y, oy, 64)
        assert torch.equal(wide[:, :off], before[:, :off]) and torch.equal(wide[:, off + n:], before[:, off + n:])


@pytest.mark.parametrize("k,n", [(65, 40), (67, 41), (451, 33)])
@pytest.mark.parametrize("dtype", [B, F])
def test_linear_neighbours_of_strided_operands_are_not_read(k, n, dtype):
    """x, the residual and dy lie in wider buffers with aligned rows whose other columns are NaN."""
    t = 150
    x, w, b, r, dy = linear_case(t, k, n, "silu", dtype, residual=True)

    def inside(a):
        wide = torch.full((t, (a.shape[1] + 23) // 16 * 16), float("nan"), dtype=a.dtype, device="cuda")
        wide[:, :a.shape[1]] = a
        return wide[:, :a.shape[1]]

    op, ref = Linear(t, k, n, "silu", dtype), Linear(t, k, n, "silu", dtype)
    y = op.forward(inside(x), w, b, inside(r), save_pre=True)
    assert torch.isfinite(y).all()
    close("y", y, od.linear_forward(f64(x), f64(w), f64(b), f64(r), "silu")[0], k)
    ref.forward(x, w, b, r, save_pre=True)
    for a, c in zip(op.backward(inside(x), w, inside(dy)), ref.backward(x, w, dy)):
        assert torch.isfinite(a).all()
        close("gradient", a, f64(c), max(t, n), True)


def test_linear_gradients_one_at_a_time():
    x, w, b, _, dy = linear_case(150, 65, 40, "gelu", B)
    op = Linear(150, 65, 40, "gelu", B)
    op.forward(x, w, b, save_pre=True)
    whole = [t.clone() for t in op.backward(x, w, dy)]
    for i, kw in enumerate((dict(need_dw=False, bias=False), dict(need_dx=False, bias=False),
                            dict(need_dx=False, need_dw=False))):
        got = op.backward(x, w, dy, **kw)
        assert torch.equal(got[i], whole[i])
        assert all(t is None for j, t in enumerate(got) if j != i)


def test_linear_gradients_of_a_gradient_without_rows():
    x, w, _, _, _ = linear_case(4, 16, 24, "none", B)
    dw = torch.ones_like(w)
    db = torch.ones(24, dtype=B, device="cuda")
    d = binding.make_linear_dims(0, 16, 24)
    binding.linear_backward(d, None, w, None, None, None, dw, db, None)
    assert not dw.any() and not db.any()


def test_linear_offsets_past_32_bits():
    """x and y are columns of a buffer of 70,000 rows of 40,000 elements: row offsets pass 2^31 elements."""
    t, ld = 70000, 40000
    wide = torch.zeros((t, ld), dtype=B, device="cuda")
    x, y = wide[:, 64:128], wide[:, 1024:1024 + 48]
    x.copy_(torch.randn(t, 64, device="cuda").to(B))
    w = (torch.randn(48, 64, device="cuda") / 8).to(B)
    Linear(t, 64, 48, "none", B).forward(x, w, out=y)
    at = torch.tensor([0, 53686, 53688, 69999], device="cuda")  # both sides of 2^31 elements
    close("y", y[at], od.linear_forward(f64(x[at]), f64(w))[0], 64)
    assert not wide[:, 128:1024].any() and not wide[:, 1024 + 48:].any()
    dy = torch.randn(t, 48, device="cuda").to(B)
    dx, dw, _ = Linear(t, 64, 48, "none", B).backward(x, w, dy, bias=False)
    close("dx", dx[at], od.linear_backward(f64(x[at]), f64(w), f64(y[at]), f64(dy[at]))[0], 48, True)
    close("dw", dw, (dy.double().t() @ x.double()).cpu().numpy(), t, True)


def test_linear_extreme_values():
    """Activations far out in both tails, and values near the largest fp32 in the split into pieces."""
    t, k = 200, 8
    x = torch.zeros(t, k, device="cuda")
    x[:, 0] = torch.linspace(-300, 300, t, device="cuda")
    w = torch.zeros(16, k, device="cuda")
    w[:, 0] = 1.0
    for act in ("silu", "gelu"):
        op = Linear(t, k, 16, act, F)
        y = op.forward(x, w, save_pre=True)
        close("y", y, np.repeat(od.act(act, f64(x[:, :1])), 16, 1), k)
        dx, _, _ = op.backward(x, w, torch.ones_like(y), bias=False)
        assert torch.isfinite(dx).all()
        # the derivative: 0 and 1 in the tails
        assert dx[0, 0].abs() < 1e-6 and (dx[-1, 0] - 16).abs() < 1e-4
    big = torch.full((20, k), 3.38e38, device="cuda")
    one = torch.zeros(8, k, device="cuda")
    one[:, 3] = 1.0
    assert torch.equal(Linear(20, k, 8, "none", F).forward(big, one), big[:, :8])


def test_linear_same_bits_again_and_on_another_stream():
    x, w, b, r, dy = linear_case(600, 200, 333, "gelu", B, residual=True)
    op = Linear(600, 200, 333, "gelu", B)
    ref = [op.forward(x, w, b, r, save_pre=True).clone()] + [t.clone() for t in op.backward(x, w, dy)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [op.forward(x, w, b, r, save_pre=True)] + list(op.backward(x, w, dy))
    s.synchronize()
    for a, c in zip(ref, got):
        assert torch.equal(a, c)


def test_linear_and_loss_in_a_cuda_graph():
    x, w, b, _, _ = linear_case(40, 64, 72, "silu", B)
    head = (torch.randn(500, 72, device="cuda") / 8).to(B)
    target = torch.randint(0, 500, (40,), device="cuda")
    op, ls = Linear(40, 64, 72, "silu", B), LmLoss(40, 72, 500, B)

    def step():
        y = op.forward(x, w, b, save_pre=True)
        loss, _ = ls.forward(y, head, target)
        dh, dhead = ls.backward(y, head, target)
        return (loss, dhead) + op.backward(x, w, dh)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ref = [t.clone() for t in step()]
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got = step()
    for t in got:
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    for a, c in zip(ref, got):
        assert torch.equal(a, c)


# ---------------------------------------------------------------------------
# loss
# ---------------------------------------------------------------------------
def loss_case(t, k, v, dtype, counted=0.6, seed=0, ld=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = draw(g, (t, k + ld), 1.0, dtype)[:, :k]
    w = draw(g, (v, k), 2 / math.sqrt(k), dtype)
    target = torch.randint(0, max(1, v - 1), (t,), generator=g, device="cuda")
    weight = torch.rand(t, generator=g, device="cuda") + 0.1
    weight[torch.rand(t, generator=g, device="cuda") > counted] = 0.0
    dloss = torch.rand(t, generator=g, device="cuda") + 0.5
    return h, w, target, weight, dloss


def check_loss(h, w, target, weight, dloss, excluded=-1, name=""):
    t, k = h.shape
    op = LmLoss(t, k, w.shape[0], h.dtype, excluded)
    loss, lse = op.forward(h, w, target, weight)
    ones = np.ones(t)
    wt, dl = ones if weight is None else f64(weight), ones if dloss is None else f64(dloss)
    hh = np.nan_to_num(f64(h), nan=0.0, posinf=0.0, neginf=0.0)
    tg = target.cpu().numpy()
    ol, os_ = od.lm_loss_forward(hh, f64(w), tg, wt, excluded)
    close("loss" + name, loss, ol, k)
    close("lse" + name, lse, os_, k)
    dh, dw = op.backward(h, w, target, weight, dloss)
    gh, gw = od.lm_loss_backward(hh, f64(w), tg, wt, dl, excluded)
    close("dh" + name, dh, gh, w.shape[0], True)
    close("dw" + name, dw, gw, t, True)
    out = (wt == 0) | (tg < 0) | (tg >= w.shape[0])
    assert not loss.cpu().numpy()[out].any() and not lse.cpu().numpy()[out].any()
    assert not dh.float().cpu().numpy()[out | (dl == 0)].any()
    if excluded >= 0:
        assert not dw[excluded].any()


@pytest.mark.parametrize("t", [1, 2, 31, 128, 130, 300])
@pytest.mark.parametrize("dtype", [B, F])
def test_loss_rows(t, dtype):
    check_loss(*loss_case(t, 64, 500, dtype, counted=1.0 if t < 3 else 0.6, seed=t))


@pytest.mark.parametrize("k,v", [(1, 2), (8, 1), (7, 33), (64, 31), (65, 257), (451, 1000), (72, 5001)])
@pytest.mark.parametrize("dtype", [B, F])
def test_loss_widths(k, v, dtype):
    check_loss(*loss_case(70, k, v, dtype, seed=k + v), excluded=v - 1 if v > 2 else -1)


def test_loss_options():
    h, w, target, weight, dloss = loss_case(90, 64, 300, B)
    check_loss(h, w, target, None, dloss)
    check_loss(h, w, target, weight, None)
    check_loss(h, w, target, None, None, excluded=0 if int(target.min()) > 0 else 299)
    check_loss(*loss_case(90, 64, 300, B, ld=8))
    check_loss(*loss_case(90, 64, 300, F, ld=3))
    dloss[::3] = 0.0
    check_loss(h, w, target, weight, dloss)


def test_loss_targets_outside_the_vocabulary_and_hidden_garbage():
    """Rows that do not count may hold anything: infinities, NaN, targets outside."""
    for dtype in (B, F):
        h, w, target, weight, dloss = loss_case(200, 64, 300, dtype, counted=1.0)
        target[3], target[77], target[130] = -1, 300, 2 ** 40
        weight[10:20] = 0.0
        h[3], h[77], h[130] = float("nan"), float("inf"), -float("inf")
        h[10:20] = float("nan")
        check_loss(h, w, target, weight, dloss)


def test_loss_no_row_counts():
    h, w, target, weight, dloss = loss_case(150, 64, 300, B)
    weight.zero_()
    op = LmLoss(150, 64, 300, B)
    loss, lse = op.forward(h, w, target, weight)
    dh, dw = op.backward(h, w, target, weight, dloss)
    assert not loss.any() and not lse.any() and not dh.any() and not dw.any()
    d = binding.make_lm_loss_dims(0, 64, 300)
    dw.fill_(1.0)
    binding.lm_loss_backward(d, None, w, None, None, None, None, None, dw, None)
    assert not dw.any()


def test_loss_target_is_the_excluded_entry_and_nothing_left():
    h, w, target, weight, _ = loss_case(40, 64, 300, B, counted=1.0)
    target[5] = 299
    op = LmLoss(40, 64, 300, B, excluded=299)
    loss, _ = op.forward(h, w, target, weight)
    dh, dw = op.backward(h, w, target, weight)
    rest = torch.arange(40, device="cuda") != 5
    assert loss[5] == float("inf") and torch.isfinite(loss[rest]).all()
    assert torch.isfinite(dh.float()).all() and torch.isfinite(dw.float()).all() and not dw[299].any()
    one = LmLoss(40, 64, 1, B, excluded=0)
    loss, lse = one.forward(h, w[:1].contiguous(), torch.zeros_like(target), weight)
    assert (loss == float("inf")).all() and (lse == -float("inf")).all()
    dh, dw = one.backward(h, w[:1].contiguous(), torch.zeros_like(target), weight)
    assert not dh.any() and not dw.any()


def test_loss_peaked_logits():
    """Log sums far from zero and probabilities next to one."""
    h, w, target, weight, dloss = loss_case(100, 64, 400, F, counted=1.0)
    h *= 20.0
    z = h.double() @ w.double().t()
    target[:50] = z.argmax(1)[:50]
    check_loss(h, w, target, weight, dloss)


@pytest.mark.parametrize("dtype,t,v", [(B, 16384, 20001), (F, 9000, 9001)])
def test_loss_vocabulary_in_pieces(dtype, t, v):
    """More logits than one piece of the backward holds; fp64 torch on the GPU as the oracle."""
    k = 40
    h, w, target, weight, dloss = loss_case(t, k, v, dtype, counted=0.3)
    op = LmLoss(t, k, v, dtype, v - 1)
    loss, lse = op.forward(h, w, target, weight)
    dh, dw = op.backward(h, w, target, weight, dloss)
    rows = torch.nonzero(weight).squeeze(1)
    ol, gh, gw = torch.zeros(t, dtype=torch.float64, device="cuda"), torch.zeros(t, k, dtype=torch.float64, device="cuda"), 0
    for part in rows.split(2000):
        z = h[part].double() @ w.double().t()
        z[:, v - 1] = -math.inf
        s = torch.logsumexp(z, 1)
        i = torch.arange(len(part), device="cuda")
        ol[part] = weight[part].double() * (s - z[i, target[part]])
        dz = torch.exp(z - s[:, None])
        dz[i, target[part]] -= 1
        dz *= (weight[part].double() * dloss[part].double())[:, None]
        gh[part] = dz @ w.double()
        gw = gw + dz.t() @ h[part].double()
    close("loss", loss, ol.cpu().numpy(), k)
    close("dh", dh, gh.cpu().numpy(), v, True)
    close("dw", dw, gw.cpu().numpy(), t, True)


def test_loss_many_rows():
    """More rows than one CTA numbers at a time, most of them not counting."""
    t = 70001
    h, w, target, weight, dloss = loss_case(t, 8, 5, F, counted=0.02)
    op = LmLoss(t, 8, 5, F)
    loss, lse = op.forward(h, w, target, weight)
    z = h.double() @ w.double().t()
    s = torch.logsumexp(z, 1)
    want = torch.where(weight != 0, weight.double() * (s - z.gather(1, target[:, None])[:, 0]), torch.zeros_like(s))
    close("loss", loss, want.cpu().numpy(), 8)
    dh, dw = op.backward(h, w, target, weight, dloss)
    g = torch.exp(z - s[:, None])
    g[torch.arange(t, device="cuda"), target] -= 1
    g *= (weight.double() * dloss.double())[:, None]
    close("dh", dh, (g @ w.double()).cpu().numpy(), 8, True)
    close("dw", dw, (g.t() @ h.double()).cpu().numpy(), t, True)


def test_loss_same_bits_again():
    h, w, target, weight, dloss = loss_case(300, 200, 3001, B)
    op = LmLoss(300, 200, 3001, B)
    ref = [t.clone() for t in op.forward(h, w, target, weight) + op.backward(h, w, target, weight, dloss)]
    got = op.forward(h, w, target, weight) + op.backward(h, w, target, weight, dloss)
    for a, c in zip(ref, got):
        assert torch.equal(a, c)


def test_gradients_against_differences():
    """Directional derivatives of the library's own fp32 outputs. A central difference of step e of a sum whose
    rounding noise is n (2^-22 of its magnitude) is good to n / e plus third derivatives times e^2."""
    t, k, n, v = 40, 24, 32, 50
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w, b, _, _ = linear_case(t, k, n, "gelu", F)
    head = draw(g, (v, n), 1.0, F)
    target = torch.randint(0, v, (t,), generator=g, device="cuda")
    op, ls = Linear(t, k, n, "gelu", F), LmLoss(t, n, v, F)

    def total(xx, ww, hh):
        return ls.forward(op.forward(xx, ww, b, save_pre=True), hh, target)[0].double().sum().item()

    total(x, w, head)
    y = op.forward(x, w, b, save_pre=True)
    dh, dhead = ls.backward(y, head, target)
    dhead = dhead.clone()
    dx, dw, _ = op.backward(x, w, dh)
    dx, dw = dx.clone(), dw.clone()
    size, e = abs(total(x, w, head)), 1e-2
    for i, (a, ga) in enumerate(((x, dx), (w, dw), (head, dhead))):
        d = draw(g, a.shape, 1.0, F)
        d /= d.norm()
        args = [x, w, head]
        args[i] = a + e * d
        hi = total(*args)
        args[i] = a - e * d
        lo = total(*args)
        want = (ga.double() * d.double()).sum().item()
        assert abs((hi - lo) / (2 * e) - want) <= 2.0 ** -22 * size / e + 10 * e * e * max(1.0, ga.norm().item())


# ---------------------------------------------------------------------------
# debug build
# ---------------------------------------------------------------------------
def test_debug_build_of_the_dense_operators():
    x, w, b, r, dy = linear_case(300, 65, 72, "gelu", B, residual=True)
    h, head, target, weight, dloss = loss_case(150, 72, 400, B)

    def run():
        op, ls = Linear(300, 65, 72, "gelu", B), LmLoss(150, 72, 400, B)
        return (op.forward(x, w, b, r, save_pre=True),) + op.backward(x, w, dy) + ls.forward(
            h, head, target, weight) + ls.backward(h, head, target, weight, dloss)

    ref = [t.clone() for t in run()]
    binding.use_debug_build(True)
    try:
        for a, c in zip(ref, run()):
            assert torch.equal(a, c)
        assert binding.bdscan_debug_set_slack(1) == 0
        for rows in (300, 4):  # the product's and the row kernel's extent
            with pytest.raises(binding.BdscanError) as e:
                Linear(rows, 64, 72, "none", B).forward(x[:rows, :64].contiguous(), w[:, :64].contiguous())
            assert e.value.code == binding.BDSCAN_ERR_DEVICE and "outside the extent" in str(e.value)
    finally:
        binding.bdscan_debug_set_slack(0)
        binding.use_debug_build(False)
