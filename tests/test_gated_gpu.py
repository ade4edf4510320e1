"""The gated linear layer on the GPU against the fp64 oracle: sizes from one row
to tiles of pairs of CTAs, odd widths, every activation and type, strides,
refused and empty calls, captured calls.

Tolerances (per tensor, tests/parity.py: max |err| - u |oracle| over max
|oracle|), fixed beforehand:
  * bf16: u = 2^-8, forward 2e-3, gradients 5e-3 (the products read dz rounded
    to bf16, half an ulp 2^-9 per term, adding up like a random walk; the
    projections are computed again and enter unrounded).
  * fp32: a sum over k terms is off by at most e(k) = 2^-23 (k / 16 + 24)
    max(1, sqrt(k) / 4) of its largest value (tests/test_dense_gpu.py). y is a
    product of two such values; its largest is at least a quarter of the product
    of the largest factors, so that either factor's error counts at most four
    times: 8 e(k) + 2e-6 (MUFU). A gradient is a sum over m terms that each
    carry a product of dy, one projection and a derivative below 1.2 of the
    other: e(m) + 10 e(k) + 2e-6.
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
from paper_2607_02805_gb300.dense import GatedLinear, Linear  # noqa: E402

B, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    assert binding.bdscan_ssd_wait_flag(1) == 0
    yield
    torch.cuda.synchronize()
    assert binding.bdscan_ssd_wait_flag(1) == 0


def e32(k):
    return 2.0 ** -23 * (k / 16 + 24) * max(1.0, math.sqrt(k) / 4)


def close(name, t, ora, tol32, grad=False):
    a = t.detach().double().cpu().numpy()
    if t.dtype == B:
        parity.assert_close(name, a, ora, parity.GRAD_TOL if grad else parity.FWD_TOL, parity.BF16_U)
    else:
        parity.assert_close(name, a, ora, tol32 + 2e-6)


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def case(t, k, n, dtype, bias=True, seed=0, ld=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(shape, std):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    x = draw((t, k + ld), 1.0)[:, :k]
    w = draw((2 * n, k), 1 / math.sqrt(k))
    b = draw((2 * n,), 0.3) if bias else None
    dy = draw((t, n + ld), 1.0)[:, :n]
    return x, w, b, dy


def check(t, k, n, act, dtype, bias=True, seed=0, ld=0):
    x, w, b, dy = case(t, k, n, dtype, bias, seed, ld)
    op = GatedLinear(t, k, n, act, dtype)
    close("y", op.forward(x, w, b), od.gated_linear_forward(f64(x), f64(w), f64(b), act), 8 * e32(k))
    dx, dw, db = op.backward(x, w, dy, b)
    gx, gw, gb = od.gated_linear_backward(f64(x), f64(w), f64(b), f64(dy), act)
    close("dx", dx, gx, e32(2 * n) + 10 * e32(k), True)
    close("dw", dw, gw, e32(t) + 10 * e32(k), True)
    if bias:
        close("dbias", db, gb, e32(t) + 10 * e32(k), True)
    else:
        assert db is None


@pytest.mark.parametrize("rows", [1, 2, 5, 8, 9, 31, 32, 33, 127, 128, 129, 257])
@pytest.mark.parametrize("dtype", [B, F])
def test_rows(rows, dtype):
    check(rows, 72, 136, "silu", dtype, seed=rows)


@pytest.mark.parametrize("k,n", [(1, 1), (1, 40), (7, 3), (8, 8), (15, 33), (64, 32), (65, 200), (451, 95), (200, 449),
                                 (40, 12), (64, 130)])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows", [3, 150])
def test_widths(rows, k, n, dtype):
    check(rows, k, n, "gelu", dtype, seed=k + n)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("bias", [False, True])
def test_options(act, dtype, bias):
    check(140, 96, 80, act, dtype, bias)
    check(4, 96, 80, act, dtype, bias)


@pytest.mark.parametrize("ld", [8, 5])
@pytest.mark.parametrize("dtype", [B, F])
def test_strided_rows(ld, dtype):
    for t in (6, 140):
        check(t, 64, 72, "silu", dtype, ld=ld)


@pytest.mark.parametrize("t,k,n", [(2000, 448, 1792), (2000, 1792, 448), (1111, 451, 1789), (33, 832, 3328)])
@pytest.mark.parametrize("dtype", [B, F])
def test_large(t, k, n, dtype):
    check(t, k, n, "silu", dtype)


def test_output_inside_a_wider_buffer():
    """Its other columns stay as they are, and so does what lies behind the last row."""
    for n, off in ((72, 8), (73, 8)):
        for t in (5, 140):
            x, w, b, _ = case(t, 64, n, B)
            wide = torch.randn(t + 3, 160, device="cuda").to(B)
            before = wide.clone()
            y = wide[:t, off:off + n]
            GatedLinear(t, 64, n).forward(x, w, b, out=y)
            close("y", y, od.gated_linear_forward(f64(x), f64(w), f64(b)), 0)
            wide[:t, off:off + n] = before[:t, off:off + n]
            assert torch.equal(wide, before)


def test_each_gradient_by_itself():
    x, w, b, dy = case(300, 72, 136, B)
    op = GatedLinear(300, 72, 136)
    dx, dw, db = (t.clone() for t in op.backward(x, w, dy, b))
    assert op.backward(x, w, dy, b, need_dw=False)[1] is None
    assert torch.equal(op.backward(x, w, dy, b, need_dw=False)[0], dx)
    assert torch.equal(op.backward(x, w, dy, b, need_dx=False)[1], dw)
    one = op.backward(x, w, dy, b, need_dx=False, need_dw=False)
    assert one[0] is None and one[1] is None and torch.equal(one[2], db)


def test_same_bits_for_the_same_call():
    x, w, b, dy = case(700, 200, 264, B)
    op = GatedLinear(700, 200, 264)
    first = [t.clone() for t in (op.forward(x, w, b), *op.backward(x, w, dy, b))]
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, (op.forward(x, w, b), *op.backward(x, w, dy, b))))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows", [4, 200])
def test_values_that_are_not_finite_stay_visible(rows, dtype):
    """A NaN or infinity in one row of x shows in that row of y and dx and in dw, and in no other row."""
    x, w, b, dy = case(rows, 64, 72, dtype)
    for bad in (math.nan, math.inf):
        xb = x.clone()
        xb[1, 3] = bad
        op = GatedLinear(rows, 64, 72, "gelu", dtype)
        y = op.forward(xb, w, b)
        dx, dw, db = op.backward(xb, w, dy, b)
        rest = torch.arange(rows, device="cuda") != 1
        assert not torch.isfinite(y[1]).any() or bad == math.inf and not torch.isfinite(y[1]).all()
        assert torch.isfinite(y[rest]).all() and torch.isfinite(dx[rest]).all()
        assert not torch.isfinite(dx[1]).any() and not torch.isfinite(dw[:, 3]).any()
        assert not torch.isfinite(db).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("n", [9728, 9731])
@pytest.mark.parametrize("dtype", [B, F])
def test_bias_gradient_of_a_few_rows_behind_values_that_are_not_finite(bad, n, dtype):
    """A product of fewer than 128 rows reads whole tiles of 128, whose other rows hold what an earlier kernel left in
    shared memory. Here that is a product of 128 rows of NaN or infinity with the same layout, on every SM (9728 columns
    of both projections are a tile each): nothing of it comes into the sums of the rows."""
    k = 136
    x, w, b, dy = case(100, k, n, dtype)
    full, dy128 = torch.full((128, k), bad, device="cuda", dtype=dtype), torch.ones(128, n, device="cuda", dtype=dtype)
    before = GatedLinear(128, k, n, "silu", dtype)
    for rows in (1, 5, 8, 9, 24, 33, 40, 70, 100):
        op = GatedLinear(rows, k, n, "silu", dtype)
        a, e = x[:rows], dy[:rows]
        _, _, db = before.backward(full, w, dy128, b, need_dx=False, need_dw=False)
        assert not torch.isfinite(db).any()
        _, _, db = op.backward(a, w, e, b, need_dx=False, need_dw=False)
        z = f64(a) @ f64(w).T + f64(b)
        g, u, s = z[:, :n], z[:, n:], 1 / (1 + np.exp(-z[:, :n]))
        want = np.concatenate(((f64(e) * u * s * (1 + g * (1 - s))).sum(0), (f64(e) * g * s).sum(0)))
        assert torch.isfinite(db).all(), rows
        close("dbias", db, want, e32(rows) + 10 * e32(k), True)


def test_no_rows():
    op = GatedLinear(0, 64, 72)
    w, b = torch.zeros(144, 64, device="cuda", dtype=B), torch.zeros(144, device="cuda", dtype=B)
    x, dy = torch.zeros(0, 64, device="cuda", dtype=B), torch.zeros(0, 72, device="cuda", dtype=B)
    assert op.forward(x, w, b).shape == (0, 72)
    dx, dw, db = op.backward(x, w, dy, b)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()


def test_gradients_against_differences():
    """fp32, single entries of x, w and bias moved both ways."""
    t, k, n = 12, 24, 40
    x, w, b, dy = case(t, k, n, F)
    op = GatedLinear(t, k, n, "silu", F)
    dx, dw, db = (v.clone() for v in op.backward(x, w, dy, b))

    def value(*inputs):
        return float((op.forward(*inputs).double() * dy.double()).sum())

    step = 2.0 ** -8
    scale = float(dw.abs().max())
    for place, grad, at in ((0, dx, (3, 5)), (1, dw, (7, 2)), (1, dw, (n + 7, 2)), (2, db, (9,)), (2, db, (n + 9,))):
        lo, hi = [v.clone() for v in (x, w, b)], [v.clone() for v in (x, w, b)]
        lo[place][at] -= step
        hi[place][at] += step
        # third-order term of the difference: step^2 times a third derivative of order one over a few terms;
        # 480 outputs of fp32 forward error 1e-6 each, like a random walk, over 2 step: 3e-3
        assert abs((value(*hi) - value(*lo)) / (2 * step) - float(grad[at])) < 1e-2 * max(1.0, scale)


def test_captured_calls_replay():
    x, w, b, dy = case(300, 72, 136, B)
    op = GatedLinear(300, 72, 136)
    want = [t.clone() for t in (op.forward(x, w, b), *op.backward(x, w, dy, b))]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        op.forward(x, w, b)
        op.backward(x, w, dy, b)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = (op.forward(x, w, b), *op.backward(x, w, dy, b))
    torch.cuda.synchronize()
    for t in got:
        t.zero_()
    x2 = x.clone()
    x.copy_(x2.flip(0))  # other inputs in the same place
    dy2 = dy.clone()
    dy.copy_(dy2.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0].flip(0)) and torch.equal(got[1], want[1].flip(0))
    x.copy_(x2), dy.copy_(dy2)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_two_streams_with_a_holder_each():
    args = [case(520, 200, 264, B, seed=i) for i in (1, 2)]
    ops = [GatedLinear(520, 200, 264) for _ in args]
    want = [[t.clone() for t in (o.forward(x, w, b), *o.backward(x, w, dy, b))] for o, (x, w, b, dy) in zip(ops, args)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(8):
        got = []
        for o, s, (x, w, b, dy) in zip(ops, streams, args):
            got.append((o.forward(x, w, b, stream=s), *o.backward(x, w, dy, b, stream=s)))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, v in zip(got, want) for p, q in zip(g, v))


def test_offsets_past_32_bits():
    """x and y are columns of a buffer of 70,000 rows of 40,000 elements: row offsets pass 2^31 elements."""
    t, k, n, ld = 70000, 64, 48, 40000
    wide = torch.zeros((t, ld), dtype=B, device="cuda")
    x, y = wide[:, 64:64 + k], wide[:, 1024:1024 + n]
    x.copy_(torch.randn(t, k, device="cuda").to(B))
    w = (torch.randn(2 * n, k, device="cuda") / 8).to(B)
    op = GatedLinear(t, k, n)
    op.forward(x, w, out=y)
    at = torch.tensor([0, 53686, 53688, 69999], device="cuda")  # both sides of 2^31 elements
    close("y", y[at], od.gated_linear_forward(f64(x[at]), f64(w)), 0)
    assert not wide[:, 128:1024].any() and not wide[:, 1024 + n:].any()
    dx, _, _ = op.backward(x, w, y)
    gx, _, _ = od.gated_linear_backward(f64(x[at]), f64(w), None, f64(y[at]))
    close("dx", dx[at], gx, 0, True)


def test_gated_block_with_its_down_projection():
    """A whole feed-forward block: gated layer, down projection onto the residual stream, and back."""
    t, k, n = 260, 96, 256
    x, w, b, _ = case(t, k, n, F)
    g = torch.Generator(device="cuda").manual_seed(5)
    wd = torch.randn(k, n, generator=g, device="cuda") / 16
    dy = torch.randn(t, k, generator=g, device="cuda")
    up, down = GatedLinear(t, k, n, "silu", F), Linear(t, n, k, dtype=F)
    a = up.forward(x, w, b)
    y = down.forward(a, wd, residual=x)
    da, dwd, _ = down.backward(a, wd, dy, bias=False)
    dx, dw, db = up.backward(x, w, da, b)
    xs, ws, bs, wds = (v.double().requires_grad_(True) for v in (x, w, b, wd))
    z = xs @ ws.t() + bs
    r = (z[:, :n] * torch.sigmoid(z[:, :n]) * z[:, n:]) @ wds.t() + xs
    gx, gw, gb, gwd = torch.autograd.grad(r, (xs, ws, bs, wds), dy.double())
    tol = 20 * e32(n)
    for name, got, want in (("y", y, r), ("dx", dx + dy, gx), ("dw", dw, gw), ("db", db, gb), ("dwd", dwd, gwd)):
        parity.assert_close(name, got.double().cpu().numpy(), want.detach().cpu().numpy(), tol + 2e-6)
