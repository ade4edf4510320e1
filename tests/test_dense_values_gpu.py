"""Values at the ends of the range through the dense operators: what is not
finite stays visible in every output that reads it, and activations far out in
both tails are those of the formula, whatever the number of rows."""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import Linear  # noqa: E402

B, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    assert binding.bdscan_ssd_wait_flag(1) == 0
    yield
    torch.cuda.synchronize()
    assert binding.bdscan_ssd_wait_flag(1) == 0


def draw(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def case(t, k, n, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (draw(g, (t, k), 1.0, dtype), draw(g, (n, k), 1 / math.sqrt(k), dtype), draw(g, (n,), 0.3, dtype),
            draw(g, (t, n), 1.0, dtype))


NOT_FINITE = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("value", NOT_FINITE)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("t,k,n", [(4, 72, 40), (150, 72, 40), (150, 71, 41)])
def test_bias_that_is_not_finite_reaches_the_gradients(t, k, n, dtype, act, value):
    """The pre-activations of column 5 are not finite: neither is what reads them, everything else is."""
    x, w, b, dy = case(t, k, n, dtype)
    b[5] = value
    op = Linear(t, k, n, act, dtype)
    y = op.forward(x, w, b, save_pre=True)
    rest = torch.arange(n, device="cuda") != 5
    assert not torch.isfinite(y[:, 5]).any() and torch.isfinite(y[:, rest]).all()
    dx, dw, db = op.backward(x, w, dy)
    assert not torch.isfinite(db[5]) and torch.isfinite(db[rest]).all()
    assert not torch.isfinite(dw[5]).any() and torch.isfinite(dw[rest]).all()
    assert not torch.isfinite(dx).any()


@pytest.mark.parametrize("value", NOT_FINITE)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("t,k,n", [(4, 72, 40), (150, 72, 40), (150, 71, 41)])
def test_input_that_is_not_finite_reaches_the_gradients(t, k, n, dtype, act, value):
    x, w, b, dy = case(t, k, n, dtype)
    x[3, 7] = value
    op = Linear(t, k, n, act, dtype)
    y = op.forward(x, w, b, save_pre=True)
    rest = torch.arange(t, device="cuda") != 3
    assert not torch.isfinite(y[3]).any() and torch.isfinite(y[rest]).all()
    dx, dw, db = op.backward(x, w, dy)
    assert not torch.isfinite(dx[3]).any() and torch.isfinite(dx[rest]).all()
    assert not torch.isfinite(dw).any() and not torch.isfinite(db).any()


# Sigmoids below 2^-60 may count as zero: |y| is then at most |z| 2^-60 for the z where that begins, -41.6 for SiLU.
TAIL = 42.0 * 2.0 ** -60


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("t,k", [(4, 8), (200, 8), (200, 7), (40, 4096), (300, 4096)])
def test_activations_far_out(t, k, dtype, act):
    """z far out in both tails: zero below and z above, by the product, by few rows and by products that are split.
    The value above is z times a sigmoid of 1 from an approximate reciprocal (2^-22), rounded to the type."""
    z = torch.tensor([42.0, 50.0, 100.0, 1e4, 1e10, 1e19, 1e20, 1e30, 3e38])
    z = torch.cat([z, -z]).to("cuda", dtype)
    n = 18
    x = torch.zeros(t, k, dtype=dtype, device="cuda")
    x[:, k - 1] = 1.0
    w = torch.zeros(n, k, dtype=dtype, device="cuda")
    w[:, k - 1] = z
    y = Linear(t, k, n, act, dtype).forward(x, w).double().cpu().numpy()
    zz = z.double().cpu().numpy()
    u = 2.0 ** -8 if dtype == B else 2.0 ** -22
    assert (np.abs(y[:, :9] - zz[:9]) <= u * zz[:9]).all()
    assert (np.abs(y[:, 9:]) <= TAIL).all()
