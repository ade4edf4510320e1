"""fp32 accuracy of the dense operators, tight enough to tell three bf16
pieces per value from two.

Tolerances, fixed beforehand. A value is p0 + p1 + p2 with |p1| <= 2^-9 |v| and
|p2| <= 2^-18 |v| (bf16 rounds to 8 bits), exact to 2^-27. Of the nine products
six are taken; the three that are not are below 2^-26 |u v| together. An output
that is one product of two values is the sum of those six, whose five additions
are cut off below 2^-23 of the sum each: 2^-26 + 5 2^-23 < 2^-20 of the exact
value (SINGLE). Two pieces leave out u0 v2 + u2 v0, up to 2^-17, and three
pieces without u1 v1 up to 2^-18.

Long sums of positive terms: within 64 of k, 24 additions cut off below 2^-23
of a partial sum that ends as the step's share of the result, then one rounding
(2^-24 of the running sum) per step: 2^-23 (24 + k / 128) of the result. Without
the sums leaving the tensor core every 64 of k it cuts off 6 k / 16 additions of
a sum that is half the result on average, 2^-24 on average each: at k = 16384
1.8e-4 against 1.8e-5.
"""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import Linear, LmLoss  # noqa: E402

F = torch.float32
SINGLE = 2.0 ** -20


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    assert binding.bdscan_ssd_wait_flag(1) == 0
    yield
    torch.cuda.synchronize()
    assert binding.bdscan_ssd_wait_flag(1) == 0


def full(g, *shape):
    """Values of all 24 bits, between 1 and 2 in magnitude."""
    v = 1 + torch.rand(shape, generator=g, device="cuda")
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.5, -v, v)


def one_per_row(g, rows, cols):
    """One value in each row, in turn over the columns, and its column."""
    at = torch.arange(rows, device="cuda") % cols
    a = torch.zeros(rows, cols, device="cuda")
    a[torch.arange(rows, device="cuda"), at] = full(g, rows)
    return a, at


def assert_single(got, want):
    assert got.dtype == F and want.dtype == torch.float64
    assert ((got.double() - want).abs() <= SINGLE * want.abs()).all()


SIZES = [(4, 72, 40), (150, 65, 40), (300, 451, 333), (33, 3328, 832), (2000, 448, 1792), (1111, 451, 1789)]


@pytest.mark.parametrize("t,k,n", SIZES)
def test_linear_outputs_of_one_product(t, k, n):
    g = torch.Generator(device="cuda").manual_seed(t)
    x, at = one_per_row(g, t, k)
    w = full(g, n, k)
    v = x.double().sum(1, keepdim=True)
    assert_single(Linear(t, k, n, "none", F).forward(x, w), v * w.double().t()[at])


@pytest.mark.parametrize("t,k,n", SIZES)
def test_linear_input_gradients_of_one_product(t, k, n):
    g = torch.Generator(device="cuda").manual_seed(t)
    dy, at = one_per_row(g, t, n)
    x, w = full(g, t, k), full(g, n, k)
    dx, _, db = Linear(t, k, n, "none", F).backward(x, w, dy)
    assert_single(dx, dy.double().sum(1, keepdim=True) * w.double()[at])


@pytest.mark.parametrize("t,k,n", SIZES)
def test_linear_weight_gradients_of_one_product(t, k, n):
    g = torch.Generator(device="cuda").manual_seed(t)
    dyt, at = one_per_row(g, n, t)  # one row for each output
    x, w = full(g, t, k), full(g, n, k)
    _, dw, db = Linear(t, k, n, "none", F).backward(x, w, dyt.t().contiguous())
    v = dyt.double().sum(1, keepdim=True)
    assert_single(dw, v * x.double()[at])
    assert_single(db, v[:, 0])


@pytest.mark.parametrize("t,k,v", [(3, 64, 40), (150, 65, 40), (300, 451, 333), (1000, 448, 8191)])
def test_loss_logits_of_one_product(t, k, v):
    """Logits of magnitude 4000 to 16000, so far apart that the log sum is the largest but for neighbours; its error is
    at most the largest error of a logit, and 1e-6 of it for the log sum's own steps."""
    g = torch.Generator(device="cuda").manual_seed(t)
    h, at = one_per_row(g, t, k)
    w = full(g, v, k)
    h *= 64.0
    w *= 64.0
    target = torch.randint(0, v, (t,), generator=g, device="cuda")
    loss, lse = LmLoss(t, k, v, F).forward(h, w, target)
    z = h.double().sum(1, keepdim=True) * w.double().t()[at]
    want = torch.logsumexp(z, 1)
    bound = (SINGLE + 1e-6) * z.abs().amax(1)
    assert ((lse.double() - want).abs() <= bound).all()
    zt = z.gather(1, target[:, None])[:, 0]
    assert ((loss.double() - (want - zt)).abs() <= 2 * bound).all()


@pytest.mark.parametrize("t,k,n", [(200, 16384, 64), (64, 4096, 333), (300, 8192, 200)])
def test_long_sums(t, k, n):
    g = torch.Generator(device="cuda").manual_seed(k)
    x, w = full(g, t, k).abs(), full(g, n, k).abs()
    tol = 2.0 ** -23 * (24 + k / 128)
    want = x.double() @ w.double().t()
    y = Linear(t, k, n, "none", F).forward(x, w)
    assert ((y.double() - want).abs() <= tol * want).all()
    # the weight gradient's sum runs over rows
    _, dw, _ = Linear(k, n, t, "none", F).backward(w.t().contiguous(), torch.zeros(t, n, device="cuda"),
                                                   x.t().contiguous(), bias=False, need_dx=False)
    assert ((dw.double() - want).abs() <= tol * want).all()
