"""The distillation loss on the GPU against the fp64 oracle: rows that count and
rows that do not, entries that are missing, excluded, doubled or impossible,
temperatures, vocabularies in several pieces, gradients.

Tolerances, fixed beforehand. A logit is a sum over k terms, off by at most e(k)
= 2^-23 (k / 16 + 24) max(1, sqrt(k) / 4) of the largest one, M
(tests/test_dense_gpu.py); the log sum by as much, and 2e-6 (1 + its size) for
the exponentials and their sum; a log probability by both:
  * lse: e(k) M / T + 2e-6 (1 + |lse|)
  * loss: |weight| (2 e(k) M / T + 4e-6 (1 + M / T))
Gradients per tensor (tests/parity.py): bf16 5e-3 beside u = 2^-8 (p - q is read
rounded to bf16); fp32 e(n) + 2 (e(k) M / T + 2e-6 (1 + M / T)) for sums over n
terms whose probabilities are off by that share. Where p and q agree, what is
left is the difference of two values off by that share s each: the terms' sizes
add up to p + q = 2, so that 2 s |weight dloss| / T times the largest value of the
other operand (for dw summed over the rows) is added to both bounds.
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
from paper_2607_02805_gb300.dense import DistillLoss, GatedLinear, Linear, LmLoss, TokenScores  # noqa: E402

B, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _no_wait_gave_up():
    assert binding.bdscan_ssd_wait_flag(1) == 0
    yield
    torch.cuda.synchronize()
    assert binding.bdscan_ssd_wait_flag(1) == 0


def e32(k):
    return 2.0 ** -23 * (k / 16 + 24) * max(1.0, math.sqrt(k) / 4)


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def within(name, got, want, tol):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), name
    bad = np.abs(got - want) - tol
    assert bad.max() <= 0, (name, bad.max())


def case(t, k, v, n, dtype, counted=0.6, ragged=True, seed=0, ld=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(t, k + ld, generator=g, device="cuda").to(dtype)[:, :k]
    w = (torch.randn(v, k, generator=g, device="cuda") * 2 / math.sqrt(k)).to(dtype)
    ids = torch.rand(t, v, generator=g, device="cuda").argsort(1)[:, :n].contiguous()
    if ids.shape[1] < n:
        ids = torch.cat((ids, torch.full((t, n - ids.shape[1]), -1, device="cuda")), 1)
    if ragged:
        ids = torch.where(torch.rand(t, n, generator=g, device="cuda") < 0.3, torch.full_like(ids, -1), ids)
    teacher = torch.randn(t, n, generator=g, device="cuda") * 2 + 5
    weight = torch.rand(t, generator=g, device="cuda") + 0.1
    weight[torch.rand(t, generator=g, device="cuda") > counted] = 0.0
    dloss = torch.rand(t, generator=g, device="cuda") + 0.5
    return h, w, ids, teacher, weight, dloss


def check(h, w, ids, teacher, weight, dloss, excluded=-1, temperature=1.0, op=None):
    t, k = h.shape
    v = w.shape[0]
    op = op or DistillLoss(t, k, v, ids.shape[1], h.dtype, excluded, temperature)
    loss, lse = op.forward(h, w, ids, teacher, weight)
    ones = np.ones(t)
    wt, dl = ones if weight is None else f64(weight), ones if dloss is None else f64(dloss)
    hh = np.nan_to_num(f64(h), nan=0.0, posinf=0.0, neginf=0.0)
    args = (hh, f64(w), ids.cpu().numpy(), f64(teacher), wt)
    ol, os_, oz = od.distill_loss_forward(*args, excluded, temperature)
    m = np.abs(hh @ f64(w).T).max()
    within("lse", lse, os_, e32(k) * m / temperature + 2e-6 * (1 + np.abs(os_)))
    within("z", op._buf["z"], oz, e32(k) * m)
    within("loss", loss, ol, np.abs(wt) * (2 * e32(k) * m / temperature + 4e-6 * (1 + m / temperature)))
    assert not loss.cpu().numpy()[ol == 0][wt[ol == 0] == 0].any()
    dh, dw = op.backward(h, w, ids, teacher, weight, dloss)
    gh, gw = od.distill_loss_backward(*args, dl, excluded, temperature)
    off = 2 * (e32(k) * m + 2e-6 * (temperature + m)) / temperature
    size = off * np.abs(wt * dl) / temperature
    for name, a, b, n, left in (("dh", dh, gh, v, size.max() * np.abs(f64(w)).max()),
                                ("dw", dw, gw, t, size.sum() * np.abs(hh).max())):
        u, tol = (parity.BF16_U, parity.GRAD_TOL) if h.dtype == B else (0.0, e32(n) + off)
        within(name, a, b, u * np.abs(b) + tol * np.abs(b).max() + left)
    known = (ids >= 0) & (ids < v) & (ids != excluded) & (teacher != -math.inf)
    out = (wt == 0) | ~known.any(1).cpu().numpy()
    assert not loss.cpu().numpy()[out].any() and not lse.cpu().numpy()[out].any()
    assert not op._buf["z"].cpu().numpy()[out].any()
    assert not dh.float().cpu().numpy()[out | (dl == 0)].any()
    if excluded >= 0:
        assert not dw[excluded].any()
    return op


@pytest.mark.parametrize("t", [1, 2, 31, 64, 65, 128, 130, 300])
@pytest.mark.parametrize("dtype", [B, F])
def test_rows(t, dtype):
    check(*case(t, 64, 500, 6, dtype, counted=1.0 if t < 3 else 0.6, ragged=t > 2, seed=t))


@pytest.mark.parametrize("k,v,n", [(1, 2, 1), (8, 1, 1), (7, 33, 40), (64, 31, 8), (65, 257, 32), (451, 1000, 33),
                                   (72, 5001, 64)])
@pytest.mark.parametrize("dtype", [B, F])
def test_widths(k, v, n, dtype):
    check(*case(70, k, v, n, dtype, seed=k + v), excluded=v - 1 if v > 2 else -1)


@pytest.mark.parametrize("temperature", [0.5, 2.0, 7.3])
@pytest.mark.parametrize("dtype", [B, F])
def test_temperatures(temperature, dtype):
    check(*case(90, 64, 300, 12, dtype), excluded=7, temperature=temperature)


def test_options():
    h, w, ids, teacher, weight, dloss = case(90, 64, 300, 5, B)
    check(h, w, ids, teacher, None, dloss)
    check(h, w, ids, teacher, weight, None)
    check(h, w, ids, teacher, None, None, excluded=0)
    check(h, w, ids, teacher, -weight, dloss)
    check(*case(90, 64, 300, 5, B, ld=8))
    check(*case(90, 64, 300, 5, F, ld=3))
    dloss[::3] = 0.0
    check(h, w, ids, teacher, weight, dloss)


@pytest.mark.parametrize("dtype", [B, F])
def test_entries_that_are_not_known(dtype):
    """Ids outside the vocabulary, the excluded one, logits of minus infinity; rows without any, with hidden garbage."""
    h, w, ids, teacher, weight, dloss = case(60, 64, 300, 4, dtype, counted=1.0, ragged=False)
    ids[0] = -1
    ids[1] = torch.tensor([300, -7, 2 ** 40, -2 ** 40], device="cuda")
    ids[2] = 299  # excluded, in all places
    ids[3, 1:] = torch.tensor([299, -1, 300], device="cuda")
    teacher[4] = -math.inf
    teacher[5, 1:] = -math.inf
    teacher[6, 0] = -1e38  # possible, but without a share
    teacher[7] = 1e30
    teacher[0] = math.nan  # beside ids that are not known
    h[0], h[1], h[2], h[4] = math.nan, math.inf, -math.inf, math.nan
    check(h, w, ids, teacher, weight, dloss, excluded=299)


@pytest.mark.parametrize("dtype", [B, F])
def test_scales_that_vanish_in_their_product(dtype):
    """A weight and a dloss whose product is below fp32: the row counts, its gradient is zero, and nothing that was
    left in memory comes into it."""
    h, w, ids, teacher, weight, dloss = case(60, 64, 300, 4, dtype, counted=1.0, ragged=False)
    weight[3], dloss[3] = 1e-30, 1e-30
    weight[4], dloss[5] = 1e30, 1e-35
    op = DistillLoss(60, 64, 300, 4, dtype)
    op.forward(h, w, ids, teacher, weight)
    op.backward(h, w, ids, teacher, weight, dloss)
    for t in [op._buf["workspace"], *op._outgrown]:
        t.fill_(255)  # NaN as bf16 and as fp32
    dh, dw = op.backward(h, w, ids, teacher, weight, dloss)
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all() and not dh[3].any()


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("v", [1, 40, 700])
def test_ids_that_come_twice(dtype, v):
    h, w, ids, teacher, weight, dloss = case(50, 32, v, 64, dtype, counted=1.0, ragged=False)
    ids = torch.randint(0, min(v, 9), ids.shape, device="cuda")
    check(h, w, ids, teacher, weight, dloss)
    check(h, w, ids, teacher * 0, weight, dloss, temperature=3.0)
    ids[:] = 0
    op = check(h, w, ids, teacher, weight, dloss)
    if v == 1:
        dh, dw = op.backward(h, w, ids, teacher, weight, dloss)
        assert dh.abs().max() < 1e-5 and dw.abs().max() < 1e-4  # the only entry has probability one on both sides


def test_one_entry_is_the_vocabulary_loss():
    """With one known entry q is one there: the same loss and the same gradients as for a target. In bf16 each side
    rounds a term of a sum twice at most (p - q with its part of the row's scale, and for dw the scaled h), by 2^-8 of
    it each, and the result once: 4 2^-8 of the sum of the terms' sizes and 2 2^-8 of the result between the two."""
    for dtype in (B, F):
        h, w, ids, teacher, weight, dloss = case(200, 64, 700, 1, dtype, ragged=False)
        a, b = DistillLoss(200, 64, 700, 1, dtype, 699), LmLoss(200, 64, 700, dtype, 699)
        target = ids[:, 0].contiguous()
        for x, y in zip(a.forward(h, w, ids, teacher, weight), b.forward(h, w, target, weight)):
            torch.testing.assert_close(x, y, rtol=1e-5, atol=2e-5)
        dz = torch.softmax(h.double() @ w.double().t(), 1)
        dz[torch.arange(200), target] -= 1
        dz = (dz * (weight * dloss)[:, None]).abs()
        sizes = (dz @ w.double().abs(), dz.t() @ h.double().abs())
        for x, y, size in zip(a.backward(h, w, ids, teacher, weight, dloss),
                              b.backward(h, w, target, weight, dloss), sizes):
            u = 2.0 ** -8 if dtype == B else 2.0 ** -16
            assert ((x.double() - y.double()).abs() <= 4 * u * size + 2 * u * y.double().abs() + 1e-7).all()


@pytest.mark.parametrize("t", [1, 2, 3, 7, 16, 17, 40, 128])
def test_gradients_of_a_few_rows_are_rounded_once(t):
    # Up to 16 rows count, and dw's rows at their entries are sums of at most 16 fp32 terms, rounded once: off by 2^-8
    # of their value at most, and by the terms' own share of them. A term's p - q is off by s = (2 e(k) M + 4e-6 (1 + M))
    # of p + q <= 2, and each sum by 16 x 2^-24; entries that are no row's own come from p rounded to bf16, 2^-8 of p, times
    # a copy of h rounded likewise: both at most 2^-8 of the terms.
    k, v, n = 448, 5000, 8
    for seed in range(6):
        h, w, ids, teacher, weight, dloss = case(t, k, v, n, B, min(1.0, 5 / t), False, 100 + seed)
        weight[torch.nonzero(weight)[16:, 0]] = 0.0
        op = DistillLoss(t, k, v, n)
        op.forward(h, w, ids, teacher, weight)
        dw = op.backward(h, w, ids, teacher, weight, dloss)[1].double().cpu()
        hd, wd, wt = h.double().cpu(), w.double().cpu(), (weight * dloss).double().cpu()
        z = hd @ wd.T
        p = torch.softmax(z, 1)
        q = torch.zeros(t, v, dtype=torch.float64)
        q.scatter_add_(1, ids.cpu(), torch.softmax(teacher.double().cpu(), 1))
        want = (wt[:, None] * (p - q)).T @ hd
        m = float(z.abs().max())
        share = 2 * (2 * e32(k) * m + 4e-6 * (1 + m)) + 16 * 2.0 ** -24
        own = torch.zeros(t, v, dtype=torch.bool).scatter_(1, ids.cpu(), True) & (wt != 0)[:, None]
        sizes = (wt.abs()[:, None] * (p + q)).T @ hd.abs()
        others = (wt.abs()[:, None] * p * ~own).T @ hd.abs()
        tol = 2.0 ** -8 * want.abs() + share * sizes + 2 * 2.0 ** -8 * others
        at = own.any(0)
        bad = ((dw - want).abs() - tol)[at]
        assert not at.any() or bad.max() <= 0, (seed, float(bad.max()))


@pytest.mark.parametrize("t", [32, 129, 256, 2500])
@pytest.mark.parametrize("count", [1, 5, 17, 32])
def test_few_rows_that_count_whatever_the_call_holds(t, count):
    """dw rounded once as above, for any number of other rows, and dh as of a call of those rows alone: with the same
    statistics the same gradients are rounded at the entries, so that what is between the two calls is each result's
    rounding, 2^-8 of it, that of p elsewhere, 2^-8 of the terms in each, and fp32 sums over the vocabulary."""
    k, v, n = 448, 5000, 24
    for seed in range(3):
        h, w, ids, teacher, _, dloss = case(t, k, v, n, B, 1.0, False, 200 + seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        at = torch.randperm(t, generator=g, device="cuda")[:count].sort().values
        weight = torch.zeros(t, device="cuda")
        weight[at] = torch.rand(count, generator=g, device="cuda") + 0.1
        op, alone = DistillLoss(t, k, v, n), DistillLoss(count, k, v, n)
        op.forward(h, w, ids, teacher, weight)
        dh, dw = op.backward(h, w, ids, teacher, weight, dloss)
        few = [u[at].contiguous() for u in (h, ids, teacher, weight, dloss)]
        alone.forward(few[0], w, *few[1:4])
        alone._buf["lse"].copy_(op._buf["lse"][at])
        alone._buf["z"].copy_(op._buf["z"][at])
        dh_alone = alone.backward(few[0], w, *few[1:])[0].double().cpu()
        hd, wd, wt = few[0].double().cpu(), w.double().cpu(), (few[3] * few[4]).double().cpu()
        z, where = hd @ wd.T, few[1].cpu()
        p, q = torch.softmax(z, 1), torch.zeros(count, v, dtype=torch.float64)
        q.scatter_add_(1, where, torch.softmax(few[2].double().cpu(), 1))
        own = torch.zeros(count, v, dtype=torch.bool).scatter_(1, where, True)
        rest, both = wt[:, None] * p * ~own, wt[:, None] * (p + q)
        share = 2 * (2 * e32(k) * float(z.abs().max()) + 4e-6 * (1 + float(z.abs().max())))
        want, got = (wt[:, None] * (p - q)).T @ hd, dw.double().cpu()
        tol = 2.0 ** -8 * (want.abs() + 2 * rest.T @ hd.abs()) + (share + 32 * 2.0 ** -24) * (both.T @ hd.abs())
        assert ((got - want).abs() - tol)[own.any(0)].max() <= 0, (seed, "dw")
        got, want = dh[at].double().cpu(), dh_alone
        tol = 2 * 2.0 ** -8 * (want.abs() + rest @ wd.abs()) + 2 * e32(v) * want.abs().max() + 1e-9
        assert ((got - want).abs() - tol).max() <= 0, (seed, "dh")
        assert not dh[weight == 0].any()


def test_a_student_that_agrees_has_no_loss():
    """Teacher and student the same over a vocabulary of which all entries are known."""
    for dtype in (B, F):
        h, w, _, _, weight, _ = case(100, 64, 48, 48, dtype, counted=1.0)
        z = h.float() @ w.float().t()
        ids = torch.arange(48, device="cuda").repeat(100, 1)
        op = DistillLoss(100, 64, 48, 48, dtype)
        loss, _ = op.forward(h, w, ids, z, weight)
        assert (loss >= 0).all() and loss.max() < 1e-5
        dh, dw = op.backward(h, w, ids, z, weight)
        assert dh.float().abs().max() < 1e-4 and dw.float().abs().max() < 1e-3


def test_values_that_are_not_finite_stay_visible():
    h, w, ids, teacher, weight, dloss = case(150, 64, 300, 4, B, counted=1.0, ragged=False)
    for what in ("h", "teacher nan", "teacher inf"):
        a, t = h.clone(), teacher.clone()
        if what == "h":
            a[5, 3] = math.nan
        else:
            t[5, 2] = math.nan if what == "teacher nan" else math.inf
        op = DistillLoss(150, 64, 300, 4, B)
        loss, _ = op.forward(a, w, ids, t, weight)
        dh, dw = op.backward(a, w, ids, t, weight, dloss)
        rest = torch.arange(150, device="cuda") != 5
        assert torch.isnan(loss[5]) and torch.isfinite(loss[rest]).all()
        assert not torch.isfinite(dh[5]).any() and torch.isfinite(dh[rest]).all()
        assert not torch.isfinite(dw).all()


@pytest.mark.parametrize("dtype", [B, F])
def test_vocabulary_in_several_pieces(dtype):
    """16384 rows: the gradient at the logits does not fit one piece; a few rows against the oracle, the rest zero."""
    t, k, v, n = 16384, 16, 40000, 8
    h, w, _, teacher, _, dloss = case(t, k, 8, n, dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    w = (torch.randn(v, k, generator=g, device="cuda") / 4).to(dtype)
    ids = torch.randint(0, v, (t, n), generator=g, device="cuda")
    weight = torch.zeros(t, device="cuda")
    at = torch.tensor([0, 1, 700, 8191, 8192, 16000, 16383], device="cuda")
    weight[at] = 1.0
    op = DistillLoss(t, k, v, n, dtype, 5, 1.5)
    loss, lse = op.forward(h, w, ids, teacher, weight)
    dh, dw = op.backward(h, w, ids, teacher, weight, dloss)
    args = (f64(h[at]), f64(w), ids[at].cpu().numpy(), f64(teacher[at]), np.ones(len(at)))
    ol, os_, _ = od.distill_loss_forward(*args, 5, 1.5)
    gh, gw = od.distill_loss_backward(*args, f64(dloss[at]), 5, 1.5)
    within("loss", loss[at], ol, 1e-4)
    within("lse", lse[at], os_, 1e-4)
    for name, a, b in (("dh", dh[at], gh), ("dw", dw, gw)):
        parity.assert_close(name, a.double().cpu().numpy(), b, parity.GRAD_TOL if dtype == B else 1e-4,
                            parity.BF16_U if dtype == B else 0.0)
    out = torch.ones(t, dtype=torch.bool, device="cuda")
    out[at] = False
    assert not loss[out].any() and not dh[out].any()


def test_offsets_past_32_bits():
    """h is columns of a buffer of 70,000 rows of 40,000 elements: row offsets pass 2^31 elements."""
    t, k, v, n, ld = 70000, 16, 300, 4, 40000
    wide = torch.zeros((t, ld), dtype=B, device="cuda")
    h = wide[:, 64:64 + k]
    h.copy_(torch.randn(t, k, device="cuda").to(B))
    w = torch.randn(v, k, device="cuda").to(B)
    ids = torch.randint(0, v, (t, n), device="cuda")
    teacher = torch.randn(t, n, device="cuda")
    at = torch.tensor([0, 53686, 53688, 69999], device="cuda")  # both sides of 2^31 elements
    weight = torch.zeros(t, device="cuda")
    weight[at] = 1.0
    op = DistillLoss(t, k, v, n, B)
    loss, _ = op.forward(h, w, ids, teacher, weight)
    dh, dw = op.backward(h, w, ids, teacher, weight)
    args = (f64(h[at]), f64(w), ids[at].cpu().numpy(), f64(teacher[at]), np.ones(4))
    within("loss", loss[at], od.distill_loss_forward(*args)[0], 1e-4)
    gh, gw = od.distill_loss_backward(*args, np.ones(4))
    parity.assert_close("dh", dh[at].double().cpu().numpy(), gh, parity.GRAD_TOL, parity.BF16_U)
    parity.assert_close("dw", dw.double().cpu().numpy(), gw, parity.GRAD_TOL, parity.BF16_U)
    assert int((loss != 0).sum()) <= 4


def test_two_streams_with_a_holder_each():
    args = [case(200, 64, 700, 9, B, seed=i) for i in (1, 2)]
    ops = [DistillLoss(200, 64, 700, 9, B, 3, 2.0) for _ in args]

    def step(o, a, s=None):
        return (*o.forward(*a[:5], stream=s), *o.backward(*a, stream=s))

    want = [[t.clone() for t in step(o, a)] for o, a in zip(ops, args)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(8):
        got = [step(o, a, s) for o, a, s in zip(ops, args, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for g, v in zip(got, want) for p, q in zip(g, v))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("k,ld", [(72, 0), (72, 3), (71, 0)])
@pytest.mark.parametrize("rows", [40, 2100])
def test_student_logits_of_entries_that_are_not_known(rows, k, ld, dtype):
    """Zero, also beside a NaN or an infinity in the row, whatever way the rows are read; what is known shows it."""
    h, w, ids, teacher, weight, _ = case(rows, k, 300, 6, dtype, counted=1.0, ragged=False, ld=ld)
    ids[3, 2], ids[3, 5], ids[4, 0], ids[5, 1:] = -1, 300, 299, -1
    teacher[4, 3] = -math.inf
    h[3, 1], h[4, 2], h[5, 3] = math.nan, math.inf, -math.inf
    op = DistillLoss(rows, k, 300, 6, dtype, 299)
    loss, _ = op.forward(h, w, ids, teacher, weight)
    z = op._buf["z"]
    known = (ids >= 0) & (ids < 299) & (teacher != -math.inf)
    at = torch.tensor([3, 4, 5], device="cuda")
    assert not z[~known].any()
    assert not torch.isfinite(z[at][known[at]]).any() and not torch.isfinite(loss[at]).any()
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.isfinite(z[rest]).all() and torch.isfinite(loss[rest]).all()


def test_no_rows():
    op = DistillLoss(0, 64, 100, 4)
    h, w = torch.zeros(0, 64, device="cuda", dtype=B), torch.ones(100, 64, device="cuda", dtype=B)
    ids, teacher = torch.zeros(0, 4, device="cuda", dtype=torch.int64), torch.zeros(0, 4, device="cuda")
    assert op.forward(h, w, ids, teacher)[0].shape == (0,)
    dh, dw = op.backward(h, w, ids, teacher)
    assert dh.shape == (0, 64) and not dw.any()


def test_gradients_against_differences():
    h, w, ids, teacher, weight, dloss = case(4, 12, 30, 5, F, counted=1.0)
    op = DistillLoss(4, 12, 30, 5, F, 29, 1.4)
    op.forward(h, w, ids, teacher, weight)
    dh, dw = (v.clone() for v in op.backward(h, w, ids, teacher, weight, dloss))

    def value(*hw):
        return float((op.forward(*hw, ids, teacher, weight)[0].double() * dloss.double()).sum())

    step = 2.0 ** -7
    for place, grad, at in ((0, dh, (1, 3)), (0, dh, (3, 11)), (1, dw, (int(ids[0].max()), 2)), (1, dw, (7, 5)),
                            (1, dw, (29, 5))):
        lo, hi = [h.clone(), w.clone()], [h.clone(), w.clone()]
        lo[place][at] -= step
        hi[place][at] += step
        # forward errors of 4e-6 over 2 step, and step^2 times a third derivative of order ten
        assert abs((value(*hi) - value(*lo)) / (2 * step) - float(grad[at])) < 2e-3


@pytest.mark.parametrize("rows", [40, 300, 2500])
def test_same_bits_and_captured_replays(rows):
    h, w, ids, teacher, weight, dloss = case(rows, 64, 700, 9, B)
    op = DistillLoss(rows, 64, 700, 9, B, 3, 2.0)

    def step():
        return (*op.forward(h, w, ids, teacher, weight), *op.backward(h, w, ids, teacher, weight, dloss))

    want = [t.clone() for t in step()]
    assert all(torch.equal(p, q) for p, q in zip(want, step()))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = step()
    old = weight.clone()
    weight.zero_()  # a replay with no row that counts
    graph.replay()
    torch.cuda.synchronize()
    assert not any(t.any() for t in got)
    weight.copy_(old)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_teacher_to_student():
    """The set as it is used: a teacher's logits give its likeliest entries, and a gated block under a head learns
    from them; loss and every gradient against 64 bits."""
    t, k, n, v, top = 130, 64, 96, 500, 8
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(t, k, generator=g, device="cuda")
    wg = torch.randn(2 * n, k, generator=g, device="cuda") / 8
    wd = torch.randn(k, n, generator=g, device="cuda") / 10
    head = torch.randn(v, k, generator=g, device="cuda") / 4
    logits = torch.randn(t, v, generator=g, device="cuda") * 3
    weight = (torch.rand(t, generator=g, device="cuda") < 0.5).float() / t
    _, _, ids, best = TokenScores(t, v, top, F, v - 1).forward(logits)
    block, down = GatedLinear(t, k, n, "silu", F), Linear(t, n, k, dtype=F)
    loss = DistillLoss(t, k, v, top, F, v - 1, 2.0)
    a = block.forward(x, wg)
    h = down.forward(a, wd, residual=x)
    per_row, _ = loss.forward(h, head, ids, best, weight)
    dh, dhead = loss.backward(h, head, ids, best, weight)
    da, dwd, _ = down.backward(a, wd, dh, bias=False)
    dx, dwg, _ = block.backward(x, wg, da)
    xs, gs, ds, hs = (u.double().requires_grad_(True) for u in (x, wg, wd, head))
    z = xs @ gs.t()
    hh = (z[:, :n] * torch.sigmoid(z[:, :n]) * z[:, n:]) @ ds.t() + xs
    zz = hh @ hs.t() / 2.0
    zz = torch.cat((zz[:, :-1], torch.full((t, 1), -math.inf, device="cuda", dtype=torch.float64)), 1)
    teacher = logits.double()[:, :-1].topk(top, 1)
    assert torch.equal(ids, teacher.indices)
    q = torch.softmax(teacher.values / 2.0, 1)
    lp = torch.log_softmax(zz, 1).gather(1, ids)
    want = (q * (q.log() - lp)).sum(1) * weight.double()
    gx, gg, gd, gh = torch.autograd.grad(want.sum(), (xs, gs, ds, hs))
    for p, r in ((per_row, want), (dx + dh, gx), (dwg, gg), (dwd, gd), (dhead, gh)):
        r = r.detach()
        assert float((p.double() - r).abs().max()) < 2e-5 * float(r.abs().max())
