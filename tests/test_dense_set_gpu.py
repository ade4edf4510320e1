"""The gated linear layer, the distillation loss and the token scores through the
functions of the binding, and through the debug build: valid calls to the bounds of the release build's tests, and an
extent that is one element short is reported by its kernel and not touched."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

import test_distill_gpu  # noqa: E402
import test_gated_gpu  # noqa: E402
import test_scores_gpu  # noqa: E402
from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import DistillLoss, GatedLinear, Linear, TokenScores  # noqa: E402

B, F = torch.bfloat16, torch.float32


@pytest.fixture
def debug():
    def call(f):
        binding.use_debug_build(True)
        try:
            return f()
        finally:
            binding.use_debug_build(False)
    yield call
    binding.use_debug_build(False)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("t,k,n", [(5, 64, 72), (300, 65, 40), (300, 64, 136)])
def test_gated(debug, dtype, t, k, n):
    debug(lambda: test_gated_gpu.check(t, k, n, "silu", dtype))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows,vocab", [(3, 900), (3, 40000), (200, 9000)])
def test_scores(debug, dtype, rows, vocab):
    z, token, dl, dh = test_scores_gpu.draw(rows, vocab, dtype)
    debug(lambda: test_scores_gpu.check(z, token, 5, 3, 0.8, dl, dh))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows", [40, 2500])
def test_distill(debug, dtype, rows):
    args = test_distill_gpu.case(rows, 64, 300, 7, dtype, counted=0.1)
    debug(lambda: test_distill_gpu.check(*args, excluded=299, temperature=1.5))


def test_scores_extent_that_is_short(debug):
    z, token, _, _ = test_scores_gpu.draw(40, 9000, B)
    op = TokenScores(40, 9000, 5, B)
    want = [v.clone() for v in op.forward(z, token)]

    def short():
        binding.bdscan_debug_set_slack(1)
        try:
            op.forward(z, token)
        finally:
            binding.bdscan_debug_set_slack(0)

    with pytest.raises(binding.BdscanError, match="k_scores") as e:
        debug(short)
    assert e.value.code == binding.BDSCAN_ERR_DEVICE
    assert all(torch.equal(p, q) for p, q in zip(want, debug(lambda: op.forward(z, token))))


def test_functions_of_the_binding():
    """The C functions by way of the binding, with memory of the caller's: what the holders give."""
    g = torch.Generator(device="cuda").manual_seed(0)

    def draw(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(B)

    def empty(*shape, dtype=B):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    def space(n):
        return torch.empty(n, device="cuda", dtype=torch.uint8) if n else None

    x, w, dy = draw(100, 64), draw(144, 64, std=0.1), draw(100, 72)
    d = binding.make_gated_linear_dims(100, 64, 72)
    y, dx, dw = empty(100, 72), empty(100, 64), empty(144, 64)
    binding.gated_linear_forward(d, x, w, None, y, space(binding.bdscan_gated_linear_forward_workspace_size(d)))
    binding.gated_linear_backward(d, x, w, None, dy, dx, dw, None,
                                  space(binding.bdscan_gated_linear_backward_workspace_size(d)))
    op = GatedLinear(100, 64, 72)
    assert torch.equal(y, op.forward(x, w)) and all(torch.equal(p, q) for p, q in zip((dx, dw), op.backward(x, w, dy)))

    z, token = draw(100, 300, std=3.0), torch.arange(100, device="cuda")
    d = binding.make_token_scores_dims(100, 300, 4, excluded=299, temperature=0.9)
    logp, entropy, best = empty(100, dtype=F), empty(100, dtype=F), empty(100, 4, dtype=F)
    stats, ids, dz = empty(100, 2, dtype=F), empty(100, 4, dtype=torch.int64), empty(100, 300)
    binding.token_scores_forward(d, z, token, logp, entropy, stats, ids, best)
    binding.token_scores_backward(d, z, token, stats, entropy, logp, entropy, dz)
    op = TokenScores(100, 300, 4, excluded=299, temperature=0.9)
    assert all(torch.equal(p, q) for p, q in zip((logp, entropy, ids, best), op.forward(z, token)))
    assert torch.equal(dz, op.backward(z, token, logp, entropy))

    h, head = draw(100, 72), draw(300, 72, std=0.2)
    d = binding.make_distill_loss_dims(100, 72, 300, 4, excluded=299, temperature=1.1)
    loss, lse, zs = empty(100, dtype=F), empty(100, dtype=F), empty(100, 4, dtype=F)
    dh, dhead = empty(100, 72), empty(300, 72)
    binding.distill_loss_forward(d, h, head, ids, best, None, loss, lse, zs,
                                 space(binding.bdscan_distill_loss_forward_workspace_size(d)))
    binding.distill_loss_backward(d, h, head, ids, best, None, lse, zs, None, dh, dhead,
                                  space(binding.bdscan_distill_loss_backward_workspace_size(d)))
    op = DistillLoss(100, 72, 300, 4, excluded=299, temperature=1.1)
    assert all(torch.equal(p, q) for p, q in zip((loss, lse), op.forward(h, head, ids, best)))
    assert all(torch.equal(p, q) for p, q in zip((dh, dhead), op.backward(h, head, ids, best)))


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("rows", [2, 40])
def test_columns_side_by_side_share_nothing(rows, dtype):
    """Inputs and outputs between one another's columns of one buffer: as with buffers of their own."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    wide = torch.randn(rows, 200, generator=g, device="cuda").to(dtype)
    w = torch.randn(128, 64, generator=g, device="cuda").to(dtype) / 8
    x, y = wide[:, 8:72], wide[:, 72:136]  # directly behind one another
    for op, weights in ((GatedLinear(rows, 64, 64, dtype=dtype), w), (Linear(rows, 64, 64, dtype=dtype), w[:64])):
        want = op.forward(x.clone(), weights).clone()
        assert torch.equal(op.forward(x, weights, out=y), want)
    linear = Linear(rows, 64, 64, dtype=dtype)
    want = linear.forward(x, w[:64], residual=y.clone()).clone()
    assert torch.equal(linear.forward(x, w[:64], residual=y, out=y), want)  # in place
    scores = TokenScores(rows, 64, 4, dtype)
    dh = torch.ones(rows, device="cuda")
    scores.forward(x)
    want = scores.backward(x, dentropy=dh).clone()
    assert torch.equal(scores.backward(x, dentropy=dh, out=y), want)
    assert torch.equal(scores.backward(x, dentropy=dh, out=x), want)
