"""The gated linear layer, the distillation loss and the token scores through the
debug build: valid calls to the bounds of the release build's tests, and an
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
from paper_2607_02805_gb300.dense import TokenScores  # noqa: E402

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


def draw(*shape, dtype, std=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


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
    z, token = draw(40, 9000, dtype=B, std=3.0), torch.arange(40, device="cuda")
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
