"""Losses that are small beside the logits: their error goes by the loss, not
by the logits."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import LmLoss  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [3, 40, 100, 300])
def test_losses_beside_large_logits(rows, dtype):
    """Every logit is one product of exact values (multiples of 1/8 up to 248), so the 64-bit loss has the library's own
    logits. What is left: an exponential good to 2^-22 per entry and a logarithm and a product in fp32, 2^-20 max(1,
    loss) with room; a log sum rounded at the size of the logits would be off by up to 248 2^-23 = 31 2^-20."""
    k, v = 64, 500
    g = torch.Generator(device="cuda").manual_seed(rows)
    h = torch.zeros(rows, k, dtype=dtype, device="cuda")
    at = torch.arange(rows, device="cuda") % k
    h[torch.arange(rows, device="cuda"), at] = 1.0
    base = torch.randint(-31, 32, (1, k), generator=g, device="cuda") * 8.0  # the size of a row's logits
    w = base + torch.randint(-64, 1, (v, k), generator=g, device="cuda") / 8.0
    w = torch.where(base.abs() > 16, base + torch.randint(-31, 1, (v, k), generator=g, device="cuda").float(), w)
    w[torch.arange(k, device="cuda"), torch.arange(k, device="cuda")] = base[0] + 4.0  # a dominant entry in each column
    w = w.to(dtype)
    z = w.double().t()[at]
    target = torch.randint(0, v, (rows,), generator=g, device="cuda")
    target[::2] = at[::2]
    loss, lse = LmLoss(rows, k, v, dtype).forward(h, w, target)
    want = torch.logsumexp(z, 1) - z.gather(1, target[:, None])[:, 0]
    assert (loss >= 0).all()
    assert ((loss.double() - want).abs() <= 2.0 ** -20 * want.clamp(min=1)).all()
    one, _ = LmLoss(rows, k, 1, dtype).forward(h, w[:1].contiguous(), torch.zeros_like(target))
    assert (one >= 0).all() and (one <= 2.0 ** -20).all()  # one entry: certain
    assert binding.bdscan_ssd_wait_flag(1) == 0
