"""examples/masked_lm_head.py: the operators together, as a training program and a server use them."""

import os
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import masked_lm_head as example  # noqa: E402


def test_training_lowers_the_loss_and_one_token_is_served():
    losses, weights = example.train(steps=5)
    # an untrained head over 8191 entries: at least the loss of equal probabilities, 9.01
    assert 8.0 < losses[0] < 12.0
    assert all(b < a for a, b in zip(losses, losses[1:]))
    x = torch.randn(1, example.WIDTH, device="cuda").bfloat16()
    logits = example.serve(x, weights)
    w_up, b_up, w_down, b_down, head = (w.double() for w in weights)
    a = torch.nn.functional.gelu(x.double() @ w_up.t() + b_up, approximate="tanh").bfloat16().double()
    h = (x.double() + a @ w_down.t() + b_down).bfloat16().double()
    want = h @ head.t()
    # two bf16 roundings on the way (of a and h, 2^-9 of each value): 2^-7 of the largest logit covers both
    assert (logits.double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()
