"""The dense half of a masked language model with the library's operators: an
MLP block (up projection with GELU, down projection onto the residual stream)
and the head's weighted cross entropy over the vocabulary, trained for a few
steps, then one token served.

    python examples/masked_lm_head.py [steps]

The hidden states stand in for a mixer's output: each clean token has an
embedding, and a masked token (half of them, as a masked objective draws them)
shows the mask's embedding plus a hint of its own. Plain SGD on the five weight
tensors; the loss of the masked tokens falls step by step. PyTorch provides
memory, the random numbers and the weight update; every forward and gradient
runs in libbdscan.
"""

import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2607_02805_gb300.dense import Linear, LmLoss  # noqa: E402

ROWS, WIDTH, HIDDEN, VOCAB = 2048, 448, 1792, 8192
MASK = VOCAB - 1  # never predicted


def train(steps=8, lr=0.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std):
        return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()

    embed = normal(VOCAB, WIDTH, std=1.0)
    w_up, b_up = normal(HIDDEN, WIDTH, std=WIDTH ** -0.5), torch.zeros(HIDDEN, device="cuda").bfloat16()
    w_down, b_down = normal(WIDTH, HIDDEN, std=HIDDEN ** -0.5), torch.zeros(WIDTH, device="cuda").bfloat16()
    head = normal(VOCAB, WIDTH, std=WIDTH ** -0.5)

    tokens = torch.randint(0, MASK, (ROWS,), generator=g, device="cuda")
    masked = torch.rand(ROWS, generator=g, device="cuda") < 0.5
    x = torch.where(masked[:, None], embed[MASK] + 0.5 * embed[tokens], embed[tokens])
    weight = masked.float() / masked.sum()  # only masked tokens count

    up = Linear(ROWS, WIDTH, HIDDEN, act="gelu")
    down = Linear(ROWS, HIDDEN, WIDTH)
    loss = LmLoss(ROWS, WIDTH, VOCAB, excluded=MASK)
    losses = []
    for _ in range(steps):
        a = up.forward(x, w_up, b_up, save_pre=True)
        h = down.forward(a, w_down, b_down, residual=x)
        per_token, _ = loss.forward(h, head, tokens, weight)
        losses.append(per_token.sum())
        dh, dhead = loss.backward(h, head, tokens, weight)
        da, dw_down, db_down = down.backward(a, w_down, dh)
        _, dw_up, db_up = up.backward(x, w_up, da, need_dx=False)
        for w, dw in ((w_up, dw_up), (b_up, db_up), (w_down, dw_down), (b_down, db_down), (head, dhead)):
            w.sub_(dw, alpha=lr)
    return torch.stack(losses).tolist(), (w_up, b_up, w_down, b_down, head)


def serve(x, weights):
    """The logits of one token in fp32, by the same operators with one row."""
    w_up, b_up, w_down, b_down, head = weights
    a = Linear(1, WIDTH, HIDDEN, act="gelu").forward(x, w_up, b_up)
    h = Linear(1, HIDDEN, WIDTH).forward(a, w_down, b_down, residual=x)
    return Linear(1, WIDTH, VOCAB, out_dtype=torch.float32).forward(h, head)


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 8
    losses, weights = train(steps)
    for i, v in enumerate(losses):
        print(f"step {i}: loss per masked token {v:.4f}")
    logits = serve(torch.randn(1, WIDTH, device="cuda").bfloat16(), weights)
    logits[:, MASK] = -float("inf")
    print("most likely token of a random state:", int(logits.argmax()))


if __name__ == "__main__":
    main()
