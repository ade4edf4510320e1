"""The bound that the fp32 tests on the GPU use for an output that is one
product, against an emulation of the pieces on the host: three pieces and six
products keep it, fewer do not."""

import pytest

torch = pytest.importorskip("torch")

SINGLE = 2.0 ** -20  # tests/test_dense_fp32_gpu.py


def pieces(v, n):
    out = []
    for _ in range(n):
        p = v.bfloat16().float()
        out.append(p.double())
        v = v - p
    return out


def product(u, v, n, pairs):
    a, b = pieces(u, n), pieces(v, n)
    return sum(a[i] * b[j] for i, j in pairs)


SIX = [(0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)]


@pytest.mark.parametrize("n,pairs,kept", [
    (3, SIX, True),
    (2, [(1, 1), (0, 1), (1, 0), (0, 0)], False),
    (2, [(0, 1), (1, 0), (0, 0)], False),
    (3, [p for p in SIX if p != (1, 1)], False),
    (3, [p for p in SIX if p != (0, 2)], False),
])
def test_bound_of_one_product(n, pairs, kept):
    g = torch.Generator().manual_seed(0)
    u, v = 1 + torch.rand(2, 4096, generator=g)
    exact = u.double() * v.double()
    worst = ((product(u, v, n, pairs) - exact).abs() / exact).max().item()
    assert worst <= SINGLE / 8 if kept else worst > SINGLE
