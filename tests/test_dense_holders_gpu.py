"""The holders' workspaces on the GPU: a CUDA graph of one kind of call stays
good when another kind of call needs a larger workspace, and calls on a stream
of their own leave other streams' memory alone."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover - collected on CPU machines
    pytest.skip("needs a CUDA GPU", allow_module_level=True)

from paper_2607_02805_gb300 import binding  # noqa: E402
from paper_2607_02805_gb300.dense import Linear  # noqa: E402

F = torch.float32


def _case():
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(300, 448, generator=g, device="cuda")
    w = torch.randn(1792, 448, generator=g, device="cuda") / 21
    return x, w, torch.randn(300, 1792, generator=g, device="cuda")


def test_graph_of_a_forward_survives_a_backward():
    x, w, dy = _case()
    op = Linear(300, 448, 1792, "gelu", F)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ref = op.forward(x, w, save_pre=True).clone()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            y = op.forward(x, w, save_pre=True)
    torch.cuda.current_stream().wait_stream(s)
    size = op._buf["workspace"].numel()
    grads = [t.clone() for t in op.backward(x, w, dy)]
    assert op._buf["workspace"].numel() > size
    torch.cuda.synchronize()
    # whatever memory the allocator has to give now belongs to others
    others = [torch.full((size // n,), 7, dtype=torch.uint8, device="cuda") for n in (1, 2, 4) for _ in range(4)]
    with torch.cuda.stream(s):
        others += [torch.full((size // n,), 7, dtype=torch.uint8, device="cuda") for n in (1, 2, 4) for _ in range(4)]
    torch.cuda.synchronize()
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, ref)
    assert all((t == 7).all() for t in others)
    for a, c in zip(op.backward(x, w, dy), grads):
        assert torch.equal(a, c)
    assert binding.bdscan_ssd_wait_flag(1) == 0


def test_calls_on_a_given_stream():
    """stream= while another stream is current, which keeps allocating and freeing."""
    x, w, dy = _case()
    ref = Linear(300, 448, 1792, "gelu", F)
    want = [ref.forward(x, w, save_pre=True).clone()] + [t.clone() for t in ref.backward(x, w, dy)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):
        op = Linear(300, 448, 1792, "gelu", F)
        y = op.forward(x, w, save_pre=True, stream=s)
        noise = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 20, 6 << 20, 13 << 20)]
        grads = op.backward(x, w, dy, stream=s)
        noise += [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 20, 6 << 20, 13 << 20)]
        s.synchronize()
        torch.cuda.synchronize()
        for a, c in zip([y, *grads], want):
            assert torch.equal(a, c)
        assert all((t == 7).all() for t in noise)
    assert binding.bdscan_ssd_wait_flag(1) == 0


def test_graph_on_a_stream_of_its_own_outlives_the_warm_up():
    """Warm-up on the current stream, capture on another: the same buffers, freed only after both."""
    x, w, dy = _case()
    op = Linear(300, 448, 1792, "gelu", F)
    want = [op.forward(x, w, save_pre=True).clone()] + [t.clone() for t in op.backward(x, w, dy)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = [op.forward(x, w, save_pre=True), *op.backward(x, w, dy)]
    for t in got:
        t.zero_()
    g.replay()
    torch.cuda.synchronize()
    for a, c in zip(got, want):
        assert torch.equal(a, c)
    del g, op, got
    torch.cuda.synchronize()
    again = Linear(300, 448, 1792, "gelu", F)
    for a, c in zip([again.forward(x, w, save_pre=True), *again.backward(x, w, dy)], want):
        assert torch.equal(a, c)
    assert binding.bdscan_ssd_wait_flag(1) == 0
