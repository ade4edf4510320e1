"""Outputs that share memory with inputs, on the host: the test of two strided
pieces of memory against one byte by byte, and the calls that are refused for it
before anything touches a GPU."""

import os
import shutil
import subprocess
import tempfile

import pytest

from paper_2607_02805_gb300 import binding as b

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02805_gb300", "csrc")

PROG = r"""
#include <vector>
#include "overlap.h"
int main() {
  using namespace bds;
  unsigned long long seed = 1;
  auto draw = [&](int lo, int hi) {
    seed = seed * 6364136223846793005ull + 1442695040888963407ull;
    return lo + (int)((seed >> 33) % (unsigned)(hi - lo + 1));
  };
  int wrong = 0, yes = 0, no = 0;
  for (int i = 0; i < 100000; ++i) {
    Span s[2];
    for (int k = 0; k < 2; ++k) {
      const int ld = k == 1 && draw(0, 1) ? (int)s[0].ld : draw(1, 20);
      s[k] = Span{"", (const void*)(uintptr_t)draw(100, 300), draw(0, 9), draw(1, ld), ld};
    }
    std::vector<char> in(1000, 0);
    bool shared = false;
    for (int k = 0; k < 2; ++k)
      for (int64_t r = 0; r < s[k].rows; ++r)
        for (int64_t c = 0; c < s[k].row; ++c) {
          char& at = in[(uintptr_t)s[k].at + r * s[k].ld + c];
          shared |= k == 1 && at == 1;
          at |= k == 0;
        }
    (shared ? yes : no) += 1;
    wrong += overlap(s[0], s[1]) != shared || overlap(s[1], s[0]) != shared;
  }
  const Span none = dense_span("", nullptr, 100), far{"", (const void*)(1ull << 46), 1 << 27, 1 << 20, 1ll << 32};
  wrong += overlap(none, none) || overlap(none, far) || overlap(dense_span("", (const void*)64, 64), far);
  wrong += !overlap(dense_span("", (const void*)((1ull << 46) + (5ll << 32) + 7), 1), far);
  std::printf("%d %d %d", wrong, yes > 1000, no > 1000);
}
"""


def test_strided_pieces_byte_by_byte():
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "t.cpp"), os.path.join(tmp, "t")
        with open(src, "w") as f:
            f.write(PROG)
        subprocess.run([gxx, "-std=c++17", "-O2", "-I" + CSRC, src, "-o", exe], check=True)
        assert subprocess.run([exe], capture_output=True, text=True, check=True).stdout == "0 1 1"


def at(i, off=0):
    """Addresses 2^36 bytes apart, which no call below dereferences: each of them is refused."""
    return (i + 1 << 36) + off


GATED = dict(rows=100, d_in=64, d_hidden=96, act=b.BDSCAN_ACT_SILU, dtype=b.BDSCAN_BF16)
SCORES = dict(rows=50, vocab=100, top=4, dtype=b.BDSCAN_BF16)
DISTILL = dict(rows=50, d_model=64, vocab=100, top=4, dtype=b.BDSCAN_F32)
CALLS = {
    "linear": (b.make_linear_dims, dict(rows=100, d_in=64, d_out=96, dtype=b.BDSCAN_BF16), b.bdscan_linear_forward,
               ["x", "w", "bias", "residual", "pre", "y"], True),
    "gated": (b.make_gated_linear_dims, GATED, b.bdscan_gated_linear_forward, ["x", "w", "bias", "y"], True),
    "gated backward": (b.make_gated_linear_dims, GATED, b.bdscan_gated_linear_backward,
                       ["x", "w", "bias", "dy", "dx", "dw", "dbias"], True),
    "scores": (b.make_token_scores_dims, SCORES, b.bdscan_token_scores_forward,
               ["logits", "token", "logp", "entropy", "stats", "top_ids", "top_logp"], False),
    "scores backward": (b.make_token_scores_dims, SCORES, b.bdscan_token_scores_backward,
                        ["logits", "token", "stats", "entropy", "dlogp", "dentropy", "dlogits"], False),
    "distill": (b.make_distill_loss_dims, DISTILL, b.bdscan_distill_loss_forward,
                ["h", "w", "ids", "teacher", "weight", "loss", "lse", "z"], True),
    "distill backward": (b.make_distill_loss_dims, DISTILL, b.bdscan_distill_loss_backward,
                         ["h", "w", "ids", "teacher", "weight", "lse", "z", "dloss", "dh", "dw"], True),
}


@pytest.mark.parametrize("call,read,written,off,dims", [
    ("linear", "x", "y", 0, {}), ("linear", "x", "y", 64, {}), ("linear", "w", "y", 0, {}), ("linear", "bias", "y", 16, {}),
    ("linear", "x", "pre", 0, {}), ("linear", "residual", "y", 16, {}), ("linear", "residual", "y", 0, dict(ld_y=104)),
    ("linear", "x", "y", 0, dict(rows=3)), ("linear", "x", "y", 16, dict(ld_x=200, ld_y=200)),
    ("linear", "x", "y", 256, dict(ld_x=200, ld_y=200)),  # its last columns are x's first of the next row
    ("gated", "x", "y", 0, {}), ("gated", "x", "y", 96, dict(ld_x=160, ld_y=160)), ("gated", "w", "y", 0, {}),
    ("gated", "bias", "y", 0, {}), ("gated", "x", "y", 64, dict(rows=2)), ("gated", "w", "y", 1600, dict(rows=1)),
    ("gated backward", "x", "dx", 0, {}), ("gated backward", "x", "dw", 0, {}), ("gated backward", "dy", "dx", 16, {}),
    ("gated backward", "w", "dw", 0, {}), ("gated backward", "bias", "dbias", 0, {}),
    ("gated backward", "w", "dbias", 160, {}),
    ("scores", "logits", "top_logp", 0, {}), ("scores", "logits", "entropy", 32, {}), ("scores", "logits", "stats", 0, {}),
    ("scores", "token", "top_ids", 0, {}), ("scores", "token", "top_ids", 400 - 16, {}), ("scores", "token", "logp", 0, {}),
    ("scores backward", "logits", "dlogits", 16, {}), ("scores backward", "token", "dlogits", 0, {}),
    ("scores backward", "logits", "dlogits", 32, dict(ld_logits=128, ld_dlogits=128)),
    ("scores backward", "logits", "dlogits", 96, dict(ld_logits=128, ld_dlogits=128)),
    ("scores backward", "stats", "dlogits", 0, {}), ("scores backward", "entropy", "dlogits", 0, {}),
    ("scores backward", "dlogp", "dlogits", 0, {}), ("scores backward", "dentropy", "dlogits", 0, {}),
    ("distill", "h", "z", 0, {}), ("distill", "w", "loss", 0, {}), ("distill", "ids", "z", 16, {}),
    ("distill", "teacher", "z", 0, {}), ("distill", "weight", "lse", 0, {}), ("distill", "weight", "loss", 16, {}),
    ("distill backward", "h", "dh", 0, {}), ("distill backward", "w", "dw", 0, {}), ("distill backward", "h", "dw", 0, {}),
    ("distill backward", "z", "dh", 0, {}), ("distill backward", "teacher", "dw", 0, {}),
    ("distill backward", "weight", "dh", 0, {}), ("distill backward", "lse", "dh", 0, {}),
    ("distill backward", "ids", "dh", 0, {}), ("distill backward", "dloss", "dh", 0, {}),
])
def test_calls_that_would_read_what_they_write(call, read, written, off, dims):
    make, kw, fn, names, workspace = CALLS[call]
    ptrs = {n: at(i) for i, n in enumerate(names)}
    ptrs[written] = ptrs[read] + off  # `off` bytes behind the input's first
    tail = (at(len(names)), 1 << 40, None) if workspace else (None,)
    assert fn(make(**{**kw, **dims}), *ptrs.values(), *tail) == b.BDSCAN_ERR_ARG
    assert f"{read} overlaps {written}, which the call writes" in b.bdscan_last_error()


def test_holders_refuse_views_that_overlap(monkeypatch):
    """Views of one buffer that share columns, an output on the weights, what the holder returned under another shape."""
    torch = pytest.importorskip("torch")
    from paper_2607_02805_gb300.dense import GatedLinear, Linear, TokenScores
    monkeypatch.setattr(b, "_stream", lambda stream: None)
    dt = torch.bfloat16
    wide = torch.zeros(4, 64, dtype=dt)
    w = torch.zeros(32, 16, dtype=dt)
    gated, linear = GatedLinear(4, 16, 16, device="cpu"), Linear(4, 16, 16, device="cpu")
    scores = TokenScores(4, 16, 16, torch.float32, device="cpu")
    logits, token = torch.zeros(4, 32), torch.zeros(4, dtype=torch.int64)
    scores._buf.update(stats=torch.zeros(4, 2), entropy=torch.zeros(4), top=torch.zeros(4, 16))
    for call, name in ((lambda: gated.forward(wide[:, :16], w, out=wide[:, 8:24]), "x"),
                       (lambda: gated.forward(wide[:, 48:], w, out=wide[:, 40:56]), "x"),
                       (lambda: gated.forward(wide[:, :16], w, out=w[:4]), "w"),
                       (lambda: linear.forward(wide[:, :16], w[:16], out=w[12:16]), "w"),
                       (lambda: scores.forward(scores._buf["top"], token), "logits"),
                       (lambda: scores.backward(logits[:, :16], token, out=logits[:, 4:20]), "logits")):
        with pytest.raises(b.BdscanError, match=f"{name} overlaps"):
            call()
