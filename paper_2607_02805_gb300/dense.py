"""Device-resident state for repeated calls of the dense operators
(include/bdscan_dense.h) from PyTorch.

PyTorch provides the device memory and the stream; every step of the
computation runs in libbdscan through ``binding``. A ``Linear`` or ``LmLoss``
holds one size's outputs, saved pre-activations, gradients and workspaces; the
inputs and weights belong to the caller. What a call returns are the holder's
buffers, valid until its next call; a holder serves one stream at a time.
"""

from __future__ import annotations

import torch

from . import binding

ACTS = {"none": binding.BDSCAN_ACT_NONE, "silu": binding.BDSCAN_ACT_SILU, "gelu": binding.BDSCAN_ACT_GELU}
CODES = {torch.float32: binding.BDSCAN_F32, torch.bfloat16: binding.BDSCAN_BF16}


def _code(dtype):
    if dtype not in CODES:
        raise ValueError(f"unsupported dtype {dtype}")
    return CODES[dtype]


def _check(name, t, shape, dtype, device):
    if t is None:
        return
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, not {dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


class _Holder:
    def __init__(self, device):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._dims = {}  # row strides -> (dims, forward workspace, backward workspace)
        self._buf = {}

    def _buffer(self, name, shape, dtype):
        t = self._buf.get(name)
        if t is None:
            t = self._buf[name] = torch.empty(shape, dtype=dtype, device=self.device)
        return t

    def _workspace(self, name, size, dims):
        """One workspace for all calls of a kind, of the largest size that its dims have asked for."""
        need = size(dims)
        t = self._buf.get(name)
        if need and (t is None or t.numel() < need):
            t = self._buf[name] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return t


class Linear(_Holder):
    """y = residual + act(x w^T + bias) for x [rows, d_in], w [d_out, d_in]."""

    def __init__(self, rows, d_in, d_out, act="none", dtype=torch.bfloat16, out_dtype=None, device="cuda"):
        super().__init__(device)
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}")
        self.rows, self.d_in, self.d_out, self.act = int(rows), int(d_in), int(d_out), act
        self.dtype, self.out_dtype = dtype, dtype if out_dtype is None else out_dtype
        _code(self.dtype), _code(self.out_dtype)
        self.pre = None

    def _get(self, x, residual, y):
        key = (binding.row_stride(x), 0 if residual is None else binding.row_stride(residual), binding.row_stride(y))
        d = self._dims.get(key)
        if d is None:
            d = self._dims[key] = binding.make_linear_dims(self.rows, self.d_in, self.d_out, ACTS[self.act],
                                                           _code(self.dtype), _code(self.out_dtype), *key)
        return d

    def forward(self, x, w, bias=None, residual=None, save_pre=False, out=None, stream=None):
        """y (the holder's buffer, or `out`); with save_pre the pre-activations
        are kept for backward(). Without an activation there is none to keep."""
        _check("x", x, (self.rows, self.d_in), self.dtype, self.device)
        _check("w", w, (self.d_out, self.d_in), self.dtype, self.device)
        _check("bias", bias, (self.d_out,), self.dtype, self.device)
        _check("residual", residual, (self.rows, self.d_out), self.out_dtype, self.device)
        _check("out", out, (self.rows, self.d_out), self.out_dtype, self.device)
        y = self._buffer("y", (self.rows, self.d_out), self.out_dtype) if out is None else out
        self.pre = None
        if save_pre and self.act != "none":
            self.pre = self._buffer("pre", (self.rows, self.d_out), self.dtype)
        d = self._get(x, residual, y)
        ws = self._workspace("ws_f", binding.bdscan_linear_forward_workspace_size, d)
        binding.linear_forward(d, x, w, bias, residual, self.pre, y, ws, stream)
        return y

    def backward(self, x, w, dy, bias=True, need_dx=True, need_dw=True, stream=None):
        """(dx, dw, dbias) of <dy, y>; dbias None without `bias`. The
        residual's gradient is dy."""
        _check("x", x, (self.rows, self.d_in), self.dtype, self.device)
        _check("w", w, (self.d_out, self.d_in), self.dtype, self.device)
        _check("dy", dy, (self.rows, self.d_out), self.out_dtype, self.device)
        if self.act != "none" and self.pre is None:
            raise ValueError("backward needs a forward with save_pre=True")
        dx = self._buffer("dx", (self.rows, self.d_in), self.dtype) if need_dx else None
        dw = self._buffer("dw", (self.d_out, self.d_in), self.dtype) if need_dw else None
        db = self._buffer("dbias", (self.d_out,), self.dtype) if bias else None
        d = self._get(x, None, dy)
        ws = self._workspace("ws_b", binding.bdscan_linear_backward_workspace_size, d)
        binding.linear_backward(d, x, w, self.pre, dy, dx, dw, db, ws, stream)
        return dx, dw, db


class LmLoss(_Holder):
    """Weighted softmax cross entropy of h w^T at the rows that count, for
    h [rows, d_model], w [vocab, d_model]; include/bdscan_dense.h has the rules."""

    def __init__(self, rows, d_model, vocab, dtype=torch.bfloat16, excluded=-1, device="cuda"):
        super().__init__(device)
        self.rows, self.d_model, self.vocab, self.dtype = int(rows), int(d_model), int(vocab), dtype
        self.excluded = int(excluded)
        _code(dtype)

    def _get(self, h):
        key = binding.row_stride(h)
        d = self._dims.get(key)
        if d is None:
            d = self._dims[key] = binding.make_lm_loss_dims(self.rows, self.d_model, self.vocab, _code(self.dtype),
                                                            self.excluded, key)
        return d

    def _check_inputs(self, h, w, target, weight):
        _check("h", h, (self.rows, self.d_model), self.dtype, self.device)
        _check("w", w, (self.vocab, self.d_model), self.dtype, self.device)
        _check("target", target, (self.rows,), torch.int64, self.device)
        _check("weight", weight, (self.rows,), torch.float32, self.device)

    def forward(self, h, w, target, weight=None, stream=None):
        """(loss, lse), fp32 per row; zero at the rows that do not count."""
        self._check_inputs(h, w, target, weight)
        loss = self._buffer("loss", (self.rows,), torch.float32)
        lse = self._buffer("lse", (self.rows,), torch.float32)
        d = self._get(h)
        ws = self._workspace("ws_f", binding.bdscan_lm_loss_forward_workspace_size, d)
        binding.lm_loss_forward(d, h, w, target, weight, loss, lse, ws, stream)
        return loss, lse

    def backward(self, h, w, target, weight=None, dloss=None, lse=None, stream=None):
        """(dh, dw) of <dloss, loss>, from the last forward's lse or the one given."""
        self._check_inputs(h, w, target, weight)
        _check("dloss", dloss, (self.rows,), torch.float32, self.device)
        _check("lse", lse, (self.rows,), torch.float32, self.device)
        if lse is None:
            lse = self._buf.get("lse")
            if lse is None:
                raise ValueError("backward needs a forward or its lse")
        dh = self._buffer("dh", (self.rows, self.d_model), self.dtype)
        dw = self._buffer("dw", (self.vocab, self.d_model), self.dtype)
        d = self._get(h)
        ws = self._workspace("ws_b", binding.bdscan_lm_loss_backward_workspace_size, d)
        binding.lm_loss_backward(d, h, w, target, weight, lse, dloss, dh, dw, ws, stream)
        return dh, dw
