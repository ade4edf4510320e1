"""Device-resident state for repeated calls of the dense operators
(include/bdscan_dense.h) from PyTorch.

PyTorch provides the device memory and the stream; every step of the
computation runs in libbdscan through ``binding``. A ``Linear`` or ``LmLoss``
holds one size's outputs, saved pre-activations, gradients and workspaces; the
inputs and weights belong to the caller. What a call returns are the holder's
buffers, valid until its next call; a holder serves one stream at a time, and
its buffers stay where they are for its life, so that a CUDA graph of its calls
can be replayed as long as it lives.
"""

from __future__ import annotations

import ctypes

import torch

from . import binding

ACTS = {"none": binding.BDSCAN_ACT_NONE, "silu": binding.BDSCAN_ACT_SILU, "gelu": binding.BDSCAN_ACT_GELU}
CODES = {torch.float32: binding.BDSCAN_F32, torch.bfloat16: binding.BDSCAN_BF16}

# The current stream's handle without a Stream object, where this PyTorch has the query.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _code(dtype):
    if dtype not in CODES:
        raise ValueError(f"unsupported dtype {dtype}")
    return CODES[dtype]


def _refuse(name, t, shape, dtype, index):
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, not {dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on {'the CPU' if index < 0 else f'cuda:{index}'}")
    raise ValueError(f"{name} is not contiguous")


# The checks run in every call: torch.Size compares with a tuple, dtypes are singletons, and the device's index is
# cheaper to ask for than the device.
def _whole(name, t, shape, dtype, index):
    """Address of a contiguous tensor (None stays None)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        _refuse(name, t, shape, dtype, index)
    return t.data_ptr()


def _rows(name, t, shape, dtype, index):
    """Address and row stride of a 2-D tensor with contiguous rows, each in memory of its own: the stride 0 of an
    expanded row would be read as "the row length"."""
    if t is None:
        return None, 0
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index:
        _refuse(name, t, shape, dtype, index)
    ld, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise ValueError(f"the rows of {name} are not contiguous")
    if shape[0] <= 1:
        return t.data_ptr(), shape[1]
    if ld < shape[1]:
        raise ValueError(f"the rows of {name} overlap: {shape[1]} elements every {ld}")
    return t.data_ptr(), ld


def _apart(name, at, *outputs):
    """Refuses an input (its address) that the call overwrites while it reads it: what the holder returned before."""
    if at and at in outputs:
        raise ValueError(f"{name} is a buffer that this call writes: pass a copy, or use a holder of its own")


class _Holder:
    def __init__(self, device):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index if self.device.type == "cuda" else -1
        self._plans = {}  # (kind, row strides) -> (dims, their reference, workspace address and bytes)
        self._buf = {}
        self._outgrown = []  # workspaces that a larger one replaced
        self._handle = self._stream = None  # of the last call

    def _enter(self, stream):
        """Handle of the call's stream. What the call allocates comes from that stream's memory, and what the holder
        allocated on others before is marked as used on it. The kernels go to the current device, which has to be the
        holder's."""
        index = self._index
        if index < 0:
            handle = binding._stream(stream)
        else:
            current = torch._C._cuda_getDevice()
            if current != index:
                raise ValueError(f"the holder is on {self.device}, the current device is cuda:{current}")
            handle = _raw_stream(index) if stream is None and _raw_stream is not None else binding._stream(stream)
        if handle != self._handle:
            if stream is None:
                stream = torch.cuda.current_stream()
            elif not isinstance(stream, torch.cuda.Stream):
                stream = torch.cuda.ExternalStream(handle, self.device)
            for t in [*self._buf.values(), *self._outgrown]:
                t.record_stream(stream)
            self._handle, self._stream = handle, stream
        return handle

    def _empty(self, shape, dtype):
        with torch.cuda.stream(self._stream):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _buffer(self, name, shape, dtype):
        t = self._buf.get(name)
        if t is None:
            t = self._buf[name] = self._empty(shape, dtype)
        return t

    def _plan(self, key, size):
        """What a kind of call passes for its row strides, asked for once: the dims, and address and size of the
        workspace. One workspace serves all calls of the holder, which run one after another. Where a kind of call
        needs more, the smaller one is kept: work in flight or a CUDA graph may still write there."""
        plan = self._plans.get(key)
        if plan is None:
            dims = self._make_dims(*key[1:])
            need = size(dims)
            ws = self._buf.get("workspace")
            if need and (ws is None or ws.numel() < need):
                if ws is not None:
                    self._outgrown.append(ws)
                ws = self._buf["workspace"] = self._empty(need, torch.uint8)
                self._plans = {k: v[:2] + (ws.data_ptr(), ws.numel()) for k, v in self._plans.items()}
            plan = (dims, ctypes.byref(dims)) + ((None, 0) if ws is None else (ws.data_ptr(), ws.numel()))
            self._plans[key] = plan
        return plan


class Linear(_Holder):
    """y = residual + act(x w^T + bias) for x [rows, d_in], w [d_out, d_in]."""

    def __init__(self, rows, d_in, d_out, act="none", dtype=torch.bfloat16, out_dtype=None, device="cuda"):
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}")
        _code(dtype), _code(dtype if out_dtype is None else out_dtype)
        super().__init__(device)
        self.rows, self.d_in, self.d_out, self.act = int(rows), int(d_in), int(d_out), act
        self.dtype, self.out_dtype = dtype, dtype if out_dtype is None else out_dtype
        self.pre = None
        self._x, self._w, self._y = (self.rows, self.d_in), (self.d_out, self.d_in), (self.rows, self.d_out)
        self._b = (self.d_out,)

    def _make_dims(self, ld_x, ld_res, ld_y):
        return binding.make_linear_dims(self.rows, self.d_in, self.d_out, ACTS[self.act], _code(self.dtype),
                                        _code(self.out_dtype), ld_x, ld_res, ld_y)

    def forward(self, x, w, bias=None, residual=None, save_pre=False, out=None, stream=None):
        """y (the holder's buffer, or `out`); with save_pre the pre-activations
        are kept for backward(). Without an activation there is none to keep."""
        dt, od, dev = self.dtype, self.out_dtype, self._index
        px, ld_x = _rows("x", x, self._x, dt, dev)
        pr, ld_r = _rows("residual", residual, self._y, od, dev)
        pw = _whole("w", w, self._w, dt, dev)
        pb = _whole("bias", bias, self._b, dt, dev)
        py, ld_y = _rows("out", out, self._y, od, dev)
        s = self._enter(stream)
        y = out
        if out is None:
            y = self._buffer("y", self._y, od)
            py, ld_y = y.data_ptr(), self.d_out
        _apart("x", px, py)
        self.pre = pp = None
        if save_pre and self.act != "none":
            self.pre = self._buffer("pre", self._y, dt)
            pp = self.pre.data_ptr()
        _, d, ws, size = self._plan(("forward", ld_x, ld_r, ld_y), binding.bdscan_linear_forward_workspace_size)
        binding._call("bdscan_linear_forward", d, px, pw, pb, pr, pp, py, ws, size, s)
        return y

    def backward(self, x, w, dy, bias=True, need_dx=True, need_dw=True, stream=None):
        """(dx, dw, dbias) of <dy, y>; dbias None without `bias`. The
        residual's gradient is dy."""
        dt, dev = self.dtype, self._index
        px, ld_x = _rows("x", x, self._x, dt, dev)
        py, ld_y = _rows("dy", dy, self._y, self.out_dtype, dev)
        pw = _whole("w", w, self._w, dt, dev)
        if self.act != "none" and self.pre is None:
            raise ValueError("backward needs a forward with save_pre=True")
        s = self._enter(stream)
        dx = self._buffer("dx", self._x, dt) if need_dx else None
        dw = self._buffer("dw", self._w, dt) if need_dw else None
        db = self._buffer("dbias", self._b, dt) if bias else None
        p = binding._ptr
        qx, qw = p(dx), p(dw)
        _apart("x", px, qx)
        _apart("dy", py, qx)
        _apart("w", pw, qw)
        _, d, ws, size = self._plan(("backward", ld_x, 0, ld_y), binding.bdscan_linear_backward_workspace_size)
        binding._call("bdscan_linear_backward", d, px, pw, p(self.pre), py, qx, qw, p(db), ws, size, s)
        return dx, dw, db


class LmLoss(_Holder):
    """Weighted softmax cross entropy of h w^T at the rows that count, for
    h [rows, d_model], w [vocab, d_model]; include/bdscan_dense.h has the rules."""

    def __init__(self, rows, d_model, vocab, dtype=torch.bfloat16, excluded=-1, device="cuda"):
        _code(dtype)
        super().__init__(device)
        self.rows, self.d_model, self.vocab, self.dtype = int(rows), int(d_model), int(vocab), dtype
        self.excluded = int(excluded)
        self._h, self._w, self._t = (self.rows, self.d_model), (self.vocab, self.d_model), (self.rows,)

    def _make_dims(self, ld_h):
        return binding.make_lm_loss_dims(self.rows, self.d_model, self.vocab, _code(self.dtype), self.excluded, ld_h)

    def _inputs(self, h, w, target, weight):
        ph, ld_h = _rows("h", h, self._h, self.dtype, self._index)
        return ld_h, (ph, _whole("w", w, self._w, self.dtype, self._index),
                      _whole("target", target, self._t, torch.int64, self._index),
                      _whole("weight", weight, self._t, torch.float32, self._index))

    def forward(self, h, w, target, weight=None, stream=None):
        """(loss, lse), fp32 per row; zero at the rows that do not count."""
        ld_h, inputs = self._inputs(h, w, target, weight)
        s = self._enter(stream)
        loss = self._buffer("loss", self._t, torch.float32)
        lse = self._buffer("lse", self._t, torch.float32)
        _, d, ws, size = self._plan(("forward", ld_h), binding.bdscan_lm_loss_forward_workspace_size)
        binding._call("bdscan_lm_loss_forward", d, *inputs, loss.data_ptr(), lse.data_ptr(), ws, size, s)
        return loss, lse

    def backward(self, h, w, target, weight=None, dloss=None, lse=None, stream=None):
        """(dh, dw) of <dloss, loss>, from the last forward's lse or the one given."""
        ld_h, inputs = self._inputs(h, w, target, weight)
        pd = _whole("dloss", dloss, self._t, torch.float32, self._index)
        if lse is None:
            lse = self._buf.get("lse")
            if lse is None:
                raise ValueError("backward needs a forward or its lse")
        pl = _whole("lse", lse, self._t, torch.float32, self._index)
        s = self._enter(stream)
        dh = self._buffer("dh", self._h, self.dtype)
        dw = self._buffer("dw", self._w, self.dtype)
        _apart("h", inputs[0], dh.data_ptr())
        _apart("w", inputs[1], dw.data_ptr())
        _, d, ws, size = self._plan(("backward", ld_h), binding.bdscan_lm_loss_backward_workspace_size)
        binding._call("bdscan_lm_loss_backward", d, *inputs, pl, pd, dh.data_ptr(), dw.data_ptr(), ws, size, s)
        return dh, dw
