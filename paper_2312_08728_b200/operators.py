"""Operators of a gated network's training step, and of its scoring, on device tensors.

    rows, labels = gather_batch(x, y, seed, chain, round, first, count)      the mini-batch of the shuffled buffer
    logits, saved = gated_ffn(rows, w_gate, w_up, w_down, save=True)         (act(X Wg) * (X Wu)) Wd
    residual, loss = softmax_residual(logits, labels)                        softmax loss and its gradient
    dx, dw_gate, dw_up, dw_down = gated_ffn_backward(residual, rows, w_gate, w_up, w_down, saved)
    adamw_step([w_gate, w_up, w_down], [dw_gate, dw_up, dw_down], m, v, control, lr=1e-3)

Between blocks:

    y, total, rstd = rms_norm(x, weight, residual=total, save=True)          norm of x + residual
    dx, dweight = rms_norm_backward(dy, total, weight, rstd, dtotal)         dx is the gradient of the residual too
    total = dropout(y, rate, seed, layer, step, residual=total)              its gradient: dropout(dtotal, rate, seed, layer, step)

Scored with weights in 8 bits, and the answer:

    codes, scale = quantize_weight(w)                                        laid out once
    q, q_scale, total = rms_norm_int8(x, weight, residual=total)             or quantize_rows(up, gate=gate)
    y = int8_linear(q, q_scale, codes, scale)
    logprob, entropy, classes, logprobs = log_probs(logits, labels, top=5)   log_probs_backward for its gradient

Argument checks and marshalling only: the computation runs in the CUDA library (include/bmgd.h), which takes bare
pointers, so whatever the tensors' own metadata can tell is refused here.  Work is ordered on `stream`, by default the
current stream of the tensors' device; nothing waits for the device, so every call can be captured into a CUDA graph.
Outputs and workspaces come from torch's allocator on that stream.  Where `stream` is not the current one, the order between
the two is the caller's (wait_stream or events); the memory of inputs and outputs is kept until both are done with it.

None of them is part of an autograd graph: gradients are outputs like others.  gated_ffn, rms_norm, rms_norm_int8, quantize_rows, int8_linear,
log_probs and dropout refuse tensors that require gradients where a graph would be recorded (call them under torch.no_grad(), with the
backward calls beside them), and dual tensors of forward-mode differentiation.  The other calls take both and give plain results.  adamw_step writes parameters and
copies in place and tells autograd so: a graph that has saved one of them refuses its backward pass (an update that is replayed from a
CUDA graph tells it only at its capture).
"""
from __future__ import annotations

import contextlib
import ctypes
import operator
import struct
from array import array
from typing import List, Optional, Sequence, Tuple, Union

import torch
from torch.autograd import forward_ad as _forward_ad

from . import binding as _binding
from .binding import BMGD_OK, BmgdError

ACT_SILU, ACT_GELU, ACT_RELU, ACT_SIGMOID = 0, 1, 2, 3
TYPE_F32, TYPE_BF16, TYPE_F16 = 0, 1, 2
SCALE_BLOCK = 256       # values that share a scale where moments are held in 8 bits
CONTROL_WORDS = 4

_TYPES = {torch.float32: TYPE_F32, torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16}


def _status(rc: int, where: str) -> None:
    if rc != BMGD_OK:
        raise BmgdError(rc, where)


_HERE = contextlib.nullcontext()


@contextlib.contextmanager
def _other(device: torch.device, stream: Optional[torch.cuda.Stream]):
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream):
                yield


def _place(device: torch.device, stream: Optional[torch.cuda.Stream]):
    """Context in which outputs are allocated and kernels launched: the tensors' device, on the stream that orders them."""
    if stream is not None and stream.device != device:
        raise ValueError(f"the stream belongs to {stream.device}, the tensors live on {device}")
    if stream is None and torch._C._cuda_getDevice() == device.index:
        return _HERE
    return _other(device, stream)


def _lend(stream: Optional[torch.cuda.Stream], device: torch.device, inputs) -> None:
    """Tell the allocator that a call on another stream reads or writes these tensors: a caller may drop them at once."""
    if stream is not None and stream != torch.cuda.current_stream(device):
        for t in inputs:
            if t is not None:
                t.record_stream(stream)


def _hand(stream: Optional[torch.cuda.Stream], device: torch.device, outputs) -> None:
    """The same for tensors allocated on that stream, which the caller goes on to use on the current one."""
    if stream is not None:
        here = torch.cuda.current_stream(device)
        if stream != here:
            for t in outputs:
                if t is not None:
                    t.record_stream(here)


def _current(device: torch.device) -> int:
    """The current stream of the device, as the library takes it (without the object that torch.cuda makes of it)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _matrix(t: torch.Tensor, name: str, rows: Optional[int], cols: Optional[int], dtype: torch.dtype, device: torch.device):
    """Refuse a tensor that is not a [rows, cols] matrix with contiguous rows; returns its size and row stride."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        want = ", ".join("any" if n is None else str(n) for n in (rows, cols))
        raise ValueError(f"{name} must be [{want}], got {tuple(shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}, got {t.device}")
    n, c = shape
    s0, s1 = t.stride()
    if c > 1 and s1 != 1:
        raise ValueError(f"{name} must have contiguous rows, got strides {(s0, s1)}")
    if n <= 1:
        return n, c, c if c > 1 else 1
    if s0 < c:
        raise ValueError(f"{name} has rows that overlap: stride {s0} for {c} columns")
    return n, c, s0


def _like(t: torch.Tensor, ld: int) -> torch.Tensor:
    """An uninitialised contiguous tensor of the size and type of the matrix t, whose row stride is ld."""
    return torch.empty_like(t) if ld == t.shape[1] else t.new_empty(t.shape)


def _device_of(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor; there is no CPU path")
    return t.device


def _no_graph(name: str, *tensors: Optional[torch.Tensor]) -> None:
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} records no autograd graph: call it under torch.no_grad(), or with detached tensors")
    if getattr(_forward_ad, "_current_level", 0) >= 0:  # (inside forward_ad.dual_level(); no_grad() does not stop it)
        for t in tensors:
            if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError(f"{name} records no autograd graph: call it without tangents, on the primal of a dual tensor")


def _vector(t: Optional[torch.Tensor], name: str, size: int, dtype: torch.dtype, device: torch.device) -> int:
    """Refuse a tensor that is not a contiguous vector of that size and type; returns its address (0 for None)."""
    if t is None:
        return 0
    if t.shape != (size,) or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} [{size}] on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


try:  # (0.9 us on the host instead of 1.5 to 2.5: as long as the checks of a whole call)
    from torch._C._dynamo.guards import _empty_strided_cuda as _strided
except ImportError:
    def _strided(size, stride, dtype):
        return torch.empty_strided(size, stride, dtype=dtype, device="cuda")


def _rows_of(n: int, c: int, dtype: torch.dtype) -> torch.Tensor:
    """An uninitialised contiguous matrix on the current device."""
    return _strided((n, c), (c, 1), dtype)


def _one_per_row(n: int, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    return _strided((n,), (1,), dtype)


def _floating(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _TYPES:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return _TYPES[t.dtype]


# ---------------------------------------------------------------- gated feed-forward block

# bmgd_gated_ffn of include/bmgd.h: rows; inputs, hidden, outputs, type, activation, reserved; x, w_gate, w_up, w_down and their
# strides; y and its stride; saved_value, saved_slope, saved_hidden, ld_saved; dy and its stride; dx, dw_gate, dw_up, dw_down
_GATED_FFN = struct.Struct("=q6i4Q4qQq3QqQq4Q")
_FORWARD, _BACKWARD = 0, 1


def _ffn_args(x, w_gate, w_up, w_down, activation):
    """The members that both passes share, and (rows, inputs, hidden, outputs)."""
    device = _device_of(x, "x")
    dtype = x.dtype
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise ValueError(f"x must be bfloat16 or float16, got {dtype}")
    if activation not in (ACT_SILU, ACT_GELU, ACT_RELU, ACT_SIGMOID):
        raise ValueError(f"unknown activation code {activation}")
    n, d, ld_x = _matrix(x, "x", None, None, dtype, device)
    _, f, ld_gate = _matrix(w_gate, "w_gate", d, None, dtype, device)
    _, _, ld_up = _matrix(w_up, "w_up", d, f, dtype, device)
    _, c, ld_down = _matrix(w_down, "w_down", f, None, dtype, device)
    if d < 1 or f < 1 or c < 1:
        raise ValueError("the block needs at least one input, one hidden unit and one output")
    return (n, d, f, c, _TYPES[dtype], activation, 0, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
            ld_x, ld_gate, ld_up, ld_down), (n, d, f, c), device


def _saved_args(saved: torch.Tensor, n: int, width: int):
    """Where the three parts of `saved` stand: act(X Wg) and (X Wu) * act'(X Wg) in fp32, their rows' product in 16 bits."""
    p = saved.data_ptr()
    return p, p + n * width * 4, p + n * width * 8, width


def _run_ffn(which: int, args: bytes, device: torch.device) -> None:
    L = _binding.load_library()
    need = ctypes.c_int64()
    rc = L.bmgd_gated_ffn_workspace_bytes(args, which, ctypes.byref(need))
    if rc == BMGD_OK:
        w = torch.empty(need.value, dtype=torch.uint8, device=device) if need.value else None
        call = L.bmgd_gated_ffn_forward if which == _FORWARD else L.bmgd_gated_ffn_backward
        rc = call(args, w.data_ptr() if w is not None else None, need.value, _current(device))
    if rc != BMGD_OK:
        raise BmgdError(rc, "bmgd_gated_ffn_forward" if which == _FORWARD else "bmgd_gated_ffn_backward")


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, activation: int = ACT_SILU,
              save: bool = False, stream: Optional[torch.cuda.Stream] = None):
    """(act(x w_gate) * (x w_up)) w_down for x [rows, inputs], w_gate and w_up [inputs, hidden], w_down [hidden, outputs].

    All four in bfloat16 or all in float16; rows contiguous, any row stride.  Sums are fp32, the product in brackets is rounded to
    that type in between (float16: it must stay below 65,504).  With save=True returns (y, saved), saved
    being what gated_ffn_backward needs beside its other arguments."""
    shared, (n, d, f, c), device = _ffn_args(x, w_gate, w_up, w_down, activation)
    _no_graph("gated_ffn", x, w_gate, w_up, w_down)
    place = _place(device, stream)
    _lend(stream, device, (x, w_gate, w_up, w_down))
    with place:
        y = x.new_empty((n, c))
        saved, kept = None, (0, 0, 0, 0)
        if save:
            width = (f + 7) // 8 * 8
            saved = x.new_empty((n, 5 * width))
            kept = _saved_args(saved, n, width)
        if n > 0:
            _run_ffn(_FORWARD, _GATED_FFN.pack(*shared, y.data_ptr(), c, *kept, 0, 0, 0, 0, 0, 0), device)
    _hand(stream, device, (y, saved))
    return (y, saved) if save else y


def gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                       saved: torch.Tensor, activation: int = ACT_SILU,
                       need_dx: bool = True, stream: Optional[torch.cuda.Stream] = None):
    """Gradients (dx, dw_gate, dw_up, dw_down) of gated_ffn for the gradient dy of its output; dx is None with need_dx=False
    (the first layer of a model has no use for it).

    `saved` is what the forward call on the same arguments returned; the gradients have the type of x."""
    shared, (n, d, f, c), device = _ffn_args(x, w_gate, w_up, w_down, activation)
    _, _, ld_dy = _matrix(dy, "dy", n, c, x.dtype, device)
    width = (f + 7) // 8 * 8
    if saved.shape != (n, 5 * width) or saved.dtype is not x.dtype or saved.device != device or not saved.is_contiguous():
        raise ValueError("saved must be what gated_ffn returned for the same rows and weights")
    place = _place(device, stream)
    _lend(stream, device, (dy, x, w_gate, w_up, w_down, saved))
    with place:
        ld_x, ld_gate, ld_up, ld_down = shared[11:]
        dx = _like(x, ld_x) if need_dx else None
        dw_gate, dw_up, dw_down = _like(w_gate, ld_gate), _like(w_up, ld_up), _like(w_down, ld_down)
        _run_ffn(_BACKWARD, _GATED_FFN.pack(*shared, 0, 0, *_saved_args(saved, n, width), dy.data_ptr(), ld_dy,
                                            dx.data_ptr() if need_dx else 0, dw_gate.data_ptr(),
                                            dw_up.data_ptr(), dw_down.data_ptr()), device)
    _hand(stream, device, (dx, dw_gate, dw_up, dw_down))
    return dx, dw_gate, dw_up, dw_down


def stream_check(stream: Optional[torch.cuda.Stream] = None) -> None:
    """Wait for the stream and raise, once, if a device-side wait of a gated-block or 8-bit product kernel on its device gave up.  What that kernel had
    not computed by then is NaN in its outputs."""
    s = stream if stream is not None else torch.cuda.current_stream()
    with torch.cuda.device(s.device):
        _status(_binding.load_library().bmgd_stream_check(s.cuda_stream), "bmgd_stream_check")


# ---------------------------------------------------------------- softmax loss, mini-batch

def softmax_residual(logits: torch.Tensor, y: torch.Tensor, scale: Optional[float] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(residual, loss) for logits [rows, C] and int32 labels y [rows]: scale (softmax - onehot), and the loss per row in
    fp32.  scale defaults to 1 / rows, the mean gradient of the mini-batch.  Rows without a label in [0, C) give zeros.

    float16 has too few exponents for the default over many rows: values below 6e-5 lose bits, those below 3e-8 are zero, and what
    gated_ffn_backward makes of them is smaller still.  Give it S / rows with a power of two S near the number of rows, and
    adamw_step grad_scale=1 / S."""
    device = _device_of(logits, "logits")
    if logits.dtype not in _TYPES:
        raise ValueError(f"logits must be float32, bfloat16 or float16, got {logits.dtype}")
    rows, C, ld = _matrix(logits, "logits", None, None, logits.dtype, device)
    if C < 1:
        raise ValueError("logits need at least one class")
    if y.dim() != 1 or y.shape[0] != rows or y.dtype != torch.int32 or y.device != device or not y.is_contiguous():
        raise ValueError(f"y must be a contiguous int32 [{rows}] on {device}")
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (logits, y))
    with place:
        residual = _like(logits, ld)
        loss = torch.empty(rows, dtype=torch.float32, device=device)
        if rows > 0:
            _status(L.bmgd_softmax_residual(logits.data_ptr(), ld, y.data_ptr(), rows, C, _TYPES[logits.dtype],
                                            1.0 / rows if scale is None else float(scale), residual.data_ptr(), C,
                                            loss.data_ptr(), _current(device)), "bmgd_softmax_residual")
    _hand(stream, device, (residual, loss))
    return residual, loss


def gather_batch(x: torch.Tensor, y: Optional[torch.Tensor], seed: int, chain: int, round: int, first: int, count: int,
                 stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rows first .. first + count - 1 of one round's order of the buffer x [rows, p], with their int32 labels: the
    mini-batch that run_rounds would take there (round `round` of chain `chain` under `seed`)."""
    device = _device_of(x, "x")
    if x.dim() != 2 or not x.is_contiguous() or x.shape[0] < 1 or x.shape[1] < 1:
        raise ValueError(f"x must be a contiguous [rows, p] with at least one row, got {tuple(x.shape)}")
    rows = x.shape[0]
    if y is not None and (y.dim() != 1 or y.shape[0] != rows or y.dtype != torch.int32 or y.device != device or not y.is_contiguous()):
        raise ValueError(f"y must be a contiguous int32 [{rows}] on {device}")
    if first < 0 or count < 0 or first + count > rows:
        raise ValueError(f"rows {first} to {first + count} of a buffer of {rows}")
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (x, y))
    with place:
        bx = torch.empty(count, x.shape[1], dtype=x.dtype, device=device)
        by = torch.empty(count, dtype=torch.int32, device=device) if y is not None else None
        _status(L.bmgd_gather_batch(x.data_ptr(), x.shape[1] * x.element_size(), y.data_ptr() if y is not None else None, rows,
                                    int(seed) & 0xFFFFFFFFFFFFFFFF, int(chain) & 0xFFFFFFFF, int(round) & 0xFFFFFFFF, first, count,
                                    bx.data_ptr(), by.data_ptr() if by is not None else None,
                                    _current(device)), "bmgd_gather_batch")
    _hand(stream, device, (bx, by))
    return bx, by


# ---------------------------------------------------------------- norm with the residual's addition, rows in 8 bits

# bmgd_rms_norm of include/bmgd.h: rows; width, type, weight_type, reserved; eps; x, residual, weight, total, y, codes, scale, rstd; strides of
# x, residual, total, y, codes; dy, dtotal, dx, dweight; strides of dy, dtotal, dx
_RMS_NORM = struct.Struct("=q4id8Q5q4Q3q")


def _norm_args(x: torch.Tensor, weight: Optional[torch.Tensor], eps: float, name: str):
    """What all the norm's calls check, and (device, rows, width, stride of x, the struct's first members, address of weight)."""
    device = _device_of(x, name)
    code = _floating(x, name)
    n, d, ld = _matrix(x, name, None, None, x.dtype, device)
    if d < 1:
        raise ValueError(f"{name} needs at least one column")
    if not 0.0 <= eps < float("inf"):
        raise ValueError(f"eps must be non-negative and finite, got {eps}")
    kind = code
    if weight is not None:
        if weight.dtype is not x.dtype and weight.dtype is not torch.float32:
            raise ValueError(f"weight must be {x.dtype} or float32, got {weight.dtype}")
        kind = _TYPES[weight.dtype]
    at = _vector(weight, "weight", d, weight.dtype if weight is not None else x.dtype, device)
    return device, n, d, ld, (n, d, code, kind, 0, float(eps)), at


def _codes_of(n: int, width: int) -> torch.Tensor:
    """Uninitialised codes [n, width] on the current device whose rows start on 16-byte boundaries."""
    return _strided((n, width), ((width + 15) // 16 * 16, 1), torch.int8)


def _run_norm(name, x, weight, residual, eps, save, quantized, stream):
    device, n, d, ld_x, head, at_weight = _norm_args(x, weight, eps, "x")
    ld_r = 0
    if residual is not None:
        _, _, ld_r = _matrix(residual, "residual", n, d, x.dtype, device)
    _no_graph(name, x, weight, residual)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (x, weight, residual))
    with place:
        total, at_total, at_residual = x, 0, 0
        if residual is not None:
            total = _rows_of(n, d, x.dtype)
            at_total, at_residual = total.data_ptr(), residual.data_ptr()
        y = codes = scale = rstd = None
        at_y = at_codes = at_scale = at_rstd = 0
        if quantized:
            codes, scale = _codes_of(n, d), _one_per_row(n)
            at_codes, at_scale = codes.data_ptr(), scale.data_ptr()
        else:
            y = _rows_of(n, d, x.dtype)
            at_y = y.data_ptr()
        if save:
            rstd = _one_per_row(n)
            at_rstd = rstd.data_ptr()
        if n > 0:
            _status(L.bmgd_rms_norm_forward(_RMS_NORM.pack(*head, x.data_ptr(), at_residual, at_weight, at_total, at_y, at_codes, at_scale, at_rstd, ld_x,
                                                           ld_r, d, d, (d + 15) // 16 * 16, 0, 0, 0, 0, 0, 0, 0), _current(device)), "bmgd_rms_norm_forward")
    if stream is not None:
        _hand(stream, device, (total if residual is not None else None, y, codes, scale, rstd))
    return y, codes, scale, total, rstd


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
             save: bool = False, stream: Optional[torch.cuda.Stream] = None):
    """(y, total) for x [rows, width] and, of the same size and type, residual: total = x + residual in that type (x itself without a
    residual), y = total / sqrt(mean(total^2) + eps) * weight.  With save=True (y, total, rstd), what rms_norm_backward needs.

    float32, bfloat16 or float16, rows contiguous, any row stride; weight [width] of that type or float32.  Sums are fp32."""
    y, _, _, total, rstd = _run_norm("rms_norm", x, weight, residual, eps, save, False, stream)
    return (y, total, rstd) if save else (y, total)


def rms_norm_int8(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(codes, scale, total): as rms_norm, with y in 8 bits as int8_linear reads it (y is about codes * scale[:, None])."""
    _, codes, scale, total, _ = _run_norm("rms_norm_int8", x, weight, residual, eps, False, True, stream)
    return codes, scale, total


def rms_norm_backward(dy: torch.Tensor, total: torch.Tensor, weight: Optional[torch.Tensor], rstd: torch.Tensor,
                      dtotal: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(dx, dweight) of rms_norm for the gradient dy of y and, where total is used further on, dtotal of total.  dx is the gradient
    of x and of the residual; dweight has the weight's type (None without a weight)."""
    device, n, d, ld_t, head, at_weight = _norm_args(total, weight, 0.0, "total")
    _, _, ld_dy = _matrix(dy, "dy", n, d, total.dtype, device)
    ld_dt = 0
    if dtotal is not None:
        _, _, ld_dt = _matrix(dtotal, "dtotal", n, d, total.dtype, device)
    at_rstd = _vector(rstd, "rstd", n, torch.float32, device)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (dy, total, weight, rstd, dtotal))
    with place:
        dx = _rows_of(n, d, total.dtype)
        dweight = _one_per_row(d, weight.dtype) if weight is not None else None
        args = _RMS_NORM.pack(*head, 0, 0, at_weight, total.data_ptr(), 0, 0, 0, at_rstd, 0, 0, ld_t, 0, 0, dy.data_ptr(),
                              dtotal.data_ptr() if dtotal is not None else 0, dx.data_ptr(), dweight.data_ptr() if weight is not None else 0, ld_dy, ld_dt, d)
        w, size = None, 0
        if weight is not None and n > 0:
            need = ctypes.c_int64()
            _status(L.bmgd_rms_norm_workspace_bytes(args, ctypes.byref(need)), "bmgd_rms_norm_workspace_bytes")
            size = need.value
            w = _one_per_row(size, torch.uint8)
        _status(L.bmgd_rms_norm_backward(args, w.data_ptr() if w is not None else None, size, _current(device)), "bmgd_rms_norm_backward")
    _hand(stream, device, (dx, dweight))
    return dx, dweight


# bmgd_quantize_rows_args: rows; width, type, activation, reserved; x, gate, codes, scale; ld_x, ld_gate, ld_codes
_QUANTIZE_ROWS = struct.Struct("=q4i4Q3q")


def quantize_rows(x: torch.Tensor, gate: Optional[torch.Tensor] = None, activation: int = ACT_SILU,
                  stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes, scale) of the rows of x [rows, width], or with a gate of the same size and type those of act(gate) * x: int8 with
    the row's largest magnitude at 127, and that magnitude / 127 in float32."""
    device = _device_of(x, "x")
    code = _floating(x, "x")
    n, d, ld_x = _matrix(x, "x", None, None, x.dtype, device)
    if d < 1:
        raise ValueError("x needs at least one column")
    ld_g = 0
    if gate is not None:
        _, _, ld_g = _matrix(gate, "gate", n, d, x.dtype, device)
    if activation not in (ACT_SILU, ACT_GELU, ACT_RELU, ACT_SIGMOID):
        raise ValueError(f"unknown activation code {activation}")
    _no_graph("quantize_rows", x, gate)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (x, gate))
    with place:
        codes, scale = _codes_of(n, d), _one_per_row(n)
        if n > 0:
            _status(L.bmgd_quantize_rows(_QUANTIZE_ROWS.pack(n, d, code, activation, 0, x.data_ptr(), gate.data_ptr() if gate is not None else 0,
                                                             codes.data_ptr(), scale.data_ptr(), ld_x, ld_g, (d + 15) // 16 * 16), _current(device)),
                    "bmgd_quantize_rows")
    _hand(stream, device, (codes, scale))
    return codes, scale


# ---------------------------------------------------------------- product in 8-bit integers

def quantize_weight(w: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes, scale) of a weight [inputs, outputs] as int8_linear reads it: int8 [outputs, inputs] with each output's largest
    magnitude at 127, and that magnitude / 127 in float32 [outputs].  Done once for a weight."""
    device = _device_of(w, "w")
    code = _floating(w, "w")
    d, c, ld = _matrix(w, "w", None, None, w.dtype, device)
    if d < 1 or c < 1:
        raise ValueError("w needs at least one input and one output")
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (w,))
    with place:
        codes, scale = _codes_of(c, d), _one_per_row(c)
        _status(L.bmgd_quantize_weight(w.data_ptr(), ld, d, c, code, codes.data_ptr(), (d + 15) // 16 * 16, scale.data_ptr(), _current(device)),
                "bmgd_quantize_weight")
    _hand(stream, device, (codes, scale))
    return codes, scale


# bmgd_quantized_linear_args: rows; inputs, outputs, type, reserved; codes, scale, weight, weight_scale, bias, y; ld_codes, ld_weight, ld_y
_QUANTIZED_LINEAR = struct.Struct("=q4i6Q3q")
_MOST_INPUTS = 131071


def int8_linear(q: torch.Tensor, q_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                dtype: torch.dtype = torch.bfloat16, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """(q w^T) * q_scale[:, None] * w_scale + bias for q [rows, inputs] and w [outputs, inputs] in int8, scales and bias in float32; the sums
    are exact, the result is rounded once to dtype (float32, bfloat16 or float16).  Up to 131,071 inputs."""
    device = _device_of(q, "q")
    n, d, ld_q = _matrix(q, "q", None, None, torch.int8, device)
    c, _, ld_w = _matrix(w, "w", None, d, torch.int8, device)
    if c < 1 or not 1 <= d <= _MOST_INPUTS:
        raise ValueError(f"the product needs 1 to {_MOST_INPUTS} inputs and at least one output, got {d} and {c}")
    if dtype not in _TYPES:
        raise ValueError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    at_q, at_w, at_b = (_vector(t, name, k, torch.float32, device) for t, name, k in ((q_scale, "q_scale", n), (w_scale, "w_scale", c), (bias, "bias", c)))
    if q_scale is None or w_scale is None:
        raise ValueError("q_scale and w_scale are needed")
    _no_graph("int8_linear", q_scale, w_scale, bias)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (q, q_scale, w, w_scale, bias))
    with place:
        y = _rows_of(n, c, dtype)
        if n > 0:
            base_q, base_w, work, size = q.data_ptr(), w.data_ptr(), None, 0
            args = _QUANTIZED_LINEAR.pack(n, d, c, _TYPES[dtype], 0, base_q, at_q, base_w, at_w, at_b, y.data_ptr(), ld_q, ld_w, c)
            if (base_q | base_w | ld_q | ld_w) % 16:  # (rows on 16-byte boundaries need no workspace, few tokens neither)
                need = ctypes.c_int64()
                _status(L.bmgd_quantized_linear_workspace_bytes(args, ctypes.byref(need)), "bmgd_quantized_linear_workspace_bytes")
                size = need.value
                work = _one_per_row(size, torch.uint8) if size else None
            _status(L.bmgd_quantized_linear(args, work.data_ptr() if work is not None else None, size, _current(device)), "bmgd_quantized_linear")
    _hand(stream, device, (y,))
    return y


# ---------------------------------------------------------------- log probabilities

# bmgd_log_probs_args: rows; C, type, top, reserved; logits, y, logprob, entropy, saved, top_class, top_logprob; ld_logits; dlogprob, dentropy,
# dlogits; ld_dlogits
_LOG_PROBS = struct.Struct("=q4i7Qq3Qq")
MOST_ALTERNATIVES = 32


def _score_args(logits: torch.Tensor, y: Optional[torch.Tensor]):
    device = _device_of(logits, "logits")
    code = _floating(logits, "logits")
    rows, C, ld = _matrix(logits, "logits", None, None, logits.dtype, device)
    if C < 1:
        raise ValueError("logits need at least one class")
    return device, code, rows, C, ld, _vector(y, "y", rows, torch.int32, device)


def log_probs(logits: torch.Tensor, y: Optional[torch.Tensor] = None, top: int = 0, save: bool = False,
              stream: Optional[torch.cuda.Stream] = None):
    """(logprob, entropy, classes, logprobs) of logits [rows, C]: the log probability of the int32 label y of each row (0 for a row whose
    label is outside [0, C), or without y), the entropy of its distribution, and its `top` (0 to 32) most probable classes with their log
    probabilities [rows, top], in falling order, equal ones by rising class.  All in float32 and int32.  With save=True a fifth,
    what log_probs_backward needs.

    Rows whose logits are all -Inf have log probability and entropy 0 and alternatives of -Inf; NaN and +Inf in a row give NaN."""
    device, code, rows, C, ld, at_y = _score_args(logits, y)
    if not 0 <= top <= min(C, MOST_ALTERNATIVES):
        raise ValueError(f"top must be 0 to {min(C, MOST_ALTERNATIVES)}, got {top}")
    _no_graph("log_probs", logits)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (logits, y))
    with place:
        logprob, entropy = _one_per_row(rows), _one_per_row(rows)
        classes, values = _strided((rows, top), (max(top, 1), 1), torch.int32), _strided((rows, top), (max(top, 1), 1), torch.float32)
        saved = _rows_of(rows, 3, torch.float32) if save else None
        if rows > 0:
            _status(L.bmgd_log_probs(_LOG_PROBS.pack(rows, C, code, top, 0, logits.data_ptr(), at_y, logprob.data_ptr(), entropy.data_ptr(),
                                                     saved.data_ptr() if save else 0, classes.data_ptr() if top else 0, values.data_ptr() if top else 0,
                                                     ld, 0, 0, 0, 0), _current(device)), "bmgd_log_probs")
    _hand(stream, device, (logprob, entropy, classes, values, saved))
    return (logprob, entropy, classes, values, saved) if save else (logprob, entropy, classes, values)


def log_probs_backward(dlogprob: Optional[torch.Tensor], dentropy: Optional[torch.Tensor], logits: torch.Tensor, y: Optional[torch.Tensor],
                       saved: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of the logits, in their type, for the gradients of log_probs' first two results (float32 [rows], None for zero).

    float16 holds no gradients of a mean over many rows: scale the two up (as softmax_residual says)."""
    device, code, rows, C, ld, at_y = _score_args(logits, y)
    at_l, at_e = _vector(dlogprob, "dlogprob", rows, torch.float32, device), _vector(dentropy, "dentropy", rows, torch.float32, device)
    if saved.shape != (rows, 3) or saved.dtype is not torch.float32 or saved.device != device or not saved.is_contiguous():
        raise ValueError("saved must be what log_probs returned for the same logits")
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (dlogprob, dentropy, logits, y, saved))
    with place:
        dlogits = _rows_of(rows, C, logits.dtype)
        if rows > 0:
            _status(L.bmgd_log_probs_backward(_LOG_PROBS.pack(rows, C, code, 0, 0, logits.data_ptr(), at_y, 0, 0, saved.data_ptr(), 0, 0, ld,
                                                              at_l, at_e, dlogits.data_ptr(), C), _current(device)), "bmgd_log_probs_backward")
    _hand(stream, device, (dlogits,))
    return dlogits


# ---------------------------------------------------------------- dropout

# bmgd_dropout_args: rows, width; type, layer; rate; seed; step; x, residual, y; ld_x, ld_residual, ld_y
_DROPOUT = struct.Struct("=2q2id5Q3q")


def dropout(x: torch.Tensor, rate: float, seed: int, layer: int = 0, step: Optional[torch.Tensor] = None,
            residual: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """x [rows, width] with a share `rate` of its values dropped and the others divided by what is kept, plus the residual.

    Which values stay follows from (seed, layer, step) and a value's place alone (bmgd_dropout in include/bmgd.h): the gradient is the same call
    on the output's gradient, without the residual.  step: an int64 [1] on the device, read when the call runs, for instance
    state["control"][:1] of adamw_state, so that a captured call draws anew with each update; None counts as 0."""
    device = _device_of(x, "x")
    code = _floating(x, "x")
    n, d, ld_x = _matrix(x, "x", None, None, x.dtype, device)
    if d < 1:
        raise ValueError("x needs at least one column")
    ld_r = 0
    if residual is not None:
        _, _, ld_r = _matrix(residual, "residual", n, d, x.dtype, device)
    if not 0.0 <= rate < 1.0 - 2.0 ** -17:
        raise ValueError(f"rate must be 0 to below 1 - 2^-17, got {rate}")
    if not 0 <= layer <= 0xFFFF:
        raise ValueError(f"layer must be 0 to 65535, got {layer}")
    at_step = _vector(step, "step", 1, torch.int64, device)
    _no_graph("dropout", x, residual)
    L = _binding.load_library()
    place = _place(device, stream)
    _lend(stream, device, (x, residual, step))
    with place:
        y = _rows_of(n, d, x.dtype)
        if n > 0:
            _status(L.bmgd_dropout(_DROPOUT.pack(n, d, code, layer, rate, int(seed) & 0xFFFFFFFFFFFFFFFF, at_step, x.data_ptr(),
                                                 residual.data_ptr() if residual is not None else 0, y.data_ptr(), ld_x, ld_r, d), _current(device)), "bmgd_dropout")
    _hand(stream, device, (y,))
    return y


# ---------------------------------------------------------------- AdamW

class _AdamwConfig(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("lr", "a", "b", "eps", "grad_scale", "max_norm")] + [("seed", ctypes.c_uint64)]


def adamw_state(params: Sequence[torch.Tensor], state_bits: int = 32) -> dict:
    """Zero moments and counters for adamw_step: keyword arguments m, v, control and, with 8 bits, m_scale and v_scale."""
    if state_bits not in (8, 32):
        raise ValueError("state_bits must be 8 or 32")
    if not params:
        raise ValueError("no parameters")
    out = {"control": torch.zeros(CONTROL_WORDS, dtype=torch.int64, device=params[0].device)}
    if state_bits == 32:
        out["m"] = [torch.zeros(p.shape, dtype=torch.float32, device=p.device) for p in params]
        out["v"] = [torch.zeros(p.shape, dtype=torch.float32, device=p.device) for p in params]
    else:
        out["m"] = [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for p in params]
        out["v"] = [torch.zeros(p.shape, dtype=torch.uint8, device=p.device) for p in params]
        for k in ("m_scale", "v_scale"):
            out[k] = [torch.zeros(-(-p.numel() // SCALE_BLOCK), dtype=torch.uint8, device=p.device) for p in params]
    return out


_dtype = operator.attrgetter("dtype")
_numel, _get_device, _is_contiguous, _data_ptr = (getattr(torch.Tensor, k) for k in ("numel", "get_device", "is_contiguous", "data_ptr"))


def _column(tensors: Sequence[torch.Tensor], name: str, counts: List[int], types: frozenset, device: int) -> List[int]:
    """Refuse a list of tensors that does not match the parameters; returns their addresses."""
    if len(tensors) != len(counts):
        raise ValueError(f"{name}: {len(tensors)} tensors for {len(counts)} parameters")
    if list(map(_numel, tensors)) != counts:
        raise ValueError(f"{name}: a tensor's size does not match its parameter's")
    found = set(map(_dtype, tensors))
    if not found <= types:
        raise ValueError(f"{name} must be {' or '.join(sorted(map(str, types)))}, got {(found - types).pop()}")
    if set(map(_get_device, tensors)) - {device}:
        raise ValueError(f"{name}: all tensors must live on one device")
    if not all(map(_is_contiguous, tensors)):
        raise ValueError(f"{name}: tensors must be contiguous")
    return list(map(_data_ptr, tensors))


_ANY, _FLOAT = frozenset(_TYPES), frozenset((torch.float32,))
_M, _V, _BYTES = frozenset((torch.float32, torch.float8_e4m3fn)), frozenset((torch.float32, torch.uint8)), frozenset((torch.uint8,))


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: Sequence[torch.Tensor], v: Sequence[torch.Tensor],
               control: torch.Tensor, lr: float, a: float = 0.9, b: float = 0.999, eps: float = 1e-8,
               weight_decay: Union[float, Sequence[float]] = 0.0, max_norm: float = 0.0, grad_scale: float = 1.0,
               m_scale: Optional[Sequence[torch.Tensor]] = None, v_scale: Optional[Sequence[torch.Tensor]] = None,
               masters: Optional[Sequence[Optional[torch.Tensor]]] = None, seed: int = 0,
               stream: Optional[torch.cuda.Stream] = None) -> None:
    """One AdamW update of all tensors, in place (formula, types and control words: bmgd_adamw_step in include/bmgd.h).

    params: float32, bfloat16 or float16, contiguous, on one device; grads: any of the three types.  m and v: both
    float32, or float8_e4m3fn and uint8 with the per-256-values scales m_scale and v_scale (adamw_state makes them); a
    list may mix the two.  masters: float32 copies (None for a parameter without one).  control: int64 [4]."""
    count = len(params)
    if count == 0:
        raise ValueError("no parameters")
    device = _device_of(params[0], "params")
    index = device.index
    counts = list(map(_numel, params))
    p_types, g_types, m_types, v_types = (set(map(_dtype, t)) for t in (params, grads, m, v))
    every = [*params, *grads, *m, *v]
    if not (len(grads) == len(m) == len(v) == count and p_types <= _ANY and g_types <= _ANY and m_types <= _M and v_types <= _V and
            list(map(_numel, every)) == counts * 4 and set(map(_get_device, every)) == {index} and all(map(_is_contiguous, every))):
        for t, name, types in ((params, "params", _ANY), (grads, "grads", _ANY), (m, "m", _M), (v, "v", _V)):
            _column(t, name, counts, types, index)  # (says which)
        raise ValueError("params, grads, m and v do not match")
    addresses = array("q", map(_data_ptr, every))
    table = array("q", bytes(88 * count))  # bmgd_adamw_tensor[count], filled column by column
    for k in range(4):
        table[k::11] = addresses[k * count:(k + 1) * count]
    if m_types == _FLOAT and v_types == _FLOAT:
        table[10::11] = array("q", range(32, 32 + (count << 32), 1 << 32))  # state_bits and index
    else:
        eight = [t.dtype is not torch.float32 for t in m]
        if eight != [t.dtype is not torch.float32 for t in v]:
            raise ValueError("m and v of a parameter must be held in the same number of bits")
        if m_scale is None or v_scale is None:
            raise ValueError("moments in 8 bits need m_scale and v_scale")
        blocks = [-(-n // SCALE_BLOCK) for n in counts]
        table[4::11] = array("q", _column(m_scale, "m_scale", blocks, _BYTES, index))
        table[5::11] = array("q", _column(v_scale, "v_scale", blocks, _BYTES, index))
        table[10::11] = array("q", [(8 if e else 32) | i << 32 for i, e in enumerate(eight)])
    if masters is not None:
        if len(masters) != count:
            raise ValueError(f"masters: {len(masters)} tensors for {count} parameters")
        held = [i for i, t in enumerate(masters) if t is not None]
        for i, at in zip(held, _column([masters[i] for i in held], "masters", [counts[i] for i in held], _FLOAT, index)):
            if params[i].dtype is torch.float32:
                raise ValueError("a float32 parameter has no master copy")
            table[11 * i + 6] = at
    if torch.float16 in p_types and (masters is None or any(t is None and p.dtype is torch.float16 for p, t in zip(params, masters))):
        raise ValueError("a float16 parameter needs a master copy")
    if control.dtype != torch.int64 or control.numel() != CONTROL_WORDS or control.device != device or not control.is_contiguous():
        raise ValueError(f"control must be a contiguous int64 [{CONTROL_WORDS}] on {device}")
    table[7::11] = array("q", counts)
    if isinstance(weight_decay, (int, float)):
        decays = array("d", [weight_decay]) * count
    else:
        decays = array("d", weight_decay)
        if len(decays) != count:
            raise ValueError(f"weight_decay: {len(decays)} values for {count} parameters")
    table[8::11] = array("q", decays.tobytes())
    if len(p_types) == 1 and len(g_types) == 1:
        table[9::11] = array("q", [_TYPES[params[0].dtype] | _TYPES[grads[0].dtype] << 32]) * count
    else:
        table[9::11] = array("q", [_TYPES[p.dtype] | _TYPES[g.dtype] << 32 for p, g in zip(params, grads)])
    cfg = _AdamwConfig(float(lr), float(a), float(b), float(eps), float(grad_scale), float(max_norm), int(seed) & 0xFFFFFFFFFFFFFFFF)
    L = _binding.load_library()
    place = _place(device, stream)
    if stream is not None:
        _lend(stream, device, [*every, control, *(m_scale or ()), *(v_scale or ()), *(masters or ())])
    with place:
        scratch, size = None, 0
        if max_norm > 0:
            size = (1 + count // 360) * 1184 * 8
            scratch = torch.empty(size, dtype=torch.uint8, device=device)
        _status(L.bmgd_adamw_step(table.buffer_info()[0], count, ctypes.byref(cfg), control.data_ptr(),
                                  scratch.data_ptr() if scratch is not None else None, size,
                                  _current(device)), "bmgd_adamw_step")
    torch._C._increment_version(params if masters is None else [*params, *(t for t in masters if t is not None)])


def decode_moments(m: torch.Tensor, m_scale: torch.Tensor, v: torch.Tensor, v_scale: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
    """The fp32 values that moments in 8 bits stand for (for reading them; adamw_step does this on its own)."""
    def per_value(scale, n):
        return scale.to(torch.int32).repeat_interleave(SCALE_BLOCK)[:n]
    n = m.numel()
    first = torch.ldexp(m.reshape(-1).float(), per_value(m_scale, n) - 134).reshape(m.shape)
    codes = v.reshape(-1).to(torch.int32)
    second = torch.ldexp(1.0 + (codes & 7).float() / 8.0, (codes >> 3) - 157 + per_value(v_scale, n))
    second = torch.where(codes == 0, 0.0, torch.where(codes == 255, float("nan"), second)).reshape(v.shape)
    return first, second
