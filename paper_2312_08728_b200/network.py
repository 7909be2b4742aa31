"""Buffered mini-batch training of a network with one gated hidden layer (Algorithm 1 beyond linear models).

The paper runs its buffering over networks too (Sections 4.3 and 4.4, with Adam in Section 4.2); the step kernels behind
`Bmgd` hold a model with one layer.  GatedSoftmax is the C-class softmax regression on a gated hidden layer,

    logits = (act(X Wg) * (X Wu)) Wd,        loss = mean over the mini-batch of  logsumexp(logits) - logit of the label,

trained the same way: buffers are copied into one of two slots behind the computation, and each buffer is visited in rounds
of freshly shuffled mini-batches, the shuffle being the one of `Bmgd` (round t under a seed draws the same partition).
Rows are bf16 or fp16; the weights are held in fp32 and in the rows' type, the update is AdamW with moments in 32 or 8
bits.  Every step is the operators of `operators.py` in a row: gather_batch, gated_ffn, softmax_residual,
gated_ffn_backward, adamw_step.

fp16 has no exponents for gradients of a mean over many rows: a probability of 1e-4 over 1,000 rows lies below its normal
values, and the gradients that follow from it lower still (1,000 rows that a net 512 -> 1024 -> 10 knows with e^9 to 1: the relative error of
dWg is 0.08, of 8,192 rows 0.43; with the loss scaled 0.0005).  So with fp16 rows the residual, and with it every gradient, is
multiplied by a power of two S, which the update divides out again in fp32; S / rows is between 1/2 and 1, S at most 2^13 and,
up to 128 rows, 1, unless the caller gives `loss_scale`.  An update whose gradients are not finite is left out
(state["control"] counts them).  Eight steps after one whose loss was a number, S falls to a quarter; it rises again by as much
after 2,000 updates without one.  (A loss that is NaN comes from the rows, or from hidden values above 65,504: no S mends that.)
"""
from __future__ import annotations

import math
import sys
from typing import Dict, List, Optional

import torch

from . import operators as ops
from .binding import ERR_CAPACITY, ERR_STATE, BmgdError, check_buffer
from .inputs import DTYPE_BF16, LOSS_SOFTMAX

_LAG = 8               # steps between an update and the look at whether it was left out: the host runs ahead that far
_RAISE = 2000          # updates in a row that were taken, before S rises again
_LEAST = 2.0 ** -20    # of the factor by which S has fallen


class GatedSoftmax:
    """The model, its optimizer state and two buffer slots of ceil(N / K) rows on one device.

    Mirrors Bmgd where the two mean the same: load_buffer, run_rounds, run_rounds_resident, get_theta, set_theta, sync."""

    def __init__(self, N: int, p: int, K: int, hidden: int, C: int, dtype: torch.dtype = torch.bfloat16,
                 activation: int = ops.ACT_SILU, device: int = 0, state_bits: int = 32, a: float = 0.9, b: float = 0.999,
                 eps: float = 1e-8, weight_decay: float = 0.0, max_norm: float = 0.0, seed: int = 0,
                 loss_scale: Optional[float] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("GatedSoftmax needs a CUDA device; there is no CPU path")
        if N < 1 or p < 1 or K < 1 or K > N or hidden < 1 or C < 2:
            raise ValueError("N, p, K, hidden and C must be positive, K at most N, C at least 2")
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"dtype must be bfloat16 or float16, got {dtype}")
        if loss_scale is not None and (dtype is not torch.float16 or not 0.0 < loss_scale < float("inf")):
            raise ValueError("loss_scale must be positive and finite, and is for float16 only")
        self.N, self.p, self.K, self.hidden, self.C, self.dtype, self.activation = N, p, K, hidden, C, dtype, activation
        self.device = torch.device("cuda", device)
        self.rows = -(-N // K)
        if dtype is torch.float16 and max_norm == 0.0:
            max_norm = sys.float_info.max   # clips nothing, and leaves an update out whose norm is not finite
        self._rule = dict(a=a, b=b, eps=eps, weight_decay=weight_decay, max_norm=max_norm, seed=seed)
        gen = torch.Generator(device=self.device).manual_seed(seed)
        shapes = ((p, hidden), (p, hidden), (hidden, C))
        self.masters: List[torch.Tensor] = [torch.randn(s, generator=gen, device=self.device) * s[0] ** -0.5 for s in shapes]
        self.weights: List[torch.Tensor] = [m.to(dtype) for m in self.masters]
        self.state: Dict = ops.adamw_state(self.weights, state_bits)
        self._slots: List[Optional[tuple]] = [None, None]    # (x, y) on the device
        self._count = [0, 0]
        self._loaded = [torch.cuda.Event() for _ in range(2)]
        self._freed = [torch.cuda.Event() for _ in range(2)]
        self._next = 0
        self.loss_scale = loss_scale
        if dtype is torch.float16:
            self._lowered, self._steps, self._lowered_at, self._left_out, self._taken = 1.0, 0, 0, 0, 0
            self._counts = torch.zeros(_LAG, ops.CONTROL_WORDS, dtype=torch.int64).pin_memory()
            self._losses = torch.zeros(_LAG).pin_memory()
            self._counted = [torch.cuda.Event() for _ in range(_LAG)]

    def load_buffer(self, host_x: torch.Tensor, host_y: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> int:
        """Start copying one buffer (pinned host tensors, labels int32) into the next slot on `stream`, behind the last
        computation that read that slot and the last copy into it; returns the slot."""
        if host_x.device.type != "cpu" or host_y.device.type != "cpu":
            raise ValueError("load_buffer takes host tensors")
        self._check(host_x, host_y)
        rows = host_x.shape[0]
        if rows > self.rows:
            raise BmgdError(ERR_CAPACITY, "load_buffer")
        if stream is not None and stream.device != self.device:
            raise ValueError(f"the stream belongs to {stream.device}, the model lives on {self.device}")
        s, current = self._next, torch.cuda.current_stream(self.device)
        copy = stream if stream is not None else current
        if self._slots[s] is None:
            with torch.cuda.device(self.device):
                self._slots[s] = (torch.empty(self.rows, self.p, dtype=self.dtype, device=self.device),
                                  torch.empty(self.rows, dtype=torch.int32, device=self.device))
            self._freed[s].record(current)  # (new memory may still be in use by work issued before)
        x, y = self._slots[s]
        copy.wait_event(self._freed[s])
        copy.wait_event(self._loaded[s])  # (a slot may be loaded again without having been trained on, on another stream)
        self._count[s] = 0  # (nothing to train on, should a copy fail)
        try:
            with torch.cuda.stream(copy):
                x[:rows].copy_(host_x, non_blocking=True)
                y[:rows].copy_(host_y, non_blocking=True)
        finally:  # (if the second copy fails the first is under way all the same)
            x.record_stream(copy)  # (the model may be dropped while a copy is under way)
            y.record_stream(copy)
            self._loaded[s].record(copy)
        self._count[s] = rows
        self._next ^= 1
        return s

    def run_rounds(self, slot: int, rounds: int, batch_size: int, lr: float, seed: int) -> torch.Tensor:
        """`rounds` rounds over the buffer in `slot` on the current stream; returns the loss of every row of the last mini-batch."""
        if slot not in (0, 1) or self._count[slot] == 0:
            raise BmgdError(ERR_STATE, "run_rounds")
        current = torch.cuda.current_stream(self.device)
        current.wait_event(self._loaded[slot])
        x, y = self._slots[slot]
        n = self._count[slot]
        try:
            return self._rounds(x[:n], y[:n], rounds, batch_size, lr, seed)
        finally:
            self._freed[slot].record(current)  # (a step that fails leaves the steps before it under way)

    def run_rounds_resident(self, dev_x: torch.Tensor, dev_y: torch.Tensor, rounds: int, batch_size: int, lr: float,
                            seed: int) -> torch.Tensor:
        """The same on a buffer the caller holds in device memory."""
        if dev_x.device != self.device or dev_y.device != self.device:
            raise ValueError("resident buffers must live on the model's device")
        self._check(dev_x, dev_y)
        return self._rounds(dev_x, dev_y, rounds, batch_size, lr, seed)

    def _check(self, x: torch.Tensor, y: torch.Tensor) -> None:
        if x.dtype != self.dtype:
            raise ValueError(f"X must be {self.dtype}, got {x.dtype}")
        check_buffer(x.view(torch.bfloat16), y, self.p, LOSS_SOFTMAX, DTYPE_BF16)  # (either 16-bit type: shapes and labels)

    def _rounds(self, x, y, rounds, batch_size, lr, seed):
        if rounds < 1 or batch_size < 1:
            raise ValueError("rounds and batch_size must be positive")
        n, loss = x.shape[0], None
        for t in range(rounds):
            for first in range(0, n, batch_size):
                loss = self.step(*ops.gather_batch(x, y, seed, 0, t, first, min(batch_size, n - first)), lr)
        return loss

    def _scale(self, rows: int) -> float:
        """S for a mini-batch of that many rows.  What is looked at is always the update _LAG steps back, whether the device is
        ahead or behind: equal runs give equal bits."""
        if self.dtype is not torch.float16:
            return 1.0
        if self._steps >= _LAG and not torch.cuda.is_current_stream_capturing():
            k = self._steps % _LAG
            self._counted[k].synchronize()
            left_out = int(self._counts[k, 1])
            self._taken = self._taken + 1 if left_out == self._left_out else 0
            if left_out > self._left_out and not math.isnan(float(self._losses[k])) and self._steps - _LAG >= self._lowered_at:
                self._lowered, self._lowered_at = max(self._lowered / 4, _LEAST), self._steps  # (it was taken with the present S)
            elif self._taken >= _RAISE and self._lowered < 1.0:
                self._lowered, self._taken = self._lowered * 4, 0
            self._left_out = left_out
        if self.loss_scale is not None:
            return self.loss_scale * self._lowered
        return (1.0 if rows <= 128 else 2.0 ** min(rows.bit_length() - 1, 13)) * self._lowered

    def step(self, x: torch.Tensor, y: torch.Tensor, lr: float) -> torch.Tensor:
        """One update from the rows of one mini-batch; returns the loss of each.  (A step captured into a graph keeps the S of its
        capture.)"""
        scale = self._scale(x.shape[0])
        logits, saved = ops.gated_ffn(x, *self.weights, self.activation, save=True)
        residual, loss = ops.softmax_residual(logits, y, None if scale == 1.0 else scale / max(x.shape[0], 1))
        _, *grads = ops.gated_ffn_backward(residual, x, *self.weights, saved, self.activation, need_dx=False)
        ops.adamw_step(self.weights, grads, lr=lr, masters=self.masters, grad_scale=1.0 / scale, **self.state, **self._rule)
        if self.dtype is torch.float16 and not torch.cuda.is_current_stream_capturing():
            k = self._steps % _LAG
            with torch.cuda.device(self.device):
                self._counts[k].copy_(self.state["control"], non_blocking=True)
                self._losses[k].copy_(loss.sum(), non_blocking=True)
                self._counted[k].record()
            self._steps += 1
        return loss

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        """The model's answer for device rows x."""
        return ops.gated_ffn(x, *self.weights, self.activation)

    def get_theta(self) -> List[torch.Tensor]:
        """Copies of the fp32 weights (Wg, Wu, Wd) on the host."""
        return [m.cpu() for m in self.masters]

    def set_theta(self, theta) -> None:
        """Overwrite the weights; the optimizer's state stays."""
        if len(theta) != 3 or any(t.shape != m.shape for t, m in zip(theta, self.masters)):
            raise ValueError("theta must be [p, hidden], [p, hidden] and [hidden, C]")
        for t, m, w in zip(theta, self.masters, self.weights):
            m.copy_(t)
            w.copy_(m)

    def sync(self) -> None:
        """Wait for everything issued on the current stream and report a device-side error if one was raised (the step concerned
        has NaN for gradients then, and so have the weights after it unless max_norm is given, which leaves such an update out)."""
        ops.stream_check(torch.cuda.current_stream(self.device))
