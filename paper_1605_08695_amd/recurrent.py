"""The recurrent layer of a language model between its embedding table and its softmax head (Section 6.4's model has
one): a gated linear recurrence, whose products are made for all tokens before its scan."""
from __future__ import annotations

from typing import NamedTuple, Optional

import numpy as np
import torch

from . import ops


class Saved(NamedTuple):
    """What GatedRecurrence.backward needs of a forward call."""
    x: torch.Tensor
    z: torch.Tensor
    lengths: Optional[torch.Tensor]
    states: torch.Tensor


class GatedRecurrence:
    """Variables W (d_in x gates d, fp32 master + bf16 shadow, the filter of a 1 x 1 convolution) and b (gates d, fp32):
    column blocks input, forget gate and, with output_gate, output gate.  h_t = s(a_t) h_(t-1) + (1 - s(a_t)) x_t and
    y_t = h_t or s(o_t) h_t, with x, a, o the blocks of input W + b and s the logistic function."""

    def __init__(self, W: np.ndarray, b: np.ndarray, output_gate: bool = True, device="cuda"):
        dev = torch.device(device)
        gates = 3 if output_gate else 2
        self.d_in, cols = W.shape
        if cols % gates or b.shape != (cols,):
            raise ValueError("W must have %d columns for each channel and b as many values" % gates)
        self.d, self.output_gate = cols // gates, output_gate
        # master weights start at their bf16 values (the values the products read)
        self.W = torch.from_numpy(np.asarray(W, np.float32)).to(torch.bfloat16).to(torch.float32).to(dev)
        self.W_lp = self.W.to(torch.bfloat16)
        self.b = torch.from_numpy(np.asarray(b, np.float32)).to(dev)

    def _product(self, x: torch.Tensor, stream) -> torch.Tensor:
        if not x.is_contiguous():
            raise ValueError("the layer's input must be contiguous")
        n = x.numel() // self.d_in
        z = ops.conv2d_fwd(x.view(n, 1, 1, self.d_in), self.W_lp.view(1, 1, self.d_in, -1), 1, (0, 0, 0, 0), stream=stream)
        return z.view(*x.shape[:-1], z.shape[-1])

    def forward(self, x: torch.Tensor, h0=None, lengths=None, save: bool = True, stream=None):
        """x (sequences x tokens x d_in, bf16, contiguous; its padding finite, as backward multiplies it by zeros):
        returns (y, the last states, what backward needs)."""
        z = self._product(x, stream)
        y, last, states = ops.gated_scan_fwd(z, self.output_gate, self.b, h0, lengths, save=save, stream=stream)
        return y, last, Saved(x, z, lengths, states) if save else None

    def backward(self, saved: Saved, dy: torch.Tensor, dh_last=None, stream=None):
        """The gradients (dx, dh0, dW, db) for dy and dh_last; what was saved is used up (dz takes z's place)."""
        x, z, lengths, states = saved
        dz, dh0 = ops.gated_scan_bwd(z, dy, states, self.output_gate, self.b, lengths, dh_last, dz=z, stream=stream)
        n = x.numel() // self.d_in
        x4, dz4 = x.view(n, 1, 1, self.d_in), dz.view(n, 1, 1, dz.shape[-1])
        w4 = self.W_lp.view(1, 1, self.d_in, -1)
        _, db = ops.bias_relu_bwd(None, dz4, dpre=dz4, stream=stream)
        dW = ops.conv2d_bwd_filter(x4, dz4, (1, 1), 1, (0, 0, 0, 0), stream=stream).view(self.d_in, -1)
        dx = ops.conv2d_bwd_input(dz4, w4, ops._empty_like(stream, x4), 1, (0, 0, 0, 0), stream=stream)
        return dx.view(x.shape), dh0, dW, db

    def step(self, x: torch.Tensor, state: torch.Tensor, slots=None, stream=None) -> torch.Tensor:
        """One token of each of n sequences being served (x: n x d_in): their states (slots x d, fp32) move on in
        place.  Returns y (n x d)."""
        return ops.gated_scan_step(self._product(x, stream), state, slots, self.output_gate, self.b, stream=stream)
