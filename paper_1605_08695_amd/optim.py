"""AdamW over all variables of a model at once, beside the updates of single variables in ``ops``."""
from __future__ import annotations

import ctypes
import operator
from typing import Optional, Sequence

import torch

from . import ops
from ._lib import check, load


class AdamW:
    """AdamW over a list of fp32 variables, updated in place with their bf16 copies (shadows, entries may be
    None).  bits=8 keeps the moments as e4m3 values with one fp32 factor for each 256 of them, and the second
    as its square root (a quarter of their memory, and 18 bytes a value moved in place of 30); bits=32 in fp32.
    weight_decay is one number, or one for each variable.

    In 8 bits a second moment follows its block's largest exactly, and its own gradients only by changes of more than
    half a code in one step: gradients that grow beside the rest of their block may take steps up to
    sqrt(1 + 0.129 / (1 - beta2)) times too large, 11 at 0.999 and 3.7 at 0.99, until they do; a beta2 of 0.99 or less
    suits it.  A step that is recorded or captured is replayed as the step t that it was.

    moments = (ms, vs, m_scales, v_scales) continues with moments that are there (the scales None with bits=32), for
    instance those of a checkpoint, with ``t`` the number of steps made.  The handle keeps all these tensors, whose
    memory must stay where it is while it is used."""

    def __init__(self, variables: Sequence[torch.Tensor], lr: float, beta1: float = 0.9, beta2: float = 0.999,
                 epsilon: float = 1e-8, weight_decay=0.0, shadows: Optional[Sequence] = None, bits: int = 32, moments=None,
                 t: int = 0):
        self.variables = list(variables)
        self.lr, self.beta1, self.beta2, self.epsilon = lr, beta1, beta2, epsilon
        self.bits, self.t = bits, operator.index(t)
        self.shadows = None if shadows is None else list(shadows)
        n = len(self.variables)
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(w) for w in weight_decay]
        if len(decay) != n:
            raise ValueError("weight_decay must be one number, or one for each variable")
        if moments is None:
            dtype = torch.float8_e4m3fn if bits == 8 else torch.float32
            zeros = lambda dt, size: [torch.zeros(size(v), dtype=dt, device=v.device) for v in self.variables]  # noqa: E731
            count = lambda v: ops.adamw_scales(v.numel())  # noqa: E731
            scales = [zeros(torch.float32, count) for _ in range(2)] if bits == 8 else [None, None]
            moments = (zeros(dtype, lambda v: v.shape), zeros(dtype, lambda v: v.shape), *scales)
        self.ms, self.vs = list(moments[0]), list(moments[1])
        self.m_scales, self.v_scales = (list(s) if s is not None else None for s in moments[2:4])
        ops._check_adamw(self.variables, self.ms, self.vs, self.m_scales, self.v_scales, self.shadows, bits)
        self._kept = [*self.variables, *self.ms, *self.vs, *(self.shadows or ())]
        if bits == 8:
            self._kept += [*self.m_scales, *self.v_scales]
        # what a call tells the library about the variables, laid out once; a step adds the gradients
        p = ops._pointers
        self._sizes = [v.numel() for v in self.variables]
        self._state = (p(self.variables), p(self.ms), p(self.vs), p(self.m_scales) if bits == 8 else None,
                       p(self.v_scales) if bits == 8 else None)
        self._ns = (ctypes.c_int64 * max(n, 1))(*self._sizes)
        self._decay = (ctypes.c_double * max(n, 1))(*decay)
        self._shadows = None if self.shadows is None else p(self.shadows)
        spans = sorted((x.data_ptr(), x.data_ptr() + x.numel() * x.element_size())
                       for x in self._kept if x is not None and x.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("variables, moments, scales and shadows must not share memory")
        devices = {t_.get_device() for t_ in self._kept if t_ is not None}
        if len(devices) > 1:
            raise ValueError("variables and moments must be on one GPU")

    def step(self, grads: Sequence[torch.Tensor], t: Optional[int] = None, stream=None) -> None:
        """One step for the gradients of all variables (fp32), as step t (default: the one after the last)."""
        ops._check_grads(grads, self._sizes)
        if not self.variables:
            return
        st = ops._on_device(stream, self.variables[0], *grads)
        t = self.t + 1 if t is None else operator.index(t)
        n = len(grads)
        check(load().tfk_apply_adamw_multi(n, self.bits, *self._state, (ctypes.c_void_p * n)(*[g.data_ptr() for g in grads]),
                                           self._ns, self._decay, self.lr, self.beta1, self.beta2, self.epsilon, t,
                                           self._shadows, st))
        self.t = t
