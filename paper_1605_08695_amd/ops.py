"""Python binding of the tfk_* C ABI over torch device tensors.

Argument marshalling only: every step runs in the HIP kernels of libtfk.so.
Tensors are NHWC torch tensors on the GPU; a 4-D tensor may be a channel
slice of a wider NHWC buffer (its pixel stride is passed to the library).
Filters are dense HWIO.  Every call is enqueued on ``stream`` (default: torch's
current stream) and raises TfkError on a non-OK status.  There is no CPU path.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import threading
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from ._lib import Nhwc, TfkError, Window, TFK_BF16, TFK_F32, check, load

__all__ = ["conv2d_fwd", "conv2d_fwd_bias_relu", "conv2d_bwd_input", "conv2d_bwd_filter", "conv2d_workspace_bytes", "bias_relu_fwd",
           "bias_relu_bwd", "bias_relu_bwd_workspace_bytes", "maxpool_fwd", "maxpool_bwd", "maxpool_bwd_relu_bwd", "apply_sgd",
           "apply_sgd_multi", "apply_momentum", "apply_adam", "softmax_xent",
           "gather_rows_t", "sampled_softmax_xent", "scatter_apply_sgd", "distill_xent", "embedding_fwd", "embedding_bwd",
           "embedding_apply_sgd", "embedding_workspace_bytes", "token_logprobs", "token_logprobs_bwd", "token_logprobs_workspace_bytes",
           "TokenLogprobs",
           "gated_scan_fwd", "gated_scan_bwd", "gated_scan_step", "gated_scan_workspace_bytes", "SCAN_BLOCK",
           "apply_adamw_multi", "adamw_scales", "stream_wait", "Program", "out_len", "nhwc",
           "window", "TfkError", "abi_version", "DeferredBias", "bias_grad_finish"]


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return TFK_F32
    if t.dtype == torch.bfloat16:
        return TFK_BF16
    raise TypeError("tfk supports float32 and bfloat16 tensors, got %s" % t.dtype)


# A small layer's kernels take a few microseconds, as long as marshalling one call did (10-12 us for a
# convolution): what follows from shapes and strides alone -- view and window descriptors, workspace
# sizes -- is computed once per distinct value and kept (bounded), and addresses and streams are
# passed as plain integers (5 us).  Nothing is kept by the identity or address of a tensor.
_KEPT = 4096


def _stream(stream) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return t.data_ptr() if t is not None else None


def _describe(shape, strides) -> Nhwc:
    n, h, w, c = shape
    s0, s1, s2, s3 = strides
    if n * h * w > 0:
        ps = s2 if w > 1 else (s1 if h > 1 else (s0 if n > 1 else c))
        if s3 != 1 or (w > 1 and s2 != ps) or (h > 1 and s1 != w * ps) or (n > 1 and s0 != h * w * ps):
            raise ValueError("tensor is not an NHWC view with unit channel stride: strides %s" % (tuple(strides),))
    else:
        ps = c
    return Nhwc(n, h, w, c, ps)


def nhwc(t: torch.Tensor) -> Nhwc:
    """Describes a 4-D NHWC tensor (or a channel slice of one) for the library."""
    if t.dim() != 4:
        raise ValueError("expected a 4-D NHWC tensor, got shape %s" % (tuple(t.shape),))
    return _describe(t.shape, t.stride())


_described = functools.lru_cache(_KEPT)(_describe)


def _view(t: torch.Tensor) -> Nhwc:
    """nhwc(t), shared between calls with tensors of one shape and strides (read only)."""
    if t.dim() != 4:
        raise ValueError("expected a 4-D NHWC tensor, got shape %s" % (tuple(t.shape),))
    return _described(t.shape, t.stride())


def window(kh, kw, stride, pads) -> Window:
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    pt, pb, pl, pr = pads
    return Window(kh, kw, sh, sw, pt, pb, pl, pr)


def _win_key(kh, kw, stride, pads) -> Tuple[int, ...]:
    """The values of window(...) as plain integers, so that equal keys are equal windows: 1.0 and True
    equal 1, and an integer tensor or array has no hash of its value."""
    sh, sw = (stride, stride) if isinstance(stride, int) else stride
    pt, pb, pl, pr = pads
    return tuple(map(operator.index, (kh, kw, sh, sw, pt, pb, pl, pr)))


@functools.lru_cache(_KEPT)
def _win_of(key) -> Window:
    return Window(*key)


def _win(kh, kw, stride, pads) -> Window:
    """window(...), shared between calls with the same values (read only)."""
    return _win_of(_win_key(kh, kw, stride, pads))


@functools.lru_cache(_KEPT)
def _conv_need(op, shape, strides, cout, key, dt) -> int:
    return load().tfk_conv2d_workspace_bytes(op, _describe(shape, strides), cout, Window(*key), dt)


def _conv_ws_need(op, x, cout, key, dt) -> int:
    """The workspace query of a convolution over x (a forward input's view), by its values."""
    return _conv_need(op, x.shape, x.stride(), cout, key, dt)


@functools.lru_cache(_KEPT)
def _bias_need(shape, strides, dt) -> int:
    return load().tfk_bias_relu_bwd_workspace_bytes(_describe(shape, strides), dt)


def out_len(n, k, s, p0, p1) -> int:
    return (n + p0 + p1 - k) // s + 1


def abi_version() -> int:
    return load().tfk_abi_version()


_recording = threading.local()     # .program: the Program recording on this thread


def _empty(stream, *args, **kw) -> torch.Tensor:
    """torch.empty on the stream the op is enqueued on: the caching allocator then hands the
    memory, once freed, only to later work on that same stream (a temporary freed on return
    cannot be reused by another stream while the kernel still runs).  A program that is recording
    keeps it: its runs use the same memory."""
    if stream is None:
        t = torch.empty(*args, **kw)
    else:
        with torch.cuda.stream(stream):
            t = torch.empty(*args, **kw)
    prog = getattr(_recording, "program", None)
    if prog is not None:
        prog.kept.append(t)
    return t


def _empty_like(stream, t: torch.Tensor) -> torch.Tensor:
    return _empty(stream, t.shape, dtype=t.dtype, device=t.device)


def _ws(nbytes: int, device, stream=None) -> Optional[torch.Tensor]:
    if nbytes == 0:
        return None
    return _empty(stream, (nbytes + 15) // 16 * 16, dtype=torch.uint8, device=device)


# ----------------------------------------------------------------------------- convolution
def conv2d_workspace_bytes(op: int, x: torch.Tensor, cout: int, kh, kw, stride, pads) -> int:
    return _conv_ws_need(operator.index(op), x, operator.index(cout), _win_key(kh, kw, stride, pads), _dt(x))


def _conv_fwd(x, w, bias, stride, pads, y, ws, stream):
    lib = load()
    kh, kw, cin, cout = w.shape
    key = _win_key(kh, kw, stride, pads)
    win = _win_of(key)
    need = _conv_ws_need(0, x, cout, key, _dt(x))
    if need and (ws is None or ws.numel() < need):
        ws = _ws(need, x.device, stream)
    if y is None:
        n, h, ww, _ = x.shape
        y = _empty(stream, (n, out_len(h, kh, win.stride_h, pads[0], pads[1]),
                         out_len(ww, kw, win.stride_w, pads[2], pads[3]), cout), dtype=x.dtype, device=x.device)
    if w.dtype != x.dtype or y.dtype != x.dtype:
        raise TypeError("x, w and y must share one dtype")
    wsp = _ptr(ws) if need else None
    if bias is None:
        check(lib.tfk_conv2d_fwd(_ptr(x), _view(x), _ptr(w), cout, win, _dt(x), _ptr(y), _view(y), wsp, need,
                                 _stream(stream)))
    else:
        if bias.dtype != torch.float32 or bias.numel() != cout or not bias.is_contiguous():
            raise ValueError("bias must be a contiguous float32 vector of cout values")
        check(lib.tfk_conv2d_fwd_bias_relu(_ptr(x), _view(x), _ptr(w), cout, _ptr(bias), win, _dt(x), _ptr(y),
                                           _view(y), wsp, need, _stream(stream)))
    return y


def conv2d_fwd(x, w, stride, pads, y=None, ws=None, stream=None):
    """y = x (*) w (cross-correlation).  x NHWC, w HWIO, pads (top, bottom, left, right)."""
    return _conv_fwd(x, w, None, stride, pads, y, ws, stream)


def conv2d_fwd_bias_relu(x, w, bias, stride, pads, y=None, ws=None, stream=None):
    """y = max(x (*) w + bias, 0) in one kernel (bias fp32, one value per output channel)."""
    return _conv_fwd(x, w, bias, stride, pads, y, ws, stream)


def conv2d_fwd_bias_relu_maxpool(x, w, bias, stride, pads, pool_hw, pool_stride, pool_pads=(0, 0, 0, 0), y=None,
                                 py=None, taps=None, ws=None, stream=None):
    """y = max(x (*) w + bias, 0) and its max-pool (py, uint8 window taps) in one call; one kernel
    where the convolution's row bands hold whole pool windows.  Returns (y, py, taps)."""
    lib = load()
    kh, kw, cin, cout = w.shape
    key = _win_key(kh, kw, stride, pads)
    win = _win_of(key)
    need = _conv_ws_need(0, x, cout, key, _dt(x))
    if need and (ws is None or ws.numel() < need):
        ws = _ws(need, x.device, stream)
    n, h, ww, _ = x.shape
    oh = out_len(h, kh, win.stride_h, pads[0], pads[1])
    ow = out_len(ww, kw, win.stride_w, pads[2], pads[3])
    if y is None:
        y = _empty(stream, (n, oh, ow, cout), dtype=x.dtype, device=x.device)
    pkh, pkw = pool_hw
    pwin = _win(pkh, pkw, pool_stride, pool_pads)
    poh = out_len(oh, pkh, pwin.stride_h, pool_pads[0], pool_pads[1])
    pow_ = out_len(ow, pkw, pwin.stride_w, pool_pads[2], pool_pads[3])
    if py is None:
        py = _empty(stream, (n, poh, pow_, cout), dtype=x.dtype, device=x.device)
    if taps is None:
        taps = _empty(stream, (n, poh, pow_, cout), dtype=torch.uint8, device=x.device)
    if not (w.dtype == y.dtype == py.dtype == x.dtype):
        raise TypeError("x, w, y and py must share one dtype")
    if taps.dtype != torch.uint8 or not taps.is_contiguous():
        raise ValueError("taps must be a dense uint8 tensor")
    if bias.dtype != torch.float32 or bias.numel() != cout or not bias.is_contiguous():
        raise ValueError("bias must be a contiguous float32 vector of cout values")
    check(lib.tfk_conv2d_fwd_bias_relu_maxpool(_ptr(x), _view(x), _ptr(w), cout, _ptr(bias), win, _dt(x), _ptr(y),
                                               _view(y), pwin, _ptr(py), _view(py), _ptr(taps),
                                               _ptr(ws) if need else None, need, _stream(stream)))
    return y, py, taps


def conv2d_bwd_input(dy, w, dx, stride, pads, beta=0.0, ws=None, stream=None):
    """dx (= or +=) conv2d_fwd^T(dy).  dx gives the forward input's shape (it is written)."""
    lib = load()
    kh, kw, cin, cout = w.shape
    if not (w.dtype == dy.dtype == dx.dtype):
        raise TypeError("dy, w and dx must share one dtype")
    key = _win_key(kh, kw, stride, pads)
    win = _win_of(key)
    need = _conv_ws_need(1, dx, cout, key, _dt(dx))
    if need and (ws is None or ws.numel() < need):
        ws = _ws(need, dx.device, stream)
    check(lib.tfk_conv2d_bwd_input(_ptr(dy), _view(dy), _ptr(w), win, _dt(dy), _ptr(dx), _view(dx), float(beta),
                                   _ptr(ws) if need else None, need, _stream(stream)))
    return dx


def conv2d_bwd_input_relu_bwd(dy, w, y, dpre, stride, pads, dbias=None, ws=None, stream=None, defer=False,
                              beta=0.0):
    """dpre = (y > 0) * (beta * dpre + conv2d_fwd^T(dy)), dbias = column sums of dpre (fp32): the
    input gradient fused with the ReLU backward of the layers that produced the input (y, dpre: its
    view); beta = 1 adds it to the gradient the input's other readers stored in dpre.
    defer=True: returns (dpre, DeferredBias) instead, the partials left in ws (see bias_grad_finish)."""
    lib = load()
    kh, kw, cin, cout = w.shape
    if not (w.dtype == dy.dtype == y.dtype == dpre.dtype):
        raise TypeError("dy, w, y and dpre must share one dtype")
    d_y, d_p = _view(y), _view(dpre)
    if d_y is not d_p and ((d_y.n, d_y.h, d_y.w, d_y.c, d_y.pixel_stride) !=
                           (d_p.n, d_p.h, d_p.w, d_p.c, d_p.pixel_stride)):
        raise ValueError("y and dpre must share one view (extents and pixel stride)")
    key = _win_key(kh, kw, stride, pads)
    win = _win_of(key)
    need = _conv_ws_need(3, dpre, cout, key, _dt(y))
    if defer:
        _need_ws(ws, need)
        dbias = None
    elif dbias is None:
        dbias = _empty(stream, cin, dtype=torch.float32, device=y.device)
    if need and (ws is None or ws.numel() < need):
        ws = _ws(need, y.device, stream)
    check(lib.tfk_conv2d_bwd_input_relu_bwd(_ptr(dy), _view(dy), _ptr(w), win, _dt(dy), _ptr(y), _ptr(dpre), d_p,
                                            float(beta), _ptr(dbias), _ptr(ws) if need else None, need,
                                            _stream(stream)))
    return dpre, (_deferred(lib, cin) if defer else dbias)


def conv2d_bwd_filter(x, dy, kernel_hw, stride, pads, dw=None, ws=None, stream=None):
    """dW (fp32 HWIO) = sum over pixels of x-gather * dy."""
    lib = load()
    kh, kw = kernel_hw
    cout = dy.shape[3]
    if dw is None:
        dw = _empty(stream, (kh, kw, x.shape[3], cout), dtype=torch.float32, device=x.device)
    if dy.dtype != x.dtype or dw.dtype != torch.float32:
        raise TypeError("x and dy share one dtype; dw is float32")
    key = _win_key(kh, kw, stride, pads)
    win = _win_of(key)
    need = _conv_ws_need(2, x, cout, key, _dt(x))
    if ws is None or ws.numel() < need:
        ws = _ws(need, x.device, stream)
    check(lib.tfk_conv2d_bwd_filter(_ptr(x), _view(x), _ptr(dy), _view(dy), win, _dt(x), _ptr(dw), _ptr(ws),
                                    need, _stream(stream)))
    return dw


def conv2d_bwd_filter_noalloc(x, dy, kernel_hw, stride, pads, dw, stream=None):
    """conv2d_bwd_filter with the library's own device scratch in place of a workspace: the call
    allocates nothing (dw must be given).  Calls that overlap in time on one GPU race."""
    kh, kw = kernel_hw
    cout = dy.shape[3]
    if dy.dtype != x.dtype or dw.dtype != torch.float32:
        raise TypeError("x and dy share one dtype; dw is float32")
    if tuple(dw.shape) != (kh, kw, x.shape[3], cout) or not dw.is_contiguous():
        raise ValueError("dw must be a contiguous float32 HWIO tensor")
    check(load().tfk_conv2d_bwd_filter_noalloc(_ptr(x), _view(x), _ptr(dy), _view(dy), _win(kh, kw, stride, pads),
                                               _dt(x), _ptr(dw), _stream(stream)))
    return dw


# ----------------------------------------------------------------------------- bias + relu
def bias_relu_fwd(y, bias, stream=None):
    """In place: y <- max(y + bias, 0)."""
    check(load().tfk_bias_relu_fwd(_ptr(y), _view(y), _ptr(bias), _dt(y), _stream(stream)))
    return y


def bias_relu_bwd_workspace_bytes(y) -> int:
    return _bias_need(y.shape, y.stride(), _dt(y))


def bias_relu_bwd(y, dy, dpre=None, dbias=None, ws=None, stream=None, defer=False):
    """dpre = dy * (y > 0) (dpre may be dy), dbias = column sums of dpre (fp32).  With y None
    (a bias-only layer) dpre = dy and dbias = column sums of dy.  defer=True: returns
    (dpre, DeferredBias) instead, the partials left in ws (see bias_grad_finish)."""
    lib = load()
    if dpre is None:
        dpre = _empty_like(stream, dy)
    view = y if y is not None else dy
    need = _bias_need(view.shape, view.stride(), _dt(view))
    if defer:
        _need_ws(ws, need)
        dbias = None
    elif dbias is None:
        dbias = _empty(stream, dy.shape[3], dtype=torch.float32, device=dy.device)
    if ws is None or ws.numel() < need:
        ws = _ws(need, dy.device, stream)
    d_y, d_dy, d_dp = _view(view), _view(dy), _view(dpre)
    if (d_y.pixel_stride, d_y.c) != (d_dy.pixel_stride, d_dy.c) or (d_y.pixel_stride, d_y.c) != (d_dp.pixel_stride, d_dp.c):
        raise ValueError("y, dy and dpre must share one view (extents and pixel stride)")
    check(lib.tfk_bias_relu_bwd(_ptr(y), _ptr(dy), d_y, _ptr(dpre), _ptr(dbias), _dt(dy), _ptr(ws), need,
                                _stream(stream)))
    return dpre, (_deferred(lib, dy.shape[3]) if defer else dbias)


def softmax_xent(logits, labels, scale, bias=None, loss=None, dlogits=None, stream=None):
    """Softmax cross-entropy of contiguous logits (rows of the last dimension) + bias against int32
    labels: returns (per-row loss fp32, dlogits = scale * (softmax - onehot)); dlogits may be logits."""
    if not logits.is_contiguous():
        raise ValueError("logits must be contiguous")
    c = logits.shape[-1]
    n = logits.numel() // c if c else 0
    if labels.dtype != torch.int32 or labels.numel() != n:
        raise ValueError("labels must be int32, one per row")
    if bias is not None and (bias.dtype != torch.float32 or bias.numel() != c):
        raise ValueError("bias must be float32 [c]")
    if loss is None:
        loss = _empty(stream, n, dtype=torch.float32, device=logits.device)
    if dlogits is None:
        dlogits = _empty_like(stream, logits)
    if dlogits.dtype != logits.dtype or dlogits.numel() != logits.numel() or not dlogits.is_contiguous():
        raise ValueError("dlogits must be a contiguous tensor like logits")
    check(load().tfk_softmax_xent(_ptr(logits), _dt(logits), n, c, _ptr(bias), _ptr(labels), float(scale),
                                  _ptr(loss), _ptr(dlogits), _stream(stream)))
    return loss, dlogits


# ----------------------------------------------------------------------------- max-pool
def maxpool_fwd(x, kernel_hw, stride, pads, y=None, argmax=None, stream=None, taps=False):
    """Returns (y, argmax).  argmax is int32 dense NHWC indices into x, or with ``taps`` uint8
    window taps kh * KW + kw (a quarter of the bytes); the backward ops accept either."""
    lib = load()
    kh, kw = kernel_hw
    win = _win(kh, kw, stride, pads)
    n, h, w, c = x.shape
    oh = out_len(h, kh, win.stride_h, pads[0], pads[1])
    ow = out_len(w, kw, win.stride_w, pads[2], pads[3])
    if y is None:
        y = _empty(stream, (n, oh, ow, c), dtype=x.dtype, device=x.device)
    if argmax is None:
        argmax = _empty(stream, (n, oh, ow, c), dtype=torch.uint8 if taps else torch.int32, device=x.device)
    fn = _argmax_fn(lib, "tfk_maxpool_fwd", argmax)
    check(fn(_ptr(x), _view(x), win, _dt(x), _ptr(y), _view(y), _ptr(argmax), _stream(stream)))
    return y, argmax


def _argmax_fn(lib, name, argmax):
    """The entry point for this argmax format: int32 dense indices, or uint8 taps (``_taps``)."""
    if not argmax.is_contiguous() or argmax.dtype not in (torch.int32, torch.uint8):
        raise ValueError("argmax must be a dense int32 (indices) or uint8 (taps) tensor")
    return getattr(lib, name + ("_taps" if argmax.dtype == torch.uint8 else ""))


def maxpool_bwd(dy, argmax, dx, kernel_hw, stride, pads, beta=0.0, stream=None):
    kh, kw = kernel_hw
    fn = _argmax_fn(load(), "tfk_maxpool_bwd", argmax)
    check(fn(_ptr(dy), _ptr(argmax), _view(dy), _win(kh, kw, stride, pads), _dt(dy), _ptr(dx), _view(dx),
             float(beta), _stream(stream)))
    return dx


def maxpool_bwd_relu_bwd(dy, argmax, y, dpre, kernel_hw, stride, pads, beta=0.0, dbias=None, ws=None, stream=None,
                         py=None, defer=False):
    """dpre = (y > 0) * (beta * dpre + max-pool gradient of dy), dbias = column sums of dpre (fp32).

    y is the pool input (the ReLU output); dpre has its shape and view.  py (optional) is the
    pool's output: with beta = 0 the mask is taken from it per window and y is not read (y may
    then be None).  defer=True: returns (dpre, DeferredBias) instead, the partials left in ws
    (see bias_grad_finish).
    """
    lib = load()
    kh, kw = kernel_hw
    fn = _argmax_fn(lib, "tfk_maxpool_bwd_relu_bwd", argmax)
    d_p = _view(dpre)
    if y is not None:
        d_y = _view(y)
        if d_y is not d_p and ((d_y.n, d_y.h, d_y.w, d_y.c, d_y.pixel_stride) !=
                           (d_p.n, d_p.h, d_p.w, d_p.c, d_p.pixel_stride)):
            raise ValueError("y and dpre must share one view (extents and pixel stride)")
    pys = 0
    if py is not None:
        if tuple(py.shape) != tuple(dy.shape) or py.dtype != dy.dtype:
            raise ValueError("py must have dy's shape and element type")
        pys = _view(py).pixel_stride
    need = _bias_need(dpre.shape, dpre.stride(), _dt(dpre))
    if defer:
        _need_ws(ws, need)
        dbias = None
    elif dbias is None:
        dbias = _empty(stream, dpre.shape[3], dtype=torch.float32, device=dpre.device)
    if ws is None or ws.numel() < need:
        ws = _ws(need, dpre.device, stream)
    check(fn(_ptr(dy), _ptr(argmax), _view(dy), _win(kh, kw, stride, pads), _dt(dy),
             _ptr(y), _ptr(py), pys, _ptr(dpre), d_p,
             float(beta), _ptr(dbias), _ptr(ws), need, _stream(stream)))
    return dpre, (_deferred(lib, dpre.shape[3]) if defer else dbias)


# ----------------------------------------------------------------------------- deferred bias gradients
class DeferredBias(NamedTuple):
    """Where a call made with defer=True left its bias-gradient partials: inside the workspace it
    was given, which must stay untouched until bias_grad_finish has run."""
    part: int          # device address
    rows: int          # partials per channel
    channels: int


def _need_ws(ws, need):
    if ws is None or ws.numel() < need:
        raise ValueError("defer=True needs a caller workspace of at least %d bytes (the partials stay in it)" % need)


def _deferred(lib, channels) -> DeferredBias:
    part, rows = ctypes.c_void_p(), ctypes.c_int32()
    check(lib.tfk_last_bias_partials(ctypes.byref(part), ctypes.byref(rows)))
    return DeferredBias(part.value or 0, rows.value, int(channels))


def bias_grad_finish(jobs, stream=None):
    """For every (DeferredBias, dbias) in jobs: dbias = the fixed-order per-channel sums of the
    partials its deferred call left (the same bits as the call given dbias), in one launch."""
    lib = load()
    n = len(jobs)
    for d, db in jobs:
        if db.dtype != torch.float32 or not db.is_contiguous() or db.numel() != d.channels:
            raise ValueError("dbias must be contiguous float32 with one value per channel")
    parts = (ctypes.c_void_p * max(n, 1))(*[d.part for d, _ in jobs])
    rows = (ctypes.c_int32 * max(n, 1))(*[d.rows for d, _ in jobs])
    chans = (ctypes.c_int32 * max(n, 1))(*[d.channels for d, _ in jobs])
    dbs = (ctypes.c_void_p * max(n, 1))(*[db.data_ptr() for _, db in jobs])
    check(lib.tfk_bias_grad_finish(n, parts, rows, chans, dbs, _stream(stream)))


# ----------------------------------------------------------------------------- update
def apply_sgd(var, grad, lr, shadow=None, stream=None):
    """In place: var <- fma(-lr, grad, var); shadow (bf16) <- bf16(var) if given."""
    if var.dtype != torch.float32 or grad.dtype != torch.float32:
        raise TypeError("var and grad are float32")
    if not (var.is_contiguous() and grad.is_contiguous()) or var.numel() != grad.numel():
        raise ValueError("var and grad must be contiguous with the same size")
    if shadow is not None and (shadow.dtype != torch.bfloat16 or shadow.numel() != var.numel()
                               or not shadow.is_contiguous()):
        raise ValueError("shadow must be a contiguous bfloat16 tensor of var's size")
    check(load().tfk_apply_sgd(_ptr(var), _ptr(grad), var.numel(), float(lr), _ptr(shadow), _stream(stream)))
    return var


def _check_update(var, grad, slots, shadow):
    for t in (var, grad, *slots):
        if t.dtype != torch.float32:
            raise TypeError("var, grad and the optimizer slots are float32")
        if not t.is_contiguous() or t.numel() != var.numel():
            raise ValueError("var, grad and the optimizer slots must be contiguous with the same size")
    if shadow is not None and (shadow.dtype != torch.bfloat16 or shadow.numel() != var.numel()
                               or not shadow.is_contiguous()):
        raise ValueError("shadow must be a contiguous bfloat16 tensor of var's size")


def apply_momentum(var, accum, grad, lr, momentum, nesterov=False, shadow=None, stream=None):
    """In place: accum <- momentum * accum + grad; var <- var - lr * accum (or, look-ahead form,
    var <- var - lr * (grad + momentum * accum)); shadow (bf16) <- bf16(var) if given."""
    _check_update(var, grad, (accum,), shadow)
    check(load().tfk_apply_momentum(_ptr(var), _ptr(accum), _ptr(grad), var.numel(), float(lr), float(momentum),
                                    int(bool(nesterov)), _ptr(shadow), _stream(stream)))
    return var


def apply_adam(var, m, v, grad, lr, beta1, beta2, epsilon, t, shadow=None, stream=None):
    """In place, Adam step t >= 1: the moments m and v and var; shadow (bf16) <- bf16(var) if given."""
    _check_update(var, grad, (m, v), shadow)
    check(load().tfk_apply_adam(_ptr(var), _ptr(m), _ptr(v), _ptr(grad), var.numel(), float(lr), float(beta1),
                                float(beta2), float(epsilon), int(t), _ptr(shadow), _stream(stream)))
    return var


def apply_sgd_multi(vars_: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], lr,
                    shadows: Optional[Sequence[Optional[torch.Tensor]]] = None, stream=None):
    count = len(vars_)
    VP = ctypes.c_void_p * max(count, 1)
    NS = ctypes.c_int64 * max(count, 1)
    v = VP(*[t.data_ptr() for t in vars_])
    g = VP(*[t.data_ptr() for t in grads])
    ns = NS(*[t.numel() for t in vars_])
    sh = None
    if shadows is not None:
        sh = VP(*[(t.data_ptr() if t is not None else 0) for t in shadows])
    check(load().tfk_apply_sgd_multi(count, v, g, ns, float(lr), sh, _stream(stream)))


def adamw_scales(n: int) -> int:
    """How many factors the 8-bit moments of a variable of n values have: one for each 256."""
    return (n + 255) // 256


def _check_adamw(vars_, ms, vs, m_scales, v_scales, shadows, bits):
    """Types, sizes and layout of the variables and of what is kept for each."""
    if bits not in (8, 32):
        raise ValueError("bits must be 8 or 32, got %r" % (bits,))
    kinds = [("m", ms, torch.float32 if bits == 32 else torch.float8_e4m3fn), ("v", vs, torch.float32 if bits == 32 else
                                                                              torch.float8_e4m3fn)]
    if bits == 8:
        if m_scales is None or v_scales is None:
            raise ValueError("moments in 8 bits need m_scales and v_scales")
        kinds += [("m_scales", m_scales, torch.float32), ("v_scales", v_scales, torch.float32)]
    if shadows is not None:
        kinds.append(("shadows", shadows, torch.bfloat16))
    for name, ts, dtype in kinds:
        if len(ts) != len(vars_):
            raise ValueError("%s must have one entry for each variable" % name)
        for i, (var, t) in enumerate(zip(vars_, ts)):
            if t is None and name == "shadows":
                continue
            n = adamw_scales(var.numel()) if name.endswith("scales") else var.numel()
            if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
                raise ValueError("%s of variable %d must be a contiguous %s tensor of %d values" %
                                 (name, i, str(dtype).split(".")[-1], n))
    for i, var in enumerate(vars_):
        if var.dtype != torch.float32 or not var.is_contiguous():
            raise ValueError("variable %d must be contiguous float32" % i)


def _pointers(ts):
    return (ctypes.c_void_p * max(len(ts), 1))(*[t.data_ptr() if t is not None else 0 for t in ts])


def _check_grads(grads, sizes):
    if len(grads) != len(sizes):
        raise ValueError("one gradient for each variable")
    for i, (g, n) in enumerate(zip(grads, sizes)):
        if g.dtype != torch.float32 or g.numel() != n or not g.is_contiguous():
            raise ValueError("the gradient of variable %d must be a contiguous float32 tensor of %d values" % (i, n))


def apply_adamw_multi(vars_: Sequence[torch.Tensor], ms, vs, grads, lr, beta1, beta2, epsilon, t, weight_decay=None,
                      shadows=None, m_scales=None, v_scales=None, bits=32, stream=None):
    """In place, AdamW step t >= 1 over all variables at once: moments ms and vs in fp32, or with bits=8 as
    float8_e4m3fn values (vs: the square root) with one fp32 factor for each 256 of them in m_scales and
    v_scales; weight_decay one number for each variable; shadows bf16 copies (entries may be None).
    optim.AdamW keeps all of this for a program."""
    _check_adamw(vars_, ms, vs, m_scales, v_scales, shadows, bits)
    sizes = [v.numel() for v in vars_]
    _check_grads(grads, sizes)
    n = len(vars_)
    if weight_decay is not None and len(weight_decay) != n:
        raise ValueError("weight_decay must have one entry for each variable")
    if n == 0:
        return
    st = _on_device(stream, *vars_, *ms, *vs, *grads, *(shadows or ()), *((*m_scales, *v_scales) if bits == 8 else ()))
    check(load().tfk_apply_adamw_multi(
        n, bits, _pointers(vars_), _pointers(ms), _pointers(vs), _pointers(m_scales) if bits == 8 else None,
        _pointers(v_scales) if bits == 8 else None, _pointers(grads), (ctypes.c_int64 * n)(*sizes),
        None if weight_decay is None else (ctypes.c_double * n)(*weight_decay), float(lr), float(beta1), float(beta2),
        float(epsilon), operator.index(t), None if shadows is None else _pointers(shadows), st))


# ----------------------------------------------------------------------------- sampled softmax
def gather_rows_t(table, idx, u_pad, out_t=None, stream=None):
    """out_t (d x u_pad) = table[idx]^T, zero past len(idx); table (rows x d) contiguous."""
    rows, d = table.shape
    u = idx.numel()
    if idx.dtype != torch.int32 or not table.is_contiguous():
        raise ValueError("idx must be int32 and table contiguous")
    if out_t is None:
        out_t = _empty(stream, d, u_pad, dtype=table.dtype, device=table.device)
    if out_t.dtype != table.dtype or out_t.numel() != d * u_pad or not out_t.is_contiguous():
        raise ValueError("out_t must be a contiguous d x u_pad tensor of table's type")
    check(load().tfk_gather_rows_t(_ptr(table), _dt(table), rows, d, _ptr(idx), u, u_pad, _ptr(out_t),
                                   _stream(stream)))
    return out_t


def sampled_softmax_xent(z, u, m, true_pos, lq_true, lq_sampled, scale, bias_c=None, loss=None, dz=None,
                         stream=None):
    """Cross-entropy over candidate logits z (n x u_pad): returns (loss per row, dz)."""
    n, u_pad = z.shape[0], z.shape[-1]
    if not z.is_contiguous() or z.numel() != n * u_pad:
        raise ValueError("z must be contiguous n x u_pad")
    if loss is None:
        loss = _empty(stream, n, dtype=torch.float32, device=z.device)
    if dz is None:
        dz = _empty_like(stream, z)
    check(load().tfk_sampled_softmax_xent(_ptr(z), _dt(z), n, u, u_pad, m, _ptr(bias_c), _ptr(true_pos),
                                          _ptr(lq_true), _ptr(lq_sampled), float(scale), _ptr(loss), _ptr(dz),
                                          _stream(stream)))
    return loss, dz


def scatter_apply_sgd(var, idx, grad_t, lr, shadow=None, stream=None):
    """var[idx[j]] -= lr * grad_t[:, j] (var rows x d fp32; grad_t d x ld fp32); shadow rewritten."""
    rows, d = var.shape if var.dim() == 2 else (var.shape[0], 1)
    ld = grad_t.shape[-1]
    if var.dtype != torch.float32 or grad_t.dtype != torch.float32 or idx.dtype != torch.int32:
        raise TypeError("var and grad_t are float32, idx int32")
    check(load().tfk_scatter_apply_sgd(_ptr(var), _ptr(shadow), rows, d, _ptr(idx), idx.numel(), _ptr(grad_t), ld,
                                       float(lr), _stream(stream)))
    return var


# ----------------------------------------------------------------------------- rows
def _width(c, name) -> int:
    """c, a number of columns that the library counts in 32 bits."""
    if c > 0x7fffffff:
        raise ValueError("%s has more than 2^31 - 1 columns" % name)
    return c


def _rows_of(t, name) -> Tuple[int, int, int]:
    """(n, c, elements between rows) of a tensor whose last dimension has unit stride and whose others
    together are n rows a fixed distance apart."""
    shape = t.shape
    if len(shape) == 2:
        n, c = shape
        s, s1 = (c, 1) if t.is_contiguous() else t.stride()
    else:
        if len(shape) < 2:
            raise ValueError("%s must have rows and columns, got shape %s" % (name, tuple(shape)))
        c = shape[-1]
        n = t.numel() // c if c else 0
        if not t.is_contiguous():
            raise ValueError("%s with more than two dimensions must be contiguous" % name)
        s, s1 = c, 1
    if n < 2:
        s = c
    if c == 0 or (c > 1 and s1 != 1 and n > 0) or s < c:
        raise ValueError("%s must be rows of unit stride that do not overlap, got shape %s, strides %s" %
                         (name, tuple(t.shape), tuple(t.stride())))
    return n, _width(c, name), s


def _vector(t, dtype, n, name):
    if t is not None and (t.dtype != dtype or t.numel() != n or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous %s tensor of %d values" % (name, str(dtype).split(".")[-1], n))


def _on_device(stream, first, *others) -> int:
    """The stream to enqueue on (given or current).  Every operand must be on the current GPU, and the
    stream of that GPU."""
    at = first.get_device()
    for t in others:
        if t is not None and t.get_device() != at:
            raise ValueError("operands must be on one GPU, got %s and %s" % (first.device, t.device))
    if at < 0:
        raise ValueError("operands must be on the GPU, got one on %s" % first.device)
    if at != torch._C._cuda_getDevice() or (stream is not None and stream.device.index != at):
        raise ValueError("operands are on GPU %d, which is not the current device or the stream's" % at)
    return torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream


# ----------------------------------------------------------------------------- distillation
def distill_xent(logits, top_idx, top, scale, temperature=1.0, top_lse=None, labels=None, alpha=1.0, weight=None,
                 bias=None, loss=None, dlogits=None, stream=None):
    """Distillation from a teacher's k largest logits: returns (loss per row, dlogits), where
    loss = weight * (alpha T^2 KL(teacher || student) + (1 - alpha) cross-entropy with labels) and
    dlogits = scale * its gradient.

    logits: rows of c classes (+ bias), dlogits the same shape and type (may be logits: in place).
    top, top_idx (n x k): the teacher's logits and their classes, -1 for none; renormalised over the
    list, or with top_lse (the log-sum-exp of all the teacher's logits / temperature) the rest of its
    mass counts as one more class.  Rows of weight 0 give loss 0 and no gradient.  Not differentiated
    through the teacher."""
    n, c, ld = _rows_of(logits, "logits")
    shape = top.shape
    if len(shape) < 2 or shape != top_idx.shape or top.numel() != n * shape[-1]:
        raise ValueError("top and top_idx must share one shape of n rows, got %s and %s" % (tuple(shape),
                                                                                          tuple(top_idx.shape)))
    if top_idx.dtype != torch.int32 or not (top_idx.is_contiguous() and top.is_contiguous()):
        raise ValueError("top_idx must be int32, top and top_idx contiguous")
    k = _width(shape[-1], "top")
    _vector(top_lse, torch.float32, n, "top_lse")
    _vector(labels, torch.int32, n, "labels")
    _vector(weight, torch.float32, n, "weight")
    _vector(bias, torch.float32, c, "bias")
    _vector(loss, torch.float32, n, "loss")
    dt, tdt = _dt(logits), _dt(top)
    dld = c if dlogits is None else ld
    if dlogits is not None and dlogits is not logits:
        if dlogits.shape != logits.shape or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits must have the logits' shape and type")
        dld = _rows_of(dlogits, "dlogits")[2]
    st = _on_device(stream, logits, top, top_idx, top_lse, labels, weight, bias, loss, dlogits)
    if loss is None:
        loss = _empty(stream, n, dtype=torch.float32, device=logits.device)
    if dlogits is None:
        dlogits = _empty_like(stream, logits)
    check(load().tfk_distill_xent(_ptr(logits), dt, n, c, ld, _ptr(bias), _ptr(top), tdt, _ptr(top_idx), k,
                                  _ptr(top_lse), _ptr(labels), _ptr(weight), float(temperature), float(alpha),
                                  float(scale), _ptr(loss), _ptr(dlogits), dld, st))
    return loss, dlogits


# ----------------------------------------------------------------------------- embedding table
def _ids(ids):
    if ids.dtype != torch.int32 or not ids.is_contiguous():
        raise ValueError("ids must be a contiguous int32 tensor")
    return ids.numel()


def embedding_fwd(table, ids, scale=1.0, out=None, out_dtype=None, stream=None):
    """out[i] = scale * table[ids[i]] (zeros for an id outside the table); table (rows x d) and out of
    either type (out_dtype, default table's).  Returns out, ids' shape with d columns."""
    n = _ids(ids)
    if table.dim() != 2:
        raise ValueError("table must be rows x d, got shape %s" % (tuple(table.shape),))
    rows, d, tld = _rows_of(table, "table")
    dt = _dt(table)
    shape = tuple(ids.shape) + (d,)
    if out is None:
        st = _on_device(stream, table, ids)
        out = _empty(stream, shape, dtype=out_dtype or table.dtype, device=table.device)
        old = d
    else:
        if tuple(out.shape) != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must be %s%s, got %s of %s" % (shape, " of %s" % out_dtype if out_dtype else "",
                                                                tuple(out.shape), out.dtype))
        if len(shape) == 1 and not out.is_contiguous():
            raise ValueError("out must be contiguous for a single id")
        old = d if len(shape) == 1 else _rows_of(out, "out")[2]
        st = _on_device(stream, table, ids, out)
    check(load().tfk_embedding_fwd(_ptr(table), dt, rows, tld, d, _ptr(ids), n, float(scale), _ptr(out), _dt(out), old,
                                   st))
    return out


def embedding_workspace_bytes(n, d, rows) -> int:
    """Workspace of embedding_bwd and embedding_apply_sgd for n tokens of a rows x d table."""
    return load().tfk_embedding_workspace_bytes(operator.index(n), _width(operator.index(d), "dy"), operator.index(rows))


_embed_need = functools.lru_cache(_KEPT)(embedding_workspace_bytes)


def _embed_args(dy, ids, stream, ws, rows, d, *more):
    """Checks dy (ids' shape with d columns) and the operands' device; returns (n, dy's row distance,
    workspace, its bytes, stream)."""
    n = _ids(ids)
    if tuple(dy.shape) != tuple(ids.shape) + (d,):
        raise ValueError("dy must be %s, got %s" % (tuple(ids.shape) + (d,), tuple(dy.shape)))
    ld = d if dy.dim() == 1 and dy.is_contiguous() else _rows_of(dy, "dy")[2]
    if ws is not None and not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    st = _on_device(stream, dy, ids, ws, *more)
    need = _embed_need(n, d, rows)
    if need and (ws is None or ws.numel() * ws.element_size() < need):
        ws = _ws(need, dy.device, stream)
    return n, ld, ws, need, st


def embedding_bwd(dy, ids, rows, scale=1.0, dtable=None, beta=0.0, ws=None, stream=None):
    """The table's dense fp32 gradient: dtable (rows x d) = beta * dtable + scale * the sum of dy over
    each row's tokens (beta 0 or 1).  Returns dtable."""
    d = _width(dy.shape[-1], "dy") if dy.dim() else 0
    rows = operator.index(rows)
    if dtable is None and beta != 0.0:
        raise ValueError("beta = 1 adds to a dtable that is given")
    if dtable is not None and (dtable.dtype != torch.float32 or tuple(dtable.shape) != (rows, d) or
                               not dtable.is_contiguous()):
        raise ValueError("dtable must be a contiguous float32 tensor of %d x %d" % (rows, d))
    dt = _dt(dy)
    n, ld, ws, need, st = _embed_args(dy, ids, stream, ws, rows, d, dtable)
    if dtable is None:
        dtable = _empty(stream, (rows, d), dtype=torch.float32, device=dy.device)
    check(load().tfk_embedding_bwd(_ptr(dy), dt, n, ld, d, _ptr(ids), rows, float(scale), float(beta), _ptr(dtable),
                                   _ptr(ws), need, st))
    return dtable


def embedding_apply_sgd(var, ids, dy, lr, scale=1.0, shadow=None, ws=None, stream=None):
    """In place: var[r] -= lr * scale * the sum of dy over the tokens of row r, for the rows that have
    tokens (ids may repeat); shadow (bf16) rewritten there.  Returns var."""
    if var.dim() != 2 or var.dtype != torch.float32 or not var.is_contiguous():
        raise ValueError("var must be a contiguous float32 tensor of rows x d")
    if shadow is not None and (shadow.dtype != torch.bfloat16 or shadow.shape != var.shape or not shadow.is_contiguous()):
        raise ValueError("shadow must be a contiguous bfloat16 tensor of var's shape")
    rows, d = var.shape[0], _width(var.shape[1], "var")
    dt = _dt(dy)
    n, ld, ws, need, st = _embed_args(dy, ids, stream, ws, rows, d, var, shadow)
    check(load().tfk_embedding_apply_sgd(_ptr(var), _ptr(shadow), rows, d, _ptr(ids), n, _ptr(dy), dt, ld, float(scale),
                                         float(lr), _ptr(ws), need, st))
    return var


# ----------------------------------------------------------------------------- log-probabilities
class TokenLogprobs(NamedTuple):
    """What token_logprobs found out about each row; logp without tokens and top_* with k = 0 are None."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    top_idx: Optional[torch.Tensor]
    top_logp: Optional[torch.Tensor]


def token_logprobs_workspace_bytes(n, c, k) -> int:
    """Workspace of token_logprobs for n rows of c classes and the k largest of them."""
    return load().tfk_token_logprobs_workspace_bytes(operator.index(n), _width(operator.index(c), "logits"), operator.index(k))


_logprob_need = functools.lru_cache(_KEPT)(token_logprobs_workspace_bytes)


def token_logprobs(logits, tokens=None, k=0, temperature=1.0, bias=None, ws=None, stream=None) -> TokenLogprobs:
    """Of each row of (logits + bias) / temperature: the log-probability of its token (int32; one outside the
    classes is padding), the entropy, the log-sum-exp and the k <= 128 largest classes with their
    log-probabilities, largest first (n x k, -1 and -inf behind the last class that is not -inf)."""
    n, c, ld = _rows_of(logits, "logits")
    k = operator.index(k)
    if not 0 <= k <= 128:
        raise ValueError("k must be in 0..128, got %d" % k)
    _vector(tokens, torch.int32, n, "tokens")
    _vector(bias, torch.float32, c, "bias")
    dt = _dt(logits)
    if ws is not None and not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    st = _on_device(stream, logits, tokens, bias, ws)
    need = _logprob_need(n, c, k)
    if need and (ws is None or ws.numel() * ws.element_size() < need):
        ws = _ws(need, logits.device, stream)
    out = _empty(stream, (2 if tokens is None else 3, n), dtype=torch.float32, device=logits.device)
    idx = top = None
    if k:
        idx = _empty(stream, (n, k), dtype=torch.int32, device=logits.device)
        top = _empty(stream, (n, k), dtype=torch.float32, device=logits.device)
    r = TokenLogprobs(None if tokens is None else out[2], out[0], out[1], idx, top)
    check(load().tfk_token_logprobs(_ptr(logits), dt, n, c, ld, _ptr(bias), _ptr(tokens), float(temperature), k, _ptr(r.logp),
                                    _ptr(r.entropy), _ptr(r.lse), _ptr(idx), _ptr(top), _ptr(ws), need, st))
    return r


def token_logprobs_bwd(logits, tokens, lse, dlogp, entropy=None, dentropy=None, temperature=1.0, bias=None, dlogits=None,
                       stream=None):
    """The logits' gradient for the gradients dlogp of token_logprobs' logp and, if given, dentropy of its entropy;
    lse and entropy as that call returned them.  dlogits may be logits (in place).  Returns dlogits."""
    n, c, ld = _rows_of(logits, "logits")
    _vector(tokens, torch.int32, n, "tokens")
    _vector(lse, torch.float32, n, "lse")
    _vector(dlogp, torch.float32, n, "dlogp")
    _vector(entropy, torch.float32, n, "entropy")
    _vector(dentropy, torch.float32, n, "dentropy")
    _vector(bias, torch.float32, c, "bias")
    if dentropy is not None and entropy is None:
        raise ValueError("dentropy needs the entropy")
    dt, dld = _dt(logits), c if dlogits is None else ld
    if dlogits is not None and dlogits is not logits:
        if dlogits.shape != logits.shape or dlogits.dtype != logits.dtype:
            raise ValueError("dlogits must have the logits' shape and type")
        dld = _rows_of(dlogits, "dlogits")[2]
    st = _on_device(stream, logits, tokens, lse, dlogp, entropy, dentropy, bias, dlogits)
    if dlogits is None:
        dlogits = _empty(stream, logits.shape, dtype=logits.dtype, device=logits.device)
    check(load().tfk_token_logprobs_bwd(_ptr(logits), dt, n, c, ld, _ptr(bias), _ptr(tokens), float(temperature), _ptr(lse),
                                        _ptr(entropy), _ptr(dlogp), _ptr(dentropy), _ptr(dlogits), dld, st))
    return dlogits


# ----------------------------------------------------------------------------- gated linear recurrence
SCAN_BLOCK = 16       # tokens between two states that gated_scan_fwd saves


@functools.lru_cache(_KEPT)
def _seq_layout(shape, strides, name, cols) -> Tuple[int, int, int, int, int]:
    if len(shape) != 3:
        raise ValueError("%s must be sequences x tokens x columns, got shape %s" % (name, tuple(shape)))
    b, n, c = shape
    if c == 0 or (cols is not None and c != cols):
        raise ValueError("%s must have %s columns, got shape %s" % (name, cols or "some", tuple(shape)))
    sb, st, sc = strides
    if b and n and c > 1 and sc != 1:
        raise ValueError("%s must have unit stride within rows, got strides %s" % (name, tuple(strides)))
    st = st if n > 1 else c
    sb = sb if b > 1 else max(1, n) * st
    if b and n and not ((st >= c and (b == 1 or sb >= (n - 1) * st + c)) or (sb >= c and st >= (b - 1) * sb + c)):
        raise ValueError("%s must have rows that do not overlap, got shape %s, strides %s" % (name, tuple(shape), tuple(strides)))
    return b, n, _width(c, name), sb, st


def _seqs(t, name, cols=None) -> Tuple[int, int, int, int, int]:
    """(b, t, columns, elements between sequences, between rows) of a b x t x columns tensor of either order."""
    return _seq_layout(t.shape, t.stride(), name, cols)


def _scan_args(z, output_gate, bias, lengths):
    gates = 3 if output_gate else 2
    b, t, cols, zb, zt = _seqs(z, "z")
    if cols % gates:
        raise ValueError("z must have %d columns for each channel, got %d" % (gates, cols))
    _vector(bias, torch.float32, cols, "bias")
    _vector(lengths, torch.int32, b, "lengths")
    return gates, b, t, cols // gates, zb, zt


def _like_seqs(stream, z, cols, zb, zt):
    """A dense b x t x cols tensor with z's order of sequences and tokens, and its two distances."""
    b, t = z.shape[:2]
    if b > 1 and t > 1 and zb < zt:
        return _empty(stream, (t, b, cols), dtype=z.dtype, device=z.device).transpose(0, 1), cols, b * cols
    return _empty(stream, (b, t, cols), dtype=z.dtype, device=z.device), t * cols, cols


def _states_of(h, b, d, name):
    if h is not None and (h.dtype != torch.float32 or tuple(h.shape) != (b, d) or not h.is_contiguous()):
        raise ValueError("%s must be a contiguous float32 tensor of %d x %d" % (name, b, d))


def gated_scan_workspace_bytes(op, b, t, d) -> int:
    """Workspace of gated_scan_fwd (op 0) or gated_scan_bwd (op 1)."""
    return load().tfk_gated_scan_workspace_bytes(operator.index(op), operator.index(b), operator.index(t),
                                                 _width(operator.index(d), "z"))


_scan_need = functools.lru_cache(_KEPT)(gated_scan_workspace_bytes)


def _scan_ws(op, b, t, d, ws, device, stream):
    need = _scan_need(op, b, t, d)
    if ws is not None and not ws.is_contiguous():
        raise ValueError("ws must be contiguous")
    if need and (ws is None or ws.numel() * ws.element_size() < need):
        ws = _ws(need, device, stream)
    return ws, need


def gated_scan_fwd(z, output_gate=False, bias=None, h0=None, lengths=None, y=None, save=False, ws=None, stream=None):
    """Gated linear recurrence over sequences: with x, a (and o, with output_gate) the column blocks of z + bias
    (b x t x 2 d or 3 d; sequence or token first) and s the logistic function,
    h_t = s(a_t) h_(t-1) + (1 - s(a_t)) x_t from h0 (b x d fp32, default 0), y_t = h_t or s(o_t) h_t.
    lengths (int32): tokens of each sequence, the rest is padding (y is 0 there).
    Returns (y, the last states, the saved states for gated_scan_bwd, or None without save)."""
    gates, b, t, d, zb, zt = _scan_args(z, output_gate, bias, lengths)
    _states_of(h0, b, d, "h0")
    dt = _dt(z)
    if y is not None and (tuple(y.shape) != (b, t, d) or y.dtype != z.dtype):
        raise ValueError("y must be %s of z's type" % ((b, t, d),))
    st = _on_device(stream, z, bias, h0, lengths, y, ws)
    if y is None:
        y, yb, yt = _like_seqs(stream, z, d, zb, zt)
    else:
        yb, yt = _seqs(y, "y", d)[3:]
    last = _empty(stream, (b, d), dtype=torch.float32, device=z.device)
    states = None
    if save:
        states = _empty(stream, (b, (t + SCAN_BLOCK - 1) // SCAN_BLOCK, d), dtype=torch.float32, device=z.device)
    ws, need = _scan_ws(0, b, t, d, ws, z.device, stream)
    check(load().tfk_gated_scan_fwd(_ptr(z), dt, b, t, d, gates, zb, zt, _ptr(bias), _ptr(h0), _ptr(lengths), _ptr(y), yb, yt,
                                    _ptr(last), _ptr(states), _ptr(ws), need, st))
    return y, last, states


def gated_scan_bwd(z, dy, states, output_gate=False, bias=None, lengths=None, dh_last=None, dz=None, ws=None, stream=None):
    """Gradient of gated_scan_fwd for dy (of y) and dh_last (of the last states, default 0), with the states that
    call saved.  dz may be z (in place).  Returns (dz, the gradient of h0); the bias's gradient is dz's
    column sums (bias_relu_bwd without y)."""
    gates, b, t, d, zb, zt = _scan_args(z, output_gate, bias, lengths)
    dt = _dt(z)
    if tuple(dy.shape) != (b, t, d) or dy.dtype != z.dtype:
        raise ValueError("dy must be %s of z's type" % ((b, t, d),))
    yb, yt = _seqs(dy, "dy", d)[3:]
    _states_of(dh_last, b, d, "dh_last")
    blocks = (t + SCAN_BLOCK - 1) // SCAN_BLOCK
    if states.dtype != torch.float32 or tuple(states.shape) != (b, blocks, d) or not states.is_contiguous():
        raise ValueError("states must be a contiguous float32 tensor of %d x %d x %d" % (b, blocks, d))
    if dz is not None and (dz.shape != z.shape or dz.dtype != z.dtype):
        raise ValueError("dz must have z's shape and type")
    st = _on_device(stream, z, dy, states, bias, lengths, dh_last, dz, ws)
    if dz is None:
        dz, gb, gt = _like_seqs(stream, z, gates * d, zb, zt)
    else:
        gb, gt = (zb, zt) if dz is z else _seqs(dz, "dz")[3:]
    dh0 = _empty(stream, (b, d), dtype=torch.float32, device=z.device)
    ws, need = _scan_ws(1, b, t, d, ws, z.device, stream)
    check(load().tfk_gated_scan_bwd(_ptr(z), dt, b, t, d, gates, zb, zt, _ptr(bias), _ptr(lengths), _ptr(dy), yb, yt,
                                    _ptr(states), _ptr(dh_last), _ptr(dz), gb, gt, _ptr(dh0), _ptr(ws), need, st))
    return dz, dh0


def gated_scan_step(z, state, slots=None, output_gate=False, bias=None, y=None, stream=None):
    """One token of each of n sequences: z (n x 2 d or 3 d) moves the states of their slots (int32, distinct; one
    outside the states is none, and y's row 0; default row i has slot i) in state (slots x d fp32) in
    place.  Returns y (n x d)."""
    gates = 3 if output_gate else 2
    if z.dim() != 2:
        raise ValueError("z must be rows x columns, got shape %s" % (tuple(z.shape),))
    n, cols, ld = _rows_of(z, "z")
    if cols % gates:
        raise ValueError("z must have %d columns for each channel, got %d" % (gates, cols))
    d = cols // gates
    if state.dim() != 2 or state.dtype != torch.float32 or state.shape[1] != d or not state.is_contiguous():
        raise ValueError("state must be a contiguous float32 tensor of slots x %d" % d)
    _vector(bias, torch.float32, cols, "bias")
    _vector(slots, torch.int32, n, "slots")
    dt = _dt(z)
    yld = d
    if y is not None:
        if tuple(y.shape) != (n, d) or y.dtype != z.dtype:
            raise ValueError("y must be %s of z's type" % ((n, d),))
        yld = _rows_of(y, "y")[2]
    st = _on_device(stream, z, state, slots, bias, y)
    if y is None:
        y = _empty(stream, (n, d), dtype=z.dtype, device=z.device)
    check(load().tfk_gated_scan_step(_ptr(z), dt, n, d, gates, ld, _ptr(bias), _ptr(slots), _ptr(state), state.shape[0],
                                     _ptr(y), yld, st))
    return y


# ----------------------------------------------------------------------------- streams and programs
def stream_wait(waiter, producer):
    """Work enqueued on ``waiter`` afterwards waits for everything enqueued on ``producer`` so far
    (an event join inside the library; recorded into a program like the ops)."""
    check(load().tfk_stream_wait(ctypes.c_void_p(waiter.cuda_stream), ctypes.c_void_p(producer.cuda_stream)))


class Mark:
    """A point on one stream that other streams can wait for (``record`` then ``wait``): unlike
    ``stream_wait``, work the producer enqueues after ``record`` is not waited for.  Recorded
    into programs like the ops; a mark must outlive every program that uses it."""

    def __init__(self):
        self._lib = load()
        h = ctypes.c_void_p()
        check(self._lib.tfk_mark_create(ctypes.byref(h)))
        self._h = h

    def record(self, stream):
        check(self._lib.tfk_mark_record(self._h, ctypes.c_void_p(stream.cuda_stream)))

    def wait(self, waiter):
        """Work enqueued on ``waiter`` afterwards starts once the latest ``record`` is reached."""
        check(self._lib.tfk_stream_wait_mark(ctypes.c_void_p(waiter.cuda_stream), self._h))

    def close(self):
        if self._h is not None and self._h.value:
            self._lib.tfk_mark_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Program:
    """A recorded sequence of library calls, issued again from C++ by ``run()``.

    ``with prog.recording(): ...`` runs the calls made inside the block as usual and records
    each one that succeeds (same pointers, shapes, scalars and streams); ``run()`` enqueues them
    again in order.  Buffers the caller gave them must stay allocated while the program is used;
    results and workspaces that the calls made themselves are kept with it."""

    def __init__(self):
        self._lib = load()
        h = ctypes.c_void_p()
        check(self._lib.tfk_program_create(ctypes.byref(h)))
        self._h = h
        self.kept = []

    def recording(self):
        prog = self

        class _Rec:
            def __enter__(self):
                check(prog._lib.tfk_program_begin(prog._h))
                prog.kept = []
                _recording.program = prog
                return prog

            def __exit__(self, *exc):
                _recording.program = None
                check(prog._lib.tfk_program_end(prog._h))
                return False

        return _Rec()

    def __len__(self) -> int:
        return int(self._lib.tfk_program_length(self._h))

    def run(self):
        check(self._lib.tfk_program_run(self._h))

    def close(self):
        if self._h is not None and self._h.value:
            self._lib.tfk_program_destroy(self._h)
        self._h = None
        self.kept = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
