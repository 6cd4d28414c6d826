"""Refusals of the recurrence, the log-probabilities and AdamW, at the C ABI (fake addresses, never dereferenced) and in
the Python binding (CPU tensors): nothing here reaches a GPU."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1605_08695_amd import _lib, ops
from paper_1605_08695_amd.optim import AdamW
from paper_1605_08695_amd.recurrent import GatedRecurrence

F32, BF16 = 0, 1
OK, NULL, SHAPE, DTYPE, ALIGN, OVERFLOW, ALIAS, WORKSPACE, HIP, ARG = range(10)
P = 0x10000000
M = 0x100000
NAN, INF = float("nan"), float("inf")
f = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def vp(a):
    return ctypes.c_void_p(a) if a else None


# ----------------------------------------------------------------------------- log-probabilities
_ROWS = [(dict(dt=7), DTYPE), (dict(n=-1), SHAPE), (dict(c=0), SHAPE), (dict(ld=99), SHAPE), (dict(T=0.0), ARG),
         (dict(T=NAN), ARG), (dict(T=1e5), ARG), (dict(n=1 << 31), OVERFLOW), (dict(n=1 << 30, ld=1 << 11), OVERFLOW),
         (dict(c=(1 << 30) + 1, n=1), OVERFLOW), (dict(z=0), NULL), (dict(z=P + 2), ALIGN), (dict(bias=P + M + 1), ALIGN),
         (dict(tokens=P + 2 * M + 2), ALIGN)]


@pytest.mark.parametrize("kw,status", _ROWS + [
    (dict(k=-1), SHAPE), (dict(k=129), SHAPE), (dict(tokens=0), NULL), (dict(idx=0), NULL), (dict(top=0), NULL),
    (dict(logp=P + 3 * M + 2), ALIGN), (dict(ent=P + 4 * M + 1), ALIGN), (dict(lse=P + 5 * M + 2), ALIGN),
    (dict(idx=P + 6 * M + 2), ALIGN), (dict(top=P + 7 * M + 1), ALIGN), (dict(logp=P), ALIAS), (dict(ent=P + M), ALIAS),
    (dict(lse=P + 2 * M), ALIAS), (dict(idx=P + 7 * M), ALIAS), (dict(ent=P + 5 * M), ALIAS),
    (dict(c=1 << 17, n=2, ws=0), WORKSPACE), (dict(c=1 << 17, n=2, wb=64), WORKSPACE), (dict(c=1 << 17, n=2, ws=P + 9 * M + 8), ALIGN),
    (dict(c=1 << 17, n=2, ws=P + 16 * M), ALIAS), (dict(c=1 << 17, n=2, ws=P + 7 * M), ALIAS),
    (dict(n=0, z=0, tokens=0, logp=0, ent=0, lse=0, idx=0, top=0), OK)], ids=str)
def test_token_logprobs(lib, kw, status):
    a = dict(z=P, dt=F32, n=4, c=100, ld=0, bias=P + M, tokens=P + 2 * M, T=1.0, k=5, logp=P + 3 * M, ent=P + 4 * M,
             lse=P + 5 * M, idx=P + 6 * M, top=P + 7 * M, ws=P + 9 * M, wb=M)
    if kw.get("c", 0) > 100:
        a.update(z=P + 16 * M, bias=P + 11 * M)
    a.update(kw)
    assert lib.tfk_token_logprobs(vp(a["z"]), a["dt"], a["n"], a["c"], a["ld"], vp(a["bias"]), vp(a["tokens"]), f(a["T"]),
                                  a["k"], vp(a["logp"]), vp(a["ent"]), vp(a["lse"]), vp(a["idx"]), vp(a["top"]),
                                  vp(a["ws"]), a["wb"], None) == status


@pytest.mark.parametrize("kw,status", _ROWS + [
    (dict(dld=99), SHAPE), (dict(tokens=0), NULL), (dict(lse=0), NULL), (dict(dlogp=0), NULL), (dict(ent=0), NULL),
    (dict(dz=0), NULL), (dict(dz=P + 3 * M + 2), ALIGN), (dict(lse=P + 4 * M + 1), ALIGN), (dict(dlogp=P + 6 * M + 2), ALIGN),
    (dict(dent=P + 7 * M + 2), ALIGN), (dict(ent=P + 5 * M + 2), ALIGN), (dict(dz=P + 4), ALIAS), (dict(dz=P, dld=128), ALIAS),
    (dict(dz=P + M), ALIAS), (dict(dz=P + 4 * M), ALIAS), (dict(dz=P + 6 * M), ALIAS),
    (dict(n=0, z=0, tokens=0, lse=0, dlogp=0, ent=0, dent=0, dz=0), OK)], ids=str)
def test_token_logprobs_bwd(lib, kw, status):
    a = dict(z=P, dt=F32, n=4, c=100, ld=0, bias=P + M, tokens=P + 2 * M, T=1.0, lse=P + 4 * M, ent=P + 5 * M, dlogp=P + 6 * M,
             dent=P + 7 * M, dz=P + 3 * M, dld=0)
    a.update(kw)
    assert lib.tfk_token_logprobs_bwd(vp(a["z"]), a["dt"], a["n"], a["c"], a["ld"], vp(a["bias"]), vp(a["tokens"]), f(a["T"]),
                                      vp(a["lse"]), vp(a["ent"]), vp(a["dlogp"]), vp(a["dent"]), vp(a["dz"]), a["dld"],
                                      None) == status


# ----------------------------------------------------------------------------- recurrence
_SCAN = [(dict(dt=7), DTYPE), (dict(b=-1), SHAPE), (dict(t=-1), SHAPE), (dict(d=0), SHAPE), (dict(gates=1), ARG),
         (dict(gates=4), ARG), (dict(b=1 << 31), OVERFLOW), (dict(t=1 << 30), OVERFLOW), (dict(d=(1 << 24) + 1), OVERFLOW),
         (dict(b=1 << 20, t=1 << 20, d=8), OVERFLOW), (dict(zt=-8), OVERFLOW), (dict(zt=(1 << 25) + 1), OVERFLOW), (dict(yt=1 << 27), OVERFLOW), (dict(zb=-8, zt=0), OVERFLOW),
         (dict(zt=23, zb=24), SHAPE), (dict(zt=24, zb=30), SHAPE), (dict(zb=24, zt=24), SHAPE), (dict(yt=7, yb=100), SHAPE),
         (dict(z=0), NULL), (dict(z=P + 2), ALIGN), (dict(bias=P + 2 * M + 2), ALIGN), (dict(lengths=P + 3 * M + 1), ALIGN)]


@pytest.mark.parametrize("kw,status", _SCAN + [
    (dict(y=0), NULL), (dict(y=P + M + 1), ALIGN), (dict(h0=P + 4 * M + 2), ALIGN), (dict(last=P + 5 * M + 2), ALIGN),
    (dict(states=P + 6 * M + 2), ALIGN), (dict(y=P + 16), ALIAS), (dict(last=P + 4 * M), ALIAS), (dict(last=P + M), ALIAS),
    (dict(states=P + 2 * M), ALIAS), (dict(y=P + 3 * M), ALIAS), (dict(last=P + 6 * M), ALIAS),
    (dict(b=0, z=0, y=0, last=0, states=0), OK), (dict(t=0, z=0, y=0, last=0, states=0, h0=0), OK)], ids=str)
def test_gated_scan_fwd(lib, kw, status):
    a = dict(z=P, dt=F32, b=3, t=5, d=8, gates=3, zb=0, zt=0, bias=P + 2 * M, h0=P + 4 * M, lengths=P + 3 * M, y=P + M, yb=0, yt=0,
             last=P + 5 * M, states=P + 6 * M, ws=P + 8 * M, wb=1 << 30)
    a.update(kw)
    assert lib.tfk_gated_scan_fwd(vp(a["z"]), a["dt"], a["b"], a["t"], a["d"], a["gates"], a["zb"], a["zt"], vp(a["bias"]),
                                  vp(a["h0"]), vp(a["lengths"]), vp(a["y"]), a["yb"], a["yt"], vp(a["last"]), vp(a["states"]),
                                  vp(a["ws"]), a["wb"], None) == status


@pytest.mark.parametrize("kw,status", _SCAN + [
    (dict(dy=0), NULL), (dict(dz=0), NULL), (dict(states=0), NULL), (dict(dy=P + M + 1), ALIGN), (dict(dz=P + 5 * M + 2), ALIGN),
    (dict(states=P + 6 * M + 2), ALIGN), (dict(dh=P + 4 * M + 2), ALIGN), (dict(dh0=P + 7 * M + 2), ALIGN),
    (dict(dz=P + 16), ALIAS), (dict(dz=P, gt=32, gb=160), ALIAS), (dict(dz=P + M), ALIAS), (dict(dz=P + 6 * M), ALIAS),
    (dict(dh0=P + 4 * M), ALIAS), (dict(dh0=P + 5 * M), ALIAS), (dict(dh0=P + 2 * M), ALIAS), (dict(gt=20, gb=500), SHAPE),
    (dict(b=0, z=0, dy=0, dz=0, states=0, dh0=0), OK), (dict(t=0, z=0, dy=0, dz=0, states=0, dh0=0), OK)], ids=str)
def test_gated_scan_bwd(lib, kw, status):
    a = dict(z=P, dt=F32, b=3, t=5, d=8, gates=3, zb=0, zt=0, bias=P + 2 * M, lengths=P + 3 * M, dy=P + M, yb=0, yt=0,
             states=P + 6 * M, dh=P + 4 * M, dz=P + 5 * M, gb=0, gt=0, dh0=P + 7 * M, ws=P + 8 * M, wb=1 << 30)
    a.update(kw)
    assert lib.tfk_gated_scan_bwd(vp(a["z"]), a["dt"], a["b"], a["t"], a["d"], a["gates"], a["zb"], a["zt"], vp(a["bias"]),
                                  vp(a["lengths"]), vp(a["dy"]), a["yb"], a["yt"], vp(a["states"]), vp(a["dh"]), vp(a["dz"]),
                                  a["gb"], a["gt"], vp(a["dh0"]), vp(a["ws"]), a["wb"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=7), DTYPE), (dict(n=-1), SHAPE), (dict(d=0), SHAPE), (dict(gates=1), ARG), (dict(ld=23), SHAPE), (dict(yld=7), SHAPE),
    (dict(slots_n=-1), SHAPE), (dict(slots=0, slots_n=3), SHAPE), (dict(slots_n=1 << 31), OVERFLOW), (dict(n=1 << 31), OVERFLOW),
    (dict(z=0), NULL), (dict(y=0), NULL), (dict(state=0), NULL), (dict(z=P + 2), ALIGN), (dict(y=P + M + 2), ALIGN),
    (dict(state=P + 2 * M + 2), ALIGN), (dict(bias=P + 3 * M + 2), ALIGN), (dict(slots=P + 4 * M + 2), ALIGN), (dict(y=P), ALIAS),
    (dict(state=P + 16), ALIAS), (dict(y=P + 2 * M), ALIAS), (dict(state=P + 4 * M), ALIAS), (dict(y=P + 3 * M), ALIAS),
    (dict(n=0, z=0, y=0, state=0, slots=0), OK)], ids=str)
def test_gated_scan_step(lib, kw, status):
    a = dict(z=P, dt=F32, n=4, d=8, gates=3, ld=0, bias=P + 3 * M, slots=P + 4 * M, state=P + 2 * M, slots_n=10, y=P + M, yld=0)
    a.update(kw)
    assert lib.tfk_gated_scan_step(vp(a["z"]), a["dt"], a["n"], a["d"], a["gates"], a["ld"], vp(a["bias"]), vp(a["slots"]),
                                   vp(a["state"]), a["slots_n"], vp(a["y"]), a["yld"], None) == status


def test_logprob_workspace(lib):
    q = lib.tfk_token_logprobs_workspace_bytes
    assert q(0, 10, 1) == q(-1, 10, 1) == q(5, 0, 1) == q(5, 10, 129) == q(5, 10, -1) == q(1 << 31, 10, 1) == q(4, 1000, 5) == 0
    assert q(5000, 1 << 17, 20) == 0 and q(2, 1 << 17, 20) >= 2 * 2 * (20 * 8 + 12)


def test_gated_scan_workspace(lib):
    q = lib.tfk_gated_scan_workspace_bytes
    assert q(2, 1, 1, 1) == q(-1, 1, 1, 1) == q(0, 0, 5, 8) == q(0, 5, 0, 8) == q(1, -1, 5, 8) == q(1, 1 << 31, 5, 8) == 0
    # too little where some is needed
    for op, fn in ((0, "fwd"), (1, "bwd")):
        need = q(op, 1, 1 << 16, 64)
        if need:
            a = [vp(P), F32, 1, 1 << 16, 64, 2, 0, 0, None]
            a += [None, None, vp(P << 4), 0, 0, vp(P << 5), None] if op == 0 else [None, vp(P << 4), 0, 0, vp(P << 5), None,
                                                                                  vp(P << 6), 0, 0, None]
            call = lambda ws, n: getattr(lib, "tfk_gated_scan_" + fn)(*a, vp(ws), n, None)  # noqa: E731
            assert call(0, need) == WORKSPACE and call(P << 7, need - 1) == WORKSPACE and call((P << 7) + 8, need) == ALIGN
            assert call(P, need) == ALIAS


# ----------------------------------------------------------------------------- AdamW
@pytest.mark.parametrize("kw,status", [
    (dict(count=-1), ARG), (dict(bits=16), ARG), (dict(lr=NAN), ARG), (dict(b1=1.0), ARG), (dict(b1=-0.1), ARG), (dict(b2=NAN), ARG),
    (dict(eps=-1.0), ARG), (dict(eps=INF), ARG), (dict(t=0), ARG), (dict(lr=1e38, b1=0.999999999), OVERFLOW),
    (dict(wd=[0.1, -1.0]), ARG), (dict(wd=[NAN, 0.0]), ARG), (dict(wd=[1e38, 0.0], lr=10.0), ARG), (dict(n=[100, -1]), SHAPE),
    (dict(n=[(1 << 38) + 1, 1]), OVERFLOW), (dict(var=[0, P + M]), NULL), (dict(m=[P + 2 * M, 0]), NULL), (dict(v=[0, P]), NULL),
    (dict(g=[0, P]), NULL), (dict(mc=[0, P]), NULL), (dict(mc=None), NULL), (dict(vc=None), NULL), (dict(var=None), NULL),
    (dict(g=None), NULL), (dict(n=None), NULL), (dict(var=[P + 2, P + M]), ALIGN), (dict(g=[P + 6 * M + 1, P + 7 * M]), ALIGN),
    (dict(mc=[P + 8 * M + 2, P + 9 * M]), ALIGN), (dict(sh=[P + 12 * M + 1, 0]), ALIGN), (dict(bits=32, m=[P + 2 * M + 2, P + 3 * M]), ALIGN),
    (dict(m=[P + 4, P + 3 * M]), ALIAS), (dict(v=[P + 2 * M + 50, P + 5 * M]), ALIAS), (dict(sh=[P + 396, 0]), ALIAS),
    (dict(g=[P, P + 7 * M]), ALIAS), (dict(mc=[P + 10 * M, P + 9 * M]), ALIAS), (dict(var=[P, P + 396]), ALIAS),
    (dict(var=[P, P]), ALIAS), (dict(var=[P + 8, P]), ALIAS), (dict(n=[0, 0], var=[0, 0], m=[0, 0], v=[0, 0], g=[0, 0], mc=[0, 0], vc=[0, 0]), OK),
    (dict(count=0, var=None, m=None, v=None, g=None, n=None), OK)], ids=str)
def test_apply_adamw_multi(lib, kw, status):
    a = dict(count=2, bits=8, var=[P, P + M], m=[P + 2 * M, P + 3 * M], v=[P + 4 * M, P + 5 * M], g=[P + 6 * M, P + 7 * M],
             mc=[P + 8 * M, P + 9 * M], vc=[P + 10 * M, P + 11 * M], n=[100, 50], wd=[0.1, 0.0], lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, t=1,
             sh=[P + 12 * M, 0])
    a.update(kw)
    ptrs = lambda x: None if x is None else (ctypes.c_void_p * 2)(*x)  # noqa: E731
    assert lib.tfk_apply_adamw_multi(
        a["count"], a["bits"], ptrs(a["var"]), ptrs(a["m"]), ptrs(a["v"]), ptrs(a["mc"]), ptrs(a["vc"]), ptrs(a["g"]),
        None if a["n"] is None else (ctypes.c_int64 * 2)(*a["n"]), (ctypes.c_double * 2)(*a["wd"]), a["lr"], a["b1"], a["b2"], a["eps"],
        a["t"], ptrs(a["sh"]), None) == status


# ----------------------------------------------------------------------------- the Python binding
def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


I32, F8 = torch.int32, torch.float8_e4m3fn
_S = torch.zeros(8)


def test_binding_refuses_host_tensors():
    z = _t(2, 3, 8)
    for call in (lambda: ops.token_logprobs(_t(3, 4)), lambda: ops.token_logprobs_bwd(_t(3, 4), _t(3, dtype=I32), _t(3), _t(3)),
                 lambda: ops.gated_scan_fwd(z), lambda: ops.gated_scan_bwd(z, _t(2, 3, 4), _t(2, 1, 4)),
                 lambda: ops.gated_scan_step(_t(3, 8), _t(3, 4)), lambda: AdamW([_t(4)], 0.1).step([_t(4)]),
                 lambda: ops.apply_adamw_multi([_t(4)], [_t(4)], [_t(4)], [_t(4)], 0.1, 0.9, 0.99, 0.0, 1)):
        with pytest.raises(ValueError, match="GPU"):
            call()


@pytest.mark.parametrize("call", [
    lambda: ops.token_logprobs(_t(3)), lambda: ops.token_logprobs(_t(4, 3).t()), lambda: ops.token_logprobs(_t(3, 0)),
    lambda: ops.token_logprobs(_t(3, 4), k=129), lambda: ops.token_logprobs(_t(3, 4), k=-1),
    lambda: ops.token_logprobs(_t(3, 4), tokens=_t(3)), lambda: ops.token_logprobs(_t(3, 4), tokens=_t(2, dtype=I32)),
    lambda: ops.token_logprobs(_t(3, 4), bias=_t(3)), lambda: ops.token_logprobs(_t(3, 4, dtype=torch.float16)),
    lambda: ops.token_logprobs_bwd(_t(3, 4), _t(3, dtype=I32), _t(3), _t(3), dentropy=_t(3)),
    lambda: ops.token_logprobs_bwd(_t(3, 4), _t(3, dtype=I32), _t(2), _t(3)),
    lambda: ops.token_logprobs_bwd(_t(3, 4), _t(3, dtype=I32), _t(3), _t(3), dlogits=_t(3, 5)),
    lambda: ops.token_logprobs_bwd(_t(3, 4), _t(3, dtype=I32), _t(3), _t(3), dlogits=_t(3, 4, dtype=torch.bfloat16)),
    lambda: ops.gated_scan_fwd(_t(3, 8)), lambda: ops.gated_scan_fwd(_t(2, 3, 7)), lambda: ops.gated_scan_fwd(_t(2, 3, 8), output_gate=True),
    lambda: ops.gated_scan_fwd(_t(2, 8, 3).transpose(1, 2)), lambda: ops.gated_scan_fwd(_t(1, 3, 8).expand(2, 3, 8)),
    lambda: ops.gated_scan_fwd(_t(2, 1, 8).expand(2, 3, 8)), lambda: ops.gated_scan_fwd(_t(2, 3, 8), bias=_t(4)),
    lambda: ops.gated_scan_fwd(_t(2, 3, 8), h0=_t(2, 5)), lambda: ops.gated_scan_fwd(_t(2, 3, 8), h0=_t(4, 2).t()),
    lambda: ops.gated_scan_fwd(_t(2, 3, 8), lengths=_t(3, dtype=I32)), lambda: ops.gated_scan_fwd(_t(2, 3, 8), y=_t(2, 3, 8)),
    lambda: ops.gated_scan_fwd(_t(2, 3, 8), y=_t(2, 3, 4, dtype=torch.bfloat16)), lambda: ops.gated_scan_fwd(_t(2, 3, 0)),
    lambda: ops.gated_scan_bwd(_t(2, 3, 8), _t(2, 3, 8), _t(2, 1, 4)), lambda: ops.gated_scan_bwd(_t(2, 3, 8), _t(2, 3, 4), _t(2, 2, 4)),
    lambda: ops.gated_scan_bwd(_t(2, 3, 8), _t(2, 3, 4), _t(2, 1, 4), dh_last=_t(2, 3)),
    lambda: ops.gated_scan_bwd(_t(2, 3, 8), _t(2, 3, 4), _t(2, 1, 4), dz=_t(2, 3, 4)),
    lambda: ops.gated_scan_step(_t(2, 3, 8), _t(3, 4)), lambda: ops.gated_scan_step(_t(2, 7), _t(3, 4)),
    lambda: ops.gated_scan_step(_t(2, 8), _t(3, 5)), lambda: ops.gated_scan_step(_t(2, 8), _t(3, 4, dtype=torch.bfloat16)),
    lambda: ops.gated_scan_step(_t(2, 8), _t(3, 4), slots=_t(3, dtype=I32)), lambda: ops.gated_scan_step(_t(2, 8), _t(3, 4), y=_t(2, 8)),
    lambda: AdamW([_t(4)], 0.1, bits=16), lambda: AdamW([_t(4, dtype=torch.bfloat16)], 0.1), lambda: AdamW([_t(4)], 0.1, weight_decay=[0.1, 0.2]),
    lambda: AdamW([_t(4)], 0.1, shadows=[_t(4)]), lambda: AdamW([_t(4, 4).t()], 0.1), lambda: AdamW([_t(4)], 0.1, bits=8, moments=([_t(4)], [_t(4)], None, None)),
    lambda: AdamW([_t(400)], 0.1, bits=8, moments=([_t(400, dtype=F8)], [_t(400, dtype=F8)], [_t(1)], [_t(2)])),
    lambda: AdamW([_S, _S], 0.1), lambda: AdamW([_S[:3], _S[2:]], 0.1), lambda: AdamW([_t(8)], 0.1, moments=([_S], [_S], None, None)),
    lambda: AdamW([_t(8), _t(8)], 0.1, moments=([_S, _t(8)], [_t(8), _S], None, None)), lambda: AdamW([_t(4)], 0.1).step([]), lambda: AdamW([_t(4)], 0.1).step([_t(5)]), lambda: AdamW([_t(4)], 0.1).step([_t(4, dtype=torch.bfloat16)]),
    lambda: ops.apply_adamw_multi([_t(4)], [_t(4)], [], [_t(4)], 0.1, 0.9, 0.99, 0.0, 1),
    lambda: GatedRecurrence(np.zeros((4, 7)), np.zeros(7), device="cpu"), lambda: GatedRecurrence(np.zeros((4, 6)), np.zeros(5), device="cpu"),
])
def test_binding_refuses(call):
    with pytest.raises((ValueError, TypeError)) as e:
        call()
    assert "GPU" not in str(e.value)


def test_binding_constants(lib):
    assert ops.SCAN_BLOCK == 16 and [ops.adamw_scales(n) for n in (0, 1, 256, 257)] == [0, 1, 1, 2]
    assert ops.gated_scan_workspace_bytes(0, 2, 3, 4) == lib.tfk_gated_scan_workspace_bytes(0, 2, 3, 4)
