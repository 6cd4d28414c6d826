"""Refusals of the embedding and distillation entry points, at the C ABI (fake addresses, never
dereferenced) and in the Python binding (CPU tensors): nothing here reaches a GPU."""
import ctypes

import pytest
import torch

from paper_1605_08695_amd import _lib, ops
from paper_1605_08695_amd.embedding import EmbeddingTable

F32, BF16 = 0, 1
OK, NULL, SHAPE, DTYPE, ALIGN, OVERFLOW, ALIAS, WORKSPACE, HIP, ARG = range(10)
P = 0x10000000
NAN, INF = float("nan"), float("inf")
f = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def vp(a):
    return ctypes.c_void_p(a) if a else None


@pytest.mark.parametrize("kw,status", [
    (dict(dt=7), DTYPE), (dict(odt=-1), DTYPE), (dict(n=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(d=0), SHAPE),
    (dict(tld=7), SHAPE), (dict(old=7), SHAPE), (dict(scale=NAN), ARG), (dict(scale=INF), ARG),
    (dict(n=1 << 31), OVERFLOW), (dict(rows=1 << 31), OVERFLOW), (dict(n=1 << 30, old=1 << 11), OVERFLOW),
    (dict(table=0), NULL), (dict(ids=0), NULL), (dict(out=0), NULL), (dict(table=P + 2), ALIGN),
    (dict(ids=P + 0x100002), ALIGN), (dict(out=P + 0x200001, odt=BF16), ALIGN), (dict(out=P + 100 * 32 - 4), ALIAS),
    (dict(out=P + 0x100000 + 36), ALIAS), (dict(n=0, table=0, ids=0, out=0), OK),
], ids=lambda v: str(v))
def test_embedding_fwd(lib, kw, status):
    a = dict(table=P, dt=F32, rows=100, tld=0, d=8, ids=P + 0x100000, n=10, scale=1.0, out=P + 0x200000, odt=F32, old=0)
    a.update(kw)
    assert lib.tfk_embedding_fwd(vp(a["table"]), a["dt"], a["rows"], a["tld"], a["d"], vp(a["ids"]), a["n"], f(a["scale"]),
                                 vp(a["out"]), a["odt"], a["old"], None) == status


_SUM = [
    (dict(dt=7), DTYPE), (dict(n=-1), SHAPE), (dict(rows=-1), SHAPE), (dict(d=0), SHAPE), (dict(ld=7), SHAPE),
    (dict(scale=NAN), ARG), (dict(n=1 << 31), OVERFLOW), (dict(rows=1 << 31), OVERFLOW), (dict(dy=0), NULL),
    (dict(ids=0), NULL), (dict(dst=0), NULL), (dict(dy=P + 0x100002), ALIGN), (dict(dst=P + 2), ALIGN),
    (dict(ids=P + 0x200002), ALIGN), (dict(ws=0), WORKSPACE), (dict(wb=8), WORKSPACE), (dict(ws=P + 0x300008), ALIGN),
    (dict(dy=P + 100 * 32 - 4), ALIAS), (dict(ids=P), ALIAS), (dict(ws=P + 16), ALIAS), (dict(ws=P + 0x100000), ALIAS),
    (dict(ws=P + 0x200000), ALIAS), (dict(rows=0, dst=0), OK), (dict(rows=0, n=0, dst=0, dy=0, ids=0, ws=0), OK),
]


def _sum_args(kw):
    a = dict(dy=P + 0x100000, dt=F32, n=10000, ld=0, d=8, ids=P + 0x200000, rows=100, scale=1.0, beta=0.0, dst=P, sh=0,
             lr=0.1, ws=P + 0x300000, wb=1 << 20)
    a.update(kw)
    return a


@pytest.mark.parametrize("kw,status", _SUM + [(dict(beta=0.5), ARG), (dict(beta=NAN), ARG),
                                              (dict(beta=1.0, n=0, dst=0, dy=0, ids=0, ws=0), OK),
                                              (dict(n=0, dst=0), NULL)], ids=lambda v: str(v))
def test_embedding_bwd(lib, kw, status):
    a = _sum_args(kw)
    assert lib.tfk_embedding_bwd(vp(a["dy"]), a["dt"], a["n"], a["ld"], a["d"], vp(a["ids"]), a["rows"], f(a["scale"]),
                                 f(a["beta"]), vp(a["dst"]), vp(a["ws"]), a["wb"], None) == status


@pytest.mark.parametrize("kw,status", _SUM + [(dict(lr=NAN), ARG), (dict(sh=P + 0x400001), ALIGN), (dict(sh=P + 64), ALIAS),
                                              (dict(sh=P + 0x100000), ALIAS), (dict(sh=P + 0x300000), ALIAS),
                                              (dict(n=0, dst=0, dy=0, ids=0, ws=0), OK)], ids=lambda v: str(v))
def test_embedding_apply_sgd(lib, kw, status):
    a = _sum_args(kw)
    assert lib.tfk_embedding_apply_sgd(vp(a["dst"]), vp(a["sh"]), a["rows"], a["d"], vp(a["ids"]), a["n"], vp(a["dy"]),
                                       a["dt"], a["ld"], f(a["scale"]), f(a["lr"]), vp(a["ws"]), a["wb"], None) == status


def test_embedding_workspace_bytes(lib):
    q = lib.tfk_embedding_workspace_bytes
    assert q(0, 8, 100) == q(-1, 8, 100) == q(10, 0, 100) == q(10, 8, 0) == q(1 << 31, 8, 100) == q(10, 8, 1 << 31) == 0
    assert q(10, 8, 100) == 0                                  # few tokens are sorted on chip
    assert q(10000, 8, 100) >= 80000 and q(1 << 30, 8, 100) >= 8 << 30


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), DTYPE), (dict(tdt=9), DTYPE), (dict(n=-1), SHAPE), (dict(c=0), SHAPE), (dict(k=0), SHAPE),
    (dict(k=1025), SHAPE), (dict(ld=99), SHAPE), (dict(dld=99), SHAPE), (dict(scale=INF), ARG), (dict(T=0.0), ARG),
    (dict(T=-1.0), ARG), (dict(T=NAN), ARG), (dict(T=1e5), ARG), (dict(alpha=0.0), ARG), (dict(alpha=1.5), ARG),
    (dict(alpha=NAN), ARG), (dict(alpha=0.5, labels=0), ARG), (dict(n=1 << 31), OVERFLOW), (dict(n=1 << 30, ld=1 << 11), OVERFLOW),
    (dict(c=(1 << 30) + 1, n=1), OVERFLOW), (dict(z=0), NULL), (dict(top=0), NULL), (dict(idx=0), NULL), (dict(loss=0), NULL), (dict(dz=0), NULL),
    (dict(z=P + 2), ALIGN), (dict(dz=P + 0x100002), ALIGN), (dict(top=P + 0x200002), ALIGN), (dict(idx=P + 0x210002), ALIGN),
    (dict(bias=P + 0x220001), ALIGN), (dict(lse=P + 0x230002), ALIGN), (dict(labels=P + 0x240002), ALIGN),
    (dict(weight=P + 0x250002), ALIGN), (dict(loss=P + 0x260002), ALIGN), (dict(dz=P + 4), ALIAS),
    (dict(dz=P, dld=128), ALIAS), (dict(dz=P + 0x200000), ALIAS), (dict(loss=P), ALIAS), (dict(loss=P + 0x100000), ALIAS),
    (dict(loss=P + 0x240000), ALIAS), (dict(loss=P + 0x210000), ALIAS),
    (dict(n=0, z=0, top=0, idx=0, loss=0, dz=0, bias=0, lse=0, labels=0, weight=0), OK),
], ids=lambda v: str(v))
def test_distill_xent(lib, kw, status):
    a = dict(z=P, dt=F32, n=4, c=100, ld=0, bias=P + 0x220000, top=P + 0x200000, tdt=F32, idx=P + 0x210000, k=5,
             lse=P + 0x230000, labels=P + 0x240000, weight=P + 0x250000, T=2.0, alpha=0.5, scale=1.0, loss=P + 0x260000,
             dz=P + 0x100000, dld=0)
    a.update(kw)
    assert lib.tfk_distill_xent(vp(a["z"]), a["dt"], a["n"], a["c"], a["ld"], vp(a["bias"]), vp(a["top"]), a["tdt"],
                                vp(a["idx"]), a["k"], vp(a["lse"]), vp(a["labels"]), vp(a["weight"]), f(a["T"]),
                                f(a["alpha"]), f(a["scale"]), vp(a["loss"]), vp(a["dz"]), a["dld"], None) == status


# ----------------------------------------------------------------------------- the Python binding
def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


I32 = torch.int32


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding_fwd(_t(10, 4), _t(3, dtype=I32))
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10)
    with pytest.raises(ValueError, match="GPU"):
        ops.embedding_apply_sgd(_t(10, 4), _t(3, dtype=I32), _t(3, 4), 0.1)
    with pytest.raises(ValueError, match="GPU"):
        ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0)


@pytest.mark.parametrize("call", [
    lambda: ops.embedding_fwd(_t(10, 4), _t(3, dtype=torch.int64)),
    lambda: ops.embedding_fwd(_t(10, 4), _t(6, dtype=I32)[::2]),
    lambda: ops.embedding_fwd(_t(10, 2, 2), _t(3, dtype=I32)),
    lambda: ops.embedding_fwd(_t(4, 10).t(), _t(3, dtype=I32)),
    lambda: ops.embedding_fwd(_t(1, 4).expand(10, 4), _t(3, dtype=I32)),
    lambda: ops.embedding_fwd(_t(10, 0), _t(3, dtype=I32)),
    lambda: ops.embedding_fwd(_t(10, 4), _t(3, dtype=I32), out=_t(3, 5)),
    lambda: ops.embedding_fwd(_t(10, 4), _t(3, dtype=I32), out=_t(4, 3).t()),
    lambda: ops.embedding_fwd(_t(10, 4), _t(3, dtype=I32), out=_t(3, 4), out_dtype=torch.bfloat16),
    lambda: ops.embedding_fwd(_t(10, 4), _t(1, dtype=I32)[0], out=_t(4, 2)[:, 0]),
    lambda: ops.embedding_bwd(_t(4, 2)[:, 0], _t(1, dtype=I32)[0], 10),
    lambda: ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10, ws=torch.zeros(64, 2, dtype=torch.uint8)[:, 0]),
    lambda: ops.embedding_bwd(_t(3, 4), _t(4, dtype=I32), 10),
    lambda: ops.embedding_bwd(_t(1, 4).expand(3, 4), _t(3, dtype=I32), 10),
    lambda: ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10, beta=1.0),
    lambda: ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10, dtable=_t(10, 5)),
    lambda: ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10, dtable=_t(10, 4, dtype=torch.bfloat16)),
    lambda: ops.embedding_apply_sgd(_t(10, 4, dtype=torch.bfloat16), _t(3, dtype=I32), _t(3, 4), 0.1),
    lambda: ops.embedding_apply_sgd(_t(10, 4), _t(3, dtype=I32), _t(3, 5), 0.1),
    lambda: ops.embedding_apply_sgd(_t(10, 4), _t(3, dtype=I32), _t(3, 4), 0.1, shadow=_t(10, 4)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=torch.int64), _t(3, 2), 1.0),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 3), 1.0),
    lambda: ops.distill_xent(_t(3, 8), _t(4, 2, dtype=I32), _t(4, 2), 1.0),
    lambda: ops.distill_xent(_t(3, 8), _t(2, 3, dtype=I32).t(), _t(2, 3).t(), 1.0),
    lambda: ops.distill_xent(_t(8, 3).t(), _t(3, 2, dtype=I32), _t(3, 2), 1.0),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, labels=_t(3, dtype=torch.int64)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, bias=_t(7)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, weight=_t(2)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, top_lse=_t(3, dtype=torch.bfloat16)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, dlogits=_t(3, 8, dtype=torch.bfloat16)),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2), 1.0, loss=_t(4)),
])
def test_binding_refuses(call):
    with pytest.raises(ValueError):
        call()


@pytest.mark.parametrize("call", [
    lambda: ops.embedding_fwd(_t(10, 4, dtype=torch.float16), _t(3, dtype=I32)),
    lambda: ops.embedding_bwd(_t(3, 4, dtype=torch.float64), _t(3, dtype=I32), 10),
    lambda: ops.embedding_bwd(_t(3, 4), _t(3, dtype=I32), 10.5),
    lambda: ops.distill_xent(_t(3, 8, dtype=torch.float16), _t(3, 2, dtype=I32), _t(3, 2), 1.0),
    lambda: ops.distill_xent(_t(3, 8), _t(3, 2, dtype=I32), _t(3, 2, dtype=torch.float64), 1.0),
])
def test_binding_refuses_types(call):
    with pytest.raises(TypeError):
        call()


def test_programs_record_the_calls(lib):
    """Calls without work enqueue nothing: they are recorded and run again like the others."""
    prog = ops.Program()
    with prog.recording():
        assert lib.tfk_embedding_fwd(None, F32, 10, 0, 8, None, 0, f(1), None, F32, 0, None) == OK
        assert lib.tfk_embedding_apply_sgd(None, None, 10, 8, None, 0, None, F32, 0, f(1), f(0.1), None, 0, None) == OK
        assert lib.tfk_embedding_bwd(None, F32, 0, 0, 8, None, 10, f(1), f(1), None, None, 0, None) == OK
        assert lib.tfk_embedding_bwd(None, F32, 0, 0, 8, None, 10, f(1), f(2), None, None, 0, None) == ARG
        assert lib.tfk_distill_xent(None, F32, 0, 10, 0, None, None, F32, None, 2, None, None, None, f(1), f(1), f(1), None,
                                    None, 0, None) == OK
    assert len(prog) == 4
    prog.run()
    prog.close()


def test_table_keeps_what_lookups_read():
    import numpy as np
    t = EmbeddingTable(np.linspace(-1, 1, 12).reshape(4, 3), lr=0.1, scale=2.0, device="cpu")
    assert t.W.dtype == torch.float32 and torch.equal(t.W, t.W_lp.float()) and (t.vocab, t.d) == (4, 3)


def test_embedding_columns(lib):
    """Sums of more columns than a launch's grid holds are refused; the lookup takes them."""
    a = _sum_args(dict(n=1, rows=1, d=(1 << 23) + 1, dst=1 << 32, dy=1 << 33, wb=0))
    assert lib.tfk_embedding_bwd(vp(a["dy"]), a["dt"], a["n"], a["ld"], a["d"], vp(a["ids"]), a["rows"], f(1.0), f(0.0),
                                 vp(a["dst"]), vp(a["ws"]), a["wb"], None) == OVERFLOW
    assert lib.tfk_embedding_apply_sgd(vp(a["dst"]), None, a["rows"], a["d"], vp(a["ids"]), a["n"], vp(a["dy"]), a["dt"],
                                       a["ld"], f(1.0), f(0.1), vp(a["ws"]), a["wb"], None) == OVERFLOW
    assert lib.tfk_embedding_workspace_bytes(100000, (1 << 23) + 1, 100) == 0
    assert lib.tfk_embedding_workspace_bytes(100000, 1 << 20, 100) > 0


def test_columns_past_32_bits():
    """Column counts are 32 bits at the C ABI: wider tensors are refused, not cut off."""
    c, one = (1 << 32) + 8, torch.zeros(1, dtype=torch.int32)
    wide = torch.empty((1, c), dtype=torch.bfloat16, device="meta")
    top = torch.zeros((1, 3))
    for call in (lambda: ops.distill_xent(wide, torch.zeros((1, 3), dtype=torch.int32), top, 1.0),
                 lambda: ops.distill_xent(torch.zeros(1, 8), torch.empty((1, c), dtype=torch.int32, device="meta"),
                                          torch.empty((1, c), device="meta"), 1.0),
                 lambda: ops.embedding_fwd(wide, one),
                 lambda: ops.embedding_bwd(wide, one, 4),
                 lambda: ops.embedding_bwd(wide[0], one[0], 4),
                 lambda: ops.embedding_apply_sgd(torch.empty((1, c), device="meta"), one, wide, 0.1),
                 lambda: ops.embedding_workspace_bytes(5, c, 4)):
        with pytest.raises(ValueError, match="columns"):
            call()
