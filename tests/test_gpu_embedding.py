"""The embedding table on the GPU: lookup, dense gradient and sparse update against float64, over
tables, widths, strides and token distributions where they can go wrong."""
import numpy as np
import pytest
import torch

from paper_1605_08695_amd import ops
from paper_1605_08695_amd.embedding import EmbeddingTable

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24                       # half a step of fp32, relative


def say(*a):
    print(*a, flush=True)


def f64(t):
    return t.detach().double()


def _tokens(rng, n, rows, kind):
    if kind == "zipf":
        ids = np.minimum((np.exp(rng.random(n) * np.log(rows + 1.0)) - 1).astype(np.int64), rows - 1)
    elif kind == "same":
        ids = np.full(n, rows // 2)
    elif kind == "distinct":
        ids = rng.permutation(rows)[:n] if n <= rows else rng.integers(0, rows, n)
    elif kind == "half":                 # half of them one word
        ids = rng.integers(0, rows, n)
        ids[rng.random(n) < 0.5] = rows - 1
    elif kind == "stride":               # rows a power of two apart
        ids = rng.integers(0, max(1, rows // 256), n) * 256 % rows
    else:                                # padding and ids outside the table among the others
        ids = rng.integers(0, rows, n)
        ids[rng.random(n) < 0.3] = -1
        ids[rng.random(n) < 0.1] = rows
        ids[::17] = 2 ** 31 - 1
        ids[5::31] = -2 ** 31
        if kind == "none":
            ids[:] = -1
    return torch.from_numpy(ids.astype(np.int32)).to(DEV)


def _strided(t, extra):
    """The same values with `extra` elements between rows, filled with NaN."""
    if not extra:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, 1:1 + t.shape[1]] = t
    return wide[:, 1:1 + t.shape[1]]


# ----------------------------------------------------------------------------- lookup
@pytest.mark.parametrize("tdt,odt", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("n,d,rows,kind,extra", [
    (1, 1, 1, "same", 0), (3, 7, 5, "bad", 0), (128, 512, 40000, "zipf", 0), (1000, 333, 2001, "bad", 0),
    (257, 64, 300, "zipf", 3), (64, 1030, 100, "bad", 5), (33, 4096, 50, "zipf", 8), (5, 16, 9, "none", 0),
    (4099, 24, 1000, "zipf", 0)])
def test_lookup(tdt, odt, n, d, rows, kind, extra):
    say("lookup", tdt, odt, n, d, rows, kind, extra)
    rng = np.random.default_rng(n + d)
    table = torch.from_numpy(rng.standard_normal((rows, d))).to(tdt).to(DEV)
    ids = _tokens(rng, n, rows, kind)
    scale = float(np.float32(np.sqrt(d)))
    out = _strided(torch.zeros(n, d, dtype=odt, device=DEV), extra)
    wide = out._base if extra else out
    before = wide.clone()
    got = ops.embedding_fwd(_strided(table, extra), ids, scale, out=out)
    torch.cuda.synchronize()
    # one fp32 product, rounded once more where the output is bf16: the same bits
    i = ids.long()
    ok = (i >= 0) & (i < rows)
    ref = (f64(table)[i.clamp(0, rows - 1)] * scale).float()
    ref[~ok] = 0
    assert torch.equal(got, ref.to(odt))
    if extra:                            # what lies between the rows stays
        keep = torch.ones_like(wide, dtype=torch.bool)
        keep[:, 1:1 + d] = False
        bits = torch.int32 if odt == F32 else torch.int16
        assert torch.equal(wide.view(bits)[keep], before.view(bits)[keep])


def test_lookup_shapes_and_defaults():
    t = torch.randn(50, 16, device=DEV)
    ids = torch.randint(0, 50, (4, 5), dtype=torch.int32, device=DEV)
    assert ops.embedding_fwd(t, ids).shape == (4, 5, 16)
    assert ops.embedding_fwd(t, ids, out_dtype=BF16).dtype == BF16
    assert torch.equal(ops.embedding_fwd(t, ids), t[ids.long()])
    one = torch.tensor(7, dtype=torch.int32, device=DEV)
    assert torch.equal(ops.embedding_fwd(t, one), t[7])
    assert ops.embedding_fwd(t, ids[:0]).shape == (0, 5, 16)
    assert torch.equal(ops.embedding_fwd(t[:0], ids), torch.zeros(4, 5, 16, device=DEV))
    torch.cuda.synchronize()


def test_lookup_offsets_past_32_bits():
    """A table and an output of more than 2^31 elements: rows at both ends of each."""
    d, rows = 4096, (1 << 19) + 9
    table = torch.zeros(rows, d, dtype=BF16, device=DEV)
    probe = [0, 1, (1 << 19) - 1, 1 << 19, rows - 1]
    for r in probe:
        table[r] = torch.arange(d, device=DEV).remainder(251).to(BF16) + r % 97
    n = rows
    ids = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    at = [0, 5, (1 << 19) - 1, 1 << 19, n - 1]
    for i, r in zip(at, probe):
        ids[i] = r
    out = ops.embedding_fwd(table, ids)
    torch.cuda.synchronize()
    for i, r in zip(at, probe):
        assert torch.equal(out[i], table[r])
    assert not out[6].any() and not out[n - 2].any()


# ----------------------------------------------------------------------------- sums
def _sums(dy, ids, rows):
    """Float64 sums of dy's rows by id, sums of their magnitudes, and tokens per row."""
    i = ids.reshape(-1).long()
    y = f64(dy).reshape(-1, dy.shape[-1])
    ok = (i >= 0) & (i < rows)
    s = torch.zeros(rows, dy.shape[-1], dtype=torch.float64, device=DEV).index_add_(0, i[ok], y[ok])
    a = torch.zeros_like(s).index_add_(0, i[ok], y[ok].abs())
    c = torch.bincount(i[ok], minlength=rows).double()[:, None]
    return s, a, c


# A sum of L fp32 terms in any order is off by at most (L - 1) half steps of the sum of magnitudes;
# the scaling adds one, and so does each later rounding.
def _sum_bound(a, c, scale):
    return (c + 1) * U * a * abs(scale) * (1 + 1e-4)


CASES = [
    (1, 1, 1, "same", 0), (1, 8, 3, "none", 0), (2, 5, 7, "same", 0), (37, 3, 11, "bad", 0), (64, 128, 64, "distinct", 0),
    (300, 33, 50, "zipf", 3), (1000, 64, 1, "same", 0), (2560, 512, 40000, "zipf", 0), (2049, 257, 700, "bad", 1),
    (4097, 96, 60000, "distinct", 0), (5000, 1000, 5000, "same", 0), (3000, 2056, 300, "zipf", 0), (777, 8200, 100, "zipf", 0),
    (20000, 40, 300000, "zipf", 0), (20011, 34, 1 << 20, "stride", 2), (70001, 64, 131072, "zipf", 0), (70000, 72, 9, "zipf", 8),
    (66000, 16, 3, "same", 0), (33333, 520, 33333, "bad", 0), (8192, 36, 491520, "zipf", 0), (8193, 130, 262144, "half", 0),
    (40000, 260, 262145, "half", 0), (300, 4, 3000000, "distinct", 0), (9000, 6, 2097152, "half", 0)]


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,rows,kind,extra", CASES)
def test_gradient(dt, n, d, rows, kind, extra):
    say("gradient", dt, n, d, rows, kind, extra)
    rng = np.random.default_rng(n + d)
    ids = _tokens(rng, n, rows, kind)
    dy = _strided(torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(dt).to(DEV), extra)
    scale = float(np.float32(0.37))
    s, a, c = _sums(dy, ids, rows)
    bound = _sum_bound(a, c, scale)
    got = torch.full((rows, d), float("nan"), device=DEV)
    ops.embedding_bwd(dy, ids, rows, scale, dtable=got)
    got2 = ops.embedding_bwd(dy, ids, rows, scale)
    old = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(DEV)
    added = ops.embedding_bwd(dy, ids, rows, scale, dtable=old.clone(), beta=1.0)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int32), got2.view(torch.int32))       # the same bits every time
    assert torch.all((f64(got) - scale * s).abs() <= bound)
    ref = f64(old) + scale * s
    assert torch.all((f64(added) - ref).abs() <= bound + U * ref.abs() * (1 + 1e-4))
    none = (c[:, 0] == 0)
    assert not got[none].any() and torch.equal(added[none], old[none])


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shadow", [True, False])
@pytest.mark.parametrize("n,d,rows,kind,extra", CASES)
def test_update(dt, shadow, n, d, rows, kind, extra):
    say("update", dt, shadow, n, d, rows, kind, extra)
    rng = np.random.default_rng(n + d + 1)
    ids = _tokens(rng, n, rows, kind)
    dy = _strided(torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(dt).to(DEV), extra)
    W = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(DEV)
    sh = torch.full((rows, d), 7.0, dtype=BF16, device=DEV) if shadow else None
    W0 = W.clone()
    scale, lr = float(np.float32(1.7)), float(np.float32(0.05))
    assert ops.embedding_apply_sgd(W, ids, dy, lr, scale, shadow=sh) is W
    torch.cuda.synchronize()
    s, a, c = _sums(dy, ids, rows)
    ref = f64(W0) - lr * scale * s
    assert torch.all((f64(W) - ref).abs() <= lr * _sum_bound(a, c, scale) + U * ref.abs() * (1 + 1e-4))
    none = c[:, 0] == 0
    assert torch.equal(W[none], W0[none])
    if shadow:
        assert torch.equal(sh[~none], W[~none].to(BF16)) and torch.all(sh[none] == 7.0)


@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,d,rows,kind,extra", [(127, 512, 900, "same", 0), (129, 200, 900, "same", 1), (4000, 64, 700, "half", 0),
                                                 (8192, 512, 30000, "same", 0), (8000, 250, 5000, "half", 3),
                                                 (6001, 1030, 2000, "half", 0), (8191, 7, 40, "half", 0)])
def test_frequent_rows_of_few_tokens(dt, n, d, rows, kind, extra):
    test_gradient(dt, n, d, rows, kind, extra)
    test_update(dt, True, n, d, rows, kind, extra)


@pytest.mark.parametrize("n", [4096, 9000])
def test_gradient_offsets_past_32_bits(n):
    """dy's rows spread over more than 2^32 bytes and elements, and a table of more than 2^31 elements."""
    d, rows, ld = 64, (1 << 25) + 9, (1 << 32) // n + 5
    free = torch.cuda.mem_get_info()[0]
    if free < n * ld * 2 + 3 * rows * d * 4:
        pytest.skip("needs %d GB" % ((n * ld * 2 + 3 * rows * d * 4) >> 30))
    rng = np.random.default_rng(n)
    wide = torch.zeros(n, ld, dtype=BF16, device=DEV)
    dy = wide[:, 3:3 + d]
    dy.copy_(torch.from_numpy(rng.integers(-4, 5, (n, d)).astype(np.float32)))      # (sums of whole numbers are exact)
    names = np.array([0, 1, 77, (1 << 25) - 1, 1 << 25, rows - 1])
    ids = names[rng.integers(0, len(names), n)]
    ids[n - 1], ids[0] = rows - 1, 0
    ids_ = torch.from_numpy(ids.astype(np.int32)).to(DEV)
    got = ops.embedding_bwd(dy, ids_, rows)
    W = torch.ones(rows, d, device=DEV)
    ops.embedding_apply_sgd(W, ids_, dy, 0.5)
    torch.cuda.synchronize()
    vals = dy.float().cpu().numpy().astype(np.float64)
    for r in names:
        s = vals[ids == r].sum(0)
        assert np.array_equal(got[int(r)].cpu().numpy(), s.astype(np.float32))
        assert np.array_equal(W[int(r)].cpu().numpy(), (1 - 0.5 * s).astype(np.float32))
        got[int(r)] = 0
        W[int(r)] = 1
    assert not got.any() and bool((W == 1).all())


@pytest.mark.parametrize("n", [500, 40000])
def test_gradient_of_the_lookup(n):
    """<dy, lookup(W + E) - lookup(W)> = <gradient, E>: the lookup is linear in the table."""
    rows, d, scale = 3000, 48, 1.5
    rng = np.random.default_rng(3)
    ids = _tokens(rng, n, rows, "bad")
    W, E = (torch.from_numpy(rng.integers(-8, 9, (rows, d)).astype(np.float32)).to(DEV) for _ in range(2))
    dy = torch.from_numpy(rng.integers(-4, 5, (n, d)).astype(np.float32)).to(DEV)
    up = f64(ops.embedding_fwd(W + E, ids, scale)) - f64(ops.embedding_fwd(W, ids, scale))
    g = ops.embedding_bwd(dy, ids, rows, scale)
    assert float((f64(dy) * up).sum()) == float((f64(g) * f64(E)).sum())      # small integers: exact


def test_empty_and_special_values():
    dy = torch.randn(3, 4, device=DEV)
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    g = torch.full((5, 4), float("nan"), device=DEV)
    ops.embedding_bwd(dy[:0], none, 5, dtable=g)
    assert torch.equal(g, torch.zeros_like(g))
    ops.embedding_bwd(dy[:0], none, 5, dtable=g.fill_(2.0), beta=1.0)
    assert torch.all(g == 2.0)
    assert ops.embedding_bwd(dy, torch.zeros(3, dtype=torch.int32, device=DEV), 0).shape == (0, 4)
    W = torch.ones(5, 4, device=DEV)
    ops.embedding_apply_sgd(W, none, dy[:0], 0.1)
    assert torch.all(W == 1.0)
    # NaN and infinities stay in their rows, and out of them where the token is padding
    ids = torch.tensor([1, -1, 3, 1], dtype=torch.int32, device=DEV)
    y = torch.ones(4, 4, device=DEV)
    y[1] = float("nan")
    y[2, 2] = float("inf")
    g = ops.embedding_bwd(y, ids, 5)
    want = torch.zeros(5, 4)
    want[1] = 2
    want[3] = 1
    want[3, 2] = float("inf")
    assert torch.equal(g.cpu(), want)
    # a single token's denormals come through
    y = torch.full((1, 4), 1e-40, device=DEV)
    assert torch.equal(ops.embedding_bwd(y, ids[:1], 5)[1], y[0])


def test_other_stream_and_workspace():
    n, d, rows = 30000, 96, 1000
    rng = np.random.default_rng(8)
    ids = _tokens(rng, n, rows, "zipf")
    dy = torch.randn(n, d, device=DEV)
    ref = ops.embedding_bwd(dy, ids, rows)
    need = ops.embedding_workspace_bytes(n, d, rows)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.embedding_bwd(dy, ids, rows, stream=side, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, ref)
    assert torch.all(ws[need:] == 0xA5)                       # nothing behind the workspace is written


@pytest.mark.parametrize("n", [600, 30000])
def test_two_calls_at_once(n):
    """Two updates and their lookups on two streams, each with a workspace of its own."""
    d, rows = 192, 5000
    rng = np.random.default_rng(12)
    jobs = []
    for kind in ("zipf", "bad"):
        ids = _tokens(rng, n, rows, kind)
        W = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(DEV)
        dy = torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(BF16).to(DEV)
        want = W.clone()
        ops.embedding_apply_sgd(want, ids, dy, 0.1)
        jobs.append((ids, W, dy, want, ops.embedding_fwd(want, ids, 3.0), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for ids, W, dy, _, _, st in jobs:
            W0 = W.clone()
            st.wait_stream(torch.cuda.current_stream())
            ops.embedding_apply_sgd(W0, ids, dy, 0.1, stream=st)
            got.append((W0, ops.embedding_fwd(W0, ids, 3.0, stream=st)))
            W0.record_stream(st)
    torch.cuda.synchronize()
    for i, (W0, y) in enumerate(got):
        assert torch.equal(W0, jobs[i % 2][3]) and torch.equal(y, jobs[i % 2][4])


@pytest.mark.parametrize("n,rows", [(700, 300), (50000, 3000)])
def test_captured_and_recorded(n, rows):
    """One program and one graph of lookup, gradient and update, run again with new tokens, with eager
    work between the runs."""
    d = 72
    rng = np.random.default_rng(9)
    table = EmbeddingTable(rng.standard_normal((rows, d)), lr=0.5, scale=2.0)
    start = table.W.clone()
    ids = _tokens(rng, n, rows, "bad")
    dy = torch.randn(n, d, device=DEV).to(BF16)
    dW = torch.zeros(rows, d, device=DEV)
    y = torch.zeros(n, d, dtype=BF16, device=DEV)

    def step():
        table.lookup(ids, out=y)
        table.gradient(ids, dy, dW=dW)
        table.update(ids, dy)

    def reset():
        table.W.copy_(start)
        table.W_lp.copy_(start)

    prog = ops.Program()
    with prog.recording():
        step()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        ids.copy_(_tokens(rng, n, rows, ("zipf", "bad", "same", "distinct")[turn]))
        dy.normal_()
        reset()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dW, table.W, table.W_lp)]
        for again in (prog.run, graph.replay):
            reset()
            dW.fill_(float("nan"))
            y.zero_()
            again()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((y, dW, table.W, table.W_lp), want))
    prog.close()
