"""The gated linear recurrence on the GPU: forward, backward and single tokens against the recurrence in float64,
at lengths, orders, strides and gates where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_1605_08695_amd import ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24                       # half a step of fp32, relative
TINY = 2.0 ** -126


def say(*a):
    print(*a, flush=True)


def f64(t):
    return t.detach().double().cpu()


def half(dt):
    return torch.finfo(dt).eps / 2


def sig(a):
    return 1.0 / (1.0 + torch.exp(-a))


# The bounds.  A gate's argument a = z + bias is rounded once and multiplied by a rounded log2(e), so its exponential
# is off by up to 3 |a| U, and with the instructions' last places (exponential, sum, reciprocal, product) the smaller of
# f and 1 - f by EG = (3 |a| + 8) U of itself.  A step moves a state by that share of x - h, so it is off by
# min(f, 1 - f) (|x| + |h|) EG and three roundings of numbers up to f |h| + (1 - f) |x|; `size` is that sum carried
# on, an upper bound of |h|.  Joined spans go through the same steps a second time, with states begun at 0, and a few
# roundings more: twice the error, and 8 U size a step.  The exponential flushes what is below TINY = 2^-126.
def reference(z, bias, h0, lengths, gates, dy=None, dh=None):
    """Float64 results and bounds of what fp32 arithmetic may add to the rounding of the outputs."""
    b, t, cols = z.shape
    d = cols // gates
    pre = f64(z) + (f64(bias) if bias is not None else 0.0)
    x, a = pre[..., :d], pre[..., d:2 * d]
    f, q = sig(a), sig(-a)
    least = torch.minimum(f, q)
    EG = (3 * a.abs() + 8) * U
    o = sig(pre[..., 2 * d:]) if gates == 3 else torch.ones_like(x)
    EO = (3 * pre[..., 2 * d:].abs() + 9) * U if gates == 3 else torch.zeros_like(x)
    h = f64(h0) if h0 is not None else torch.zeros(b, d, dtype=torch.float64)
    n = [t] * b if lengths is None else [min(max(int(v), 0), t) for v in lengths]
    live = torch.tensor([[i < m for i in range(t)] for m in n], dtype=torch.bool).view(b, t, 1)
    M, E = h.abs(), torch.zeros_like(h)
    hs, es, ms = [h], [E], [M]
    for i in range(t):
        l = live[:, i]
        size = f[:, i] * M + q[:, i] * x[:, i].abs()
        E = torch.where(l, f[:, i] * E + 2 * (least[:, i] * EG[:, i] + TINY) * (x[:, i].abs() + M) + 8 * size * U, E)
        M = torch.where(l, size, M)
        h = torch.where(l, f[:, i] * h + q[:, i] * x[:, i], h)
        hs.append(h), es.append(E), ms.append(M)
    if t:
        H, EH = torch.stack(hs[1:], 1), torch.stack(es[1:], 1)
    else:
        H = EH = torch.zeros(b, 0, d, dtype=torch.float64)
    zero = torch.zeros((), dtype=torch.float64)
    out = dict(y=torch.where(live, o * H, zero), Ey=torch.where(live, o * EH + (o * H).abs() * (EO + 2 * U), zero), last=h,
               Elast=E)
    if dy is None:
        return out
    up = torch.where(live, f64(dy), zero)
    g = f64(dh) if dh is not None else torch.zeros(b, d, dtype=torch.float64)
    mag, Eg = g.abs(), torch.zeros_like(g)
    dz = torch.zeros(b, t, cols, dtype=torch.float64)
    Edz = torch.zeros_like(dz)
    for i in reversed(range(t)):
        l = live[:, i]
        inc = up[:, i] * o[:, i]
        g1, mag1 = g + inc, mag + inc.abs()
        # every |g| is at most mag; what comes from behind is joined as the states are
        E1 = Eg + 2 * inc.abs() * (EO[:, i] + 2 * U) + 4 * mag1 * U
        F, Q, X = f[:, i], q[:, i], x[:, i]
        away, Eaway = Q * g1, Q * E1 + mag1 * (Q * (EG[:, i] + 2 * U) + TINY)
        diff = hs[i] - X
        Ediff = es[i] + (ms[i] + X.abs()) * 4 * U
        parts = [(away, Eaway), (F * away * diff, F * (Eaway * diff.abs() + Ediff * Q * mag1 + Eaway * Ediff) +
                                 mag1 * diff.abs() * (F * Q * (2 * EG[:, i] + 6 * U) + TINY))]
        if gates == 3:
            slope = o[:, i] * (1 - o[:, i]) * up[:, i]
            v = slope * hs[i + 1]
            parts.append((v, v.abs() * (2 * EO[:, i] + 8 * U) + slope.abs() * (es[i + 1] + 4 * U * ms[i + 1])))
        dz[:, i] = torch.cat([torch.where(l, p, zero) for p, _ in parts], 1)
        Edz[:, i] = torch.cat([torch.where(l, e, zero) for _, e in parts], 1)
        g, mag = torch.where(l, F * g1, g), torch.where(l, F * mag1, mag)
        Eg = torch.where(l, F * E1 + 2 * (least[:, i] * EG[:, i] + TINY) * mag1 + 8 * F * mag1 * U, Eg)
    out.update(dz=dz, Edz=Edz, dh0=g, Edh0=Eg)
    return out


def near(got, want, bound, dt, what):
    got = f64(got)
    tol = bound * (1 + half(dt)) + half(dt) * want.abs() + 1e-37
    off = (got - want).abs() - tol
    assert torch.isfinite(got).all(), what
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0, (what, worst, (got - want).abs().max().item())


def make(b, t, d, gates, dt, seed, order="b", pad=0, hard=False):
    """z with its rows `pad` elements apart in either order, NaN between them; with `hard` gates wide open and shut."""
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((b, t, gates * d))
    v[..., d:] *= 3.0
    if hard:
        v[..., d:2 * d] += rng.choice([-90.0, -12.0, 0.0, 9.0, 14.0, 95.0], size=d)
    return strided(torch.from_numpy(v).to(dt).to(DEV), order, pad)


def strided(v, order, pad):
    b, t, c = v.shape
    if order == "b":
        wide = torch.full((b, t, c + pad), float("nan"), dtype=v.dtype, device=DEV)
        view = wide[..., pad // 2:pad // 2 + c]
    else:
        wide = torch.full((t, b, c + pad), float("nan"), dtype=v.dtype, device=DEV)
        view = wide[..., pad // 2:pad // 2 + c].transpose(0, 1)
    view.copy_(v)
    return view


CASES = [(1, 1, 1, "b", 0, None), (3, 1, 7, "t", 0, None), (2, 2, 64, "b", 0, None), (2, 127, 65, "b", 3, None),
         (2, 128, 64, "t", 0, None), (3, 129, 130, "b", 0, "mixed"), (1, 700, 33, "b", 1, None), (7, 260, 24, "t", 5, "mixed"),
         (5, 40, 200, "b", 8, "short"), (2, 300, 512, "b", 0, "none"), (1, 5000, 3, "b", 0, None), (70, 3, 10, "t", 0, "mixed"),
         # long runs in segments, short runs of several strips, and strips enough to be read by a workgroup each
         (4, 2100, 600, "b", 0, None), (6, 4200, 131, "t", 2, "mixed"), (2, 1000, 512, "t", 0, None),
         (520, 140, 40, "b", 0, "mixed")]


def _lengths(kind, b, t):
    if kind is None:
        return None
    v = {"mixed": [t, 0, 1, t + 5, -3, t // 2, max(0, t - 1)], "short": [0, 1, 2, 3, 0], "none": [0]}[kind]
    return torch.tensor([v[i % len(v)] for i in range(b)], dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dt", [F32, BF16], ids=str)
@pytest.mark.parametrize("gates", [2, 3])
@pytest.mark.parametrize("b,t,d,order,pad,kind", CASES)
def test_forward_and_backward(b, t, d, order, pad, kind, gates, dt):
    say("recurrence", b, t, d, gates, dt, order, pad, kind)
    rng = np.random.default_rng(b * 1000 + t)
    z = make(b, t, d, gates, dt, 1, order, pad)
    up = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().to(DEV)  # noqa: E731
    bias, h0, dh = up(gates * d), up(b, d), up(b, d)
    dy = strided(up(b, t, d).to(dt), order, pad)
    lengths = _lengths(kind, b, t)
    y, last, saved = ops.gated_scan_fwd(z, gates == 3, bias, h0, lengths, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved, gates == 3, bias, lengths, dh)
    torch.cuda.synchronize()
    r = reference(z, bias, h0, lengths, gates, dy, dh)
    near(y, r["y"], r["Ey"], dt, "y")
    near(last, r["last"], r["Elast"], F32, "last")
    near(dz, r["dz"], r["Edz"], dt, "dz")
    near(dh0, r["dh0"], r["Edh0"], F32, "dh0")
    again = ops.gated_scan_fwd(z, gates == 3, bias, h0, lengths)
    assert again[2] is None and torch.equal(again[0], y) and torch.equal(again[1], last)
    # in place, into a buffer with room between its rows, and without what may be left out
    room = strided(torch.zeros(b, t, d, dtype=dt, device=DEV), order, pad)
    assert torch.equal(ops.gated_scan_fwd(z, gates == 3, bias, h0, lengths, y=room)[0], y)
    mine = z.clone() if not pad else strided(z, order, pad)
    assert torch.equal(ops.gated_scan_bwd(mine, dy, saved, gates == 3, bias, lengths, dh, dz=mine)[0], dz)
    if pad:
        whole = mine._base
        assert whole.isnan().sum().item() == whole.numel() - mine.numel()
    y0, last0, saved0 = ops.gated_scan_fwd(z, gates == 3, save=True)
    dz0, dh00 = ops.gated_scan_bwd(z, dy, saved0, gates == 3)
    torch.cuda.synchronize()
    r = reference(z, None, None, None, gates, dy)
    near(y0, r["y"], r["Ey"], dt, "y")
    near(last0, r["last"], r["Elast"], F32, "last")
    near(dz0, r["dz"], r["Edz"], dt, "dz")
    near(dh00, r["dh0"], r["Edh0"], F32, "dh0")


@pytest.mark.parametrize("gates", [2, 3])
@pytest.mark.parametrize("b,t,d", [(1, 1, 5), (2, 400, 70), (1, 3000, 8)])
def test_gates_open_and_shut(b, t, d, gates):
    """Gates that keep a state for millions of tokens, and ones that keep nothing."""
    say("hard gates", b, t, d, gates)
    z = make(b, t, d, gates, F32, 3, hard=True)
    g = torch.Generator(device=DEV).manual_seed(3)
    h0, dy = torch.randn(b, d, generator=g, device=DEV), torch.randn(b, t, d, generator=g, device=DEV)
    y, last, saved = ops.gated_scan_fwd(z, gates == 3, h0=h0, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved, gates == 3)
    torch.cuda.synchronize()
    r = reference(z, None, h0, None, gates, dy)
    near(y, r["y"], r["Ey"], F32, "y")
    near(last, r["last"], r["Elast"], F32, "last")
    near(dz, r["dz"], r["Edz"], F32, "dz")
    near(dh0, r["dh0"], r["Edh0"], F32, "dh0")


def test_nearly_open_gates_keep_steady_values():
    """A state that forgets a part in 10^5 a token: after 20000 equal inputs it is where the formula puts it, which a
    gate rounded to fp32 (f = 1 - 1e-5, off by 3e-8) would miss by 3e-3 of the way."""
    t, d = 20000, 64
    a = float(np.log(1e5))
    z = torch.zeros(1, t, 2 * d, device=DEV)
    z[..., :d], z[..., d:] = 1.0, a
    _, last, _ = ops.gated_scan_fwd(z)
    torch.cuda.synchronize()
    q = 1.0 / (1.0 + np.exp(float(np.float32(a))))
    want = 1.0 - (1.0 - q) ** t
    # each state is rounded to half a step of 2^-24 of itself, at most 20000 times, with signs that do not agree; the
    # share q is off by (3 a + 8) U of itself
    tol = (3 * a + 8) * U * q * t + 2 * U * np.sqrt(t) * 8
    assert abs(last.double().cpu().numpy() - want).max() < tol


def test_forgotten_states_leave_nothing():
    """A state of 1e20 meets a gate that keeps a part in 10^30 of it: nothing of its roundings is left."""
    b, t, d = 2, 300, 66
    z = make(b, t, d, 2, F32, 9)
    z[0, 130, :d] = 1e20
    z[:, 131:134, d:] = -40.0
    z[1, 0, d:] = -120.0
    h0 = torch.full((b, d), 3e20, device=DEV)
    dy = torch.randn(b, t, d, device=DEV)
    dy[:, 133] = 1e20
    y, last, saved = ops.gated_scan_fwd(z, h0=h0, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved)
    torch.cuda.synchronize()
    r = reference(z, None, h0, None, 2, dy)
    near(y, r["y"], r["Ey"], F32, "y")
    near(last, r["last"], r["Elast"], F32, "last")
    near(dz, r["dz"], r["Edz"], F32, "dz")
    near(dh0, r["dh0"], r["Edh0"], F32, "dh0")


def test_gradient_against_differences():
    """The kernels' gradients along random directions against central differences of the formula in float64."""
    b, t, d, gates = 2, 150, 6, 3
    z = make(b, t, d, gates, F32, 5)
    rng = np.random.default_rng(5)
    up = lambda *s: torch.from_numpy(rng.standard_normal(s)).float().to(DEV)  # noqa: E731
    bias, h0, dh, dy = up(gates * d), up(b, d), up(b, d), up(b, t, d)
    lengths = torch.tensor([t, 90], dtype=torch.int32, device=DEV)
    _, _, saved = ops.gated_scan_fwd(z, True, bias, h0, lengths, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved, True, bias, lengths, dh)
    torch.cuda.synchronize()
    r = reference(z, bias, h0, lengths, gates, dy, dh)

    def loss(e, vz, vh):
        q = reference(f64(z) + e * vz, bias, f64(h0) + e * vh, lengths, gates)
        return (q["y"] * f64(dy)).sum() + (q["last"] * f64(dh)).sum()

    for _ in range(3):
        vz, vh = torch.from_numpy(rng.standard_normal(z.shape)), torch.from_numpy(rng.standard_normal((b, d)))
        e = 1e-4
        diff = (loss(e, vz, vh) - loss(-e, vz, vh)) / (2 * e)
        mine = (f64(dz) * vz).sum() + (f64(dh0) * vh).sum()
        # the kernels' bounds, and a difference's own error: e^2 / 6 of a third derivative, itself taken from a step
        # twice as wide
        wide = (loss(2 * e, vz, vh) - loss(-2 * e, vz, vh)) / (4 * e)
        tol = ((r["Edz"] + U * r["dz"].abs()) * vz.abs()).sum() + ((r["Edh0"] + U * r["dh0"].abs()) * vh.abs()).sum()
        assert abs(mine - diff) <= tol + abs(wide - diff) + 1e-7 * abs(diff)


def test_padding_is_not_read_and_nan_stays_in_its_channel():
    b, t, d = 3, 200, 96
    z = make(b, t, d, 3, F32, 7)
    lengths = torch.tensor([150, 0, 200], dtype=torch.int32, device=DEV)
    dy = torch.randn(b, t, d, device=DEV)
    want = ops.gated_scan_fwd(z, True, lengths=lengths, save=True)
    wantg = ops.gated_scan_bwd(z, dy, want[2], True, lengths=lengths)
    bad, bdy = z.clone(), dy.clone()
    for v in (bad, bdy):
        v[0, 150:] = float("nan")
        v[1] = float("inf")
    got = ops.gated_scan_fwd(bad, True, lengths=lengths, save=True)
    gotg = ops.gated_scan_bwd(bad, bdy, got[2], True, lengths=lengths)
    assert all(torch.equal(g, w) for g, w in zip(got[:2] + gotg, want[:2] + wantg))
    for col in (5, d + 5):
        bad = z.clone()
        bad[2, 60, col] = float("nan")
        y = ops.gated_scan_fwd(bad, True, lengths=lengths)[0]
        assert y[2, 60:, 5].isnan().all()
        y[2, 60:, 5] = want[0][2, 60:, 5]
        assert torch.equal(y, want[0])
    torch.cuda.synchronize()


def like(got, want, bound, dt, what):
    """near() where a result is finite, and the same infinities and NaN elsewhere."""
    got = f64(got)
    fin = torch.isfinite(want)
    wrong = ((got.isnan() != want.isnan()) | (torch.isinf(want) & (got != want))).nonzero().tolist()
    assert not wrong, (what, len(wrong), wrong[:3])
    assert torch.isfinite(bound[fin]).all().item()
    near(got[fin], want[fin], bound[fin], dt, what)


@pytest.mark.parametrize("dt", [F32, BF16], ids=str)
@pytest.mark.parametrize("gates", [2, 3])
@pytest.mark.parametrize("b,t,d", [(3, 1, 9), (2, 40, 70), (3, 300, 65), (1, 3000, 64), (520, 140, 6)])
def test_infinite_inputs_give_what_the_formula_gives(b, t, d, gates, dt):
    """Infinities in x, in the first states and in dy, at gates on both sides of 0: the state is infinite from there on,
    NaN where two of different signs meet, and no other channel or earlier row knows of it."""
    say("infinite", b, t, d, gates, dt)
    inf = float("inf")
    z = make(b, t, d, gates, dt, 4)
    g = torch.Generator(device=DEV).manual_seed(4)
    h0, dh = (torch.randn(b, d, generator=g, device=DEV) for _ in range(2))
    dy = torch.randn(b, t, d, generator=g, device=DEV).to(dt)
    last = b - 1
    z[0, t // 3, 0], z[0, t // 3, d] = inf, 2.0
    z[0, t // 3, 1], z[0, t // 3, d + 1] = -inf, -2.0
    z[last, t // 2, 2] = inf
    z[last, t - 1, 2] = -inf
    h0[0, 3], h0[last, 4] = -inf, inf
    z[last, t // 2, 4] = -inf
    dy[last, t // 2, 5] = inf
    dh[0, 5] = -inf
    y, end, saved = ops.gated_scan_fwd(z, gates == 3, h0=h0, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved, gates == 3, dh_last=dh)
    torch.cuda.synchronize()
    r = reference(z, None, h0, None, gates, dy, dh)
    like(y, r["y"], r["Ey"], dt, "y")
    like(end, r["last"], r["Elast"], F32, "last")
    like(dz, r["dz"], r["Edz"], dt, "dz")
    like(dh0, r["dh0"], r["Edh0"], F32, "dh0")
    state = h0.clone()
    ys = ops.gated_scan_step(z[:, 0].contiguous(), state, None, gates == 3)
    r = reference(z[:, :1], None, h0, None, gates)
    like(ys, r["y"][:, 0], r["Ey"][:, 0], dt, "step")
    like(state, r["last"], r["Elast"], F32, "state")


def test_empty_batches_and_sequences():
    for b, t in ((0, 5), (3, 0), (0, 0)):
        z = torch.zeros(b, t, 8, device=DEV)
        h0, dh = torch.randn(b, 4, device=DEV), torch.randn(b, 4, device=DEV)
        y, last, saved = ops.gated_scan_fwd(z, h0=h0, save=True)
        dz, dh0 = ops.gated_scan_bwd(z, torch.zeros(b, t, 4, device=DEV), saved, dh_last=dh)
        assert y.shape == (b, t, 4) and dz.shape == z.shape
        assert torch.equal(last, h0) and torch.equal(dh0, dh)
    assert ops.gated_scan_step(torch.zeros(0, 8, device=DEV), torch.zeros(3, 4, device=DEV)).shape == (0, 4)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dt", [F32, BF16], ids=str)
@pytest.mark.parametrize("gates", [2, 3])
@pytest.mark.parametrize("n,d,slots,pad", [(1, 1, 1, 0), (5, 33, 9, 0), (128, 512, 300, 0), (33, 771, 40, 3), (1000, 64, 2000, 8)])
def test_step(n, d, slots, pad, gates, dt):
    say("step", n, d, slots, pad, gates, dt)
    rng = np.random.default_rng(n)
    z = strided(torch.from_numpy(rng.standard_normal((1, n, gates * d)) * 2).to(dt).to(DEV), "b", pad)[0]
    bias = torch.from_numpy(rng.standard_normal(gates * d)).float().to(DEV)
    state = torch.from_numpy(rng.standard_normal((slots, d))).float().to(DEV)
    at = torch.from_numpy(rng.permutation(slots)[:n].astype(np.int32)).to(DEV)
    if n > 4:
        at[3], at[4] = -1, slots
    before = state.clone()
    room = strided(torch.zeros(1, n, d, dtype=dt, device=DEV), "b", pad)[0]
    y = ops.gated_scan_step(z, state, at, gates == 3, bias, y=room)
    torch.cuda.synchronize()
    rows = [i for i in range(n) if 0 <= int(at[i]) < slots]
    used = [int(at[i]) for i in rows]
    r = reference(z[rows][:, None], bias, before[used], None, gates)
    near(y[rows], r["y"][:, 0], r["Ey"][:, 0], dt, "y")
    near(state[used], r["last"], r["Elast"], F32, "state")
    rest = [s for s in range(slots) if s not in set(used)]
    assert torch.equal(state[rest], before[rest])
    assert not y[[i for i in range(n) if i not in rows]].any()
    # without slots: row i has state i
    if n <= slots:
        mine, direct = before.clone(), before.clone()
        all_ = torch.arange(n, dtype=torch.int32, device=DEV)
        assert torch.equal(ops.gated_scan_step(z, mine, None, gates == 3, bias),
                           ops.gated_scan_step(z, direct, all_, gates == 3, bias))
        assert torch.equal(mine, direct)


def test_steps_follow_the_sequence():
    """Token by token as all at once, and a sequence cut in two with its states handed on."""
    b, t, d = 4, 150, 40
    z = make(b, t, d, 3, F32, 11)
    bias = torch.randn(3 * d, device=DEV)
    y, last, _ = ops.gated_scan_fwd(z, True, bias)
    state = torch.zeros(b, d, device=DEV)
    ys = torch.stack([ops.gated_scan_step(z[:, i], state, None, True, bias) for i in range(t)], 1)
    r = reference(z, bias, None, None, 3)
    near(ys, r["y"], r["Ey"], F32, "y")
    near(state, r["last"], r["Elast"], F32, "last")
    ya, mid, _ = ops.gated_scan_fwd(z[:, :77], True, bias)
    yb, end, _ = ops.gated_scan_fwd(z[:, 77:], True, bias, h0=mid)
    near(torch.cat([ya, yb], 1), r["y"], r["Ey"], F32, "y")
    near(end, r["last"], r["Elast"], F32, "last")
    near(last, r["last"], r["Elast"], F32, "last")


def test_offsets_past_32_bits():
    """A batch of more than 2^31 elements: the last channels of the last sequence."""
    b, t, d = 3, 1500, 1 << 18
    z = torch.zeros(b, t, 2 * d, dtype=BF16, device=DEV)
    part = torch.randn(t, 64, device=DEV).to(BF16)
    for c in (d - 64, 2 * d - 64):
        z[-1, :, c:c + 64] = part
    small = torch.cat([z[-1:, :, d - 64:d], z[-1:, :, 2 * d - 64:]], 2).contiguous()
    dy = torch.zeros(b, t, d, dtype=BF16, device=DEV)
    dy[-1, :, -64:] = part
    y, last, saved = ops.gated_scan_fwd(z, save=True)
    dz, dh0 = ops.gated_scan_bwd(z, dy, saved, dz=z)
    torch.cuda.synchronize()
    r = reference(small, None, None, None, 2, dy[-1:, :, -64:])
    near(y[-1:, :, -64:], r["y"], r["Ey"], BF16, "y")
    near(last[-1:, -64:], r["last"], r["Elast"], F32, "last")
    near(torch.cat([dz[-1:, :, d - 64:d], dz[-1:, :, -64:]], 2), r["dz"], r["Edz"], BF16, "dz")
    near(dh0[-1:, -64:], r["dh0"], r["Edh0"], F32, "dh0")
    assert not y[0, -1].any() and not dz[0, -1].any() and not dz[-1, :, :64].any()


def test_two_streams_and_a_captured_graph():
    b, t, d = 2, 2000, 96
    zs = [make(b, t, d, 3, BF16, s) for s in (1, 2)]
    dy = torch.randn(b, t, d, device=DEV).to(BF16)

    def both(z, stream=None):
        y, last, saved = ops.gated_scan_fwd(z, True, save=True, stream=stream)
        return (y, last) + ops.gated_scan_bwd(z, dy, saved, True, stream=stream)

    want = [both(z) for z in zs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in zs]
    got = [both(z, s) for z, s in zip(zs, streams)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, c) for a, c in zip(g, w))
    # two graphs of one size, replayed in turn with eager work between
    graphs = []
    ins = [z.clone() for z in zs]
    side = torch.cuda.Stream()
    for z in ins:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = both(z)
        graphs.append((g, out))
    for k in range(4):
        i = k % 2
        ins[i].copy_(zs[(k // 2 + i) % 2])
        graphs[i][0].replay()
        both(zs[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(graphs[i][1], want[(k // 2 + i) % 2]))


def test_program_replays():
    z = make(2, 300, 40, 2, F32, 1)
    prog = ops.Program()
    state = torch.zeros(2, 40, device=DEV)
    with prog.recording():
        y, last, saved = ops.gated_scan_fwd(z, save=True)
        dz, dh0 = ops.gated_scan_bwd(z, y, saved)
        ops.gated_scan_step(z[:, 0], state)
    assert len(prog) == 3
    new = make(2, 300, 40, 2, F32, 2)
    z.copy_(new)
    state.zero_()
    prog.run()
    w = ops.gated_scan_fwd(new, save=True)
    wz, wh = ops.gated_scan_bwd(new, w[0], w[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in ((y, w[0]), (last, w[1]), (dz, wz), (dh0, wh)))
