"""AdamW over many variables on the GPU, moments in fp32 and in 8 bits, against float64."""
import numpy as np
import pytest
import torch

from paper_1605_08695_amd import ops
from paper_1605_08695_amd.optim import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, FP8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


def say(*a):
    print(*a, flush=True)


def spread(x, n):
    """A factor for each 256 values, to each value."""
    return x.repeat_interleave(256)[:n]


class Model:
    """Variables of given sizes, each `offset` values into a buffer of its own with guards around, and their moments."""

    def __init__(self, sizes, bits, seed, offset=0, shadow=True, first=False):
        rng = np.random.default_rng(seed)
        self.sizes, self.bits = sizes, bits
        up = lambda a: torch.from_numpy(np.asarray(a)).float().to(DEV)  # noqa: E731
        self.bufs = []

        def room(v):
            buf = torch.full((v.numel() + offset + 9,), 77.0, device=DEV).to(v.dtype)
            at = buf[offset:offset + v.numel()]
            at.copy_(v)
            self.bufs.append((buf, offset, v.numel()))
            return at

        self.vars, self.grads, self.ms, self.vs, self.mc, self.vc, self.sh = [], [], [], [], [], [], []
        for n in sizes:
            size = np.exp(rng.standard_normal(n) * 2 - 6)
            self.vars.append(room(up(rng.standard_normal(n))))
            self.grads.append(room(up(rng.standard_normal(n) * size)))
            m, v = up(rng.standard_normal(n) * size * 0.3), up(size ** 2 * rng.random(n))
            if first:
                m, v = torch.zeros_like(m), torch.zeros_like(v)
            if bits == 8:
                b = ops.adamw_scales(n)
                mc = up(np.exp(rng.standard_normal(b) - 9)) * (0.0 if first else 1.0)
                vc = up(np.exp(rng.standard_normal(b) - 9)) * (0.0 if first else 1.0)
                self.mc.append(room(mc)), self.vc.append(room(vc))
                self.ms.append(room((m / spread(mc, n).clamp(min=1e-30)).clamp(-448, 448).to(FP8)))
                self.vs.append(room((v.sqrt() / spread(vc, n).clamp(min=1e-30)).clamp(0, 448).to(FP8)))
            else:
                self.ms.append(room(m)), self.vs.append(room(v))
            self.sh.append(room(torch.zeros(n, device=DEV).to(BF16)) if shadow else None)

    def moments(self, i):
        m, v = self.ms[i].double(), self.vs[i].double()
        if self.bits == 8:
            m = m * spread(self.mc[i], m.numel()).double()
            v = (v * spread(self.vc[i], v.numel()).double()) ** 2
        return m, v

    def guards(self):
        return all((b[:o].float() == f).all() and (b[o + n:].float() == f).all()
                   for b, o, n in self.bufs for f in [float(torch.tensor(77.0).to(b.dtype))])

    def args(self):
        return dict(shadows=self.sh, bits=self.bits, **(dict(m_scales=self.mc, v_scales=self.vc) if self.bits == 8 else {}))


# Bounds.  In 8 bits the old moments are a product of two stored numbers (one rounding; the second squared, two more):
# 1 and 4 U of themselves.  m: two products and a sum, 4 U (|b1 m| + |(1 - b1) g|); v: sums of numbers >= 0, 8 U v.
# The step: the moments' errors, its coefficients' and instructions' roundings, 20 U of itself beside m's.
def reference(md, i, lr, b1, b2, eps, wd, t):
    m, v = md.moments(i)
    g, var = md.grads[i].double(), md.vars[i].double()
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    dm, dv = 6 * U * ((b1 * m).abs() + ((1 - b1) * g).abs()), 12 * U * v1 + 2.0 ** -140
    root = torch.sqrt(v1 / (1 - b2 ** t)) + eps
    k = lr / (1 - b1 ** t)
    step = k * m1 / root
    out = var - lr * wd * var - step
    # sqrt of a v that is off by dv, subnormal ones among them
    droot = dv / (1 - b2 ** t) / torch.sqrt(v1 / (1 - b2 ** t) + 1e-300)
    dstep = k * dm / root + step.abs() * (20 * U + droot / root)
    return m1, v1, out, dm, dv, dstep + 4 * U * (var.abs() + step.abs()) + 2 * U * lr * wd * var.abs()


def near(got, want, tol, what):
    off = (got.double() - want).abs() - tol
    assert not off.isnan().any() and (off <= 1e-43).all(), (what, off.max().item())


def verify(md, before, lr, b1, b2, eps, wds, t):
    for i, n in enumerate(md.sizes):
        if n == 0:
            continue
        m1, v1, out, dm, dv, dvar = reference(before, i, lr, b1, b2, eps, wds[i], t)
        near(md.vars[i], out, dvar, "var")
        if md.sh[i] is not None:
            assert torch.equal(md.sh[i], md.vars[i].to(BF16))
        if md.bits == 32:
            near(md.ms[i], m1, dm, "m")
            near(md.vs[i], v1, dv, "v")
            continue
        r1, dr = torch.sqrt(v1), dv / (2 * torch.sqrt(v1 + 1e-300)) + 2 * U * torch.sqrt(v1)
        for x, dx, val, sc, what in ((m1, dm, md.ms[i], md.mc[i], "m"), (r1, dr, md.vs[i], md.vc[i], "v")):
            rows = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
            err = torch.nn.functional.pad(dx, (0, -n % 256)).view(-1, 256).amax(1)
            top = rows.abs().amax(1)
            near(sc, top / 448, (err + 2 * U * top) / 448, what + "'s scale")
            s = spread(sc, n).double()
            near_ = (val.double() * s - x).abs()
            # half a step of e4m3, 2^-4 of the value, or half of its smallest; a root that is there is at least that
            tol = 2.0 ** -4 * x.abs() * (1 + 16 * U) + s * 2.0 ** -10 + 2 * dx
            if what == "v":
                tol = torch.maximum(tol, s * 2.0 ** -9 * 1.001)
                assert ((val.double() > 0) | (x == 0) | (s == 0)).all()
            assert (near_ <= tol).all(), (what, (near_ - tol).max().item())


HYPER = [(1e-3, 0.9, 0.999, 1e-8, 0.1, 1), (0.5, 0.0, 0.5, 1e-3, 0.0, 7), (1e-2, 0.95, 0.99, 0.0, 1e-2, 100000)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("hyper", HYPER)
@pytest.mark.parametrize("sizes,offset", [([1], 0), ([255, 256, 257], 0), ([5, 0, 4096, 1000003], 1), ([64] * 130 + [3000], 0),
                                          ([70001, 3, 128], 3)])
def test_step(sizes, offset, hyper, bits):
    say("adamw", sizes[:4], len(sizes), offset, hyper, bits)
    lr, b1, b2, eps, wd, t = hyper
    md, before = Model(sizes, bits, len(sizes), offset), Model(sizes, bits, len(sizes), offset)
    if len(sizes) > 1:
        md.sh[1] = before.sh[1] = None
    wds = [wd if i % 2 == 0 else 0.0 for i in range(len(sizes))]
    ops.apply_adamw_multi(md.vars, md.ms, md.vs, md.grads, lr, b1, b2, eps, t, weight_decay=wds, **md.args())
    torch.cuda.synchronize()
    verify(md, before, lr, b1, b2, eps, wds, t)
    assert md.guards()
    assert all(torch.equal(a, b) for a, b in zip(md.grads, before.grads))


@pytest.mark.parametrize("bits", [32, 8])
def test_handle_steps_from_zero(bits):
    """The handle's own moments, five steps, against steps of single calls; then continued from its moments."""
    sizes = [300, 7, 2048]
    md, other = Model(sizes, bits, 3, first=True), Model(sizes, bits, 3, first=True)
    opt = AdamW(md.vars, 1e-2, 0.9, 0.99, 1e-8, 0.1, shadows=md.sh, bits=bits)
    for t in range(1, 6):
        opt.step(md.grads)
        before = [Model(sizes, bits, 3, first=True) for _ in range(1)][0]
        for a, b in ((before.vars, other.vars), (before.ms, other.ms), (before.vs, other.vs), (before.mc, other.mc), (before.vc, other.vc)):
            for x, y in zip(a, b):
                x.copy_(y)
        ops.apply_adamw_multi(other.vars, other.ms, other.vs, other.grads, 1e-2, 0.9, 0.99, 1e-8, t, weight_decay=[0.1] * 3,
                              **other.args())
        torch.cuda.synchronize()
        verify(other, before, 1e-2, 0.9, 0.99, 1e-8, [0.1] * 3, t)
    assert opt.t == 5
    bytes_ = lambda x: x.view(torch.uint8) if x.dtype == FP8 else x  # noqa: E731
    for a, b in ((md.vars, other.vars), (opt.ms, other.ms), (opt.vs, other.vs), (md.sh, other.sh)):
        assert all(torch.equal(bytes_(x), bytes_(y)) for x, y in zip(a, b))
    more = AdamW(other.vars, 1e-2, 0.9, 0.99, 1e-8, 0.1, shadows=other.sh, bits=bits,
                 moments=(other.ms, other.vs, other.mc if bits == 8 else None, other.vc if bits == 8 else None), t=5)
    opt.step(md.grads), more.step(other.grads)
    torch.cuda.synchronize()
    assert more.t == 6 and all(torch.equal(x, y) for x, y in zip(md.vars, other.vars))


def test_eight_bits_where_they_could_go_wrong():
    """Blocks of zeros, of numbers too small for a factor, with one large value, with NaN and infinities."""
    n = 256 * 7
    g = torch.zeros(n, device=DEV)
    g[256:512] = 1e-32                   # its moments fall below 2^-100
    g[512:768] = 1e-3
    g[512] = 1e6                         # 2^30 times the others
    g[768] = NAN
    g[1024] = INF
    g[1280:1536] = -5.0
    g[1536:] = 3e-15                     # squares near fp32's smallest, roots as any others
    var = torch.zeros(n, device=DEV)
    opt = AdamW([var], 1.0, 0.9, 0.99, 1e-8, bits=8)
    opt.step([g])
    torch.cuda.synchronize()
    m, v = opt.ms[0].float().view(7, 256), opt.vs[0].float().view(7, 256)
    ms, vs = opt.m_scales[0], opt.v_scales[0]
    assert not m[0].any() and not v[0].any() and ms[0] == 0 and vs[0] == 0 and not var[:256].any()
    assert not m[1].any() and ms[1] == 0
    assert m[2, 0] == 448 and v[2, 0] == 448 and (m[2, 1:] == 0).all() and (v[2, 1:] == 2.0 ** -9).all()
    assert ms[3].isnan() and vs[3].isnan() and ms[4].isnan() and vs[4].isnan()
    assert (m[5] == -448).all() and (v[5] == 448).all() and (v[6] == 448).all()
    assert var[768].isnan() and torch.isfinite(var[769:1024]).all()
    # a later step with small gradients stays small where a rounded second moment is larger than its own
    at = var[513:768].clone()
    opt.step([torch.full_like(g, 1e-3)])
    torch.cuda.synchronize()
    assert (var[513:768] - at).abs().max() <= 1.0


def test_steps_in_8_bits_move_as_far_as_their_roundings_allow():
    """Equal gradients: the first moment's ratio to the gradient, r, goes to r' = b1 r + 1 - b1, rounded by at most 2^-4 of
    itself, the second's root's R to sqrt(b2 R^2 + 1 - b2), likewise; so in each step both lie between what the least
    and the largest roundings give."""
    n, k, lr, b1, b2 = 1000, 50, 1e-3, 0.9, 0.99
    gen = torch.Generator(device=DEV).manual_seed(1)
    g = (1.0 + torch.rand(n, generator=gen, device=DEV)) * torch.randn(n, generator=gen, device=DEV).sign()
    var = torch.zeros(n, device=DEV)
    opt = AdamW([var], lr, b1, b2, 0.0, bits=8)
    least = most = 0.0
    lo, hi, LO, HI = 0.0, 0.0, 0.0, 0.0
    for t in range(1, k + 1):
        opt.step([g])
        lo, hi = b1 * lo + 1 - b1, b1 * hi + 1 - b1
        LO, HI = (b2 * LO ** 2 + 1 - b2) ** 0.5, (b2 * HI ** 2 + 1 - b2) ** 0.5
        c = (1 - b2 ** t) ** 0.5 / (1 - b1 ** t)
        least, most = least + c * lo / HI, most + c * hi / LO
        lo, LO, hi, HI = lo * (1 - 2.0 ** -4), LO * (1 - 2.0 ** -4), hi * (1 + 2.0 ** -4), HI * (1 + 2.0 ** -4)
    torch.cuda.synchronize()
    move = -(var / g.sign()).double() / lr
    assert move.min().item() >= least * (1 - 1e-4) and move.max().item() <= most * (1 + 1e-4)


def test_large_variable_and_two_streams():
    n = (1 << 31) + 300
    var, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    g[-1] = g[(1 << 31) + 5] = 1.0
    opt = AdamW([var], 0.5, bits=8)
    opt.step([g])
    torch.cuda.synchronize()
    assert var[-1] == -0.5 and var[(1 << 31) + 5] == -0.5 and var[1 << 31] == 0
    del var, g, opt
    a, b = Model([5000, 77], 8, 1), Model([5000, 77], 8, 2)
    wa, wb = Model([5000, 77], 8, 1), Model([5000, 77], 8, 2)
    for md, st in ((a, torch.cuda.Stream()), (b, torch.cuda.Stream()), (wa, None), (wb, None)):
        ops.apply_adamw_multi(md.vars, md.ms, md.vs, md.grads, 1e-3, 0.9, 0.99, 1e-8, 3, stream=st, **md.args())
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for p, q in ((a, wa), (b, wb)) for x, y in zip(p.vars, q.vars))


def test_captured_and_recorded():
    for bits in (32, 8):
        md, want = Model([3000, 5], bits, 1), Model([3000, 5], bits, 1)
        opt = AdamW(md.vars, 1e-3, shadows=md.sh, bits=bits)
        ref = AdamW(want.vars, 1e-3, shadows=want.sh, bits=bits)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            opt.step(md.grads, t=2)
        prog = ops.Program()
        with prog.recording():
            opt.step(md.grads, t=2)
        ref.step(want.grads, t=2)
        for _ in range(3):
            graph.replay()
            ref.step(want.grads, t=2)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(md.vars, want.vars))
        prog.run()
        ref.step(want.grads, t=2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(md.vars, want.vars))


def test_codes_agree_with_elementary_operations():
    """Each operation on the moments is rounded as it is written, so the codes and factors are, bit by bit, those of
    elementary tensor operations in the same order, also for values next to a border between two codes."""
    n, lr, b1, b2, eps = 256 * 8000, 1e-3, 0.9, 0.999, 1e-8
    md = Model([n], 8, 31)
    m, v, mc, vc = (x[0].clone() for x in (md.ms, md.vs, md.mc, md.vc))
    g = md.grads[0].view(-1, 256)
    for t in (1, 2, 3):
        ops.apply_adamw_multi(md.vars, md.ms, md.vs, md.grads, lr, b1, b2, eps, t, m_scales=md.mc, v_scales=md.vc, bits=8)
        m1 = b1 * (m.float().view(-1, 256) * mc[:, None]) + (1 - b1) * g
        root = torch.sqrt(b2 * (v.float().view(-1, 256) * vc[:, None]).square() + (1 - b2) * g * g)
        top = m1.abs().amax(1), root.amax(1)
        m = (m1 * (448.0 / top[0])[:, None]).clamp(-448, 448).to(FP8).view(-1)
        v = (root * (448.0 / top[1])[:, None]).clamp(2.0 ** -9, 448).to(FP8).view(-1)
        mc, vc = top[0] / 448.0, top[1] / 448.0
        for got, want in ((md.ms[0], m), (md.vs[0], v)):
            assert torch.equal(got.view(torch.uint8), want.view(torch.uint8)), t
        assert torch.equal(md.mc[0], mc) and torch.equal(md.vc[0], vc), t


# A root r beside a steady |g| is rounded back to where it was, relative to its block's largest, while b2 r^2 + (1 - b2) g^2
# lies below (1 + 2^-4)^2 r^2, half of e4m3's widest step above it: until g^2 > (1 + (2^-3 + 2^-8) / (1 - b2)) r^2.  Beyond
# that each step moves it up a code, 2^-4 of itself or more.  The largest is exact, and at the end as far from its own |g|
# as b2^t says; the rest of the block was scaled with it, so each root lies between the bound (and its rounding, 2^-4) and
# the larger of its |g| before and after, rounded.
@pytest.mark.parametrize("b2", [0.9, 0.99, 0.999])
def test_second_moments_in_8_bits_follow_as_far_as_stated(b2):
    say("follow", b2)
    k = 1 - b2
    steps = first = int(12 / k)
    sizes = torch.ones(256, device=DEV)
    sizes[0] = 2000.0
    before, after = sizes.clone(), sizes.clone()
    for i, (a, b) in enumerate([(1.0, 1.3), (1.0, 6.0), (1.0, 100.0), (3.0, 1500.0), (100.0, 1.0), (40.0, 30.0)]):
        before[1 + 40 * i:31 + 40 * i], after[1 + 40 * i:31 + 40 * i] = a, b
    gen = torch.Generator(device=DEV).manual_seed(2)
    var = [torch.zeros(256, device=DEV) for _ in range(2)]
    short, exact = AdamW(var[:1], 1e-3, 0.9, b2, bits=8), AdamW(var[1:], 1e-3, 0.9, b2, bits=32)
    for t in range(first + steps):
        g = (before if t < first else after) * (torch.rand(256, generator=gen, device=DEV) - 0.5).sign()
        short.step([g]), exact.step([g])
    torch.cuda.synchronize()
    r = short.vs[0].double() * short.v_scales[0].double()
    full = exact.vs[0].double().sqrt()
    # b2^steps < e^-12 of what was there before is left: (before / after)^2 e^-12 of v, half of that of its root
    assert ((full / after - 1).abs() <= ((before / after).double() ** 2 + 1) * np.exp(-12) / 2 + 1e-4).all().item()
    assert abs(r[0].item() / 2000.0 - 1) < 1e-3
    least = after.double() / (1 + (2.0 ** -3 + 2.0 ** -8) / k) ** 0.5
    most = torch.maximum(before, after).double()
    say("follow", b2, "of the exact root, least", (r / full).min().item(), "most", (r / full).max().item())
    assert (r >= least * (1 - 2.0 ** -4) * (1 - 1e-3)).all().item()
    assert (r <= most * (1 + 2.0 ** -4) * (1 + 1e-3)).all().item()
    steady = before == after
    assert ((r / full - 1).abs()[steady] <= 2.0 ** -4 * (1 + 1e-2)).all().item()
