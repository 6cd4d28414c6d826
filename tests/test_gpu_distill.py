"""Distillation from a teacher's top logits on the GPU: loss and gradient against the formula in
float64, within bounds that count the roundings; the formula's gradient against differences."""
import math

import numpy as np
import pytest
import torch

from paper_1605_08695_amd import ops
from paper_1605_08695_amd.embedding import EmbeddingTable
from paper_1605_08695_amd.sampled import FullSoftmaxHead

gpu = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24                       # half a step of fp32, relative
INF = float("inf")


def say(*a):
    print(*a, flush=True)


# ----------------------------------------------------------------------------- the formula
class Ref:
    """Loss and gradient in float64 from the inputs' values, and how far fp32 arithmetic may be off."""

    def __init__(self, z, idx, t, scale, T=1.0, lse=None, labels=None, alpha=1.0, weight=None, bias=None):
        x = z.double()
        n, c = x.shape
        dev = x.device
        if bias is not None:
            x = x + bias.double()
        idx = idx.long()
        valid = (idx >= 0) & (idx < c)
        t = torch.where(valid, t.double(), torch.full((), -INF, dtype=torch.float64, device=dev))
        hard = labels is not None and alpha < 1.0
        soft = torch.ones(n, dtype=torch.bool, device=dev)
        if lse is None:
            soft = (t > -INF).any(1) | torch.isnan(t).any(1)
            ent = torch.softmax(t / T, 1)                  # entry probabilities
            ent[~soft] = 0
        else:
            ent = torch.exp(t / T - lse.double()[:, None])
        at = torch.where(valid, idx, torch.full_like(idx, c))
        p = torch.zeros(n, c + 1, dtype=torch.float64, device=dev).scatter_add_(1, at, torch.where(valid, ent, 0.0))[:, :c]
        K = torch.zeros(n, c + 1, dtype=torch.bool, device=dev).scatter_(1, at, valid)[:, :c]
        pr = torch.clamp(1 - p.sum(1), min=0) if lse is not None else torch.zeros(n, dtype=torch.float64, device=dev)
        logq = torch.log_softmax(x / T, 1)
        logqr = torch.logsumexp(torch.where(K, torch.full_like(x, -INF), logq), 1)
        q, qr = torch.exp(logq), torch.exp(logqr)
        term = torch.where(K & (p != 0), p * (torch.log(p) - logq), torch.zeros_like(x))
        rest = torch.where(pr != 0, pr * (torch.log(pr) - logqr), torch.zeros_like(pr))
        sl = torch.where(soft, term.sum(1) + rest, torch.zeros_like(pr))
        others = torch.where(K, torch.full_like(x, -INF), x)
        share = torch.softmax(others / T, 1)               # of the classes outside K among themselves
        share = torch.where((others == -INF).all(1, keepdim=True), torch.zeros_like(x), share)
        gq = torch.where(K, q - p, share * (qr - pr)[:, None])
        gq = torch.where(soft[:, None], gq, torch.zeros_like(x))
        loss, g = alpha * T * T * sl, alpha * T * gq
        w = torch.ones(n, dtype=torch.float64, device=dev) if weight is None else weight.double()
        if hard:
            lab = labels.long()
            bad = (lab < 0) | (lab >= c)
            lc = lab.clamp(0, c - 1)
            lsm = torch.log_softmax(x, 1)
            hl = -lsm.gather(1, lc[:, None])[:, 0]
            hg = torch.exp(lsm)
            hg.scatter_add_(1, lc[:, None], torch.full((n, 1), -1.0, dtype=torch.float64, device=dev))
            hl[bad] = float("nan")
            hg[bad] = float("nan")
            loss, g = loss + (1 - alpha) * hl, g + (1 - alpha) * hg
        zero = (w == 0)
        self.q, self.share = q, share
        self.loss = torch.where(zero, torch.zeros_like(loss), w * loss)
        self.grad = torch.where(zero[:, None], torch.zeros_like(g), scale * w[:, None] * g)
        # ---- bounds.  Logits that count (not masked) give the spans of the exponents.
        live = x > -1e30
        big = torch.where(live, x.abs(), torch.zeros_like(x)).amax(1)
        span = 2 * big
        # x is rounded once, x - m once, its product with log2(e) / T twice (that factor's own rounding
        # too), and an exponential is within 2 half steps of its argument's value
        delta = U * (2 * big + 4 * span) * max(1.0, 1.0 / T) + 4 * U
        # positive terms: at least 64 threads sum a row, each one's chain and a tree of joins
        chain = (c / 64 + 40) * U
        rq = (2 * delta + 2 * chain + 8 * U)[:, None]       # relative, of q, q_r and the shares
        tb = torch.where(torch.isfinite(t), t.abs(), torch.zeros_like(t)).amax(1) / T
        rp = (U * (6 * tb + (lse.double().abs() if lse is not None else 2 * tb) + idx.shape[1] + 16))[:, None]
        epr = rp[:, 0] * p.sum(1) + (idx.shape[1] + 2) * U if lse is not None else torch.zeros_like(pr)
        eg = torch.where(K, q * rq + p * rp, share * (qr * rq[:, 0] * 2 + epr + pr * rq[:, 0])[:, None])
        eg = alpha * T * torch.where(soft[:, None], eg, torch.zeros_like(eg))
        fin = lambda v: torch.where(torch.isfinite(v), v, torch.zeros_like(v))      # noqa: E731
        elq = (delta + chain)[:, None] + 4 * U * (fin(logq).abs() + big[:, None] / min(T, 1.0))
        el = (p * (rp * (1 + fin(torch.log(p) - logq).abs()) + elq + 4 * U * fin(torch.log(p)).abs())).sum(1)
        lpr = fin(torch.log(torch.maximum(pr, epr))).abs() + fin(logqr).abs()
        el = el + epr * (1 + lpr) + pr * (2 * (delta + 2 * chain) + 8 * U * (lpr + big / min(T, 1.0)))
        el = alpha * T * T * torch.where(soft, fin(el), torch.zeros_like(el))
        if hard:
            eg = eg + (1 - alpha) * (torch.exp(lsm) * rq + 4 * U)
            el = el + (1 - alpha) * (delta + chain + 4 * U * (2 * big + math.log(c) + 1))
        self.eloss = (w.abs() * (el + 8 * U * loss.abs())) * 1.01
        self.egrad = (abs(scale) * w.abs()[:, None] * (fin(eg) + 4 * U * g.abs())) * 1.01

    def check(self, loss, dz, what=""):
        def held(name, got, ref, tol):
            got, fine = got.double(), torch.isfinite(ref)
            # a logit at the type's lowest value makes terms of 3.4e38: where the bound around the exact
            # value reaches past the largest fp32 number, a result within the bound may have no finite
            # fp32 value, and infinity of its sign is its rounding
            past = fine & (ref.abs() + tol > torch.finfo(F32).max)
            got = torch.where(past & torch.isinf(got) & (torch.sign(got) == torch.sign(ref)), ref, got)
            assert torch.equal(fine, torch.isfinite(got)), (what, name, "finite where it should not be, or not")
            assert torch.equal(torch.isnan(ref), torch.isnan(got)), (what, name, "NaN")
            inf = torch.isinf(ref)
            assert torch.equal(ref[inf], got[inf]), (what, name, "infinite")
            d, tol = (got - ref).abs()[fine], tol[fine]
            worst = float((d / tol.clamp(min=1e-300)).max()) if d.numel() else 0.0
            say("  %s %-5s worst error / bound %.3f" % (what, name, worst))
            assert torch.all(d <= tol), (what, name, worst)

        held("loss", loss, self.loss, torch.nan_to_num(self.eloss, nan=0.0) + 1e-44)
        half = torch.finfo(dz.dtype).eps / 2               # the one rounding of the result
        held("dz", dz.reshape(self.grad.shape), self.grad,
             torch.nan_to_num(self.egrad, nan=0.0) + half * (torch.nan_to_num(self.grad.abs(), nan=0.0) + torch.nan_to_num(self.egrad, nan=0.0)) + 1e-40)


def test_formula_against_differences():
    """The reference's gradient is the slope of the reference's loss (float64, CPU)."""
    g = torch.Generator().manual_seed(1)
    n, c, k = 3, 7, 3
    z = torch.randn(n, c, generator=g, dtype=torch.float64)
    idx = torch.tensor([[2, 0, 5], [1, -1, 6], [4, 4, 3]])
    t = torch.randn(n, k, generator=g, dtype=torch.float64)
    bias = torch.randn(c, generator=g, dtype=torch.float64)
    w = torch.tensor([1.0, 0.5, 2.0], dtype=torch.float64)
    for T in (1.0, 2.5):
        for lse in (None, torch.logsumexp(t / T, 1) + 0.7):
            for alpha, labels in ((1.0, None), (0.3, torch.tensor([2, 0, 6]))):
                kw = dict(T=T, lse=lse, alpha=alpha, labels=labels, weight=w, bias=bias)
                r = Ref(z, idx, t, 1.0, **kw)
                h = 1e-6
                for j in range(c):
                    e = torch.zeros_like(z)
                    e[:, j] = h
                    num = (Ref(z + e, idx, t, 1.0, **kw).loss - Ref(z - e, idx, t, 1.0, **kw).loss) / (2 * h)
                    assert torch.allclose(num, r.grad[:, j], rtol=1e-6, atol=1e-8)


# ----------------------------------------------------------------------------- inputs
def _case(seed, n, c, k, dt, tdt, T, spread=2.0, lift=5.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)      # noqa: E731
    z = rnd(n, c) * spread
    first = torch.arange(k + 1, device=DEV) * c // k
    wide = first[1:] - first[:-1]
    idx = first[:-1] + torch.minimum((torch.rand(n, k, generator=g, device=DEV) * wide).long(), wide - 1)
    idx = torch.gather(idx, 1, torch.rand(n, k, generator=g, device=DEV).argsort(1))
    z.scatter_add_(1, idx, rnd(n, k) + lift)
    t = (torch.gather(z, 1, idx) + rnd(n, k)).to(tdt)
    lse = (torch.logsumexp(t.double() / T, 1) + 0.3 * torch.rand(n, generator=g, device=DEV)).float()
    labels = torch.randint(0, c, (n,), generator=g, device=DEV)
    labels = torch.where(torch.rand(n, generator=g, device=DEV) < 0.5, idx[:, 0], labels).to(torch.int32)
    weight = torch.rand(n, generator=g, device=DEV) + 0.5
    weight[torch.rand(n, generator=g, device=DEV) < 0.1] = 0.0
    return dict(z=z.to(dt), idx=idx.to(torch.int32), t=t, lse=lse, labels=labels, weight=weight, bias=rnd(c) * 0.5)


def _run(v, scale, T, rest, alpha, **kw):
    a = dict(temperature=T, top_lse=v["lse"] if rest else None, labels=v["labels"] if alpha < 1 else None, alpha=alpha,
             weight=v["weight"], bias=v["bias"])
    a.update(kw)
    return ops.distill_xent(v["z"], v["idx"], v["t"], scale, **a)


def _ref(v, scale, T, rest, alpha):
    return Ref(v["z"], v["idx"], v["t"], scale, T, v["lse"] if rest else None, v["labels"], alpha, v["weight"], v["bias"])


SHAPES = [(1, 1, 1), (1, 2, 1), (3, 2, 2), (5, 9, 9), (17, 63, 4), (4, 64, 64), (33, 65, 7), (2, 1024, 1024), (64, 1000, 5),
          (19, 1027, 33), (7, 4096, 64), (130, 2051, 17), (5, 8191, 100), (3, 16385, 12), (9, 40000, 32), (4, 50021, 20),
          (2, 65536, 64), (3, 65537, 300), (2, 98305, 8), (2, 131072, 64), (3, 131079, 5), (1, 262147, 1000)]


@gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,rest,alpha", [(1.0, False, 1.0), (2.0, True, 0.6), (1.0, True, 0.5), (4.0, False, 0.9),
                                          (0.5, True, 1.0), (1.5, False, 0.3)])
@pytest.mark.parametrize("n,c,k", SHAPES)
def test_distill(dt, T, rest, alpha, n, c, k):
    say("distill", dt, T, rest, alpha, n, c, k)
    tdt = BF16 if (n + c) % 2 else F32
    v = _case(n * 1000 + c, n, c, k, dt, tdt, T)
    loss, dz = _run(v, 1.0 / n, T, rest, alpha)
    r = _ref(v, 1.0 / n, T, rest, alpha)
    # in place, and again: the same bits
    z = v["z"].clone()
    loss2, dz2 = _run({**v, "z": z}, 1.0 / n, T, rest, alpha, dlogits=z)
    torch.cuda.synchronize()
    r.check(loss, dz)
    assert dz2 is z and torch.equal(loss, loss2) and torch.equal(dz, dz2)


@gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,c,zx,dx", [(5, 1000, 3, 0), (6, 777, 0, 5), (3, 40001, 7, 2), (4, 131075, 1, 1), (1, 50, 9, 4)])
def test_strided_rows(dt, n, c, zx, dx):
    say("distill strided", dt, n, c, zx, dx)
    v = _case(5, n, c, min(c, 20), dt, F32, 2.0)
    wide = torch.full((n, c + zx), float("nan"), dtype=dt, device=DEV)
    out = torch.full((n, c + dx), 3.0, dtype=dt, device=DEV)
    wide[:, zx:] = v["z"]
    r = _ref(v, 0.25, 2.0, True, 0.5)
    loss, dz = _run({**v, "z": wide[:, zx:]}, 0.25, 2.0, True, 0.5, dlogits=out[:, :c])
    torch.cuda.synchronize()
    r.check(loss, dz)
    assert torch.all(out[:, c:] == 3.0)
    z = wide[:, zx:]
    loss2, _ = _run({**v, "z": z}, 0.25, 2.0, True, 0.5, dlogits=z)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(z, dz) and bool(torch.isnan(wide[:, :zx]).all())


@gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [6, 300, 5000, 70000, 140000])
@pytest.mark.parametrize("T,rest,alpha", [(1.0, False, 1.0), (2.0, True, 0.6), (1.0, True, 0.5), (1.5, True, 0.4)])
def test_lists_and_masks(dt, c, T, rest, alpha):
    """Rows whose lists are short, empty, doubled or all -inf, whose logits are masked, far apart or
    not finite, whose labels are outside and whose weight is zero, one kind a row."""
    say("distill special", dt, c, T, rest, alpha)
    k = 6
    v = _case(c, 20, c, k, dt, F32, T)
    z, idx, t, lse, labels, weight = (v[q] for q in ("z", "idx", "t", "lse", "labels", "weight"))
    weight.fill_(1.0)
    inside = idx[:, 0].clone()
    idx[0, 3:] = -1                                    # a shorter list
    idx[1] = -1                                        # no list
    idx[2, 0], idx[2, 4] = c, 2 ** 31 - 1              # entries outside
    idx[3, 3], idx[3, 5] = idx[3, 0], idx[3, 0]        # a class listed three times
    idx[4] = idx[4, 2]                                 # one class only
    t[5, :2] = -INF                                    # entries without probability
    t[6] = -INF
    keep = idx[7].long()
    m = torch.full((c,), True, device=DEV)
    m[keep] = False
    z[7, m] = -INF                                     # only the listed classes are allowed
    z[8, idx[8, 1].long()] = -INF                      # a listed class is not
    z[9] = torch.where(m, torch.finfo(dt).min, z[9].float()).to(dt)      # masked by the lowest value
    z[10] = torch.finfo(dt).min                        # all of it the lowest value: uniform
    z[11] = -INF                                       # nothing allowed
    z[12, int(idx[12, 0])] = float("nan")
    z[13, (int(idx[13, 0]) + 1) % c] = INF
    z[14, idx[14].long()] += 300.0                     # the others underflow next to the listed
    z[15, idx[15].long()] -= 300.0                     # and the other way round
    labels[16] = c
    labels[17] = -1
    z[18], weight[18] = float("nan"), 0.0              # a padding row
    labels[18], idx[18] = -5, 2 ** 31 - 1
    lse[19] = torch.logsumexp(t[19].double() / T, 0).float() - 1e-3       # the list holds more than all: no rest
    labels[7], labels[9] = inside[7].to(torch.int32), idx[7, 0]
    v["bias"][:] = 0.25
    r = _ref(v, 0.5, T, rest, alpha)
    loss, dz = _run(v, 0.5, T, rest, alpha)
    torch.cuda.synchronize()
    if rest and c > k:
        # q_r = 0 where p_r > 0: the loss is infinite
        assert math.isinf(float(loss[7]))
    assert float(loss[18]) == 0.0 and not dz[18].any()
    r.check(loss, dz)


# ----------------------------------------------------------------------------- finite masks
def _masks(T):
    """Finite values that put a class out of play, from the ordinary ones to past 1e30, and both sides of
    2^24 steps of the exponents."""
    near = 2.0 ** 24 * math.log(2) * min(T, 1.0)
    return [-0.99 * near, -1.02 * near, -1e8, -1e9, -1e10, -1e12, -1e15, -1e20, -1e25, -1e30, -1.5e30]


REST, ALL, FIRST, MOST, LAST, HALF, HIGH, LIST = range(8)


def _masked_rows(c, dt, T, rest, alpha, copies=1, masks=None):
    """Inputs with a row per mask and place of it, and their reference: the formula's values on logits with
    the same probabilities that are small (a class that a mask puts out of play has less than e^-150, which
    no bound can see, whatever the mask's size), and the loss by the masks themselves."""
    masks, k = masks or _masks(T), 6
    n = len(masks) * 8 * copies
    v = _case(c + 7, n, c, k, dt, F32, T)
    v["weight"].fill_(1.0)
    v["bias"][:] = 0.25
    row = torch.arange(n, device=DEV)
    kind, M = row % 8, torch.tensor(masks, device=DEV)[row // 8 % len(masks)][:, None]
    idx, j = v["idx"].long(), torch.arange(c, device=DEV)[None]
    K = torch.zeros(n, c, dtype=torch.bool, device=DEV).scatter_(1, idx, True)
    is_ = lambda q: (kind == q)[:, None]                          # noqa: E731
    hit = torch.rand(n, c, generator=torch.Generator(device=DEV).manual_seed(c), device=DEV) < 0.5
    out = (is_(REST) | is_(HIGH) | (is_(FIRST) & (j < c // 2)) | (is_(MOST) & (j < c - 3)) | (is_(LAST) & (j >= c // 3)) |
           (is_(HALF) & hit)) & ~K
    out = out | is_(ALL) | (is_(LIST) & K)
    # the label: listed, or (where the list is masked; where the rest is, every other row) the first class that is not
    other = torch.argmax((~K).int(), 1)
    masked_label = (kind == REST) & (row // 8 % 2 == 1)
    v["labels"] = torch.where((kind == LIST) | masked_label, other, idx[:, 0]).to(torch.int32)
    z = v["z"].float()
    far = 150.0 * max(T, 1.0)
    low = torch.where(is_(REST) | is_(LIST), z.amin(1, keepdim=True) - far,
                      torch.where(is_(HIGH), z.amax(1, keepdim=True) + far, torch.where(is_(ALL), 0.0, -INF)))
    args = (v["idx"], v["t"], 0.5, T, v["lse"] if rest else None, v["labels"], alpha, v["weight"], v["bias"])
    r = Ref(torch.where(out, low, z), *args)
    v["z"] = torch.where(out, torch.where(is_(HIGH), -M, M), z).to(dt)
    true = Ref(v["z"], *args)
    # the loss by the masks: a probability, off by eP, times a difference D / T that is rounded by less than 8 half
    # steps (of the operands, the difference, the quotient, the sum with the logarithms and the product)
    t = v["t"].double() / T
    p = torch.exp(t - v["lse"].double()[:, None]).sum(1) if rest else torch.ones(n, dtype=torch.float64, device=DEV)
    rp = U * (6 * t.abs().amax(1) + (v["lse"].double().abs() if rest else 2 * t.abs().amax(1)) + k + 16)
    pr = torch.clamp(1 - p, min=0) if rest else torch.zeros_like(p)
    epr = rp * p + (k + 2) * U if rest else torch.zeros_like(p)
    D = v["z"].double().abs().amax(1) + 50.0
    soft = torch.where(kind == REST, epr + 8 * U * pr, torch.where((kind == HIGH) | (kind == LIST), p * (rp + 8 * U), 0.0))
    hard = torch.where(masked_label | (kind == HIGH), 4 * U, 0.0) if alpha < 1 else 0.0
    by_mask = (kind == REST) | (kind == HIGH) | (kind == LIST)
    r.loss = torch.where(by_mask, true.loss, r.loss)
    r.eloss = r.eloss + torch.where(by_mask, D * (alpha * T * soft + (1 - alpha) * hard) + 16 * U * true.loss.abs(), 0.0)
    return v, r


@gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c,copies", [(40, 1), (300, 1), (5000, 1), (24001, 4), (41003, 4), (70001, 1), (140000, 1), (300007, 1)])
@pytest.mark.parametrize("T,rest,alpha", [(1.0, False, 1.0), (1.0, True, 0.5), (2.0, True, 0.6), (4.0, True, 0.5),
                                          (1.5, True, 0.4), (0.01, True, 1.0), (0.01, True, 0.5)])
def test_finite_masks(dt, c, copies, T, rest, alpha):
    """Classes masked by a finite value of any size: outside the list, throughout, in blocks and scattered; the
    list itself; and logits as far above the others.  (copies: more rows than compute units.)"""
    say("distill finite masks", dt, c, T, rest, alpha)
    T = float(np.float32(T))
    v, r = _masked_rows(c, dt, T, rest, alpha, copies)
    loss, dz = _run(v, 0.5, T, rest, alpha)
    z = v["z"].clone()
    loss2, dz2 = _run({**v, "z": z}, 0.5, T, rest, alpha, dlogits=z)
    torch.cuda.synchronize()
    r.check(loss, dz)
    assert torch.equal(loss, loss2) and torch.equal(dz, dz2)


@gpu
@pytest.mark.parametrize("dt", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("c", [40, 5000, 70001, 140000])
@pytest.mark.parametrize("T,rest,alpha", [(0.5, True, 1.0), (0.5, False, 0.5), (0.01, True, 0.6), (1.0, False, 0.5)])
def test_lowest_masks(dt, c, T, rest, alpha):
    """The type's lowest (and largest) values where x / T, or a sum of their shares, has no fp32 value, but the loss has."""
    say("distill lowest masks", dt, c, T, rest, alpha)
    T = float(np.float32(T))
    v, r = _masked_rows(c, dt, T, rest, alpha, masks=[torch.finfo(dt).min, torch.finfo(dt).min / 2])
    loss, dz = _run(v, 0.5, T, rest, alpha)
    torch.cuda.synchronize()
    r.check(loss, dz)


@gpu
@pytest.mark.parametrize("dt,n,c", [(BF16, 300, 41003), (BF16, 257, 65535), (F32, 300, 20490), (F32, 257, 32767), (BF16, 256, 50001)])
@pytest.mark.parametrize("T,rest,alpha", [(1.0, False, 1.0), (2.0, True, 0.6), (4.0, True, 0.5), (1.5, True, 0.4)])
def test_more_rows_than_compute_units(dt, n, c, T, rest, alpha):
    say("distill rows", dt, n, c, T, rest, alpha)
    v = _case(n + c, n, c, 9, dt, F32, T)
    loss, dz = _run(v, 1.0 / n, T, rest, alpha)
    torch.cuda.synchronize()
    _ref(v, 1.0 / n, T, rest, alpha).check(loss, dz)


@gpu
@pytest.mark.parametrize("T,alpha", [(1.0, 1.0), (2.0, 0.5), (4.0, 0.5), (3.0, 0.5)])
@pytest.mark.parametrize("c", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 300, 1001, 2055, 8193, 20481, 70001, 140001])
def test_rows_between_words(c, T, alpha):
    """Rows of bf16 that begin at odd elements, with the classes at the ends of pieces and of words listed or
    the label."""
    say("distill odd rows", c, T, alpha)
    n = 9
    want = [j for j in (0, 1, 7, 8, 9, 24, 25, 31, 32, 33, 63, 64, c // 2, c - 9, c - 2, c - 1) if 0 <= j < c]
    k = len(want)
    v = _case(c, n, c, 1, BF16, F32, T)
    v["weight"].fill_(1.0)
    v["idx"] = torch.tensor(want, dtype=torch.int32, device=DEV).repeat(n, 1)
    for i in range(k):                                 # row by row one more of them left out (doubles stay doubles)
        v["idx"][i % n, i] = -1
    v["t"] = torch.gather(v["z"].float(), 1, torch.tensor(want, device=DEV).repeat(n, 1)) + 0.5
    v["lse"] = torch.logsumexp(v["t"].double() / T, 1).float() + 0.25
    v["labels"] = torch.tensor([want[(3 * i) % k] for i in range(n)], dtype=torch.int32, device=DEV)
    wide = torch.full((n, c + 4 + c % 2), float("nan"), dtype=BF16, device=DEV)
    out = torch.full((n, c + 5 - c % 2), 3.0, dtype=BF16, device=DEV)
    for at in (1, 2):
        z = wide[:, at:at + c]
        z.copy_(v["z"])
        loss, dz = _run({**v, "z": z}, 0.5, T, True, alpha, dlogits=out[:, at:at + c])
        torch.cuda.synchronize()
        _ref(v, 0.5, T, True, alpha).check(loss, dz, "at %d" % at)
        assert torch.all(out[:, :at] == 3.0) and torch.all(out[:, at + c:] == 3.0)
        out.fill_(3.0)


@gpu
def test_probabilities_of_the_rest():
    """A student that agrees with the teacher has no loss and no gradient, whichever way the mass of the
    rest is spread."""
    n, c, k, T = 4, 3000, 8, 2.0
    v = _case(3, n, c, k, F32, F32, T)
    x = v["z"].double() + v["bias"].double()
    v["t"] = torch.gather(x, 1, v["idx"].long()).float()
    v["lse"] = torch.logsumexp(x / T, 1).float()
    v["weight"].fill_(1.0)
    loss, dz = _run(v, 1.0, T, True, 1.0)
    torch.cuda.synchronize()
    assert float(loss.abs().max()) < 1e-4 and float(dz.abs().max()) < 1e-5


@gpu
def test_two_calls_at_once():
    """Losses on two streams at a time, rows in registers and long ones."""
    jobs = []
    for c in (3000, 140000):
        v = _case(c, 70, c, 9, BF16, F32, 2.0)
        jobs.append((v, _run(v, 0.1, 2.0, True, 0.5), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for v, _, st in jobs:
            st.wait_stream(torch.cuda.current_stream())
            got.append(_run(v, 0.1, 2.0, True, 0.5, stream=st))
    torch.cuda.synchronize()
    for i, (loss, dz) in enumerate(got):
        assert torch.equal(loss, jobs[i % 2][1][0]) and torch.equal(dz, jobs[i % 2][1][1])


@gpu
def test_shapes_and_defaults():
    v = _case(4, 6, 50, 3, F32, F32, 1.0)
    one, d1 = ops.distill_xent(v["z"], v["idx"], v["t"], 1.0)
    two, d2 = ops.distill_xent(v["z"].view(6, 1, 1, 50), v["idx"].view(2, 3, 3), v["t"].view(2, 3, 3), 1.0)
    assert d2.shape == (6, 1, 1, 50) and torch.equal(one, two) and torch.equal(d1, d2.view(6, 50))
    Ref(v["z"], v["idx"], v["t"], 1.0).check(one, d1)
    # labels are not read where alpha is 1
    bad = torch.full((6,), -9, dtype=torch.int32, device=DEV)
    three, d3 = ops.distill_xent(v["z"], v["idx"], v["t"], 1.0, labels=bad)
    assert torch.equal(one, three) and torch.equal(d1, d3)
    none, dn = ops.distill_xent(v["z"][:0], v["idx"][:0], v["t"][:0], 1.0, alpha=0.5, labels=bad[:0])
    assert none.shape == (0,) and dn.shape == (0, 50)
    with pytest.raises(ops.TfkError):
        ops.distill_xent(v["z"], v["idx"], v["t"], 1.0, alpha=0.5)
    with pytest.raises(ops.TfkError):
        ops.distill_xent(v["z"], v["idx"], v["t"], 1.0, temperature=0.0)


@gpu
def test_offsets_past_32_bits():
    """More than 2^31 logits: the last rows are as they are alone."""
    n, c, k = 16400, 131075, 4
    z = torch.zeros(n, c, dtype=BF16, device=DEV)
    v = _case(6, 2, c, k, BF16, F32, 1.0)
    z[-2:] = v["z"]
    idx = torch.zeros(n, k, dtype=torch.int32, device=DEV)
    t = torch.zeros(n, k, device=DEV)
    idx[-2:], t[-2:] = v["idx"], v["t"]
    weight = torch.zeros(n, device=DEV)
    weight[-2:] = 1.0
    loss, _ = ops.distill_xent(z, idx, t, 1.0, weight=weight, dlogits=z)
    one, dz = ops.distill_xent(v["z"], v["idx"], v["t"], 1.0)
    torch.cuda.synchronize()
    assert torch.equal(loss[-2:], one) and torch.equal(z[-2:], dz) and not z[:-2:997].any()


# ----------------------------------------------------------------------------- together
def _half(x, dt):
    return torch.finfo(dt).eps / 2 * x.abs()


@gpu
@pytest.mark.parametrize("n,d,vocab", [(96, 64, 704), (509, 128, 5003)])
def test_language_model_step(n, d, vocab):
    """Token lookup, distilled head and sparse table update as one training step: each part against the
    formula on what it was given, then the whole as a captured graph and a recorded program, replayed
    with new tokens between eager steps."""
    say("lm step", n, d, vocab)
    rng = np.random.default_rng(n)
    table = EmbeddingTable(rng.standard_normal((vocab, d)) / math.sqrt(d), lr=0.5, scale=math.sqrt(d))
    head = FullSoftmaxHead(rng.standard_normal((vocab, d)) / math.sqrt(d), rng.standard_normal(vocab) * 0.1, lr=0.1)
    k, T, alpha = 8, 2.0, 0.75
    ids = torch.zeros(n, dtype=torch.int32, device=DEV)
    v = dict(idx=torch.zeros(n, k, dtype=torch.int32, device=DEV), t=torch.zeros(n, k, device=DEV),
             lse=torch.zeros(n, device=DEV), labels=torch.zeros(n, dtype=torch.int32, device=DEV),
             weight=torch.ones(n, device=DEV))

    def fill(seed):
        r = np.random.default_rng(seed)
        w = np.minimum((np.exp(r.random(n) * np.log(vocab + 1.0)) - 1).astype(np.int64), vocab - 1).astype(np.int32)
        pad = r.random(n) < 0.1
        w[pad] = -1
        ids.copy_(torch.from_numpy(w))
        idx = np.stack([r.permutation(vocab)[:k] for _ in range(n)]).astype(np.int32)
        v["idx"].copy_(torch.from_numpy(idx))
        t = r.standard_normal((n, k)) * 2 + 3
        v["t"].copy_(torch.from_numpy(t.astype(np.float32)))
        v["lse"].copy_(torch.from_numpy((np.log(np.exp(t / T).sum(1)) + 0.2).astype(np.float32)))
        v["labels"].copy_(torch.from_numpy(r.integers(0, vocab, n).astype(np.int32)))
        v["weight"].copy_(torch.from_numpy(1.0 - pad.astype(np.float32)))

    state = [table.W, table.W_lp, head.W, head.W_lp, head.b]
    start = [s.clone() for s in state]

    def reset():
        for s, s0 in zip(state, start):
            s.copy_(s0)

    def step():
        h = table.lookup(ids)
        loss, dh = head.run_distill(h, v["idx"], v["t"], T, top_lse=v["lse"], labels=v["labels"], alpha=alpha,
                                    weight=v["weight"])
        table.update(ids, dh)
        return h, loss, dh

    fill(0)
    h, loss, dh = step()
    torch.cuda.synchronize()
    ok = ids >= 0
    want_h = (start[1].double()[ids.clamp(min=0).long()] * table.scale).float().to(BF16)
    want_h[~ok] = 0
    assert torch.equal(h, want_h)
    # the head keeps its logits in bf16: the loss and dh follow from logits that are off by half a step,
    # which moves a log-softmax by at most twice the largest such step, and p by that share of itself
    z = h.double() @ start[3].double()
    r = Ref(z, v["idx"], v["t"], 1.0 / n, T, v["lse"], v["labels"], alpha, v["weight"], start[4])
    E = _half(z, BF16).amax(1) + d * U * (h.double().abs() @ start[3].double().abs()).amax(1)
    # soft: T^2 of a term that moves by 2 E / T for every unit of probability, hard: 2 E
    le = v["weight"].double() * (alpha * T * T * 2 * E / T * 2 + (1 - alpha) * 2 * E)
    assert torch.all((loss.double() - r.loss).abs() <= le + r.eloss)
    x = z + start[4].double()
    # q and the shares of the rest move by at most exp(2 E / T) - 1 of themselves, softmax(x) by exp(2 E) - 1
    eg = v["weight"].double()[:, None] / n * (alpha * T * torch.expm1(4 * E / T)[:, None] * (r.q + r.share)
                                              + (1 - alpha) * torch.expm1(2 * E)[:, None] * torch.softmax(x, 1)) + r.egrad
    eg = eg + _half(r.grad.abs() + eg, BF16)
    want = r.grad @ start[3].double().t()
    e_dh = eg @ start[3].double().abs().t() + vocab * U * (r.grad.abs() @ start[3].double().abs().t())
    assert torch.all((dh.double() - want).abs() <= e_dh + _half(want.abs() + e_dh, BF16))
    # the table: exactly the rows of the batch's tokens, by the gradient that the head returned
    i = ids.long()[ok]
    s = torch.zeros(vocab, d, dtype=torch.float64, device=DEV).index_add_(0, i, dh.double()[ok])
    a = torch.zeros_like(s).index_add_(0, i, dh.double()[ok].abs())
    cnt = torch.bincount(i, minlength=vocab).double()[:, None]
    refW = start[0].double() - table.lr * table.scale * s
    assert torch.all((table.W.double() - refW).abs() <= (cnt + 2) * U * table.lr * table.scale * a + U * refW.abs() * 1.001)
    assert torch.equal(table.W_lp, table.W.to(BF16)) and torch.equal(table.W[cnt[:, 0] == 0], start[0][cnt[:, 0] == 0])

    prog = ops.Program()
    with prog.recording():
        kept = step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(1, 4):
        fill(turn)
        reset()
        eager = step()
        torch.cuda.synchronize()
        after = [s.clone() for s in state]
        for again, res in ((graph.replay, out), (prog.run, kept)):
            reset()
            again()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(res, eager))
            assert all(torch.equal(p, q) for p, q in zip(state, after))
    prog.close()


@gpu
def test_full_softmax_step_is_what_it_was():
    """The head's step with labels, against the same calls made one by one."""
    rng = np.random.default_rng(2)
    n, d, vocab = 64, 64, 512
    W, b = rng.standard_normal((vocab, d)) * 0.1, rng.standard_normal(vocab) * 0.1
    head = FullSoftmaxHead(W, b, lr=0.1)
    h = torch.from_numpy(rng.standard_normal((n, d))).to(BF16).to(DEV)
    labels = torch.from_numpy(rng.integers(0, vocab, n).astype(np.int32)).to(DEV)
    w4 = head.W_lp.clone().view(1, 1, d, vocab)
    b0, W0 = head.b.clone(), head.W.clone()
    loss, dh = head.run(h, labels)
    z = ops.conv2d_fwd(h.view(n, 1, 1, d), w4, 1, (0, 0, 0, 0))
    want, dz = ops.softmax_xent(z, labels, 1.0 / n, bias=b0)
    dx = ops.conv2d_bwd_input(dz, w4, torch.empty_like(h.view(n, 1, 1, d)), 1, (0, 0, 0, 0))
    dw = ops.conv2d_bwd_filter(h.view(n, 1, 1, d), dz, (1, 1), 1, (0, 0, 0, 0))
    ops.apply_sgd(W0.view(-1), dw.view(-1), head.lr)
    torch.cuda.synchronize()
    assert torch.equal(loss, want) and torch.equal(dh, dx.view(n, d)) and torch.equal(head.W, W0)
