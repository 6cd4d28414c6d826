"""The language-model operators of this framework as cases that can be timed and compared: the embedding
table's lookup, gradient and update, and the distillation loss from a teacher's top logits.

``own`` False computes each in its plain form (elementary torch operations in fp32, rounded once);
``own`` True makes the calls of a training program on the same inputs and buffers.

Kinds of cases:

* ``lookup``: out[i] = scale * table[ids[i]], zero rows for padding ids.
* ``grad``: the dense gradient of the table, fp32 (beta 1 adds to a gradient that is there already).
* ``sgd``: the table's update by its tokens' gradients, fp32 variable and bf16 copy, in place.
* ``distill``: loss per row and logit gradient of alpha T^2 KL(teacher || student) + (1 - alpha)
  cross-entropy, the teacher given by its k largest logits (renormalised, or with the rest of its mass
  as one more class: ``rest``).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
LR = 0.05


# ----------------------------------------------------------------------------- the cases
def listed():
    return [
        # one time step of a recurrent language model's batch: 128 tokens (latency)
        dict(name="lookup_128", kind="lookup", n=128, d=512, rows=40000, dtype="bf16", out="bf16"),
        # ragged fp32 rows, as a model trained in single precision has them
        dict(name="lookup_f32_ragged", kind="lookup", n=20011, d=771, rows=50021, dtype="f32", out="f32"),
        # the tokens of a large batch, wide rows
        dict(name="lookup_64k", kind="lookup", n=65536, d=2048, rows=131072, dtype="bf16", out="bf16"),
        # 128 sequences x 20 steps over 40 000 words: the table's dense gradient
        dict(name="grad_lm", kind="grad", n=2560, d=512, rows=40000, dtype="bf16", beta=0),
        # ragged, fp32, added to the gradient that the tied head left
        dict(name="grad_f32_ragged", kind="grad", n=5003, d=333, rows=20011, dtype="f32", beta=1),
        # the dense gradient of a large batch over a large vocabulary
        dict(name="grad_64k", kind="grad", n=65536, d=1024, rows=131072, dtype="bf16", beta=0),
        # 128 sequences x 20 steps: the sparse update of one training step
        dict(name="sgd_lm", kind="sgd", n=2560, d=512, rows=40000, dtype="bf16"),
        # the sparse update of a large batch over a large vocabulary
        dict(name="sgd_64k", kind="sgd", n=65536, d=1024, rows=131072, dtype="bf16"),
        # an image classifier of 1000 classes, batch 128, fp32 logits, with its labels
        dict(name="distill_1000", kind="distill", n=128, c=1000, k=5, dtype="f32", top="f32", T=4.0, alpha=0.9,
             hard=True, rest=False),
        # 128 sequences x 20 steps over 40 000 words, teacher's 32 largest logits
        dict(name="distill_lm", kind="distill", n=2560, c=40000, k=32, dtype="bf16", top="bf16", T=2.0, alpha=1.0,
             hard=False, rest=False),
        # rows that no vector load is aligned to, the rest of the teacher's mass as one class
        dict(name="distill_ragged", kind="distill", n=1021, c=50021, k=20, dtype="bf16", top="f32", T=1.0, alpha=1.0,
             hard=False, rest=True),
        # a large batch over a large vocabulary, with labels and the rest of the teacher's mass
        dict(name="distill_131k", kind="distill", n=4096, c=131072, k=64, dtype="bf16", top="bf16", T=2.0, alpha=0.7,
             hard=True, rest=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Row widths as tables have them: mostly whole multiples of 64 or 8, now and then any number."""
    d = _log(rng, lo, hi)
    u = rng.random()
    step = 1 if u < 0.25 else (8 if u < 0.4 else 64)
    return max(step, (d + step // 2) // step * step)


def draw(rng):
    most = {c["name"]: work(c)["bytes"] for c in listed()}
    while True:
        kind = rng.choice(("lookup", "grad", "sgd", "distill", "distill"))
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        if kind == "distill":
            c = _log(rng, 10, 160000)
            hard = rng.random() < 0.5
            case = dict(kind=kind, n=_log(rng, 1, 8192), c=c, k=min(c, _log(rng, 1, 128)), dtype=dtype,
                        top=rng.choice(("bf16", "f32")), T=rng.choice((1.0, 1.5, 2.0, 4.0)),
                        alpha=rng.choice((0.3, 0.5, 0.9)) if hard else 1.0, hard=hard, rest=rng.random() < 0.5)
            if work(case)["bytes"] <= most["distill_131k"]:
                return case
            continue
        case = dict(kind=kind, n=_log(rng, 1, 65536), d=_width(rng, 16, 4096), rows=_log(rng, 100, 200000), dtype=dtype)
        if kind == "lookup":
            case["out"] = dtype if rng.random() < 0.8 else rng.choice(("bf16", "f32"))
            top = most["lookup_64k"]
        elif kind == "grad":
            case["beta"] = int(rng.random() < 0.3)
            top = most["grad_64k"]
        else:
            top = most["sgd_64k"]
        if work(case)["bytes"] <= top:
            return case


# ----------------------------------------------------------------------------- inputs
class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, *shape, scale=1.0):
        return torch.randn(shape, generator=self.g, device=DEV).mul_(scale)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def zipf(self, n, classes):
        """Words of a text: log-uniform frequencies, the most frequent first."""
        w = torch.exp(self.uniform(n).double() * math.log(classes + 1.0)) - 1.0
        return w.long().clamp_(0, classes - 1).to(torch.int32)


def _tokens(r, case):
    """Zipfian token ids; the ends of the shorter sequences are padding (-1), about one in thirty."""
    ids = r.zipf(case["n"], case["rows"])
    return torch.where(r.uniform(case["n"]) < 1 / 30, torch.full_like(ids, -1), ids)


def _distill_inputs(case, seed):
    r, n, c, k = _Rand(seed), case["n"], case["c"], case["k"]
    z = r.normal(n, c, scale=2.0)
    # k distinct classes a row, one in each k-th of them, where teacher and student both see something
    first = torch.arange(k + 1, device=DEV) * c // k
    wide = first[1:] - first[:-1]
    idx = first[:-1] + torch.minimum((r.uniform(n, k).double() * wide).long(), wide - 1)
    z.scatter_add_(1, idx, r.normal(n, k, scale=1.5) + 5.0)
    t = (torch.gather(z, 1, idx) + r.normal(n, k)).sort(dim=1, descending=True)
    idx, t = torch.gather(idx, 1, t.indices), t.values
    # the teacher's log-sum-exp over all its classes at this temperature: the top ones hold most of it
    top = torch.logsumexp(t.double() / case["T"], dim=1)
    lse = (top + 0.02 + 0.5 * r.uniform(n).double()).float()
    labels = torch.where(r.uniform(n) < 0.8, idx[:, 0], r.zipf(n, c).long()).to(torch.int32)
    # teachers that kept fewer classes for a row pad its list with -1
    short = (r.uniform(n, 1) < 0.1) & (torch.arange(k, device=DEV)[None, :] > k // 2)
    idx = torch.where(short, torch.full_like(idx, -1), idx)
    # rows behind the end of a sequence count for nothing
    weight = (r.uniform(n) >= 1 / 30).float()
    return dict(z=z.to(_DT[case["dtype"]]), bias=r.normal(c, scale=0.1), idx=idx.to(torch.int32),
                t=t.to(_DT[case["top"]]), lse=lse if case["rest"] else None, labels=labels if case["hard"] else None,
                weight=weight)


def _inputs(case, seed):
    if case["kind"] == "distill":
        return _distill_inputs(case, seed)
    r, n, d, rows, dt = _Rand(seed), case["n"], case["d"], case["rows"], _DT[case["dtype"]]
    s = dict(ids=_tokens(r, case))
    if case["kind"] == "lookup":
        s["table"] = r.normal(rows, d, scale=1.0 / math.sqrt(d)).to(dt)
        return s
    s["dy"] = r.normal(n, d, scale=1.0 / math.sqrt(n)).to(dt)
    if case["kind"] == "sgd":
        s["W"] = r.normal(rows, d, scale=1.0 / math.sqrt(d))
        s["shadow"] = s["W"].to(torch.bfloat16)
    elif case["beta"]:
        s["dW"] = r.normal(rows, d, scale=1.0 / math.sqrt(n))
    return s


def _scale(case):
    return math.sqrt(case["d"])


# ----------------------------------------------------------------------------- prepare
def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "lookup":
        s["y"] = torch.empty(case["n"], case["d"], dtype=_DT[case["out"]], device=DEV)
    elif case["kind"] == "grad" and not case["beta"]:
        s["dW"] = torch.empty(case["rows"], case["d"], dtype=torch.float32, device=DEV)
    elif case["kind"] == "distill":
        s["loss"] = torch.empty(case["n"], dtype=torch.float32, device=DEV)
        s["dz"] = torch.empty_like(s["z"])
    return s


# ----------------------------------------------------------------------------- run
def _plain_distill(s, case):
    T, alpha = case["T"], case["alpha"]
    n, c = s["z"].shape
    x = s["z"].float() + s["bias"]
    idx = s["idx"].long()
    valid = idx >= 0
    at = idx.clamp(min=0)
    # teacher
    t = torch.where(valid, s["t"].float() / T, torch.full((), -math.inf, device=DEV))
    if case["rest"]:
        logp = t - s["lse"][:, None]
        p_r = (1.0 - torch.exp(logp).sum(1)).clamp_(min=0.0)
    else:
        m = t.amax(1, keepdim=True)
        logp = t - m - torch.log(torch.exp(t - m).sum(1, keepdim=True))
        p_r = torch.zeros(n, device=DEV)
    p = torch.exp(logp)
    # student at temperature T, the teacher's classes and the others apart
    top = torch.zeros(n, c + 1, dtype=torch.bool, device=DEV)
    top.scatter_(1, torch.where(valid, idx, torch.full_like(idx, c)), True)
    top = top[:, :c]
    u = x / T
    m = u.amax(1, keepdim=True)
    e = torch.exp(u - m)
    total = e.sum(1)
    others = torch.where(top, torch.zeros((), device=DEV), e).sum(1)
    q = e / total[:, None]
    del e
    q_r = others / total
    logq = torch.gather(u, 1, at) - m - torch.log(total)[:, None]
    del u
    soft = torch.where(p > 0, p * (logp - logq), torch.zeros((), device=DEV)).sum(1)
    soft = soft + torch.where(p_r > 0, p_r * (torch.log(p_r) - torch.log(q_r)), torch.zeros((), device=DEV))
    ratio = torch.where(q_r > 0, 1.0 - p_r / q_r, torch.zeros((), device=DEV))
    g = torch.where(top, q, q * ratio[:, None])
    del q, top
    g.scatter_add_(1, at, torch.where(valid, -p, torch.zeros((), device=DEV)))
    loss, g = alpha * T * T * soft, g.mul_(alpha * T)
    if case["hard"]:
        lab = s["labels"].long()[:, None]
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        total = e.sum(1, keepdim=True)
        loss = loss + (1.0 - alpha) * (m + torch.log(total) - torch.gather(x, 1, lab))[:, 0]
        g.add_(e.div_(total), alpha=1.0 - alpha)
        g.scatter_add_(1, lab, torch.full(lab.shape, alpha - 1.0, device=DEV))
    g.mul_((s["weight"] / n)[:, None])
    return dict(loss=loss * s["weight"], dz=g.to(s["z"].dtype))


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if own:
        from paper_1605_08695_amd import ops
        if kind == "lookup":
            return ops.embedding_fwd(s["table"], s["ids"], scale=_scale(case), out=s["y"])
        if kind == "grad":
            return ops.embedding_bwd(s["dy"], s["ids"], case["rows"], scale=_scale(case), dtable=s["dW"],
                                     beta=float(case["beta"]))
        if kind == "sgd":
            ops.embedding_apply_sgd(s["W"], s["ids"], s["dy"], LR, scale=_scale(case), shadow=s["shadow"])
            return dict(W=s["W"], shadow=s["shadow"])
        loss, dz = ops.distill_xent(s["z"], s["idx"], s["t"], 1.0 / case["n"], temperature=case["T"], top_lse=s["lse"],
                                    labels=s["labels"], alpha=case["alpha"], weight=s["weight"], bias=s["bias"],
                                    loss=s["loss"], dlogits=s["dz"])
        return dict(loss=loss, dz=dz)
    if kind == "distill":
        return _plain_distill(s, case)
    valid = (s["ids"] >= 0)[:, None]
    at = s["ids"].clamp(min=0).long()
    if kind == "lookup":
        y = s["table"][at].float() * _scale(case)
        return torch.where(valid, y, torch.zeros((), device=DEV)).to(_DT[case["out"]])
    dy = torch.where(valid, s["dy"].float() * _scale(case), torch.zeros((), device=DEV))
    if kind == "grad":
        dW = s["dW"] if case["beta"] else s["dW"].zero_()
        return dW.index_add_(0, at, dy)
    s["W"].index_add_(0, at, dy, alpha=-LR)
    s["shadow"][at] = s["W"][at].to(torch.bfloat16)
    return dict(W=s["W"], shadow=s["shadow"])


# ----------------------------------------------------------------------------- work
def _distinct(n, rows):
    """Expected distinct words among n Zipfian tokens."""
    i = np.arange(rows, dtype=np.float64)
    p = np.log((i + 2.0) / (i + 1.0)) / math.log(rows + 1.0)
    return float(np.sum(-np.expm1(n * np.log1p(-p))))


def work(case):
    if case["kind"] == "distill":
        n, c, k = case["n"], case["c"], case["k"]
        el = _SIZE[case["dtype"]]
        by = 2 * n * c * el + n * k * (4 + _SIZE[case["top"]]) + 4 * c + 4 * n * (2 + int(case["hard"]) + int(case["rest"]))
        return dict(bytes=by, flops=(8.0 + 4.0 * (case["hard"] and case["T"] != 1.0)) * n * c)
    n, d, rows = case["n"], case["d"], case["rows"]
    u, el = min(n, _distinct(n, rows)), _SIZE[case["dtype"]]
    if case["kind"] == "lookup":
        return dict(bytes=4 * n + u * d * el + n * d * _SIZE[case["out"]], flops=float(n) * d)
    by = 4 * n + n * d * el
    if case["kind"] == "grad":
        return dict(bytes=by + (2 * u if case["beta"] else rows) * d * 4, flops=2.0 * n * d)
    return dict(bytes=by + u * d * (4 + 4 + 2), flops=2.0 * n * d)


# ----------------------------------------------------------------------------- exact
def _exact_distill(case, seed):
    """Row block by row block, each class's share of the loss and its gradient by the definitions."""
    s = _distill_inputs(case, seed)
    n, c, T, a = case["n"], case["c"], case["T"], case["alpha"]
    loss = torch.zeros(n, dtype=torch.float64, device=DEV)
    dz = torch.zeros(n, c, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // c)
    for r0 in range(0, n, step):
        rows = slice(r0, min(n, r0 + step))
        x = s["z"][rows].double() + s["bias"].double()
        pick = s["idx"][rows].long()
        t = s["t"][rows].double() / T
        row, col = torch.nonzero(pick >= 0, as_tuple=True)
        cls = pick[row, col]
        logp = torch.full_like(x, -math.inf)             # the teacher's log-probability, class by class
        logp[row, cls] = t[row, col]
        if case["rest"]:
            logp -= s["lse"][rows].double()[:, None]
        else:
            logp -= torch.logsumexp(logp, 1, keepdim=True)
        p = torch.exp(logp)
        listed_ = torch.zeros_like(x, dtype=torch.bool)
        listed_[row, cls] = True
        logq = torch.log_softmax(x / T, 1)
        kl = torch.where(listed_ & (p > 0), p * (logp - logq), torch.zeros_like(x)).sum(1)
        g = torch.exp(logq) - p
        if case["rest"]:
            pr = torch.clamp(1.0 - p.sum(1), min=0.0)
            logqr = torch.logsumexp(torch.where(listed_, torch.full_like(x, -math.inf), logq), 1)
            kl += torch.where(pr > 0, pr * (torch.log(pr) - logqr), torch.zeros_like(pr))
            # within the rest the teacher's mass goes by the student's own shares
            inside = torch.where(torch.isfinite(logqr)[:, None], torch.exp(logq - logqr[:, None]), torch.zeros_like(x))
            g -= torch.where(listed_, torch.zeros_like(x), pr[:, None] * inside)
        out, g = a * T * T * kl, a * T * g
        if case["hard"]:
            lab = s["labels"][rows].long()
            lsm = torch.log_softmax(x, 1)
            each = torch.arange(lab.numel(), device=DEV)
            out = out - (1.0 - a) * lsm[each, lab]
            g += (1.0 - a) * torch.exp(lsm)
            g[each, lab] -= 1.0 - a
        w = s["weight"][rows].double()
        loss[rows] = w * out
        dz[rows] = g * (w / n)[:, None]
    return dict(loss=loss, dz=dz)


def exact(case, seed):
    if case["kind"] == "distill":
        return _exact_distill(case, seed)
    s = _inputs(case, seed)
    rows, d = case["rows"], case["d"]
    here = torch.nonzero(s["ids"] >= 0)[:, 0]
    at = s["ids"][here].long()
    if case["kind"] == "lookup":
        y = torch.zeros(case["n"], d, dtype=torch.float64, device=DEV)
        y[here] = torch.index_select(s["table"], 0, at).double() * _scale(case)
        return y
    # the sum over each row's tokens, column block by column block: tokens grouped by row, then
    # differences of running sums (about 2^16 terms, so 64 bits keep ten digits)
    order = torch.argsort(at, stable=True)
    words, count = torch.unique_consecutive(at[order], return_counts=True)
    end = torch.cumsum(count, 0)
    total = torch.zeros(rows, d, dtype=torch.float64, device=DEV)
    for c0 in range(0, d, 256):
        run_ = torch.cumsum(s["dy"][here[order], c0:c0 + 256].double(), 0)[end - 1] if at.numel() else None
        if run_ is not None:
            total[words, c0:c0 + 256] = torch.diff(run_, dim=0, prepend=torch.zeros_like(run_[:1]))
    total *= _scale(case)
    if case["kind"] == "grad":
        return total + s["dW"].double() if case["beta"] else total
    W = s["W"].double() - LR * total
    shadow = s["shadow"].double()
    shadow[words] = W[words]
    return dict(W=W, shadow=shadow)
