"""What a recurrent language model runs between its embedding table and its softmax head, after the head and at
the end of a step, as cases that can be timed and compared: a gated linear recurrence (training, whole prompts,
single tokens), log-probabilities of given tokens with the entropy and the largest alternatives (and their
gradient), and an AdamW step over all variables at once with its states in 32 or in 8 bits.

``own`` False computes each in its plain form (elementary torch operations in fp32, rounded once);
``own`` True makes the calls of a program on the same inputs and buffers.

Kinds of cases:

* ``scan``: x, f, o the column blocks of z + bias; h_t = s(f) h_(t-1) + (1 - s(f)) x, y = h or s(o) h, s the
  logistic function; sequences of ragged lengths in one padded batch, batch or time first.  ``train``: y, the last
  states and the gradients of z and of the first states; else y and the last states.
* ``step``: one token of each of n sequences, their states in a cache of more slots.
* ``score``: log-probability of each row's token, entropy, log-sum-exp and the k largest classes with their
  log-probabilities.  ``train``: the logits' gradient for given gradients of the log-probability and the entropy.
* ``adamw``: variables, moments and bf16 copies in place; 8-bit moments are e4m3 values times one fp32 scale for
  each 256, the second moment as its square root.
"""
import math
import random

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f32": 4}
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.99, 1e-8, 1e-3, 0.1


# ----------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of each of 128 sequences being served, their states among 1024 slots (latency)
        dict(name="step_128", kind="step", n=128, d=512, slots=1024, gates=3, dtype="bf16"),
        # 128 sequences x 20 steps, the steps of truncated backpropagation, time first
        dict(name="scan_train_lm", kind="scan", b=128, t=20, d=512, gates=3, dtype="bf16", train=True, ragged=False,
             first="t"),
        # a few prompts of different lengths read in, fp32 rows that no vector load is aligned to
        dict(name="scan_prefill_ragged", kind="scan", b=5, t=5003, d=771, gates=2, dtype="f32", train=False, ragged=True,
             first="b"),
        # a training batch of ordinary documents, padded to the longest
        dict(name="scan_train_4k", kind="scan", b=8, t=4096, d=2048, gates=2, dtype="bf16", train=True, ragged=True,
             first="b"),
        # one very long document, few channels: the time axis is all there is to share out
        dict(name="scan_train_64k", kind="scan", b=1, t=65536, d=768, gates=3, dtype="bf16", train=True, ragged=False,
             first="b"),
        # 16 sequences being served over a large vocabulary, half of it ruled out: the 20 largest to choose from
        dict(name="score_decode", kind="score", n=16, c=131072, k=20, dtype="bf16", T=0.8, tokens=False, masked=True,
             bias=False, train=False),
        # a teacher's 32 largest classes at temperature 2 for 128 sequences x 20 steps over 40 000 words
        dict(name="score_lm", kind="score", n=2560, c=40000, k=32, dtype="bf16", T=2.0, tokens=True, masked=False,
             bias=True, train=False),
        # ragged fp32 rows, trained on their tokens' log-probabilities and the entropy
        dict(name="score_train_ragged", kind="score", n=1021, c=50021, k=5, dtype="f32", T=1.0, tokens=True,
             masked=False, bias=True, train=True),
        # a large batch over a large vocabulary, trained on log-probabilities
        dict(name="score_train_131k", kind="score", n=4096, c=131072, k=0, dtype="bf16", T=1.0, tokens=True,
             masked=False, bias=True, train=True),
        # the variables of one recurrent layer, fp32 moments (latency)
        dict(name="adamw_layer", kind="adamw", count=2, total=787968, spread="layer", bits=32),
        # the filters and biases of a deep image model: 190 variables from 64 values up, fp32 moments
        dict(name="adamw_many", kind="adamw", count=190, total=24000000, spread="many", bits=32),
        # a language model over a large vocabulary, moments in 8 bits
        dict(name="adamw8_lm", kind="adamw", count=9, total=277000003, spread="lm", bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths as layers have them: mostly whole multiples of 64 or 8, now and then any number."""
    d = _log(rng, lo, hi)
    u = rng.random()
    step = 1 if u < 0.25 else (8 if u < 0.4 else 64)
    return max(step, (d + step // 2) // step * step)


def draw(rng):
    most = {c["name"]: work(c)["bytes"] for c in listed()}
    while True:
        kind = rng.choice(("scan", "scan", "step", "score", "score", "adamw"))
        dtype = "f32" if rng.random() < 0.3 else "bf16"
        if kind == "scan":
            case = dict(kind=kind, b=_log(rng, 1, 128), t=_log(rng, 1, 65536), d=_width(rng, 16, 4096),
                        gates=rng.choice((2, 3)), dtype=dtype, train=rng.random() < 0.6, ragged=rng.random() < 0.5,
                        first=rng.choice("bt"))
            top = most["scan_train_64k"]
        elif kind == "step":
            n = _log(rng, 1, 4096)
            case = dict(kind=kind, n=n, d=_width(rng, 16, 4096), slots=n + _log(rng, 1, 2048), gates=rng.choice((2, 3)),
                        dtype=dtype)
            top = most["scan_train_64k"]
        elif kind == "score":
            c, train = _log(rng, 10, 160000), rng.random() < 0.5
            case = dict(kind=kind, n=_log(rng, 1, 8192), c=c, k=min(c, rng.choice((0, _log(rng, 1, 128)))), dtype=dtype,
                        T=rng.choice((0.7, 1.0, 1.5, 2.0)), tokens=train or rng.random() < 0.5,
                        masked=rng.random() < 0.3, bias=rng.random() < 0.5, train=train)
            top = most["score_train_131k"]
        else:
            count = _log(rng, 1, 200)
            case = dict(kind=kind, count=count, total=max(300 * count, _log(rng, 1000, 200000000)), spread="many",
                        bits=rng.choice((8, 32)))
            top = most["adamw8_lm"]
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


def _gate_bias(r, d, gates):
    """Forget gates begin mostly open, with time constants from a few to some hundreds of tokens."""
    return torch.cat([r.normal(d, scale=0.1), 1.0 + 4.0 * r.uniform(d)] + [r.normal(d, scale=0.5)] * (gates - 2))


def _scan_inputs(case, seed):
    r, b, t, d, k, dt = _Rand(seed), case["b"], case["t"], case["d"], case["gates"], _DT[case["dtype"]]
    shape = (b, t) if case["first"] == "b" else (t, b)
    s = dict(z=r.normal(*shape, k * d).to(dt), bias=_gate_bias(r, d, k), h0=r.normal(b, d, scale=0.5))
    s["lengths"] = None
    if case["ragged"]:
        lengths = (t * (0.4 + 0.6 * r.uniform(b))).ceil().to(torch.int32)
        lengths[0] = t
        # a place of the batch that no document was left for
        s["lengths"] = torch.where(torch.arange(b, device=DEV) % 16 == 15, torch.zeros_like(lengths), lengths)
    if case["train"]:
        s["dy"] = r.normal(*shape, d).to(dt)
        s["dh"] = r.normal(b, d)
    if case["first"] == "t":
        for name in ("z", "dy"):
            if name in s:
                s[name] = s[name].transpose(0, 1)
    return s


def _step_inputs(case, seed):
    r, n, d, k = _Rand(seed), case["n"], case["d"], case["gates"]
    slots = torch.randperm(case["slots"], generator=r.g, device=DEV)[:n].to(torch.int32)
    # places of the batch without a sequence
    slots = torch.where(r.uniform(n) < 1 / 30, torch.full_like(slots, -1), slots)
    return dict(z=r.normal(n, k * d).to(_DT[case["dtype"]]), bias=_gate_bias(r, d, k), slots=slots,
                state=r.normal(case["slots"], d, scale=0.5))


def _score_inputs(case, seed):
    r, n, c = _Rand(seed), case["n"], case["c"]
    z = r.normal(n, c, scale=2.0)
    # a few likely classes a row, one in each eighth of them
    likely = torch.arange(8, device=DEV) * c // 8 + (r.uniform(n, 8) * (c // 8)).long()
    z.scatter_add_(1, likely, 4.0 + 3.0 * r.uniform(n, 8))
    tokens = torch.where(r.uniform(n) < 0.7, z.argmax(1), r.zipf(n, c).long())
    if case["masked"]:
        z.masked_fill_((r.uniform(c) < 0.5) & (torch.arange(c, device=DEV) > 0), -math.inf)
    tokens = torch.where(r.uniform(n) < 1 / 30, torch.full_like(tokens, -1), tokens).to(torch.int32)
    s = dict(z=z.to(_DT[case["dtype"]]), bias=r.normal(c, scale=0.1) if case["bias"] else None,
             tokens=tokens if case["tokens"] else None)
    if case["train"]:
        s["dlogp"], s["dentropy"] = r.normal(n, scale=1.0 / n), r.normal(n, scale=0.1 / n)
    return s


def _sizes(case):
    """How many values each variable has."""
    total, count = case["total"], case["count"]
    if case["spread"] == "layer":                    # 512 x 1536 and its bias
        return [512 * 1536, 1536]
    if case["spread"] == "lm":                       # table and head over 131072 words, layers of 1024 and biases
        return [131072 * 1024, 131072 * 1024, 131072] + [1024 * 2048, 2048] * 2 + [1024 * 1024 + 3, 1024]
    rng = random.Random(1000 * count + total % 997)
    w = [math.exp(rng.uniform(math.log(64.0), math.log(2.0e6))) for _ in range(count)]
    left = total - 64 * count
    return [64 + int(left * x / sum(w)) for x in w]


def _spans(sizes, step):
    """First place of each variable in one buffer, a whole number of `step` places apart."""
    at, end = [], 0
    for n in sizes:
        at.append(end)
        end += -(-n // step) * step
    return at, end


def _q8(x):
    """Blocks of 256 values over their scales, so that each block's largest is e4m3's, and the scales."""
    top = x.abs().amax(1)
    y = torch.where(top[:, None] > 0, x * (448.0 / top)[:, None], torch.zeros((), device=DEV))
    return y.clamp_(-448.0, 448.0), top / 448.0


def _decay(sizes):
    """Weight decay of the matrices, none of the biases."""
    return [DECAY if n > 4096 else 0.0 for n in sizes]


def _adamw_inputs(case, seed):
    r, sizes = _Rand(seed), _sizes(case)
    at, end = _spans(sizes, 256)
    inside = torch.zeros(end, dtype=torch.bool, device=DEV)
    decay = torch.zeros(end // 256, device=DEV)
    for a, n, w in zip(at, sizes, _decay(sizes)):
        inside[a:a + n] = True
        decay[a // 256:(a + n + 255) // 256] = w
    s = dict(at=at, sizes=sizes, decay=decay, var=r.normal(end, scale=0.02).mul_(inside))
    size = 1e-3 * torch.exp(2.0 * r.normal(end // 256)).repeat_interleave(256)
    s["grad"] = r.normal(end).mul_(size).mul_(inside)
    m = r.normal(end).mul_(size).mul_(0.3).mul_(inside)
    v = size.square_().mul_(0.3 + r.uniform(end)).mul_(inside)
    s["shadow"] = s["var"].to(torch.bfloat16)
    if case["bits"] == 8:
        y, s["m_scale"] = _q8(m.view(-1, 256))
        s["m"] = y.view(-1).to(torch.float8_e4m3fn)
        y, s["v_scale"] = _q8(v.sqrt_().view(-1, 256))
        s["v"] = y.view(-1).to(torch.float8_e4m3fn)
    else:
        s["m"], s["v"] = m, v
    return s


def _inputs(case, seed):
    return {"scan": _scan_inputs, "step": _step_inputs, "score": _score_inputs, "adamw": _adamw_inputs}[case["kind"]](case, seed)


# ----------------------------------------------------------------------------- prepare
def _views(s, name):
    """Each variable's part of the buffer s[name]."""
    return [s[name][a:a + n] for a, n in zip(s["at"], s["sizes"])]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "adamw":
        s["vars"], s["grads"], s["shadows"] = _views(s, "var"), _views(s, "grad"), _views(s, "shadow")
        s["ms"], s["vs"] = _views(s, "m"), _views(s, "v")
        if case["bits"] == 8:
            blocks = [(a // 256, -(-n // 256)) for a, n in zip(s["at"], s["sizes"])]
            s["m_scales"] = [s["m_scale"][a:a + n] for a, n in blocks]
            s["v_scales"] = [s["v_scale"][a:a + n] for a, n in blocks]
        if own:
            from paper_1605_08695_amd.optim import AdamW
            s["opt"] = AdamW(s["vars"], LR, BETA1, BETA2, EPS, _decay(s["sizes"]), shadows=s["shadows"], bits=case["bits"],
                             moments=(s["ms"], s["vs"], s.get("m_scales"), s.get("v_scales")))
    return s


# ----------------------------------------------------------------------------- run
def _recur(f, b):
    """h_t = f_t h_(t-1) + b_t along dimension 1 from 0: spans of 1, 2, 4 ... tokens joined (f and b are lost)."""
    span = 1
    while span < b.shape[1]:
        b = torch.cat([b[:, :span], torch.addcmul(b[:, span:], f[:, span:], b[:, :-span])], 1)
        f = torch.cat([f[:, :span], f[:, span:] * f[:, :-span]], 1)
        span *= 2
    return b


def _plain_scan(s, case):
    b, t, d, dt = case["b"], case["t"], case["d"], _DT[case["dtype"]]
    zero = torch.zeros((), device=DEV)
    pre = s["z"].float() + s["bias"]
    x, f = pre[..., :d], torch.sigmoid(pre[..., d:2 * d])
    o = torch.sigmoid(pre[..., 2 * d:]) if case["gates"] == 3 else None
    here = None
    if s["lengths"] is not None:
        here = (torch.arange(t, device=DEV)[None, :] < s["lengths"][:, None])[..., None]
    keep = f if here is None else torch.where(here, f, torch.ones((), device=DEV))
    put = (1.0 - f) * x if here is None else torch.where(here, (1.0 - f) * x, zero)
    put = torch.cat([torch.addcmul(put[:, :1], keep[:, :1], s["h0"][:, None]), put[:, 1:]], 1)
    h = _recur(keep, put)
    del put
    y = h if o is None else o * h
    y = (y if here is None else torch.where(here, y, zero)).to(dt)
    out = dict(y=y, last=h[:, -1].clone())
    if not case["train"]:
        return out
    dy = s["dy"].float()
    dy = dy if here is None else torch.where(here, dy, zero)
    dh = dy if o is None else dy * o
    dh = torch.cat([dh[:, :-1], dh[:, -1:] + s["dh"][:, None]], 1)
    after = torch.cat([keep[:, 1:], torch.zeros_like(keep[:, :1])], 1)
    dh = _recur(after.flip(1), dh.flip(1)).flip(1)
    before = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    parts = [(1.0 - f) * dh, f * (1.0 - f) * (before - x) * dh] + ([dy * h * o * (1.0 - o)] if o is not None else [])
    dz = torch.cat(parts, 2)
    out["dz"] = (dz if here is None else torch.where(here, dz, zero)).to(dt)
    out["dfirst"] = keep[:, 0] * dh[:, 0]
    return out


def _plain_step(s, case):
    d = case["d"]
    pre = s["z"].float() + s["bias"]
    at = s["slots"].clamp(min=0).long()
    live = (s["slots"] >= 0)[:, None]
    f = torch.sigmoid(pre[:, d:2 * d])
    h = f * s["state"][at] + (1.0 - f) * pre[:, :d]
    y = h if case["gates"] == 2 else torch.sigmoid(pre[:, 2 * d:]) * h
    rows = torch.nonzero(s["slots"] >= 0)[:, 0]
    s["state"][at[rows]] = h[rows]
    return dict(y=torch.where(live, y, torch.zeros((), device=DEV)).to(s["z"].dtype), state=s["state"])


def _plain_score(s, case):
    k, T = case["k"], case["T"]
    n, c = s["z"].shape
    zero = torch.zeros((), device=DEV)
    x = s["z"].float()
    if s["bias"] is not None:
        x = x + s["bias"]
    live = torch.ones(n, dtype=torch.bool, device=DEV) if s["tokens"] is None else s["tokens"] >= 0
    top = x.amax(1, keepdim=True)
    u = (x - top) / T
    e = torch.exp(u)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total[:, 0] - torch.where(e > 0, e * u, zero).sum(1) / total[:, 0]
    out = dict(entropy=torch.where(live, entropy, zero), lse=torch.where(live, (top / T + log_total)[:, 0], zero))
    if s["tokens"] is not None:
        at = s["tokens"].clamp(min=0).long()[:, None]
        out["logp"] = torch.where(live, (torch.gather(u, 1, at) - log_total)[:, 0], zero)
    if k:
        # the order of the values as whole numbers, then the lower class first
        bits = (x + 0.0).view(torch.int32)
        bits = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * 2 ** 32 + torch.arange(c - 1, -1, -1, device=DEV)
        first = c - 1 - torch.topk(bits, k, 1).values % 2 ** 32
        logp = torch.gather(u, 1, first) - log_total
        there = live[:, None] & (logp > -math.inf)
        out["top_idx"] = torch.where(there, first, torch.full_like(first, -1)).to(torch.int32)
        out["top_logp"] = torch.where(there, logp, torch.full((), -math.inf, device=DEV))
    if case["train"]:
        p = e / total
        logp = u - log_total
        g = torch.where(p > 0, p * (logp + entropy[:, None]), zero).mul_(-s["dentropy"][:, None])
        g.sub_(p * s["dlogp"][:, None])
        g.scatter_add_(1, at, s["dlogp"][:, None])
        out["dz"] = torch.where(live[:, None], g / T, zero).to(s["z"].dtype)
    return out


def _plain_adamw(s, case):
    """All variables at once: what lies between them in the buffers is 0 and stays 0."""
    t = 100
    var, grad, m, v = (s[name].view(-1, 256) for name in ("var", "grad", "m", "v"))
    m1, v1 = m, v
    if case["bits"] == 8:
        m1, v1 = m.float() * s["m_scale"][:, None], (v.float() * s["v_scale"][:, None]).square_()
    m1 = BETA1 * m1 + (1.0 - BETA1) * grad
    v1 = BETA2 * v1 + (1.0 - BETA2) * grad * grad
    step = (m1 / (1.0 - BETA1 ** t)) / (torch.sqrt(v1 / (1.0 - BETA2 ** t)) + EPS)
    var.mul_(1.0 - LR * s["decay"][:, None]).sub_(LR * step)
    s["shadow"].copy_(s["var"])
    if case["bits"] == 32:
        m.copy_(m1)
        v.copy_(v1)
        return
    y, s["m_scale"][:] = _q8(m1)
    m.copy_(y)
    root = torch.sqrt(v1)
    y, s["v_scale"][:] = _q8(root)
    # a second moment that is there never becomes 0
    v.copy_(torch.where(root > 0, y.clamp(min=2.0 ** -9), torch.zeros((), device=DEV)))


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if kind == "adamw":
        if own:
            s["opt"].step(s["grads"], t=100)
        else:
            _plain_adamw(s, case)
        return {name: s[name] for name in ("var", "m", "v", "shadow", "m_scale", "v_scale") if name in s}
    if not own:
        return {"scan": _plain_scan, "step": _plain_step, "score": _plain_score}[kind](s, case)
    from paper_1605_08695_amd import ops
    if kind == "scan":
        gated = case["gates"] == 3
        y, last, saved = ops.gated_scan_fwd(s["z"], output_gate=gated, bias=s["bias"], h0=s["h0"], lengths=s["lengths"],
                                            save=case["train"])
        out = dict(y=y, last=last)
        if case["train"]:
            out["dz"], out["dfirst"] = ops.gated_scan_bwd(s["z"], s["dy"], saved, output_gate=gated, bias=s["bias"],
                                                          lengths=s["lengths"], dh_last=s["dh"])
        return out
    if kind == "step":
        y = ops.gated_scan_step(s["z"], s["state"], slots=s["slots"], output_gate=case["gates"] == 3, bias=s["bias"])
        return dict(y=y, state=s["state"])
    r = ops.token_logprobs(s["z"], tokens=s["tokens"], k=case["k"], temperature=case["T"], bias=s["bias"])
    out = dict(entropy=r.entropy, lse=r.lse)
    if s["tokens"] is not None:
        out["logp"] = r.logp
    if case["k"]:
        out["top_idx"], out["top_logp"] = r.top_idx, r.top_logp
    if case["train"]:
        out["dz"] = ops.token_logprobs_bwd(s["z"], s["tokens"], r.lse, s["dlogp"], entropy=r.entropy,
                                           dentropy=s["dentropy"], temperature=case["T"], bias=s["bias"])
    return out


# ----------------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind == "scan":
        # forward: z read, y written; backward, after the loss has been formed: z and dy read, dz written
        b, t, d, k, el = case["b"], case["t"], case["d"], case["gates"], _SIZE[case["dtype"]]
        cells = b * t * d * (0.7 if case["ragged"] and b > 1 else 1.0)
        by, fl = cells * el * (k + 1) + 8 * b * d, 10.0 * cells
        if case["train"]:
            by, fl = by + cells * el * (2 * k + 1) + 8 * b * d, 4.0 * fl
        return dict(bytes=by, flops=fl)
    if kind == "step":
        n, d, k = case["n"], case["d"], case["gates"]
        return dict(bytes=n * d * ((k + 1) * _SIZE[case["dtype"]] + 8) + 4 * n + 4 * k * d, flops=10.0 * n * d)
    if kind == "score":
        n, c, el = case["n"], case["c"], _SIZE[case["dtype"]]
        by = n * c * el * (3 if case["train"] else 1) + 4 * c * case["bias"] + 8 * n * case["k"] + 16 * n
        return dict(bytes=by, flops=(16.0 if case["train"] else 8.0) * n * c)
    n = float(sum(_sizes(case)))
    return dict(bytes=n * (30 if case["bits"] == 32 else 18 + 16 / 256), flops=(16.0 if case["bits"] == 32 else 40.0) * n)


# ----------------------------------------------------------------------------- exact
def _exact_scan(case, seed):
    """Token by token, as the recurrence is written."""
    s = _scan_inputs(case, seed)
    b, t, d, k = case["b"], case["t"], case["d"], case["gates"]
    bias = s["bias"].double()
    lengths = torch.full((b,), t, device=DEV) if s["lengths"] is None else s["lengths"]
    h = s["h0"].double()
    hs = torch.empty(t + 1, b, d, dtype=torch.float64, device=DEV)
    fs = torch.empty(t, b, d, dtype=torch.float64, device=DEV)
    hs[0] = h
    live = (lengths[None, :] > torch.arange(t, device=DEV)[:, None])[..., None]
    for i in range(t):
        fs[i] = 1.0 / (1.0 + torch.exp(-(s["z"][:, i, d:2 * d].double() + bias[d:2 * d])))
        new = s["z"][:, i, :d].double() + bias[:d]
        h = torch.where(live[i], new + fs[i] * (h - new), h)
        hs[i + 1] = h
    hs = hs.transpose(0, 1)
    fs = fs.transpose(0, 1)
    live = live.transpose(0, 1)
    out = dict(last=h)
    o = None
    if k == 3:
        o = 1.0 / (1.0 + torch.exp(-(s["z"][..., 2 * d:].double() + bias[2 * d:])))
    y = hs[:, 1:] * (1.0 if o is None else o)
    out["y"] = y.masked_fill(~live, 0.0)
    if not case["train"]:
        return out
    g = s["dh"].double()
    gs = torch.empty(b, t, d, dtype=torch.float64, device=DEV)
    for i in reversed(range(t)):
        up = s["dy"][:, i].double()
        gs[:, i] = g + (up if o is None else up * o[:, i])
        g = torch.where(live[:, i], fs[:, i] * gs[:, i], g)
    dz = torch.empty(b, t, k * d, dtype=torch.float64, device=DEV)
    dz[..., :d] = gs - fs * gs
    # the gate's own slope times how far h_t moves with it
    dz[..., d:2 * d] = (hs[:, :-1] - (s["z"][..., :d].double() + bias[:d])) * gs * (fs - fs * fs)
    if o is not None:
        dz[..., 2 * d:] = s["dy"].double() * hs[:, 1:] * (o - o * o)
    out["dz"] = dz.masked_fill(~live, 0.0)
    out["dfirst"] = g
    return out


def _exact_step(case, seed):
    s = _step_inputs(case, seed)
    d = case["d"]
    rows = torch.nonzero(s["slots"] >= 0)[:, 0]
    at = s["slots"][rows].long()
    pre = s["z"][rows].double() + s["bias"].double()
    f = 1.0 / (1.0 + torch.exp(-pre[:, d:2 * d]))
    state = s["state"].double()
    h = pre[:, :d] + f * (state[at] - pre[:, :d])
    state[at] = h
    y = torch.zeros(case["n"], d, dtype=torch.float64, device=DEV)
    y[rows] = h if case["gates"] == 2 else h / (1.0 + torch.exp(-pre[:, 2 * d:]))
    return dict(y=y, state=state)


def _exact_score(case, seed):
    """Row block by row block, through the log-softmax."""
    s = _score_inputs(case, seed)
    n, c, k, T = case["n"], case["c"], case["k"], case["T"]
    f64 = dict(dtype=torch.float64, device=DEV)
    out = dict(entropy=torch.zeros(n, **f64), lse=torch.zeros(n, **f64))
    if s["tokens"] is not None:
        out["logp"] = torch.zeros(n, **f64)
    if k:
        out["top_idx"] = None
        out["top_logp"] = torch.full((n, k), -math.inf, **f64)
    if case["train"]:
        out["dz"] = torch.zeros(n, c, **f64)
    step = max(1, (1 << 26) // c)
    for r0 in range(0, n, step):
        rows = torch.arange(r0, min(n, r0 + step), device=DEV)
        if s["tokens"] is not None:
            rows = rows[s["tokens"][rows] >= 0]
            if not rows.numel():
                continue
        x = s["z"][rows].double()
        if s["bias"] is not None:
            x = x + s["bias"].double()
        x /= T
        out["lse"][rows] = torch.logsumexp(x, 1)
        logp = torch.log_softmax(x, 1)
        finite = torch.where(logp > -math.inf, logp, torch.zeros_like(logp))
        p = torch.exp(logp)
        H = -(p * finite).sum(1)
        out["entropy"][rows] = H
        if k:
            out["top_logp"][rows] = torch.topk(logp, k, 1).values
        if s["tokens"] is None:
            continue
        tok = s["tokens"][rows].long()
        each = torch.arange(rows.numel(), device=DEV)
        out["logp"][rows] = logp[each, tok]
        if case["train"]:
            a, e = s["dlogp"][rows].double()[:, None], s["dentropy"][rows].double()[:, None]
            g = -p * (a + e * (finite + H[:, None]))
            g[each, tok] += a[:, 0]
            out["dz"][rows] = g / T
    return out


def _exact_adamw(case, seed):
    """Variable by variable."""
    s = _adamw_inputs(case, seed)
    t = 100
    names = ("var", "shadow", "m", "v") + (("m_scale", "v_scale") if case["bits"] == 8 else ())
    out = {name: s[name].double() for name in names}
    for a, n, w in zip(s["at"], s["sizes"], _decay(s["sizes"])):
        whole = slice(a, a + -(-n // 256) * 256)
        blocks = slice(whole.start // 256, whole.stop // 256)
        m, v, g = out["m"][whole], out["v"][whole], s["grad"][whole].double()
        if case["bits"] == 8:
            m = (m.view(-1, 256) * out["m_scale"][blocks, None]).view(-1)
            v = (v.view(-1, 256) * out["v_scale"][blocks, None]).view(-1) ** 2
        m = m + (1.0 - BETA1) * (g - m)
        v = v + (1.0 - BETA2) * (g * g - v)
        move = m / (1.0 - BETA1 ** t) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + EPS)
        out["var"][whole] -= LR * (w * out["var"][whole] + move)
        out["shadow"][whole] = out["var"][whole]
        for name, x in (("m", m), ("v", v)):
            if case["bits"] == 8:
                # the values before they are rounded to 8 bits
                x = (x if name == "m" else torch.sqrt(x)).view(-1, 256)
                out[name + "_scale"][blocks] = x.abs().amax(1) / 448.0
                x = (x / out[name + "_scale"][blocks, None].clamp(min=1e-300)).view(-1)
            out[name][whole] = x
    return out


def exact(case, seed):
    return {"scan": _exact_scan, "step": _exact_step, "score": _exact_score, "adamw": _exact_adamw}[case["kind"]](case, seed)
