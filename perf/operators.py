"""Performance cases of the output head's operators: the cross entropy over the
vocabulary and its gradient, the distillation from a teacher's top logits and
its gradient, and the selection of those top logits.

A case names the operator ("op") and its sizes: T tokens, V words of the
vocabulary, D the width of the hidden state, K the listed teacher logits.
"empty" is the share of tokens that take no part (a prompt's tokens, padding),
"pad" the elements by which a row of the hidden state (or of the logits) is
longer than what the call reads, "tau" the temperature.

own = False computes the operators in elementary operations in fp32, rounded
once at the end; own = True calls the package's entry points.
"""
import math

import torch

own = False

DEV = "cuda"
OPS = ("loss", "loss_grad", "distill", "distill_grad", "top")

_BASE = dict(op="loss", T=0, V=0, D=0, K=0, tau=1.0, empty=0.0, pad=0, mass=False, weighted=False,
             dtype="bf16")


def _case(**kw):
    return dict(_BASE, **kw)


def listed():
    return [
        # Evaluating a short answer with a small model: launches and latency.
        _case(name="loss_small", op="loss", T=7, V=1000, D=96),
        # One token of an 8B model scored: the weight is read once.
        _case(name="loss_8b_one", op="loss", T=1, V=128256, D=4096),
        # The loss of a micro-batch of 4096 tokens, an eighth of it padding.
        _case(name="loss_8b", op="loss", T=4096, V=128256, D=4096, empty=0.125),
        # A small model's gradient at odd sizes, tokens weighted.
        _case(name="loss_grad_odd", op="loss_grad", T=333, V=5003, D=321, empty=0.1, pad=7,
              weighted=True),
        # A dialogue batch of which half the tokens are prompt.
        _case(name="loss_grad_32k", op="loss_grad", T=4096, V=32000, D=2048, empty=0.5),
        # The gradient of the 8B micro-batch: the largest.
        _case(name="loss_grad_8b", op="loss_grad", T=4096, V=128256, D=4096),
        # The student's loss on a public batch against 64 teacher logits.
        _case(name="distill_8b", op="distill", T=1000, V=128256, D=4096, K=64, tau=2.0, mass=True),
        # A short public batch, a few of its tokens without a teacher.
        _case(name="distill_grad_short", op="distill_grad", T=64, V=50257, D=1024, K=16, tau=1.5,
              empty=0.25),
        # The student's gradient on a batch.
        _case(name="distill_grad_8b", op="distill_grad", T=2048, V=128256, D=4096, K=32, tau=2.0),
        # One token's top logits from a padded vocabulary, in fp32.
        _case(name="top_one", op="top", T=1, V=50257, K=8, pad=47, dtype="fp32"),
        # A teacher's micro-batch of bf16 logits.
        _case(name="top_8b", op="top", T=2048, V=128256, K=64, tau=2.0),
        # Fewer rows than compute units, fp32, an odd vocabulary.
        _case(name="top_100", op="top", T=100, V=100003, K=100, pad=5, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


WIDTHS = (64, 128, 256, 320, 512, 768, 896, 1024, 1280, 1536, 2048, 2560, 4096)


def draw(rng):
    op = rng.choice(OPS)
    c = dict(_BASE, op=op)
    c["T"] = _log_int(rng, 1, 2048 if op == "top" else 4096)
    c["V"] = _log_int(rng, 512, 128256)
    if op != "top":
        c["D"] = rng.choice([_log_int(rng, 64, 4096)] + [rng.choice(WIDTHS)] * 3)
        c["empty"] = rng.choice([0.0, 0.0, round(rng.uniform(0.05, 0.7), 3)])
        c["weighted"] = op.endswith("grad") and rng.random() < 0.5
    if op == "top":
        c["dtype"] = rng.choice(["bf16", "fp32"])
    if op not in ("loss", "loss_grad"):
        c["K"] = _log_int(rng, 1, 128)
        c["tau"] = rng.choice([1.0, 1.5, 2.0, 4.0])
    if op.startswith("distill"):
        c["mass"] = rng.random() < 0.5
    c["pad"] = rng.choice([0, 0, rng.randint(1, 64)])
    return c


# ---- inputs ----------------------------------------------------------------

ROWS = 512   # rows of logits at a time while inputs are made


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    g = _gen(seed)
    T, V, D, K, op, tau = (case[k] for k in ("T", "V", "D", "K", "op", "tau"))
    if op == "top":
        # logits of a trained model: a spread of 2.5, and some words far above
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        base = torch.empty(T, V + case["pad"], device=DEV, dtype=dt)
        for r in range(0, T, ROWS):
            x = _randn(g, min(ROWS, T - r), V + case["pad"]) * 2.5
            base[r:r + ROWS] = x + (x > 7.5).float() * 2.0 * (x - 7.5)
        return dict(case=case, logits=base[:, :V], values=torch.empty(T, K, device=DEV),
                    ids=torch.empty(T, K, device=DEV, dtype=torch.int32),
                    lse=torch.empty(T, device=DEV))
    # A hidden state of unit variance and a weight that gives logits a spread of 2.5.
    hidden = _randn(g, T, D + case["pad"]).bfloat16()[:, :D]
    weight = (_randn(g, V, D) * (2.5 / math.sqrt(D))).bfloat16()
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    n_empty = min(T - 1, int(round(case["empty"] * T)))
    keep[torch.randperm(T, generator=g, device=DEV)[:n_empty]] = False
    s = dict(case=case, hidden=hidden, weight=weight)
    w32 = weight.float()
    lse, tgt = torch.zeros(T, device=DEV), torch.zeros(T, max(K, 1), device=DEV)
    labels = torch.full((T,), -100, dtype=torch.int64, device=DEV)
    ids = torch.full((T, max(K, 1)), -1, dtype=torch.int32, device=DEV)
    a = torch.zeros(T, max(K, 1), device=DEV)
    alse = torch.zeros(T, device=DEV)
    for r in range(0, T, ROWS):
        e = min(r + ROWS, T)
        z = hidden[r:e].float() @ w32.t()
        k = keep[r:e]
        lse[r:e] = torch.where(k, torch.logsumexp(z / tau, 1), 0.0)
        if K == 0:
            # labels as the model itself would draw them
            u = torch.rand(z.shape, generator=g, device=DEV).clamp_(1e-9, 1.0 - 1e-6)
            y = (z - torch.log(-torch.log(u))).argmax(1)
            labels[r:e] = torch.where(k, y, -100)
            tgt[r:e, 0] = torch.where(k, z.gather(1, y[:, None])[:, 0], 0.0)
        else:
            # the teacher: the student's logits and noise of its own
            az = z + _randn(g, *z.shape)
            v, i = az.topk(K, dim=1)
            ids[r:e] = torch.where(k[:, None], i.int(), -1)
            a[r:e] = torch.where(k[:, None], v, 0.0)
            alse[r:e] = torch.where(k, torch.logsumexp(az / tau, 1), 0.0)
            tgt[r:e] = torch.where(k[:, None], z.gather(1, i), 0.0)
    if K and K > 2:   # a few rows list fewer words than the others
        few = keep & (torch.rand(T, generator=g, device=DEV) < 0.1)
        ids[few, K // 2:] = -1
        tgt[few, K // 2:] = 0.0
    if K == 0:
        s.update(labels=labels, target=tgt[:, 0].contiguous())
    else:
        s.update(ids=ids, teacher=a, teacher_lse=alse if case["mass"] else None, target=tgt)
    if op.endswith("grad"):
        dl = torch.full((T,), 1.0 / max(1, T - n_empty), device=DEV)
        if case["weighted"]:
            dl = dl * (0.5 + torch.rand(T, generator=g, device=DEV))
        s.update(lse=lse, dloss=dl, dhidden=torch.empty(T, D, device=DEV, dtype=torch.bfloat16),
                 dweight=torch.empty(V, D, device=DEV, dtype=torch.bfloat16))
    else:
        s.update(loss=torch.empty(T, device=DEV), lse_out=torch.empty(T, device=DEV),
                 target_out=torch.empty(T, max(K, 1), device=DEV))
        if K == 0:
            s["target_out"] = s["target_out"][:, 0]
    return s


# ---- one pass --------------------------------------------------------------


def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    return {"loss": _loss, "loss_grad": _loss_grad, "distill": _distill,
            "distill_grad": _distill_grad, "top": _top}[op](s)


def _run_own(s, op):
    import paper_2609_20359_amd as P

    c = s["case"]
    if op == "top":
        P.fl_top_logits(s["logits"], c["K"], c["tau"], s["values"], s["ids"], s["lse"])
        return dict(values=s["values"], ids=s["ids"], lse=s["lse"])
    if op == "loss":
        P.fl_head_loss(s["hidden"], s["weight"], s["labels"], s["loss"], s["lse_out"],
                       s["target_out"])
    elif op == "distill":
        P.fl_head_distill(s["hidden"], s["weight"], s["ids"], s["teacher"], s["teacher_lse"],
                          c["tau"], s["loss"], s["lse_out"], s["target_out"])
    elif op == "loss_grad":
        P.fl_head_loss_grad(s["hidden"], s["weight"], s["labels"], s["lse"], s["target"],
                            s["dloss"], s["dhidden"], s["dweight"])
    else:
        P.fl_head_distill_grad(s["hidden"], s["weight"], s["ids"], s["teacher"],
                               s["teacher_lse"], c["tau"], s["lse"], s["target"], s["dloss"],
                               s["dhidden"], s["dweight"])
    if op.endswith("grad"):
        return dict(dhidden=s["dhidden"], dweight=s["dweight"])
    return dict(loss=s["loss"], lse=s["lse_out"], target=s["target_out"])


def _loss(s):
    z = s["hidden"].float() @ s["weight"].float().t()
    keep = s["labels"] >= 0
    m = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - m).sum(1)) + m[:, 0]
    t = z.gather(1, s["labels"].clamp(min=0)[:, None])[:, 0]
    return dict(loss=torch.where(keep, lse - t, 0.0), lse=torch.where(keep, lse, 0.0),
                target=torch.where(keep, t, 0.0))


def _loss_grad(s):
    h, w = s["hidden"].float(), s["weight"].float()
    keep = s["labels"] >= 0
    c = torch.where(keep, s["dloss"], 0.0)
    g = torch.exp(h @ w.t() - s["lse"][:, None]) * c[:, None]
    g = torch.where(keep[:, None], g, 0.0)
    g.scatter_add_(1, s["labels"].clamp(min=0)[:, None], -c[:, None])
    return dict(dhidden=(g @ w).bfloat16(), dweight=(g.t() @ h).bfloat16())


def _teacher(s):
    """(listed, keep, log p, p) of the teacher."""
    there = s["ids"] >= 0
    a = torch.where(there, s["teacher"] / s["case"]["tau"], -math.inf)
    keep = there.any(1)
    if s["teacher_lse"] is not None:
        logp = a - s["teacher_lse"][:, None]
    else:
        m = torch.where(keep, a.amax(1), 0.0)[:, None]
        logp = a - m - torch.log(torch.exp(a - m).sum(1, keepdim=True))
    logp = torch.where(there, logp, 0.0)
    return there, keep, logp, torch.where(there, torch.exp(logp), 0.0)


def _distill(s):
    tau = s["case"]["tau"]
    there, keep, logp, p = _teacher(s)
    z = s["hidden"].float() @ s["weight"].float().t()
    t = z.gather(1, s["ids"].clamp(min=0).long())
    z = z / tau
    m = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - m).sum(1)) + m[:, 0]
    loss = tau * tau * (p * (logp - t / tau + lse[:, None])).sum(1)
    return dict(loss=torch.where(keep, loss, 0.0), lse=torch.where(keep, lse, 0.0),
                target=torch.where(there, t, 0.0))


def _distill_grad(s):
    tau = s["case"]["tau"]
    h, w = s["hidden"].float(), s["weight"].float()
    there, keep, logp, p = _teacher(s)
    c = torch.where(keep, s["dloss"] * tau, 0.0)[:, None]
    g = torch.exp((h @ w.t()) / tau - s["lse"][:, None]) * (c * p.sum(1, keepdim=True))
    g = torch.where(keep[:, None], g, 0.0)
    g.scatter_add_(1, s["ids"].clamp(min=0).long(), -c * p)
    return dict(dhidden=(g @ w).bfloat16(), dweight=(g.t() @ h).bfloat16())


def _top(s):
    x = s["logits"].float() + 0.0
    # one whole number that orders a row's words by value, then by the lower id
    bits = x.view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
    key = (order << 32) | (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
    key = key.topk(s["case"]["K"], dim=1).values
    ids = 0x7FFFFFFF - (key & 0xFFFFFFFF)
    z = x / s["case"]["tau"]
    m = z.amax(1, keepdim=True)
    return dict(values=x.gather(1, ids), ids=ids.int(),
                lse=torch.log(torch.exp(z - m).sum(1)) + m[:, 0])


# ---- what a pass cannot do without, and its results in 64 bits ---------------


def work(case):
    T, V, D, K, op = (case[k] for k in ("T", "V", "D", "K", "op"))
    if op == "top":
        e = 2 if case["dtype"] == "bf16" else 4
        return dict(bytes=T * V * e + T * (8 * K + 4), flops=3 * T * V)
    live = T - min(T - 1, int(round(case["empty"] * T)))   # tokens that take part
    per_token = 8 * T if K == 0 else 8 * T * K + (4 * T if case["mass"] else 0)
    inputs = 2 * D * (live + V) + per_token
    if op.endswith("grad"):
        return dict(bytes=inputs + 2 * D * (T + V) + T * (8 + 4 * max(K, 1)),
                    flops=6 * live * V * D)
    return dict(bytes=inputs + T * (8 + 4 * max(K, 1)), flops=2 * live * V * D)


def exact(case, seed):
    s = prepare(case, seed)
    op, tau = case["op"], case["tau"]
    if op == "top":
        x = s["logits"].double()
        v, i = torch.sort(x, dim=1, descending=True, stable=True)
        return dict(values=v[:, :case["K"]], ids=i[:, :case["K"]].int(),
                    lse=torch.logsumexp(x / tau, 1))
    h, w = s["hidden"].double(), s["weight"].double()
    T = h.shape[0]
    # the target distribution as lists of (row, word, probability)
    if case["K"] == 0:
        live = (s["labels"] >= 0).nonzero()[:, 0]
        row, word = live, s["labels"][live]
        prob = torch.ones(len(live), dtype=torch.float64, device=h.device)
        scale = 1.0
    else:
        row, k = (s["ids"] >= 0).nonzero(as_tuple=True)
        word = s["ids"][row, k].long()
        e = torch.exp(s["teacher"].double()[row, k] / tau)
        if s["teacher_lse"] is not None:
            prob = e / torch.exp(s["teacher_lse"].double())[row]
        else:
            total = torch.zeros(T, dtype=torch.float64, device=h.device).index_add_(0, row, e)
            prob = e / total[row]
        live = row.unique()
        scale = tau
    z = h @ w.t()
    at = z[row, word]
    lse = torch.logsumexp(z / tau, 1)
    if op.endswith("grad"):
        mass = torch.zeros(T, dtype=torch.float64, device=h.device).index_add_(0, row, prob)
        c = s["dloss"].double() * scale
        z.div_(tau).sub_(lse[:, None]).exp_().mul_((c * mass)[:, None])
        z.index_put_((row, word), -c[row] * prob, accumulate=True)
        return dict(dhidden=z @ w, dweight=z.t() @ h)
    part = prob * (torch.log(prob) - at / tau + lse[row])
    loss = torch.zeros(T, dtype=torch.float64, device=h.device).index_add_(0, row, part)
    on = torch.zeros(T, dtype=torch.float64, device=h.device)
    on[live] = 1.0
    target = torch.zeros(T, max(case["K"], 1), dtype=torch.float64, device=h.device)
    if case["K"] == 0:
        target[row, 0] = at
        target = target[:, 0]
    else:
        target[row, k] = at
    return dict(loss=loss * scale * scale, lse=lse * on, target=target)
