"""Layer norm and distillation from a teacher's top logits, each with its gradients, as cases to be measured.

``run`` computes a case with elementary torch operations in 32 bits or, with ``own`` set, through the library's entry points."""

import math

import torch

own = False

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


def listed():
    return [
        # one token while decoding: latency
        dict(name="norm-token", op="norm", m=1, n=4096, x="bf16", w="bf16"),
        # a packed batch of hidden states
        dict(name="norm-batch", op="norm", m=8192, n=4096, x="bf16", w="bf16"),
        # rows that end on no boundary, weights kept in 32 bits
        dict(name="norm-ragged", op="norm", m=5001, n=2035, x="fp16", w="fp32"),
        # a few answer tokens of a small model, backward
        dict(name="norm-grad-few", op="norm-grad", m=60, n=304, x="bf16", w="bf16"),
        # a full training batch, backward, weights kept in 32 bits
        dict(name="norm-grad-batch", op="norm-grad", m=16384, n=4096, x="bf16", w="fp32"),
        dict(name="norm-grad-ragged", op="norm-grad", m=3001, n=1031, x="fp16", w="fp16"),
        # wide rows in 32 bits
        dict(name="norm-grad-wide", op="norm-grad", m=2048, n=16384, x="fp32", w="fp32"),
        # evaluation of a student: a few tokens, and a batch
        dict(name="distill-few", op="distill", t=24, d=1024, v=32768, k=32, x="bf16", logit="fp32", tau=1.0, reduction="mean"),
        dict(name="distill-batch", op="distill", t=4096, d=2048, v=32768, k=64, x="bf16", logit="bf16", tau=2.0, reduction="mean"),
        # training steps: a few answer tokens; ragged with weights per token; a full batch
        dict(name="distill-step-few", op="distill-step", t=16, d=4096, v=65536, k=20, x="bf16", logit="fp32", tau=1.0, reduction="mean"),
        dict(name="distill-step-ragged", op="distill-step", t=777, d=1032, v=20011, k=17, x="fp16", logit="fp32", tau=1.5, reduction="none"),
        dict(name="distill-step-batch", op="distill-step", t=8192, d=4096, v=131072, k=100, x="bf16", logit="bf16", tau=2.0, reduction="mean"),
    ]


def _between(rng, low, high):
    """Spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "norm-grad", "distill", "distill-step"])
    if op.startswith("norm"):
        m, n, x = _between(rng, 1, 32768), _between(rng, 8, 20000), rng.choice(["bf16", "fp16", "fp32"])
        n = rng.choice([n, (n + 7) // 8 * 8])          # hidden sizes are mostly multiples of 8, not always
        while m * n > 16384 * 4096:
            m = (m + 1) // 2
        return dict(op=op, m=m, n=n, x=x, w=rng.choice([x, "fp32"]))
    t, d, v = _between(rng, 1, 8192), 8 * _between(rng, 4, 512), _between(rng, 500, 131072)
    return dict(op=op, t=t, d=d, v=v, k=_between(rng, 1, 128), x=rng.choice(["bf16", "fp16"]), logit=rng.choice(["fp32", "bf16", "fp16"]),
                tau=rng.choice([0.5, 1.0, 1.5, 2.0, 4.0]), reduction=rng.choice(["mean", "sum", "none"]))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    s = dict(case)
    if case["op"].startswith("norm"):
        m, n, bits, wbits = case["m"], case["n"], BITS[case["x"]], BITS[case["w"]]
        # hidden states: a few channels far larger than the rest, rows of different scale, means beside zero
        big = torch.where(uniform(n) < 0.01, 20.0, 1.0)
        s["x"] = ((normal(m, n) * big + 0.3) * (0.5 + uniform(m, 1))).to(bits)
        s["gamma"], s["beta"] = (1 + 0.2 * normal(n)).to(wbits), (0.2 * normal(n)).to(wbits)
        s["mean"], s["rstd"] = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
        s["out"] = torch.empty_like(s["x"])             # y, or dx
        if case["op"] == "norm-grad":
            s["dy"] = (normal(m, n) * 0.1).to(bits)
            x = s["x"].float()                          # what the forward pass has left
            s["mean"] = x.mean(1)
            s["rstd"] = ((x - s["mean"][:, None]).square().mean(1) + EPS).rsqrt()
            s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
        return s
    t, d, v, k, bits = case["t"], case["d"], case["v"], case["k"], BITS[case["x"]]
    s["h"] = normal(t, d).to(bits)                              # normed hidden states
    s["w"] = (normal(v, d) * (2.5 / math.sqrt(d))).to(bits)     # scores with a deviation of 2.5
    # the teacher's words: distinct in a row, frequent (low) ones more often, in the order of their logits
    at = torch.arange(k, device="cuda")
    word = (v * ((at + uniform(t, k)) / k).square()).long().clamp_(max=v - 1)
    word = (word - at).cummax(1).values + at
    word = word.gather(1, uniform(t, k).argsort(1))
    logit = (12 + 2.5 * normal(t, k)).sort(1, descending=True).values
    # one token in four is clear, to the teacher and to the student
    clear = torch.arange(t, device="cuda") % 4 == 3
    logit[:, 0] += torch.where(clear, 12.0, 0.0)
    s["h"] = torch.where(clear[:, None], (s["w"][word[:, 0]].float() * 2).to(bits), s["h"])
    # some tokens keep fewer words, and a masked prompt comes before the answer
    fewer = torch.where(uniform(t) < 0.25, 1 + (uniform(t) * k).long(), k)
    word = torch.where(at < fewer[:, None], word, -1)
    if t > 8:
        word[: t // 8] = -1
    s["word"], s["logit"] = word.contiguous(), logit.to(BITS[case["logit"]]).contiguous()
    s["lse"], s["diff"] = torch.empty(t, device="cuda"), torch.empty(t, k, device="cuda")
    s["loss"] = torch.empty(t if case["reduction"] == "none" else 1, device="cuda")
    if case["op"] == "distill-step":
        # fp16 steps are scaled up against underflow, as mixed-precision training does
        up = 1024.0 if case["x"] == "fp16" else 1.0
        s["grad"] = (0.5 + uniform(t)) * up if case["reduction"] == "none" else torch.full((1,), up, device="cuda")
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    return s


def run(state):
    op = state["op"]
    if own:
        import paper_2508_20258_b200 as sp
        if op == "norm":
            sp.layernorm(state["x"], state["gamma"], state["beta"], state["out"], state["mean"], state["rstd"], eps=EPS)
            return state["out"], state["mean"], state["rstd"]
        if op == "norm-grad":
            sp.layernorm_grad(state["dy"], state["x"], state["gamma"], state["mean"], state["rstd"], state["out"], state["dgamma"], state["dbeta"])
            return state["out"], state["dgamma"], state["dbeta"]
        sp.linear_distill(state["h"], state["w"], state["word"], state["logit"], state["lse"], state["diff"], state["loss"],
                          temperature=state["tau"], reduction=state["reduction"])
        if op == "distill":
            return state["loss"], state["lse"], state["diff"]
        sp.linear_distill_grad(state["h"], state["w"], state["word"], state["lse"], state["diff"], state["grad"], state["dh"], state["dw"],
                               temperature=state["tau"], reduction=state["reduction"])
        return state["loss"], state["dh"], state["dw"]
    if op == "norm":
        x = state["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = (c.square().mean(1) + EPS).rsqrt()
        y = c * rstd[:, None] * state["gamma"].float() + state["beta"].float()
        return y.to(state["x"].dtype), mean, rstd
    if op == "norm-grad":
        dy, rstd = state["dy"].float(), state["rstd"][:, None]
        xh = (state["x"].float() - state["mean"][:, None]) * rstd
        u = dy * state["gamma"].float()
        dx = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
        return dx.to(state["x"].dtype), (dy * xh).sum(0).to(state["gamma"].dtype), dy.sum(0).to(state["gamma"].dtype)
    h, w, tau, word = state["h"], state["w"], state["tau"], state["word"]
    z = (h.float() @ w.float().T) / tau
    top = z.amax(1, keepdim=True)
    z -= top
    used = word >= 0
    kept = used.any(1)
    at = torch.where(used, word, 0)
    own_z = z.gather(1, at)                                     # scores of the teacher's words
    z.exp_()
    total = z.sum(1, keepdim=True)
    log_total = total.log()
    lse = torch.where(kept, (top + log_total)[:, 0], math.inf)
    logit = torch.where(used, state["logit"].float() / tau, -math.inf)
    logit = logit - torch.where(kept, logit.amax(1), 0.0)[:, None]
    mass = logit.exp()
    share = mass.sum(1, keepdim=True)
    q = torch.where(used, mass / share, 0.0)
    log_p = own_z - log_total
    each = tau * tau * torch.where(q > 0, q * (logit - share.log() - log_p), 0.0).sum(1)
    loss = each if state["reduction"] == "none" else each.sum()[None] if state["reduction"] == "sum" else (each.sum() / kept.sum())[None]
    if op == "distill":
        return loss, lse, torch.where(used, log_p.exp() - q, 0.0)
    coef = state["grad"] / kept.sum() if state["reduction"] == "mean" else state["grad"]
    z /= total
    z.scatter_add_(1, at, -q)
    z *= torch.where(kept, tau * coef, 0.0)[:, None]
    return loss, (z @ w.float()).to(h.dtype), (z.T @ h.float()).to(w.dtype)


def work(case):
    if case["op"].startswith("norm"):
        m, n, e, ew = case["m"], case["n"], SIZE[case["x"]], SIZE[case["w"]]
        if case["op"] == "norm":
            return {"bytes": 2 * m * n * e + 2 * n * ew + 8 * m, "flops": 8 * m * n}
        return {"bytes": 3 * m * n * e + 3 * n * ew + 8 * m, "flops": 14 * m * n}
    t, d, v, k, e = case["t"], case["d"], case["v"], case["k"], SIZE[case["x"]]
    inputs, losses = (t + v) * d * e + t * k * (8 + SIZE[case["logit"]]), 4 * (t if case["reduction"] == "none" else 1)
    if case["op"] == "distill":
        return {"bytes": inputs + losses + 4 * t + 4 * t * k, "flops": 2 * t * v * d}
    # three products; making the scores a second time is the price of not keeping them, and not counted
    return {"bytes": inputs + 2 * losses + (t + v) * d * e, "flops": 6 * t * v * d}


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"].startswith("norm"):
        x, gamma, beta = s["x"].to(f64), s["gamma"].to(f64), s["beta"].to(f64)
        if case["op"] == "norm":
            var, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = 1.0 / torch.sqrt(var + EPS)
            return torch.addcmul(beta, torch.mul(x.sub_(mean[:, None]), rstd[:, None]), gamma), mean, rstd
        dy, rstd = s["dy"].to(f64), s["rstd"].to(f64)[:, None]
        x.sub_(s["mean"].to(f64)[:, None]).mul_(rstd)
        dgamma, dbeta = torch.einsum("mn,mn->n", dy, x), torch.sum(dy, dim=0)
        dy.mul_(gamma)
        along = torch.einsum("mn,mn->m", dy, x) / case["n"]
        flat = torch.mean(dy, dim=1)
        return dy.sub_(flat[:, None]).sub_(x.mul_(along[:, None])).mul_(rstd), dgamma, dbeta
    tau, t, word = float(case["tau"]), case["t"], s["word"]
    h, w = s["h"].to(f64), s["w"].to(f64)
    z = torch.matmul(h, w.t()).div_(tau)
    lse = torch.logsumexp(z, dim=1)
    logp = z.sub_(lse[:, None])
    teacher = s["logit"].to(f64).div(tau).masked_fill(word < 0, -math.inf)
    rows = torch.nonzero((word >= 0).sum(1) > 0)[:, 0]
    logq = torch.full_like(teacher, -math.inf)
    logq[rows] = torch.log_softmax(teacher[rows], dim=1)
    q = torch.exp(logq)
    mine = torch.gather(logp, 1, word.clamp(min=0))
    each = (tau * tau) * torch.sum(torch.where(word >= 0, q * (logq.clamp(min=-1e4) - mine), torch.zeros_like(q)), dim=1)
    loss = each if case["reduction"] == "none" else torch.sum(each).reshape(1)
    if case["reduction"] == "mean":
        loss = loss / rows.numel()
    if case["op"] == "distill":
        left = torch.full_like(lse, math.inf)
        left[rows] = lse[rows]
        return loss, left, torch.where(word >= 0, torch.exp(mine) - q, torch.zeros_like(q))
    weight = torch.zeros_like(lse)
    weight[rows] = tau * s["grad"].to(f64).expand(t)[rows]
    if case["reduction"] == "mean":
        weight = weight / rows.numel()
    prob = logp.exp_()
    prob.scatter_add_(1, word.clamp(min=0), -q)
    prob.mul_(weight[:, None])
    return loss, torch.matmul(prob, w), torch.matmul(prob.t(), h)
