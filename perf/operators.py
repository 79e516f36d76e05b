"""The language-model operators of this library, as cases to be measured: the 8-bit integer linear layer and the vocabulary
product with its softmax cross entropy and gradients.

``run`` computes a case with elementary torch operations in 32 bits (64 where a rounding border has to be met exactly), or,
with ``own`` set, through the library's entry points."""

import math

import torch

own = False

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
IGNORE = -100


def listed():
    return [
        # one token through a square projection: decoding with a batch of one, where latency counts
        dict(name="linear-token", op="linear", m=1, n=4096, k=4096, x="bf16", out="bf16"),
        # a small decoding batch through a wide projection: bound by reading the weights
        dict(name="linear-batch", op="linear", m=24, n=16384, k=8192, x="bf16", out="bf16"),
        # a prompt whose length, width and inner size fit no tile; fp16 activations, fp32 result (a last layer's scores)
        dict(name="linear-ragged", op="linear", m=2001, n=4999, k=2035, x="fp16", out="fp32"),
        # a long packed prompt through a large square projection: bound by the tensor cores
        dict(name="linear-prompt", op="linear", m=8192, n=8192, k=8192, x="bf16", out="bf16"),
        # tokens quantised once and used by several projections: the product alone
        dict(name="product-square", op="product", m=4096, n=4096, k=4096, x="fp32", out="bf16"),
        dict(name="product-tall", op="product", m=16384, n=2048, k=8192, x="fp32", out="fp16"),
        # the score of one token under a vocabulary (ranking an answer token by token)
        dict(name="loss-token", op="loss", t=1, d=4096, v=32768, x="bf16", reduction="mean"),
        # evaluation of a batch: perplexity of a few packed sequences
        dict(name="loss-batch", op="loss", t=4096, d=2048, v=32768, x="bf16", reduction="mean"),
        # ragged in every size, a loss for each token (weighted outside), fp16
        dict(name="loss-ragged", op="loss", t=1001, d=1032, v=50001, x="fp16", reduction="none"),
        # training steps: a few answer tokens behind a masked prompt; ragged with weights per token; a full batch
        dict(name="step-few", op="step", t=16, d=4096, v=65536, x="bf16", reduction="mean"),
        dict(name="step-ragged", op="step", t=777, d=1032, v=20011, x="fp16", reduction="none"),
        dict(name="step-batch", op="step", t=8192, d=4096, v=131072, x="bf16", reduction="mean"),
    ]


def _between(rng, low, high):
    """Spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "product", "loss", "step"])
    if op in ("linear", "product"):
        m, n, k = _between(rng, 1, 16384), _between(rng, 16, 16384), _between(rng, 16, 8192)
        if op == "product":                      # quantised rows are padded to 16 bytes
            k = max(16, k // 16 * 16)
        while m * n * k > 8192 ** 3:
            m = (m + 1) // 2
        x = rng.choice(["bf16", "fp16", "fp32"]) if op == "linear" else "fp32"
        return dict(op=op, m=m, n=n, k=k, x=x, out=rng.choice(["bf16", "fp16", "fp32"]))
    t, d, v = _between(rng, 1, 8192), 8 * _between(rng, 4, 512), _between(rng, 500, 131072)
    return dict(op=op, t=t, d=d, v=v, x=rng.choice(["bf16", "fp16"]), reduction=rng.choice(["mean", "sum", "none"]))


def _pad16(k):
    return (k + 15) // 16 * 16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = dict(case)
    if case["op"] in ("linear", "product"):
        m, n, k = case["m"], case["n"], case["k"]
        kp = _pad16(k)
        # weights quantised per output channel, once, as a user's program keeps them: rows padded to 16 bytes
        w = torch.randint(-127, 128, (n, kp), device="cuda", generator=g, dtype=torch.int32).to(torch.int8)
        w[:, k:] = 0
        s["w"] = w
        s["w_scale"] = (0.5 + torch.rand(n, device="cuda", generator=g)) * (0.02 / 127)
        s["y"] = torch.empty(m, n, device="cuda", dtype=BITS[case["out"]])
        if case["op"] == "linear":
            # activations: a few channels are much larger than the rest, as in trained models
            big = torch.where(torch.rand(k, device="cuda", generator=g) < 0.01, 20.0, 1.0)
            s["x"] = (normal(m, k) * big).to(BITS[case["x"]])
            s["q"] = torch.empty(m, kp, device="cuda", dtype=torch.int8)
            s["q_scale"] = torch.empty(m, device="cuda")
        else:
            s["q"] = (normal(m, kp) * 30).round().clamp(-127, 127).to(torch.int8)
            s["q_scale"] = (0.5 + torch.rand(m, device="cuda", generator=g)) * (4.0 / 127)
        s["x_type"], s["out_type"] = case["x"], case["out"]
        return s
    t, d, v = case["t"], case["d"], case["v"]
    bits = BITS[case["x"]]
    s["h"] = normal(t, d).to(bits)                              # normed hidden states
    s["w"] = (normal(v, d) * (2.5 / math.sqrt(d))).to(bits)     # scores with a deviation of 2.5
    target = torch.randint(0, v, (t,), device="cuda", generator=g)
    if t > 8:                                                   # a masked prompt before the answer
        target[: t // 8] = IGNORE
    s["target"] = target
    s["lse"] = torch.empty(t, device="cuda")
    s["loss"] = torch.empty(t if case["reduction"] == "none" else 1, device="cuda")
    if case["op"] == "step":
        # fp16 steps are scaled up against underflow, as mixed-precision training does
        up = 1024.0 if case["x"] == "fp16" else 1.0
        if case["reduction"] == "none":
            s["grad"] = (0.5 + torch.rand(t, device="cuda", generator=g)) * up
        else:
            s["grad"] = torch.full((1,), up, device="cuda")
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    return s


def _quantized(x):
    x = x.float()
    scale = (x.abs().amax(1).double() / 127).float()            # correctly rounded: a step beside it moves exact halves
    q = (x.double() / scale.double()[:, None]).round()          # half to even, of the exact quotient
    return torch.where(scale[:, None] > 0, q, 0.0).float(), scale


def _scores(h, w, target):
    z = h.float() @ w.float().T
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lse = (top + total.log())[:, 0]
    kept = target != IGNORE
    at = torch.where(kept, target, 0)[:, None]
    each = torch.where(kept, lse - z.gather(1, at)[:, 0], 0.0)
    return e, total, lse, kept, at, each


def run(state):
    op = state["op"]
    if own:
        import paper_2508_20258_b200 as sp
        if op == "linear":
            sp.linear_i8(state["x"], state["q"], state["q_scale"], state["w"], state["w_scale"], state["y"])
            return state["y"], state["q_scale"]
        if op == "product":
            sp.gemm_i8(state["q"], state["q_scale"], state["w"], state["w_scale"], state["y"])
            return state["y"]
        sp.linear_ce(state["h"], state["w"], state["target"], state["lse"], state["loss"], reduction=state["reduction"], ignore_index=IGNORE)
        if op == "loss":
            return state["loss"], state["lse"]
        sp.linear_ce_grad(state["h"], state["w"], state["target"], state["lse"], state["grad"], state["dh"], state["dw"],
                          reduction=state["reduction"], ignore_index=IGNORE)
        return state["loss"], state["dh"], state["dw"]
    if op == "linear":
        q, scale = _quantized(state["x"])
        y = (q @ state["w"][:, : q.shape[1]].float().T) * scale[:, None] * state["w_scale"]
        return y.to(state["y"].dtype), scale
    if op == "product":
        y = (state["q"].float() @ state["w"].float().T) * state["q_scale"][:, None] * state["w_scale"]
        return y.to(state["y"].dtype)
    h, w, target = state["h"], state["w"], state["target"]
    e, total, lse, kept, at, each = _scores(h, w, target)
    loss = each if state["reduction"] == "none" else each.sum()[None] if state["reduction"] == "sum" else (each.sum() / kept.sum())[None]
    if op == "loss":
        return loss, lse
    share = state["grad"] / kept.sum() if state["reduction"] == "mean" else state["grad"]
    g = e / total
    g.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    g = g * torch.where(kept, share, 0.0)[:, None]
    return loss, (g @ w.float()).to(h.dtype), (g.T @ h.float()).to(w.dtype)


def work(case):
    if case["op"] in ("linear", "product"):
        m, n, k = case["m"], case["n"], _pad16(case["k"])
        read = m * case["k"] * SIZE[case["x"]] if case["op"] == "linear" else m * k + 4 * m
        return {"bytes": read + n * k + 4 * n + m * n * SIZE[case["out"]] + (4 * m if case["op"] == "linear" else 0), "flops": 2 * m * n * case["k"]}
    t, d, v, e = case["t"], case["d"], case["v"], SIZE[case["x"]]
    inputs, losses = (t + v) * d * e + 8 * t, 4 * (t if case["reduction"] == "none" else 1)
    if case["op"] == "loss":
        return {"bytes": inputs + losses + 4 * t, "flops": 2 * t * v * d}
    # three products (scores, both gradients); making the scores a second time is the price of not keeping them, and not counted
    return {"bytes": inputs + losses + 4 * losses + (t + v) * d * e, "flops": 6 * t * v * d}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("linear", "product"):
        w = s["w"].to(torch.float64)
        w *= s["w_scale"].to(torch.float64)[:, None]
        if case["op"] == "product":
            a = s["q"].to(torch.float64) * s["q_scale"].to(torch.float64)[:, None]
            return torch.matmul(a, w.t())
        x = s["x"].to(torch.float64)
        step = (torch.max(torch.abs(x), dim=1).values / 127.0).to(torch.float32).to(torch.float64)   # the scale is a 32-bit number
        a = torch.round(x / step[:, None]) * step[:, None]
        return torch.matmul(a, w[:, : case["k"]].t()), step
    h, w, y = s["h"].to(torch.float64), s["w"].to(torch.float64), s["target"]
    z = torch.matmul(h, w.t())
    lse = torch.logsumexp(z, dim=1)
    rows = torch.nonzero(y != IGNORE)[:, 0]
    each = torch.zeros_like(lse)
    each[rows] = lse[rows] - z[rows, y[rows]]
    loss = each if case["reduction"] == "none" else torch.sum(each).reshape(1)
    if case["reduction"] == "mean":
        loss = loss / rows.numel()
    if case["op"] == "loss":
        return loss, lse
    weight = torch.zeros_like(lse)
    weight[rows] = (s["grad"].to(torch.float64).expand(case["t"]))[rows]
    if case["reduction"] == "mean":
        weight = weight / rows.numel()
    z.sub_(lse[:, None]).exp_()
    z[rows, y[rows]] -= 1.0
    z.mul_(weight[:, None])
    return loss, torch.matmul(z, w), torch.matmul(z.t(), h)
