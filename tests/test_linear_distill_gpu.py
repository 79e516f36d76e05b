"""Distillation from a teacher's top logits and its gradients against the formulas in float64.

Tolerances, from the arithmetic (u = 2^-23; e = eps / 2 of the 16-bit type; z the scores over the temperature).
  z      16 products at a time are added to an accumulator that may cut instead of rounding, 512 at a time in fp32: (D / 16 + D / 512 + 2) u sum_d |h_d W_vd| /
         temperature, the largest over v: dz.
  p      an exponent z log2 e - m is rounded up to three times on its way, is at most 2 log2(e) max|z|, and the hardware's 2^x is good to 2^-22; so is the sum
         of all of them, its additions within 2^-17: relative s = 2 dz + 2 (6 log2(e) max|z| + 4) u + 2^-17.
  q      the same for logits that lie up to `span` / temperature apart, with K / 32 + 8 additions: rq = (4 log2(e) span + K / 16 + 32) u.
  lse    s and its rounding.
  loss   d = log q - log p is off by dd = s + rq + 4 u (|log q| + |log p|); where p and q are above 1/2 it is made from 1 - p and 1 - q and off by 2 (s + (K + 8) u) (1 - p) +
         2 (rq + (K + 8) u) (1 - q).  A word adds q d - q + p >= 0: for |d| below 1/2 by a series, off by q (|1 - e^-d| dd + dd^2) and (rq + 8 u) of itself; beyond by its
         terms, q dd + (rq + 4 u) q (|d| + 1) + (s + 4 u) p.  The other words' p: s.  Additions: (K + 8) u of all.  (The float64 value is made of the same terms, and its own d off
         by up to 2^-45.)
  diff   (s + 4 u) p + (rq + 4 u) q, and where p is above 1/2 that of 1 - p and 1 - q instead, with K u for the additions.  (The float64 values' own p and q are off by
         up to 2^-53 times the size of z and of the sums, below 2^-45, which counts where both are 1.)
  g      s p, or at the teacher's words that of diff; then half a step of the 16-bit type: e |g| (fp16: 2^-25 at the scale 2^14 / max c).
  dh, dW those summed, (V + 2) u and (T + 2) u of the absolute sums for the additions, and the result's own rounding."""

import pytest

import paper_2508_20258_b200 as sp
from oracle import distill as DI

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = 2.0 ** -23
LOG2E = 1.4426950408889634
INF = float("inf")


def inputs(T, V, D, K, dtype, logit="fp32", scale=2.5, seed=0, agree=0.0):
    """Random scores and teachers; words in any order, some twice, some not used, some with a logit of minus infinity, every fifth token without any.  agree: share of
    the tokens whose state points along the teacher's first word."""
    g = torch.Generator(device="cuda").manual_seed(seed * 1000 + T + V + D + K)
    h = torch.randn(T, D, device="cuda", generator=g).to(BITS[dtype])
    W = (torch.randn(V, D, device="cuda", generator=g) * (scale / D ** 0.5)).to(BITS[dtype])
    index = torch.randint(0, V, (T, K), device="cuda", generator=g)
    top = torch.randn(T, K, device="cuda", generator=g) * 3
    gone = torch.rand(T, K, device="cuda", generator=g)
    index = torch.where(gone < 0.1, torch.full_like(index, -7), index)
    top = torch.where(gone > 0.93, -INF, top)
    if T > 3:
        index[1::5] = -1
    if agree:
        sure = torch.rand(T, device="cuda", generator=g) < agree
        index[:, 0] = torch.where(sure, index[:, 0].clamp(min=0), index[:, 0])
        top[:, 0] = torch.where(sure, 3 + torch.rand(T, device="cuda", generator=g) * 20, top[:, 0])
        along = W[index[:, 0].clamp(min=0)].float() * (torch.linspace(1, 7, T, device="cuda") / scale ** 2 * 4)[:, None]
        h = torch.where(sure[:, None], along.to(h.dtype), h)
        if T > 3:
            index[1::5] = -1
    return h, W, index.contiguous(), top.to(BITS[logit]).contiguous()


class Result:
    def __init__(self, h, W, index, top, tau, red, grad=None, want="both", stream=None, **kw):
        T, K = index.shape
        n = T if red == "none" else 1
        lb, db, ob = (torch.full((m + 8,), 97.0, device="cuda") for m in (T, T * K, n))
        self.lse, self.diff, self.loss = lb[:T], db[:T * K].view(T, K), ob[:n]
        torch.cuda.synchronize()
        sp.linear_distill(h, W, index, top, self.lse, self.diff, self.loss, temperature=tau, reduction=red, stream=stream, **kw)
        if want:
            hb, wb = (torch.full((x.numel() + 64,), 97.0, dtype=x.dtype, device="cuda") for x in (h, W))
            self.dh = hb[:h.numel()].view_as(h) if want != "dW" else None
            self.dW = wb[:W.numel()].view_as(W) if want != "dh" else None
            torch.cuda.synchronize()
            sp.linear_distill_grad(h, W, index, self.lse, self.diff, grad, self.dh, self.dW, temperature=tau, reduction=red, stream=stream)
        assert sp.get_status(stream) == 0
        torch.cuda.synchronize()
        assert (lb[T:] == 97).all() and (db[T * K:] == 97).all() and (ob[n:] == 97).all()
        if want:
            assert (hb[h.numel():] == 97).all() and (wb[W.numel():] == 97).all()


def reference(h, W, index, top, tau, red, grad, dtype):
    """Values and tolerances of the module's docstring, in float64."""
    hd, Wd = h.double(), W.double()
    (T, D), V, K = h.shape, W.shape[0], index.shape[1]
    e = torch.finfo(BITS[dtype]).eps / 2
    z = hd @ Wd.t() / tau
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    p = logp.exp()
    used = (index >= 0) & (top != -INF)
    kept = used.any(1)
    t = torch.where(used, top.double() / tau, -INF)
    m = torch.where(kept, t.amax(1), 0.0)[:, None]
    span = (m - torch.where(used, t, m)).amax(1)
    w = torch.where(used, (t - m).exp(), 0.0)
    w = w / torch.where(kept, w.sum(1), 1.0)[:, None]
    q = torch.zeros_like(p).scatter_add_(1, index.clamp(min=0), w)
    size = (hd.abs() @ Wd.abs().t()).amax(1) / tau
    s = 2 * (D / 16 + D / 512 + 2) * U * size + 2 * (6 * LOG2E * z.abs().amax(1) + 4) * U + 2.0 ** -17
    rq = (4 * LOG2E * span + K / 16 + 32) * U
    s, rq = s[:, None], rq[:, None]
    has = q > 0
    logq = torch.where(has, q, 1.0).log()
    d = torch.where(has, logq - logp, 0.0)
    dd = s + rq + 4 * U * (logq.abs() + logp.abs())
    p_less, q_less = (1 - p).clamp(min=0), (1 - q).clamp(min=0)
    most = 2 * (s + (K + 8) * U) * p_less + 2 * (rq + (K + 8) * U) * q_less
    dd = torch.where((p > 0.51) & (q > 0.51), most, torch.where((p > 0.49) & (q > 0.49), torch.maximum(most, dd), dd)) + 2.0 ** -45
    word = torch.where(has, q * (d + torch.expm1(-d)), 0.0)
    near = q * (torch.expm1(-d).abs() * dd + dd * dd) + (rq + 8 * U) * word
    far = q * dd + (rq + 4 * U) * q * (d.abs() + 1) + (s + 4 * U) * p
    off = torch.where(has, torch.where(d.abs() < 0.49, near, torch.maximum(near, far)), 0.0)
    rest = torch.where(has, 0.0, p)
    each = torch.where(kept, tau ** 2 * (word + rest).sum(1), 0.0)
    d_each = tau ** 2 * ((off + s * rest).sum(1) + (K + 8) * U * (word + rest).sum(1)) + 4 * U * each.abs()
    d_each = torch.where(kept, d_each, 0.0)
    n = kept.sum()
    loss, d_loss = (each, d_each) if red == "none" else (each.sum()[None], d_each.sum()[None] + U * each.sum().abs())
    if red == "mean":
        loss, d_loss = loss / n, d_loss / n
    low, high = (s + 4 * U) * p + (rq + 4 * U) * q, (s + (K + 4) * U) * p_less + (rq + (K + 4) * U) * q_less
    off = torch.where(p < 0.49, low, torch.where(p > 0.51, high, torch.maximum(low, high))) + 2.0 ** -45
    at = index.clamp(min=0)
    there = (index >= 0) & kept[:, None]
    diff, d_diff = (torch.where(there, x.gather(1, at), 0.0) for x in (p - q, off))
    # entries of g that a word of the teacher's list stands for are diff, whether its q is 0 or not
    listed = torch.zeros_like(p).scatter_add_(1, at, there.double()) > 0
    c = torch.where(kept, grad.double().expand(T), 0.0) * tau / (n if red == "mean" else 1)
    g = c[:, None] * (p - q)
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    dg = c.abs()[:, None] * torch.where(listed, off, s * p)
    dg = dg + e * (g.abs() + dg) + tiny * c.abs().max() / 2.0 ** 14
    dh, dW = g @ Wd, g.t() @ hd
    tol_h = dg @ Wd.abs() + (V + 2) * U * (g.abs() @ Wd.abs())
    tol_W = dg.t() @ hd.abs() + (T + 2) * U * (g.abs().t() @ hd.abs())
    tol_h, tol_W = (x + (e + 2 * U) * (y.abs() + x) + tiny for x, y in ((tol_h, dh), (tol_W, dW)))
    lse = torch.where(kept, lse, INF)
    return kept, (lse, diff, loss, dh, dW), (s[:, 0] + 2 * U * lse.abs(), d_diff, d_loss, tol_h, tol_W)


def check(r, ref, names=("lse", "diff", "loss", "dh", "dW")):
    kept, want, tol = ref
    assert (r.lse[~kept] == INF).all() and (r.diff[~kept] == 0).all()
    for name, w, t in zip(("lse", "diff", "loss", "dh", "dW"), want, tol):
        if name not in names:
            continue
        got = getattr(r, name).double()
        if name == "lse":
            got, w, t = got[kept], w[kept], t[kept]
        assert torch.isfinite(got).all(), name
        worst = ((got - w).abs() / (t + 1e-300)).max() if got.numel() else torch.zeros(())
        assert float(worst) <= 1, f"{name}: {float(worst):.3g} of the tolerance"


# one token; a vocabulary of two, of a tile and one more; more words than the vocabulary has; the largest lists, by a warp and by a block; both tile heights and their edges; a
# copy of h (D no multiple of 64, many tokens); sums of 512 and several
SHAPES = [(1, 2, 8, 1), (1, 2, 8, 5), (3, 1, 8, 2), (1, 999, 2056, 17), (2, 257, 72, 256), (5, 1000, 136, 257), (7, 3000, 64, 1024), (31, 513, 1032, 33), (33, 511, 64, 32), (128, 300, 64, 100),
          (129, 4097, 128, 64), (256, 256, 64, 3), (300, 2049, 520, 128), (60, 40001, 64, 20), (1030, 5001, 72, 9)]


@pytest.mark.parametrize("T,V,D,K", SHAPES)
@pytest.mark.parametrize("dtype,logit,tau", [("bf16", "fp32", 1.0), ("bf16", "bf16", 2.0), ("fp16", "fp16", 0.5), ("fp16", "fp32", 5.0)])
def test_against_the_formulas(T, V, D, K, dtype, logit, tau):
    h, W, index, top = inputs(T, V, D, K, dtype, logit)
    for red in ("none", "mean", "sum"):
        up = 64.0 if dtype == "fp16" else 1.0
        grad = (torch.rand(T if red == "none" else 1, device="cuda", generator=torch.Generator(device="cuda").manual_seed(T)) + 0.5) * up
        ref = reference(h, W, index, top, tau, red, grad, dtype)
        if red == "mean" and not ref[0].any():
            continue
        r = Result(h, W, index, top, tau, red, grad)
        check(r, ref)
        if red == "mean":
            for only in ("dh", "dW"):
                assert torch.equal(getattr(Result(h, W, index, top, tau, red, grad, want=only), only), getattr(r, only))


@pytest.mark.parametrize("T,V,D,K", [(1, 1001, 256, 1), (40, 3001, 256, 1), (200, 1001, 128, 8), (300, 9001, 520, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("tau", [0.5, 1.0])
def test_small_losses_and_differences_keep_their_digits(T, V, D, K, dtype, tau):
    h, W, index, top = inputs(T, V, D, K, dtype, scale=3.0, agree=1.0)
    grad = torch.ones(T, device="cuda")
    ref = reference(h, W, index, top, tau, "none", grad, dtype)
    if T > 1:
        small = ref[1][2][ref[0]]
        assert (small < 1e-3).any() and (small > 1e-1).any()
    check(Result(h, W, index, top, tau, "none", grad), ref)


def test_the_oracle_agrees():
    h, W, index, top = inputs(23, 300, 64, 12, "bf16")
    for red in ("none", "mean", "sum"):
        grad = torch.ones(23 if red == "none" else 1, device="cuda")
        _, (lse, diff, loss, dh, dW), _ = reference(h, W, index, top, 1.5, red, grad, "bf16")
        args = [x.double().cpu().numpy() for x in (h, W)] + [index.cpu().numpy(), top.double().cpu().numpy()]
        o = DI.linear_distill(*args, 1.5, red)
        for got, want in zip((loss, lse, diff), o):
            assert torch.allclose(got.cpu().reshape(-1), torch.as_tensor(want).reshape(-1), rtol=1e-10, atol=1e-12)
        for got, want in zip((dh, dW), DI.linear_distill_grad(*args, grad.cpu().numpy(), 1.5, red)):
            assert torch.allclose(got.cpu(), torch.as_tensor(want), rtol=1e-9, atol=1e-11)


def test_a_vocabulary_in_pieces():
    # T V above 2^27: several pieces, whose words are placed piece by piece; a slice of the rows and of the words is checked in float64
    T, V, D, K = 3000, 70001, 64, 40
    h, W, index, top = inputs(T, V, D, K, "bf16")
    index[:, 3] = V - 1
    grad = torch.ones(1, device="cuda")
    r = Result(h, W, index, top, 1.0, "sum", grad)
    for rows in (slice(0, 40), slice(T - 40, T)):
        ref = reference(h[rows], W, index[rows], top[rows], 1.0, "sum", grad, "bf16")
        part = Result(h[rows].contiguous(), W, index[rows].contiguous(), top[rows].contiguous(), 1.0, "none", torch.ones(40, device="cuda"))
        r2 = type("R", (), dict(lse=r.lse[rows], diff=r.diff[rows], dh=r.dh[rows]))
        check(r2, ref, ("lse", "diff", "dh"))
        assert torch.equal(part.lse, r2.lse) and torch.equal(part.diff, r2.diff)
    want, size = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(want)
    for i in range(0, T, 250):
        rows = slice(i, i + 250)
        _, v, t = reference(h[rows], W, index[rows], top[rows], 1.0, "sum", grad, "bf16")
        want += v[4]
        tol += t[4]
    e = 2.0 ** -8
    assert ((r.dW.double() - want).abs() <= tol + e * want.abs()).all()


def test_gradients_against_differences_of_the_loss():
    # central differences of the kernel's own loss: off by step^2 / 6 times the third derivative (tau^2 times a third cumulant of numbers within R / tau: (2 R)^3 / tau), and by the noise of the losses over the step
    g = torch.Generator().manual_seed(2)
    T, V, D, tau = 3, 37, 16, 2.0
    h = (torch.randint(-8, 9, (T, D), generator=g) / 8).bfloat16().cuda()
    W = (torch.randint(-8, 9, (V, D), generator=g) / 16).bfloat16().cuda()
    index = torch.tensor([[4, 30, 7], [-1, -1, -1], [36, 36, 0]]).cuda()
    top = torch.randn(T, 3, generator=g).cuda()
    r = Result(h, W, index, top, tau, "sum")
    step = 2.0 ** -4

    def loss_at(hh, ww):
        return float(Result(hh, ww, index, top, tau, "sum", want=None).loss.double())

    for x, grad, other, first in ((h, r.dh, W, True), (W, r.dW, h, False)):
        R = float(other.double().abs().max())
        for i in [(0, 0), (0, 15), (1, 3), (2, 7)] + ([] if first else [(4, 2), (36, 9), (20, 4)]):
            e = torch.zeros_like(x)
            e[i] = step
            assert torch.equal((x + e).double() - e.double(), x.double())
            num = (loss_at(x + e, W) - loss_at(x - e, W) if first else loss_at(h, x + e) - loss_at(h, x - e)) / (2 * step)
            tol = T * step ** 2 / 6 * (2 * R) ** 3 + 2 * T * tau ** 2 * 2.0 ** -17 / step + 2.0 ** -7 * (abs(num) + R * T * V * tau * 2.0 ** -8)
            assert abs(num - float(grad[i].double())) <= tol


@pytest.mark.parametrize("T", [6, 200])
def test_tokens_that_do_not_count(T):
    h, W, index, top = inputs(T, 700, 64, 5, "bf16")
    for empty, logits in ((torch.full_like(index, -1), top), (index.clamp(min=0), torch.full_like(top, -INF))):
        for red, want in (("mean", float("nan")), ("sum", 0.0), ("none", 0.0)):
            r = Result(h, W, empty, logits, 1.0, red)
            assert (torch.isnan(r.loss) if want != want else r.loss == want).all()
            assert (r.lse == INF).all() and (r.diff == 0).all() and (r.dh == 0).all() and (r.dW == 0).all()
    # an overflowed loss scale: the tokens that do not count still have nothing
    r = Result(h, W, index, top, 1.0, "sum", torch.full((1,), INF, device="cuda"))
    out = r.lse == INF
    assert out.any() and (r.dh[out] == 0).all() and not torch.isfinite(r.dh[~out]).all()


@pytest.mark.parametrize("T,V,D", [(40, 300, 64), (300, 700, 72), (150, 3001, 264)])
@pytest.mark.parametrize("value", [float("nan"), INF, 65504.0])
def test_rows_of_tokens_that_do_not_count_may_hold_anything(T, V, D, value):
    h, W, index, top = inputs(T, V, D, 6, "fp16")
    good = Result(h, W, index, top, 1.0, "mean")
    bad = h.clone()
    bad[good.lse == INF] = value
    r = Result(bad, W, index, top, 1.0, "mean")
    for name in ("lse", "diff", "loss", "dh", "dW"):
        assert torch.equal(getattr(r, name), getattr(good, name)), name


def test_words_outside_the_vocabulary_and_wild_logits_are_loud_and_stay_alone():
    h, W, index, top = inputs(40, 300, 64, 6, "bf16")
    good = Result(h, W, index, top, 1.0, "none")
    row = 2
    for kind in ("word", "far word", "nan", "inf"):
        i2, t2 = index.clone(), top.clone()
        i2[row] = torch.arange(6, device="cuda")
        t2[row] = 0.0
        if kind == "word":
            i2[row, 3] = 300
        elif kind == "far word":
            i2[row, 3] = 1 << 40
        else:
            t2[row, 3] = float(kind)
        r = Result(h, W, i2, t2, 1.0, "none")
        assert torch.isnan(r.loss[row]) and torch.isnan(r.diff[row]).any() and torch.isnan(r.dh[row]).all(), kind
        others = torch.arange(40, device="cuda") != row
        for name in ("loss", "lse", "diff", "dh"):
            assert torch.equal(getattr(r, name)[others], getattr(good, name)[others]), (kind, name)
    # not used: what stands beside it does not matter
    t2 = torch.where(index < 0, float("nan"), top)
    r = Result(h, W, index, t2, 1.0, "none")
    for name in ("loss", "lse", "diff", "dh", "dW"):
        assert torch.equal(getattr(r, name), getattr(good, name)), name


def test_order_and_equal_words():
    # the words' order changes nothing but the order of diff; a word that stands twice is a word with the sum
    h, W, index, top = inputs(50, 700, 64, 24, "bf16")
    index = torch.stack([torch.randperm(700, generator=torch.Generator().manual_seed(i))[:24] for i in range(50)]).cuda()
    top = top.masked_fill(top == -INF, -1.0)
    a = Result(h, W, index, top, 1.0, "none")
    turn = torch.randperm(24, generator=torch.Generator().manual_seed(9)).cuda()
    b = Result(h, W, index[:, turn].contiguous(), top[:, turn].contiguous(), 1.0, "none")
    assert torch.equal(a.lse, b.lse) and torch.equal(a.diff[:, turn], b.diff) and torch.equal(a.dh, b.dh) and torch.equal(a.dW, b.dW) and torch.equal(a.loss, b.loss)
    half = torch.cat([index, index], 1).contiguous()
    c = Result(h, W, half, torch.cat([top, top], 1).contiguous(), 1.0, "none")
    check(c, reference(h, W, half, torch.cat([top, top], 1), 1.0, "none", torch.ones(50, device="cuda"), "bf16"))
    assert torch.equal(c.diff[:, :24], c.diff[:, 24:]) and torch.equal(c.lse, a.lse)


@pytest.mark.parametrize("T,V,D,K", [(20, 3000, 64, 20), (300, 5001, 136, 64)])
def test_same_bits_every_time_captured_replayed_and_on_another_stream(T, V, D, K):
    h, W, index, top = inputs(T, V, D, K, "bf16", agree=0.3)
    want = Result(h, W, index, top, 2.0, "mean")
    side = torch.cuda.Stream()
    names = ("lse", "diff", "loss", "dh", "dW")
    again = Result(h, W, index, top, 2.0, "mean", stream=side)
    assert all(torch.equal(getattr(want, n), getattr(again, n)) for n in names)
    out = {n: torch.empty_like(getattr(want, n)) for n in names}
    ws = [torch.empty(sp.linear_distill_workspace(T, V, D, K, grad=g), dtype=torch.uint8, device="cuda") for g in (False, True)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sp.linear_distill(h, W, index, top, out["lse"], out["diff"], out["loss"], temperature=2.0, workspace=ws[0])
        sp.linear_distill_grad(h, W, index, out["lse"], out["diff"], None, out["dh"], out["dW"], temperature=2.0, workspace=ws[1])
    keep = index.clone(), h.clone()
    for _ in range(3):
        index.copy_(torch.where(torch.rand(T, K, device="cuda") < 0.5, -1, keep[0]))      # other words between the replays
        h.copy_(torch.randn(T, D, device="cuda"))
        graph.replay()
        index.copy_(keep[0])
        h.copy_(keep[1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(want, n), out[n]) for n in names)


def test_end_of_a_students_training_step():
    # norm, distillation, gradients and the norm's gradients in a row, as they are used, against float64 of the whole chain: the hidden state in between is rounded to 16
    # bits (2^-8 of it, on either way), which bounds the differences
    T, V, D, K, tau = 120, 2000, 256, 16, 2.0
    h, W, index, top = inputs(T, V, D, K, "bf16")
    x = torch.randn(T, D, device="cuda").bfloat16()
    gamma, beta = (1 + 0.1 * torch.randn(D, device="cuda")), 0.1 * torch.randn(D, device="cuda")
    mean, rstd = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    lse, diff, loss = torch.empty(T, device="cuda"), torch.empty(T, K, device="cuda"), torch.empty(1, device="cuda")
    dh, dW, dx, dgamma, dbeta = torch.empty_like(h), torch.empty_like(W), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    sp.layernorm(x, gamma, beta, h, mean, rstd)
    sp.linear_distill(h, W, index, top, lse, diff, loss, temperature=tau)
    sp.linear_distill_grad(h, W, index, lse, diff, None, dh, dW, temperature=tau)
    sp.layernorm_grad(dh, x, gamma, mean, rstd, dx, dgamma, dbeta)
    assert sp.get_status() == 0
    xd, gd, bd, Wd = (v.double().requires_grad_() for v in (x, gamma, beta, W))
    hidden = torch.nn.functional.layer_norm(xd, (D,), gd, bd, 1e-5)
    hidden.retain_grad()
    logp = torch.log_softmax(hidden @ Wd.t() / tau, 1)
    used = (index >= 0) & (top != -INF)
    t = torch.where(used, top.double() / tau, -INF)
    kept = used.any(1)
    q = torch.zeros_like(logp).scatter_add(1, index.clamp(min=0), torch.where(used, torch.softmax(torch.where(kept[:, None], t, 0.0), 1), 0.0))
    each = tau ** 2 * (torch.special.entr(q).neg() - q * logp).sum(1)
    total = torch.where(kept, each, 0.0).sum() / kept.sum()
    total.backward()
    total = total.detach()
    # norms: half a step of rounding in h moves the scores by 2^-9 of their size (random signs), p and with it g by as much relative
    far = lambda got, want: float((got.double() - want).norm() / want.norm())  # noqa: E731
    assert abs(float(loss) - float(total)) <= 2.0 ** -7 * float(total)
    for got, want in ((dh, hidden.grad), (dW, Wd.grad), (dx, xd.grad), (dgamma, gd.grad), (dbeta, bd.grad)):
        assert far(got, want) <= 2.0 ** -6


def test_refusals_of_the_binding():
    h, W, index, top = inputs(4, 30, 64, 3, "bf16")
    lse, diff, loss = torch.empty(4, device="cuda"), torch.empty(4, 3, device="cuda"), torch.empty(1, device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        sp.linear_distill(h, W, index.t().contiguous().t(), top, lse, diff, loss)
    for kw in (dict(temperature=0.0), dict(temperature=1e6), dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(sp.SpError) as e:
            sp.linear_distill(h, W, index, top, lse, diff, loss, **kw)
        assert e.value.status == sp.ERR_INVALID_ARG
    with pytest.raises(sp.SpError) as e:
        sp.linear_distill_grad(h, W, index, lse, diff, None, h, torch.empty_like(W))
    assert e.value.status == sp.ERR_INVALID_ARG
    assert sp.get_status() == 0


# a word per lane, several, and lists that are read where they are needed; of a warp's lanes some without any
@pytest.mark.parametrize("K", [1, 2, 20, 40, 200])
@pytest.mark.parametrize("place", ["lowest", "middle", "highest", "none"])
@pytest.mark.parametrize("value", [float("nan"), INF, -INF])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_row_of_W_that_is_not_finite(K, place, value, dtype):
    if K == 1 and place == "middle":
        pytest.skip("one word is the lowest and the highest")
    T, V, D, bad, at = 12, 700, 64, 350, 3
    h, W, _, _ = inputs(T, V, D, K, dtype)
    g = torch.Generator().manual_seed(K)
    h[:, at] = torch.where(torch.arange(T, device="cuda") % 2 == 0, 1.0, -1.0)
    below = {"lowest": 0, "middle": K // 2, "highest": K - 1, "none": K // 2}[place]
    above = K - below - (place != "none")
    index = torch.stack([torch.cat([torch.randperm(bad, generator=g)[:below], torch.tensor([bad] if place != "none" else [], dtype=torch.int64),
                                    bad + 1 + torch.randperm(V - bad - 1, generator=g)[:above]])[torch.randperm(K, generator=g)] for _ in range(T)]).cuda()
    top = torch.randn(T, K, generator=g).cuda()
    out = torch.arange(T, device="cuda") % 6 == 5
    index[out] = -1
    W[bad, at] = -60000.0      # the words' scores 0 of itself under a softmax, or above all others
    low = Result(h, W, index, top, 1.0, "none")
    W[bad, at] = 60000.0
    high = Result(h, W, index, top, 1.0, "none")
    W[bad, at] = value
    r = Result(h, W, index, top, 1.0, "none")
    assert (r.lse[out] == INF).all() and (r.loss[out] == 0).all() and (r.diff[out] == 0).all() and (r.dh[out] == 0).all()
    # a score of minus infinity: p is 0 there, as of one of -60000, and only the loss tells them apart, where the teacher has the word
    gone = ~out & (h[:, at] * value == -INF)
    finite = low if value < 0 else high
    assert value != value or gone.sum() >= 4
    assert torch.equal(r.lse[gone], finite.lse[gone]) and torch.equal(r.diff[gone], finite.diff[gone])
    assert (r.loss[gone] == INF).all() if place != "none" else torch.equal(r.loss[gone], finite.loss[gone])
    others = torch.arange(D, device="cuda") != at
    assert torch.equal(r.dh[gone][:, others], finite.dh[gone][:, others])
    # a NaN, or plus infinity: all of the token is NaN
    rest = ~out & ~gone
    assert rest.sum() >= 4 and all(torch.isnan(x[rest]).all() for x in (r.lse, r.loss, r.diff, r.dh)) and torch.isnan(r.dW).all()
    for red in ("mean", "sum"):
        assert torch.isnan(Result(h, W, index, top, 1.0, red, want=None).loss).all()


@pytest.mark.parametrize("value", [float("nan"), INF])
@pytest.mark.parametrize("T,K", [(20, 3), (40, 33), (300, 150)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_token_that_counts_and_is_not_finite_stays_alone(T, K, dtype, value):
    h, W, index, top = inputs(T, 700, 64, K, dtype)
    index[2], top[2] = torch.arange(K, device="cuda"), 0.0
    good = Result(h, W, index, top, 1.0, "none")
    h[2, 5] = value
    r = Result(h, W, index, top, 1.0, "none")
    assert all(torch.isnan(x[2]).all() for x in (r.lse, r.loss, r.diff, r.dh)) and torch.isnan(r.dW).all()
    others = torch.arange(T, device="cuda") != 2
    for name in ("loss", "lse", "diff", "dh"):
        assert torch.equal(getattr(r, name)[others], getattr(good, name)[others]), name


@pytest.mark.parametrize("D", [1024, 4096])
def test_the_score_of_a_settled_word_is_not_cut_off(D):
    # fp16 states along their word's row of W, all other rows 0: p - q is -(V - 1) / (V - 1 + e^z), and with p next to 1 its relative error that of z itself.  Products of fp16 numbers are exact
    # in fp32.  Cut off, z is always too small (2e-7 of itself); rounded to nearest its n = 1 + 2 + D / 256 + 5 roundings, each at most u = 2^-24 of z, are as often up as down, and the mean over T
    # tokens is beyond u sqrt(n) sqrt(2 ln(2e9) / T) of z once in 1e9 (Hoeffding).  log2 e in fp32: 2^-25 of z.  Two exponentials, good to 2^-22, and four roundings, whatever z is.
    T, V, word = 8192, 512, 300
    g = torch.Generator(device="cuda").manual_seed(D)
    W = torch.zeros(V, D, dtype=torch.float16, device="cuda")
    W[word] = (0.5 + torch.rand(D, device="cuda", generator=g)) * torch.where(torch.rand(D, device="cuda", generator=g) < 0.5, -1.0, 1.0)
    h = ((0.1 + torch.rand(T, D, device="cuda", generator=g)) * (25 / (0.6 * D)) * W[word].sign()).half()
    index, top = torch.full((T, 1), word, device="cuda"), torch.zeros(T, 1, device="cuda")
    r = Result(h, W, index, top, 1.0, "none", want=None)
    z = h.double() @ W[word].double()
    assert float(z.min()) > 20 and float(z.max()) < 30
    odds = (V - 1) * torch.exp(-z)
    off = ((r.diff[:, 0].double() / (-odds / (1 + odds)) - 1) / z).mean()
    u, n = 2.0 ** -24, 1 + 2 + D / 256 + 5
    assert abs(float(off)) <= u * (n * 2 * 21.5 / T) ** 0.5 + 2.0 ** -25 + (2 * 2.0 ** -22 + 4 * u) / 20, float(off)


@pytest.mark.parametrize("T,V,D,K", [(1, 4001, 256, 8), (16, 3001, 512, 20), (64, 2001, 256, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gradients_of_few_tokens_are_as_good_as_rounded_once(T, V, D, K, dtype):
    # Up to 64 tokens g is held with its rounding errors, to e^2 (2^-16, 2^-22) of an entry, and the scores' errors move it by 1e-6 to 1e-5: at most a twentieth of what rounding a gradient once does
    # (a uniform error of up to e of a value, about e / 2 in the norm: 2^-9, 2^-12), which adds 1 / 800 to the norm.  g rounded without them adds as much as the rounding itself: sqrt 2 where a
    # gradient is one product.
    h, W, index, top = inputs(T, V, D, K, dtype)
    top = top.masked_fill(top == -INF, -1.0)
    grad = torch.full((T,), 64.0 if dtype == "fp16" else 1.0, device="cuda")
    r = Result(h, W, index, top, 1.0, "none", grad)
    kept, (_, _, _, dh, dW), _ = reference(h, W, index, top, 1.0, "none", grad, dtype)
    listed = torch.zeros(V, dtype=torch.bool, device="cuda")
    listed[index[kept].clamp(min=0).flatten()] = True
    for got, want in ((r.dh, dh), (r.dW[listed], dW[listed]), (r.dW[~listed], dW[~listed])):
        once = (want.to(BITS[dtype]).double() - want).norm()
        assert float(once) > 0 and float((got.double() - want).norm() / once) <= 1.02


@pytest.mark.parametrize("tau", [sp.DISTILL_MIN_TEMPERATURE, 0.01, 100.0, sp.DISTILL_MAX_TEMPERATURE])
@pytest.mark.parametrize("T,V,D", [(5, 1000, 112), (150, 3000, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_temperatures_from_end_to_end(T, V, D, dtype, tau):
    # One word per token, so that no q is too small for float64.  Scores of 1e5: p falls below what fp32 and bf16 hold, 2^-126, which is all that is lost of g there, as held, before its factor.
    h, W, index, top = inputs(T, V, D, 1, dtype)
    grad = torch.full((T,), (64.0 if dtype == "fp16" else 1.0) / max(tau, 1.0), device="cuda")
    ref = reference(h, W, index, top, tau, "none", grad, dtype)
    r = Result(h, W, index, top, tau, "none", grad)
    check(r, ref, ("lse", "diff", "loss", "dh"))
    lost = T * 2.0 ** -126 * float(h.abs().max()) * max(1.0, float(grad.max()) * tau)
    assert ((r.dW.double() - ref[1][4]).abs() <= ref[2][4] + lost).all()
