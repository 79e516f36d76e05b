"""The vocabulary cross entropy and its gradients against the oracle (float64 of the formulas).

Tolerances, from the arithmetic.  u = 2^-23 bounds one fp32 addition on the tensor cores (which may cut instead of rounding).
  score     products of 16-bit numbers are exact in fp32; D of them are summed: dz = D u max_v sum_d |h_d W_vd|.
  lse       every score is off by at most dz; an exponent z log2 e - m of size up to E = |z log2 e| + |m| is rounded once or twice and the hardware's
            2^x is good to 2^-22, so a term is off by r = (E + 4) 2^-23 relative; so is a sum of such terms, plus a few 2^-24
            for the additions (256-column tiles in four chains, then joined: below 2^-17 in all); the result is rounded
            once: |lse| 2^-23.
  loss      the same, plus dz for the target's own score.
  g         p is off by dp = 2 dz + 2 r relative (a score and the lse), then g is rounded to 16 bits: half a step, e = eps / 2
            (and fp16's smallest number, 2^-25, at the scale 2^14 / max c that the coefficients are brought to).
  (Scores are summed 512 products at a time, so this bound is generous; what it would hide, the test on exact scores shows.)
  dh        sum_v (e |g| + (1 + e) c p dp) |W| + V u sum_v |g W|, then rounded to 16 bits: e |dh| (fp16: + 2^-25).
  dW        the same over the tokens, with |h| and T u."""

import numpy as np
import pytest

import paper_2508_20258_b200 as sp
from oracle import linear as LN

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0 ** -23
LOG2E = 1.4426950408889634


def inputs(T, V, D, dtype, seed=0, scale=2.5, ignored=True):
    g = torch.Generator().manual_seed(seed * 1000 + T + V + D)
    h = torch.randn(T, D, generator=g).to(BITS[dtype])
    W = (torch.randn(V, D, generator=g) * (scale / D ** 0.5)).to(BITS[dtype])
    t = torch.randint(0, V, (T,), generator=g)
    t[0], t[-1] = V - 1, 0
    if ignored and T > 3:
        t[1::5] = -100
    return h, W, t


def forward(h, W, t, red, stream=None, **kw):
    T = h.shape[0]
    lb, ob = torch.full((T + 8,), 97.0, device="cuda"), torch.full(((T if red == "none" else 1) + 8,), 97.0, device="cuda")
    lse, loss = lb[:T], ob[:-8]
    sp.linear_ce(h, W, t, lse, loss, reduction=red, stream=stream, **kw)
    assert sp.get_status(stream) == 0
    assert (lb[T:] == 97).all() and (ob[-8:] == 97).all()
    return lse, loss


def backward(h, W, t, lse, grad, red, want="both", **kw):
    dh = torch.full_like(h, float("nan")) if want != "dW" else None
    wb = torch.full((W.numel() + 64,), 97.0, dtype=W.dtype, device="cuda")
    dW = wb[:W.numel()].view_as(W) if want != "dh" else None
    if dW is not None:
        dW.fill_(float("nan"))
    sp.linear_ce_grad(h, W, t, lse, grad, dh, dW, reduction=red, **kw)
    assert sp.get_status() == 0
    assert (wb[W.numel():] == 97).all()
    return dh, dW


def bounds(h, W, t, grad, red, dtype):
    """Oracle values and the tolerances of the module's docstring."""
    hd, Wd, tn = h.double().numpy(), W.double().numpy(), t.numpy()
    T, D = hd.shape
    V = Wd.shape[0]
    e = float(torch.finfo(BITS[dtype]).eps) / 2
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    loss, lse, each, kept = LN.linear_ce(hd, Wd, tn, red)
    size = (np.abs(hd) @ np.abs(Wd).T).max(axis=1)
    dz = D * U * size
    r = (2 * LOG2E * size + 4) * U
    dlse = dz + r + 2.0 ** -17 + np.abs(lse) * U
    dloss = dlse + dz + np.abs(each) * U
    if red == "sum":
        dloss = dloss[kept].sum() + abs(loss) * U
    elif red == "mean":
        dloss = (dloss[kept].mean() if kept.any() else 0) + abs(loss) * U
    dh, dW, g, p, c = LN.linear_ce_grad(hd, Wd, tn, grad.double().numpy(), red)
    dp = (2 * dz + 2 * r + 2.0 ** -17)[:, None]
    top = np.abs(c).max() if len(c) else 0.0
    dg = e * np.abs(g) + (1 + e) * np.abs(c)[:, None] * p * dp + tiny * top / 2.0 ** 14
    tol_h = dg @ np.abs(Wd) + V * U * (np.abs(g) @ np.abs(Wd)) + (e + 2 * U) * np.abs(dh) + tiny
    tol_W = dg.T @ np.abs(hd) + T * U * (np.abs(g).T @ np.abs(hd)) + (e + 2 * U) * np.abs(dW) + tiny
    return (loss, lse, dh, dW), (dloss, dlse, tol_h, tol_W)


def inside(got, ref, tol):
    d = np.abs(got.double().cpu().numpy() - ref)
    return bool((d <= tol).all())


# one token (by rows, in one and several reads of a row, and too long for it); a vocabulary of two, of a tile and one more, odd; one stage of D, one
# sum of 512 and several, ragged ones; both tile heights and their edges
SHAPES = [(1, 2, 8), (3, 1, 8), (1, 256, 64), (1, 999, 2056), (1, 300, 16384), (1, 257, 16392), (130, 300, 1544), (2, 257, 72), (5, 1000, 136), (31, 513, 1032), (33, 511, 64), (128, 300, 64), (129, 4097, 128), (256, 256, 64), (300, 2049, 520)]


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("red", ["none", "mean", "sum"])
def test_against_the_formulas(T, V, D, dtype, red):
    h, W, t = inputs(T, V, D, dtype)
    up = 64.0 if dtype == "fp16" else 1.0
    grad = torch.rand(T if red == "none" else 1, generator=torch.Generator().manual_seed(T)) * up + 0.5 * up
    ref, tol = bounds(h, W, t, grad, red, dtype)
    dev = [v.cuda() for v in (h, W, t)]
    lse, loss = forward(*dev, red)
    assert inside(lse, ref[1], tol[1])
    assert inside(loss, np.reshape(ref[0], -1), tol[0])
    dh, dW = backward(*dev, lse, grad.cuda(), red)
    assert inside(dh, ref[2], tol[2])
    assert inside(dW, ref[3], tol[3])
    only_h, _ = backward(*dev, lse, grad.cuda(), red, want="dh")
    _, only_W = backward(*dev, lse, grad.cuda(), red, want="dW")
    assert torch.equal(only_h, dh) and torch.equal(only_W, dW)


def test_exact_scores_leave_only_the_exponentials():
    # small integers: the scores are exact in fp32, so lse and loss are held to the error of 2^x and log alone
    g = torch.Generator().manual_seed(5)
    for T, V, D in [(1, 1000, 64), (70, 777, 40), (200, 5000, 64)]:
        h, W = torch.randint(-1, 2, (T, D), generator=g).bfloat16(), torch.randint(-1, 2, (V, D), generator=g).bfloat16()
        t = torch.randint(0, V, (T,), generator=g)
        loss, lse, each, _ = LN.linear_ce(h.double().numpy(), W.double().numpy(), t.numpy(), "none")
        got_lse, got = forward(h.cuda(), W.cuda(), t.cuda(), "none")
        tol = (2 * LOG2E * D + 4) * U + 2.0 ** -17
        assert inside(got_lse, lse, tol) and inside(got, loss, tol)


def test_gradients_against_differences_of_the_loss():
    # central differences of the kernel's own loss: off by step^2 / 6 times the third derivative (a third cumulant of numbers within
    # +-R: at most (2 R)^3), and by the fp32 noise of the losses over the step
    g = torch.Generator().manual_seed(2)
    T, V, D = 3, 37, 16
    h = (torch.randint(-8, 9, (T, D), generator=g) / 8).bfloat16()
    W = (torch.randint(-8, 9, (V, D), generator=g) / 16).bfloat16()
    t = torch.tensor([4, -100, 36])
    dev_t = t.cuda()
    lse, _ = forward(h.cuda(), W.cuda(), dev_t, "sum")
    dh, dW = backward(h.cuda(), W.cuda(), dev_t, lse, None, "sum")
    step = 2.0 ** -4

    def loss_at(hh, ww):
        return float(forward(hh.cuda(), ww.cuda(), dev_t, "sum")[1].double())

    for x, grad, other, first in ((h, dh, W, True), (W, dW, h, False)):
        R = float(other.double().abs().max())
        for i in [(0, 0), (0, 15), (1, 3), (2, 7)] + ([] if first else [(4, 2), (36, 9), (20, 20 % D)]):
            e = torch.zeros_like(x)
            e[i] = step                                            # exact: x and the step are multiples of 1/16, |x| < 2
            assert torch.equal((x + e).double() - e.double(), x.double())
            num = (loss_at(x + e, W) - loss_at(x - e, W) if first else loss_at(h, x + e) - loss_at(h, x - e)) / (2 * step)
            tol = T * step ** 2 / 6 * (2 * R) ** 3 + 2 * T * 2.0 ** -17 / step + 2.0 ** -7 * (abs(num) + R * T * V * 2.0 ** -8)
            assert abs(num - float(grad[i].double())) <= tol


@pytest.mark.parametrize("T", [6, 200])
def test_tokens_that_do_not_count(T):
    V, D = 700, 64
    h, W, t = inputs(T, V, D, "bf16")
    none_left = torch.full_like(t, -100).cuda()
    for red, want in (("mean", float("nan")), ("sum", 0.0), ("none", 0.0)):
        lse, loss = forward(h.cuda(), W.cuda(), none_left, red)
        assert (torch.isnan(loss) if np.isnan(want) else loss == want).all() and torch.isfinite(lse).all()
        dh, dW = backward(h.cuda(), W.cuda(), none_left, lse, None, red)
        assert (dh == 0).all() and (dW == 0).all()
    # another index to ignore, one that is a token of the vocabulary
    t2 = torch.where(t == -100, torch.tensor(7), t)
    for red in ("none", "mean"):
        a = forward(h.cuda(), W.cuda(), t.cuda(), red)
        kept7 = torch.where(t2 == 7, torch.tensor(-100), t2)
        b = forward(h.cuda(), W.cuda(), t2.cuda(), red, ignore_index=7)
        if torch.equal(kept7, t):
            assert torch.equal(a[1], b[1])
    # an overflowed loss scale: the tokens that are ignored still have nothing
    lse, _ = forward(h.cuda(), W.cuda(), t.cuda(), "sum")
    dh, _ = backward(h.cuda(), W.cuda(), t.cuda(), lse, torch.full((1,), float("inf"), device="cuda"), "sum")
    assert (dh[t.cuda() == -100] == 0).all() and not torch.isfinite(dh[t.cuda() != -100]).all()


@pytest.mark.parametrize("T,V,D", [(40, 300, 64), (300, 700, 72), (150, 3000, 264)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 65504.0])
def test_rows_of_ignored_tokens_may_hold_anything(T, V, D, value):
    h, W, t = inputs(T, V, D, "fp16")
    h[t == -100] = 0
    ref = forward(h.cuda(), W.cuda(), t.cuda(), "mean")
    bad = h.clone()
    bad[t == -100] = value
    lse, loss = forward(bad.cuda(), W.cuda(), t.cuda(), "mean")
    assert torch.equal(loss, ref[1])
    got = backward(bad.cuda(), W.cuda(), t.cuda(), lse, None, "mean")
    good = backward(h.cuda(), W.cuda(), t.cuda(), ref[0], None, "mean")
    assert torch.equal(got[0], good[0]) and torch.equal(got[1], good[1])


def test_targets_outside_the_vocabulary_are_loud():
    h, W, t = inputs(20, 300, 64, "bf16", ignored=False)
    for wrong in (300, 511, -1, 1 << 40, -(1 << 40)):
        t2 = t.clone()
        t2[4] = wrong
        lse, loss = forward(h.cuda(), W.cuda(), t2.cuda(), "none")
        assert torch.isnan(loss[4]) and torch.isfinite(loss[[i for i in range(20) if i != 4]]).all() and torch.isfinite(lse).all()
        assert torch.isnan(forward(h.cuda(), W.cuda(), t2.cuda(), "mean")[1]).all()
        dh, dW = backward(h.cuda(), W.cuda(), t2.cuda(), lse, None, "mean")
        assert torch.isnan(dh[4]).all() and torch.isnan(dW).any()


def test_large_scores_minus_infinity_and_nan():
    T, V, D = 9, 600, 64
    h, W = torch.zeros(T, D), torch.zeros(V, D)
    h[:, 0], W[:, 0] = 1.0, torch.linspace(-3e4, 3e4, V)         # exponents far outside fp32's without the maximum
    h[1, 0] = -1.0
    h[2, 0] = 0.0
    W[5, 1] = -float("inf")
    h[:, 1] = 1.0                                                # score 5 is minus infinity: probability 0
    h[3, 2] = float("nan")
    h, W = h.bfloat16(), W.bfloat16()
    t = torch.tensor([0, 0, 300, 7, 599, 5, 1, 2, -100])
    lse, loss = forward(h.cuda(), W.cuda(), t.cuda(), "none")
    z = h.double() @ torch.where(torch.isinf(W), 0.0, W.double()).t()
    z[:, 5] = -float("inf")
    want = torch.logsumexp(z, 1)
    keep = [0, 1, 2, 4, 6, 7, 8]
    assert ((lse.double().cpu() - want)[keep].abs() <= 3e4 * 2.0 ** -21 + 2.0 ** -17).all()
    assert torch.isnan(lse[3]) and torch.isnan(loss[3])
    assert loss[5] == float("inf")                               # the target itself has probability 0
    assert loss[8] == 0 and torch.isfinite(loss[[0, 1, 2, 4, 6, 7]]).all()


def test_a_tile_of_the_vocabulary_with_nothing_finite():
    # 256 columns of minus infinity leave a tile with no maximum; the other tiles decide
    T, V, D = 130, 600, 64
    h, W, t = inputs(T, V, D, "bf16", ignored=False)
    h[:, 0] = 1.0
    W[256:512, 0] = -float("inf")
    t = t % 256
    z = h.double() @ torch.where(torch.isinf(W), 0.0, W.double()).t()
    z[:, 256:512] = -float("inf")
    for rows in (T, 3):
        lse, loss = forward(h[:rows].cuda(), W.cuda(), t[:rows].cuda(), "mean")
        assert ((lse.double().cpu() - torch.logsumexp(z, 1)[:rows]).abs() < 1e-4).all() and torch.isfinite(loss).all()


def test_the_same_bits_every_time_and_whatever_the_buffers_hold():
    h, W, t = inputs(600, 9000, 264, "bf16")
    dev = [v.cuda() for v in (h, W, t)]
    first = None
    for fill in (0, 255, 127):
        f = torch.full((sp.linear_ce_workspace(600, 9000, 264),), fill, dtype=torch.uint8, device="cuda")
        b = torch.full((sp.linear_ce_workspace(600, 9000, 264, True),), fill, dtype=torch.uint8, device="cuda")
        lse, loss = forward(*dev, "mean", workspace=f)
        got = [lse, loss, *backward(*dev, lse, None, "mean", workspace=b)]
        first = first or got
        assert all(torch.equal(a, c) for a, c in zip(first, got))


# many pieces of the vocabulary (128 Mi entries of g each), few rows and many slices, both at once; references row by row on the GPU in float64
@pytest.mark.parametrize("T,V,D,dtype", [(600, 45001, 1000, "bf16"), (40000, 120001, 16, "bf16"), (3, 300001, 64, "fp16"), (16384, 50000, 264, "bf16"), (2048, 200000, 16, "fp16")])
def test_pieces_and_slices(T, V, D, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(T, D, device="cuda", generator=g).to(BITS[dtype])
    W = (torch.randn(V, D, device="cuda", generator=g) * (2 / D ** 0.5)).to(BITS[dtype])
    t = torch.randint(0, V, (T,), device="cuda", generator=g)
    t[T // 2] = -100
    c = torch.rand(T, device="cuda", generator=g) + 0.5
    lse, loss = forward(h, W, t, "none")
    dh, dW = backward(h, W, t, lse, c, "none")
    e = float(torch.finfo(BITS[dtype]).eps) / 2
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    rW, sW = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for i in range(0, T, 4096):
        hd, td, cd = h[i:i + 4096].double(), t[i:i + 4096], c[i:i + 4096].double()
        z = hd @ W.double().t()
        want = torch.logsumexp(z, 1)
        size = float((hd.abs().amax(1) * D * W.double().abs().max()).max())
        dz, r = D * U * size, (2 * LOG2E * size + 4) * U
        assert ((lse[i:i + 4096].double() - want).abs() <= dz + r + 2.0 ** -17 + want.abs() * U).all()
        kept = td != -100
        at = torch.where(kept, td, 0)[:, None]
        own = torch.where(kept, want - z.gather(1, at)[:, 0], 0.0)
        assert ((loss[i:i + 4096].double() - own).abs() <= 2 * dz + r + 2.0 ** -17 + 2 * want.abs() * U).all()
        p = (z - want[:, None]).exp() * (cd * kept)[:, None]
        gd = p.scatter_add(1, at, -(cd * kept)[:, None])
        dp = 2 * dz + 2 * r + 2.0 ** -17
        dg = e * gd.abs() + (1 + e) * dp * p + tiny * 2 / 2.0 ** 14
        rh = gd @ W.double()
        tol = dg @ W.double().abs() + V * U * (gd.abs() @ W.double().abs()) + (e + 2 * U) * rh.abs() + tiny
        assert ((dh[i:i + 4096].double() - rh).abs() <= tol).all()
        rW += gd.t() @ hd
        sW += dg.t() @ hd.abs() + T * U * (gd.abs().t() @ hd.abs())
        del z, p, gd, dg
    assert ((dW.double() - rW).abs() <= sW + (e + 2 * U) * rW.abs() + tiny).all()


def test_offsets_beyond_32_bits_in_the_weights():
    T, V, D = 4, 600000, 4096                                   # 2.5e9 elements
    W = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    W[-1], W[V // 2] = 1.0 / 64, -1.0 / 64
    h = torch.ones(T, D, dtype=torch.bfloat16, device="cuda")
    h[1] = -1.0
    t = torch.tensor([V - 1, V // 2, 0, V - 1], device="cuda")
    lse, loss = forward(h, W, t, "none")
    want = np.log(V - 2 + np.exp(64.0) + np.exp(-64.0))
    assert (np.abs(lse.double().cpu().numpy() - want) < 1e-3).all()
    assert (np.abs(loss.double().cpu().numpy() - np.array([0.0, 0.0, want, 0.0])) < 1e-3).all()
    dh, dW = backward(h, W, t, lse, None, "none")
    # token 2 alone has a gradient: p of row V - 1 is 1 and of row 0 is -1
    assert (dW[V - 1].float() == 1).all() and (dW[0].float() == -1).all() and float(dW[1:V - 1].float().abs().max()) < 1e-6
    assert (np.abs(dh[2].float().cpu().numpy() - 1.0 / 64) < 1e-4).all() and float(dh[[0, 1, 3]].float().abs().max()) < 1e-6


def test_captured_and_replayed_beside_another_stream():
    T, V, D = 50, 3000, 128
    h, W, t = [v.cuda() for v in inputs(T, V, D, "bf16")]
    lse, loss, dh, dW = torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(h), torch.empty_like(W)

    def step(*o):
        sp.linear_ce(h, W, t, o[0], o[1])
        sp.linear_ce_grad(h, W, t, o[0], None, o[2], o[3])

    step(lse, loss, dh, dW)
    graphs = []
    outs = [[torch.empty_like(v) for v in (lse, loss, dh, dW)] for _ in range(2)]
    for o in outs:                                              # two graphs, each with workspaces of its own
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(*o)
        graphs.append(gr)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for seed in range(3):
        h.copy_(torch.randn(T, D, generator=torch.Generator().manual_seed(seed)).bfloat16())
        for o in outs:
            for v in o:
                v.fill_(float("nan"))
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        step(lse, loss, dh, dW)
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(o, (lse, loss, dh, dW)))
    assert sp.get_status() == 0


def test_a_stream_that_is_not_the_current_one():
    h, W, t = [v.cuda() for v in inputs(300, 2000, 64, "fp16")]
    want = forward(h, W, t, "mean")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, int(side.cuda_stream)):
        for _ in range(5):                                      # workspaces from torch's allocator are held until the side stream is done
            lse, loss = torch.empty(300, device="cuda"), torch.empty(1, device="cuda")
            torch.cuda.synchronize()
            sp.linear_ce(h, W, t, lse, loss, stream=stream)
            junk = torch.full((1 << 20,), 7.0, device="cuda")   # would land in a workspace given back too early
            assert sp.get_status(stream) == 0
            assert torch.equal(lse, want[0]) and torch.equal(loss, want[1])
            del junk


def test_the_default_stream_by_its_handle_beside_another_current_one():
    h, W, t = [v.cuda() for v in inputs(100, 900, 64, "bf16")]
    want = forward(h, W, t, "sum")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        lse, loss = torch.empty(100, device="cuda"), torch.empty(1, device="cuda")
        torch.cuda.synchronize()
        sp.linear_ce(h, W, t, lse, loss, reduction="sum", stream=0)
        assert sp.get_status(0) == 0
    assert torch.equal(lse, want[0]) and torch.equal(loss, want[1])


def test_a_head_trained_on_an_8_bit_trunk():
    """The operators as they are used together: a frozen 8-bit layer, its output scored under a vocabulary, the head's gradient, one
    step down it, and the loss again, all on the library's kernels; every link against its oracle."""
    T, K, D, V = 70, 200, 136, 1001
    g = torch.Generator().manual_seed(8)
    x = torch.randn(T, K, generator=g).bfloat16()
    trunk = torch.randn(D, K, generator=g)
    wq, ws = torch.empty(D, 208, dtype=torch.int8, device="cuda"), torch.empty(D, device="cuda")
    sp.quantize_i8(trunk.cuda(), wq, ws)
    q, s, h = torch.empty(T, 208, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    sp.linear_i8(x.cuda(), q, s, wq, ws, h)
    rq, rs = LN.quantize_i8(x.double().numpy())
    rw, rws = LN.quantize_i8(trunk.double().numpy())
    want_h = torch.from_numpy(LN.gemm_i8(rq, rs, rw, rws)).bfloat16()
    assert torch.equal(h.cpu(), want_h)
    head, t = (torch.randn(V, D, generator=g) * 0.01).bfloat16(), torch.randint(0, V, (T,), generator=g)
    grad = torch.ones(1)
    ref, tol = bounds(want_h, head, t, grad, "mean", "bf16")
    lse, loss = forward(h, head.cuda(), t.cuda(), "mean")
    dh, dW = backward(h, head.cuda(), t.cuda(), lse, None, "mean")
    assert inside(loss, np.reshape(ref[0], -1), tol[0]) and inside(dh, ref[2], tol[2]) and inside(dW, ref[3], tol[3])
    stepped = (head.cuda().float() - 0.05 * dW.float()).bfloat16()
    again, tol2 = bounds(want_h, stepped.cpu(), t, grad, "mean", "bf16")
    _, loss2 = forward(h, stepped, t.cuda(), "mean")
    assert inside(loss2, np.reshape(again[0], -1), tol2[0])
