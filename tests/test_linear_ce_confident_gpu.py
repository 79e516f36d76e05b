"""The vocabulary cross entropy where a token is nearly certain of its word: 1 - p from 1e-1 down to 1e-7.  The loss is then about
1 - p and the gradient at the token's own word is p - 1, so both are held to errors relative to themselves, not to the scores.

Tolerances, from the arithmetic (u = 2^-23; e = eps / 2 of the 16-bit type).
  score     16 products at a time are added to an accumulator that may cut instead of rounding, 512 products at a time in fp32:
            dz = (D / 16 + D / 512 + 2) u sum_d |h_d W_vd|, the largest over v.
  2^x       of z log2 e - m: the argument is rounded up to three times on its way (product, part to row, row to lse), |argument| <=
            2 log2(e) max|z|, and the hardware's 2^x is good to 2^-22:  r = (6 log2(e) max|z| + 4) u, relative.
  loss      log(1 + sum_{v != y} e^(z_v - z_y)): relative error at most that of the sum, 2 dz + 2 r, and 2^-17 for the additions (as in
            test_linear_ce_gpu) and the logarithm.
  g         every p is off by q = 2 dz + 2 r + 2^-17 relative; lse is a 32-bit number, off by |lse| u / 2, which r covers.  A token's own
            entry is minus the sum of the others' p (relative q), or p - 1 where 1 - p is at least |lse| 2^-9, in which case it
            is off by |lse| u / (1 - p) <= 2^-13 relative.  Then half a step of the 16-bit type: e |g|.
  dh, dW    those errors summed, (V + 2) u and (T + 2) u of the absolute sums for the additions, and the result's own rounding."""

import numpy as np
import pytest

import paper_2508_20258_b200 as sp

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0 ** -23
LOG2E = 1.4426950408889634


def confident(T, V, D, dtype, seed=0, shift=24.0, sure=1.0):
    """Hidden states along their target's row of W, so long that 1 - p runs from 1e-1 to 1e-7 (the first ``sure`` of the tokens; the
    others are random), and `shift` added to every score."""
    g = torch.Generator(device="cuda").manual_seed(seed * 1000 + T + V + D)
    W = torch.randn(V, D, device="cuda", generator=g) / D ** 0.5
    W[:, 0] = 1.0
    W = W.to(BITS[dtype])
    t = torch.randint(0, V, (T,), device="cuda", generator=g)
    far = torch.linspace(0.5, 17.0, T, device="cuda")[torch.randperm(T, device="cuda", generator=g)] if T > 1 else torch.full((1,), 9.0, device="cuda")
    goal = np.log(V) + far
    a = D - (D * D - 2 * D * goal).clamp_min(0).sqrt()       # a - a^2 / (2 D) = log V + far: the others' scores have deviation a / sqrt D
    h = a[:, None] * W[t].float()
    n = int(round(T * sure))
    if n < T:
        h[n:] = torch.randn(T - n, D, device="cuda", generator=g) * 2
    h[:, 0] = shift
    h = h.to(BITS[dtype])
    if T > 3:
        t[3::7] = -100
    return h, W, t


def reference(h, W, t, c):
    """Loss, lse, 1 - p, p, g and gradients in float64, the sum of the others taken as such."""
    hd, Wd = h.double(), W.double()
    z = hd @ Wd.t()
    kept = t != -100
    at = torch.where(kept, t, 0)[:, None]
    zy = z.gather(1, at)
    others = (z - zy).exp().scatter(1, at, 0.0).sum(1)       # over p of the target
    loss = torch.where(kept, torch.log1p(others), 0.0)
    lse = torch.logsumexp(z, 1)
    rest = others / (1 + others)
    g = (z - lse[:, None]).exp().scatter(1, at, 0.0)
    g = g.scatter(1, at, -rest[:, None]) * torch.where(kept, c, 0.0)[:, None]
    size = (hd.abs() @ Wd.abs().t()).amax(1)
    zmax = z.abs().amax(1)
    return loss, lse, rest, g, size, zmax, kept


def slack(size, zmax, D):
    return 2 * (D / 16 + D / 512 + 2) * U * size + 2 * (6 * LOG2E * zmax + 4) * U + 2.0 ** -17


@pytest.mark.parametrize("T,V,D", [(1, 1001, 256), (1, 999, 16392), (4, 3001, 256), (60, 1001, 512), (128, 40001, 256), (300, 1001, 256), (700, 9001, 1032)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_small_losses_keep_their_digits(T, V, D, dtype):
    h, W, t = confident(T, V, D, dtype)
    lse, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    sp.linear_ce(h, W, t, lse, loss, reduction="none")
    want, want_lse, rest, _, size, zmax, kept = reference(h, W, t, torch.ones(T, device="cuda"))
    if T > 50:
        assert float(rest[kept].min()) < 1e-6 and float(rest[kept].max()) > 1e-2
    assert (loss >= 0).all()
    assert ((loss.double() - want).abs() <= slack(size, zmax, D) * want).all()
    assert ((lse.double() - want_lse).abs() <= slack(size, zmax, D) + want_lse.abs() * U).all()


def near(got, want, tol):
    """Within the tolerance, or infinite where the type ends within it (a scaled-up gradient may leave fp16's range)."""
    over = (want.abs() + tol > torch.finfo(got.dtype).max) & torch.isinf(got) & (got.sign() == want.sign())
    return bool((((got.double() - want).abs() <= tol) | over).all())


def check_gradients(h, W, t, reduction, dtype, up):
    T, D = h.shape
    V = W.shape[0]
    e = float(torch.finfo(BITS[dtype]).eps) / 2
    tiny = 2.0 ** -25 if dtype == "fp16" else 0.0
    lse, loss = torch.empty(T, device="cuda"), torch.empty(T if reduction == "none" else 1, device="cuda")
    sp.linear_ce(h, W, t, lse, loss, reduction=reduction)
    gen = torch.Generator(device="cuda").manual_seed(1)
    grad = (torch.rand(T if reduction == "none" else 1, device="cuda", generator=gen) + 0.5) * up
    dh, dW = torch.full_like(h, float("nan")), torch.full_like(W, float("nan"))
    sp.linear_ce_grad(h, W, t, lse, grad, dh, dW, reduction=reduction)
    assert sp.get_status() == 0
    kept = t != -100
    c = grad.double().expand(T) / (kept.sum() if reduction == "mean" else 1)
    hd, Wd = h.double(), W.double()
    rW, sW = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for i in range(0, T, 512):
        part = slice(i, i + 512)
        _, _, rest, g, size, zmax, _ = reference(h[part], W, t[part], c[part])
        dg = (e + slack(size, zmax, D) + 2.0 ** -13)[:, None] * g.abs() + torch.where(kept[part], c.max() * tiny / 2.0 ** 14, 0.0)[:, None]
        rh, sh = g @ Wd, dg @ Wd.abs() + (V + 2) * U * (g.abs() @ Wd.abs())
        assert near(dh[part], rh, sh + (e + 2 * U) * rh.abs() + tiny)
        rW += g.t() @ hd[part]
        sW += dg.t() @ hd[part].abs() + (T + 2) * U * (g.abs().t() @ hd[part].abs())
        assert (dh[part][~kept[part]] == 0).all()
    assert near(dW, rW, sW + (e + 2 * U) * rW.abs() + tiny)


@pytest.mark.parametrize("T,V,D", [(1, 1001, 256), (2, 2, 64), (4, 3001, 256), (60, 1001, 512), (128, 40001, 256), (300, 1001, 256), (700, 9001, 1032)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("reduction", ["none", "mean", "sum"])
def test_gradients_of_confident_tokens(T, V, D, dtype, reduction):
    h, W, t = confident(T, V, D, dtype)
    check_gradients(h, W, t, reduction, dtype, (4096.0 if dtype == "fp16" else 1.0) * (T if reduction == "mean" else 1))


# the vocabulary in pieces (more than 128 Mi entries of g): all tokens sure, some, one, none
@pytest.mark.parametrize("T,V,D,dtype,sure", [(2048, 70001, 256, "bf16", 1.0), (2048, 70001, 256, "fp16", 0.3), (3000, 50000, 264, "bf16", 1 / 3000), (3000, 50000, 264, "fp16", 0.0),
                                              (130, 1100000, 256, "bf16", 0.5), (100, 1400001, 256, "fp16", 0.5)])
def test_gradients_of_confident_tokens_in_pieces(T, V, D, dtype, sure):
    h, W, t = confident(T, V, D, dtype, sure=sure)
    check_gradients(h, W, t, "none", dtype, 4096.0 if dtype == "fp16" else 1.0)


@pytest.mark.parametrize("T", [2, 300])
def test_scores_made_again_are_those_of_the_forward(T):
    # All scores are one large sum of equal products, so all p are 1 / V.  An accumulator that cuts off every addition of such a sum (2048 of them) leaves
    # the score 0.03 too small, and every p with it.  Sums of 512 lose at most 32 x 2^-23 x 247 in their own additions and 64 x 2^-24 x 247 in
    # those of the sums: 1.9e-3.
    V, D = 64, 32768
    # 11-bit factors: products of 22 bits, whose sums need rounding from the first hundred on
    h, W = torch.full((T, D), 4 / 3, dtype=torch.float16, device="cuda"), torch.full((V, D), 150 / D * 1.2346, dtype=torch.float16, device="cuda")
    t = torch.zeros(T, dtype=torch.int64, device="cuda")
    lse, loss, dh, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(h), torch.empty_like(W)
    sp.linear_ce(h, W, t, lse, loss, reduction="none")
    sp.linear_ce_grad(h, W, t, lse, None, dh, dW, reduction="none")
    # p: 3.8e-3 (scores made twice), g's rounding and the result's: 2^-11 each
    assert ((dW[1:].double() * V / T / h[0].double() - 1).abs() <= 3.8e-3 + 2 * 2.0 ** -11 + 2.0 ** -16).all()


def test_sums_over_many_tokens_and_many_words_are_not_cut_off():
    # Sums of 65536 positive terms.  What is common to all entries is what the additions cut off: 32 x 2^-23 in a sum of 512, against 4e-4 if
    # one accumulator took them all; g is off by lse's 32 bits (|lse| <= 12: 12 x 2^-24 and as much again on its way) and 2^x (2^-22).  The roundings to 16 bits
    # are the results' own: `off` compares with the rounded reference, mean with mean.  An entry next to a border then
    # moves by a whole step, but as many as the common error would move on average, so twice that error bounds the mean; the chance part
    # (g's own roundings, 2^-11 / sqrt(3 x 65536) per entry) moves n entries' mean by at most 5 times that / sqrt n.
    g = torch.Generator(device="cuda").manual_seed(0)
    T, V, D = 65536, 64, 64
    h, W = (torch.rand(T, D, device="cuda", generator=g) + 0.5).half(), (torch.randn(V, D, device="cuda", generator=g) * 0.01).half()
    t = torch.randint(0, 8, (T,), device="cuda", generator=g)
    lse, loss, up = torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.full((1,), 1024.0, device="cuda")
    dh, dW = torch.empty_like(h), torch.empty_like(W)
    sp.linear_ce(h, W, t, lse, loss)
    sp.linear_ce_grad(h, W, t, lse, up, dh, dW)
    p = (h.double() @ W.double().t()).softmax(1)[:, 8:]                 # words that are nobody's target
    want = p.t() @ h.double() * 1024 / T
    off, common = (dW[8:].double() - want.half().double()) / want, 32 * U + 12 * U + 2 * U
    assert abs(float(off.mean())) <= 2 * common + 5 * 2.0 ** -11 / (3 * T * off.numel()) ** 0.5 * 2
    T, V, D = 2048, 65536, 2560                                         # tiles of dh for every SM: no slices of the vocabulary
    h, W = (torch.randn(T, D, device="cuda", generator=g) * 0.1).half(), (torch.rand(V, D, device="cuda", generator=g) * 0.01 + 0.005).half()
    W[:8] = 0
    t = torch.randint(0, 8, (T,), device="cuda", generator=g)
    lse, dh = torch.empty(T, device="cuda"), torch.empty_like(h)
    sp.linear_ce(h, W, t, lse, loss, reduction="sum")
    sp.linear_ce_grad(h, W, t, lse, up, dh, None, reduction="sum")
    z = h.double() @ W.double().t()
    want = z.softmax(1) @ W.double() * 1024
    off = (dh.double() - want.half().double()) / want
    assert abs(float(off.mean())) <= 2 * common + 5 * 2.0 ** -11 / (3 * V * off.numel()) ** 0.5 * 2


# dh in slices of the vocabulary, in whole tiles, in pieces
@pytest.mark.parametrize("T,V,D", [(4, 700, 64), (300, 700, 72), (2560, 600, 2048), (2048, 70001, 64)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_rows_of_dh_of_ignored_tokens_are_zero_whatever_w_holds(T, V, D, value):
    g = torch.Generator(device="cuda").manual_seed(T)
    h, W = torch.randn(T, D, device="cuda", generator=g).bfloat16(), torch.randn(V, D, device="cuda", generator=g).bfloat16()
    t = torch.randint(0, V, (T,), device="cuda", generator=g)
    t[1::3] = -100
    W[5, 1] = value
    lse, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    dh, dW = torch.full_like(h, 7.0), torch.empty_like(W)
    sp.linear_ce(h, W, t, lse, loss, reduction="none")
    sp.linear_ce_grad(h, W, t, lse, None, dh, dW, reduction="none")
    assert sp.get_status() == 0
    assert (dh[t == -100] == 0).all() and torch.isnan(dh[t != -100]).any()


def test_a_workspace_on_another_stream_is_not_memory_still_in_use():
    # what the current stream has given back but is still writing must not become the workspace of a call on another stream
    T, V, D = 700, 9000, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    h, W = torch.randn(T, D, device="cuda", generator=g).bfloat16(), torch.randn(V, D, device="cuda", generator=g).bfloat16()
    t = torch.randint(0, V, (T,), device="cuda", generator=g)
    want = [torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(h), torch.empty_like(W)]
    sp.linear_ce(h, W, t, want[0], want[1])
    sp.linear_ce_grad(h, W, t, want[0], None, want[2], want[3])
    big = torch.randn(8192, 8192, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, int(side.cuda_stream)):
        got = [torch.full_like(v, 3.0) for v in want]
        torch.cuda.synchronize()
        used = [torch.empty(sp.linear_ce_workspace(T, V, D, grad), dtype=torch.uint8, device="cuda") for grad in (False, True)]
        for _ in range(10):
            big @ big                                           # some milliseconds
        for u in used:
            u.fill_(255)
        del used, u
        sp.linear_ce(h, W, t, got[0], got[1], stream=stream)
        sp.linear_ce_grad(h, W, t, got[0], None, got[2], got[3], stream=stream)
        torch.cuda.synchronize()
        assert sp.get_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(want, got))


# Many pieces of the vocabulary, few rows and many slices, both; the sizes of test_linear_ce_gpu's test of pieces, whose bound is so wide at a D of 1000
# that it holds without the softmax's part of dh.  Sums: V / 16 + V / 512 additions, fewer than V / 8.
@pytest.mark.parametrize("T,V,D,dtype", [(600, 45001, 1000, "bf16"), (600, 45001, 1000, "fp16"), (40000, 120001, 16, "bf16"), (3, 300001, 64, "fp16"),
                                         (16384, 50000, 264, "bf16"), (2048, 200000, 16, "fp16")])
def test_every_part_of_the_sums_in_pieces_and_slices_is_there(T, V, D, dtype):
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn(T, D, device="cuda", generator=gen).to(BITS[dtype])
    W = (torch.randn(V, D, device="cuda", generator=gen) * (2 / D ** 0.5)).to(BITS[dtype])
    t = torch.randint(0, V, (T,), device="cuda", generator=gen)
    t[T // 2] = -100
    c = torch.rand(T, device="cuda", generator=gen) + 0.5
    e, tiny = float(torch.finfo(BITS[dtype]).eps) / 2, 2.0 ** -25 if dtype == "fp16" else 0.0
    lse, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    sp.linear_ce(h, W, t, lse, loss, reduction="none")
    dh, dW = torch.full_like(h, float("nan")), torch.full_like(W, float("nan"))
    sp.linear_ce_grad(h, W, t, lse, c, dh, dW, reduction="none")
    assert sp.get_status() == 0
    kept, Wd, cut = t != -100, W.double(), V - V // 8
    rW, sW, own = (torch.zeros(V, D, dtype=torch.float64, device="cuda") for _ in range(3))
    seen = [0, 0]
    for i in range(0, T, 512):
        part = slice(i, i + 512)
        hd, kp = h[part].double(), kept[part]
        want, want_lse, rest, g, size, zmax, _ = reference(h[part], W, t[part], c[part].double())
        q = slack(size, zmax, D)
        assert ((loss[part].double() - want).abs() <= q * (1 - (-want).exp()) + 2 * U * want).all() and ((lse[part].double() - want_lse).abs() <= q + want_lse.abs() * U).all()
        dg = (e + q + 2.0 ** -13)[:, None] * g.abs() + torch.where(kp, c.max() * tiny / 2.0 ** 14, 0.0)[:, None]
        rh = g @ Wd
        tol = dg @ Wd.abs() + (V + 2) * U / 8 * (g.abs() @ Wd.abs()) + (e + 2 * U) * rh.abs() + tiny
        assert near(dh[part], rh, tol)
        at = torch.where(kp, t[part], 0)[:, None]
        mine = g.gather(1, at)                                  # the own words' entries
        p = g.scatter(1, at, 0.0)
        # the bound sees a dh without the softmax's part, and one without the last eighth of it
        for k, gone in enumerate((p @ Wd, p[:, cut:] @ Wd[cut:])):
            seen[k] += int(((gone.abs() > 2 * tol).any(1) & kp).sum())
        rW += g.t() @ hd
        sW += dg.t() @ hd.abs() + (T + 2) * U / 8 * (g.abs().t() @ hd.abs())
        own.index_add_(0, at[:, 0], mine * hd * kp[:, None])
    assert near(dW, rW, sW + (e + 2 * U) * rW.abs() + tiny)
    assert seen[0] > 0.9 * T - 1 and seen[1] > 0.5 * T - 1
    assert float(((rW - own).abs() > 2 * (sW + (e + 2 * U) * rW.abs() + tiny)).double().mean()) > 0.1


def test_many_more_tokens_than_a_piece_holds_words():
    h, W, t = confident(300000, 1500, 64, "bf16", shift=0.0, sure=0.0)      # pieces of 1024 words
    t[7::11] = -100
    h[::5] = 8 * W[t[::5].clamp_min(0)]                                      # some sure, not all to the same degree
    check_gradients(h, W, t, "none", "bf16", 1.0)


@pytest.mark.parametrize("T,V,D", [(60, 1001, 512), (2048, 70001, 256)])
def test_captured_once_and_replayed_on_tokens_as_sure_as_they_come(T, V, D):
    h, W, t = confident(T, V, D, "bf16", sure=0.0)
    lse, loss, dh, dW = torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(h), torch.empty_like(W)
    grad = torch.full((1,), -0.75, device="cuda")
    spaces = [torch.empty(16 + sp.linear_ce_workspace(T, V, D, g), dtype=torch.uint8, device="cuda")[16:] for g in (False, True)]      # 16-byte aligned, no more

    def step(lse, loss, dh, dW):
        sp.linear_ce(h, W, t, lse, loss, workspace=spaces[0])
        sp.linear_ce_grad(h, W, t, lse, grad, dh, dW, workspace=spaces[1])

    step(lse, loss, dh, dW)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(lse, loss, dh, dW)
    for seed, sure in enumerate((0.5, 1.0, 0.0, 0.02)):
        h2, W2, t2 = confident(T, V, D, "bf16", seed=seed + 5, sure=sure)
        h.copy_(h2), W.copy_(W2), t.copy_(t2)
        for v in (lse, loss, dh, dW):
            v.fill_(float("nan"))
        for s in spaces:
            s.fill_(255)
        graph.replay()
        got = [v.clone() for v in (lse, loss, dh, dW)]
        step(lse, loss, dh, dW)
        assert sp.get_status() == 0
        assert all(torch.equal(a, b) for a, b in zip(got, (lse, loss, dh, dW)))
        kept = t != -100
        c = torch.full((T,), -0.75, dtype=torch.float64, device="cuda") / kept.sum()
        _, _, _, g, size, zmax, _ = reference(h, W, t, c)
        e = 2.0 ** -8
        dg = (e + slack(size, zmax, D) + 2.0 ** -13)[:, None] * g.abs()
        rh = g @ W.double()
        assert near(dh, rh, dg @ W.double().abs() + (V + 2) * U * (g.abs() @ W.double().abs()) + (e + 2 * U) * rh.abs())


@pytest.mark.parametrize("T", [1, 5, 300])
def test_a_vocabulary_of_one_word_leaves_nothing_to_learn(T):
    h, W, t = torch.randn(T, 64, device="cuda").bfloat16() * 4, torch.randn(1, 64, device="cuda").bfloat16(), torch.zeros(T, dtype=torch.int64, device="cuda")
    lse, loss, dh, dW = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(h), torch.empty_like(W)
    sp.linear_ce(h, W, t, lse, loss, reduction="none")
    sp.linear_ce_grad(h, W, t, lse, None, dh, dW, reduction="none")
    assert (loss == 0).all() and (dh == 0).all() and (dW == 0).all()
