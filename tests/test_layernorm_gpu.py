"""Layer norm and its gradients against the oracle (float64 of the formulas).

Tolerances, from the arithmetic.  u = 2^-24 bounds one fp32 rounding, relative to its value.  A sum over a row passes through at most 16 additions in a
thread, 5 of lanes, 8 of warps and 8 of blocks: 37, so it is off by at most 40 u times the sum of its terms' sizes (the terms' own roundings included).
  mean   the rounded mean (off by 40 u mean |x|) is corrected by the mean of the differences to it, itself off by 40 u mean |x - mean|, and rounded:
         40 u mean |x - mean| + 2 u |mean|, and a second-order term, 40 u of 40 u mean |x|.
  rstd   the mean of squares is off by 42 u relative, its root's inverse by half of that, and 4 u for the root: 26 u.
  y      (x - mean) rstd gamma + beta: the mean's error, rstd's, and a rounding for each step: u (40 mean |xh| + 32 |xh|) |gamma| + 2 u |beta|, then the output's
         rounding, half a step: eps / 2 relative (fp16: or 2^-25 below its normal range).
  dx     xh is off by 2 u, u_n = dy gamma by u, their sums by 44 u of their sizes: rstd u (4 |u_n| + 48 mean |u| + 56 |xh| mean |u xh|), then the rounding.
  dgamma, dbeta   at most M / 37 rows in one chain (a group of warps; at least 37 of them share the rows), 8 groups, 19 blocks, 16 chains of these:
         u (M / 37 + 64) times the sum of the terms' sizes, then the rounding."""

import numpy as np
import pytest

import paper_2508_20258_b200 as sp
from oracle import layernorm as LN

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BITS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = 2.0 ** -24


def half_step(value, dtype):
    low = {"bf16": 0.0, "fp16": 2.0 ** -25, "fp32": 0.0}[dtype]
    return np.abs(value) * (torch.finfo(BITS[dtype]).eps / 2) * (1 + 1e-6) + low


def within(got, want, tol, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: values that are not finite"
    worst = np.max(np.abs(got - want) / (tol + 1e-300))
    assert worst <= 1, f"{what}: {worst:.3g} of the tolerance"


class Case:
    """Inputs `off` elements behind an allocation (or, unless `alike`, a multiple of them), outputs between guards."""

    def __init__(self, M, N, x="bf16", w="bf16", off=0, scale=1.0, shift=0.3, seed=0, weights=True, alike=False):
        g = torch.Generator().manual_seed(seed * 100003 + M * 7 + N)
        self.M, self.N, self.xt, self.wt = M, N, x, w
        self.guards = []
        self.x = self.place(torch.randn(M, N, generator=g) * scale + shift, x, off)
        self.dy = self.place(torch.randn(M, N, generator=g), x, off * (1 if alike else 3))
        self.gamma = self.place(1 + 0.3 * torch.randn(N, generator=g), w, off) if weights else None
        self.beta = self.place(torch.randn(N, generator=g), w, off) if weights else None
        nan = float("nan")
        self.y = self.place(torch.full((M, N), nan), x, off * (1 if alike else 2), guard=True)
        self.dx = self.place(torch.full((M, N), nan), x, off, guard=True)
        self.dgamma, self.dbeta = (self.place(torch.full((N,), nan), w, off, guard=True) for _ in range(2))
        self.mean, self.rstd = (self.place(torch.full((M,), nan), "fp32", off, guard=True) for _ in range(2))

    def place(self, values, dtype, off, guard=False):
        n = values.numel()
        whole = torch.full((n + off + 24,), 7.0, dtype=BITS[dtype], device="cuda")
        view = whole[off:off + n].view(values.shape)
        view.copy_(values)
        if guard:
            self.guards.append((whole, off, n))
        return view

    def check_guards(self):
        for whole, off, n in self.guards:
            assert (whole[:off] == 7).all() and (whole[off + n:] == 7).all(), "written outside an output"

    def forward(self, eps=1e-5, **kw):
        sp.layernorm(self.x, self.gamma, self.beta, self.y, self.mean, self.rstd, eps=eps, **kw)

    def backward(self, **kw):
        sp.layernorm_grad(self.dy, self.x, self.gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, **kw)

    def host(self, t):
        return None if t is None else t.double().cpu().numpy()

    def check_forward(self, eps=1e-5):
        x, gamma, beta = self.host(self.x), self.host(self.gamma), self.host(self.beta)
        y, mean, rstd = LN.layernorm(x, gamma, beta, eps)
        spread = np.abs(x - mean[:, None]).mean(axis=1)
        within(self.mean, mean, U * (40 * spread + 2 * np.abs(mean) + 1600 * U * np.abs(x).mean(axis=1)), "mean")
        within(self.rstd, rstd, 26 * U * rstd, "rstd")
        xh = np.abs(x - mean[:, None]) * rstd[:, None]
        gm, bt = (1.0 if v is None else np.abs(v) for v in (gamma, beta))
        own = U * (40 * xh.mean(axis=1, keepdims=True) + 32 * xh + 1600 * U * (np.abs(x).mean(axis=1) * rstd)[:, None]) * gm + 2 * U * bt
        within(self.y, y, own + half_step(np.abs(y) + own, self.xt), "y")

    def check_backward(self):
        dx, dgamma, dbeta, xh, u = LN.layernorm_grad(self.host(self.dy), self.host(self.x), self.host(self.gamma), self.host(self.mean), self.host(self.rstd))
        rstd = self.host(self.rstd)[:, None]
        xa, ua = np.abs(xh), np.abs(u)
        own = rstd * U * (4 * ua + 48 * ua.mean(axis=1, keepdims=True) + 56 * xa * (ua * xa).mean(axis=1, keepdims=True))
        within(self.dx, dx, own + half_step(np.abs(dx) + own, self.xt), "dx")
        dy = np.abs(self.host(self.dy))
        chain = U * (self.M / 37 + 64)
        for got, want, size, name in ((self.dgamma, dgamma, (dy * xa).sum(axis=0), "dgamma"), (self.dbeta, dbeta, dy.sum(axis=0), "dbeta")):
            within(got, want, chain * size + half_step(np.abs(want) + chain * size, self.wt), name)


# widths at the edges of a lane's, a warp's, a group's, a block's and a cluster's share
WIDTHS = [1, 2, 7, 8, 9, 31, 64, 255, 304, 511, 512, 513, 520, 1024, 1031, 1040, 2035, 2048, 2056, 4095, 4096, 4097, 4104, 5001, 8192, 8200, 12345, 16384, 20001, 32767, 32768]


@pytest.mark.parametrize("N", WIDTHS)
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")], ids="-".join)
def test_widths(N, types):
    for M in (1, 13):
        c = Case(M, N, *types)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()
        c.check_guards()


@pytest.mark.parametrize("alike", [False, True])
@pytest.mark.parametrize("off", [1, 3, 4, 7, 8])
@pytest.mark.parametrize("M,N", [(1, 5), (300, 3), (9, 1031), (5, 1032), (3, 4095), (3, 4104), (2, 9001), (3, 17001), (40, 96)])
@pytest.mark.parametrize("types", [("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")], ids="-".join)
def test_any_address(M, N, types, off, alike):
    c = Case(M, N, *types, off=off, alike=alike)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.check_guards()


@pytest.mark.parametrize("M,N", [(2, 4096), (4095, 64), (700, 1031), (1500, 2048), (900, 5000), (20011, 40), (3000, 512), (1300, 4104), (700, 12288), (800, 9001), (400, 20008)])
def test_many_rows(M, N):
    c = Case(M, N, "bf16", "fp32")
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.check_guards()


@pytest.mark.parametrize("M,N", [(300, 10008), (310, 12291), (300, 16384), (160, 24583), (170, 32768)])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")], ids="-".join)
def test_many_wide_rows(M, N, types):
    c = Case(M, N, *types)
    c.forward()
    c.backward()
    c.check_backward()
    c.check_guards()
    first = [t.clone() for t in (c.dx, c.dgamma, c.dbeta)]
    c.backward()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.dx, c.dgamma, c.dbeta)))


@pytest.mark.parametrize("N", [300, 4096, 9001])
def test_rows_far_from_zero_and_of_small_and_large_scale(N):
    for scale, shift in ((1.0, 1000.0), (1e-3, 0.0), (1e15, 0.0), (1.0, -30000.0)):
        c = Case(6, N, "fp32", "fp32", scale=scale, shift=shift)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


def test_equal_values_give_beta_and_without_eps_nan():
    c = Case(4, 520, "fp32", "fp32")
    c.x.fill_(3.7)
    c.forward()
    c.check_forward()
    assert torch.equal(c.y, c.beta.expand(4, -1))
    c.forward(eps=0.0)
    assert torch.isnan(c.y).all() and torch.isinf(c.rstd).all()


def test_eps_is_the_callers():
    c = Case(5, 130, "fp32", "fp32", scale=0.1)
    for eps in (0.0, 1e-12, 0.5):
        c.forward(eps=eps)
        c.check_forward(eps)


@pytest.mark.parametrize("N", [96, 4095, 8192])
def test_without_weights_and_statistics(N):
    c = Case(9, N, "bf16", "bf16", weights=False)
    c.forward()
    c.check_forward()
    y = c.y.clone()
    c.backward()
    c.check_backward()
    c.y.fill_(0)
    sp.layernorm(c.x, None, None, c.y)
    assert torch.equal(c.y, y)
    ones, zeros = torch.ones(N, device="cuda"), torch.zeros(N, device="cuda")
    c.y.fill_(0)
    sp.layernorm(c.x, ones, zeros, c.y)
    assert torch.equal(c.y, y)


@pytest.mark.parametrize("N", [304, 1031, 8192])
def test_each_gradient_alone_has_the_same_bits(N):
    c = Case(77, N, "fp16", "fp32")
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.dx, c.dgamma, c.dbeta)]
    for only in range(3):
        for both in (False, True):
            outs = [t if (i == only) != both else None for i, t in enumerate((c.dx, c.dgamma, c.dbeta))]
            for t in outs:
                if t is not None:
                    t.fill_(float("nan"))
            sp.layernorm_grad(c.dy, c.x, c.gamma, c.mean, c.rstd, *outs)
            for t, w in zip(outs, want):
                assert t is None or torch.equal(t, w)
    c.check_guards()


@pytest.mark.parametrize("N", [64, 1031, 4096, 8200])
def test_a_row_that_is_not_finite_stays_alone(N):
    c = Case(40, N, "fp32", "fp32")
    c.forward()
    c.backward()
    y, dx = c.y.clone(), c.dx.clone()
    c.x[3, N // 2], c.x[17, 0], c.x[39, N - 1] = float("inf"), float("nan"), float("-inf")
    c.forward()
    c.backward()
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 17, 39]] = True
    assert torch.isnan(c.y[bad]).all() and torch.isnan(c.dx[bad]).all() and torch.isnan(c.rstd[bad]).all()
    assert torch.equal(c.y[~bad], y[~bad]) and torch.equal(c.dx[~bad], dx[~bad])
    assert torch.isnan(c.dgamma).all() and torch.isfinite(c.dbeta).all()


@pytest.mark.parametrize("M,N", [(333, 1024), (200, 1031), (64, 8200)])
def test_same_bits_every_time_captured_replayed_and_on_another_stream(M, N):
    c = Case(M, N, "bf16", "fp32")
    outs = (c.y, c.mean, c.rstd, c.dx, c.dgamma, c.dbeta)
    c.forward()
    c.backward()
    want = [t.clone() for t in outs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c.forward(stream=side)
    c.backward(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(outs, want))
    ws = torch.empty(sp.layernorm_workspace(M, N), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward(workspace=ws)
    x = c.x.clone()
    for k in range(3):
        c.x.copy_(torch.randn_like(x))      # other values between the replays
        graph.replay()
        c.x.copy_(x)
        for t in outs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outs, want)), k
    c.check_guards()


def test_offsets_beyond_32_bits():
    M, N = 70001, 32768      # 2.3e9 elements: the last rows are beyond 2^32 bytes
    x = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 5000):
        x[i:i + 5000].normal_()
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    sp.layernorm(x, None, None, y, mean, rstd)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    sp.layernorm_grad(y, x, None, mean, rstd, dx, dgamma, dbeta)
    for rows in (slice(0, 3), slice(65534, 65540), slice(M - 3, M)):
        c = Case(x[rows].shape[0], N, weights=False)
        c.x.copy_(x[rows])
        c.dy.copy_(y[rows])
        c.forward()
        c.backward()
        assert torch.equal(c.y, y[rows]) and torch.equal(c.mean, mean[rows]) and torch.equal(c.dx, dx[rows])
        c.check_forward()
        c.check_backward()


def test_refusals_of_the_binding():
    c = Case(4, 64)
    with pytest.raises(ValueError, match="contiguous"):
        sp.layernorm(c.x.t().contiguous().t(), c.gamma, c.beta, c.y)
    with pytest.raises(sp.SpError) as e:
        sp.layernorm(c.x, c.gamma, c.beta, c.x)
    assert e.value.status == sp.ERR_INVALID_ARG
    with pytest.raises(sp.SpError) as e:
        sp.layernorm_grad(c.dy, c.x, c.gamma, c.mean, c.rstd, c.dx, c.dgamma, c.dbeta, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == sp.ERR_INVALID_ARG
    with pytest.raises(sp.SpError) as e:
        sp.layernorm(torch.empty(1, sp.LAYERNORM_MAX_N + 8, device="cuda"), None, None, torch.empty(1, sp.LAYERNORM_MAX_N + 8, device="cuda"))
    assert e.value.status == sp.ERR_UNSUPPORTED
    assert sp.get_status() == 0


# rows whose places in shared memory are used several times: 148, 74, 33 groups share them
@pytest.mark.parametrize("M,N", [(1200, 40), (700, 1031), (400, 17001)])
@pytest.mark.parametrize("types", [("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")], ids="-".join)
def test_many_rows_at_unequal_addresses(M, N, types):
    c = Case(M, N, *types, off=1)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.check_guards()


@pytest.mark.parametrize("M,N", [(600, 16384), (400, 17001), (400, 24583), (310, 32768)])
@pytest.mark.parametrize("types", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")], ids="-".join)
def test_many_wide_rows_forward(M, N, types):
    c = Case(M, N, *types)
    c.forward()
    c.check_forward()
    c.check_guards()


@pytest.mark.parametrize("M,N", [(400, 9001), (400, 16384), (400, 20001), (150, 32768)])
@pytest.mark.parametrize("types", [("fp16", "fp32"), ("fp32", "fp32")], ids="-".join)
def test_each_gradient_of_wide_rows_alone_has_the_same_bits(M, N, types):
    c = Case(M, N, *types)
    c.forward()
    c.backward()
    c.check_backward()
    want = [t.clone() for t in (c.dx, c.dgamma, c.dbeta)]
    for only in range(3):
        for both in (False, True):
            outs = [t if (i == only) != both else None for i, t in enumerate((c.dx, c.dgamma, c.dbeta))]
            for t in outs:
                if t is not None:
                    t.fill_(float("nan"))
            sp.layernorm_grad(c.dy, c.x, c.gamma, c.mean, c.rstd, *outs)
            for t, w in zip(outs, want):
                assert t is None or torch.equal(t, w)
    c.check_guards()


@pytest.mark.parametrize("N", [64, 1031, 20001])
def test_squares_beyond_fp32_leave_beta(N):
    c = Case(3, N, "fp32", "fp32", scale=1e20, shift=0.0)      # some of them beyond 1.9e19, whose square is beyond 3.4e38
    c.forward()
    assert (c.rstd == 0).all() and torch.equal(c.y, c.beta.expand(3, -1))
    c.check_guards()
