"""Layer norm without a GPU: pins of its oracle, refusals on the host, workspace sizes, argument checks of the binding."""

import numpy as np
import pytest

import paper_2508_20258_b200 as sp
from oracle import layernorm as LN

# never dereferenced: every check below fails on the host first
A, B, C, D, E, F, G, H, I = (0x1000000 * (i + 1) for i in range(9))


def test_oracle_on_values_worked_by_hand():
    y, mean, rstd = LN.layernorm([[1.0, 3.0], [5.0, 5.0]], gamma=[2.0, 10.0], beta=[0.5, -1.0], eps=3.0)
    assert mean.tolist() == [2.0, 5.0] and rstd.tolist() == [0.5, 1 / np.sqrt(3.0)]
    assert y.tolist() == [[-0.5, 4.0], [0.5, -1.0]]


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, gamma, beta, dy = rng.standard_normal((4, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((4, 7))
    _, mean, rstd = LN.layernorm(x, gamma, beta)
    dx, dgamma, dbeta, *_ = LN.layernorm_grad(dy, x, gamma, mean, rstd)
    f = lambda x_, g_, b_: float((LN.layernorm(x_, g_, b_)[0] * dy).sum())  # noqa: E731
    for k, (v, d) in enumerate(((x, dx), (gamma, dgamma), (beta, dbeta))):
        for i in np.ndindex(v.shape):
            e = np.zeros_like(v)
            e[i] = 1e-5
            args = [[x, gamma, beta], [x, gamma, beta]]
            args[0][k], args[1][k] = v + e, v - e
            assert abs((f(*args[0]) - f(*args[1])) / 2e-5 - d[i]) < 1e-8


def _fwd(x=A, gamma=B, beta=C, y=D, mean=E, rstd=F, M=8, N=64, dtype=sp.BF16, w=sp.BF16, eps=1e-5):
    return sp.lib().sp_layernorm(x, gamma, beta, y, mean, rstd, M, N, dtype, w, eps, None)


def _grad(dy=A, x=B, gamma=C, mean=D, rstd=E, dx=F, dgamma=G, dbeta=H, M=8, N=64, dtype=sp.BF16, w=sp.BF16, ws=I, n=1 << 40):
    return sp.lib().sp_layernorm_grad(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, M, N, dtype, w, ws, n, None)


def _refused_alike(f):
    for name in ("M", "N"):
        assert f(**{name: 0}) == sp.ERR_INVALID_ARG and f(**{name: -3}) == sp.ERR_INVALID_ARG
    assert f(M=1 << 31) == sp.ERR_UNSUPPORTED and f(N=sp.LAYERNORM_MAX_N + 1) == sp.ERR_UNSUPPORTED
    assert f(dtype=3) == sp.ERR_UNSUPPORTED and f(w=sp.FP16) == sp.ERR_UNSUPPORTED and f(dtype=sp.FP32, w=sp.BF16) == sp.ERR_UNSUPPORTED


def test_refusals_of_the_forward_pass():
    _refused_alike(_fwd)
    for name in ("x", "y"):
        assert _fwd(**{name: None}) == sp.ERR_INVALID_ARG
    for name in ("x", "gamma", "beta", "y"):
        assert _fwd(**{name: A * 10 + 1}) == sp.ERR_ALIGNMENT
    assert _fwd(mean=E + 2) == sp.ERR_ALIGNMENT and _fwd(rstd=F + 2) == sp.ERR_ALIGNMENT and _fwd(gamma=B + 2, w=sp.FP32) == sp.ERR_ALIGNMENT
    for eps in (-1e-5, float("nan"), float("inf")):
        assert _fwd(eps=eps) == sp.ERR_INVALID_ARG
    assert _fwd(y=A) == sp.ERR_INVALID_ARG and _fwd(y=A + 2) == sp.ERR_INVALID_ARG                       # in place, and beside it
    assert _fwd(mean=A + 8 * 64 * 2 - 4) == sp.ERR_INVALID_ARG and _fwd(rstd=E + 4) == sp.ERR_INVALID_ARG
    assert _fwd(y=B + 64 * 2 - 2) == sp.ERR_INVALID_ARG and _fwd(mean=C) == sp.ERR_INVALID_ARG
    assert sp.last_error() != ""


def test_refusals_of_the_gradient():
    _refused_alike(_grad)
    for name in ("dy", "x", "mean", "rstd", "ws"):
        assert _grad(**{name: None}) == sp.ERR_INVALID_ARG
    assert _grad(dx=None, dgamma=None, dbeta=None) == sp.ERR_INVALID_ARG
    assert _grad(n=sp.layernorm_workspace(8, 64) - 1) == sp.ERR_INVALID_ARG
    for name in ("dy", "x", "gamma", "dx", "dgamma", "dbeta"):
        assert _grad(**{name: A * 10 + 1}) == sp.ERR_ALIGNMENT
    assert _grad(mean=D + 2) == sp.ERR_ALIGNMENT and _grad(rstd=E + 1) == sp.ERR_ALIGNMENT and _grad(ws=I + 8) == sp.ERR_ALIGNMENT
    assert _grad(dgamma=G + 2, w=sp.FP32) == sp.ERR_ALIGNMENT
    for out in ("dx", "dgamma", "dbeta", "ws"):
        for other in (A, B, C, D, E):
            assert _grad(**{out: other}) == sp.ERR_INVALID_ARG
    assert _grad(dx=I) == sp.ERR_INVALID_ARG and _grad(dgamma=H) == sp.ERR_INVALID_ARG and _grad(dx=G - 16) == sp.ERR_INVALID_ARG


def test_workspace_holds_two_rows_of_sums_for_every_block():
    for M, N in ((1, 1), (60, 304), (5000, 1031), (1 << 20, 4096), (7, sp.LAYERNORM_MAX_N), ((1 << 31) - 1, sp.LAYERNORM_MAX_N)):
        n = sp.layernorm_workspace(M, N)
        row = 2 * (N + 15) // 16 * 16 * 4
        assert n % 16 == 0 and row <= n <= 296 * 2 * (N + 15) * 4
    for M, N in ((0, 4), (4, 0), (1 << 31, 4), (4, sp.LAYERNORM_MAX_N + 1)):
        with pytest.raises(sp.SpError):
            sp.layernorm_workspace(M, N)


def test_binding_checks_shapes_and_types_before_the_library():
    torch = pytest.importorskip("torch")
    x, g, s = torch.zeros(3, 8), torch.ones(8), torch.zeros(3)
    with pytest.raises(ValueError, match="CUDA"):
        sp.layernorm(x, g, g, torch.zeros(3, 8))
    with pytest.raises(ValueError, match="shape and type of y"):
        sp.layernorm(x, g, g, torch.zeros(8, 3))
    with pytest.raises(ValueError, match="shape and type of y"):
        sp.layernorm(x, g, g, torch.zeros(3, 8, dtype=torch.float16))
    with pytest.raises(ValueError, match="weight"):
        sp.layernorm(x, g, torch.ones(7), torch.zeros(3, 8))
    with pytest.raises(ValueError, match="weight"):
        sp.layernorm(x, g, g.half(), torch.zeros(3, 8))
    with pytest.raises(ValueError, match="mean"):
        sp.layernorm(x, g, g, torch.zeros(3, 8), torch.zeros(4))
    with pytest.raises(ValueError, match="mean"):
        sp.layernorm_grad(x, x, g, s.double(), s, x, g, g)
    with pytest.raises(ValueError, match="shape and type of dx"):
        sp.layernorm_grad(x, x, g, s, s, x.half(), g, g)
    with pytest.raises(ValueError, match="shape and type of dy"):
        sp.layernorm_grad(x[:2], x, g, s, s, x, g, g)
    with pytest.raises(ValueError, match="element type"):
        sp.layernorm(x.double(), g, g, x.double())


def test_workspace_is_at_most_148_rows_of_sums():
    for M in (1, 13, 148, 5000, 1 << 20, (1 << 31) - 1):
        for N in (1, 8, 17, 304, 1031, 4096, 8193, 12291, 16385, sp.LAYERNORM_MAX_N):
            row = 2 * ((N + 15) // 16 * 16) * 4
            n = sp.layernorm_workspace(M, N)
            assert n % row == 0 and row <= n <= 148 * row
    assert sp.layernorm_workspace(1 << 20, 1) == 148 * 2 * 16 * 4
