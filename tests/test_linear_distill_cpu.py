"""Distillation without a GPU: pins of its oracle, refusals on the host, workspace sizes, argument checks of the binding."""

import numpy as np
import pytest

import paper_2508_20258_b200 as sp
from oracle import distill as DI
from oracle import linear as LN

# never dereferenced: every check below fails on the host first
A, B, C, D, E, F, G, H, I, J = (0x10000000 * (i + 1) for i in range(10))


def test_oracle_on_values_worked_by_hand():
    # one dimension: scores are W itself; q = (3/4, 1/4) on words 0 and 2, p = (1, 2, 1) / 4
    h, W = np.array([[1.0]]), np.log(np.array([[1.0], [2.0], [1.0]]))
    loss, lse, diff, *_ = DI.linear_distill(h, W, np.array([[2, 0]]), np.log(np.array([[1.0, 3.0]])), 1.0, "sum")
    assert np.allclose(loss, 0.75 * np.log(3.0) + 0.25 * np.log(1.0)) and np.allclose(lse, np.log(4.0))
    assert np.allclose(diff, [[0.0, -0.5]])


def test_oracle_with_one_word_is_the_cross_entropy():
    rng = np.random.default_rng(0)
    h, W, t = rng.standard_normal((5, 4)), rng.standard_normal((9, 4)), np.array([3, 0, -1, 8, 8])
    logit = rng.standard_normal((5, 1))
    loss, lse, diff, *_ = DI.linear_distill(h, W, t[:, None], logit, 1.0, "none")
    want, want_lse, *_ = LN.linear_ce(h, W, t, "none", -1)
    assert np.allclose(loss, want) and np.allclose(lse[t >= 0], want_lse[t >= 0]) and np.isinf(lse[2]) and diff[2, 0] == 0
    for got, ref in zip(DI.linear_distill_grad(h, W, t[:, None], logit, 1.0, 1.0, "mean"), LN.linear_ce_grad(h, W, t, 1.0, "mean", -1)):
        assert np.allclose(got, ref)


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(1)
    h, W = rng.standard_normal((4, 3)), rng.standard_normal((7, 3))
    index = np.array([[0, 3, 3], [6, -1, 2], [-1, -1, -1], [5, 1, 0]])
    logit = rng.standard_normal((4, 3))
    logit[3, 1] = -np.inf
    for tau in (0.5, 1.0, 3.0):
        grad = rng.uniform(0.5, 2.0, 4)
        f = lambda a, b: float((DI.linear_distill(a, b, index, logit, tau, "none")[0] * grad).sum())  # noqa: E731
        dh, dW = DI.linear_distill_grad(h, W, index, logit, grad, tau, "none")
        for x, d, first in ((h, dh, True), (W, dW, False)):
            for i in np.ndindex(x.shape):
                e = np.zeros_like(x)
                e[i] = 1e-5
                num = (f(h + e, W) - f(h - e, W) if first else f(h, W + e) - f(h, W - e)) / 2e-5
                assert abs(num - d[i]) < 1e-7


def _fwd(h=A, W=B, index=C, logit=D, top=sp.FP32, lse=E, diff=F, loss=G, T=8, V=100, DD=64, K=4, dtype=sp.BF16, tau=1.0, red=1, ws=H, n=1 << 40):
    return sp.lib().sp_linear_distill(h, W, index, logit, top, lse, diff, loss, T, V, DD, K, dtype, tau, red, ws, n, None)


def _grad(h=A, W=B, index=C, lse=D, diff=E, g=F, dh=G, dW=H, T=8, V=100, DD=64, K=4, dtype=sp.BF16, tau=1.0, red=1, ws=I, n=1 << 40):
    return sp.lib().sp_linear_distill_grad(h, W, index, lse, diff, g, dh, dW, T, V, DD, K, dtype, tau, red, ws, n, None)


@pytest.mark.parametrize("f", [_fwd, _grad])
def test_refusals_of_both_calls(f):
    for name in ("h", "W", "index", "lse", "diff", "ws"):
        assert f(**{name: None}) == sp.ERR_INVALID_ARG
    for name in ("T", "V", "DD", "K"):
        assert f(**{name: 0}) == sp.ERR_INVALID_ARG and f(**{name: -1}) == sp.ERR_INVALID_ARG
    for name in ("T", "V"):
        assert f(**{name: 1 << 31}) == sp.ERR_UNSUPPORTED
    assert f(K=sp.DISTILL_MAX_TOP + 1) == sp.ERR_UNSUPPORTED and f(T=1 << 30, V=1 << 30) == sp.ERR_UNSUPPORTED
    assert f(dtype=sp.FP32) == sp.ERR_UNSUPPORTED and f(DD=60) == sp.ERR_ALIGNMENT
    assert f(red=3) == sp.ERR_INVALID_ARG and f(red=-1) == sp.ERR_INVALID_ARG
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-5, 1e5):
        assert f(tau=tau) == sp.ERR_INVALID_ARG
    assert f(h=A + 8) == sp.ERR_ALIGNMENT and f(W=B + 2) == sp.ERR_ALIGNMENT and f(ws=J + 8) == sp.ERR_ALIGNMENT
    assert f(index=C + 4) == sp.ERR_ALIGNMENT and f(lse=J + 2) == sp.ERR_ALIGNMENT and f(diff=J + 1) == sp.ERR_ALIGNMENT
    assert sp.last_error() != ""


def test_refusals_of_the_forward_pass():
    assert _fwd(loss=None) == sp.ERR_INVALID_ARG and _fwd(logit=None) == sp.ERR_INVALID_ARG
    assert _fwd(top=3) == sp.ERR_UNSUPPORTED and _fwd(logit=D + 2) == sp.ERR_ALIGNMENT and _fwd(loss=G + 2) == sp.ERR_ALIGNMENT
    assert _fwd(n=sp.linear_distill_workspace(8, 100, 64, 4) - 1) == sp.ERR_INVALID_ARG
    for out in ("lse", "diff", "loss", "ws"):
        for other in (A, B, C, D):
            assert _fwd(**{out: other}) == sp.ERR_INVALID_ARG
    assert _fwd(lse=F) == sp.ERR_INVALID_ARG and _fwd(loss=F + 4 * 8 * 4 - 4) == sp.ERR_INVALID_ARG and _fwd(diff=H + 16) == sp.ERR_INVALID_ARG


def test_refusals_of_the_gradient():
    assert _grad(dh=None, dW=None) == sp.ERR_INVALID_ARG
    assert _grad(dh=G + 8) == sp.ERR_ALIGNMENT and _grad(dW=H + 2) == sp.ERR_ALIGNMENT and _grad(g=F + 1) == sp.ERR_ALIGNMENT
    assert _grad(n=sp.linear_distill_workspace(8, 100, 64, 4, grad=True) - 1) == sp.ERR_INVALID_ARG
    for out in ("dh", "dW", "ws"):
        for other in (A, B, C, D, E, F):
            assert _grad(**{out: other}) == sp.ERR_INVALID_ARG
    assert _grad(dh=H) == sp.ERR_INVALID_ARG and _grad(dW=I) == sp.ERR_INVALID_ARG


def test_workspace_sizes():
    assert sp.linear_distill_workspace(4096, 32768, 2048, 64) >= 4096 * (256 * 10 + 64 * 20)
    assert sp.linear_distill_workspace(8192, 131072, 4096, 100) < 8192 * (1024 * 13 + 100 * 24)
    assert sp.linear_distill_workspace(65, 100, 64, 4, grad=True) == sp.linear_ce_workspace(65, 100, 64, grad=True)
    assert sp.linear_distill_workspace(64, 100, 64, 4, grad=True) > sp.linear_ce_workspace(64, 100, 64, grad=True)      # rounding errors have rows of their own
    for sizes in ((0, 1, 8, 1), (1, 0, 8, 1), (1, 1, 0, 1), (1, 1, 8, 0), (1, 1, 8, sp.DISTILL_MAX_TOP + 1), (1 << 31, 1, 8, 1)):
        with pytest.raises(sp.SpError):
            sp.linear_distill_workspace(*sizes)


def test_binding_checks_shapes_and_types_before_the_library():
    torch = pytest.importorskip("torch")
    h, W = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16)
    index, logit, lse, diff, loss = torch.zeros(3, 2, dtype=torch.int64), torch.zeros(3, 2), torch.zeros(3), torch.zeros(3, 2), torch.zeros(1)
    good = dict(h=h, W=W, top_index=index, top_logit=logit, lse=lse, diff=diff, loss=loss)
    with pytest.raises(ValueError, match="CUDA"):
        sp.linear_distill(**good)
    for name, wrong in (("W", W[:, :4]), ("top_index", index[:2]), ("top_logit", logit[:, :1]), ("lse", lse[:2]), ("diff", diff.t()), ("loss", lse)):
        with pytest.raises(ValueError, match="shapes"):
            sp.linear_distill(**{**good, name: wrong})
    for name, wrong in (("W", W.half()), ("top_index", index.int()), ("lse", lse.double()), ("diff", diff.half()), ("loss", loss.double())):
        with pytest.raises(ValueError, match="types"):
            sp.linear_distill(**{**good, name: wrong})
    with pytest.raises(ValueError, match="reduction"):
        sp.linear_distill(**good, reduction="max")
    with pytest.raises(ValueError, match="element type"):
        sp.linear_distill(**{**good, "top_logit": logit.double()})
    back = dict(h=h, W=W, top_index=index, lse=lse, diff=diff, grad_loss=None, dh=h.clone(), dW=W.clone())
    with pytest.raises(ValueError, match="CUDA"):
        sp.linear_distill_grad(**back)
    with pytest.raises(ValueError, match="gradient"):
        sp.linear_distill_grad(**{**back, "dh": h.half()})
    with pytest.raises(ValueError, match="grad_loss"):
        sp.linear_distill_grad(**{**back, "grad_loss": lse})
