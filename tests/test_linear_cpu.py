"""The linear-layer operators without a GPU: pins of their oracle, refusals on the host, workspace sizes, argument checks of the binding."""

import ctypes
import re
import os

import numpy as np
import pytest

import paper_2508_20258_b200 as sp
from paper_2508_20258_b200 import binding
from oracle import linear as LN

A, B = 0x100000, 0x200000     # never dereferenced: every check below fails on the host first


def test_oracle_quantiser_on_values_worked_by_hand():
    x = np.array([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5, 0.49], [0.0] * 7, [1.0, np.inf, 0, 0, 0, 0, 0], [np.nan, 1.0, 0, 0, 0, 0, 0]])
    q, s = LN.quantize_i8(x)
    assert q.shape == (4, 16)
    assert list(q[0, :7]) == [127, -127, 0, 2, 2, 0, 0] and (q[0, 7:] == 0).all() and s[0] == 1.0      # halves to even
    assert (q[1:] == 0).all() and s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3])


def test_oracle_quantiser_is_within_half_a_step():
    x = np.random.default_rng(0).standard_normal((50, 33))
    q, s = LN.quantize_i8(x)
    assert (np.abs(q[:, :33] * s[:, None].astype(np.float64) - x) <= 0.5 * s[:, None] * (1 + 1e-6)).all()
    assert (np.abs(q).max(axis=1) == 127).all()


def test_oracle_cross_entropy_against_direct_formulas_and_differences():
    rng = np.random.default_rng(1)
    h, W = rng.standard_normal((6, 5)), rng.standard_normal((9, 5))
    t = np.array([0, 8, -100, 3, 3, 1])
    for red in ("none", "mean", "sum"):
        grad = rng.uniform(0.5, 2.0, 6) if red == "none" else np.array([1.7])
        loss, lse, each, kept = LN.linear_ce(h, W, t, red)
        z = h @ W.T
        assert np.allclose(lse, np.log(np.exp(z).sum(axis=1)), rtol=1e-13)
        assert each[2] == 0 and kept.sum() == 5
        dh, dW, *_ = LN.linear_ce_grad(h, W, t, grad, red)
        f = lambda hh, ww: float(np.sum(LN.linear_ce(hh, ww, t, red)[0] * grad)) if red == "none" else float(LN.linear_ce(hh, ww, t, red)[0] * grad[0])  # noqa: E731
        for x, d, first in ((h, dh, True), (W, dW, False)):
            for i in np.ndindex(x.shape):
                e = np.zeros_like(x)
                e[i] = 1e-5
                num = (f(h + e, W) - f(h - e, W) if first else f(h, W + e) - f(h, W - e)) / 2e-5
                assert abs(num - d[i]) < 1e-8
        assert (dh[2] == 0).all()


def test_quantize_refusals():
    q = sp.lib().sp_quantize_i8
    assert q(None, sp.BF16, 4, 4, B, B, None) == sp.ERR_INVALID_ARG
    assert q(A, sp.BF16, 4, 4, None, B, None) == sp.ERR_INVALID_ARG
    assert q(A, sp.BF16, 4, 4, B, None, None) == sp.ERR_INVALID_ARG
    assert q(A, sp.BF16, 0, 4, B, B, None) == sp.ERR_INVALID_ARG
    assert q(A, sp.BF16, 4, -1, B, B, None) == sp.ERR_INVALID_ARG
    assert q(A, 3, 4, 4, B, B, None) == sp.ERR_INVALID_ARG
    assert q(A, sp.BF16, 1 << 31, 4, B, B, None) == sp.ERR_UNSUPPORTED
    assert q(A, sp.BF16, 4, 4, B + 8, B, None) == sp.ERR_ALIGNMENT
    assert q(A + 1, sp.BF16, 4, 4, B, B, None) == sp.ERR_ALIGNMENT
    assert q(A + 2, sp.FP32, 4, 4, B, B, None) == sp.ERR_ALIGNMENT
    assert q(A, sp.BF16, 4, 4, B, B + 2, None) == sp.ERR_ALIGNMENT
    assert sp.last_error() != ""


def _gemm(a=A, sa=A, b=A, sb=A, c=B, M=256, N=256, K=256, scheme=sp.ORDER_AUTO, **kw):
    p = sp.make_params(**{"b_layout": 1, **kw})
    return sp.lib().sp_gemm_i8(a, sa, b, sb, c, M, N, K, scheme, ctypes.byref(p), None)


def test_gemm_i8_refusals():
    for name in ("a", "sa", "b", "sb", "c"):
        assert _gemm(**{name: None}) == sp.ERR_INVALID_ARG
    for name in ("M", "N", "K"):
        assert _gemm(**{name: 0}) == sp.ERR_INVALID_ARG
    assert _gemm(K=264) == sp.ERR_ALIGNMENT
    assert _gemm(a=A + 8) == sp.ERR_ALIGNMENT and _gemm(b=A + 1) == sp.ERR_ALIGNMENT
    assert _gemm(sa=A + 1) == sp.ERR_ALIGNMENT and _gemm(c=B + 1) == sp.ERR_ALIGNMENT
    assert _gemm(c=B + 2, out_dtype=sp.FP32) == sp.ERR_ALIGNMENT
    assert _gemm(K=sp.I8_MAX_K + 16) == sp.ERR_UNSUPPORTED
    assert _gemm(M=1 << 31) == sp.ERR_UNSUPPORTED
    assert _gemm(b_layout=0) == sp.ERR_UNSUPPORTED
    assert _gemm(out_dtype=3) == sp.ERR_INVALID_ARG
    assert _gemm(tile_m=256, tile_n=512) == sp.ERR_UNSUPPORTED and _gemm(tile_m=128, tile_n=256) == sp.ERR_UNSUPPORTED
    assert _gemm(tile_m=256, tile_n=0) == sp.ERR_UNSUPPORTED
    assert _gemm(flags=sp.FLAG_STREAM_K) == sp.ERR_INVALID_ARG
    assert _gemm(scheme=-2) == sp.ERR_INVALID_ARG and _gemm(scheme=sp.GROUP_M, group=0) == sp.ERR_INVALID_ARG
    assert _gemm(M=256, N=512, scheme=sp.CUSTOM, tile_m=256, tile_n=256, custom_perm=[1, 1]) == sp.ERR_NOT_BIJECTIVE
    assert _gemm(M=256, N=512, scheme=sp.CUSTOM, custom_perm=[0, 1]) == sp.ERR_INVALID_ARG          # whose grid?
    assert _gemm(c=A) == sp.ERR_INVALID_ARG
    assert _gemm(M=1280, N=512, scheme=sp.XCD, tile_m=256, tile_n=256, num_xcds=4) == sp.ERR_NOT_BIJECTIVE
    p = sp.make_params(b_layout=1)
    p.struct_size = 4
    assert sp.lib().sp_gemm_i8(A, A, A, A, B, 256, 256, 256, 0, ctypes.byref(p), None) == sp.ERR_INVALID_ARG


def test_linear_i8_refuses_what_its_two_calls_refuse():
    f = sp.lib().sp_linear_i8
    p = sp.make_params(b_layout=1)
    assert f(None, sp.BF16, A, A, A, A, B, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG
    assert f(A, 7, A, A, A, A, B, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG
    assert f(A, sp.BF16, A, A, None, A, B, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG
    assert f(A, sp.BF16, A, A, A, A, B, 4, 0, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG
    assert f(A, sp.BF16, A, A, A, A, B, 4, 4, sp.I8_MAX_K + 1, -1, ctypes.byref(p), None) == sp.ERR_UNSUPPORTED
    assert f(A, sp.BF16, A + 4, A, A, A, B, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_ALIGNMENT
    assert f(A, sp.BF16, 2 * A, A, A, A, A, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG      # y = x
    assert f(A, sp.BF16, B, A, A, A, B, 4, 4, 4, -1, ctypes.byref(p), None) == sp.ERR_INVALID_ARG          # y = q


def _ce(h=A, W=A, t=A, lse=A, loss=B, T=8, V=100, D=64, dtype=sp.BF16, red=1, ws=B, n=1 << 40):
    return sp.lib().sp_linear_ce(h, W, t, lse, loss, T, V, D, dtype, -100, red, ws, n, None)


def _ce_grad(h=A, W=A, t=A, lse=A, g=A, dh=B, dW=B, T=8, V=100, D=64, dtype=sp.BF16, red=1, ws=B, n=1 << 40):
    return sp.lib().sp_linear_ce_grad(h, W, t, lse, g, dh, dW, T, V, D, dtype, -100, red, ws, n, None)


@pytest.mark.parametrize("f", [_ce, _ce_grad])
def test_linear_ce_refusals(f):
    for name in ("h", "W", "t", "lse", "ws"):
        assert f(**{name: None}) == sp.ERR_INVALID_ARG
    for name in ("T", "V", "D"):
        assert f(**{name: 0}) == sp.ERR_INVALID_ARG
        assert f(**{name: (1 << 31)}) == sp.ERR_UNSUPPORTED
    assert f(D=60) == sp.ERR_ALIGNMENT
    for name in ("h", "W", "ws"):
        assert f(**{name: A + 8}) == sp.ERR_ALIGNMENT
    assert f(t=A + 4) == sp.ERR_ALIGNMENT and f(lse=A + 2) == sp.ERR_ALIGNMENT
    assert f(dtype=sp.FP32) == sp.ERR_UNSUPPORTED
    assert f(red=3) == sp.ERR_INVALID_ARG
    assert f(n=sp.linear_ce_workspace(8, 100, 64, f is _ce_grad) - 1) == sp.ERR_INVALID_ARG


def test_linear_ce_refusals_of_one_call():
    assert _ce(loss=None) == sp.ERR_INVALID_ARG and _ce(loss=B + 2) == sp.ERR_ALIGNMENT
    assert _ce_grad(dh=None, dW=None) == sp.ERR_INVALID_ARG
    assert _ce_grad(dh=A) == sp.ERR_INVALID_ARG and _ce_grad(dW=A) == sp.ERR_INVALID_ARG      # in place
    assert _ce_grad(dh=B + 8) == sp.ERR_ALIGNMENT and _ce_grad(dW=B + 8) == sp.ERR_ALIGNMENT and _ce_grad(g=A + 2) == sp.ERR_ALIGNMENT


def test_workspace_is_in_pieces_and_never_holds_the_scores():
    for T, V, D in [(1, 2, 8), (16, 65536, 4096), (8192, 131072, 4096), (65536, 262144, 1024), (1 << 20, 1000, 64), (100, 1 << 24, 8)]:
        fwd, grad = sp.linear_ce_workspace(T, V, D), sp.linear_ce_workspace(T, V, D, True)
        rows = T * (D + 64) * 2                                                 # the tokens once more
        assert 0 < fwd <= T * ((V + 127) // 128 * 8 + 8) + rows + 4096         # a pair per 128 scores
        sums = 64 * T * D * 4                                                   # at most 64 slices of dh
        assert 0 < grad <= max(256 << 20, T * 1024 * 2) + T * 20 + T * 128 + sums + rows + 4096
    L = sp.lib()
    for bad in [(0, 8, 8), (8, -1, 8), (8, 8, 0), (1 << 31, 8, 8)]:
        assert L.sp_linear_ce_workspace(*bad, 0) == -1
        with pytest.raises(sp.SpError):
            sp.linear_ce_workspace(*bad)


def test_binding_checks_its_tensors():
    torch = pytest.importorskip("torch")
    x, q, s = torch.zeros(4, 20), torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4)
    w, y = torch.zeros(8, 32, dtype=torch.int8), torch.zeros(4, 8)
    ws = torch.zeros(8)
    for bad in [lambda: sp.quantize_i8(x, q[:, :16].contiguous(), s), lambda: sp.quantize_i8(x, q.int(), s), lambda: sp.quantize_i8(x, q, s.double()),
                lambda: sp.quantize_i8(x, q, s),                                                   # not on a GPU
                lambda: sp.linear_i8(x, q, s, w[:, :16].contiguous(), ws, y), lambda: sp.linear_i8(x, q, s, w, s, y),
                lambda: sp.linear_i8(x, q, s, w, ws, y.t().contiguous()), lambda: sp.linear_i8(x, q, s, w, ws, y),
                lambda: sp.gemm_i8(q, s, w[:, :16].contiguous(), ws, y), lambda: sp.gemm_i8(q, ws, w, ws, y), lambda: sp.gemm_i8(q, s, w, ws, y)]:
        with pytest.raises(ValueError):
            bad()
    h, W, t, lse, one = torch.zeros(4, 16).bfloat16(), torch.zeros(9, 16).bfloat16(), torch.zeros(4, dtype=torch.int64), torch.zeros(4), torch.zeros(1)
    for bad in [lambda: sp.linear_ce(h, W.half(), t, lse, one), lambda: sp.linear_ce(h, W[:, :8], t, lse, one), lambda: sp.linear_ce(h, W, t.int(), lse, one),
                lambda: sp.linear_ce(h, W, t, lse, lse), lambda: sp.linear_ce(h, W, t, lse, one, reduction="none"), lambda: sp.linear_ce(h, W, t, lse, one, reduction="avg"),
                lambda: sp.linear_ce(h.float(), W.float(), t, lse, one), lambda: sp.linear_ce(h, W, t, lse, one),
                lambda: sp.linear_ce_grad(h, W, t, lse, lse, h.clone(), None), lambda: sp.linear_ce_grad(h, W, t, lse, one, W, None),
                lambda: sp.linear_ce_grad(h, W, t, lse, one, h.clone(), W.clone())]:
        with pytest.raises(ValueError):
            bad()


def test_constants_match_the_header():
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "swizzleperf.h")).read()
    defs = {m.group(1): int(m.group(2)) for m in re.finditer(r"#define\s+SP_([A-Z_0-9]+)\s+\(?(-?\d+)\)?", text)}
    for name in ("BF16", "FP32", "FP16", "ORDER_AUTO", "I8_MAX_K", "REDUCE_NONE", "REDUCE_MEAN", "REDUCE_SUM"):
        assert defs[name] == getattr(binding, name), name


def test_a_workspace_is_taken_for_the_stream_it_is_used_on(monkeypatch):
    torch = pytest.importorskip("torch")
    import contextlib
    active, taken = ["current"], []

    class Stream:
        def __init__(self, handle):
            self.cuda_stream = handle

    @contextlib.contextmanager
    def use(stream):
        active.append(stream.cuda_stream)
        yield
        active.pop()

    class Like:
        def new_empty(self, n, dtype):
            taken.append(active[-1])
            return torch.empty(n, dtype=dtype)

    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(11))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 11, raising=False)
    for stream, want in ((None, "current"), (Stream(11), "current"), (11, "current"), (Stream(77), 77), (77, 77), (0, 0)):
        for grad in (0, 1):
            buf, n = binding._ce_workspace(None, Like(), (8, 100, 64), grad, stream)
            assert buf.numel() == n == sp.linear_ce_workspace(8, 100, 64, bool(grad)) and taken.pop() == want


# Addresses far apart, one for each argument, and then one output moved into another argument: to its start, its last element, or so that it ends in it.
FAR = {name: (i + 1) << 24 for i, name in enumerate("abcdefghij")}


def _moved(call, sizes, outs):
    """``call`` with every output moved into every other argument; ``sizes``: bytes of each argument."""
    at = {name: FAR["abcdefghij"[i]] for i, name in enumerate(sizes)}
    for out in outs:
        for other in sizes:
            if other != out:
                first = at[other]
                for where in (first, first + (sizes[other] - 1) // 16 * 16, first - (sizes[out] - 1) // 16 * 16):
                    assert call(**{**at, out: where}) == sp.ERR_INVALID_ARG, (out, other, where - first)
                    assert "overlap" in sp.last_error()


def test_what_is_written_must_not_lie_in_anything_else_of_the_call():
    L = sp.lib()
    p = sp.make_params(b_layout=1)
    M, N, K, kp = 70, 130, 300, 304
    _moved(lambda x, q, s: L.sp_quantize_i8(x, sp.BF16, M, K, q, s, None), dict(x=M * K * 2, q=M * kp, s=M * 4), ["q", "s"])
    _moved(lambda a, sa, b, sb, c: L.sp_gemm_i8(a, sa, b, sb, c, M, N, kp, -1, ctypes.byref(p), None), dict(a=M * kp, sa=M * 4, b=N * kp, sb=N * 4, c=M * N * 2), ["c"])
    _moved(lambda x, q, s, w, ws, y: L.sp_linear_i8(x, sp.FP32, q, s, w, ws, y, M, N, K, -1, ctypes.byref(p), None),
           dict(x=M * K * 4, q=M * kp, s=M * 4, w=N * kp, ws=N * 4, y=M * N * 2), ["q", "s", "y"])
    T, V, D = 40, 500, 64
    for red, n in ((sp.REDUCE_NONE, T), (sp.REDUCE_SUM, 1)):
        f, g = sp.linear_ce_workspace(T, V, D), sp.linear_ce_workspace(T, V, D, True)
        _moved(lambda h, W, t, lse, loss, ws: L.sp_linear_ce(h, W, t, lse, loss, T, V, D, sp.BF16, -100, red, ws, f, None),
               dict(h=T * D * 2, W=V * D * 2, t=T * 8, lse=T * 4, loss=n * 4, ws=f), ["lse", "loss", "ws"])
        _moved(lambda h, W, t, lse, grad, dh, dW, ws: L.sp_linear_ce_grad(h, W, t, lse, grad, dh, dW, T, V, D, sp.BF16, -100, red, ws, g, None),
               dict(h=T * D * 2, W=V * D * 2, t=T * 8, lse=T * 4, grad=n * 4, dh=T * D * 2, dW=V * D * 2, ws=g), ["dh", "dW", "ws"])


def test_arguments_side_by_side_are_accepted():
    # one byte behind the other: the checks pass, and the call ends where it asks for a device (or runs, on a GPU: not here)
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    L = sp.lib()
    M, K = 32, 64
    assert L.sp_quantize_i8(FAR["a"], sp.BF16, M, K, FAR["a"] + M * K * 2, FAR["a"] + M * K * 3, None) not in (sp.OK, sp.ERR_INVALID_ARG)
    T, V, D = 32, 64, 64
    n = sp.linear_ce_workspace(T, V, D)
    at = [FAR["a"]]
    for size in (T * D * 2, V * D * 2, T * 8, T * 4, T * 4):
        at.append(at[-1] + size)
    assert L.sp_linear_ce(at[0], at[1], at[2], at[3], at[4], T, V, D, sp.BF16, -100, sp.REDUCE_NONE, at[5], n, None) not in (sp.OK, sp.ERR_INVALID_ARG)


@pytest.mark.parametrize("f", [_ce, _ce_grad])
def test_sizes_that_no_grid_of_tiles_holds_are_refused_before_anything_is_launched(f):
    L = sp.lib()
    for T, V, D in [(1 << 24, 1 << 18, 64), (1 << 30, 1, 1 << 20), (1, 1 << 30, 1 << 20), ((1 << 31) - 1024, (1 << 31) - 1024, 8), ((1 << 31) - 1024, 8, (1 << 31) - 1024)]:
        assert f(T=T, V=V, D=D, n=(1 << 62)) == sp.ERR_UNSUPPORTED
        assert L.sp_linear_ce_workspace(T, V, D, 0) == L.sp_linear_ce_workspace(T, V, D, 1) == -1
    for T, V, D in [(1 << 22, 1 << 16, 64), (1 << 20, 1 << 18, 1 << 12), (8, 1 << 24, 1 << 14)]:
        for grad in (0, 1):
            assert 0 < L.sp_linear_ce_workspace(T, V, D, grad) < 1 << 46


def test_the_current_stream_is_found_by_torchs_public_interface(monkeypatch):
    torch = pytest.importorskip("torch")

    class Stream:
        cuda_stream = 11

    def private(device):
        return 12

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", private, raising=False)
    assert binding._stream_handle(None) == 11 and binding._stream_on(0, None) == 12
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert binding._stream_handle(None) == binding._stream_on(0, None) == 11
    assert binding._stream_on(0, 7) == 7 and binding._stream_on(0, Stream()) == 11
