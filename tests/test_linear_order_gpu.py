"""The linear-layer calls in front of a launch that does not wait for its predecessor (SP_FLAG_OVERLAP).  Such a launch may run beside the call
before it, of which it is independent, but it may read what the call before that one wrote."""

import pytest

import paper_2508_20258_b200 as sp

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def randn(*shape, seed, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def int8(*shape, seed):
    return torch.randint(-127, 128, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed), dtype=torch.int32).to(torch.int8)


def quantiser():
    x, q, s = randn(3, 512, seed=1), torch.empty(3, 512, dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
    return lambda: sp.quantize_i8(x, q, s), [q, s]


def linear(tokens, k=1024, dtype=torch.bfloat16):
    n = 512
    x, w, ws = randn(tokens, k, seed=2, dtype=dtype), int8(n, k, seed=3), torch.full((n,), 0.01, device="cuda")
    q, s, y = torch.empty(tokens, k, dtype=torch.int8, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty(tokens, n, device="cuda")
    return lambda: sp.linear_i8(x, q, s, w, ws, y), [q, s, y]


def product(tokens):
    a, w, one = int8(tokens, 256, seed=4), int8(512, 256, seed=5), torch.ones(600, device="cuda")
    y = torch.empty(tokens, 512, device="cuda")
    return lambda: sp.gemm_i8(a, one[:tokens].contiguous(), w, one[:512].contiguous(), y), [y]


def loss(T, V=700, D=64, reduction="mean"):
    h, W, t = randn(T, D, seed=6), randn(V, D, seed=7), torch.arange(T, device="cuda") % V
    lse, out, ws = torch.empty(T, device="cuda"), torch.empty(1, device="cuda"), torch.empty(sp.linear_ce_workspace(T, V, D), dtype=torch.uint8, device="cuda")
    return lambda: sp.linear_ce(h, W, t, lse, out, reduction=reduction, workspace=ws), [lse, out]


def gradient(T, V=700, D=64, dh=True, dW=True):
    h, W, t = randn(T, D, seed=8), randn(V, D, seed=9), torch.arange(T, device="cuda") % V
    lse, out = torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    sp.linear_ce(h, W, t, lse, out)
    dh, dW = torch.empty_like(h) if dh else None, torch.empty_like(W) if dW else None
    ws = torch.empty(sp.linear_ce_workspace(T, V, D, True), dtype=torch.uint8, device="cuda")
    return lambda: sp.linear_ce_grad(h, W, t, lse, None, dh, dW, workspace=ws), [v for v in (dh, dW) if v is not None]


def gemm():
    a, b, y = randn(256, 64, seed=13), randn(64, 256, seed=14), torch.empty(256, 256, dtype=torch.bfloat16, device="cuda")
    return lambda: sp.gemm(a, b, y, sp.ROW_MAJOR, sp.make_params(tile_m=128, tile_n=128)), [y]


CALLS = {"bf16 product": gemm, "quantiser": quantiser, "linear 1": lambda: linear(1), "linear 1 long": lambda: linear(1, 16384), "linear 1 fp32": lambda: linear(1, dtype=torch.float32),
         "linear 24": lambda: linear(24), "linear 300": lambda: linear(300), "product 2": lambda: product(2), "product 20": lambda: product(20), "product 300": lambda: product(300),
         "loss 1": lambda: loss(1), "loss 20": lambda: loss(20), "loss 200": lambda: loss(200, reduction="sum"), "loss copied": lambda: loss(400, 900000, 72),
         "gradient 1": lambda: gradient(1), "gradient 20": lambda: gradient(20), "gradient dh": lambda: gradient(20, dW=False), "gradient dW": lambda: gradient(20, dh=False),
         "gradient whole": lambda: gradient(2560, 600, 2048), "gradient pieces": lambda: gradient(2048, 70001, 64)}


@pytest.mark.parametrize("name", list(CALLS))
def test_an_overlapping_product_behind_a_linear_call_sees_what_came_before(name):
    call, outs = CALLS[name]()
    call()
    want = [v.clone() for v in outs]
    M, N, K = 8192, 2048, 8192                                          # X takes a tenth of a millisecond and more
    A, B, B2 = randn(M, K, seed=10), randn(K, N, seed=11), randn(N, 512, seed=12)
    X, C = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), torch.zeros(M, 512, dtype=torch.bfloat16, device="cuda")
    first, second = sp.make_params(tile_m=256, tile_n=256), sp.make_params(tile_m=128, tile_n=128, flags=sp.FLAG_OVERLAP)
    sp.gemm(A, B, X, sp.ROW_MAJOR, first)
    sp.gemm(X, B2, C, sp.ROW_MAJOR, sp.make_params(tile_m=128, tile_n=128))
    assert sp.get_status() == 0
    want_C = C.clone()
    for _ in range(3):
        for v in (X, C, *outs):
            v.zero_()
        torch.cuda.synchronize()
        sp.gemm(A, B, X, sp.ROW_MAJOR, first)
        call()
        sp.gemm(X, B2, C, sp.ROW_MAJOR, second)                         # independent of `call`, not of X's product
        assert sp.get_status() == 0
        assert torch.equal(C, want_C)
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
