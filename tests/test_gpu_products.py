"""The product in the linear kernels' epilogues, held to its bound by a check that neither NaN nor a wrong sign passes."""
import math

import pytest
import torch

from test_gpu_ffn import GLU_SHAPES, act64, gen, normal


def product_errors(H, G, U, act):
    """Where H is not fp16(act(G) U).  Finite G and U; the bounds are those of assert_product_close (the exponent's argument |z| 2^-22, the
    exponential (2 + 1.173 |z|) ulp, sum, quotient and product 2^-21 together, the fp16 store 2^-11 or 2^-25; |H| < 65504^2 2^-126 where the
    quotient is flushed).  A product of 65504 and more is at least 65472 in magnitude, and has its sign."""
    g, u = G.double(), U.double()
    z = g if act == "silu" else math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
    # (not g / (1 + exp(-z)): infinite over infinite far below zero)
    ref = g * torch.sigmoid(z) * u
    zz = z.abs().clamp(max=90.0)
    rel = 2.0 ** -11 + zz * 2.0 ** -22 + (2 + 1.173 * zz) * 2.0 ** -23 + 2.0 ** -21
    h = H.double()
    fits = ref.abs() < 65504.0
    right = torch.where(fits, (h - ref).abs() <= ref.abs() * rel + 2.0 ** -25, (h.abs() >= 65472.0) & (h.sign() == ref.sign()))
    return ~right


def test_the_check_sees_nan_and_signs():
    g = torch.tensor([1.0, -2.0, 300.0, -60000.0, 0.0], dtype=torch.float16)
    u = torch.tensor([3.0, 0.5, -300.0, 60000.0, 7.0], dtype=torch.float16)
    for act in ("silu", "gelu_tanh"):
        h = act64(g.double(), act) * u.double()
        h = torch.where(h.isnan(), 0.0, h).half()
        assert not product_errors(h, g, u, act).any()
        for i in range(5):
            bad = h.clone()
            bad[i] = float("nan")
            assert product_errors(bad, g, u, act).tolist() == [j == i for j in range(5)]
        bad = h.clone()
        bad[2] = float("inf")                       # -90000, that is -inf
        assert product_errors(bad, g, u, act).tolist() == [j == 2 for j in range(5)]


@pytest.fixture(scope="module")
def aser():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2411_07762_b200 as aser
    return aser


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,F,K,r,kernel", GLU_SHAPES)
def test_product_of_gates_of_every_size(aser, M, F, K, r, kernel, act):
    """Every kernel's epilogue: gates from 2^-24 to beyond fp16 by the channel scales, of either sign; where both factors are finite the
    product is right and no NaN."""
    N = 2 * F
    assert aser.lib.aser_linear_kernel(M, N, K) == kernel
    g = gen(M * 3 + F)
    layer = aser.AserLinear(normal(g, N, K, scale=2.0 / math.sqrt(K)), None, normal(g, r, K, scale=0.02) if r else None,
                            normal(g, N, r, scale=0.05) if r else None, M)
    layer.w_scale *= torch.exp2(torch.linspace(-20, 18, F, device="cuda"))[torch.randperm(F, device="cuda", generator=g)].repeat_interleave(2)
    layer.w_scale[1::2] = layer.w_scale[1::2].clamp(max=1.0)
    X = normal(g, M, K)
    layer.quant(X)
    layer.linear(M)
    Y = layer.Y.clone()
    H = aser.linear_w4a8_lr_glu(layer.Xq, layer.a_scale, layer.Wk, layer.w_scale, layer.T, layer.L_B, N, layer.ws, act)
    G, U = Y[:, 0::2], Y[:, 1::2]
    fin = torch.isfinite(G) & torch.isfinite(U)
    assert fin.any()
    bad = product_errors(torch.where(fin, H, 0), torch.where(fin, G, 0), torch.where(fin, U, 0), act)
    assert not bad.any(), "%d of %d wrong" % (int(bad.sum()), bad.numel())
