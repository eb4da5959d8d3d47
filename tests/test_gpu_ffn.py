"""Gated feed-forward block on the GPU: the product in the linear kernels' epilogues against 64 bits, the whole block
against its steps, refusals, streams, graphs and workspaces."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aser():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2411_07762_b200 as aser
    return aser


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, scale=1.0):
    return torch.randn(*shape, device="cuda", dtype=torch.float16, generator=g) * scale


def act64(z, act):
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))


def assert_product_close(H, G, U, act):
    """H = fp16(act(G) U) with fp16 G and U.  Relative error of the fp32 evaluation: the exponent's argument carries four
    roundings (|z| 2^-22), __expf is off by 2 + 1.173 |z| ulp (CUDA's bound), the sum, the quotient (2 ulp) and the product by
    2^-21 together; the fp16 store by 2^-11, or 2^-25 below the normal range.  The quotient is 0 where 1 + exp(-z) is above 2^126
    (|z| > 87): there |H| < 65504^2 2^-126."""
    g, u = G.double(), U.double()
    z = g if act == "silu" else math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
    ref = act64(g, act) * u
    zz = z.abs().clamp(max=90.0)
    rel = 2.0 ** -11 + zz * 2.0 ** -22 + (2 + 1.173 * zz) * 2.0 ** -23 + 2.0 ** -21
    fits = ref.abs() < 65504.0
    err = (H.double() - ref).abs()
    bad = (err > ref.abs() * rel + 2.0 ** -25) & fits
    assert not bad.any(), "%d wrong, worst error / bound %.3f" % (int(bad.sum()), float((err / (ref.abs() * rel + 2.0 ** -25))[fits].max()))
    assert (H[~fits].double().abs() >= 65472.0).all()


# every kernel that serves the projection, at whole and ragged tiles: (tokens, F, K, rank, the kernel by aser_linear_kernel)
GLU_SHAPES = [
    (1, 256, 128, 0, 0), (1, 7168, 1024, 64, 0), (8, 2048, 4096, 16, 0), (9, 264, 512, 128, 0), (16, 1000, 640, 256, 0),
    (5, 14336, 256, 32, 0), (16, 7168, 2048, 0, 0),
    (17, 512, 1024, 64, 3), (64, 1024, 2048, 0, 3), (100, 4096, 4096, 128, 3), (333, 1024, 1152, 48, 3), (511, 1040, 1024, 256, 3),
    (1024, 4096, 1024, 64, 2), (2048, 4104, 1024, 0, 2), (2048, 8200, 512, 256, 2), (600, 16384, 4096, 128, 2), (777, 3592, 4096, 192, 2),
    (130, 40, 384, 64, 2), (300, 16, 640, 80, 2),
    (20, 264, 256, 16, 1), (40, 120, 512, 0, 1), (65, 72, 256, 192, 1), (700, 4096, 1024, 64, 1), (1025, 8192, 512, 256, 1),
    (1100, 2048, 4096, 80, 1), (16, 32768, 2176, 32, 1), (33, 32768, 1024, 16, 1),
]


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M,F,K,r,kernel", GLU_SHAPES)
def test_product_in_the_epilogue(aser, M, F, K, r, kernel, act):
    """The channels that the ordinary launch stores, and their product: the gated launch stores exactly act(G) * U."""
    N = 2 * F
    assert aser.lib.aser_linear_kernel(M, N, K) == kernel
    g = gen(M * 7 + F)
    layer = aser.AserLinear(normal(g, N, K, scale=2.0 / math.sqrt(K)), None, normal(g, r, K, scale=0.02) if r else None,
                            normal(g, N, r, scale=0.05) if r else None, M)
    X = normal(g, M, K)
    layer.quant(X)
    layer.linear(M)
    Y = layer.Y.clone()
    H = torch.full((M + 1, F), 7.0, device="cuda", dtype=torch.float16)
    aser.linear_w4a8_lr_glu(layer.Xq, layer.a_scale, layer.Wk, layer.w_scale, layer.T, layer.L_B, N, layer.ws, act, H=H)
    aser.check_status(layer.ws)
    assert (H[M] == 7.0).all()                      # the row behind the last token
    assert_product_close(H[:M], Y[:, 0::2], Y[:, 1::2], act)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M", [3, 16, 40, 700])
def test_values_of_every_size(aser, M, act):
    """Gates from the smallest to the largest fp16 magnitude, both signs, and infinite ones, set through the channel scales."""
    F, K = 1024, 1024
    g = gen(M)
    layer = aser.AserLinear(normal(g, 2 * F, K, scale=2.0 / math.sqrt(K)), None, None, None, M)
    layer.w_scale *= torch.exp2(torch.linspace(-24, 15, F, device="cuda")).repeat_interleave(2)
    layer.w_scale[1::2] = layer.w_scale[1::2].clamp(max=1e-2)
    layer.w_scale[0::512] *= 1e5
    X = normal(g, M, K)
    layer.quant(X)
    layer.linear(M)
    Y = layer.Y.clone()
    H = aser.linear_w4a8_lr_glu(layer.Xq, layer.a_scale, layer.Wk, layer.w_scale, None, None, 2 * F, layer.ws, act)
    G, U = Y[:, 0::2], Y[:, 1::2]
    fin = torch.isfinite(G)
    assert (~fin).any()
    assert_product_close(torch.where(fin, H, 0), torch.where(fin, G, 0), torch.where(fin, U, 0), act)
    up = G == float("inf")                          # act(inf) = inf
    some = up & (U != 0)
    assert torch.equal(H[some], torch.where(U[some] > 0, float("inf"), float("-inf")).half())


def make_block(aser, g, M, K, F, N, r, r_down, act, smooth=True):
    W = [normal(g, F, K, scale=1.0 / math.sqrt(K)) for _ in range(2)]
    Wd = normal(g, N, F, scale=1.0 / math.sqrt(F))
    s = sd = None
    if smooth:
        s = torch.ones(K, device="cuda")
        s[torch.randperm(K, device="cuda", generator=g)[:3]] = 11.0
        sd = torch.ones(F, device="cuda")
        sd[torch.randperm(F, device="cuda", generator=g)[:3]] = 7.0
    f = lambda k, n, rr: (normal(g, rr, k, scale=0.02), normal(g, n, rr, scale=0.02)) if rr else (None, None)
    LA, LB = f(K, 2 * F, r)
    LAd, LBd = f(F, N, r_down)
    return (W[0], W[1], s, LA, LB, Wd, sd, LAd, LBd), aser.AserGatedFFN(W[0], W[1], s, LA, LB, Wd, sd, LAd, LBd, M, activation=act)


BLOCKS = [(1, 512, 1024, 512, 64, 64, "silu"), (8, 256, 640, 264, 0, 16, "gelu_tanh"), (16, 4096, 2048, 4096, 128, 0, "silu"),
          (17, 1024, 1152, 1000, 32, 32, "silu"), (47, 512, 256, 8, 0, 0, "silu"), (128, 1024, 2048, 1024, 64, 128, "gelu_tanh"),
          (333, 2048, 4096, 2048, 64, 64, "silu"), (1100, 1024, 4096, 1024, 256, 192, "silu"), (2100, 4096, 1024, 512, 64, 64, "gelu_tanh")]


class Steps:
    """The block's steps, each through its own entry point."""

    def __init__(self, aser, ops, M):
        Wg, Wu, s, LA, LB, Wd, sd, LAd, LBd = ops
        F = Wg.shape[0]
        self.aser, self.F = aser, F
        self.first = aser.AserLinear(aser.interleave_gate_up(Wg, Wu), s, LA,
                                     None if LB is None else aser.interleave_gate_up(LB[:F], LB[F:]), M)
        self.down = aser.AserLinear(Wd, sd, LAd, LBd, M)

    def __call__(self, X, act):
        f, M = self.first, X.shape[0]
        self.aser.quant_act_fine(X, f.s, f.L_A, f.ws, out=(f.Xq, f.a_scale, f.T))
        f.linear(M)
        H = self.aser.linear_w4a8_lr_glu(f.Xq[:M], f.a_scale, f.Wk, f.w_scale, f.T, f.L_B, 2 * self.F, f.ws, act)
        return f.Y[:M], H, self.down(H)


@pytest.mark.parametrize("M,K,F,N,r,r_down,act", BLOCKS)
def test_block_is_its_steps(aser, M, K, F, N, r, r_down, act):
    """The whole block has the bits of its steps; the steps are held to 64 bits."""
    g = gen(M + K + F)
    ops, block = make_block(aser, g, M, K, F, N, r, r_down, act)
    X = normal(g, M, K)
    Y = block(X).clone()
    aser.check_status(block.ws)
    steps = Steps(aser, ops, M)
    assert torch.equal(steps.first.Wk, block.Wk)
    GU, H, want = steps(X, act)
    assert_product_close(H, GU[:, 0::2], GU[:, 1::2], act)
    assert torch.equal(want, Y)
    # the projections' channels and the result against 64 bits (the project's bound for a layer's output: 2e-3 of the row's largest)
    for layer, x, out in ((steps.first, X, GU), (steps.down, H, Y)):
        ref = layer.Xq.double() @ dequantized(layer).T * layer.a_scale.double()[:, None]
        if layer.r:
            xs = x.float() / layer.s
            ref += (xs.double() @ layer.L_A.double().T) @ layer.L_B.double().T
        assert ((out.double() - ref).abs() <= 2e-3 * ref.abs().amax(1, keepdim=True)).all()


def dequantized(layer):
    w = layer.Wq
    lo = (w & 15).to(torch.int16)
    hi = (w >> 4).to(torch.int16)
    q = torch.stack([lo, hi], dim=2).reshape(layer.N, layer.K)
    q = torch.where(q > 7, q - 16, q)
    return q.double() * layer.w_scale.double()[:, None]


def test_block_without_smoothing_and_fewer_tokens(aser):
    """One block and one workspace for calls of different sizes in turn."""
    g = gen(5)
    ops, block = make_block(aser, g, 300, 512, 1024, 512, 32, 32, "silu", smooth=False)
    steps = Steps(aser, ops, 300)
    X = normal(g, 300, 512)
    for m in (300, 0, 1, 17, 64, 65, 299, 300):
        part = block(X[:m].contiguous())
        assert part.shape == (m, 512)
        if m:
            assert torch.equal(part, steps(X[:m].contiguous(), "silu")[2])


def test_factors_made_apart(aser):
    """Gate and up with factors of their own, in the stacked form given in the header: the channels are those of the two
    layers.  Either side is within 2e-3 of the row's largest value of the exact one, so they are within twice that."""
    g = gen(11)
    M, K, F = 33, 512, 1024
    W = [normal(g, F, K, scale=0.05) for _ in range(2)]
    A = [normal(g, r, K, scale=0.05) for r in (16, 32)]
    B = [normal(g, F, r, scale=0.05) for r in (16, 32)]
    LB = torch.zeros(2, F, 48, device="cuda", dtype=torch.float16)
    LB[0, :, :16], LB[1, :, 16:] = B
    X = normal(g, M, K)
    block = aser.AserGatedFFN(W[0], W[1], None, torch.cat(A), LB.reshape(2 * F, 48), normal(g, 256, F, scale=0.03), None, None, None, M)
    steps = Steps(aser, (W[0], W[1], None, torch.cat(A), LB.reshape(2 * F, 48), normal(g, 256, F, scale=0.03), None, None, None), M)
    assert torch.equal(block.L_B, steps.first.L_B) and torch.equal(block.Wk, steps.first.Wk)
    GU = steps(X, "silu")[0]
    for i in range(2):
        want = aser.AserLinear(W[i], None, A[i], B[i], M)(X).double()
        assert ((GU[:, i::2].double() - want).abs() <= 4e-3 * want.abs().amax(1, keepdim=True)).all()


def test_streams_and_graphs(aser):
    """On a stream of its own, captured and replayed with new inputs, and two graphs with workspaces of their own at once."""
    g = gen(3)
    M, K, F = 16, 512, 1024
    blocks = [make_block(aser, g, M, K, F, K, 32, 32, "silu")[1] for _ in range(2)]
    Xs = [normal(g, M, K) for _ in range(2)]
    want = [[b(x).clone() for x in Xs] for b in blocks]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = blocks[0](Xs[0]).clone()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0][0])
    graphs, ins = [], []
    for b in blocks:
        x = Xs[0].clone()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            b(x)
        graphs.append(gr)
        ins.append(x)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(4):
        for i in range(2):
            ins[i].copy_(Xs[(rep + i) % 2])
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(blocks[i].Y, want[i][(rep + i) % 2])


def test_rows_of_zeros(aser):
    g = gen(9)
    _, block = make_block(aser, g, 20, 512, 1024, 512, 32, 32, "silu")
    X = normal(g, 20, 512)
    X[3] = 0
    Y = block(X)
    assert (Y[3] == 0).all() and torch.isfinite(Y).all()


def test_refusals(aser):
    g = gen(1)
    ops, block = make_block(aser, g, 4, 256, 512, 256, 16, 16, "silu")
    X = normal(g, 4, 256)
    with pytest.raises(TypeError):
        block(X.float())
    with pytest.raises(TypeError):
        block(X[:, ::2])
    with pytest.raises(TypeError):
        block(X.cpu())
    with pytest.raises(ValueError):
        block(normal(g, 5, 256))
    Wg, Wu, s, LA, LB, Wd, sd, LAd, LBd = ops
    for bad in ((Wg[:256].contiguous(), Wu, s, LA, LB, Wd, sd, LAd, LBd), (Wg, Wu, s, LA, None, Wd, sd, LAd, LBd),
                (Wg, Wu, s, LA, LB[:512].contiguous(), Wd, sd, LAd, LBd), (Wg, Wu, s[:128].contiguous(), LA, LB, Wd, sd, LAd, LBd),
                (Wg, Wu, s, LA[:8].contiguous(), LB[:, :8].contiguous(), Wd, sd, LAd, LBd)):
        with pytest.raises((ValueError, aser.AserError)):
            aser.AserGatedFFN(*bad, 4)
    with pytest.raises(ValueError):
        aser.AserGatedFFN(*ops, 4, activation="relu")
    f = Steps(aser, ops, 4).first
    f.quant(X)
    for rows, cols in ((3, 512), (4, 504)):
        with pytest.raises(ValueError):
            aser.linear_w4a8_lr_glu(f.Xq, f.a_scale, f.Wk, f.w_scale, f.T, f.L_B, 1024, f.ws, H=normal(g, rows, cols))
