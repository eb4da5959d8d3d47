"""A decoder layer's projections as a serving step runs them: a fused query/key/value projection with the adapters of many
requests on its column ranges, an output projection with its own, and a gated feed-forward block, planned once; and layers
of a group with more tiles than the GPU holds at once."""
import math

import pytest
import torch

from test_gpu_adapters import assert_close, expected, make
from test_gpu_ffn import assert_product_close, dequantized, Steps

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


def divisors(g, K):
    s = torch.ones(K, device="cuda")
    s[torch.randperm(K, device="cuda", generator=g)[:4]] = 9.0
    return s


class Block:
    """Heads of 128: 8 for queries, 2 for keys and values; the values stand in for attention's result."""

    def __init__(self, aser, g, M, K=1024, F=1024, slots=5):
        self.aser, self.M, self.K = aser, M, K
        s, q, kv = divisors(g, K), K, 256
        self.layers = [aser.AserLinear(normal(g, n, K, scale=1 / math.sqrt(K)), s, normal(g, 32, K, scale=0.02), normal(g, n, 32, scale=0.02), M)
                       for n in (q, kv, kv)]
        self.qkv = aser.AserSharedInputCat(self.layers, M)
        self.o = aser.AserLinear(normal(g, K, kv, scale=1 / math.sqrt(kv)), divisors(g, kv), normal(g, 16, kv, scale=0.02), normal(g, K, 16, scale=0.02), M)
        W = [normal(g, F, K, scale=1 / math.sqrt(K)) for _ in range(2)]
        self.ffn_ops = (W[0], W[1], divisors(g, K), normal(g, 32, K, scale=0.02), normal(g, 2 * F, 32, scale=0.02),
                        normal(g, K, F, scale=1 / math.sqrt(F)), divisors(g, F), normal(g, 32, F, scale=0.02), normal(g, K, 32, scale=0.02))
        self.ffn = aser.AserGatedFFN(*self.ffn_ops, M)
        self.pools = []
        for k, n, r in ((K, q, 16), (K, kv, 64), (kv, K, 128)):             # queries, values, output
            A, B, ranks, scale, _ = make(g, M, k, n, r, slots)
            self.pools.append(aser.AserAdapters(A, B, scale=scale, ranks=ranks))

    def __call__(self, X, slot, plan):
        plan.update(slot)
        q, k, v = self.qkv(X)
        self.pools[0].add(X, q, plan)
        self.pools[1].add(X, v, plan)
        h = v.contiguous()
        o = self.o(h, adapters=self.pools[2], plan=plan)
        return q, k, v, h, o, self.ffn(o)


@pytest.mark.parametrize("M", [1, 7, 16, 48, 700])
def test_a_step_of_a_decoder_layer(aser, M):
    g = gen(M)
    block = Block(aser, g, M)
    X = normal(g, M, block.K)
    slot = torch.randint(-1, 5, (M,), device="cuda", generator=g, dtype=torch.int32)
    plan = aser.AdapterPlan(slot, 5)
    q, k, v, h, o, y = [t.clone() for t in block(X, slot, plan)]
    base = [t.clone() for t in block.qkv(X)]
    assert torch.equal(k, base[1])
    for pool, x, before, after in ((block.pools[0], X, base[0], q), (block.pools[1], X, base[2], v), (block.pools[2], h, block.o(h).clone(), o)):
        ranks = pool.ranks.clamp(0, pool.r)
        assert_close(after, *expected(x, before, pool.A, pool.B, ranks, pool.scale, slot))
    steps = Steps(aser, block.ffn_ops, M)
    GU, H, want = steps(o, "silu")
    assert_product_close(H, GU[:, 0::2], GU[:, 1::2], "silu")
    assert torch.equal(want, y)

    # captured, replayed with other requests and activations; a padded batch
    graph = torch.cuda.CUDAGraph()
    x_in, slot_in = X.clone(), slot.clone()
    with torch.cuda.graph(graph):
        outs = block(x_in, slot_in, plan)
    for rep in range(3):
        x_in.copy_(normal(g, M, block.K))
        slot_in.copy_(torch.randint(-1, 6, (M,), device="cuda", generator=g))
        slot_in[M - rep:] = -1
        graph.replay()
        got = [t.clone() for t in outs]
        eager = block(x_in, slot_in, plan)
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


@pytest.mark.parametrize("M", [1, 8, 9, 16])
@pytest.mark.parametrize("N,K,r", [((14336, 14344), 512, (32, 32)), ((8192, 8192, 8200), 640, (16, 48, 0)), ((28672, 128), 128, (256, 16))])
def test_groups_of_more_tiles_than_the_gpu_holds(aser, M, N, K, r):
    """A CTA goes from one layer's tile to another's; the layers one by one have the same bits."""
    g = gen(M + K)
    s = divisors(g, K)
    layers = [aser.AserLinear(normal(g, n, K, scale=0.05), s, normal(g, max(rr, 16), K, scale=0.02)[:rr] if rr else None,
                              normal(g, n, rr, scale=0.05) if rr else None, M) for n, rr in zip(N, r)]
    for layer in layers:
        assert aser.lib.aser_linear_kernel(M, layer.N, K) == 0
    X = normal(g, M, K)
    group = aser.AserSharedInput(layers, M)
    out = [y.clone() for y in group(X)]
    for layer, y in zip(layers, out):
        assert torch.equal(layer(X), y)


# few tokens by clusters along K: two, three and four CTAs to 16 channels, whole and ragged, with every share of a low-rank term
SPLIT = [(8192, 4096, 64), (7176, 8192, 0), (8200, 4224, 256), (7168, 6144, 16), (4096, 14336, 64), (4616, 10240, 128), (4000, 11008, 0), (1024, 8192, 192),
         (8, 8192, 16), (2048, 14336, 256), (3720, 8320, 48), (40, 16384, 112)]


@pytest.mark.parametrize("M", [1, 3, 8, 9, 16])
@pytest.mark.parametrize("N,K,r", SPLIT)
def test_long_rows_of_few_tokens(aser, M, N, K, r):
    """Integer sums are exact.  Y = fp16(sum a_scale w_scale + T L_B^T) in fp32: r / 16 slices of 16 exact products, each addition
    off by at most 2^-22 of the sum of magnitudes (r / 16 + 16 of them), the scale's two products, the conversion of the sum
    and the last addition by 2^-22 together, and the store by 2^-11 or 2^-25."""
    g = gen(M + N + K)
    layer = aser.AserLinear(normal(g, N, K, scale=0.03), None, normal(g, r, K, scale=0.02) if r else None,
                            normal(g, N, r, scale=0.05) if r else None, M)
    assert aser.lib.aser_linear_kernel(M, N, K) == 0
    layer.quant(normal(g, M, K))
    acc = torch.zeros(M, N, device="cuda", dtype=torch.int32)
    layer.Y.fill_(7.0)
    layer.linear(M, acc_debug=acc)
    w = dequantized(layer) / layer.w_scale.double()[:, None].clamp_min(1e-30)
    want = layer.Xq.double() @ w.round().T
    assert torch.equal(acc.double(), want)
    ref = want * layer.a_scale.double()[:, None] * layer.w_scale.double()
    bound = 2.0 ** -22 * ref.abs()
    if r:
        T, LB = layer.T[:, :r].double(), layer.L_B.double()
        ref = ref + T @ LB.T
        bound = bound + (r / 16 + 16) * 2.0 ** -22 * (T.abs() @ LB.abs().T) + 2.0 ** -22 * ref.abs()
    bound = bound + 2.0 ** -11 * (ref.abs() + bound) + 2.0 ** -25
    assert ((layer.Y.double() - ref).abs() <= bound).all()
    again = layer.Y.clone()
    layer.linear(M)
    assert torch.equal(layer.Y, again)


@pytest.mark.parametrize("M", [2, 16])
@pytest.mark.parametrize("F,K,r,act", [(4096, 4096, 64, "silu"), (512, 8192, 32, "gelu_tanh"), (2048, 14336, 0, "silu"), (1800, 8192, 128, "silu")])
def test_product_of_long_rows(aser, M, F, K, r, act):
    g = gen(M + F)
    layer = aser.AserLinear(normal(g, 2 * F, K, scale=2.0 / math.sqrt(K)), None, normal(g, r, K, scale=0.02) if r else None,
                            normal(g, 2 * F, r, scale=0.05) if r else None, M)
    layer.quant(normal(g, M, K))
    layer.linear(M)
    H = aser.linear_w4a8_lr_glu(layer.Xq, layer.a_scale, layer.Wk, layer.w_scale, layer.T, layer.L_B, 2 * F, layer.ws, act)
    assert_product_close(H, layer.Y[:, 0::2], layer.Y[:, 1::2], act)


@pytest.mark.parametrize("M", [1, 16])
@pytest.mark.parametrize("N,K,r", [((1032, 512, 640), 8192, (32, 16, 128)), ((4096, 3208), 4096, (64, 64)), ((2048, 2048, 520), 10240, (16, 0, 256))])
def test_a_group_of_long_rows(aser, M, N, K, r):
    g = gen(M + K)
    s = divisors(g, K)
    layers = [aser.AserLinear(normal(g, n, K, scale=0.05), s, normal(g, rr, K, scale=0.02) if rr else None,
                              normal(g, n, rr, scale=0.05) if rr else None, M) for n, rr in zip(N, r)]
    X = normal(g, M, K)
    out = [y.clone() for y in aser.AserSharedInput(layers, M)(X)]
    for layer, y in zip(layers, out):
        assert torch.equal(layer(X), y)


@pytest.mark.parametrize("M,K,r", [(1, 512, 16), (20, 14336, 48), (33, 512, 32), (64, 4096, 64), (64, 28672, 32), (100, 8192, 96), (130, 1152, 16), (200, 4096, 32),
                                   (333, 2048, 64), (64, 14336, 128)])
def test_projection_of_divided_columns(aser, M, K, r):
    """T of up to a few hundred tokens, where all weight lies on columns with a divisor, kept to 16 bits as pairs.  A quotient is
    multiplied as the sum of two fp16 numbers, off by 2^-22 of it, or by 2^-25 where the second is subnormal, and quotients
    beyond fp16's range come through; K / 128 + 40 additions on a sum's longest way, each off by at most 2^-21 of the sum of magnitudes
    (truncated additions of 16 products); a pair of bf16 numbers is off by 2^-16."""
    g = gen(M + K + r)
    X = normal(g, M, K)
    cols = torch.randperm(K, device="cuda", generator=g)[:max(8, K // 100)]
    s = torch.ones(K, device="cuda")
    s[cols] = torch.exp2(8 * torch.rand(cols.numel(), device="cuda", generator=g) - 2)
    s[cols[0]] = 2.5e-3
    X[0, cols[0]] = 200.0                            # x~ = 80000
    LA = normal(g, r, K, scale=2.0 ** -6)
    rest = torch.ones(K, device="cuda", dtype=torch.bool)
    rest[cols] = False
    LA[:, rest] = 0
    xq, sc, T = aser.quant_act(X, s, LA, t_pair=True)
    t = T[:, :r].double() + T[:, r:].double()
    x = X.double() / s.double()
    ref, l1 = x @ LA.double().T, x.abs() @ LA.double().abs().T
    bound = 2.0 ** -16 * ref.abs() + (2.0 ** -22 + (K / 128 + 40) * 2.0 ** -21) * l1 + 2.0 ** -25 * LA.double().abs().sum(1)
    assert ((t - ref).abs() <= bound).all()


@pytest.mark.parametrize("M,K,r,divided", [(20, 512, 16, 9), (100, 4096, 64, 41), (450, 4096, 64, 41), (500, 8192, 192, 82), (333, 8192, 48, 128), (700, 14336, 128, 143),
                                           (1500, 4096, 256, 128), (4100, 1024, 32, 1), (129, 2048, 256, 100), (300, 128, 256, 128)])
def test_fine_projection(aser, M, K, r, divided):
    """T of any number of tokens with all weight on the divided columns: the bound of test_projection_of_divided_columns with T's one
    rounding to bf16 (2^-8).  Quotients beyond fp16's range come through.  Codes and scales are those of the plain step."""
    g = gen(M + K + r)
    X = normal(g, M, K)
    cols = torch.randperm(K, device="cuda", generator=g)[:divided]
    s = torch.ones(K, device="cuda")
    s[cols] = torch.exp2(8 * torch.rand(cols.numel(), device="cuda", generator=g) - 2)
    s[cols[0]] = 2.5e-3
    X[M - 1, cols[0]] = 200.0                        # x~ = 80000
    LA = normal(g, r, K, scale=2.0 ** -6)
    rest = torch.ones(K, device="cuda", dtype=torch.bool)
    rest[cols] = False
    LA[:, rest] = 0
    Xq, sc, T = aser.quant_act_fine(X, s, LA)
    plain = aser.quant_act(X, s, LA)
    assert torch.equal(Xq, plain[0]) and torch.equal(sc, plain[1])
    x = X.double() / s.double()
    ref, l1 = x @ LA.double().T, x.abs() @ LA.double().abs().T
    bound = 2.0 ** -8 * ref.abs() + 2 * ((2.0 ** -22 + (K / 128 + 40) * 2.0 ** -21) * l1 + 2.0 ** -25 * LA.double().abs().sum(1))
    assert ((T.double() - ref).abs() <= bound).all()
    again = aser.quant_act_fine(X, s, LA)
    assert all(torch.equal(a, b) for a, b in zip((Xq, sc, T), again))


@pytest.mark.parametrize("M,K,r,launches", [(230, 6400, 128, 2), (230, 11008, 64, 1), (230, 11008, 128, 2), (700, 2432, 128, 2), (448, 5120, 96, 2),
                                            (320, 13824, 48, 2), (1000, 1152, 128, 2), (300, 4992, 112, 2)])
def test_activation_step_of_uneven_rows(aser, M, K, r, launches):
    """Row lengths that sixteen CTAs do not share evenly go through the two kernels in a forward pass: codes and scales of the one
    launch, T from fp32 sums of the same quotients (rounded to fp16; not by the one launch up to a few hundred tokens): (K / 128 + 40) additions off by 2^-21 of the sum of magnitudes each on either
    side, and either side's rounding to bf16."""
    assert aser.forward_act_launches(M, K, r) == launches
    g = gen(M + K)
    layer = aser.AserLinear(normal(g, 128, K, scale=0.03), divisors(g, K), normal(g, r, K, scale=0.02), normal(g, 128, r, scale=0.05), M)
    X = normal(g, M, K)
    layer.quant(X)
    Xq, sc, T = aser.quant_act(X, layer.s, layer.L_A)
    assert torch.equal(layer.Xq, Xq) and torch.equal(layer.a_scale, sc)
    x16 = (X.float() / layer.s).half().double() if launches == 2 else X.double() / layer.s.double()
    ref, l1 = x16 @ layer.L_A.double().T, x16.abs() @ layer.L_A.double().abs().T
    for t in (layer.T, T):
        assert ((t.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1.01 * (K / 128 + 40) * 2.0 ** -21 * l1).all()
