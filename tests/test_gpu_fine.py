"""The fine activation step where a slice of K has more divided columns than its kernel gathers."""
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


# (tokens, K, r, divided columns, those of the first columns alone): whole rows; slices with and without a second turn side by side, one column
# beyond what is gathered; more units of eight columns than the divisors' cache holds; both kernels behind it, one to two groups of L_A
MANY = [(450, 4096, 64, 4096, False), (600, 14336, 64, 5000, False), (700, 512, 192, 512, False), (4100, 1024, 32, 1024, False),
        (129, 2048, 256, 2048, False), (500, 8192, 256, 900, True), (450, 4096, 64, 300, True), (333, 8192, 48, 1024, True),
        (4100, 14336, 16, 14336, False), (600, 256, 32, 129, True), (513, 4096, 256, 700, True), (300, 256, 16, 256, False), (40, 4992, 144, 4992, False)]


@pytest.mark.parametrize("M,K,r,divided,first", MANY)
def test_many_divided_columns(aser, M, K, r, divided, first):
    """All weight on the divided columns, quotients beyond fp16's range among them.  A quotient is multiplied as the sum of two fp16
    numbers, off by 2^-22 of it, or by 2^-25 where the second is subnormal; K / 128 + 40 additions on a sum's longest way (the second
    numbers' are of sums 2^-11 as large), each off by at most 2^-21 of the sum of magnitudes; T is rounded once to bf16 (2^-8 of it, which
    the factor 2 on the other terms covers).  Codes and scales are those of the plain step, and a second call has the same bits."""
    g = gen(M + K + r)
    X = normal(g, M, K)
    cols = torch.arange(divided, device="cuda") if first else torch.randperm(K, device="cuda", generator=g)[:divided]
    s = torch.ones(K, device="cuda")
    s[cols] = torch.exp2(8 * torch.rand(divided, device="cuda", generator=g) - 2)
    s[cols[0]], s[cols[-1]] = 2.5e-3, -2e-3
    X[M - 1, cols[0]] = 200.0                        # x~ = 80000
    X[0, cols[-1]] = 200.0                           # x~ = -100000
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
    bad = ~((T.double() - ref).abs() <= bound)
    assert not bad.any(), "%d wrong, worst error / bound %.3f" % (int(bad.sum()), float(((T.double() - ref).abs() / bound).max()))
    again = aser.quant_act_fine(X, s, LA)
    assert all(torch.equal(a, b) for a, b in zip((Xq, sc, T), again))


@pytest.mark.parametrize("M,K,r", [(4096, 4096, 128), (1000, 8192, 64), (600, 14336, 96), (1500, 2048, 256)])
def test_few_values_a_step_off(aser, M, K, r):
    """T is the rounded exact sum but where the sum's own error carries it over the middle between two bf16 numbers: seldomer than for a
    product in fp32, whose additions are rounded one by one."""
    g = gen(M + K)
    X, LA = normal(g, M, K), normal(g, r, K, scale=0.02)
    s = torch.ones(K, device="cuda")
    s[torch.randperm(K, device="cuda", generator=g)[:K // 100]] = 7.0
    exact = ((X.double() / s.double()) @ LA.double().T).to(torch.bfloat16)
    assert not torch.backends.cuda.matmul.allow_tf32
    plain = ((X.float() / s) @ LA.float().T).to(torch.bfloat16)
    T = aser.quant_act_fine(X, s, LA)[2]
    off, off_plain = int((T != exact).sum()), int((plain != exact).sum())
    assert off <= off_plain, "%d of %d values off, of a product in fp32 %d" % (off, T.numel(), off_plain)
