"""Low-rank adapters of many requests on the GPU against 64 bits: sizes, ranks, strides, tokens without an adapter, values out
of range, plans, graphs and refusals."""
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


def expected(X, Y, A, B, ranks, scale, slot):
    """The update in 64 bits, and how far the kernel may be from it, element by element:
      * S = A x in fp32: the products of two fp16 numbers are exact; K / 128 + 32 additions on a sum's longest way (an
        instruction adds 16 products, 8 warps and more share K, then their sums are added), each off by at most 2^-22 of the
        sum of magnitudes (a truncated addition in the tensor cores);
      * S to fp16: 2^-11 of each entry, or 2^-25 2^(e - 14) <= 2^-38 of the token's largest below the normal range;
      * B S in fp32: r / 16 + 8 additions, as above; the factor and the final addition 2^-22 of the update and Y;
      * the result to fp16: 2^-11, or 2^-25 below the normal range."""
    K = X.shape[1]
    ref = Y.double().clone()
    bound = torch.zeros_like(ref)
    for a in sorted(set(slot.tolist())):
        if not 0 <= a < A.shape[0]:
            continue
        r = int(ranks[a])
        if r == 0:
            continue
        rows = (slot == a).nonzero().flatten()
        x, aa, bb = X[rows].double(), A[a, :r].double(), B[a, :, :r].double()
        s = x @ aa.T
        l1 = x.abs() @ aa.abs().T
        ds = (K / 128 + 32) * 2.0 ** -22 * l1 + 2.0 ** -11 * s.abs() + 2.0 ** -38 * s.abs().amax(1, keepdim=True)
        f = abs(float(scale[a]))
        ref[rows] += float(scale[a]) * (s @ bb.T)
        bound[rows] = f * (ds @ bb.abs().T + (r / 16 + 8 + 1) * 2.0 ** -22 * (s.abs() @ bb.abs().T)) * (1 + 2.0 ** -9) \
            + 2.0 ** -22 * Y[rows].double().abs()
        bound[rows] += 2.0 ** -11 * (ref[rows].abs() + bound[rows]) + 2.0 ** -25
    return ref, bound


def assert_close(out, ref, bound):
    err = (out.double() - ref).abs()
    bad = ~(err <= bound)
    assert not bad.any(), "%d wrong, worst error / bound %.3f" % (int(bad.sum()), float((err / bound.clamp_min(1e-30)).max()))


def make(g, M, K, N, r, slots, bare=0.2, spread=True):
    A, B = normal(g, slots, r, K, scale=0.05), normal(g, slots, N, r, scale=0.05)
    ranks = torch.randint(0, r // 16 + 1, (slots,), device="cuda", generator=g, dtype=torch.int32) * 16 if spread else \
        torch.full((slots,), r, device="cuda", dtype=torch.int32)
    for a in range(slots):                          # what lies behind an adapter's rank is not read
        A[a, int(ranks[a]):] = float("nan")
        B[a, :, int(ranks[a]):] = float("nan")
    scale = torch.randn(slots, device="cuda", generator=g)
    slot = torch.randint(0, slots, (M,), device="cuda", generator=g, dtype=torch.int32)
    none = torch.rand(M, device="cuda", generator=g) < bare
    slot[none] = torch.where(torch.rand(int(none.sum()), device="cuda", generator=g) < 0.5, -1, slots + 5).int()
    return A, B, ranks, scale, slot


def launches_two(aser, M, K, N, r, slots):
    return aser.lib.aser_adapters_workspace_bytes(M, N, K, r, slots) > 0


# one token to many, odd sizes, every number of 16-rank steps' remainder, one adapter to more than there are tokens
SHAPES = [(1, 128, 8, 16, 1), (1, 4096, 4096, 16, 8), (1, 640, 264, 256, 3), (2, 256, 40, 32, 70), (5, 1152, 1000, 48, 4), (16, 512, 512, 64, 1),
          (17, 128, 24, 16, 2), (33, 4096, 1024, 80, 5), (64, 2048, 4104, 128, 40), (100, 384, 88, 112, 300), (130, 14336, 72, 64, 3),
          (257, 1024, 2056, 32, 2), (501, 512, 8, 256, 6), (1000, 640, 1032, 48, 1), (1025, 256, 264, 16, 4096), (2050, 1024, 520, 144, 3),
          (33, 4096, 4096, 128, 1), (700, 512, 1024, 256, 2), (4100, 128, 64, 16, 9)]


@pytest.mark.parametrize("bare,spread", [(0.2, True), (0.0, False)])
@pytest.mark.parametrize("M,K,N,r,slots", SHAPES)
def test_update(aser, M, K, N, r, slots, bare, spread):
    g = gen(M + K + N + r)
    A, B, ranks, scale, slot = make(g, M, K, N, r, slots, bare, spread)
    X, Y = normal(g, M, K), normal(g, M, N)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    plan = pool.plan(slot)
    ref, bound = expected(X, Y, A, B, ranks, scale, slot)
    out = torch.full((M + 1, N), 7.0, device="cuda", dtype=torch.float16)
    pool.add(X, Y, plan, out=out[:M])
    assert_close(out[:M], ref, bound)
    assert (out[M] == 7.0).all()                    # the row behind the last token
    again = torch.empty_like(Y)
    assert torch.equal(pool.add(X, Y, plan, out=again), out[:M])
    inplace = Y.clone()
    assert pool.add(X, inplace, plan) is inplace
    assert torch.equal(inplace, out[:M])
    idle = (slot < 0) | (slot >= slots)
    assert torch.equal(inplace[idle], Y[idle])


# prompts: runs of tokens that follow one another, of lengths around the tiles' and the copies' sizes, with adapters of many ranks
RUNS = [(200, 14336, 72, 64, (128, 72)), (300, 128, 16384, 32, (255, 45)), (1021, 1024, 136, 128, (127, 1, 129, 33, 500, 31, 200)), (640, 4096, 512, 256, (320, 320)),
        (900, 256, 4104, 16, (32, 96, 64, 700, 8)), (1500, 14336, 200, 96, (1, 2, 3, 1494)), (2500, 512, 1032, 48, (1250, 1250)), (600, 14336, 264, 256, (333, 267)),
        (390, 7680, 520, 144, (129, 128, 133))]


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("M,K,N,r,lengths", RUNS)
def test_prompts(aser, M, K, N, r, lengths, mixed):
    """Tokens that follow one another and the same ones scattered; rows of X, Y and out apart from one another."""
    assert launches_two(aser, M, K, N, r, len(lengths))
    g = gen(M + r)
    A, B, ranks, scale, _ = make(g, M, K, N, r, len(lengths), spread=False)
    ranks[1::2] = torch.tensor([max(16, r // 32 * 16)], device="cuda", dtype=torch.int32)
    slot = torch.cat([torch.full((n,), a, device="cuda", dtype=torch.int32) for a, n in enumerate(lengths)])
    slot = torch.cat([slot[:M // 2], torch.full((M - slot.numel(),), -1, device="cuda", dtype=torch.int32), slot[M // 2:]])
    if mixed:
        slot = slot[torch.randperm(M, device="cuda", generator=g)].contiguous()
    X = normal(g, M, K + 8)[:, :K]
    wide = normal(g, M, 2 * N + 16)
    Y = wide[:, 8:8 + N]
    keep = wide.clone()
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    plan = pool.plan(slot)
    ref, bound = expected(X, Y, A, B, ranks, scale, slot)
    guard = torch.full((M + 2, N + 24), 5.0, device="cuda", dtype=torch.float16)
    out = guard[1:M + 1, 16:16 + N]
    pool.add(X, Y, plan, out=out)
    assert_close(out, ref, bound)
    assert torch.equal(wide, keep)
    pool.add(X, Y, plan)
    assert torch.equal(Y, out)
    wide[:, 8:8 + N] = keep[:, 8:8 + N]
    assert torch.equal(wide, keep)                  # nothing beside the range
    out.fill_(5.0)
    assert (guard == 5.0).all()


def test_prompts_on_two_streams_and_in_a_graph(aser):
    """One pool and one plan from two streams at once, and captured; every call has a workspace of its own."""
    g = gen(31)
    M, K, N, r = 1200, 2048, 1024, 64
    assert launches_two(aser, M, K, N, r, 4)
    A, B, ranks, scale, slot = make(g, M, K, N, r, 4)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    plan = pool.plan(slot)
    Xs, Ys = [normal(g, M, K) for _ in range(2)], [normal(g, M, N) for _ in range(2)]
    want = [pool.add(x, y, plan, out=torch.empty_like(y)) for x, y in zip(Xs, Ys)]
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(y) for y in Ys]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                pool.add(Xs[i], Ys[i], plan, out=outs[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    x, y = Xs[0].clone(), Ys[0].clone()
    with torch.cuda.graph(graph):
        pool.add(x, y, plan, out=outs[0])
    for i in (1, 0, 1):
        x.copy_(Xs[i])
        y.copy_(Ys[i])
        graph.replay()
        assert torch.equal(outs[0], want[i])


def test_defaults_and_layout(aser):
    """No ranks, no factors; X, Y and out as column ranges of wider matrices, what lies beside them left alone."""
    g = gen(2)
    M, K, N, r, slots = 75, 512, 384, 32, 4
    A, B, _, _, slot = make(g, M, K, N, r, slots, spread=False)
    wide_x, wide_y = normal(g, M, K + 64), normal(g, M, 3 * N)
    X, Y = wide_x[:, 8:8 + K], wide_y[:, N:2 * N]
    keep = wide_y.clone()
    pool = aser.AserAdapters(A, B)
    ones = torch.ones(slots, device="cuda")
    ref, bound = expected(X, Y, A, B, torch.full((slots,), r), ones, slot)
    pool.add(X, Y, pool.plan(slot))
    assert_close(wide_y[:, N:2 * N], ref, bound)
    assert torch.equal(wide_y[:, :N], keep[:, :N]) and torch.equal(wide_y[:, 2 * N:], keep[:, 2 * N:])


@pytest.mark.parametrize("M", [3, 200])
def test_token_order_does_not_matter(aser, M):
    """A token's result depends on its own row and adapter only."""
    g = gen(M)
    A, B, ranks, scale, slot = make(g, M, 512, 264, 48, 5)
    X, Y = normal(g, M, 512), normal(g, M, 264)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    out = pool.add(X, Y, pool.plan(slot), out=torch.empty_like(Y))
    p = torch.randperm(M, device="cuda", generator=g)
    out2 = pool.add(X[p].contiguous(), Y[p].contiguous(), pool.plan(slot[p].contiguous()), out=torch.empty_like(Y))
    assert torch.equal(out2, out[p])


@pytest.mark.parametrize("M", [4, 300])
def test_values_out_of_range(aser, M):
    """S beyond fp16 on both sides, and rows with infinities and NaN that leave every other row alone."""
    g = gen(M + 1)
    K, N, r, slots = 512, 128, 32, 3
    A, B, ranks, scale, slot = make(g, M, K, N, r, slots, bare=0.0, spread=False)
    slot[:3] = torch.tensor([0, 1, 2], device="cuda")
    A[0] *= 1000.0                                  # S of about 1e6 ...
    B[0] *= 1e-3                                    # (subnormal entries of B, too)
    scale[0] = 1e-3
    A[1] *= 2.0 ** -14                              # ... and of about 1e-4
    B[1] *= 1000.0
    X, Y = normal(g, M, K), normal(g, M, N)
    X[slot == 0] *= 100.0
    ref, bound = expected(X, Y, A, B, ranks, scale, slot)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    plan = pool.plan(slot)
    assert_close(pool.add(X, Y, plan, out=torch.empty_like(Y)), ref, bound)
    clean = pool.add(X, Y, plan, out=torch.empty_like(Y))
    X[M - 1, 5] = float("nan")
    X[M - 2, 7] = float("inf")
    X[0] = 0.0
    out = pool.add(X, Y, plan, out=torch.empty_like(Y))
    assert torch.equal(out[1:M - 2], clean[1:M - 2]) and torch.equal(out[0], Y[0])
    assert out[M - 1].isnan().all() and not torch.isfinite(out[M - 2]).any()


def test_unused_adapters_are_not_read(aser):
    g = gen(4)
    A, B, ranks, scale, slot = make(g, 40, 256, 64, 16, 6, spread=False)
    slot[slot == 2] = 1
    A[2] = float("nan")
    B[2] = float("inf")
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    assert torch.isfinite(pool.add(normal(g, 40, 256), normal(g, 40, 64), pool.plan(slot))).all()


def test_ranks_that_are_no_ranks(aser):
    """Ranks are taken down to multiples of 16 between 0 and r."""
    g = gen(6)
    A, B, _, scale, slot = make(g, 30, 256, 64, 32, 5, bare=0.0, spread=False)
    X, Y = normal(g, 30, 256), normal(g, 30, 64)
    odd = aser.AserAdapters(A, B, scale=scale, ranks=torch.tensor([-3, 15, 31, 33, 1000], device="cuda", dtype=torch.int32))
    even = aser.AserAdapters(A, B, scale=scale, ranks=torch.tensor([0, 0, 16, 32, 32], device="cuda", dtype=torch.int32))
    plan = odd.plan(slot)
    assert torch.equal(odd.add(X, Y, plan, out=torch.empty_like(Y)), even.add(X, Y, plan, out=torch.empty_like(Y)))


def read_plan(plan):
    w = plan.data.view(torch.int32).cpu()
    M, S = plan.M, plan.n_slots
    head, at, tiles = w[:5].tolist(), 8, []
    for size, words, n in ((16, 20, head[2]), (128, 4, head[3])):
        bound = M // size + min(S + 1, M)
        assert n <= bound
        tiles.append(w[at:at + words * n].reshape(-1, words).tolist())
        at += words * bound
    return head, tiles, w[at:at + M].tolist()


@pytest.mark.parametrize("M,slots", [(1, 1), (1, 4096), (31, 2), (1024, 7), (1025, 1), (3000, 50), (5000, 4096), (4096, 1500)])
def test_plan(aser, M, slots):
    g = gen(M + slots)
    slot = torch.randint(-2, slots + 2, (M,), device="cuda", generator=g, dtype=torch.int32)
    head, tiles, tokens = read_plan(aser.AdapterPlan(slot, slots))
    s = [a if 0 <= a < slots else -1 for a in slot.tolist()]
    want = sorted(range(M), key=lambda m: (s[m] if s[m] >= 0 else slots, m))
    assert head[:2] == [M, slots] and tokens == want
    assert head[4] == sum(a >= 0 for a, *_ in tiles[1])
    for size, ts in zip((16, 128), tiles):
        at = 0
        for a, first, count, run, *own in ts:
            assert first == at and 1 <= count <= size and all(s[m] == a for m in tokens[first:first + count])
            assert not own or own[:count] == tokens[first:first + count]
            mine = tokens[first:first + count]
            assert own or run == (mine[0] if mine == list(range(mine[0], mine[0] + count)) else -1)
            at += count
        assert at == M


def test_projection_with_adapters(aser):
    """The whole call has the bits of its two steps; without a low-rank term, and with fewer tokens than the layer holds."""
    g = gen(8)
    K, N = 1024, 520
    layer = aser.AserLinear(normal(g, N, K, scale=0.03), None, normal(g, 32, K, scale=0.02), normal(g, N, 32, scale=0.02), 600)
    for M in (1, 16, 40, 600):
        A, B, ranks, scale, slot = make(g, M, K, N, 32, 4)
        pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
        plan = pool.plan(slot)
        X = normal(g, M, K)
        for lowrank in (True, False):
            base = layer(X, lowrank=lowrank).clone()
            want = pool.add(X, base, plan)
            assert torch.equal(layer(X, lowrank=lowrank, adapters=pool, plan=plan), want)


def test_graph_follows_the_slots(aser):
    """A captured step that plans and adds, replayed with other slots and inputs; a padded batch; another stream beside it."""
    g = gen(12)
    M, K, N, slots = 48, 512, 264, 6
    A, B, ranks, scale, slot = make(g, M, K, N, 32, slots, spread=False)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    X, Y, out = normal(g, M, K), normal(g, M, N), torch.empty(M, N, device="cuda", dtype=torch.float16)
    plan = pool.plan(slot)
    pool.add(X, Y, plan, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.update(slot)
        pool.add(X, Y, plan, out=out)
    other = torch.cuda.Stream()
    out_b = torch.empty_like(out)
    for rep in range(5):
        slot.copy_(torch.randint(-1, slots, (M,), device="cuda", generator=g))
        slot[M - 3 * rep:] = -1                     # padding
        X.copy_(normal(g, M, K))
        plan_b = pool.plan(slot)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(other):
            pool.add(X, Y, plan_b, out=out_b)
        torch.cuda.synchronize()
        assert_close(out, *expected(X, Y, A, B, ranks, scale, slot))
        assert torch.equal(out, out_b)


def test_refusals(aser):
    g = gen(1)
    A, B, ranks, scale, slot = make(g, 8, 256, 64, 16, 3)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    plan = pool.plan(slot)
    X, Y = normal(g, 8, 256), normal(g, 8, 64)
    for bad in ((X[:, :128], Y), (X.float(), Y), (X, Y.cpu()), (X, Y[:7]), (X[:1].expand(8, 256), Y), (X, Y[:1].expand(8, 64)),
                (X.T.contiguous().T, Y)):
        with pytest.raises(TypeError):
            pool.add(bad[0], bad[1], plan)
    with pytest.raises(ValueError):
        pool.add(X[:7], Y[:7], plan)
    with pytest.raises(ValueError):
        pool.add(X, Y, aser.AdapterPlan(slot, 4))
    with pytest.raises(ValueError):
        pool.add(X, Y, None)
    with pytest.raises(aser.AserError):
        pool.add(X, normal(g, 8, 68)[:, :64], plan)          # rows 68 elements apart
    with pytest.raises(TypeError):
        pool.plan(slot.long())
    with pytest.raises(ValueError):
        plan.update(slot[:5])
    for args in ((A, B[:2].contiguous()), (A[0], B[0]), (A, B, scale[:2].contiguous())):
        with pytest.raises(ValueError):
            aser.AserAdapters(*args)
    with pytest.raises(TypeError):
        aser.AserAdapters(A.float(), B)
    layer = aser.AserLinear(normal(g, 128, 256, scale=0.03), None, None, None, 8)
    with pytest.raises(ValueError):
        layer(X, adapters=pool, plan=plan)                   # another number of channels
    with pytest.raises(ValueError):
        layer(X, plan=plan)


@pytest.mark.parametrize("M", [1, 20, 300, 3000])
def test_no_rank(aser, M):
    """A pool of rank 0 copies, or leaves alone."""
    g = gen(M)
    pool = aser.AserAdapters(torch.empty(3, 0, 256, device="cuda", dtype=torch.float16), torch.empty(3, 136, 0, device="cuda", dtype=torch.float16))
    X, Y = normal(g, M, 256), normal(g, M, 136)
    plan = pool.plan(torch.randint(-1, 3, (M,), device="cuda", generator=g, dtype=torch.int32))
    out = torch.full((M + 1, 136), 7.0, device="cuda", dtype=torch.float16)
    assert torch.equal(pool.add(X, Y, plan, out=out[:M]), Y) and (out[M] == 7.0).all()
    keep = Y.clone()
    assert torch.equal(pool.add(X, Y, plan), keep)


@pytest.mark.parametrize("M", [40, 1500])
def test_no_token_has_an_adapter(aser, M):
    """Nor a rank: with other adapters' tokens in the next call, one call after the other on a stream."""
    g = gen(M)
    A, B, ranks, scale, slot = make(g, M, 1024, 1032, 32, 3, spread=False)
    X, Y = normal(g, M, 1024), normal(g, M, 1032)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    ref, bound = expected(X, Y, A, B, ranks, scale, slot)
    none, some = torch.full_like(slot, -1), slot.clone()
    empty = aser.AserAdapters(A, B, scale=scale, ranks=torch.zeros_like(ranks))
    plan = pool.plan(none)
    for rep in range(3):
        out = torch.full_like(Y, 3.0)
        plan.update(none)
        assert torch.equal(pool.add(X, Y, plan, out=out), Y)
        plan.update(some)
        assert torch.equal(empty.add(X, Y, plan, out=out), Y)
        assert_close(pool.add(X, Y, plan, out=out), ref, bound)


def test_no_tokens(aser):
    g = gen(1)
    A, B, ranks, scale, _ = make(g, 8, 256, 64, 16, 3)
    pool = aser.AserAdapters(A, B, scale=scale, ranks=ranks)
    none = torch.empty(0, device="cuda", dtype=torch.int32)
    Y = torch.empty(0, 64, device="cuda", dtype=torch.float16)
    assert pool.add(torch.empty(0, 256, device="cuda", dtype=torch.float16), Y, pool.plan(none)).shape == (0, 64)


def test_far_offsets(aser):
    """Rows, adapters and results beyond 2^31 elements of their tensors' starts."""
    g = gen(21)
    K, N, r, slots = 32768, 32768, 64, 1100                 # A and B: 2.3e9 elements each
    A = torch.zeros(slots, r, K, device="cuda", dtype=torch.float16)
    B = torch.zeros(slots, N, r, device="cuda", dtype=torch.float16)
    last = slots - 1
    A[last], B[last] = normal(g, r, K, scale=0.02), normal(g, N, r, scale=0.02)
    slot = torch.tensor([last, -1, 0], device="cuda", dtype=torch.int32)
    X, Y = normal(g, 3, K), normal(g, 3, N)
    pool = aser.AserAdapters(A, B)
    out = pool.add(X, Y, pool.plan(slot), out=torch.empty_like(Y))
    ref, bound = expected(X, Y, A[last:], B[last:], [r], [1.0], torch.where(slot == last, 0, -1))
    assert_close(out[:1], ref[:1], bound[:1])
    assert torch.equal(out[1:], Y[1:])
    del A, B, pool
    # 70000 rows of 32768: the last row starts at 2.3e9
    M = 70000
    X, Y = torch.zeros(M, 128, device="cuda", dtype=torch.float16), torch.zeros(M, N, device="cuda", dtype=torch.float16)
    X[M - 1] = normal(g, 128)
    A, B = normal(g, 2, 16, 128, scale=0.1), normal(g, 2, N, 16, scale=0.1)
    slot = torch.full((M,), -1, device="cuda", dtype=torch.int32)
    slot[M - 1], slot[0] = 1, 0
    pool = aser.AserAdapters(A, B)
    pool.add(X, Y, pool.plan(slot))
    ref, bound = expected(X[M - 1:], torch.zeros_like(Y[:1]), A, B, [16, 16], [1.0, 1.0], slot[M - 1:])
    assert_close(Y[M - 1:], ref, bound)
    assert (Y[:M - 1] == 0).all()
