"""Adapters whose X lies under what the call writes: refused before anything is launched; matrices beside each other are not."""
import ctypes as C

import pytest
import torch

SHAPE = -3
BASE = 0x100000


@pytest.fixture(scope="module")
def lib():
    from paper_2411_07762_b200 import build
    build.build()
    from paper_2411_07762_b200 import binding
    return binding.lib


GOOD = C.c_void_p(0x90000000)


@pytest.mark.parametrize("x,y,out,ldx,ldy,ldo", [
    (0, 0, 0, 256, 64, 64),                 # X is what is updated
    (0, 1024, 1024, 256, 64, 64),           # ... begins inside X
    (128, 0, 0, 256, 64, 64),               # X begins inside it
    (0, 4096, 240, 320, 320, 320),          # column ranges of one matrix that share columns 240 .. 255
    (0, 4096, 320 - 32, 320, 320, 320),     # ... that reach into the next row of X
    (0, 8192, 248, 256, 64, 64),            # the last element of the first row
    (8192, 0, 32, 256, 64, 64),             # Y and out overlap, X lies elsewhere
    (8192, 0, 64, 256, 128, 136),           # ... at distances of their own
])
def test_overlaps_are_refused(lib, x, y, out, ldx, ldy, ldo):
    at = lambda e: C.c_void_p(BASE + 2 * e)
    rc = lib.aser_adapters_add(at(x), ldx, GOOD, GOOD, None, None, GOOD, 1 << 20, 8, 64, 256, 16, 4, at(y), ldy, at(out), ldo, None, 0, None)
    assert rc == SHAPE and b"overlap" in lib.aser_last_error()


@pytest.mark.parametrize("x,y", [(0, 0), (0, 1000), (200, 0)])
def test_a_layer_over_its_input_is_refused(lib, x, y):
    """(the layer itself is checked first: with a bad workspace that is what is said)"""
    at = lambda e: C.c_void_p(BASE + 2 * e - 2 * e % 16)
    call = lambda ws: lib.aser_forward_adapters(at(x), None, GOOD, GOOD, GOOD, GOOD, 8, 64, 256, 16, GOOD, GOOD, GOOD, at(y), ws, 1 << 26, GOOD, GOOD,
                                                None, None, GOOD, 1 << 20, 16, 4, None, 0, None)
    assert call(None) == -4
    if torch.cuda.is_available():
        assert call(GOOD) == SHAPE and b"overlap" in lib.aser_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 600])
def test_columns_beside_each_other(lib, M):
    """X, Y and out as column ranges of one matrix; a layer on its own output."""
    import paper_2411_07762_b200 as aser
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    normal = lambda *shape, scale=1.0: torch.randn(*shape, device="cuda", dtype=torch.float16, generator=g) * scale
    K = N = 256
    pool = aser.AserAdapters(normal(3, 32, K, scale=0.05), normal(3, N, 32, scale=0.05))
    plan = pool.plan(torch.randint(-1, 3, (M,), device="cuda", generator=g, dtype=torch.int32))
    wide = normal(M, 3 * K)
    X, Y, out = wide[:, :K], wide[:, K:2 * K], wide[:, 2 * K:]
    want = pool.add(X.contiguous(), Y.contiguous(), plan)
    assert torch.equal(pool.add(X, Y, plan, out=out), want)
    for bad_out in (wide[:, 8:8 + K], wide[:, K + 8:2 * K + 8]):
        with pytest.raises(aser.AserError):
            pool.add(X, Y, plan, out=bad_out)
    layer = aser.AserLinear(normal(N, K, scale=0.06), None, None, None, M)
    own = layer(X.contiguous(), adapters=pool, plan=plan)
    first = own.clone()
    with pytest.raises(aser.AserError):
        layer(own, adapters=pool, plan=plan)
    assert torch.equal(own, first)
    second = layer(first, adapters=pool, plan=plan).clone()
    assert torch.equal(second, pool.add(first, layer(first), plan))
