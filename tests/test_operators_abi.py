"""Refusals of the entry points for feed-forward blocks and adapters: bad arguments are rejected with an error code before
anything is launched (no GPU needed)."""
import ctypes as C

import pytest

OK, NULL, ALIGN, SHAPE, WORKSPACE = 0, -1, -2, -3, -4
GOOD, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)


@pytest.fixture(scope="module")
def lib():
    from paper_2411_07762_b200 import build
    build.build()
    from paper_2411_07762_b200 import binding
    return binding.lib


def test_gated_linear_is_refused(lib):
    def call(M=4, N=256, K=128, r=16, act=0, Xq=GOOD, T=GOOD, LB=GOOD, H=GOOD, ws=GOOD, nbytes=1 << 26):
        return lib.aser_linear_w4a8_lr_glu(Xq, GOOD, GOOD, GOOD, T, LB, M, N, K, r, act, H, ws, nbytes, None)
    assert call(M=0, Xq=None, ws=None) == OK
    assert call(N=264) == SHAPE and call(K=100) == SHAPE and call(r=8) == SHAPE and call(r=272) == SHAPE and call(M=-1) == SHAPE
    assert call(act=2) == SHAPE and call(act=-1) == SHAPE
    assert call(Xq=None) == NULL and call(T=None) == NULL and call(LB=None) == NULL and call(H=None) == NULL
    assert call(H=ODD) == ALIGN
    assert call(ws=None) == WORKSPACE and call(nbytes=1000) == WORKSPACE and call(ws=ODD) == WORKSPACE


def test_fine_activation_step_is_refused(lib):
    def call(M=40, K=256, r=16, X=GOOD, s=GOOD, LA=GOOD, Xq=GOOD, T=GOOD, ws=GOOD, nbytes=1 << 26):
        return lib.aser_quant_act_fine(X, s, LA, M, K, r, Xq, GOOD, T, ws, nbytes, None)
    assert call(M=0, X=None, ws=None) == OK
    assert call(K=200) == SHAPE and call(r=24) == SHAPE and call(r=272) == SHAPE and call(M=-1) == SHAPE
    assert call(X=None) == NULL and call(LA=None) == NULL and call(T=None) == NULL and call(Xq=None) == NULL and call(s=ODD) == ALIGN
    assert call(ws=None) == WORKSPACE and call(nbytes=1000) == WORKSPACE


def test_feed_forward_is_refused(lib):
    def call(M=4, K=128, F=256, N=128, r=16, rd=16, act=0, X=GOOD, LA=GOOD, LAd=GOOD, sd=None, Y=GOOD, ws=GOOD, nbytes=1 << 26):
        return lib.aser_forward_ffn(X, None, LA, GOOD, GOOD, GOOD, sd, LAd, GOOD, GOOD, GOOD, M, K, F, N, r, rd, act, Y, ws,
                                    nbytes, None)
    assert call(M=0, X=None, ws=None) == OK
    assert call(F=200) == SHAPE and call(K=130) == SHAPE and call(N=4) == SHAPE and call(rd=24) == SHAPE and call(F=0) == SHAPE
    assert call(act=7) == SHAPE and call(M=-2) == SHAPE and call(F=-128) == SHAPE
    assert call(X=None) == NULL and call(LA=None) == NULL and call(LAd=None) == NULL and call(Y=None) == NULL
    assert call(sd=ODD) == ALIGN and call(Y=ODD) == ALIGN
    need = lib.aser_forward_ffn_workspace_bytes(4, 128, 256, 128, 16, 16)
    assert need > 0 and call(nbytes=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE
    assert lib.aser_forward_ffn_workspace_bytes(4, 128, 200, 128, 16, 16) == 0
    assert lib.aser_forward_ffn_workspace_bytes(4, 128, 256, 128, 16, 17) == 0


@pytest.mark.parametrize("K,F,N,r,rd", [(4096, 14336, 4096, 64, 64), (512, 1024, 512, 256, 16), (128, 128, 8, 0, 256), (1024, 512, 64, 0, 0)])
def test_a_workspace_serves_fewer_tokens(lib, K, F, N, r, rd):
    need = [lib.aser_forward_ffn_workspace_bytes(m, K, F, N, r, rd) for m in range(1, 2100)]
    assert all(a <= b for a, b in zip(need, need[1:]))


def test_adapter_plan_is_refused(lib):
    assert lib.aser_adapters_plan_bytes(-1, 4) == 0 and lib.aser_adapters_plan_bytes(8, 0) == 0
    assert lib.aser_adapters_plan_bytes(8, 4097) == 0 and lib.aser_adapters_plan_bytes((1 << 24) + 1, 4) == 0
    need = lib.aser_adapters_plan_bytes(8, 4)
    assert need >= 4 * (4 + 8)
    call = lambda slot=GOOD, M=8, S=4, plan=GOOD, nbytes=need: lib.aser_adapters_plan(slot, M, S, plan, nbytes, None)
    assert call(M=0, slot=None, plan=None, nbytes=0) == OK
    assert call(S=0) == SHAPE and call(M=-1) == SHAPE and call(S=5000) == SHAPE
    assert call(slot=None) == NULL and call(plan=None) == NULL and call(plan=ODD) == ALIGN
    assert call(nbytes=need - 1) == WORKSPACE


def test_adapters_are_refused(lib):
    def call(M=8, N=64, K=256, r=16, S=4, X=GOOD, A=GOOD, B=GOOD, ranks=None, plan=GOOD, nbytes=1 << 20, Y=GOOD, out=GOOD, ldx=0,
             ldy=0, ldo=0, ws=GOOD, wbytes=1 << 20):
        return lib.aser_adapters_add(X, ldx, A, B, ranks, None, plan, nbytes, M, N, K, r, S, Y, ldy, out, ldo, ws, wbytes,
                                     None)
    assert call(M=0, X=None, plan=None, nbytes=0) == OK and call(N=0, Y=None) == OK
    assert call(K=200) == SHAPE and call(N=60) == SHAPE and call(r=24) == SHAPE and call(r=272) == SHAPE and call(M=-1) == SHAPE
    assert call(M=(1 << 24) + 1) == SHAPE and call(S=0) == SHAPE and call(S=4097) == SHAPE
    assert call(N=1 << 20, S=2048) == SHAPE
    assert call(ldx=128) == SHAPE and call(ldx=260) == SHAPE and call(ldy=68, ldo=68) == SHAPE and call(ldo=56) == SHAPE
    assert call(ldy=128) == SHAPE                   # in place, rows of one matrix
    assert call(X=None) == NULL and call(A=None) == NULL and call(B=None) == NULL and call(plan=None) == NULL
    assert call(Y=None) == NULL and call(out=None) == NULL and call(ranks=ODD) == ALIGN and call(out=ODD) == ALIGN
    assert call(nbytes=lib.aser_adapters_plan_bytes(8, 4) - 1) == WORKSPACE
    need = lib.aser_adapters_workspace_bytes(5000, 64, 256, 16, 4)
    assert need == 5000 * (2 * 16 + 4) and lib.aser_adapters_workspace_bytes(32, 64, 256, 16, 1) == 0
    assert lib.aser_adapters_workspace_bytes(5000, 64, 256, 24, 4) == 0 and lib.aser_adapters_workspace_bytes(-1, 64, 256, 16, 4) == 0
    assert call(M=5000, ws=None) == WORKSPACE and call(M=5000, wbytes=need - 1) == WORKSPACE and call(M=5000, ws=ODD) == WORKSPACE


def test_projection_with_adapters_is_refused(lib):
    def call(M=8, N=64, K=256, r=16, ra=16, X=GOOD, LA=GOOD, Y=GOOD, ws=GOOD, A=GOOD, plan=GOOD, nbytes=1 << 20):
        return lib.aser_forward_adapters(X, None, LA, GOOD, GOOD, GOOD, M, N, K, r, GOOD, GOOD, GOOD, Y, ws, 1 << 26, A, GOOD, None,
                                         None, plan, nbytes, ra, 4, None, 0, None)
    assert call(M=0, X=None, ws=None) == OK
    assert call(K=100) == SHAPE and call(ra=8) == SHAPE and call(r=8) == SHAPE and call(N=12) == SHAPE
    assert call(X=None) == NULL and call(LA=None) == NULL and call(A=None) == NULL and call(plan=None) == NULL
    assert call(ws=None) == WORKSPACE and call(nbytes=8) == WORKSPACE


def test_adapters_of_no_rank_need_no_workspace(lib):
    """Without a rank there is nothing to multiply: the launch that copies serves any number of tokens."""
    for M in (1, 33, 200, 5000, 1 << 20):
        assert lib.aser_adapters_workspace_bytes(M, 4096, 4096, 0, 4) == 0


class Placed:
    """What the argument checks see of a tensor that lies on some GPU."""

    def __init__(self, device, shape=(4, 64), dtype=None, stride=None):
        import torch
        self.shape, self.dtype, self.device = torch.Size(shape), dtype or torch.float16, device
        self.strides = stride or (shape[1], 1)

    def get_device(self):
        return self.device

    def stride(self):
        return self.strides


def test_rows_are_on_the_current_gpu(lib):
    """(no GPU: the check alone, on what it reads)"""
    import torch
    from paper_2411_07762_b200.binding import _rows
    assert _rows(Placed(1), (4, 64), "X", 1) == 64
    assert _rows(Placed(1, stride=(80, 1)), (4, 64), "X", 1) == 80
    assert _rows(Placed(0, shape=(1, 64), stride=(1, 1)), (1, 64), "X", 0) == 64
    assert _rows(Placed(0, shape=(1, 64), stride=(640, 1)), (1, 64), "X", 0) == 64
    for bad in (Placed(0), Placed(-1), Placed(1, shape=(4, 72)), Placed(1, dtype=torch.bfloat16), Placed(1, stride=(0, 1)),
                Placed(1, stride=(32, 1)), Placed(1, stride=(1, 4)), Placed(1, stride=(128, 2))):
        with pytest.raises(TypeError):
            _rows(bad, (4, 64), "X", 1)


def test_a_plan_and_a_pool_are_on_the_current_gpu(lib):
    from types import SimpleNamespace
    from paper_2411_07762_b200.binding import AserAdapters
    pool = AserAdapters.__new__(AserAdapters)
    pool.n_slots, pool.device = 3, 1
    pool._check_plan(SimpleNamespace(M=4, n_slots=3, device=1), 4, 1)
    for plan, device in ((SimpleNamespace(M=4, n_slots=3, device=0), 1), (SimpleNamespace(M=4, n_slots=3, device=1), 0),
                         (SimpleNamespace(M=5, n_slots=3, device=1), 1), (SimpleNamespace(M=4, n_slots=2, device=1), 1), (None, 1)):
        with pytest.raises(ValueError):
            pool._check_plan(plan, 4, device)
