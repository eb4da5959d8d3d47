"""The status of adapter calls: kept in the plan, read and cleared by aser_adapters_check_status."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2411_07762_b200 import build
    build.build()
    from paper_2411_07762_b200 import binding
    return binding.lib


def test_bad_plans_are_refused(lib):
    assert lib.aser_adapters_check_status(None, None) == -1
    assert lib.aser_adapters_check_status(C.c_void_p(0x1004), None) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("M", [5, 900])
def test_status_of_a_plan(lib, M):
    """Calls leave it alone; a word as a wait that gave up leaves it is reported once, and a new plan starts without."""
    import paper_2411_07762_b200 as aser
    g = torch.Generator(device="cuda")
    g.manual_seed(M)
    normal = lambda *shape: torch.randn(*shape, device="cuda", dtype=torch.float16, generator=g) * 0.1
    pool = aser.AserAdapters(normal(3, 32, 512), normal(3, 256, 32))
    slot = torch.randint(-1, 3, (M,), device="cuda", generator=g, dtype=torch.int32)
    plan = pool.plan(slot)
    X, Y = normal(M, 512), normal(M, 256)
    want = pool.add(X, Y, plan, out=torch.empty_like(Y)).clone()
    plan.check_status()
    plan.data.view(torch.int32)[6] = 1
    assert torch.equal(pool.add(X, Y, plan, out=torch.empty_like(Y)), want)
    with pytest.raises(aser.AserError) as e:
        plan.check_status()
    assert e.value.code == -6
    plan.check_status()
    plan.data.view(torch.int32)[6] = 1
    plan.update(slot)
    plan.check_status()
    pool.plan(slot[:0]).check_status()
