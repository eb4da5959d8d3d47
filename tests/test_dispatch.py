"""Which kernels serve a size (no GPU needed: what the library says of itself)."""
import pytest


@pytest.fixture(scope="module")
def aser():
    from paper_2411_07762_b200 import build
    build.build()
    import paper_2411_07762_b200 as aser
    return aser


@pytest.mark.parametrize("M,K,r,launches", [(225, 4608, 128, 2), (256, 5120, 128, 2), (257, 4608, 96, 2), (225, 4096, 128, 1), (320, 4096, 96, 1),
                                            (343, 5120, 64, 1), (449, 4608, 16, 1), (528, 5120, 32, 1), (200, 5120, 128, 1), (160, 5120, 128, 1)])
def test_activation_step_of_rows_of_4096_to_5120_columns(aser, M, K, r, launches):
    """A forward pass takes one launch up to 400 CTAs, at high ranks of rows that have not 4096 columns up to 340."""
    assert aser.forward_act_launches(M, K, r) == launches
