"""A gated feed-forward block of tensors that lie on another GPU than the current one, or on none, is refused before any kernel is
launched (no GPU needed: stand-ins tell where they lie)."""
import pytest
import torch

NAMES = ("W_gate", "W_up", "s", "L_A", "L_B", "W_down", "s_down", "L_A_down", "L_B_down")


class Placed:
    def __init__(self, device):
        self.device = device

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        raise AssertionError("%s was looked at" % name)


@pytest.fixture
def block(monkeypatch):
    from paper_2411_07762_b200 import build
    build.build()
    from paper_2411_07762_b200 import binding
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return binding.AserGatedFFN


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("where", [1, -1])
def test_tensors_of_another_gpu_are_refused(block, name, where):
    with pytest.raises(ValueError, match=name + " needs"):
        block(*(Placed(where if n == name else 0) for n in NAMES), 4)
