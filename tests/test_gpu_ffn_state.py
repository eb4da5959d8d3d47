"""What a gated feed-forward block keeps."""
import pytest
import torch

from test_gpu_ffn import gen, normal


@pytest.fixture(scope="module")
def aser():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2411_07762_b200 as aser
    return aser


@pytest.mark.gpu
def test_weights_are_kept_once(aser):
    """A block holds its packed weights in one layout: half a byte a weight, beside factors, workspace and output."""
    g = gen(2)
    K, F, M = 2048, 4096, 16
    ops = (normal(g, F, K), normal(g, F, K), None, None, None, normal(g, K, F), None, None, None)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    block = aser.AserGatedFFN(*ops, M)
    held = torch.cuda.memory_allocated() - before
    assert held < 3 * K * F // 2 + block.ws.numel() + 2 * M * K + 4 * (2 * F + K) + 16 * 512
