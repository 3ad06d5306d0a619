"""A layer's passes wait for the GPU nowhere: what is timed around them is their
work. Needs an MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("experts", [0, 6])
def test_no_waits(experts):
    from workloads import measured as M
    layer = M.WholeLayer(96, 64, 72, experts, 2, seed=3)
    x, dy = torch.randn(70, 96, device="cuda").bfloat16(), torch.randn(70, 96, device="cuda").bfloat16()
    want = layer.forward(x)
    layer.backward(dy)
    torch.cuda.synchronize()
    before = torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        y = layer.forward(x)
        layer.backward(dy)
    finally:
        torch.cuda.set_sync_debug_mode(before)
    assert torch.equal(y, want)
    assert layer.documents.tolist() == [0, 70] and layer.documents.dtype == torch.int32
