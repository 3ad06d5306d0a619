"""The feed-forward operators record nothing for autograd: a tensor that
requires a gradient is refused where torch would expect it to be recorded.
Needs an MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def test_requires_grad(H):
    g = torch.Generator(device="cuda").manual_seed(0)
    x, w, r, dy = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((6, 32), (32, 32), (6, 32), (6, 32)))
    wi, b, p = torch.randn(64, 32, generator=g, device="cuda").bfloat16(), torch.randn(32, generator=g, device="cuda").bfloat16(), x.new_empty(6, 64)
    calls = {"linear": (lambda x, w, b, r: H.heddle_linear(x, w, bias=b, residual=r), [x, w, b, r]),
             "linear backward": (lambda dy, x, w: H.heddle_linear_backward(dy, x, w)["dx"], [dy, x, w]),
             "block": (lambda x, wi, w, r: H.heddle_gated_ffn(x, wi, w, residual=r, preact=p), [x, wi, w, r]),
             "block backward": (lambda dy, x, wi, w: H.heddle_gated_ffn_backward(dy, x, wi, w, p)["dx"], [dy, x, wi, w])}
    for name, (call, args) in calls.items():
        want = call(*args)
        for i in range(len(args)):
            given = [a.clone().requires_grad_(i == j) for j, a in enumerate(args)]
            with pytest.raises(H.HeddleError) as e:
                call(*given)
            assert e.value.code == H.HEDDLE_E_INVAL and "no_grad" in str(e.value), (name, i)
            with torch.no_grad():
                assert torch.equal(call(*given), want), (name, i)


def test_clipping_of_recorded_gradients(H):
    """clipping changes gradients, whose own history nothing follows: as before"""
    g = [torch.full((5,), 2.0, device="cuda").requires_grad_(True) * 3]
    assert abs(H.heddle_clip_grad_norm(g, 1.0).item() - 180 ** 0.5) < 1e-5
    assert abs(H.heddle_grad_norm(g).item() - 1) < 1e-5
