"""A gate below float16's range is kept as -infinity; the forward pass, in fp32,
had an activation of 0 there, and so has the backward pass: no NaN comes of it.
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


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("t", [3, 70])
def test_gate_below_the_range(H, act, t):
    print("gate", act, t, flush=True)
    d, f, a = 24, 40, H.ACTIVATIONS[act]
    g = torch.Generator(device="cuda").manual_seed(t)
    x = torch.rand(t, d, generator=g, device="cuda").half() + 1
    wi, wo = torch.randn(2 * f, d, generator=g, device="cuda").half(), torch.randn(d, f, generator=g, device="cuda").half()
    dy = torch.randn(t, d, generator=g, device="cuda").half()
    low = list(range(0, f, 3))
    wi[low] = -8000                                     # gates of 24 x -8000 and below
    p = torch.empty(t, 2 * f, dtype=torch.half, device="cuda")
    y = H.heddle_gated_ffn(x, wi, wo, act=a, preact=p)
    assert bool((p[:, low] == -float("inf")).all()) and bool(torch.isfinite(y).all())
    got = H.heddle_gated_ffn_backward(dy, x, wi, wo, p, act=a)
    assert all(bool(torch.isfinite(v).all()) for v in got.values())
    # those units have no part in anything
    assert not got["dw_in"][low].any() and not got["dw_in"][[f + j for j in low]].any() and not got["dw_out"][:, low].any()
    rest = [j for j in range(f) if j not in low]
    small = H.heddle_gated_ffn_backward(dy, x, wi[rest + [f + j for j in rest]], wo[:, rest].contiguous(),
                                        p[:, rest + [f + j for j in rest]].contiguous(), act=a)
    assert torch.equal(got["dw_out"][:, rest], small["dw_out"])


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
def test_derivatives_at_infinity(H, act):
    """of kept values: 0 at -infinity, 1 at +infinity, a NaN at a NaN"""
    z = torch.tensor([[-float("inf")], [float("inf")], [float("nan")], [-6e4], [6e4]], device="cuda").half()
    one = torch.ones(1, 1, device="cuda").half()
    for rows in (z, z.repeat(20, 1)):
        dx = H.heddle_linear_backward(torch.ones_like(rows), torch.zeros_like(rows), one, act=H.ACTIVATIONS[act], preact=rows,
                                      want_dw=False)["dx"].view(-1, 5)
        assert bool((dx[:, [0, 3]] == 0).all()) and bool((dx[:, [1, 4]] == 1).all()) and bool(torch.isnan(dx[:, 2]).all())
