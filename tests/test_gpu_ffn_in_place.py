"""Outputs that may lie on inputs, because the call has read them by then: the
same bits as with outputs of their own; and the ones that may not. Needs an MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu

D, F = 264, 520


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def normal(g, *shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(scale).bfloat16()


# few rows, tiles, a divided reduction, large tiles; rows on odd addresses are copied first
@pytest.mark.parametrize("t", [3, 70, 300, 4100])
@pytest.mark.parametrize("odd", [0, 1])
def test_block(H, t, odd):
    print("in place", t, odd, flush=True)
    g = torch.Generator(device="cuda").manual_seed(t)
    wide = normal(g, t, D + odd)
    x = wide[:, odd:]
    wi, wo, dy = normal(g, 2 * F, D, scale=D ** -0.5), normal(g, D, F, scale=F ** -0.5), normal(g, t, D)
    p = x.new_empty(t, 2 * F)
    want = H.heddle_gated_ffn(x, wi, wo, residual=x, preact=p)
    plain = H.heddle_gated_ffn(x, wi, wo)
    grads = H.heddle_gated_ffn_backward(dy, x, wi, wo, p)
    for residual in (True, False):
        y = wide.clone()[:, odd:]
        assert H.heddle_gated_ffn(y, wi, wo, residual=y if residual else None, out=y) is y
        assert torch.equal(y, want if residual else plain), residual
    y = wide.clone()[:, odd:]
    H.heddle_gated_ffn(x, wi, wo, residual=y, out=y)
    assert torch.equal(y, want)
    d = dy.clone()
    got = H.heddle_gated_ffn_backward(d, x, wi, wo, p, dx=d, want_dw=False, dw_in=torch.empty_like(wi))
    assert torch.equal(d, grads["dx"]) and torch.equal(got["dw_in"], grads["dw_in"])
    for f in (lambda: H.heddle_gated_ffn_backward(d, x, wi, wo, p, dx=d), lambda: H.heddle_gated_ffn_backward(dy, x, wi, wo, p, dx=x)):
        with pytest.raises(H.HeddleError, match="overlaps"):
            f()


@pytest.mark.parametrize("m", [3, 70, 4100])
def test_linear(H, m):
    g = torch.Generator(device="cuda").manual_seed(m)
    x, w, dy = normal(g, m, D), normal(g, D, D, scale=D ** -0.5), normal(g, m, D)
    z = torch.empty_like(x)
    want = H.heddle_linear(x, w, act=H.HEDDLE_A_SILU, residual=dy, preact=z)
    y = dy.clone()
    H.heddle_linear(x, w, act=H.HEDDLE_A_SILU, residual=y, out=y)
    assert torch.equal(y, want)
    grads = H.heddle_linear_backward(dy, x, w, act=H.HEDDLE_A_SILU, preact=z, want_db=True)
    d = dy.clone()
    got = H.heddle_linear_backward(d, x, w, act=H.HEDDLE_A_SILU, preact=z, want_db=True, dx=d)
    assert all(torch.equal(got[k], grads[k]) for k in grads)
    # side by side in one allocation
    both = torch.cat([x, torch.zeros_like(x)], 1)
    H.heddle_linear(both[:, :D], w, act=H.HEDDLE_A_SILU, residual=dy, out=both[:, D:])
    assert torch.equal(both[:, D:], want) and torch.equal(both[:, :D], x)
    for f in (lambda: H.heddle_linear(x, w, out=x), lambda: H.heddle_linear(x, w, out=z, preact=z),
              lambda: H.heddle_linear(both[:, :D], w, out=both[:, D - 1:2 * D - 1]), lambda: H.heddle_linear_backward(d, x, w, dx=d),
              lambda: H.heddle_linear_backward(dy, x, w, dx=x), lambda: H.heddle_linear_backward(dy, x, w, dw=w, dx=w[:m] if m < D else w)):
        with pytest.raises(H.HeddleError, match="overlaps|shape"):
            f()
