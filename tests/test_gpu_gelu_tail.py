"""The exact GELU far out on its negative side, where it is small but not zero:
every value and derivative to a relative error. Needs an MI355X."""
import math

import pytest
import torch

from ffn_reference import E, act, act_grad, tiny, unit

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def fp32_error(z):
    """Relative, of Phi(z): exp(-z^2 / 2) in fp32 is off by z^2 / 2 units for its argument's rounding
    and once more for that of the power of two's; 16 units for the rest. Twice that for rcp and exp."""
    return 2 * E * (z * z + 16)


def check(got, want, bound, z, what):
    off = (got.double() - want).abs()
    bad = (~(off <= bound)).nonzero().flatten()
    assert not len(bad), (f"{what}: {len(bad)} values off, first at z = {z[bad[0]].item()}: {got[bad[0]].item()} for "
                          f"{want[bad[0]].item()}, bound {bound[bad[0]].item():.3g}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [20, 3000])
def test_gelu_tail(H, dtype, rows):
    """z = x exactly: one column, a weight of one; few rows and tiles"""
    print("gelu", dtype, rows, flush=True)
    z = torch.linspace(-12.5, 12.5, rows, device="cuda").to(dtype)
    zd, one = z.double(), torch.ones(1, 1, dtype=dtype, device="cuda")
    want, slope = act("gelu", zd), act_grad("gelu", zd)
    cdf = 0.5 * torch.special.erfc(-zd / math.sqrt(2))
    parts = cdf + zd.abs() * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)     # what the derivative is the sum of
    ev = want.abs() * (unit(dtype) + fp32_error(zd)) + tiny(dtype)
    ed = slope.abs() * unit(dtype) + 1.01 * parts * fp32_error(zd) + tiny(dtype)
    A = H.HEDDLE_A_GELU

    y = H.heddle_linear(z[:, None], one, act=A)
    check(y[:, 0], want, ev, z, "linear")
    got = H.heddle_linear_backward(torch.ones_like(y), z[:, None], one, act=A, preact=z[:, None], want_dw=False)
    check(got["dx"][:, 0], slope, ed, z, "linear's gradient")

    # gate z, up 1; y's first column is H
    x = torch.stack([z, torch.ones_like(z)], 1)
    eye, first = torch.eye(2, dtype=dtype, device="cuda"), torch.eye(2, dtype=dtype, device="cuda")[:, :1].contiguous()
    p = torch.empty(rows, 2, dtype=dtype, device="cuda")
    y = H.heddle_gated_ffn(x, eye, first, act=A, preact=p)
    assert torch.equal(p, x)
    check(y[:, 0], want, ev, z, "block")
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    got = H.heddle_gated_ffn_backward(dy, x, eye, first, p, act=A, want_dw=False)
    check(got["dx"][:, 0], slope, ed, z, "block's gradient of the gate")
    check(got["dx"][:, 1], want, ev, z, "block's gradient of the up projection")
