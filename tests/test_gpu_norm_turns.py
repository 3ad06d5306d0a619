"""Layer normalisation whose workgroups take several rows in turn, by its values. Needs an
MI355X."""
import pytest
import torch

import layer_reference as R
from layer_common import near
from test_gpu_norm import run

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


@pytest.mark.parametrize("n,dtype,wdtype", [(2056, BF16, BF16), (4096, BF16, FP32), (3001, FP16, FP16), (8192, BF16, BF16), (5003, FP16, FP32),
                                            (2048, FP32, FP32), (1027, FP32, FP32), (4096, FP32, FP32), (8192, FP32, FP32), (6001, FP32, FP32),
                                            (20000, BF16, FP32), (12289, FP32, FP32)])
@pytest.mark.parametrize("m", [513, 1100])
def test_rows_of_512_lanes(H, m, n, dtype, wdtype):
    """three turns and more, the last one not all workgroups', with one to four pieces a lane; long rows"""
    run(H, m + n, m, n, dtype, wdtype)
    run(H, m, m, n, dtype, wdtype, residual=False, w=False)


@pytest.mark.parametrize("n", [520, 515])
def test_more_rows_than_workgroups(H, n):
    """a forward pass of more than 2^20 rows, a workgroup each"""
    m = (1 << 20) + 77
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(m, n, generator=g, device="cuda", dtype=BF16)
    w, b = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    stats = torch.empty(m, 2, device="cuda")
    y = H.heddle_layer_norm(x, w, b, stats=stats)
    for at in (slice(0, 90), slice(m - 90, m)):
        want, bound, ws, bs = R.layer_norm(x[at], w, b, 1e-5, BF16, FP32)
        near(y[at], want, bound, "y")
        near(stats[at], ws, bs, "stats")
    again = H.heddle_layer_norm(x[:1 << 20], w, b)
    assert torch.equal(again, y[:1 << 20])
