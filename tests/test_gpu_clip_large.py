"""Clipping of 32 MiB and more, whose kernels take larger chunks: several
launches of them, more chunks than workgroups, every alignment, in place and
into outputs that start anywhere. Needs an MI355X."""
import pytest
import torch

from test_gpu_clip import BF16, F16, F32, H, check, tensors  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = (F32, BF16, F16)
SPECS = {
    # just above the bound on both sizes of values
    "one": [(8388609, F32, 1)],
    "types": [(5000001, F32, 3), (6000007, BF16, 1), (9000005, F16, 7), (0, BF16, 0), (1, F16, 5)],
    # several launches of 120 tensors, most of a few chunks and some of none
    "many": [((0, 17, 30001, 90001, 300007)[i % 5] + i, TYPES[i % 3], i % 9) for i in range(301)],
    # more chunks of 32 KB than the 2048 workgroups of a launch, whole and partial last ones
    "long": [(40000003, BF16, 5), (16384 * 700, F16, 0), (8192 * 300 + 1, F32, 2)],
}


def test_sizes():
    """all of them are large calls, and `long` has more chunks than workgroups"""
    for name, spec in SPECS.items():
        total = sum(n * dt.itemsize for n, dt, _ in spec)
        assert total >= 32 << 20, name
    assert sum(n * dt.itemsize for n, dt, _ in SPECS["long"]) > 2048 * 32768


@pytest.mark.parametrize("name", sorted(SPECS))
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clip(H, name, max_norm):  # noqa: F811
    check(H, tensors(SPECS[name], 1), max_norm)
    grads = tensors(SPECS[name], 2)
    out = [torch.full((g.numel() + 3,), float("nan"), device="cuda", dtype=g.dtype)[1:g.numel() + 1] for g in grads]
    check(H, grads, max_norm, out)
    for o in out:
        whole = torch.as_strided(o, (o.numel() + 3,), (1,), 0)
        assert bool(torch.isnan(whole[:1]).all()) and bool(torch.isnan(whole[-2:]).all()), "values outside an output were written"


def test_same_bits(H):  # noqa: F811
    """the norm's sums are in one order: the same bits twice, and in a replayed graph"""
    g = tensors(SPECS["many"], 4)
    out = [torch.empty_like(t) for t in g]
    a = H.heddle_clip_grad_norm(g, 0.1, out=out)
    first = [t.clone() for t in out]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = H.heddle_clip_grad_norm(g, 0.1, out=out)
    for i in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, a) and all(torch.equal(x, y) for x, y in zip(out, first)), i
        b = H.heddle_clip_grad_norm(g, 0.1, out=out)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and all(torch.equal(x, y) for x, y in zip(out, first)), i
