"""The global gradient norm and clipping against 64 bits. Needs an MI355X."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def tensors(spec, seed=0, scale=1.0):
    """spec: (size, type, values before the first) each"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(shift + n + 8, generator=g, device="cuda").mul_(scale).to(dt)[shift:shift + n] for n, dt, shift in spec]


def norm64(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def check(H, grads, max_norm, out=None):
    print("clip", len(grads), sum(g.numel() for g in grads), max_norm, out is not None, flush=True)
    before = [g.clone() for g in grads]
    want = norm64(before)
    alone = H.heddle_grad_norm(grads)
    norm = H.heddle_clip_grad_norm(grads, max_norm, out=out)
    assert torch.equal(alone, norm)
    # fp64 sums of at most 2^40 terms, one rounding to fp32
    assert abs(norm.item() - want) <= 2.0 ** -23 * want
    factor = min(1.0, max_norm / (norm.item() + 1e-6))
    for g, b, o in zip(grads, before, out or grads):
        w = b.double() * factor
        if out is not None:
            assert torch.equal(g, b), "an input was written"
        # the factor is off by 3 fp32 roundings, the product by one, the output by one of its type
        assert bool(((o.double() - w).abs() <= (4 * 2.0 ** -24 + 1.01 * UNIT[o.dtype]) * w.abs() + 2.0 ** -25).all())
        if factor == 1.0:
            assert torch.equal(o, b)


SPECS = {
    "one": [(1, F32, 0)],
    "odd": [(1, BF16, 1), (3, F16, 3), (17, F32, 1), (1000, BF16, 5), (8191, F32, 3), (16385, BF16, 0), (16384, F16, 1)],
    "empty": [(0, F32, 0), (5, BF16, 0), (0, F16, 0)],
    "long": [(5000001, BF16, 1), (3000000, F32, 1), (4000003, F16, 7)],
    "many": [(1 + 37 * i % 4001, (F32, BF16, F16)[i % 3], i % 9) for i in range(300)],
}


@pytest.mark.parametrize("name", sorted(SPECS))
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clip(H, name, max_norm):
    check(H, tensors(SPECS[name], 1), max_norm)
    grads = tensors(SPECS[name], 2)
    out = [torch.full((g.numel() + 3,), float("nan"), device="cuda", dtype=g.dtype)[1:g.numel() + 1] for g in grads]
    check(H, grads, max_norm, out)
    for o in out:
        whole = torch.as_strided(o, (o.numel() + 3,), (1,), 0)
        assert bool(torch.isnan(whole[:1]).all()) and bool(torch.isnan(whole[-2:]).all()), "values outside an output were written"


def test_no_tensors(H):
    assert H.heddle_clip_grad_norm([], 1.0).item() == 0.0
    assert H.heddle_clip_grad_norm(tensors([(0, F32, 0)]), 1.0).item() == 0.0


def test_squares_beyond_fp32(H):
    """values whose squares no fp32 holds, large and small"""
    for v in (3e30, 1e-30):
        g = torch.full((100,), v, device="cuda")
        assert abs(H.heddle_grad_norm([g]).item() / (10 * v) - 1) < 1e-6


def test_nonfinite(H):
    for bad in (float("nan"), float("inf")):
        for dt in (F32, BF16, F16):
            g = tensors([(5000, dt, 1), (40, F32, 0)])
            g[0][4321] = bad
            n = H.heddle_clip_grad_norm(g, 1.0).item()
            assert math.isnan(n) if math.isnan(bad) else n == math.inf
            if math.isnan(bad):
                assert all(bool(torch.isnan(t).all()) for t in g)
            else:
                assert math.isnan(g[0][4321].item()) and not g[1].any()


def test_parts(H):
    """norm of shards joined by the caller, then clipped"""
    g = tensors([(3000, BF16, 0), (777, F32, 1)], 3)
    a, b = H.heddle_grad_norm(g[:1]), H.heddle_grad_norm(g[1:])
    norm = (a * a + b * b).sqrt()
    both = [t.clone() for t in g]
    H.heddle_clip_grad_norm(both, 0.25)
    H.heddle_clip_grads(g, norm, 0.25)
    # the joined norm differs by fp32 roundings only: by at most one unit of the outputs' type
    for x, y in zip(g, both):
        assert bool(((x.double() - y.double()).abs() <= (2 * UNIT[x.dtype] + 8 * 2.0 ** -24) * y.double().abs()).all())


def test_repeat_stream_and_graph(H):
    g = tensors(SPECS["many"], 4)
    out = [torch.empty_like(t) for t in g]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = H.heddle_clip_grad_norm(g, 0.1, out=out, stream=s)
    s.synchronize()
    first = [t.clone() for t in out]
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


def test_refusals(H):
    g = tensors([(64, F32, 0)])
    bad = [lambda: H.heddle_clip_grad_norm(g, 0.0), lambda: H.heddle_clip_grad_norm(g, float("nan")),
           lambda: H.heddle_clip_grad_norm(g, float("inf")), lambda: H.heddle_clip_grad_norm(g, -1.0),
           lambda: H.heddle_grad_norm([g[0].double()]), lambda: H.heddle_grad_norm([g[0].cpu()]),
           lambda: H.heddle_grad_norm([g[0][::2]]), lambda: H.heddle_clip_grad_norm(g, 1.0, out=[]),
           lambda: H.heddle_clip_grad_norm(g, 1.0, out=[g[0].half()]), lambda: H.heddle_clip_grad_norm(g, 1.0, out=[g[0][:5]]),
           lambda: H.heddle_clip_grads(g, torch.ones(2, device="cuda"), 1.0), lambda: H.heddle_clip_grads(g, torch.ones(1), 1.0)]
    for i, f in enumerate(bad):
        with pytest.raises(H.HeddleError) as e:
            f()
        assert e.value.code == H.HEDDLE_E_INVAL, i
