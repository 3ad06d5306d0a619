"""The operators together: layers trained with them, and plans priced with
times measured on this GPU. Needs an MI355X."""
import numpy as np
import pytest
import torch

from oracle import oracle as O
from workloads.gen import load_config, make_workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    assert torch.cuda.is_available(), "no GPU"
    from workloads import measured
    return measured


def plain(layer, w, x, picked):
    """the layer in fp64, differentiable"""
    block = lambda r, wi, wo: (torch.nn.functional.silu(r @ wi[:wi.shape[0] // 2].t()) * (r @ wi[wi.shape[0] // 2:].t())) @ wo.t()  # noqa: E731
    h = x + (x @ w["kv"].t())[:, layer.width:] @ w["out"].t()
    if not layer.experts:
        return h + block(h, w["in"], w["down"])
    rows = [sum(block(h[t:t + 1], w["in"][e], w["down"][e]) for e in picked[t].tolist()) for t in range(len(h))]
    return h + torch.cat(rows) / layer.top_k


@pytest.mark.parametrize("experts", [0, 6])
def test_layer_against_autograd(M, experts):
    """the bf16 roundings of a chain of four products: an error of a few units of 2^-8 relative to the gradient's norm"""
    layer = M.Layer(96, 64, 72, experts, 2, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(40, 96, generator=g, device="cuda").bfloat16() for _ in range(2))
    picked = torch.rand(40, experts, generator=g, device="cuda").topk(2, 1).indices if experts else None
    y = layer.forward(x, picked)
    dx, grads = layer.backward(dy)
    w = {k: v.double().requires_grad_(True) for k, v in layer.w.items()}
    xd = x.double().requires_grad_(True)
    want = plain(layer, w, xd, picked)
    want.backward(dy.double())
    for name, got, ref in [("y", y, want.detach()), ("dx", dx, xd.grad)] + [(k, grads[k], w[k].grad) for k in ("kv", "out", "in", "down")]:
        assert float((got.double() - ref).norm()) <= 8 * 2.0 ** -8 * float(ref.norm()), name
    assert not grads["q"].any()


@pytest.mark.parametrize("experts", [0, 6])
def test_training_lowers_the_loss(M, experts):
    layers = [M.Layer(128, 64, 96, experts, 2, seed=s) for s in range(2)]
    g = torch.Generator(device="cuda").manual_seed(9)
    x, target = (torch.randn(200, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    picked = torch.rand(200, experts, generator=g, device="cuda").topk(2, 1).indices if experts else None
    # gradients are clipped to a norm of 0.02: an update is far below the weights' norm of about 40
    runs = [tuple(float(v) for v in M.train(layers, x, target, picked, rate=20.0, max_norm=0.02)) for _ in range(12)]
    losses = [r[0] for r in runs]
    assert all(np.isfinite(losses)) and losses[-1] < losses[0] and all(r[1] > 0 for r in runs)


def test_plans_with_measured_times(M):
    """measured layer times price like any others: the oracle's results, bit for bit"""
    from paper_2609_34244_amd import heddle as H
    w = make_workload("c1_tiny_dense", n=200)
    profile, times = M.measure(load_config("c1_tiny_dense"), w.profile, repeat=2)
    assert times and all(t > 0 for pair in times.values() for t in pair)
    assert (profile.layer_ns[1:] == w.profile.layer_ns[1:]).all()
    ns, st = H.to_device(w.n_stages, w.stages)
    m = [int(x) for x in w.m]
    out = H.alloc_outputs(w.n, len(m), w.s_max, 0)
    H.heddle_price_plans(H.heddle_load_profile(profile), ns, st, m, 0, out)
    torch.cuda.synchronize()
    want = O.price_plans(O.OracleProfile(profile), w.n_stages, w.stages, w.m, 0)
    for k in ("status", "layers", "peak_mem", "iter", "bottleneck"):
        assert np.array_equal(out[k].cpu().numpy(), want[k]), k
