"""The layer's operators together: norms, attention within documents, products,
experts picked by a router, its balance loss, all gradients and a training step.
Needs an MI355X."""
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


def plain(layer, w, x, picked, lengths):
    """the layer in fp64, differentiable: (y, balance loss)"""
    norm = lambda v, i: torch.nn.functional.layer_norm(v, v.shape[1:], w[f"norm{i}"], w[f"shift{i}"], 1e-5)  # noqa: E731
    block = lambda r, wi, wo: (torch.nn.functional.silu(r @ wi[:wi.shape[0] // 2].t()) * (r @ wi[wi.shape[0] // 2:].t())) @ wo.t()  # noqa: E731
    n, d = norm(x, 1), layer.width // layer.heads
    q, kv = n @ w["q"].t(), n @ w["kv"].t()
    parts, row = [], 0
    for length in lengths:
        at = slice(row, row + length)
        hidden = torch.ones(length, length, dtype=torch.bool, device=x.device).triu(1)
        heads = []
        for h in range(layer.heads):
            c = slice(h * d, (h + 1) * d)
            s = (q[at, c] @ kv[at, :layer.width][:, c].t()) * d ** -0.5
            heads.append(torch.softmax(s.masked_fill(hidden, -float("inf")), 1) @ kv[at, layer.width:][:, c])
        parts.append(torch.cat(heads, 1))
        row += length
    h = x + torch.cat(parts) @ w["out"].t()
    n = norm(h, 2)
    if not layer.experts:
        return h + block(n, w["in"], w["down"]), 0.0
    counts = torch.bincount(picked.flatten(), minlength=layer.experts).double()
    loss = layer.BALANCE * layer.experts * (counts / counts.sum() * torch.softmax(n @ w["router"].t(), 1).mean(0)).sum()
    rows = [sum(block(n[t:t + 1], w["in"][e], w["down"][e]) for e in picked[t].tolist()) for t in range(len(h))]
    return h + torch.cat(rows) / layer.top_k, loss


@pytest.mark.parametrize("experts", [0, 6])
@pytest.mark.parametrize("width", [64, 192])
def test_layer_against_autograd(M, experts, width):
    """the bf16 roundings of a chain of ten operators, each of a unit of 2^-8 relative to its output's norm"""
    layer = M.WholeLayer(96, width, 72, experts, 2, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy = (torch.randn(70, 96, generator=g, device="cuda").bfloat16() for _ in range(2))
    lengths = [33, 0, 1, 36]
    offsets = torch.tensor([0, 33, 33, 34, 70], dtype=torch.int32, device="cuda")
    y = layer.forward(x, documents=offsets)
    dx, grads = layer.backward(dy)
    w = {k: v.double().requires_grad_(True) for k, v in layer.w.items()}
    xd = x.double().requires_grad_(True)
    want, loss = plain(layer, w, xd, layer.picked if experts else None, lengths)
    (want * dy.double()).sum().add(loss).backward()
    assert set(grads) == set(w)
    if experts:
        assert abs(float(layer.loss) - loss.item()) <= 2.0 ** -8 * loss.item()
    for name, got, ref in [("y", y, want.detach()), ("dx", dx, xd.grad)] + [(k, grads[k], v.grad) for k, v in w.items()]:
        assert float((got.double() - ref).norm()) <= 10 * 2.0 ** -8 * float(ref.norm()), name


@pytest.mark.parametrize("experts", [0, 6])
def test_training_step(M, experts):
    layers = [M.WholeLayer(128, 64, 96, experts, 2, seed=s) for s in range(2)]
    g = torch.Generator(device="cuda").manual_seed(9)
    x, target = (torch.randn(200, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    before = {(i, k): v.clone() for i, layer in enumerate(layers) for k, v in layer.w.items()}
    loss, norm = M.train(layers, x, target, rate=0.1)
    assert bool(torch.isfinite(loss)) and float(norm) > 0
    changed = [not torch.equal(v, layers[i].w[k]) for (i, k), v in before.items()]
    assert sum(changed) > len(changed) // 2


def test_plans_with_measured_times(M):
    """times of whole layers price like any others: the oracle's results, bit for bit"""
    from paper_2609_34244_amd import heddle as H
    w = make_workload("c1_tiny_dense", n=200)
    profile, times = M.measure(load_config("c1_tiny_dense"), w.profile, repeat=2, whole=True)
    assert times and all(t > 0 for pair in times.values() for t in pair)
    ns, st = H.to_device(w.n_stages, w.stages)
    m = [int(x) for x in w.m]
    out = H.alloc_outputs(w.n, len(m), w.s_max, 0)
    H.heddle_price_plans(H.heddle_load_profile(profile), ns, st, m, 0, out)
    torch.cuda.synchronize()
    want = O.price_plans(O.OracleProfile(profile), w.n_stages, w.stages, w.m, 0)
    for k in ("status", "layers", "peak_mem", "iter", "bottleneck"):
        assert np.array_equal(out[k].cpu().numpy(), want[k]), k
