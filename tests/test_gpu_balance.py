"""Expert counts, the balance loss and its gradient against the plain 64-bit
form, every value within the bound that the roundings allow. Needs an MI355X."""
import pytest
import torch

import layer_reference as R
from layer_common import Maker, near

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def run(H, seed, t, e, k, dtype=FP32, picks=torch.int64, padding=False, residual=True, gap=0, shift=0, scale=0.01, dloss=None, spread=1.0):
    print(f"balance {t} {e} {k} {dtype} {picks} padding={padding} residual={residual} gap={gap} shift={shift}", flush=True)
    mk = Maker(seed)
    z = mk.part((t, e), dtype, (e + gap, 1), shift, spread)
    out = mk.part((t, e), dtype, (e + gap, 1), shift)
    r = mk.part((t, e), dtype, (e + gap, 1), shift, 1e-4) if residual else None
    picked = torch.rand(t, e, generator=mk.g, device="cuda").topk(k, 1).indices.to(picks)
    if padding and t:
        picked[::3] = -1
        picked[1::7, 0] = e
        picked[::5, k - 1] = 2**31 - 1 if picks == torch.int32 else 2**40
        z[0] = float("nan")                                   # a padded row's logits do not matter
        picked[0] = -1
    got = H.heddle_expert_balance(z, picked, scale=scale)
    counts, rows, mean, em, loss, el = R.balance(torch.nan_to_num(z), picked, scale)
    assert got["counts"].tolist() == counts.tolist() and got["rows"].tolist() == [rows]
    assert got["offsets"].tolist() == [0] + counts.cumsum(0).tolist()
    near(got["mean"], mean, em + R.E * mean, "mean")
    near(got["loss"], loss.reshape(1), (el + R.E * loss.abs()).reshape(1), "loss")
    d = None if dloss is None else torch.tensor([dloss], device="cuda")
    H.heddle_expert_balance_backward(z, picked, got["counts"], got["rows"], dloss=d, scale=scale, residual=r, out=out)
    want, bound = R.balance_backward(torch.nan_to_num(z), picked, counts, rows, 1.0 if dloss is None else float(d), scale, r, dtype)
    near(out, want, bound, "dlogits")
    mk.untouched()


@pytest.mark.parametrize("e", [1, 2, 7, 8, 9, 16, 17, 32, 33, 63, 64, 65, 100, 128, 130, 256, 257, 500, 1000, 1024, 2047, 2048])
@pytest.mark.parametrize("t", [1, 5, 33, 700])
def test_sizes(H, e, t):
    run(H, e + t, t, e, min(2, e), BF16 if e % 2 else FP32, torch.int32 if t % 2 else torch.int64)


@pytest.mark.parametrize("k", [1, 2, 3, 8, 20])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("padding", [False, True])
def test_picks(H, k, dtype, padding):
    run(H, k, 130, 40, k, dtype, torch.int64, padding, residual=k % 2 == 0, dloss=None if k == 1 else 0.5)
    run(H, k, 50, 20, k, dtype, torch.int32, padding, dloss=-2.0)


@pytest.mark.parametrize("gap,shift", [(3, 0), (0, 3), (5, 1)])
@pytest.mark.parametrize("e", [6, 64, 300])
def test_strides(H, gap, shift, e):
    run(H, e, 77, e, 2, FP32, gap=gap, shift=shift)
    run(H, e, 77, e, 2, BF16, gap=gap, shift=shift)


@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_spread(H, spread):
    """equal probabilities; one expert takes all"""
    run(H, 3, 200, 64, 2, FP32, spread=spread)


def test_large(H):
    run(H, 4, 50000, 64, 4, BF16)
    run(H, 5, 3000, 2000, 8, FP32)


def test_the_same_expert_twice(H):
    z = torch.randn(3, 4, device="cuda")
    picked = torch.tensor([[1, 1], [2, 0], [3, 3]], device="cuda")
    got = H.heddle_expert_balance(z, picked)
    assert got["counts"].tolist() == [1, 2, 1, 2] and got["rows"].item() == 3 and got["offsets"].tolist() == [0, 1, 3, 4, 6]


def test_masked_experts(H):
    """logits of -infinity: no probability and no gradient; a row of nothing else adds none"""
    z = torch.randn(40, 10, device="cuda")
    z[:, 3], z[7] = -float("inf"), -float("inf")
    picked = torch.randint(0, 3, (40, 2), device="cuda")
    got = H.heddle_expert_balance(z, picked, scale=2.0)
    p = torch.nan_to_num(torch.softmax(z.double(), 1))
    near(got["mean"], p.mean(0), 64 * R.E * p.mean(0) + 1e-30, "mean")
    d = H.heddle_expert_balance_backward(z, picked, got["counts"], got["rows"], scale=2.0)
    assert not d[:, 3].any() and not d[7].any() and bool(torch.isfinite(d).all())


def test_no_rows_and_no_picks(H):
    z, none = torch.randn(4, 6, device="cuda"), torch.full((4, 2), -1, device="cuda")
    for got in (H.heddle_expert_balance(z, none), H.heddle_expert_balance(z[:0], none[:0])):
        assert not any(got[k].any() for k in ("counts", "offsets", "rows", "mean", "loss"))
    got = H.heddle_expert_balance(z, none)
    assert not H.heddle_expert_balance_backward(z, none, got["counts"], got["rows"]).any()
    assert H.heddle_expert_balance_backward(z[:0], none[:0], got["counts"], got["rows"]).numel() == 0


def test_gradient_against_differences(H):
    g = torch.Generator(device="cuda").manual_seed(7)
    z = torch.randn(30, 12, generator=g, device="cuda")
    picked = torch.randint(0, 12, (30, 2), generator=g, device="cuda")
    got = H.heddle_expert_balance(z, picked, scale=3.0)
    d = H.heddle_expert_balance_backward(z, picked, got["counts"], got["rows"], scale=3.0)
    step = torch.randn(30, 12, generator=g, device="cuda").double()
    f = lambda h: float(R.balance(z.double() + h * step, picked, 3.0)[4])  # noqa: E731
    slope = (f(1e-5) - f(-1e-5)) / 2e-5
    assert abs(slope - float((d.double() * step).sum())) <= 1e-5 * float(d.double().norm() * step.norm())


def test_in_place_stream_and_graph(H):
    g = torch.Generator(device="cuda").manual_seed(1)
    z, r = (torch.randn(5000, 64, generator=g, device="cuda") for _ in range(2))
    picked = torch.randint(0, 64, (5000, 2), generator=g, device="cuda")
    got = H.heddle_expert_balance(z, picked)
    want = H.heddle_expert_balance_backward(z, picked, got["counts"], got["rows"], residual=r)
    for over in ("z", "r"):
        a, b = z.clone(), r.clone()
        assert torch.equal(H.heddle_expert_balance_backward(a, picked, got["counts"], got["rows"], residual=b, out=a if over == "z" else b), want)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    there = H.heddle_expert_balance(z, picked, stream=other)
    other.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one = H.heddle_expert_balance(z, picked)
        d = H.heddle_expert_balance_backward(z, picked, one["counts"], one["rows"], residual=r)
    for _ in range(3):
        for t in (d, *one.values()):
            t.zero_()
        graph.replay()
        again = H.heddle_expert_balance(z, picked)
        torch.cuda.synchronize()
        assert torch.equal(d, want)
        for k, t in got.items():
            assert torch.equal(one[k], t) and torch.equal(again[k], t) and torch.equal(there[k], t), k


def test_counts_feed_the_experts(H):
    """router, balance and grouped products together: rows sorted by expert use the offsets as they are"""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(50, 32, generator=g, device="cuda").to(BF16)
    wr, w = torch.randn(8, 32, generator=g, device="cuda").to(BF16), torch.randn(8, 40, 32, generator=g, device="cuda").to(BF16)
    logits = H.heddle_linear(x, wr)
    picked = logits.float().topk(2, 1).indices
    got = H.heddle_expert_balance(logits, picked)
    order = torch.argsort(picked.flatten(), stable=True)
    y = H.heddle_linear(x[order // 2], w, offsets=got["offsets"])
    want = torch.stack([x[i // 2].double() @ w[picked.flatten()[i]].double().t() for i in order.tolist()])
    near(y, want, want.abs() * 2.0 ** -8 + 40 * R.E * (x.double().abs().amax() * w.double().abs().amax() * 32), "y")


def test_refusals(H):
    z, p = torch.ones(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    got = H.heddle_expert_balance(z, p)
    c, n = got["counts"], got["rows"]
    big = torch.ones(1, 2049, device="cuda")
    for call in (lambda: H.heddle_expert_balance(z, p[:3]), lambda: H.heddle_expert_balance(z, p.float()), lambda: H.heddle_expert_balance(z[0], p),
                 lambda: H.heddle_expert_balance(z, p.repeat(1, 5)), lambda: H.heddle_expert_balance(big, p[:1]), lambda: H.heddle_expert_balance(z.double(), p),
                 lambda: H.heddle_expert_balance(z, p, scale=float("inf")), lambda: H.heddle_expert_balance(z.cpu(), p),
                 lambda: H.heddle_expert_balance(z.clone().requires_grad_(True), p), lambda: H.heddle_expert_balance_backward(z, p, c[:4], n),
                 lambda: H.heddle_expert_balance_backward(z, p, c, c), lambda: H.heddle_expert_balance_backward(z, p, c, n, dloss=torch.ones(2, device="cuda")),
                 lambda: H.heddle_expert_balance_backward(z, p, c, n, residual=z.half()), lambda: H.heddle_expert_balance_backward(z, p, c, n, out=z[:, :4])):
        with pytest.raises(H.HeddleError) as e:
            call()
        assert e.value.code == H.HEDDLE_E_INVAL


def test_loss_gradient_requires_grad(H):
    z, p = torch.ones(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    got = H.heddle_expert_balance(z, p)
    given = torch.full((1,), 0.5, device="cuda")
    want = H.heddle_expert_balance_backward(z, p, got["counts"], got["rows"], dloss=given)
    given.requires_grad_(True)
    with pytest.raises(H.HeddleError, match="no_grad"):
        H.heddle_expert_balance_backward(z, p, got["counts"], got["rows"], dloss=given)
    with torch.no_grad():
        assert torch.equal(H.heddle_expert_balance_backward(z, p, got["counts"], got["rows"], dloss=given), want)
