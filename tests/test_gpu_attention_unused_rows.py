"""Rows of no sequence: of an output that the call makes they are zeros, as a product over
all rows adds them up, in one that it is given they stay. Needs an MI355X."""
import pytest
import torch

from layer_common import ints

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def leave_nan():
    """memory that the allocator hands out next holds NaN"""
    held = [torch.full((n,), float("nan"), dtype=BF16, device="cuda") for n in (1 << 23, 1 << 19, 1 << 18, 1 << 16, 1 << 12) for _ in range(8)]
    torch.cuda.synchronize()
    del held


def tensors(shape_q, shape_k, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v, dy = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in (shape_q, shape_k, shape_k, shape_q))
    return q, k, v, dy, torch.zeros(shape_q[:-1], device="cuda")


def both_ways(H, shape_q, shape_k, dtype, used_q, used_k, how):
    q, k, v, dy, lse = tensors(shape_q, shape_k, dtype)
    mark = {n: torch.full(s, 7.0, dtype=dtype, device="cuda") for n, s in (("y", shape_q), ("dq", shape_q), ("dk", shape_k), ("dv", shape_k))}
    H.heddle_attention(q, k, v, lse=lse, out=mark["y"], **how)
    leave_nan()
    y = H.heddle_attention(q, k, v, **how)
    grads = {n: mark[n] for n in ("dq", "dk", "dv")}
    H.heddle_attention_backward(dy, q, k, v, mark["y"], lse, **grads, **how)
    leave_nan()
    made = dict(H.heddle_attention_backward(dy, q, k, v, mark["y"], lse, **how), y=y)
    for n, used in (("y", used_q), ("dq", used_q), ("dk", used_k), ("dv", used_k)):
        assert not made[n][~used].any(), n
        assert torch.equal(made[n][used], mark[n][used]), n
        assert bool((mark[n][~used] == 7).all()), n
    # one given, one made
    leave_nan()
    dk = torch.full(shape_k, 7.0, dtype=dtype, device="cuda")
    got = H.heddle_attention_backward(dy, q, k, v, mark["y"], lse, want_dq=False, dk=dk, **how)
    assert torch.equal(dk, mark["dk"]) and torch.equal(got["dv"], made["dv"])


def used_rows(n, rows, lengths):
    return torch.arange(rows, device="cuda")[None] < torch.tensor(lengths, device="cuda").clamp(0, rows)[:, None]


@pytest.mark.parametrize("dim", [64, 36, 128])
@pytest.mark.parametrize("lq,lk", [([70, 1, 0, 40], [70, 100, 30, 0]), ([0, 0, 0, 0], [3, 0, 0, 0]), ([90, 70, 80, -5], [120, 400, 99, 1])])
def test_padded_batch(H, dim, lq, lk):
    both_ways(H, (4, 90, 4, dim), (4, 120, 2, dim), BF16, used_rows(4, 90, lq), used_rows(4, 120, lk),
              dict(causal=True, q_lengths=ints(lq), k_lengths=ints(lk)))


def test_one_length_alone(H):
    every = used_rows(2, 50, [50, 50])
    both_ways(H, (2, 50, 2, 64), (2, 50, 2, 64), FP16, used_rows(2, 50, [9, 50]), every, dict(q_lengths=ints([9, 50])))
    both_ways(H, (2, 50, 2, 64), (2, 50, 2, 64), FP16, every, used_rows(2, 50, [50, 1]), dict(k_lengths=ints([50, 1])))


@pytest.mark.parametrize("offsets_q,offsets_k", [([0, 5, 90], [0, 7, 100]), ([9, 9, 60], [20, 50, 50]), ([30], [10]), ([0, 0], [0, 0]), ([100, 100], [120, 120]), ([-9, 40], [5, 500])])
@pytest.mark.parametrize("dim", [64, 33])
def test_documents(H, offsets_q, offsets_k, dim):
    def used(rows, off):
        at, off = torch.arange(rows, device="cuda"), [min(max(o, 0), rows) for o in off]
        return (at >= off[0]) & (at < off[-1])

    both_ways(H, (100, 4, dim), (120, 2, dim), BF16, used(100, offsets_q), used(120, offsets_k),
              dict(causal=True, q_offsets=ints(offsets_q), k_offsets=ints(offsets_k)))


def test_captured(H):
    """lengths that change between replays"""
    q, k, v, dy, lse = tensors((2, 40, 2, 64), (2, 40, 2, 64), BF16)
    lengths = ints([40, 40])
    leave_nan()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = H.heddle_attention(q, k, v, lse=lse, q_lengths=lengths, k_lengths=lengths)
        grads = H.heddle_attention_backward(dy, q, k, v, y, lse, q_lengths=lengths, k_lengths=lengths)
    for now in ([40, 40], [3, 17], [0, 40]):
        lengths.copy_(ints(now))
        graph.replay()
        torch.cuda.synchronize()
        used = used_rows(2, 40, now)
        for n, t in (("y", y), *grads.items()):
            assert not t[~used].any() and bool(torch.isfinite(t).all()), (n, now)
        assert torch.equal(y, H.heddle_attention(q, k, v, q_lengths=lengths, k_lengths=lengths))


@pytest.mark.parametrize("n,lq,lk,hq,hk,dim", [(2, 640, 640, 104, 52, 64), (2, 600, 700, 54, 54, 128), (4, 300, 290, 44, 22, 128), (300, 3, 40, 2, 2, 64), (700, 2, 5, 1, 1, 24),
                                               (40, 1, 3000, 8, 8, 128), (3, 2, 4000, 8, 2, 64)])
def test_kernels(H, n, lq, lk, hq, hk, dim):
    """256 and 128 rows and keys a workgroup, few of them, more sequences than workgroups that clear, keys in one part and several"""
    queries, keys = [(7 * j) % (lq + 1) for j in range(n)], [lk - (31 * j) % lk for j in range(n)]
    both_ways(H, (n, lq, hq, dim), (n, lk, hk, dim), BF16, used_rows(n, lq, queries), used_rows(n, lk, keys),
              dict(causal=True, q_lengths=ints(queries), k_lengths=ints(keys)))


@pytest.mark.parametrize("lengths,heads,kv_heads", [([700, 0, 513, 640, 1, 1200, 900], 32, 16), ([300, 0, 129, 257, 1], 60, 60), ([640] * 66, 4, 2), ([1, 2, 1], 4, 4)])
@pytest.mark.parametrize("lead,tail", [(0, 0), (300, 0), (0, 1), (5, 2000)])
def test_kernels_of_documents(H, lengths, heads, kv_heads, lead, tail):
    rows, offsets = lead + sum(lengths) + tail, [lead + sum(lengths[:i]) for i in range(len(lengths) + 1)]
    at = torch.arange(rows, device="cuda")
    used = (at >= lead) & (at < rows - tail)
    both_ways(H, (rows, heads, 64), (rows, kv_heads, 64), FP16, used, used, dict(causal=True, q_offsets=ints(offsets), k_offsets=ints(offsets)))
