"""Attention and its gradients against the plain 64-bit form, every value
within the bound that the roundings allow. Needs an MI355X."""
import itertools
import random

import pytest
import torch

import layer_reference as R
from ffn_reference import rounded
from layer_common import Maker, ints, near

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def strides_of(layout, n, rows, heads, dim):
    """strides of [n, rows, heads, dim]"""
    if layout == "heads":                    # [n][heads][rows][dim]
        return [heads * rows * dim, dim, rows * dim, 1]
    if layout == "odd":
        return [rows * (heads * (dim + 1) + 3) + 5, heads * (dim + 1) + 3, dim + 1, 1]
    if layout == "fused":                    # a part of wider rows
        return [rows * (heads * dim + 64), heads * dim + 64, dim, 1]
    return [rows * heads * dim, heads * dim, dim, 1]


def run(H, seed, queries, keys, hq, hk, dim, dtype=BF16, causal=False, cap=0.0, slopes=False, prefix=None, packed=False, layout="plain",
        room=(0, 0), scale=None, train=True, magnitude=1.0, lead=0):
    """queries, keys: lengths of the sequences. Not packed: rows of room more than the longest. lead: rows before
    the first packed document, which belong to none."""
    print(f"attention {queries} {keys} {hq}/{hk} {dim} {dtype} causal={causal} cap={cap} slopes={slopes} prefix={prefix} packed={packed} "
          f"{layout} room={room}", flush=True)
    mk, n = Maker(seed), len(queries)
    if packed:
        rq, rk = lead + sum(queries) + room[0], lead + sum(keys) + room[1]
        oq, ok = [lead + sum(queries[:i]) for i in range(n + 1)], [lead + sum(keys[:i]) for i in range(n + 1)]
    else:
        rq, rk = max(queries) + room[0], max(keys) + room[1]

    def tensor(rows, heads, size=None, shift=0):
        st = strides_of(layout, 1 if packed else n, rows, heads, dim)
        shape = [rows, heads, dim] if packed else [n, rows, heads, dim]
        return mk.part(shape, dtype, st[1:] if packed else st, shift if layout in ("odd", "fused") else 0, size)

    q, k, v = tensor(rq, hq, magnitude, 3 if layout == "odd" else 8), tensor(rk, hk, magnitude, 1 if layout == "odd" else 16), tensor(rk, hk, 1.0, 8)
    y, dy = tensor(rq, hq), tensor(rq, hq, 1.0)
    dq, dk, dv = tensor(rq, hq), tensor(rk, hk), tensor(rk, hk)
    lse = torch.full(q.shape[:-1], float("nan"), device="cuda")
    sl = torch.tensor([2.0 ** (-0.5 * (h + 1)) for h in range(hq)], device="cuda") if slopes else None

    def rows_of(i, which):
        if packed:
            return slice((oq if which == "q" else ok)[i], (oq if which == "q" else ok)[i + 1])
        return (i, slice(0, (queries if which == "q" else keys)[i]))

    # rows of no sequence hold NaN, and their outputs a value that has to stay
    mark = 7.0
    used = {"q": torch.zeros(q.shape[:-2], dtype=torch.bool, device="cuda"), "k": torch.zeros(k.shape[:-2], dtype=torch.bool, device="cuda")}
    for i in range(n):
        used["q"][rows_of(i, "q")] = True
        used["k"][rows_of(i, "k")] = True
    for t, which in ((q, "q"), (dy, "q"), (k, "k"), (v, "k")):
        t[~used[which]] = float("nan")
    for t in (y, dq, dk, dv):
        t.fill_(mark)
    how = dict(scale=scale, causal=causal, cap=cap, slopes=sl, prefix=None if prefix is None else ints(prefix))
    if packed:
        how.update(q_offsets=ints(oq), k_offsets=ints(ok))
    elif room != (0, 0) or len(set(queries)) > 1 or len(set(keys)) > 1:
        how.update(q_lengths=ints(queries), k_lengths=ints(keys))
    H.heddle_attention(q, k, v, lse=lse, out=y, **how)
    if train:
        y[~used["q"]] = float("nan")
        H.heddle_attention_backward(dy, q, k, v, y, lse, dq=dq, dk=dk, dv=dv, **how)
        y[~used["q"]] = mark
    torch.cuda.synchronize()
    for name, t, which in (("y", y, "q"), ("dq", dq, "q"), ("dk", dk, "k"), ("dv", dv, "k")):
        assert bool((t[~used[which]] == mark).all()), f"{name}: rows of no sequence were written"
    assert bool(torch.isnan(lse[~used["q"]]).all())
    group, sc = hq // hk, dim ** -0.5 if scale is None else scale
    for i in range(n):
        for h in range(hk):
            sums = {}
            for g in range(group):
                at = h * group + g
                p = dict(scale=sc, causal=causal, cap=cap, slope=None if sl is None else float(sl[at]), prefix=0 if prefix is None else prefix[i])
                qi, ki, vi = q[rows_of(i, "q")][:, at], k[rows_of(i, "k")][:, h], v[rows_of(i, "k")][:, h]
                yi, li = y[rows_of(i, "q")][:, at], lse[rows_of(i, "q")][:, at]
                want, bound, wl, bl = R.attention(qi, ki, vi, dtype, **p)
                near(li, wl, bl, f"lse of sequence {i}, head {at}")
                near(yi, want, bound, f"y of sequence {i}, head {at}")
                if train:
                    got = R.attention_backward(dy[rows_of(i, "q")][:, at], qi, ki, vi, yi, wl, bl, dtype, **p)
                    w, e = got["dq"]
                    near(dq[rows_of(i, "q")][:, at], w, rounded(w, e, dtype), f"dq of sequence {i}, head {at}")
                    for name in ("dk", "dv"):
                        w, e = sums.get(name, (0.0, 0.0))
                        sums[name] = (w + got[name][0], e + got[name][1] + group * R.E * got[name][0].abs())
            if train:
                for name, t in (("dk", dk), ("dv", dv)):
                    w, e = sums[name]
                    near(t[rows_of(i, "k")][:, h], w, rounded(w, e, dtype), f"{name} of sequence {i}, head {h}")
    mk.untouched()


LENGTHS = [(1, 1), (1, 2), (2, 1), (3, 3), (1, 31), (1, 32), (1, 33), (1, 300), (5, 64), (31, 65), (32, 32), (33, 33), (63, 64), (64, 63), (65, 129),
           (127, 128), (128, 127), (129, 129), (200, 77), (77, 200), (257, 257)]


@pytest.mark.parametrize("lq,lk", LENGTHS)
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(H, lq, lk, causal):
    run(H, lq * 3 + lk, [lq], [lk], 2, 1, 64, BF16, causal)
    run(H, lq * 5 + lk, [lq], [lk], 1, 1, 128, FP16, causal)


@pytest.mark.parametrize("dim", [1, 2, 7, 8, 15, 16, 24, 40, 56, 63, 64, 65, 72, 80, 96, 100, 112, 120, 127, 128])
@pytest.mark.parametrize("lq", [1, 70])
def test_widths(H, dim, lq):
    run(H, dim, [lq], [90], 2, 2, dim, BF16 if dim % 2 else FP16, True)


@pytest.mark.parametrize("cap,slopes,prefix,causal", [c for c in itertools.product([0.0, 5.0], [False, True], [None, 20, 500, -3], [True, False])])
@pytest.mark.parametrize("lq,lk", [(1, 75), (90, 75), (75, 150)])
def test_masks(H, cap, slopes, prefix, causal, lq, lk):
    """rows that see nothing among them: more queries than keys"""
    run(H, 11, [lq], [lk], 2, 1, 64, BF16, causal, cap, slopes, None if prefix is None else [prefix])


@pytest.mark.parametrize("cap,slopes", [(0.0, False), (30.0, False), (0.0, True), (20.0, True)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_modified_wide(H, cap, slopes, dtype):
    run(H, 12, [140], [140], 2, 1, 128, dtype, True, cap, slopes, [50])


@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (3, 1), (5, 1), (8, 2), (12, 4), (64, 8), (16, 1)])
@pytest.mark.parametrize("lq", [1, 4, 40])
def test_heads(H, hq, hk, lq):
    run(H, hq + lq, [lq, lq], [60, 60], hq, hk, 64, BF16, True, 0.0, hq % 2 == 0)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lead", [0, 150])
def test_documents(H, causal, lead):
    run(H, 21, [5, 0, 130, 1, 64, 0, 129], [5, 0, 130, 1, 64, 0, 129], 4, 2, 64, BF16, causal, packed=True, room=(9, 9), lead=lead)
    run(H, 22, [40, 3, 0, 90], [10, 70, 20, 90], 2, 2, 128, FP16, causal, 0.0, True, [0, 30, 5, 45], packed=True, room=(70, 3), lead=lead)


def test_many_documents(H):
    """more than a search looks at in a step, most of them short"""
    r = random.Random(3)
    lengths = [r.choice([0, 1, 1, 2, 3, 9, 33]) for _ in range(300)]
    run(H, 23, lengths, lengths, 1, 1, 64, BF16, True, packed=True, room=(2, 0))
    run(H, 24, [1] * 70, [r.randint(0, 40) for _ in range(70)], 4, 1, 64, BF16, True, packed=True)


@pytest.mark.parametrize("causal", [False, True])
def test_batches_with_room(H, causal):
    """lengths of their own, garbage behind them"""
    run(H, 31, [70, 1, 0, 40], [70, 100, 30, 0], 4, 2, 64, BF16, causal, room=(3, 60))
    run(H, 32, [1, 1, 1], [1, 257, 64], 8, 1, 128, FP16, causal, 10.0, True, room=(0, 40))
    run(H, 33, [3, 2], [500, 90], 4, 4, 64, BF16, causal, room=(0, 0))


@pytest.mark.parametrize("layout", ["plain", "heads", "odd", "fused"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dim", [64, 36, 128])
def test_layouts(H, layout, packed, dim):
    if packed and layout == "heads":
        pytest.skip("packed rows have no sequences to stride over")
    run(H, 41, [50, 20], [50, 70], 4, 2, dim, BF16, True, packed=packed, layout=layout, room=(2, 2))
    run(H, 42, [1, 2], [80, 70], 4, 2, dim, FP16, True, packed=packed, layout=layout, room=(0, 6))


@pytest.mark.parametrize("magnitude", [0.0, 0.01, 6.0])
@pytest.mark.parametrize("lq", [1, 100])
def test_magnitudes(H, magnitude, lq):
    """uniform rows, and rows whose maximum moves far while keys pass"""
    run(H, 51, [lq], [400], 2, 2, 64, BF16, True, magnitude=magnitude)
    run(H, 52, [lq], [400], 2, 2, 64, FP16, False, 50.0, magnitude=magnitude, train=magnitude < 1)


@pytest.mark.parametrize("cap,scale", [(0.5, None), (4096.0, 0.3), (0.0, 2.0), (0.0, 1e-6), (1e-3, 1.0)])
def test_extremes_of_cap_and_scale(H, cap, scale):
    run(H, 55, [40], [90], 2, 1, 64, BF16, True, cap, scale=scale)
    run(H, 56, [1], [300], 4, 1, 64, BF16, True, cap, True, scale=scale)


@pytest.mark.parametrize("lq,lk,hq,hk", [(1, 5000, 4, 1), (2, 3001, 2, 2), (1, 20000, 1, 1), (16, 2100, 4, 4), (100, 4000, 4, 2)])
def test_long_caches(H, lq, lk, hq, hk):
    """keys divided over workgroups"""
    run(H, 61, [lq], [lk], hq, hk, 128, BF16, True, 0.0, True, train=False)
    run(H, 62, [lq, lq, lq], [lk, 100, lk // 2 + 1], hq, hk, 64, FP16, True, 20.0, train=False, room=(0, 1))


def test_long(H):
    run(H, 63, [1500], [1500], 2, 1, 128, BF16, True)


def test_nothing(H):
    q, k = torch.empty(2, 0, 4, 64, dtype=BF16, device="cuda"), torch.ones(2, 5, 2, 64, dtype=BF16, device="cuda")
    assert H.heddle_attention(q, k, k).shape == (2, 0, 4, 64)
    got = H.heddle_attention_backward(q, q, k, k, q, torch.empty(2, 0, 4, device="cuda"))
    assert got["dq"].numel() == 0 and not got["dk"].any() and not got["dv"].any()
    empty = torch.empty(0, 4, 64, dtype=BF16, device="cuda")
    assert H.heddle_attention(empty, empty, empty, q_offsets=ints([0]), k_offsets=ints([0])).numel() == 0
    q, k = torch.ones(1, 3, 4, 64, dtype=BF16, device="cuda"), torch.empty(1, 0, 4, 64, dtype=BF16, device="cuda")
    lse = torch.zeros(1, 3, 4, device="cuda")
    assert not H.heddle_attention(q, k, k, lse=lse).any() and bool((lse == -float("inf")).all())
    assert not H.heddle_attention_backward(q, q, k, k, torch.zeros_like(q), lse)["dq"].any()


@pytest.mark.parametrize("offsets", [[0, 300, 20], [50, 10, 400], [-7, 30, 90], [90, 90, 90], [0, 2**31 - 1, -2**31]])
def test_offsets_that_are_none(H, offsets):
    """no access leaves the tensors, and the call ends"""
    mk = Maker(5)
    q, k, v, dy = (mk.part((100, 2, 64), BF16, scale=1.0) for _ in range(4))
    y, dq, dk, dv = (mk.part((100, 2, 64), BF16) for _ in range(4))
    for t in (y, dq, dk, dv):
        t.zero_()
    lse = torch.zeros(100, 2, device="cuda")
    how = dict(causal=True, q_offsets=ints(offsets), k_offsets=ints(offsets))
    H.heddle_attention(q, k, v, out=y, lse=lse, **how)
    H.heddle_attention_backward(dy, q, k, v, y, lse, dq=dq, dk=dk, dv=dv, **how)
    mk.untouched()


def test_parts_of_the_gradient(H):
    mk = Maker(6)
    q, k, v, dy = (mk.part((1, 60, 2, 64), BF16, scale=1.0) for _ in range(4))
    lse = torch.empty(1, 60, 2, device="cuda")
    y = H.heddle_attention(q, k, v, causal=True, lse=lse)
    both = H.heddle_attention_backward(dy, q, k, v, y, lse, causal=True)
    one = H.heddle_attention_backward(dy, q, k, v, y, lse, causal=True, want_dkv=False)
    two = H.heddle_attention_backward(dy, q, k, v, y, lse, causal=True, want_dq=False)
    assert set(one) == {"dq"} and set(two) == {"dk", "dv"}
    for part in (one, two):
        for name, t in part.items():
            assert torch.equal(t, both[name]), name


@pytest.mark.parametrize("cap", [0.0, 4.0])
def test_gradients_against_differences(H, cap):
    """sum dy y along a direction: a central difference of the exact form, off by h^2 of its third derivative; the call's
    gradients are off by the bounds of test_masks, here taken as 3% of the gradient's norm"""
    g = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, dy = (torch.randn(1, 24, 1, 16, generator=g, device="cuda").to(FP16) for _ in range(4))
    lse = torch.empty(1, 24, 1, device="cuda")
    y = H.heddle_attention(q, k, v, causal=True, cap=cap, lse=lse)
    got = H.heddle_attention_backward(dy, q, k, v, y, lse, causal=True, cap=cap)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        step = torch.randn(t.shape, generator=g, device="cuda").double()
        f = lambda h: float((dy[0, :, 0].double() * R.attention(*(x[0, :, 0].double() + (h * step[0, :, 0] if x is t else 0) for x in (q, k, v)),  # noqa: E731
                                                                FP16, 0.25, True, cap)[0]).sum())
        slope = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(slope - float((got[name].double() * step).sum())) <= 0.03 * float(got[name].double().norm()) + 1e-4, name


def test_two_streams_and_a_graph(H):
    """a call on another stream than the current one, and a captured pair of calls replayed between eager ones"""
    mk = Maker(9)
    q, k, v, dy = (mk.part((2, 100, 4, 64), BF16, scale=1.0) for _ in range(4))
    lse = torch.empty(2, 100, 4, device="cuda")
    want = H.heddle_attention(q, k, v, causal=True, lse=lse)
    grads = H.heddle_attention_backward(dy, q, k, v, want, lse, causal=True)
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = H.heddle_attention(q, k, v, causal=True, stream=other)
    other.synchronize()
    assert torch.equal(got, want)
    q1, k1 = q[:, -1:].contiguous(), k.repeat(1, 8, 1, 1)                   # a decode step in parts
    v1 = v.repeat(1, 8, 1, 1)
    one = H.heddle_attention(q1, k1, v1)
    graph, g = torch.cuda.CUDAGraph(), {}
    with torch.cuda.graph(graph):
        l2 = torch.empty_like(lse)
        g["y"] = H.heddle_attention(q, k, v, causal=True, lse=l2)
        g.update(H.heddle_attention_backward(dy, q, k, v, g["y"], l2, causal=True))
        g["one"] = H.heddle_attention(q1, k1, v1)
    for _ in range(3):
        for t in g.values():
            t.zero_()
        graph.replay()
        again = H.heddle_attention(q, k, v, causal=True)
        torch.cuda.synchronize()
        assert torch.equal(again, want) and torch.equal(g["y"], want) and torch.equal(g["one"], one)
        for name, t in grads.items():
            assert torch.equal(g[name], t), name


def test_far_into_a_cache(H):
    """sequences whose values lie past 2^31 elements"""
    k = torch.zeros(3, 9000, 8, 10000, dtype=BF16, device="cuda")[..., :64]   # 2.16e9 elements, 4.3 GB
    g = torch.Generator(device="cuda").manual_seed(1)
    k.copy_(torch.randn(3, 9000, 8, 64, generator=g, device="cuda"))
    q = torch.randn(3, 1, 8, 64, generator=g, device="cuda").to(BF16)
    y = H.heddle_attention(q, k, k, k_lengths=ints([9000, 17, 8999]))
    for i, n in ((0, 9000), (1, 17), (2, 8999)):
        for h in (0, 7):
            want, bound, _, _ = R.attention(q[i, :, h], k[i, :n, h], k[i, :n, h], BF16, 0.125)
            near(y[i, :, h], want, bound, f"sequence {i}, head {h}")


def test_requires_grad(H):
    q, k, v = (torch.ones(1, 4, 2, 16, dtype=BF16, device="cuda") for _ in range(3))
    want = H.heddle_attention(q, k, v)
    for i in range(3):
        given = [t.clone().requires_grad_(i == j) for j, t in enumerate((q, k, v))]
        with pytest.raises(H.HeddleError, match="no_grad"):
            H.heddle_attention(*given)
        with torch.no_grad():
            assert torch.equal(H.heddle_attention(*given), want)


def test_refusals(H):
    q, k = torch.ones(1, 4, 4, 16, dtype=BF16, device="cuda"), torch.ones(1, 6, 2, 16, dtype=BF16, device="cuda")
    o = ints([0, 4])
    lse = torch.zeros(1, 4, 4, device="cuda")
    for call in (lambda: H.heddle_attention(q, k, k[:, :5]), lambda: H.heddle_attention(q, k.half(), k), lambda: H.heddle_attention(q.cpu(), k, k),
                 lambda: H.heddle_attention(q, k[:, :, :, :8], k[:, :, :, :8]), lambda: H.heddle_attention(q[:, :, :3], k, k),
                 lambda: H.heddle_attention(q, k, k, scale=0.0), lambda: H.heddle_attention(q, k, k, scale=float("nan")),
                 lambda: H.heddle_attention(q, k, k, cap=-1.0), lambda: H.heddle_attention(q, k, k, prefix=o),
                 lambda: H.heddle_attention(q, k, k, q_offsets=o, k_offsets=o), lambda: H.heddle_attention(q[0], k[0], k[0], q_offsets=o),
                 lambda: H.heddle_attention(q, k, k, slopes=torch.ones(3, device="cuda")), lambda: H.heddle_attention(q, k, k, k_lengths=o.long()[:1]),
                 lambda: H.heddle_attention(q, k, k, out=q), lambda: H.heddle_attention(q.float(), k.float(), k.float()),
                 lambda: H.heddle_attention(q, k, k.transpose(2, 3).contiguous().transpose(2, 3)), lambda: H.heddle_attention(q, k, k, lse=lse[..., 0]),
                 lambda: H.heddle_attention_backward(q, q, k, k, q, None), lambda: H.heddle_attention_backward(q, q, k, k, q, lse, dk=k),
                 lambda: H.heddle_attention(torch.ones(1, 2, 1, 136, dtype=BF16, device="cuda"), *2 * [torch.ones(1, 2, 1, 136, dtype=BF16, device="cuda")])):
        with pytest.raises(H.HeddleError) as e:
            call()
        assert e.value.code == H.HEDDLE_E_INVAL


@pytest.mark.parametrize("a,b,c,want", [(2.0 ** -12, 2.0 ** -11, 2.0 ** 10, 2.0 ** -13), (2.0 ** -7, 2.0 ** -6, 2.0 ** 10, 2.0 ** -3),
                                        (2.0 ** -13, 2.0 ** -12, 2.0 ** 10, 0.0), (2.0 ** 8, 2.0 ** 8, 2.0 ** -3, 2.0 ** 13),
                                        (2.0 ** 9, 2.0 ** 9, 2.0 ** -4, float("inf"))])
def test_range_of_float16_gradients(H, a, b, c, want):
    """Two keys of equal scores, values b and -b, dy a: y = 0, D = 0, dS = a b / 2 and -a b / 2, dq = 2 c dS for keys c and
    -c. dS is 2^-24 (the smallest float16), 2^-14, 2^-26 (0 when rounded), 2^15 and 2^17 (past the largest). P is off by
    some 2^-22, far from half a step of dS, and all else is a power of two: dq is what it should be, to its rounding."""
    q, k, v, dy = torch.zeros(1, 1, 1, 16), torch.zeros(1, 2, 1, 16), torch.zeros(1, 2, 1, 16), torch.zeros(1, 1, 1, 16)
    k[0, :, 0, 0], v[0, :, 0, 0], dy[..., 0] = torch.tensor([c, -c]), torch.tensor([b, -b]), a
    q, k, v, dy = (t.half().cuda() for t in (q, k, v, dy))
    lse = torch.empty(1, 1, 1, device="cuda")
    y = H.heddle_attention(q, k, v, scale=1.0, lse=lse)
    dq = float(H.heddle_attention_backward(dy, q, k, v, y, lse, scale=1.0)["dq"][0, 0, 0, 0])
    assert dq == want or abs(dq - want) <= 2.0 ** -11 * want, dq
