"""Attention's outputs on what it reads, in every order of dimensions. Without a GPU; the
addresses are of no memory."""
import itertools
import random

import pytest

from paper_2609_34244_amd import heddle as H
from test_layer_abi import MB, attention, no_gpu, refused, three

P = 300 * MB                           # far from the tensors that are not named

pytestmark = no_gpu


@pytest.fixture(scope="module")
def L():
    return H.lib()


def strides(order, sizes, gaps=(0, 0, 0)):
    """(sequence, row, head) distances; order: the dimensions from the innermost on; gaps: values left out after each"""
    st, extent = [0, 0, 0], sizes[3]
    for i, gap in zip(order, gaps):
        st[i] = extent + gap
        extent += (sizes[i] - 1) * st[i] + gap
    return st


def values(p, st, sizes):
    return {p // 2 + s * st[0] + r * st[1] + h * st[2] + c for s in range(sizes[0]) for r in range(sizes[1]) for h in range(sizes[2]) for c in range(sizes[3])}


@pytest.mark.parametrize("order", itertools.permutations(range(3)))
def test_a_row_into_an_input(L, order):
    """y on q's memory, some rows or values on: with the same strides, dense and with gaps that hold another tensor"""
    sizes = (2, 40, 4, 64)
    dense = strides(order, sizes)
    assert refused(L, attention(y=P, q=P, q_strides=three(*dense), y_strides=three(*dense)), "forward")
    for d in dense:
        assert refused(L, attention(q=P, y=P + 2 * d, q_strides=three(*dense), y_strides=three(*dense)), "forward"), d
        assert refused(L, attention(q=P + 2 * d, y=P, q_strides=three(*dense), y_strides=three(*dense)), "forward"), d
    total = 2 * 40 * 4 * 64
    assert not refused(L, attention(q=P, y=P + 2 * total, q_strides=three(*dense), y_strides=three(*dense)), "forward")
    wide = strides(order, sizes, (64, 0, 0))
    for at, apart in ((64, True), (63, False), (65, False), (64 + 3 * 128, True), (3 * 128, False), (-64, True), (-63, False), (64 - 5 * 128, True)):
        d = attention(q=P, y=P + 2 * at, q_strides=three(*wide), y_strides=three(*wide))
        assert refused(L, d, "forward") != apart, at
        d = attention(dy=P, dq=P + 2 * at, dy_strides=three(*wide), dq_strides=three(*wide))
        assert refused(L, d, "backward") != apart, at


def test_gradients_in_one_buffer(L):
    """[sequences][heads of q, k and v][rows][64]: apart by whole heads, not by less"""
    st = three(8 * 50 * 64, 64, 50 * 64)
    one = dict(k_len=40, **{f"{t}_strides": st for t in ("dq", "dk", "dv")})
    head = 2 * 50 * 64
    assert not refused(L, attention(**one, dq=P, dk=P + 4 * head, dv=P + 6 * head), "backward")
    for dk, dv in ((3, 6), (4, 5), (7, 6), (4, 7)):
        assert refused(L, attention(**one, dq=P, dk=P + dk * head, dv=P + dv * head), "backward"), (dk, dv)


def test_against_all_addresses(L):
    """small tensors of random orders, gaps and distances between them"""
    rng, seen = random.Random(5), set()
    for _ in range(1500):
        n, lq, lk, hk, group, dim = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 2), rng.randint(1, 2), rng.choice([1, 2, 3, 8])
        t = {}
        for name, rows, heads in (("q", lq, hk * group), ("k", lk, hk), ("y", lq, hk * group)):
            sizes = (n, rows, heads, dim)
            if name == "y" and rng.random() < 0.4:
                st = t["q"][1]
            else:
                st = strides(rng.sample(range(3), 3), sizes, [rng.choice([0, 0, 1, dim, 9]) for _ in range(3)])
            t[name] = (P + 2 * (0 if name == "q" else rng.randint(-120, 120)), st, sizes)
        d = dict(sequences=n, q_len=lq, k_len=lk, heads=hk * group, kv_heads=hk, dim=dim)
        for name, (p, st, _) in t.items():
            d[name], d[f"{name}_strides"] = p, three(*st)
        d.update(v_strides=three(*t["k"][1]))
        all_ = {name: values(*v) for name, v in t.items()}
        want = bool(all_["y"] & (all_["q"] | all_["k"]))
        seen.add(want)
        assert refused(L, attention(**d), "forward") == want, (d, t)
    assert seen == {True, False}


def test_long_tensors(L):
    """the largest sizes and distances: an answer at once"""
    far = three(2 ** 61, 2 ** 22, 64)
    d = dict(sequences=65535, q_len=2 ** 20, k_len=2 ** 30, heads=512, kv_heads=512, q_strides=far, k_strides=far, v_strides=far)
    for y in (P, P + 2 ** 23 * 77 + 2):
        desc = attention(**d, q=P, y=y, y_strides=three(2 ** 61, 2 ** 22, 64))
        assert L.heddle_attention(H.C.byref(desc), 512 << 20, 1 << 60, None) in (H.HEDDLE_E_INVAL, H.HEDDLE_E_RANGE)
    long = dict(sequences=1, q_len=2 ** 20, k_len=2 ** 20, heads=1, kv_heads=1, q=P, k=P + 2 ** 34, v=P + 2 ** 35)
    assert not refused(L, attention(**long, q_strides=three(0, 300, 64), y=P + 2 ** 36, y_strides=three(0, 256, 64)), "forward")
    assert refused(L, attention(**long, q_strides=three(0, 300, 64), y=P + 2, y_strides=three(0, 257, 64)), "forward")
