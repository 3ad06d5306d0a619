"""Outputs of the feed-forward and gradient operators that lie on what the call
reads, or on each other: refused on the host, before any device work. The
addresses are of no memory; a call that is not refused ends for want of a GPU."""
import ctypes as C
import itertools
import random

import pytest
import torch

from paper_2609_34244_amd import heddle as H

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run on no memory")

M, N, K = 40, 96, 64            # rows, columns of Y and of X
MB = 1 << 20


@pytest.fixture(scope="module")
def L():
    return H.lib()


def place(names):
    """an address apart from the others for every name"""
    return {n: MB * (i + 16) for i, n in enumerate(names)}


def linear(**over):
    d = dict(dtype=H.HEDDLE_T_BF16, act=H.HEDDLE_A_NONE, m=M, n=N, k=K, ldx=K, ldw=K, ldr=N, ldp=N, ldy=N, lddy=N, lddx=K, lddw=K)
    d.update(place(["x", "w", "bias", "residual", "preact", "y", "dy", "dx", "dw", "db"]))
    d.update(over)
    return H.heddle_linear_desc(**d)


def ffn(**over):
    d = dict(dtype=H.HEDDLE_T_BF16, act=H.HEDDLE_A_SILU, t=M, d=K, f=N, ldx=K, ldw_in=K, ldw_out=N, ldr=K, ldp=2 * N, ldy=K,
             lddy=K, lddx=K, lddw_in=K, lddw_out=N)
    d.update(place(["x", "w_in", "w_out", "residual", "preact", "y", "dy", "dx", "dw_in", "dw_out"]))
    d.update(over)
    return H.heddle_gated_ffn_desc(**d)


def run(call, desc):
    """True: refused as an overlap"""
    rc = call(C.byref(desc), 256 * MB, 64 * MB, None)
    if rc == H.HEDDLE_E_INVAL:
        assert "overlaps" in H.heddle_last_error(), H.heddle_last_error()
        return True
    assert rc == H.HEDDLE_E_DEVICE, (rc, H.heddle_last_error())
    return False


def at(desc, name):
    return getattr(desc, name)


FORWARD = [("y", "x"), ("y", "w"), ("y", "bias"), ("y", "preact"), ("preact", "x"), ("preact", "w"), ("preact", "bias"),
           ("preact", "residual")]


@pytest.mark.parametrize("m", [3, M])
@pytest.mark.parametrize("out,on", FORWARD)
def test_linear(L, m, out, on):
    d = linear(m=m, n=K, ldy=K, ldr=K, ldp=K)
    assert not run(L.heddle_linear, d)
    for shift in (0, 2, -2):
        assert run(L.heddle_linear, linear(m=m, n=K, ldy=K, ldr=K, ldp=K, **{out: at(d, on) + shift})), shift


def test_linear_residual(L):
    """y may be the residual itself, but not lie on another row's residual"""
    d = linear()
    assert not run(L.heddle_linear, linear(y=at(d, "residual")))
    assert run(L.heddle_linear, linear(y=at(d, "residual") + 2 * N))
    assert run(L.heddle_linear, linear(y=at(d, "residual"), ldy=2 * N))
    assert not run(L.heddle_linear, linear(m=1, y=at(d, "residual"), ldy=2 * N))


@pytest.mark.parametrize("out,on,act", [(o, i, a) for (o, i), a in itertools.product(
    [("dx", "dy"), ("dx", "w"), ("dx", "x"), ("dx", "dw"), ("dw", "x"), ("dw", "dy"), ("db", "dy"), ("db", "x"), ("db", "w"),
     ("db", "dx"), ("db", "dw")], [H.HEDDLE_A_NONE, H.HEDDLE_A_SILU])] + [("db", "preact", H.HEDDLE_A_SILU)])
def test_linear_backward(L, out, on, act):
    d = linear(act=act)
    assert not run(L.heddle_linear_backward, d)
    # with an activation the products read dZ, not dy
    fine = act != H.HEDDLE_A_NONE and on == "dy" and out != "db"
    assert run(L.heddle_linear_backward, linear(act=act, **{out: at(d, on)})) == (not fine)


def test_linear_backward_reads_only_what_it_needs(L):
    d = linear()
    assert not run(L.heddle_linear_backward, linear(dx=at(d, "x"), dw=None))
    assert not run(L.heddle_linear_backward, linear(dw=at(d, "w"), dx=None))
    assert not run(L.heddle_linear_backward, linear(db=at(d, "preact")))


@pytest.mark.parametrize("out,on", [("y", "w_out"), ("y", "preact"), ("preact", "x"), ("preact", "w_in"), ("preact", "w_out"),
                                    ("preact", "residual")])
def test_ffn(L, out, on):
    d = ffn()
    assert run(L.heddle_gated_ffn, ffn(**{out: at(d, on)}))


def test_ffn_in_place(L):
    """y over x: the block has read x when it writes y"""
    d = ffn()
    assert not run(L.heddle_gated_ffn, d)
    assert not run(L.heddle_gated_ffn, ffn(y=at(d, "x"), residual=at(d, "x")))
    assert not run(L.heddle_gated_ffn, ffn(y=at(d, "residual")))
    assert run(L.heddle_gated_ffn, ffn(y=at(d, "residual") + 2))


@pytest.mark.parametrize("out,on", [("dx", "w_in"), ("dx", "x"), ("dx", "dy"), ("dx", "dw_in"), ("dx", "dw_out"), ("dw_in", "x"),
                                    ("dw_in", "dy"), ("dw_in", "dw_out"), ("dw_out", "dy")])
def test_ffn_backward(L, out, on):
    d = ffn()
    assert not run(L.heddle_gated_ffn_backward, d)
    assert run(L.heddle_gated_ffn_backward, ffn(**{out: at(d, on)}))


def test_ffn_backward_reads_only_what_it_needs(L):
    d = ffn()
    assert not run(L.heddle_gated_ffn_backward, ffn(dx=at(d, "dy"), dw_out=None))
    assert not run(L.heddle_gated_ffn_backward, ffn(dx=at(d, "x"), dw_in=None))


def test_matrices_in_one(L):
    """two matrices side by side in wider rows do not overlap, shifted by a column they do; x: [M][K], y: [M][N]"""
    wide = K + N
    base = 16 * MB
    fine = dict(x=base, ldx=wide, y=base + 2 * K, ldy=wide, m=M)
    assert not run(L.heddle_linear, linear(**fine))
    assert run(L.heddle_linear, linear(**{**fine, "y": base + 2 * K - 2}))
    assert run(L.heddle_linear, linear(**{**fine, "y": base + 2 * K + 2}))       # its rows end in x's next ones
    assert not run(L.heddle_linear, linear(**{**fine, "y": base + 2 * K + 2, "m": 1}))
    assert not run(L.heddle_linear, linear(**{**fine, "y": base - 2 * N, "x": base}))
    # stacked: y's first row after x's last
    assert not run(L.heddle_linear, linear(x=base, ldx=wide, y=base + 2 * ((M - 1) * wide + K), ldy=wide))
    # a run of values in the gap of wider rows, and one into the next row
    assert not run(L.heddle_linear, linear(x=base, ldx=wide, bias=None, m=M, y=64 * MB, preact=base + 2 * K, ldp=wide))
    one = dict(m=1, n=N, x=17 * MB, w=base, ldw=K + N)
    assert not run(L.heddle_linear, linear(**one, y=base + 2 * K))
    assert run(L.heddle_linear, linear(**one, y=base + 2 * K + 2))


def test_groups(L):
    g = dict(groups=3, d_offsets=15 * MB, stride_w=N * K, stride_dw=N * K)
    assert not run(L.heddle_linear, linear(**g))
    d = linear(**g)
    assert run(L.heddle_linear, linear(**g, y=at(d, "w") + 2 * 2 * N * K))
    assert not run(L.heddle_linear, linear(**g, y=at(d, "w") + 2 * 3 * N * K))
    assert run(L.heddle_linear_backward, linear(**g, dx=at(d, "dw") + 2 * (3 * N * K - 1)))
    # groups apart: y in the gap between two
    far = {**g, "stride_w": N * K + M * N}
    assert not run(L.heddle_linear, linear(**far, y=at(d, "w") + 2 * N * K))
    assert run(L.heddle_linear, linear(**far, y=at(d, "w") + 2 * (2 * far["stride_w"] + 5)))


def test_against_every_value(L):
    """x and y of one distance between rows, or of one row: as comparing their values' addresses says"""
    rng, seen = random.Random(7), [0, 0]
    for _ in range(3000):
        m, k, n = rng.choice([1, 2, 3, 5]), rng.randint(1, 9), rng.randint(1, 9)
        ldx = max(k, n) + rng.randint(0, 12)
        ldy = ldx if m > 1 else n
        shift = rng.randint(-3 * ldx - 12, 3 * ldx + 12)
        values = lambda p, ld, cols: {p + i * ld + j for i in range(m) for j in range(cols)}  # noqa: E731
        want = bool(values(0, ldx, k) & values(shift, ldy, n))
        base = 200 * MB
        got = run(L.heddle_linear, linear(m=m, n=n, k=k, x=base, ldx=ldx, y=base + 2 * shift, ldy=ldy, residual=None, preact=None))
        assert got == want, (m, k, n, ldx, shift)
        seen[want] += 1
    assert min(seen) > 500, seen


def test_clipping(L):
    def call(shift, n=100, dtype=H.HEDDLE_T_F32):
        g = H.heddle_grad_desc(g=16 * MB, out=16 * MB + shift, n=n, dtype=dtype)
        rc = L.heddle_clip_grad_norm(C.byref(g), 1, 1.0, 17 * MB, 18 * MB, MB, None)
        assert rc in (H.HEDDLE_E_INVAL, H.HEDDLE_E_DEVICE), rc
        return rc == H.HEDDLE_E_INVAL

    assert not call(0) and not call(400) and not call(-400)
    assert call(4) and call(-4) and call(396) and call(-396)
    assert call(198, dtype=H.HEDDLE_T_BF16) and not call(200, dtype=H.HEDDLE_T_BF16)
