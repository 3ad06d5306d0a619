"""Every tile kernel by its values: each shape of tile with each memory order
and epilogue, whole and divided reductions, with and without expert groups.
The sizes are small ones that the library's rules send there; which ones they
reach is asked of the library itself, without a GPU, so that a rule that
changes cannot leave a kernel untested. Values need an MI355X."""
import ctypes as C

import pytest
import torch

import ffn_reference as R
from paper_2609_34244_amd import heddle as HD
from test_gpu_ffn import Maker, group_offsets, near, run_linear

# rows, model width, hidden units, expert groups (0: without offsets)
BLOCKS = [(37, 138, 4231, 1), (53, 129, 4124, 0), (829, 801, 45, 0), (4412, 44, 1228, 0), (4616, 1756, 43, 0), (5512, 264, 307, 1),
          (5465, 320, 137, 0), (4945, 400, 3526, 0), (334, 4187, 5699, 0), (1201, 222, 4185, 6), (2202, 3024, 45, 1), (2202, 5798, 350, 0),
          (5823, 1564, 586, 5), (393, 61, 5577, 25), (305, 5299, 45, 29), (3340, 135, 3605, 0), (2447, 129, 5863, 1), (4354, 4553, 276, 0)]
# rows, k, columns
LINEARS = [(3900, 2050, 4002), (2050, 4100, 2100), (4090, 523, 4099), (600, 2048, 520), (1100, 96, 1000), (4412, 1228, 44)]

TILES = {0: "256x256", 1: "128x128", 2: "64x128", 3: "64x256"}


class Shape(C.Structure):
    _fields_ = [("cfg", C.c_int), ("splits", C.c_int), ("split_tiles", C.c_int)]


def rules():
    """the library's own choice: shape_of and third_buffer (linear.hip)"""
    lib = HD.lib()
    shape, third = lib._ZN6heddle2mm8shape_ofElllibNS0_5OrderE, lib._ZN6heddle2mm12third_bufferEllibbi
    shape.restype, shape.argtypes = Shape, [C.c_int64] * 3 + [C.c_int, C.c_bool, C.c_int]
    third.restype, third.argtypes = C.c_bool, [C.c_int64] * 2 + [C.c_int, C.c_bool, C.c_bool, C.c_int]
    return shape, third


def kernel(what, m, n, k, groups, gated, order):
    """(product, with groups, tile, whether the reduction is divided); order: of shape_of"""
    shape, third = rules()
    s = shape(m, n, k, groups, gated, order)
    buffers = " 3" if s.cfg == 2 and third(m, n, groups, gated, order == 2, s.splits) else " 2" if s.cfg == 2 else ""
    return what, groups > 0, TILES[s.cfg] + buffers, s.splits > 1


def of_block(t, d, f, groups):
    assert t > 32 and t > 10 * groups, "few enough rows for the kernel without tiles"
    return {kernel("gate and up", t, f, d, groups, True, 0), kernel("rows", t, d, f, groups, False, 0),
            kernel("dP and H", t, f, d, groups, False, 1), kernel("dX", t, d, 2 * f, groups, False, 1),
            kernel("dW", 2 * f, d, t, groups, False, 2), kernel("dW", d, f, t, groups, False, 2)}


def of_linear(m, k, n):
    assert m > 32
    return {kernel("rows", m, n, k, 0, False, 0), kernel("dX", m, k, n, 0, False, 1), kernel("dW", n, k, m, 0, False, 2)}


def test_every_kernel_is_reached():
    got = set().union(*(of_block(*b) for b in BLOCKS), *(of_linear(*a) for a in LINEARS))
    tiles = ["256x256", "128x128", "64x128 2", "64x128 3"]
    want = {(what, False, tile, divided) for what in ("gate and up", "rows", "dP and H", "dX", "dW") for tile in tiles
            for divided in (False, True)}
    want |= {(what, True, tile, False) for what in ("gate and up", "rows", "dP and H", "dX") for tile in tiles + ["64x256"]}
    want |= {("dW", True, tile, False) for tile in tiles}
    assert got == want, (sorted(want - got), sorted(got - want))


def test_rows_and_columns_of_linear():
    """the epilogue with everything in it, too, on each tile"""
    tiles = {k[2] for a in LINEARS for k in of_linear(*a) if k[0] == "rows"}
    assert tiles == {"256x256", "128x128", "64x128 2", "64x128 3"}, tiles


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    return HD


class Even(Maker):
    """matrices as they are where their rows are on 4-byte boundaries, else with one value between rows:
    no operand is copied first; `wide`: with more between rows, and a first one off 16 bytes"""

    def __init__(self, seed, dtype, wide):
        super().__init__(seed, dtype)
        self.wide = wide

    def matrix(self, *shape, scale=None):
        return self.part(shape, shape[-1] % 2 + (6 if self.wide else 0), 2 if self.wide else 0, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,act,wide", [(torch.bfloat16, "silu", False), (torch.float16, "gelu_tanh", True)])
@pytest.mark.parametrize("t,d,f,groups", BLOCKS)
def test_block(H, t, d, f, groups, dtype, act, wide):
    print(f"block {t} {d} {f} groups={groups} {act} {dtype}", flush=True)
    mk = Even(t, dtype, wide)
    off = group_offsets("uneven", t, groups, torch.Generator().manual_seed(t)) if groups else [0, t]
    lead = (groups,) if groups else ()
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda") if groups else None
    x, r, dy = mk.matrix(t, d, scale=1.0), mk.matrix(t, d, scale=1.0), mk.matrix(t, d, scale=1.0)
    wi, wo = mk.matrix(*lead, 2 * f, d, scale=d ** -0.5), mk.matrix(*lead, d, f, scale=f ** -0.5)
    y, p, dx = mk.matrix(t, d), mk.matrix(t, 2 * f), mk.matrix(t, d)
    dwi, dwo = mk.matrix(*lead, 2 * f, d), mk.matrix(*lead, d, f)
    a = H.ACTIVATIONS[act]
    H.heddle_gated_ffn(x, wi, wo, act=a, residual=r, preact=p, out=y, offsets=offsets)
    H.heddle_gated_ffn_backward(dy, x, wi, wo, p, act=a, offsets=offsets, dx=dx, dw_in=dwi, dw_out=dwo)
    for e in range(len(off) - 1):
        s = slice(off[e], off[e + 1])
        i = (lambda q: q[e]) if groups else (lambda q: q)
        wy, by, wp, bp = R.ffn(x[s], i(wi), i(wo), act, r[s], dtype)
        near(p[s], wp, bp, f"preact, group {e}")
        near(y[s], wy, by, f"y, group {e}")
        want = R.ffn_backward(dy[s], x[s], i(wi), i(wo), act, p[s], dtype)
        near(dx[s], *want["dx"], f"dx, group {e}")
        near(i(dwi), *want["dw_in"], f"dw_in, group {e}")
        near(i(dwo), *want["dw_out"], f"dw_out, group {e}")
    torch.cuda.synchronize()
    mk.untouched()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,act,wide", [(torch.bfloat16, "gelu", True), (torch.float16, "silu", False)])
@pytest.mark.parametrize("m,k,n", LINEARS)
def test_linear(H, m, k, n, dtype, act, wide):
    print(f"linear {m} {k} {n} {act} {dtype}", flush=True)
    mk = Even(m, dtype, wide)
    x, w, r, dy = mk.matrix(m, k, scale=1.0), mk.matrix(n, k, scale=k ** -0.5), mk.matrix(m, n, scale=1.0), mk.matrix(m, n, scale=1.0)
    b = torch.randn(n, generator=mk.g, device="cuda").to(dtype)
    y, z, dx, dw = mk.matrix(m, n), mk.matrix(m, n), mk.matrix(m, k), mk.matrix(n, k)
    a = H.ACTIVATIONS[act]
    H.heddle_linear(x, w, bias=b, act=a, residual=r, preact=z, out=y)
    wy, by, wz, bz = R.linear(x, w, b, act, r, dtype)
    near(z, wz, bz, "preact")
    near(y, wy, by, "y")
    got = H.heddle_linear_backward(dy, x, w, act=a, preact=z, dx=dx, dw=dw, want_db=True)
    for key, (c, e) in R.linear_backward(dy, x, w, act, z, dtype).items():
        near(got[key], c, e, key)
    torch.cuda.synchronize()
    mk.untouched()


# few rows: the kernel without tiles divides k among 16 wavefronts (k from 4096 on), 8 or 4 (1024 workgroups
# without), for up to 16 rows at a time or 32, rows on 4-byte boundaries or not
FEW = [(5, 4160, 50, 0), (5, 4100, 50, 0), (5, 4099, 70, 0), (20, 4100, 50, 0), (32, 6000, 33, 2), (3, 72, 16400, 0), (3, 71, 16400, 0),
       (20, 72, 16400, 0), (31, 70, 16389, 2), (9, 200, 16390, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("m,k,n,gap", FEW)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_few_rows(H, m, k, n, gap, dtype):
    run_linear(H, k, m, k, n, "silu", True, True, dtype, gap, 0, backward=False)


@pytest.mark.gpu
@pytest.mark.parametrize("groups,rows,k,n,gap", [(64, 150, 72, 264, 0), (64, 150, 71, 264, 0), (130, 200, 200, 140, 0), (64, 500, 130, 270, 1),
                                                 (3, 9, 4100, 40, 0), (3, 28, 4099, 40, 0)])
def test_few_rows_of_groups(H, groups, rows, k, n, gap):
    print(f"few rows {groups} {rows} {k} {n} {gap}", flush=True)
    dtype = torch.bfloat16
    mk = Maker(rows, dtype)
    off = group_offsets("uneven", rows, groups, torch.Generator().manual_seed(rows))
    x, w = mk.part((rows, k), gap, 0, 1.0), mk.part((groups, n, k), gap, 0, k ** -0.5)
    b, y, z = torch.randn(groups, n, generator=mk.g, device="cuda").to(dtype), mk.part((rows, n), gap), mk.part((rows, n), gap)
    H.heddle_linear(x, w, bias=b, act=H.HEDDLE_A_SILU, preact=z, out=y, offsets=torch.tensor(off, dtype=torch.int32, device="cuda"))
    for e in range(groups):
        s = slice(off[e], off[e + 1])
        wy, by, wz, bz = R.linear(x[s], w[e], b[e], "silu", None, dtype)
        near(z[s], wz, bz, f"preact of group {e}")
        near(y[s], wy, by, f"y of group {e}")
    torch.cuda.synchronize()
    mk.untouched()
