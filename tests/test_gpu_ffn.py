"""The feed-forward operators (products, gated block, expert groups, their
gradients) against plain 64-bit forms, every value within the bound that the
roundings allow. Needs an MI355X."""
import itertools

import pytest
import torch

import ffn_reference as R

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


class Maker:
    """Random device matrices, and matrices that are parts of larger ones:
    `gap` more values a row, `shift` values before the first; what lies outside
    the matrix is NaN, and must neither be used nor written."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = dtype
        self.whole = []

    def part(self, shape, gap=0, shift=0, scale=None):
        lead, rows, cols = shape[:-2], shape[-2], shape[-1]
        n = 1
        for v in lead:
            n *= v
        flat = torch.full((shift + n * rows * (cols + gap) + 64,), float("nan"), dtype=self.dtype, device="cuda")
        view = flat[shift:shift + n * rows * (cols + gap)].view(*lead, rows, cols + gap)[..., :cols]
        if scale is not None:
            view.copy_(torch.randn(shape, generator=self.g, device="cuda").mul_(scale))
        self.whole.append((flat, view))
        return view

    def untouched(self):
        for flat, view in self.whole:
            at = torch.zeros_like(flat, dtype=torch.bool)
            torch.as_strided(at, view.shape, view.stride(), view.storage_offset()).fill_(True)
            assert bool(torch.isnan(flat[~at]).all()), "values outside a matrix were written"


def near(got, want, bound, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first {i}: {got[i].item()} for "
                             f"{want[i].item()}, off {off[i].item():.3g}, bound {bound[i].item():.3g}")


def run_linear(H, seed, m, k, n, act, bias, residual, dtype, gap=0, shift=0, backward=True):
    print(f"linear {m} {k} {n} {act} bias={bias} residual={residual} {dtype} gap={gap} shift={shift}", flush=True)
    mk = Maker(seed, dtype)
    x, w = mk.part((m, k), gap, shift, 1.0), mk.part((n, k), gap, shift, k ** -0.5)
    b = torch.randn(n, generator=mk.g, device="cuda").to(dtype) if bias else None
    r = mk.part((m, n), gap, shift, 1.0) if residual else None
    y, z = mk.part((m, n), gap, shift), mk.part((m, n), gap, shift)
    H.heddle_linear(x, w, bias=b, act=H.ACTIVATIONS[act], residual=r, preact=z, out=y)
    wy, by, wz, bz = R.linear(x, w, b, act, r, dtype)
    near(z, wz, bz, "preact")
    near(y, wy, by, "y")
    if backward:
        dy = mk.part((m, n), gap, shift, 1.0)
        dx, dw = mk.part((m, k), gap, shift), mk.part((n, k), gap, shift)
        got = H.heddle_linear_backward(dy, x, w, act=H.ACTIVATIONS[act], preact=None if act == "none" else z, dx=dx, dw=dw,
                                       want_db=True)
        for key, (c, e) in R.linear_backward(dy, x, w, act, z, dtype).items():
            near(got[key], c, e, key)
    torch.cuda.synchronize()
    mk.untouched()


SIZES = [(1, 1, 1), (1, 64, 16), (2, 7, 3), (3, 65, 33), (5, 128, 129), (16, 40, 24), (17, 200, 136), (31, 512, 72),
         (64, 64, 128), (65, 63, 127), (100, 321, 257), (129, 1024, 130), (255, 72, 511), (256, 256, 256), (300, 130, 770)]


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_sizes(H, m, k, n, dtype):
    run_linear(H, m * 7 + k, m, k, n, "none", False, False, dtype)
    run_linear(H, m * 7 + n, m, k, n, "silu", True, True, dtype)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("bias,residual", list(itertools.product([False, True], repeat=2)))
def test_linear_epilogue(H, act, bias, residual):
    run_linear(H, 5, 70, 96, 200, act, bias, residual, torch.bfloat16)
    run_linear(H, 6, 9, 104, 88, act, bias, residual, torch.float16)


@pytest.mark.parametrize("gap,shift", [(8, 0), (8, 8), (2, 2), (4, 6), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("m,k,n", [(4, 96, 80), (40, 104, 264), (150, 70, 62)])
def test_linear_strides(H, gap, shift, m, k, n):
    """rows apart, rows on 16-, 8-, 4- and 2-byte boundaries"""
    run_linear(H, gap + shift, m, k, n, "gelu", True, True, torch.bfloat16, gap, shift)


@pytest.mark.parametrize("m,k,n", [(600, 2048, 520), (2, 8192, 300), (40, 6000, 100), (1100, 96, 1000)])
def test_linear_large(H, m, k, n):
    """long reductions, several tiles each way"""
    run_linear(H, 9, m, k, n, "gelu_tanh", True, True, torch.bfloat16)


def test_linear_no_rows(H):
    x, w = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda"), torch.ones(16, 24, dtype=torch.bfloat16, device="cuda")
    assert H.heddle_linear(x, w).shape == (0, 16)
    got = H.heddle_linear_backward(x.new_empty(0, 16), x, w, want_db=True)
    assert got["dx"].shape == (0, 24) and not got["dw"].any() and not got["db"].any()


def test_linear_nonfinite(H):
    """infinities and NaN stay in their own rows and columns"""
    x, w = torch.randn(70, 136, device="cuda").bfloat16(), torch.randn(150, 136, device="cuda").bfloat16()
    clean = H.heddle_linear(x, w, act=H.HEDDLE_A_SILU)
    x[3, 5], x[40, 135], w[7, 0] = float("inf"), float("nan"), float("nan")
    y = H.heddle_linear(x, w, act=H.HEDDLE_A_RELU)
    rows = torch.tensor([r not in (3, 40) for r in range(70)], device="cuda")
    cols = torch.tensor([c != 7 for c in range(150)], device="cuda")
    assert bool(torch.isfinite(y[rows][:, cols]).all()) and bool(torch.isnan(y[40]).all()) and bool(torch.isnan(y[:, 7]).all())
    assert bool(torch.isfinite(clean).all())
    z = torch.tensor([[-3e4, 3e4, -100.0, 0.0, float("inf")]], device="cuda").half()
    eye = torch.eye(5, device="cuda").half()
    z[0, 4] = 100
    for act in ("relu", "silu", "gelu", "gelu_tanh"):
        got = H.heddle_linear(z, eye, act=H.ACTIVATIONS[act])
        assert got.tolist() == [[0.0, z[0, 1].item(), 0.0, 0.0, 100.0]], act


def group_offsets(kind, rows, groups, gen):
    """host offsets: `even`, `one` (all rows in one group) or `uneven` with empty groups"""
    if kind == "one":
        counts = [0] * groups
        counts[groups // 2] = rows
    elif kind == "even":
        counts = [rows // groups + (i < rows % groups) for i in range(groups)]
    else:
        pick = torch.randint(0, groups, (rows,), generator=gen)
        pick = torch.where(pick % 3 == 0, pick * 0, pick)
        counts = torch.bincount(pick, minlength=groups).tolist()
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


GROUPS = [("uneven", 40, 8), ("uneven", 7, 16), ("one", 300, 5), ("even", 260, 4), ("uneven", 500, 70), ("even", 3, 1)]


@pytest.mark.parametrize("kind,rows,groups", GROUPS)
@pytest.mark.parametrize("k,n,gap,shift", [(64, 96, 0, 0), (70, 33, 1, 0), (136, 200, 8, 2)])
def test_linear_groups(H, kind, rows, groups, k, n, gap, shift):
    dtype = torch.bfloat16
    print("groups", kind, rows, groups, k, n, gap, shift, flush=True)
    mk = Maker(rows + groups, dtype)
    off = group_offsets(kind, rows, groups, torch.Generator().manual_seed(rows))
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    x, w = mk.part((rows, k), gap, shift, 1.0), mk.part((groups, n, k), gap, shift, k ** -0.5)
    b = torch.randn(groups, n, generator=mk.g, device="cuda").to(dtype)
    r, dy = mk.part((rows, n), gap, shift, 1.0), mk.part((rows, n), gap, shift, 1.0)
    y, z = mk.part((rows, n), gap, shift), mk.part((rows, n), gap, shift)
    act = H.HEDDLE_A_GELU
    H.heddle_linear(x, w, bias=b, act=act, residual=r, preact=z, out=y, offsets=offsets)
    dx, dw = mk.part((rows, k), gap, shift), mk.part((groups, n, k), gap, shift)
    got = H.heddle_linear_backward(dy, x, w, act=act, preact=z, offsets=offsets, dx=dx, dw=dw, want_db=True)
    for e in range(groups):
        s = slice(off[e], off[e + 1])
        wy, by, wz, bz = R.linear(x[s], w[e], b[e], "gelu", r[s], dtype)
        near(z[s], wz, bz, f"preact of group {e}")
        near(y[s], wy, by, f"y of group {e}")
        want = R.linear_backward(dy[s], x[s], w[e], "gelu", z[s], dtype)
        near(dx[s], *want["dx"], f"dx of group {e}")
        near(dw[e], *want["dw"], f"dw of group {e}")
        near(got["db"][e], *want["db"], f"db of group {e}")
    torch.cuda.synchronize()
    mk.untouched()


@pytest.mark.parametrize("rows,k,n", [(1500, 72, 40), (100, 2048, 72), (20, 4096, 24)])
def test_linear_one_group(H, rows, k, n):
    """one expert's rows: the same as without offsets, also where that product's reduction is divided"""
    mk = Maker(rows, torch.bfloat16)
    x, w, dy = mk.part((rows, k), 0, 0, 1.0), mk.part((n, k), 0, 0, k ** -0.5), mk.part((rows, n), 0, 0, 1.0)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    y, by, _, _ = R.linear(x, w, None, "none", None, torch.bfloat16)
    near(H.heddle_linear(x, w[None], offsets=off), y, by, "y")
    got = H.heddle_linear_backward(dy, x, w[None], offsets=off, want_db=True)
    for key, (c, e) in R.linear_backward(dy, x, w, "none", None, torch.bfloat16).items():
        near(got[key].view(c.shape), c, e, key)


@pytest.mark.parametrize("groups,rows,k,n", [(70, 900, 2600, 1030), (40, 300, 1000, 1100)])
def test_linear_groups_wide(H, groups, rows, k, n):
    """weights of many tiles for few rows: several of a group's tiles go through one workgroup"""
    dtype = torch.bfloat16
    mk = Maker(groups, dtype)
    off = group_offsets("uneven", rows, groups, torch.Generator().manual_seed(groups))
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    x, w, dy = mk.part((rows, k), 0, 0, 1.0), mk.part((groups, n, k), 0, 0, k ** -0.5), mk.part((rows, n), 2, 2, 1.0)
    got = H.heddle_linear_backward(dy, x, w, offsets=offsets, dx=mk.part((rows, k)), dw=mk.part((groups, n, k), 2, 2))
    for e in range(groups):
        s = slice(off[e], off[e + 1])
        want = R.linear_backward(dy[s], x[s], w[e], "none", None, dtype)
        near(got["dx"][s], *want["dx"], f"dx of group {e}")
        near(got["dw"][e], *want["dw"], f"dw of group {e}")
    torch.cuda.synchronize()
    mk.untouched()


def run_ffn(H, seed, t, d, f, act, residual, dtype, off=None, gap=0, shift=0):
    print(f"ffn {t} {d} {f} {act} residual={residual} {dtype} groups={off and len(off) - 1} gap={gap} shift={shift}", flush=True)
    mk = Maker(seed, dtype)
    lead = (len(off) - 1,) if off else ()
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda") if off else None
    x = mk.part((t, d), gap, shift, 1.0)
    wi, wo = mk.part((*lead, 2 * f, d), gap, shift, d ** -0.5), mk.part((*lead, d, f), gap, shift, f ** -0.5)
    r = mk.part((t, d), gap, shift, 1.0) if residual else None
    y, p, dy = mk.part((t, d), gap, shift), mk.part((t, 2 * f), gap, shift), mk.part((t, d), gap, shift, 1.0)
    a = H.ACTIVATIONS[act]
    H.heddle_gated_ffn(x, wi, wo, act=a, residual=r, preact=p, out=y, offsets=offsets)
    dx = mk.part((t, d), gap, shift)
    dwi, dwo = mk.part((*lead, 2 * f, d), gap, shift), mk.part((*lead, d, f), gap, shift)
    H.heddle_gated_ffn_backward(dy, x, wi, wo, p, act=a, offsets=offsets, dx=dx, dw_in=dwi, dw_out=dwo)
    for e in range(len(off) - 1 if off else 1):
        s = slice(off[e], off[e + 1]) if off else slice(0, t)
        i = (lambda q: q[e]) if off else (lambda q: q)
        wy, by, wp, bp = R.ffn(x[s], i(wi), i(wo), act, None if r is None else r[s], dtype)
        near(p[s], wp, bp, f"preact, group {e}")
        near(y[s], wy, by, f"y, group {e}")
        want = R.ffn_backward(dy[s], x[s], i(wi), i(wo), act, p[s], dtype)
        near(dx[s], *want["dx"], f"dx, group {e}")
        near(i(dwi), *want["dw_in"], f"dw_in, group {e}")
        near(i(dwo), *want["dw_out"], f"dw_out, group {e}")
    torch.cuda.synchronize()
    mk.untouched()


@pytest.mark.parametrize("t,d,f", [(1, 64, 64), (1, 1, 1), (2, 10, 6), (3, 136, 204), (16, 96, 40), (17, 520, 65), (33, 72, 408),
                                   (64, 128, 128), (65, 129, 17), (130, 264, 300), (300, 512, 520)])
@pytest.mark.parametrize("dtype", TYPES)
def test_ffn_sizes(H, t, d, f, dtype):
    run_ffn(H, t + d, t, d, f, "silu", t % 2 == 0, dtype)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("t", [1, 50, 200])
def test_ffn_activations(H, act, t):
    run_ffn(H, 3, t, 200, 168, act, True, torch.bfloat16)


@pytest.mark.parametrize("gap,shift", [(8, 8), (2, 4), (4, 2), (1, 0), (0, 1)])
@pytest.mark.parametrize("t", [2, 70])
def test_ffn_strides(H, gap, shift, t):
    run_ffn(H, 4, t, 104, 140, "silu", True, torch.bfloat16, None, gap, shift)


@pytest.mark.parametrize("kind,rows,groups", GROUPS)
@pytest.mark.parametrize("d,f,gap,shift", [(128, 204, 0, 0), (72, 51, 1, 0), (64, 104, 2, 2)])
def test_ffn_groups(H, kind, rows, groups, d, f, gap, shift):
    off = group_offsets(kind, rows, groups, torch.Generator().manual_seed(rows))
    run_ffn(H, rows, rows, d, f, "silu", rows % 2 == 0, torch.bfloat16, off, gap, shift)


def test_ffn_no_rows(H):
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    wi, wo = x.new_ones(96, 64), x.new_ones(64, 48)
    assert H.heddle_gated_ffn(x, wi, wo).shape == (0, 64)
    got = H.heddle_gated_ffn_backward(x, x, wi, wo, x.new_empty(0, 96))
    assert got["dx"].shape == (0, 64) and not got["dw_in"].any() and not got["dw_out"].any()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    got = H.heddle_gated_ffn_backward(x, x, x.new_ones(3, 96, 64), x.new_ones(3, 64, 48), x.new_empty(0, 96), offsets=off)
    assert got["dw_in"].shape == (3, 96, 64) and not got["dw_in"].any() and not got["dw_out"].any()


def test_gradients_against_differences(H):
    """directional differences of the 64-bit forward pass. fp16: each
    gradient's relative error is a few units of 2^-11, its sum with a random
    direction's at most sqrt(n) times larger than the terms' mean square; the
    central difference's own error is of order h^2 = 1e-8."""
    mk = Maker(17, torch.float16)
    t, d, f = 24, 40, 56
    x, wi, wo = mk.part((t, d), 0, 0, 1.0), mk.part((2 * f, d), 0, 0, d ** -0.5), mk.part((d, f), 0, 0, f ** -0.5)
    dy, p = mk.part((t, d), 0, 0, 1.0), mk.part((t, 2 * f))
    H.heddle_gated_ffn(x, wi, wo, preact=p)
    got = H.heddle_gated_ffn_backward(dy, x, wi, wo, p)

    def loss(x, wi, wo):
        q = x @ wi.t()
        return float(((R.act("silu", q[:, :f]) * q[:, f:]) @ wo.t() * dy.double()).sum())

    h = 1e-4
    args = [x.double(), wi.double(), wo.double()]
    for i, key in enumerate(("dx", "dw_in", "dw_out")):
        for _ in range(4):
            v = torch.randn(args[i].shape, generator=mk.g, device="cuda", dtype=torch.float64)
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * v, args[i] - h * v
            want = (loss(*up) - loss(*down)) / (2 * h)
            terms = got[key].double() * v
            # 8 units: own rounding, p, dp or h, each at most one unit of every term, and the sums' spread
            assert abs(float(terms.sum()) - want) <= 8 * 2.0 ** -11 * float(terms.square().sum().sqrt()) * 4 + 1e-5 * abs(want), key


def test_offsets_beyond_32_bits(H):
    """rows far apart: byte offsets above 2^32 in x, dy and the outputs"""
    m, ld, k, n = 9000, 300000, 72, 40
    x = torch.empty(m, ld, dtype=torch.bfloat16, device="cuda")[:, 7:7 + k + 1][:, 1:]
    x.copy_(torch.randn(m, k, device="cuda"))
    w = torch.randn(n, k, device="cuda").mul_(k ** -0.5).bfloat16()
    y = torch.empty(m, ld, dtype=torch.bfloat16, device="cuda")[:, 16:16 + n]
    H.heddle_linear(x, w, out=y)
    wy, by, _, _ = R.linear(x, w, None, "none", None, torch.bfloat16)
    near(y, wy, by, "y")
    got = H.heddle_linear_backward(y, x, w)
    for key in ("dx", "dw"):
        near(got[key], *R.linear_backward(y, x, w, "none", None, torch.bfloat16)[key], key)


def test_other_stream_and_repeat(H):
    """on a stream of the caller's, with its own tensors; the same bits twice"""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x, wi, wo = (torch.randn(*z, device="cuda").mul_(0.1).bfloat16() for z in ((90, 200), (2 * 152, 200), (200, 152)))
        p = x.new_empty(90, 304)
    s.synchronize()
    a = H.heddle_gated_ffn(x, wi, wo, preact=p, stream=s)
    ga = H.heddle_gated_ffn_backward(a, x, wi, wo, p, stream=s)
    s.synchronize()
    b = H.heddle_gated_ffn(x, wi, wo, preact=p)
    gb = H.heddle_gated_ffn_backward(b, x, wi, wo, p)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and all(torch.equal(ga[k], gb[k]) for k in ga)


@pytest.mark.parametrize("t,experts", [(1, 1), (48, 1), (40, 6)])
def test_graph_replays(H, t, experts):
    """captured once, replayed over new inputs, each replay as the eager call"""
    lead = (experts,) if experts > 1 else ()
    x, dy = (torch.randn(t, 264, device="cuda").bfloat16() for _ in range(2))
    wi, wo = (torch.randn(*lead, *z, device="cuda").mul_(0.05).bfloat16() for z in ((2 * 204, 264), (264, 204)))
    off = torch.tensor(group_offsets("uneven", t, experts, torch.Generator().manual_seed(1)), dtype=torch.int32,
                       device="cuda") if experts > 1 else None

    def step():
        p = x.new_empty(t, 408)
        y = H.heddle_gated_ffn(x, wi, wo, preact=p, offsets=off)
        return [y, *H.heddle_gated_ffn_backward(dy, x, wi, wo, p, offsets=off).values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(3):
        x.copy_(torch.randn(t, 264, device="cuda"))
        g.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_offsets_out_of_range_stay_inside(H):
    """offsets are clamped to the rows; what they leave out is not written"""
    x, w = torch.randn(50, 64, device="cuda").bfloat16(), torch.randn(3, 32, 64, device="cuda").mul_(0.1).bfloat16()
    off = torch.tensor([-5, 20, 30, 1000], dtype=torch.int32, device="cuda")
    fine = torch.tensor([0, 20, 30, 50], dtype=torch.int32, device="cuda")
    assert torch.equal(H.heddle_linear(x, w, offsets=off), H.heddle_linear(x, w, offsets=fine))
    y = torch.full((50, 32), 7.0, device="cuda").bfloat16()
    H.heddle_linear(x, w, out=y, offsets=torch.tensor([10, 20, 15, 40], dtype=torch.int32, device="cuda"))
    assert bool((y[:10] == 7).all()) and bool((y[40:] == 7).all())


def test_refusals(H):
    x, w = torch.ones(4, 32, device="cuda").bfloat16(), torch.ones(8, 32, device="cuda").bfloat16()
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    bad = [lambda: H.heddle_linear(x.float(), w.float()), lambda: H.heddle_linear(x, w.half()), lambda: H.heddle_linear(x, w[:, :31]),
           lambda: H.heddle_linear(x.t(), w), lambda: H.heddle_linear(x.cpu(), w.cpu()), lambda: H.heddle_linear(x, w.cpu()),
           lambda: H.heddle_linear(x, w, act=9), lambda: H.heddle_linear(x, w, bias=x[0]), lambda: H.heddle_linear(x, w, out=x),
           lambda: H.heddle_linear(x, w, offsets=off), lambda: H.heddle_linear(x, w[None], offsets=off.long()),
           lambda: H.heddle_linear(x, w[None], offsets=off[:1]), lambda: H.heddle_linear(x[0], w),
           lambda: H.heddle_linear(x, w.t().contiguous().t()),
           lambda: H.heddle_linear_backward(x[:, :8], x, w, act=H.HEDDLE_A_RELU),
           lambda: H.heddle_gated_ffn(x, w[:7], w), lambda: H.heddle_gated_ffn(x, w, w), lambda: H.heddle_gated_ffn(x, w, w.t()),
           lambda: H.heddle_gated_ffn_backward(x, x, w, x.new_ones(32, 4), x)]
    for i, f in enumerate(bad):
        with pytest.raises(H.HeddleError) as e:
            f()
        assert e.value.code == H.HEDDLE_E_INVAL, i
