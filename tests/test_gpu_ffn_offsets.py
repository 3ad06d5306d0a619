"""Expert offsets that are out of order: every operator reads them as their
running maximum, so the results are those of the ordered offsets, bit for bit.
Needs an MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def ordered(offsets, rows):
    out, most = [], 0
    for o in offsets:
        most = max(most, min(max(o, 0), rows))
        out.append(most)
    return out


def zigzag(groups, rows, low, high):
    """every second offset is `low`, the others rise to `high`; then the row count"""
    return [0] + [low if i % 2 else high * (i + 2) // (groups + 1) for i in range(groups - 1)] + [rows]


CASES = {
    # ranges that, taken one by one, have more rows and tiles than there are
    "tiles": (1024, [0, 500, 0, 500, 0, 500, 0, 1024]),
    "few rows": (6, [0, 4, 0, 4, 0, 4, 0, 6]),
    "first one late": (300, [100, 20, 60, 150, 90, 300]),
    "out of range too": (200, [-7, 90, 2**31 - 1, -2**31, 50, 200]),
    # beyond one wavefront's 64 offsets, the disorder across its end
    "many": (900, zigzag(150, 900, 3, 800)),
    "last of 64": (400, [0] + [min(6 * i, 350) for i in range(1, 63)] + [390, 10] + [20] * 20 + [400]),
}


@pytest.mark.parametrize("name", sorted(CASES))
@pytest.mark.parametrize("d,f", [(136, 72), (264, 520)])
def test_offsets_out_of_order(H, name, d, f):
    rows, off = CASES[name]
    print("offsets", name, rows, len(off) - 1, d, f, flush=True)
    groups = len(off) - 1
    g = torch.Generator(device="cuda").manual_seed(rows)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(scale).bfloat16()

    x, dy, z0 = normal(rows, d), normal(rows, d), normal(rows, 2 * f)
    wi, wo, b = normal(groups, 2 * f, d, scale=d ** -0.5), normal(groups, d, f, scale=f ** -0.5), normal(groups, 2 * f)
    dz = normal(rows, 2 * f)

    def calls(offsets):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        # what no group has keeps what was there
        p, z = torch.full_like(z0, 7.0), torch.full_like(z0, 7.0)
        out = {"p": p, "z": z}
        out["y"] = H.heddle_gated_ffn(x, wi, wo, preact=p, out=torch.full_like(x, 7.0), offsets=o)
        out["t"] = H.heddle_linear(x, wi, bias=b, act=H.HEDDLE_A_SILU, preact=z, out=torch.full_like(z0, 7.0), offsets=o)
        for k, v in H.heddle_gated_ffn_backward(dy, x, wi, wo, p, offsets=o, dx=torch.full_like(x, 7.0)).items():
            out["ffn " + k] = v
        for k, v in H.heddle_linear_backward(dz, x, wi, act=H.HEDDLE_A_SILU, preact=z, offsets=o, want_db=True,
                                             dx=torch.full_like(x, 7.0)).items():
            out["linear " + k] = v
        return out

    want = ordered(off, rows)
    assert want != off and want[-1] == rows
    a, b2 = calls(off), calls(want)
    torch.cuda.synchronize()
    for k in a:
        assert torch.equal(a[k], b2[k]), k
    assert bool((a["y"][:want[0]] == 7).all()) and not bool((a["y"][want[0]:] == 7).all(1).any())
