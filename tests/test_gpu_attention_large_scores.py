"""Attention where the scores are far larger than a float's digits reach: the keys
of the largest score share the row, whatever its size. Needs an MI355X."""
import pytest
import torch

from ffn_reference import E, unit
from layer_common import near

pytestmark = pytest.mark.gpu


def means(w, v):
    """of the values and of their sizes, with weights w [sequences, keys, heads]: [sequences, 1, heads, dim]"""
    w = (w / w.sum(1, keepdim=True))[..., None]
    return (w * v.double()).sum(1, keepdim=True), (w * v.double().abs()).sum(1, keepdim=True)


# (sequences, queries, keys, heads): 32 rows a workgroup, the same with the keys in parts, 128 rows, 256 rows
SHAPES = [(2, 1, 300, 4), (1, 1, 5000, 2), (1, 200, 130, 3), (4, 1024, 70, 32)]


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "no GPU"
    from paper_2609_34244_amd import heddle
    heddle.lib()
    return heddle


def inputs(shape, dtype, dim, first, second, seed):
    """q, k, v of which q k is first[0] first[1] + second k, a whole number of fp32, with k from `second` of the generator"""
    n, lq, lk, h = shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k = torch.zeros(n, lq, h, dim, device="cuda"), torch.zeros(n, lk, h, dim, device="cuda")
    c = second(n, lk, h, g)
    q[..., 0], k[..., 0], q[..., 1], k[..., 1] = first[0], first[1], 1, c
    v = torch.randint(-64, 65, (n, lk, h, dim), generator=g, device="cuda").float()
    assert torch.equal(k, k.to(dtype).float())
    return q.to(dtype), k.to(dtype), v.to(dtype), c


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,biased", [(64, False), (128, True)])
@pytest.mark.parametrize("power", [10, 20, 24, 28, 34, 60])
def test_largest_scores_alone(H, shape, dtype, dim, biased, power):
    """scores 2^power c of whole c from -7 to 7: two neighbours are e^-(2^10) apart at the least, 0 in fp32, so that y is the mean of
    the values of the largest. Their probabilities are one number, which may differ from 1 (by less than 2^8) and is rounded by u;
    the sum of at most lk values (lk e), a division (3 e) and y's own rounding"""
    n, lq, lk, h = shape
    print(f"large scores {shape} {dtype} {dim} 2^{power}", flush=True)
    q, k, v, c = inputs(shape, dtype, dim, (0, 0), lambda n, lk, h, g: torch.randint(-7, 8, (n, lk, h), generator=g, device="cuda").float(), power)
    lse = torch.empty(n, lq, h, device="cuda")
    y = H.heddle_attention(q, k, v, scale=2.0 ** power, slopes=torch.zeros(h, device="cuda") if biased else None, lse=lse)
    top = c.amax(1, keepdim=True)
    want, size = means((c == top).double(), v)
    near(y, want.expand(y.shape), (unit(dtype) * want.abs() + (1.01 * unit(dtype) + (lk + 4) * E) * size).expand(y.shape), "y")
    ln = (top.double() * 2.0 ** power + (c == top).double().sum(1, keepdim=True).log()).expand(lse.shape)
    near(lse, ln, 8 * E * (ln.abs() + 20), "lse")


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,biased", [(64, True), (128, False)])
def test_small_differences_of_large_scores(H, shape, dtype, dim, biased):
    """scores 2^22 + 8 c, c whole sixteenths to 4: sums below 2^24 sixteenths are exact. A probability is off by the rounding of
    8 c log2(e) (4 e 32 1.5), the exponential's 2 e and its rounding to 16 bits, below 2^-24 by 2^-25"""
    n, lq, lk, h = shape
    q, k, v, c = inputs(shape, dtype, dim, (2.0 ** 10, 2.0 ** 9), lambda n, lk, h, g: torch.randint(-64, 65, (n, lk, h), generator=g, device="cuda") / 16.0, 3)
    y = H.heddle_attention(q, k, v, scale=8.0, slopes=torch.zeros(h, device="cuda") if biased else None)
    want, size = means(torch.exp(8.0 * (c - c.amax(1, keepdim=True)).double()), v)
    bound = unit(dtype) * want.abs() + (unit(dtype) * 1.01 + (2 * lk + 400) * E) * size + lk * 2.0 ** -25 * 64
    near(y, want.expand(y.shape), bound.expand(y.shape), "y")
