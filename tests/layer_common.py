"""What the GPU tests of attention, layer normalisation and expert balance share."""
import torch


class Maker:
    """Random device tensors that are parts of larger ones: what lies outside them is NaN, and must neither be
    used nor written."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.whole = []

    def part(self, shape, dtype, strides=None, shift=0, scale=None):
        """strides: elements between values of each dimension (contiguous without), shift: values before the first"""
        if strides is None:
            strides, n = [], 1
            for s in reversed(shape):
                strides.insert(0, n)
                n *= s
        size = shift + 1 + sum((s - 1) * st for s, st in zip(shape, strides) if s) + 40
        flat = torch.full((size,), float("nan"), dtype=dtype, device="cuda")
        view = torch.as_strided(flat, shape, strides, shift)
        if scale is not None and view.numel():
            view.copy_(torch.randn(shape, generator=self.g, device="cuda").mul_(scale))
        self.whole.append((flat, view))
        return view

    def untouched(self):
        torch.cuda.synchronize()
        for flat, view in self.whole:
            at = torch.zeros_like(flat, dtype=torch.bool)
            if view.numel():
                torch.as_strided(at, view.shape, view.stride(), view.storage_offset()).fill_(True)
            assert bool(torch.isnan(flat[~at]).all()), "values outside a tensor were written"


def near(got, want, bound, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~((off <= bound) | ((got.double() == want) & torch.isinf(want)))
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off, first {i}: {got[i].item()} for "
                             f"{want[i].item()}, off {off[i].item():.3g}, bound {bound[i].item():.3g}")


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")
