"""Bounds for the operators of a transformer block against a 64-bit evaluation, from the arithmetic they use.

An output is off by at most half a step of its type (HALF, relative), plus the error of the sums: every addition and
product in the sums' type is off by at most ACC relative (binary32 sums: 2^-23, which also covers sums that are cut off instead of
rounded), plus half the smallest step of the type (TINY) where it underflows.
"""
import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "f64": torch.float64}
HALF = {k: torch.finfo(t).eps / 2 for k, t in DT.items()}
ACC = {"f32": 2.0 ** -23, "f16": 2.0 ** -23, "bf16": 2.0 ** -23, "f64": 2.0 ** -51}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f64": 0.0}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, kind, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float64) * std + mean).to(DT[kind])


class Buffer:
    """An output of `shape` with guard words on both sides, filled with a pattern."""
    PAD = 64

    def __init__(self, shape, dtype, fill=0x5A):
        n = 1
        for s in shape:
            n *= s
        self.full = torch.empty(n + 2 * self.PAD, dtype=dtype, device="cuda")
        self.full.view(torch.uint8).fill_(fill)
        self.t = self.full[self.PAD:self.PAD + n].view(shape)
        self.fill = fill

    def intact(self):
        raw, pad = self.full.view(torch.uint8), self.PAD * self.full.element_size()
        return bool((raw[:pad] == self.fill).all()) and bool((raw[raw.numel() - pad:] == self.fill).all())


def within(name, got, want, bound):
    """Every element of `got` within `bound` of `want` (both float64); non-finite ones equal."""
    got = got.double()
    assert got.shape == want.shape, name
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{name}: NaN in other places"
    off = (got - want).abs()
    bad = fine & ~(off <= bound)
    worst = (off / bound.clamp(min=1e-300))[fine].max().item() if fine.any() else 0.0
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {worst:.2f} times"
    other = ~fine & ~torch.isnan(want)
    assert torch.equal(got[other], want[other]), f"{name}: infinities"
