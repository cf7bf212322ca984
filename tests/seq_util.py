"""Helpers of the tests of the operators over sequences: arrays as they may lie in memory, and comparison within the bounds
that the oracle derives."""
import numpy as np
import torch

from paper_1606_03401_b200 import synth

EPS = 2.0 ** -24
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}       # rounding to the type, relative to the value
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}
SENTINEL = 977.0


def rounded(a, dtype):
    return synth.round_to_bf16(a) if dtype == "bf16" else synth.round_to_fp32(a)


def device(a, dtype="fp32"):
    """A dense CUDA tensor of the type, or None."""
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to(TORCH[dtype])


class Laid:
    """An array [t, batch, width] that lies in memory as the layout says; what is around it holds a sentinel."""

    def __init__(self, shape, dtype, layout, fill=None):
        t, n, d = shape
        new = dict(dtype=TORCH[dtype], device="cuda")
        if layout == "batch":
            self.memory = torch.full((n, t, d), SENTINEL, **new)
            self.x = self.memory.transpose(0, 1)
        elif layout == "sliced":                 # columns of a wider array, on 16-byte boundaries where the width allows
            self.memory = torch.full((t, n, 2 * d + 8), SENTINEL, **new)
            self.x = self.memory[:, :, d:2 * d]
        elif layout == "odd":                    # an odd place, gaps behind columns, rows and steps
            self.memory = torch.full((t * (n * (d + 3) + 5) + 1,), SENTINEL, **new)
            self.x = self.memory.as_strided((t, n, d), (n * (d + 3) + 5, d + 3, 1), 1)
        else:
            self.memory = torch.full((t, n, d), SENTINEL, **new)
            self.x = self.memory
        self.mask = torch.ones_like(self.memory, dtype=torch.bool)
        self.mask.as_strided(self.x.shape, self.x.stride(), self.x.storage_offset()).fill_(False)
        if fill is not None:
            self.x.copy_(torch.from_numpy(np.ascontiguousarray(fill)))

    strides = property(lambda self: (self.x.stride(0), self.x.stride(1)))

    def untouched(self):
        return bool((self.memory[self.mask] == SENTINEL).all())

    def numpy(self):
        return self.x.double().cpu().numpy()


def numpy(x):
    return x.double().cpu().numpy()


def assert_within(name, got, ref, bound, dtype):
    """Every element: the bound of the float32 computation, and then the rounding to the type that it is stored in."""
    got, ref = np.asarray(got, np.float64).reshape(np.shape(ref)), np.asarray(ref)
    allowed = EPS * bound
    allowed = allowed + HALF_STEP[dtype] * (np.abs(ref) + allowed) + 1e-37
    off = np.abs(got - ref)
    bad = ~(off <= allowed)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(off / allowed)), np.argwhere(bad)[:3].tolist())
