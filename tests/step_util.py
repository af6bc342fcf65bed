"""Helpers for the tests of the operators around the layers: device tensors
with guarded surroundings, and the rounding of a result's type."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                       # half a step of fp32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def tdt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def values(x, dtype):
    """fp64 numpy values of x as `dtype` holds them."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(tdt(dtype)).double().numpy()


def dev(x, dtype="f32", offset=0):
    """A device tensor of x's values; its first entry lies `offset` entries behind an allocation's start."""
    import torch
    x = np.asarray(x)
    buf = torch.empty(x.size + offset, dtype=tdt(dtype), device="cuda")
    t = buf[offset:].view(x.shape)
    t.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)))
    return t


GUARD = 64                           # entries; the marker 776 = 97 * 8 is exact in bf16


class Guarded:
    """An output tensor between two runs of a marker value that the call has to leave as they are."""

    def __init__(self, shape, dtype, offset=0):
        import torch
        n = int(np.prod(shape))
        self.buf = torch.full((n + 2 * GUARD + offset,), 776.0, dtype=tdt(dtype), device="cuda")
        self.lo, self.n = GUARD + offset, n
        self.t = self.buf[self.lo:self.lo + n].view(shape)

    def np(self):
        out = self.t.double().cpu().numpy()
        around = self.buf.double().cpu().numpy()
        assert (around[:self.lo] == 776.0).all() and (around[self.lo + self.n:] == 776.0).all(), "written outside"
        return out


def within(got, ref, bound):
    """|got - ref| <= bound everywhere (bound: array of absolute errors)."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert np.isfinite(got).all()
    over = np.abs(got - ref) - bound
    assert (over <= 0).all(), f"max |error| {np.abs(got - ref).max():.3g}, over the bound by {over.max():.3g}"
