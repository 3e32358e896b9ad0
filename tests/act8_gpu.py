"""Shared by the GPU tests of the 8-bit activations: types, guarded buffers, steps of rounding."""
from __future__ import annotations

import numpy as np
import torch

import act8_reference as ref
import paper_2002_11082_b200 as ogq

DTYPES = {"f32": (ogq.OGQ_F32, torch.float32), "f16": (ogq.OGQ_F16, torch.float16), "bf16": (ogq.OGQ_BF16, torch.bfloat16)}
ACTS = {"none": (ogq.OGQ_ACT_NONE, ref.NONE), "relu": (ogq.OGQ_ACT_RELU, ref.RELU), "silu": (ogq.OGQ_ACT_SILU, ref.SILU),
        "gelu": (ogq.OGQ_ACT_GELU, ref.GELU)}
U24 = 2.0 ** -24  # half a step of fp32, relative


def half_step(dt: torch.dtype) -> float:
    return torch.finfo(dt).eps / 2


def smallest(dt: torch.dtype) -> float:
    """Half a step of the subnormal numbers."""
    return float(torch.finfo(dt).smallest_normal) * torch.finfo(dt).eps / 2


class Guarded:
    """A matrix [rows, cols] with row stride ld inside a larger buffer, `shift` elements behind its 256-byte boundary;
    check() finds whatever was written outside the matrix."""

    def __init__(self, rows, cols, ld, dtype, shift=0, data=None):
        self.rows, self.cols, self.ld, self.shift = rows, cols, ld, shift
        n = max(rows, 1) * ld + shift + 64
        if dtype.is_floating_point:
            self.buf = torch.full((n,), -77.0, dtype=dtype, device="cuda")
        else:
            self.buf = torch.full((n,), 0x55, dtype=dtype, device="cuda")
        self.before = self.buf.clone()
        self.t = self.buf[shift:shift + max(rows, 1) * ld].view(max(rows, 1), ld)[:rows, :cols]
        if data is not None:
            self.t.copy_(data)

    def check(self):
        torch.cuda.synchronize()
        same = self.buf.view(torch.uint8).view(len(self.buf), -1) == self.before.view(torch.uint8).view(len(self.buf), -1)
        same = same.all(1)
        same[self.shift:self.shift + max(self.rows, 1) * self.ld].view(max(self.rows, 1), self.ld)[:self.rows, :self.cols] = True
        assert bool(same.all()), "written outside the matrix"

    def numpy(self):
        torch.cuda.synchronize()
        return self.t.double().cpu().numpy()


def kept(rows, cols, shift=0):
    return Guarded(rows, cols, cols, torch.int8, shift), Guarded(rows, ref.groups(cols), ref.groups(cols), torch.uint8, shift)


def activations(rng, rows, cols, dt):
    """Normal values with a scale per column, rounded to the type: groups with small values beside large ones, some groups all zero."""
    x = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal(cols))
    if rows > 1 and cols > 32:
        x[0, :32] = 0.0
    return torch.from_numpy(x).to(dt)


def assert_near(got, want, tol, what=""):
    d = np.abs(got - want)
    bad = ~(d <= tol) & ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, the worst {float(np.nanmax(np.where(bad, d, 0)))} at {np.argwhere(bad)[:3].tolist()}"
