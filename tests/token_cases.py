"""Helpers of the token operators' GPU tests: tensors with row strides and odd base addresses whose surroundings
are checked, and the error that one rounding to the storage format makes."""
import numpy as np
import torch

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS32 = 2.0 ** -24  # half the spacing of fp32 above 1: the largest relative error of one fp32 rounding
# the same of the formats, and half the spacing of their subnormal numbers
UNIT = {"bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25), "f32": (2.0 ** -24, 2.0 ** -150)}
GUARD = -77.0  # in what surrounds a tensor's rows; held by every format


def precision(D, kind):
    """The library that a case runs on, and the element type that it is given."""
    return D.precision("f16" if kind == "f16" else "bf16"), D.DBL_F32 if kind == "f32" else D.DBL_BF16


class Rows:
    """[rows, c] at row stride ld and `offset` elements after an aligned address, guards everywhere else."""

    def __init__(self, kind, rows, c, ld=0, offset=0, values=None):
        self.rows, self.c, self.ld = rows, c, ld or c
        self.buf = torch.full((offset + rows * self.ld + 64,), GUARD, dtype=DTYPE[kind], device="cuda")
        self.offset = offset
        if values is not None:
            self.view().copy_(torch.as_tensor(np.ascontiguousarray(values)).reshape(rows, c))

    def view(self):
        return self.buf.as_strided((self.rows, self.c), (self.ld, 1), self.offset)

    def ptr(self):
        return self.buf.data_ptr() + self.offset * self.buf.element_size()

    def values(self):
        return self.view().double().cpu().numpy()

    def check_guards(self):
        whole = self.buf.clone()
        whole.as_strided((self.rows, self.c), (self.ld, 1), self.offset).fill_(GUARD)
        assert bool((whole == GUARD).all()), "written outside the rows"


def rounding(kind, value):
    u, sub = UNIT[kind]
    return u * np.abs(value) + sub


def assert_within(got, want, tol, what):
    got, want, tol = (np.asarray(a, np.float64) for a in (got, want, tol))
    tol = np.broadcast_to(tol, want.shape)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    if bad.any():
        i = np.unravel_index(int(np.argmax(np.where(bad, np.abs(got - want) / np.maximum(tol, 1e-300), 0))), want.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, worst at {i}: {got[i]!r} for {want[i]!r}, "
                             f"tolerance {tol[i]!r}")
