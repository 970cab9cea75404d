"""The weight gradient's error in its norm, over long groups: chains of 512 rows on the tensor cores, whose sums are added in
fp32, in one piece or in parts.

A tensor core takes 16 rows a step: it adds 16 products and the sum so far, of each of which it cuts the digits below fp32's of
the largest, half a unit in the mean and a unit at the most, a unit being at most 2^-23 of the running sum.  A chain has 32 steps.
  Terms of both signs: the running sum grows as the root of the steps, so that it has 2/3 of the chain's size in the mean and its
  square 1/2.  The sum's own cuts go one way: 32 * 2^-24 * 2/3.  The products' have the signs of the products, independent of each
  other, with a root mean square of a unit / sqrt(3): sqrt(16 * 32 / 2) * 2^-23 / sqrt(3).
  Positive terms: the running sum has half of the chain's size in the mean, and all cuts go one way: 17 * 32 * 2^-24 / 2.  (A
  product of bf16 values has 16 digits, of which few are cut; one of fp16 values has 22.)
Each addition of chains and parts afterwards rounds to nearest: 2^-24 / sqrt(3) of the sum in the root mean square at the most,
which add up in squares.  One chain over all rows of the unsplit cases would be off by 16 times the first terms, parts held in 16
bits by 2^-9."""
import pytest
import torch

from gpu_common import check_status, load_dbl, ws
from token_cases import DTYPE, precision

pytestmark = pytest.mark.gpu

CASES = [  # rows of a group, groups, n_in, n_out, split
    (8192, 19, 512, 512, False), (8189, 38, 256, 512, False), (65000, 1, 512, 512, True), (20011, 2, 512, 264, True)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_weight_gradient_of_long_groups(kind, positive, accumulate, case):
    D = load_dbl()
    rows, groups, n_in, n_out, split = case
    gen = torch.Generator(device="cuda").manual_seed(rows)
    new = lambda c: torch.randn((groups * rows, c), device="cuda", generator=gen)
    x, dy = (t.abs() if positive else t for t in (new(n_in), new(n_out)))
    x, dy = x.to(DTYPE[kind]), dy.to(DTYPE[kind])
    off = torch.arange(groups + 1, dtype=torch.int32, device="cuda") * rows
    dw = torch.ones((groups, n_out, n_in), device="cuda")
    fmt, _ = precision(D, kind)
    with fmt:
        shape = D.grouped_shape(groups * rows, groups, n_in, n_out)
        need = D.dbl_grouped_workspace_bytes(shape, D.DBL_PASS_WGRAD)
        parts = max(1, need // (dw.numel() * 4))
        assert (parts > 1) == split
        D.dbl_grouped_wgrad(shape, x, dy, off, dw, accumulate, ws(need), need)
    check_status(D)
    size = off_by = 0.0
    for g in range(groups):
        a, b = (t[g * rows:(g + 1) * rows].double() for t in (x, dy))
        want = b.t() @ a + (1.0 if accumulate else 0.0)
        size += float(want.square().sum())
        off_by += float((dw[g].double() - want).square().sum())
    additions = -(-rows // 512) + parts + 1
    if positive:
        limit = 17 * 32 * 2.0 ** -24 / 2
    else:
        limit = 32 * 2.0 ** -24 * 2 / 3 + (16 * 32 / 2) ** 0.5 * 2.0 ** -23 / 3 ** 0.5
    limit += additions ** 0.5 * 2.0 ** -24 / 3 ** 0.5
    error = (off_by / size) ** 0.5
    print(f"error {error:.3e}, limit {limit:.3e}")
    assert error <= limit
