"""Rows of logits without a distribution, in every kernel that takes rows: NaN in the loss and the gradient of that row,
all of it, and nowhere else."""
import numpy as np
import pytest

from gpu_common import load_dbl
from test_gpu_distill import call, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    return load_dbl()


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
# a warp each, a block each, a cluster each, from memory
@pytest.mark.parametrize("v,k", [(1000, 4), (9001, 4), (9001, 100), (70001, 4), (131071, 80), (2000003, 4)])
@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.5), (1.0, 0.0)])
def test_rows_without_a_distribution_are_nan_everywhere(D, kind, v, k, tau, alpha):
    rows = 6
    z, top, cls, labels = problem(kind, rows, v, k, 3)
    z[1] = -np.inf
    z[2, 17] = np.nan
    z[3, v - 1] = np.inf
    z[4, 0], z[4, v // 2] = np.inf, -np.inf
    _, row, loss, dz = call(D, kind, z, top, cls, labels if alpha < 1 else None, None, tau, alpha)
    bad, rest = [1, 2, 3, 4], [0, 5]
    assert np.isnan(row[bad]).all() and np.isnan(loss)
    assert np.isnan(dz[bad]).all()
    assert np.isfinite(row[rest]).all() and np.isfinite(dz[rest]).all()
