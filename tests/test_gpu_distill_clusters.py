"""Rows that clusters of blocks share: blocks that have begun at different times, beside rows that end at once."""
import numpy as np
import pytest

from gpu_common import load_dbl
from test_gpu_distill import call, check, problem

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def D():
    return load_dbl()


# sizes that take 2 to 16 blocks a row on 152 SMs; parts of a few units at the row's end among them
@pytest.mark.parametrize("kind,rows,v", [("f16", 9, 131071), ("f32", 5, 65537), ("bf16", 60, 60001), ("bf16", 200, 50257),
                                         ("f32", 300, 50001), ("bf16", 3, 8193), ("f32", 1, 4 * 16 * 128 + 1)])
def test_rows_of_a_cluster_beside_rows_of_weight_0(D, kind, rows, v):
    z, top, cls, labels = problem(kind, rows, v, 5, 11)
    w = np.linspace(0.5, 1.5, rows).astype(np.float32)
    w[1::3] = 0.0
    first = None
    for _ in range(5):
        got = call(D, kind, z, top, cls, labels, w, 2.0, 0.5, 64.0)
        if first is None:
            first = got
            check(kind, got[0], got, top, cls, labels, w, 2.0, 0.5, 64.0)
        assert all(np.array_equal(a, b) for a, b in zip(first, got))
