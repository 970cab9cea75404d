"""Every worker draws its dropout masks from a seed of its own, also where none is given, and every place of it (no GPU)."""
import pytest

from oracle import experts as orc
from paper_2509_26092_gb300 import build_lib


@pytest.fixture(scope="module")
def TS():
    build_lib.build()
    from paper_2509_26092_gb300 import token_step
    return token_step


def seeds(TS, n, **kw):
    worker = TS.TokenWorker(TS.TokenSpec(64, 2, 10, 4, 64), n, 5, 2, device="cpu", dropout=0.5, **kw)
    return [shape.seed for shape in worker.drops]


def test_workers_without_a_seed_draw_other_masks(TS):
    large, small = seeds(TS, 4), seeds(TS, 1)  # as a program makes the two workers of an iteration
    every = large + small + seeds(TS, 4) + seeds(TS, 4, seed=0) + seeds(TS, 4, seed=1)
    assert len(large) == 4 and len(set(every)) == len(every)
    masks = [orc.dropout_mask(5, 64, 0.5, s, 0).tobytes() for s in large + small]
    assert len(set(masks)) == len(masks)


def test_a_given_seed_is_the_workers(TS):
    assert seeds(TS, 4, seed=99) == seeds(TS, 1, seed=99) != seeds(TS, 1, seed=98)
    assert seeds(TS, 1, seed=99) == [99 ^ (0x9E3779B97F4A7C15 * (i + 1)) % 2 ** 64 for i in range(4)]
    assert seeds(TS, 1, seed=-1) == seeds(TS, 1, seed=2 ** 64 - 1)
