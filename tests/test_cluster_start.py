"""Distributed shared memory may be touched only in a block that is known to have begun: in every kernel, a barrier of the
cluster comes before the first access to another block's shared memory (read from the sources, no GPU)."""
import glob
import os
import re

import pytest

from paper_2509_26092_gb300 import build_lib

# a barrier of the cluster that has been waited for, and the calls that begin with one
BARRIER = r"\b(?:cluster_sync_all|cluster_wait|links_init|ex\.init)\s*\("
# stores, loads and arrivals at an address of another block, and the calls that begin with one
REMOTE = r"\b(?:st_cluster_v4|st_async2|st_async4|ld_cluster_f32x4|ld_cluster_f32|mbar_arrive_cluster|mapa_shared|ex\.all)\s*\("


def kernels(path):
    text = re.sub(r"//[^\n]*", "", open(path).read())
    starts = [m.start() for m in re.finditer(r"__global__", text)]
    for a, b in zip(starts, starts[1:] + [len(text)]):
        body = text[a:b]
        yield re.search(r"(\w+)\s*\(", re.sub(r"__launch_bounds__\s*\([^()]*(?:\([^()]*\))?[^()]*\)", "", body)).group(1), body


SOURCES = sorted(glob.glob(os.path.join(build_lib.CSRC, "*.cu")))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_a_cluster_barrier_comes_before_remote_shared_memory(path):
    for name, body in kernels(path):
        remote = re.search(REMOTE, body)
        if remote is None:
            continue
        barrier = re.search(BARRIER, body)
        assert barrier and barrier.start() < remote.start(), f"{os.path.basename(path)}: {name}"


def test_the_kernels_that_exchange_are_seen():
    seen = {name for path in SOURCES for name, body in kernels(path) if re.search(REMOTE, body)}
    assert {"distill_kernel", "scan_fwd_kernel", "scan_bwd_kernel", "ln_fwd_kernel", "ln_bwd_kernel"} <= seen
