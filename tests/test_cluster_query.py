"""How many clusters a device holds, as the token operators ask it: only the device's own answers are kept.  A small
program compiled against the header, with a stand-in for the query (no GPU)."""
import os
import subprocess

from paper_2509_26092_gb300 import build_lib

PROGRAM = r"""
#include <cuda_runtime.h>
#include <cstdio>

static cudaError_t g_answer = cudaSuccess;
static int g_count = 0, g_asked = 0;
template <class K>
cudaError_t query(int* n, K, const cudaLaunchConfig_t*)
{
    ++g_asked;
    *n = g_answer == cudaSuccess ? g_count : -7;
    return g_answer;
}
#define cudaOccupancyMaxActiveClusters query
#include "dbl_elem.cuh"

namespace dbl {
int set_error(int code, const char*, ...) { return code; }
void count_launch() {}
int max_cluster() { return 8; }
int sm_count() { return 152; }
}
__global__ void kernel() {}

int main()
{
    auto ask = [](cudaError_t e, int count, int dev, int S) {
        g_answer = e, g_count = count;
        return dbl::clusters_held<kernel>(dev, S, 256, 0);
    };
    int bad = 0;
    auto expect = [&](int got, int want, int asked, const char* what) {
        if (got != want || g_asked != asked) std::printf("%s: %d for %d, asked %d for %d\n", what, got, want, g_asked, asked), bad = 1;
    };
    expect(ask(cudaErrorMemoryAllocation, 5, 0, 4), 0, 1, "an error is no answer");
    expect(ask(cudaSuccess, 5, 0, 4), 5, 2, "asked again after it");
    expect(ask(cudaErrorMemoryAllocation, 9, 0, 4), 5, 2, "an answer stays");
    expect(ask(cudaErrorInvalidClusterSize, 0, 0, 8), 0, 3, "a size that the device does not have");
    expect(ask(cudaSuccess, 5, 0, 8), 0, 3, "is an answer");
    expect(ask(cudaSuccess, 0, 1, 4), 0, 4, "another device");
    expect(ask(cudaSuccess, 5, 1, 4), 0, 4, "none is an answer too");
    expect(ask(cudaSuccess, 5, 0, 16), 0, 4, "above the largest cluster");
    return bad;
}
"""


def test_only_the_devices_answers_are_kept(tmp_path):
    src, exe = tmp_path / "query.cu", tmp_path / "query"
    src.write_text(PROGRAM)
    cmd = [build_lib._nvcc()] + build_lib.ARCH + ["-std=c++17", "-I", build_lib.CSRC, "-I", build_lib.INCLUDE, str(src), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""))
    assert r.returncode == 0, r.stdout + r.stderr
