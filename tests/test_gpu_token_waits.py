"""The bounded waits that the token operators' kernels share, made to run out: a program of its own, compiled against the
header, whose barrier nothing arrives at.  The wait gives up after its limit of two seconds, says so in the status word,
no further wait of the block takes long, the cluster's blocks leave together, and the context stays usable."""
import subprocess

import pytest

from gpu_common import need_gpu
from paper_2509_26092_gb300 import build_lib

pytestmark = pytest.mark.gpu

PROGRAM = r"""
#include <cstdio>
#include "dbl_elem.cuh"

namespace dbl {
int set_error(int code, const char*, ...) { return code; }
void count_launch() {}
int max_cluster() { return 16; }
int sm_count() { return 1; }
}
using namespace dbl::dev;

__device__ int g_status;
struct Out { unsigned long long first, second, leave; int abort, value; };

// Two blocks: the first waits at a barrier that nothing arrives at (`stall`), or at one that it arrives at itself; then it
// sends a pair to the second, which waits for it.
__global__ void __cluster_dims__(2) kernel(int stall, Out* out)
{
    __shared__ alignas(8) unsigned long long bar_[2];
    __shared__ int abort_;
    __shared__ alignas(8) float2 pair;
    uint64_t* bar = reinterpret_cast<uint64_t*>(bar_);
    const int rank = (int)cluster_ctarank();
    if (threadIdx.x == 0) {
        mbar_init(&bar[0], 1);
        mbar_init(&bar[1], 1);
        abort_ = 0, pair = make_float2(0.f, 0.f);
        fence_mbar_init();
    }
    cluster_sync_all();
    uint64_t t0 = globaltimer(), t1 = t0, t2 = t0;
    if (rank == 0) {
        if (threadIdx.x == 0 && !stall) mbar_arrive(&bar[0]);
        bounded_wait(&bar[0], 0, &abort_, &g_status);
        t1 = globaltimer();
        __syncthreads();
        if (stall) bounded_wait(&bar[0], 0, &abort_, &g_status);
        t2 = globaltimer();
        if (threadIdx.x == 0)
            st_async2(mapa_shared(smem_u32(&pair), 1), mapa_shared(smem_u32(&bar[1]), 1), make_float2(3.f, 4.f));
    } else {
        if (threadIdx.x == 0) mbar_arrive_expect_tx(&bar[1], sizeof(float2));
        bounded_wait(&bar[1], 0, &abort_, &g_status);
        t1 = t2 = globaltimer();
    }
    __syncthreads();
    const int value = (int)(pair.x + pair.y);  // the second block's, if it came in time
    linger(&abort_);
    cluster_leave();
    if (threadIdx.x == 0) out[rank] = {t1 - t0, t2 - t1, globaltimer() - t2, abort_, value};
}

int run(int stall, Out* out, int* status)
{
    Out* d;
    if (cudaMalloc(&d, 2 * sizeof(Out)) != cudaSuccess) return 1;
    kernel<<<2, 64>>>(stall, d);
    if (cudaDeviceSynchronize() != cudaSuccess) return 2;
    if (cudaMemcpy(out, d, 2 * sizeof(Out), cudaMemcpyDeviceToHost) != cudaSuccess) return 3;
    if (dbl::status_read(g_status, status) != DBL_OK || dbl::status_clear(g_status) != DBL_OK) return 4;
    return cudaFree(d) != cudaSuccess;
}

int main()
{
    const double ms = 1e-6;
    for (int stall : {0, 1, 0}) {
        Out o[2];
        int status = -1;
        if (const int e = run(stall, o, &status)) return std::printf("error %d\n", e), 1;
        for (const Out& b : o)
            std::printf("stall %d: first %.3f ms, second %.3f ms, leave %.3f ms, abort %d, value %d, status %d\n", stall, b.first * ms,
                        b.second * ms, b.leave * ms, b.abort, b.value, status);
        if (!stall) {
            if (status != DBL_OK || o[0].abort || o[1].abort || o[1].value != 7 || (o[0].first + o[1].first) * ms > 100) return 2;
        } else {
            // the second block may have given up as well: its limit runs from the same time
            if (status != DBL_ERR_TIMEOUT || !o[0].abort || o[0].first * ms < 1900 || o[0].first * ms > 4000) return 3;
            if (o[0].second * ms > 500 || o[1].first * ms > 4000 || (!o[1].abort && o[1].value != 7)) return 4;
            if (o[0].leave * ms > 1500 || o[1].leave * ms > 1500) return 5;
        }
    }
    return 0;
}
"""


def test_a_wait_that_runs_out_is_reported_and_the_context_survives(tmp_path):
    need_gpu()
    src, exe = tmp_path / "waits.cu", tmp_path / "waits"
    src.write_text(PROGRAM)
    cmd = [build_lib._nvcc()] + build_lib.ARCH + ["-std=c++17", "-I", build_lib.CSRC, "-I", build_lib.INCLUDE, str(src), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
