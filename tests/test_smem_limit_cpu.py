"""Two host threads on the first calls of one kernel with different amounts of shared memory: whichever comes second, neither is left
with a limit below what it asked for.  The library's host code with a stand-in for the call that sets the limit; no GPU."""
import os
import subprocess

from paper_2607_08991_gb300 import build

SOURCE = r"""
#include <cuda_runtime.h>
#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>
static std::atomic<int> limit{0};
template <typename K> static cudaError_t slow_set(K, cudaFuncAttribute, int bytes)
{
    limit = bytes;                                                   // as the runtime does: the last one counts
    std::this_thread::sleep_for(std::chrono::milliseconds(200));     // (a descheduled thread)
    return cudaSuccess;
}
#define cudaFuncSetAttribute slow_set
#include "tc_common.cuh"

__global__ void kernel() {}

int main()
{
    static std::atomic<int> configured[64];
    std::atomic<int> below{0};
    const auto call = [&](int wait_ms, int bytes) {
        std::this_thread::sleep_for(std::chrono::milliseconds(wait_ms));
        const cudaError_t e = sats::tc::set_smem(kernel, bytes, configured);
        if (e != cudaSuccess || limit < bytes) ++below;              // the launch behind it would fail
    };
    std::thread a(call, 0, 110000), b(call, 50, 104000), c(call, 500, 112000);
    a.join();
    b.join();
    c.join();
    const int after = limit;
    call(0, 111000);                                                 // (and what the record says is there)
    std::printf("%d below, limit %d\n", below.load(), after);
    return below.load();
}
"""


def test_concurrent_first_calls(tmp_path):
    src, exe = tmp_path / "limit.cu", tmp_path / "limit"
    src.write_text(SOURCE)
    subprocess.check_call([build.nvcc(), *build.ARCH, "-std=c++17", "-O1", "-w", "-I", build.INCLUDE, "-I", build.CSRC, str(src), "-o",
                           str(exe), "-cudart", "static", "-lpthread"])
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert done.returncode == 0, done.stdout + done.stderr
