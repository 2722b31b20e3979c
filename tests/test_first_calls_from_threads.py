"""The entry point of the driver that encodes tensor maps, looked up by the first call: from several threads at once, with a look-up that takes its time."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_07139_b200", "csrc")
PROGRAM = r"""
#include <atomic>
#include <chrono>
#include <thread>
#include <vector>
#include <cuda_runtime.h>
static cudaError_t slow_look_up(const char*, void** p, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* q)
{
    static std::atomic<int> calls{0};
    std::this_thread::sleep_for(std::chrono::milliseconds(100));
    *p = reinterpret_cast<void*>(&slow_look_up);
    *q = cudaDriverEntryPointSuccess;
    return calls.fetch_add(1) == 0 ? cudaErrorUnknown : cudaSuccess;         // the first one fails
}
#define cudaGetDriverEntryPointByVersion slow_look_up
#include "fq_umma.cuh"
int main()
{
    if (fq::tensor_map_encoder()) return 100;                                // a failure is one call's, not the process's
    std::atomic<int> none{0}, waiting{8};
    std::vector<std::thread> threads;
    for (int i = 0; i < 8; i++)
        threads.emplace_back([&] {
            waiting--;
            while (waiting > 0) std::this_thread::yield();
            if (!fq::tensor_map_encoder()) none++;
        });
    for (auto& t : threads) t.join();
    return none;
}
"""


@pytest.mark.skipif(shutil.which("nvcc") is None, reason="no nvcc")
def test_all_of_them_get_it(tmp_path):
    source, program = tmp_path / "first.cu", tmp_path / "first"
    source.write_text(PROGRAM)
    subprocess.check_call(["nvcc", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static", "-I", CSRC, "-o", str(program), str(source),
                           "-lpthread"])
    assert subprocess.run([str(program)], timeout=60).returncode == 0
