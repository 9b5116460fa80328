"""First calls that two host threads make at the same time: what is looked up once for the process is whole before anyone uses it."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_26558_b200", "csrc")

# A runtime whose look-up takes a while, in place of CUDA's: the second thread asks while the first one's is under way.
_SLOW_LOOKUP = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include "tc.cuh"
static int found;
static std::atomic<int> lookups{0};
extern "C" cudaError_t CUDARTAPI cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    ++lookups;
    std::this_thread::sleep_for(std::chrono::milliseconds(300));
    *fn = &found;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
int main() {
    void *a = nullptr, *b = nullptr;
    std::thread first([&] { a = (void*)cass::encode_fn(); });
    std::this_thread::sleep_for(std::chrono::milliseconds(100));
    std::thread second([&] { b = (void*)cass::encode_fn(); });
    first.join();
    second.join();
    std::printf("%d %d %d\n", a == &found, b == &found, lookups.load());
}
"""


def test_tensor_map_encoder_is_looked_up_once_for_all_threads(tmp_path):
    from paper_2605_26558_b200 import build
    src, exe = tmp_path / "lookup.cu", tmp_path / "lookup"
    src.write_text(_SLOW_LOOKUP)
    r = subprocess.run([build.NVCC, "-std=c++17", "--expt-relaxed-constexpr", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "shared", "-I", CSRC,
                        str(src), "-o", str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.split() == ["1", "1", "1"], (r.stdout, r.stderr)
