"""First calls that two host threads make at the same time: what is looked up once for the process is whole before anyone uses it."""
import os
import subprocess
import sys

import pytest

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


# An encoder that wants a context bound, as CUDA's does, in a thread that has none.
_UNBOUND = r"""
#include <cstdio>
#include "tc.cuh"
extern "C" int bound;
static int asked;
static CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                       CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    ++asked;
    return bound ? CUDA_SUCCESS : CUDA_ERROR_INVALID_CONTEXT;
}
extern "C" cudaError_t CUDARTAPI cudaGetDriverEntryPoint(const char*, void** fn, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    *fn = (void*)&encode;
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
int main() {
    CUtensorMap map;
    const int first = cass::tc_matrix_map(&map, &map, 64, 64, 16), again = cass::tc_matrix_map(&map, &map, 64, 64, 16);
    std::printf("%d %d %d\n", first, again, asked);
}
"""
_DEVICE_3 = r"""
extern "C" {
int bound = 0;
int cudaGetDevice(int* dev) { *dev = 3; return 0; }
int cudaSetDevice(int dev) { bound = dev == 3; return 0; }
}
"""


def _output(tmp_path, source, runtime=""):
    from paper_2605_26558_b200 import build
    src, more, exe = tmp_path / "host.cu", tmp_path / "runtime.cpp", tmp_path / "host"
    src.write_text(source)
    more.write_text(runtime)
    r = subprocess.run([build.NVCC, "-std=c++17", "--expt-relaxed-constexpr", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "shared", "-I", CSRC,
                        str(src), str(more), "-o", str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    return r.stdout.split()


def test_tensor_map_encoder_is_looked_up_once_for_all_threads(tmp_path):
    assert _output(tmp_path, _SLOW_LOOKUP) == ["1", "1", "1"]


def test_tensor_maps_in_a_thread_without_a_context(tmp_path):
    assert _output(tmp_path, _UNBOUND, _DEVICE_3) == ["0", "0", "3"]


_TWO_FIRST_CALLS = r"""
import threading
import torch
import paper_2605_26558_b200 as cass

B, NQ, NK, D, P = 40, 8, 2, 128, 700
geom, attn = cass.CacheGeom(cass.BF16, B, NK, D, 0, 0, 0, 0), cass.SharedAttn(NQ, 1, NQ * D, NQ * D, D, NQ * D, NQ * D, D, P, NK * D, D, 0.0)
q, kp, vp = (torch.randn(*n, device="cuda").to(torch.bfloat16) for n in ((B, 1, NQ, D), (P, NK, D), (P, NK, D)))
out = [torch.zeros_like(q) for _ in range(2)]
scratch = [torch.zeros(cass.cass_shared_prefix_scratch_bytes(geom, attn), dtype=torch.uint8, device="cuda") for _ in range(2)]
status = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)]
streams, start, errors = [torch.cuda.Stream() for _ in range(2)], threading.Barrier(2), []
torch.cuda.synchronize()

def call(i):
    start.wait()
    try:
        cass.cass_shared_prefix_attention(geom, attn, q, kp, vp, None, None, None, out[i], None, None, None, scratch[i], scratch[i].numel(), status[i], streams[i])
    except Exception as e:
        errors.append(repr(e))

threads = [threading.Thread(target=call, args=(i,)) for i in range(2)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert not errors, errors
assert torch.equal(out[0], out[1]) and out[0].abs().amax() > 0 and not any(int(s) for s in status)
"""


@pytest.mark.gpu
def test_two_threads_call_first():
    r = subprocess.run([sys.executable, "-c", _TWO_FIRST_CALLS], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
