"""First calls from several threads at once: what the library looks up once per process is there for every one of them.  On the host, against
a stand-in for the CUDA runtime's lookup of a driver function."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
NVCC = os.environ.get("NVCC", os.path.join(CUDA, "bin", "nvcc"))

HARNESS = r"""
#include "tma.cu"

#include <atomic>
#include <chrono>
#include <cstdio>
#include <thread>

static std::atomic<int> lookups{0}, encodings{0};
static CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                       CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
  ++encodings;
  return CUDA_SUCCESS;
}
// takes its time: the other threads meet it half done
extern "C" cudaError_t CUDARTAPI cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* r) {
  ++lookups;
  std::this_thread::sleep_for(std::chrono::milliseconds(300));
  *f = reinterpret_cast<void*>(&encode);
  *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}

int main() {
  std::atomic<int> done{0};
  std::thread threads[8];
  for (std::thread& t : threads)
    t = std::thread([&] {
      CUtensorMap m;
      const uint64_t dims[2] = {64, 64}, stride[1] = {64};
      const uint32_t box[2] = {64, 8};
      done += ssdi8::encode_tensor_map(&m, nullptr, 1, 2, dims, stride, box, 0);
    });
  for (std::thread& t : threads) t.join();
  std::printf("%d %d %d\n", done.load(), encodings.load(), lookups.load());
}
"""


@pytest.mark.skipif(not shutil.which(NVCC), reason="no nvcc")
def test_tensor_maps_from_several_threads(tmp_path):
    (tmp_path / "first.cu").write_text(HARNESS)
    exe = str(tmp_path / "first")
    subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "shared", "-I", os.path.join(ROOT, "paper_2608_21952_b200", "csrc"),
                    "-Xlinker", "-rpath=" + os.path.join(CUDA, "lib64"), "-o", exe, str(tmp_path / "first.cu")], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["8", "8", "1"]   # every thread had its map, and one of them looked the function up
