"""The table of tensor maps without memory: a small program around it, with a driver that only counts and an allocator that fails (no GPU needed)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cuda.h>
#include <cuda_runtime.h>
static int encodes = 0;
static CUresult encode(CUtensorMap* m, ...) { ++encodes; *reinterpret_cast<unsigned char*>(m) = 7; return CUDA_SUCCESS; }
static cudaError_t entry_point(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* q) {
    *f = (void*)encode; *q = cudaDriverEntryPointSuccess; return cudaSuccess;
}
#define cudaGetDriverEntryPoint entry_point
#include "csrc/tensor_map.cu"
extern bool no_memory;
int main() {
    alignas(64) CUtensorMap m;
    const cuuint64_t dims[2] = {64, 128}, strides[1] = {128};
    const cuuint32_t box[2] = {64, 128};
    auto ask = [&]() { return dr::tmap_tiled(&m, 2, (void*)4096, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE); };
    setenv("A_TUNABLE_WITH_A_LONG_NAME_OF_ITS_OWN", "5", 1);
    no_memory = true;
    const int a = ask(), b = ask(), t = dr::tunable("A_TUNABLE_WITH_A_LONG_NAME_OF_ITS_OWN", 3);
    no_memory = false;
    const int c = ask(), d = ask();
    printf("%d %d %d %d tunable %d encodes %d\n", a, b, c, d, t, encodes);
    return 0;
}
"""

ALLOCATOR = r"""
#include <cstdlib>
#include <new>
bool no_memory = false;
void* operator new(size_t n) {
    if (no_memory) throw std::bad_alloc();
    return malloc(n);
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }
"""


def test_no_memory_for_the_table_is_no_error(tmp_path):
    src, alloc, exe = tmp_path / "memo.cu", tmp_path / "alloc.cpp", tmp_path / "memo"
    src.write_text(PROGRAM)
    alloc.write_text(ALLOCATOR)
    pkg = os.path.join(ROOT, "paper_1708_04728_b200")
    subprocess.run(["nvcc", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", pkg, "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src), str(alloc)],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    # each of the first two calls encodes (nothing is kept), then one more whose answer the last call finds
    assert r.returncode == 0 and r.stdout.split() == "0 0 0 0 tunable 5 encodes 3".split(), (r.returncode, r.stdout, r.stderr)
