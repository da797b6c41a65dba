"""The build refuses a library whose kernels spill vector registers (CPU: hipcc cross-compiles)."""
import os

import pytest

from paper_2609_36757_amd import build

# sixteen registers for sixty-four values that all stay live; and an array indexed by data, which goes to scratch
SPILLS = """
#include <hip/hip_runtime.h>
extern "C" __global__ __attribute__((amdgpu_num_vgpr(16))) void too_many_values(float* x) {
  float v[64];
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i] = x[i * 64 + threadIdx.x];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 64; ++i) x[(63 - i) * 64 + threadIdx.x] = v[i] * v[(i * 7 + 3) % 64];
}
"""
SCRATCH = """
#include <hip/hip_runtime.h>
extern "C" __global__ void indexed_array(float* x, const int* at) {
  float v[64];
  for (int i = 0; i < 64; ++i) v[at[i] & 63] = x[i];
  x[threadIdx.x] = v[at[threadIdx.x] & 63];
}
"""
CLEAN = """
#include <hip/hip_runtime.h>
extern "C" __global__ void fine(float* x) { x[threadIdx.x] *= 2.f; }
"""


@pytest.fixture
def library(tmp_path, monkeypatch):
    def write(text):
        (tmp_path / "k.hip").write_text(text)
        return build.build()
    monkeypatch.setattr(build, "CSRC", str(tmp_path))
    monkeypatch.setattr(build, "SOURCES", ["k.hip"])
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib.so"))
    return write


@pytest.mark.parametrize("text,name", [(SPILLS, "too_many_values"), (SCRATCH, "indexed_array")],
                         ids=["registers", "scratch"])
def test_spilling_kernels_are_refused(library, tmp_path, text, name):
    path = library(CLEAN)
    before = os.stat(path).st_mtime_ns, os.path.getsize(path)
    with pytest.raises(RuntimeError, match=name):
        library(text + CLEAN.replace("#include <hip/hip_runtime.h>", ""))
    # the library that was there stays, and nothing is left beside it
    assert (os.stat(path).st_mtime_ns, os.path.getsize(path)) == before
    assert sorted(os.listdir(tmp_path)) == ["k.hip", "lib.so"]


def test_a_failed_compile_still_says_why(library):
    with pytest.raises(RuntimeError, match="no_such_name"):
        library(CLEAN + "int f() { return no_such_name; }\n")
