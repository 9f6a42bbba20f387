"""Products of tiles on the host: every thread of a workgroup, with checked array indexes and matrix instructions that count themselves."""
import subprocess

import pytest

from tests.test_activation_texts import CSRC

CLANG = "/opt/rocm/llvm/bin/clang++"

# what device code takes from the compiler, for a host: a matrix instruction adds one to its sums
STUBS = r"""
#include <cstdint>
#include <cstdio>
#define __device__
#define __shared__ static
struct Dim { unsigned x; } threadIdx, blockIdx, gridDim;
struct __amdgpu_buffer_rsrc_t { const void* p; };
#define __builtin_amdgcn_readfirstlane(x) (x)
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) ((c) + 1.f)
#define __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, x, y, z) ((c) + 1.0)
#define __builtin_amdgcn_make_buffer_rsrc(p, a, b, c) (__amdgpu_buffer_rsrc_t{p})
#define __builtin_amdgcn_raw_buffer_load_b32(b, o, x, y) (0u)
#define __builtin_amdgcn_raw_buffer_load_b64(b, o, x, y) (u32x2{0, 0})
#define __builtin_amdgcn_raw_buffer_load_b128(b, o, x, y) (u32x4{0, 0, 0, 0})
"""

MAIN = r"""
#include "product.hpp"
using namespace cgtp;
int main() {
  typedef %(type)s T;
  typedef Results<T, %(rows)d, %(columns)d, %(up)d, %(across)d> R;
  static Operand<T, %(rows)d, %(by)s> left;
  static Operand<T, %(columns)d, %(by)s> right;
  for (threadIdx.x = 0; threadIdx.x < R::kThreads; ++threadIdx.x) {
    R r;
    r.multiply(left, right);
    for (int i = 0; i < R::RT; ++i)
      for (int j = 0; j < R::CT; ++j)
        for (int k = 0; k < 4; ++k)
          if (r.acc[i][j][k] != (sizeof(T) == 4 ? 6 : 8)) return std::printf("thread %%u: %%g products of tile %%d %%d\n", threadIdx.x, (double)r.acc[i][j][k], i, j), 1;
  }
}
"""


# of A with 32, 64, 96 and 128 rows (orth_kernels.hpp), and of the tiles of results
@pytest.mark.parametrize("type_,rows,columns,up,across,by", [
    ("float", 32, 32, 2, 2, "kApart"), ("float", 64, 64, 2, 2, "kApart"), ("float", 64, 64, 2, 4, "kApart"), ("float", 96, 96, 2, 3, "kApart"), ("float", 128, 128, 2, 4, "kApart"),
    ("double", 32, 32, 2, 2, "kApart"), ("double", 64, 64, 2, 2, "kApart"), ("double", 96, 96, 2, 2, "kApart"), ("double", 128, 128, 2, 2, "kApart"),
    ("float", 128, 128, 2, 2, "kWholeRows"), ("float", 128, 64, 2, 2, "kWholeRows"), ("float", 64, 128, 2, 2, "kWholeRows"), ("float", 64, 64, 2, 2, "kWholeRows"),
    ("double", 64, 64, 2, 2, "kWholeRows"), ("double", 32, 64, 2, 2, "kWholeRows")])
def test_products_stay_inside_their_tiles(type_, rows, columns, up, across, by, tmp_path):
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text(STUBS)
    (tmp_path / "main.cpp").write_text(MAIN % dict(type=type_, rows=rows, columns=columns, up=up, across=across, by=by))
    program = str(tmp_path / "main")
    made = subprocess.run([CLANG, "-std=c++17", "-O0", "-w", "-fsanitize=bounds", "-fsanitize-trap=bounds", "-I", str(tmp_path), "-I", CSRC, str(tmp_path / "main.cpp"), "-o", program],
                          capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-2000:]
    ran = subprocess.run([program], capture_output=True, text=True)
    assert ran.returncode == 0, (ran.returncode, ran.stdout)
