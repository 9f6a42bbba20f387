// Gated feed-forward block: out = act(x Wg + bg) * (x Wu + bu), and its gradients.
//
// With g = x Wg + bg, u = x Wu + bu and t = dE/dout:   dg = t u act'(g),  du = t act(g),
//     gx = dg Wg^T + du Wu^T,   gWg = x^T dg,   gWu = x^T du,   gbg = sum dg,   gbu = sum du.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "act.hpp"
#include "layer.hpp"

namespace cgtp {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

// 64 x 64 results a workgroup, 4 x 4 a thread, both projections; operands in steps of 16 through LDS.
template <class T, int kAct, bool kBack>
__global__ void __launch_bounds__(kThreads) k_gated_tile(GatedArgs a, int64_t row0, int64_t rows, T* dg, T* du) {
  __shared__ T sx[kStep][kTile + 1], sg[kStep][kTile + 1], su[kStep][kTile + 1];
  const T *x = (const T*)a.x, *Wg = (const T*)a.Wg, *Wu = (const T*)a.Wu;
  const int64_t n = a.d_out, K = a.d_in, n_tiles = (n + kTile - 1) / kTile;
  const int64_t r0 = blockIdx.x / n_tiles * kTile, c0 = blockIdx.x % n_tiles * kTile;
  const int t = threadIdx.x, tr = t / 16, tc = t % 16;
  T ag[4][4] = {}, au[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += kStep) {
    for (int i = t; i < kTile * kStep; i += kThreads) {
      const int r = i / kStep, k = i % kStep;
      sx[k][r] = r0 + r < rows && k0 + k < K ? x[(row0 + r0 + r) * a.ld_x + k0 + k] : T(0);
      const int c = i % kTile, kk = i / kTile;
      const bool in = c0 + c < n && k0 + kk < K;
      sg[kk][c] = in ? Wg[(k0 + kk) * n + c0 + c] : T(0);
      su[kk][c] = in ? Wu[(k0 + kk) * n + c0 + c] : T(0);
    }
    __syncthreads();
    for (int k = 0; k < kStep; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
          ag[i][j] += sx[k][tr * 4 + i] * sg[k][tc + 16 * j];
          au[i][j] += sx[k][tr * 4 + i] * su[k][tc + 16 * j];
        }
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + tr * 4 + i, c = c0 + tc + 16 * j;
      if (r >= rows || c >= n) continue;
      const T g = ag[i][j] + (a.bg ? ((const T*)a.bg)[c] : T(0)), u = au[i][j] + (a.bu ? ((const T*)a.bu)[c] : T(0));
      T v, d;
      act_both<kAct>(g, v, d);
      if (kBack) {
        const T o = ((const T*)a.gout)[(row0 + r) * a.ld_gout + c];
        dg[r * n + c] = o * u * d;
        du[r * n + c] = o * v;
      } else {
        ((T*)a.out)[(row0 + r) * a.ld_out + c] = v * u;
      }
    }
}

// gx = dg Wg^T + du Wu^T for one piece of rows
template <class T>
__global__ void __launch_bounds__(kThreads) k_gated_gx(GatedArgs a, int64_t row0, int64_t rows, const T* dg, const T* du) {
  __shared__ T sg[kStep][kTile + 1], su[kStep][kTile + 1], wg[kStep][kTile + 1], wu[kStep][kTile + 1];
  const T *Wg = (const T*)a.Wg, *Wu = (const T*)a.Wu;
  const int64_t n = a.d_out, K = a.d_in, k_tiles = (K + kTile - 1) / kTile;
  const int64_t r0 = blockIdx.x / k_tiles * kTile, c0 = blockIdx.x % k_tiles * kTile;
  const int t = threadIdx.x, tr = t / 16, tc = t % 16;
  T acc[4][4] = {};
  for (int64_t n0 = 0; n0 < n; n0 += kStep) {
    for (int i = t; i < kTile * kStep; i += kThreads) {
      const int r = i / kStep, k = i % kStep;
      const bool in = r0 + r < rows && n0 + k < n, win = c0 + r < K && n0 + k < n;
      sg[k][r] = in ? dg[(r0 + r) * n + n0 + k] : T(0);
      su[k][r] = in ? du[(r0 + r) * n + n0 + k] : T(0);
      wg[k][r] = win ? Wg[(c0 + r) * n + n0 + k] : T(0);
      wu[k][r] = win ? Wu[(c0 + r) * n + n0 + k] : T(0);
    }
    __syncthreads();
    for (int k = 0; k < kStep; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
          acc[i][j] += sg[k][tr * 4 + i] * wg[k][tc + 16 * j] + su[k][tr * 4 + i] * wu[k][tc + 16 * j];
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + tr * 4 + i, c = c0 + tc + 16 * j;
      if (r < rows && c < K) ((T*)a.gx)[(row0 + r) * a.ld_gx + c] = acc[i][j];
    }
}

// gW += x^T d for one piece of rows; the workgroups of the first 64 columns of x add up the biases' gradients too
template <class T>
__global__ void __launch_bounds__(kThreads) k_gated_gw(GatedArgs a, int64_t row0, int64_t rows, const T* d, T* gW, T* gb, int first) {
  __shared__ T sx[kStep][kTile + 1], sd[kStep][kTile + 1];
  const T* x = (const T*)a.x;
  const int64_t n = a.d_out, K = a.d_in, n_tiles = (n + kTile - 1) / kTile;
  const int64_t k0 = blockIdx.x / n_tiles * kTile, c0 = blockIdx.x % n_tiles * kTile;
  const int t = threadIdx.x, tr = t / 16, tc = t % 16;
  T acc[4][4] = {}, sum[4] = {};
  for (int64_t r0 = 0; r0 < rows; r0 += kStep) {
    for (int i = t; i < kTile * kStep; i += kThreads) {
      const int r = i / kTile, c = i % kTile;
      sx[r][c] = r0 + r < rows && k0 + c < K ? x[(row0 + r0 + r) * a.ld_x + k0 + c] : T(0);
      sd[r][c] = r0 + r < rows && c0 + c < n ? d[(r0 + r) * n + c0 + c] : T(0);
    }
    __syncthreads();
    for (int r = 0; r < kStep; ++r) {
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] += sx[r][tr * 4 + i] * sd[r][tc + 16 * j];
      for (int j = 0; j < 4; ++j) sum[j] += sd[r][tc + 16 * j];
    }
    __syncthreads();
  }
  for (int j = 0; j < 4; ++j) {
    const int64_t c = c0 + tc + 16 * j;
    if (c >= n) continue;
    for (int i = 0; i < 4; ++i) {
      const int64_t k = k0 + tr * 4 + i;
      if (k < K) gW[k * n + c] = acc[i][j] + (first ? T(0) : gW[k * n + c]);
    }
    if (gb && k0 == 0 && tr == 0) gb[c] = sum[j] + (first ? T(0) : gb[c]);
  }
}

// ---- fp32, up to 128 columns of x ----------------------------------------------------------------------------------------
//
// Products on the matrix cores in bf16, 16 x 16 results from 32 terms an instruction: sixteen times the rate of the fp32 ones.  A
// factor is the sum of three bf16 numbers, which hold its 24 bits; of the nine products of parts the six largest are formed, the
// others are below 2^-25 of the product.  Sums are held in fp32.
//
// A wave keeps the parts of its columns of Wg and Wu in registers for the whole call and walks over rows, whose parts the workgroup
// puts into LDS once for its four waves.

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct Parts {
  bf16x8 p[3];
};

// two numbers as three pairs of bf16
__device__ inline void split(float a, float b, unsigned* p) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
    p[i] = h;
    if (i == 2) break;
    a -= __builtin_bit_cast(float, h << 16);
    b -= __builtin_bit_cast(float, h & 0xffff0000u);
  }
}

__device__ inline Parts split8(const float* v) {
  unsigned w[4][3];
#pragma unroll
  for (int i = 0; i < 4; ++i) split(v[2 * i], v[2 * i + 1], w[i]);
  Parts r;
#pragma unroll
  for (int i = 0; i < 3; ++i) r.p[i] = __builtin_bit_cast(bf16x8, u32x4{w[0][i], w[1][i], w[2][i], w[3][i]});
  return r;
}

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// which parts meet: the smallest products first
constexpr int kPairA[6] = {2, 0, 1, 1, 0, 0}, kPairB[6] = {0, 2, 1, 0, 1, 0};

constexpr int kRows = 64;        // rows in LDS at a time
constexpr int kMaxIn = 128;      // columns of x that the kernels below take

// Rows go through buffer descriptors of at most 64 rows: what lies outside reads as zero and is not written, without a branch.  A
// place that is not wanted inside the descriptor's range gets the offset kNowhere, behind every range (64 rows of 2^22 numbers of
// 8 bytes at most).
constexpr unsigned kNowhere = 0x80000000u;
constexpr int kNonTemporal = 2;
using Buffer = __amdgpu_buffer_rsrc_t;

__device__ inline Buffer rows_of(const void* base, int64_t first, int64_t rows, int64_t ld, int64_t width, int element) {
  const int64_t have = rows - first < kRows ? rows - first : kRows;
  const char* p = (const char*)base + (have > 0 ? first * ld * element : 0);
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, have > 0 ? (int)(((have - 1) * ld + width) * element) : 0, 0x00020000);
}

// Four neighbouring numbers of a row from column k, zero beyond its end.  vec: rows and widths are multiples of four.
__device__ inline f32x4 load4(Buffer B, unsigned row, int k, int K, bool vec) {
  if (vec) return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(B, k < K ? row + k * 4 : kNowhere, 0, 0));
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(B, k + i < K ? row + (k + i) * 4 : kNowhere, 0, 0));
  return v;
}

// The parts of a column of W, terms 32 s + 8 q + (0..7), as the right operand
__device__ inline Parts column_parts(const float* W, int64_t n, int64_t c, int k0, int K) {
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool in = k0 + j < K && c < n;
    const float e = W[in ? (int64_t)(k0 + j) * n + c : 0];
    v[j] = in ? e : 0.f;
  }
  return split8(v);
}

template <int KS>
struct RowParts {   // 64 rows of x in parts; a row is padded by 16 bytes so that eight rows fill all banks once
  static constexpr int kPitch = KS * 32 + 8;
  __bf16 v[3][kRows][kPitch];
};

// One column of 16 x NT results a lane; results of a row tile: rows 4 q + i, columns NT (lane % 16) + t of the wave's 16 NT.
template <int KS, int NT, int kAct, bool kVec>
__global__ void __launch_bounds__(kThreads, 2) k_gated_fwd(GatedArgs a, int col_tiles, int splits) {
  __shared__ RowParts<KS> X;
  constexpr int KP = KS * 32, kQuads = KP / 4, kPer = kRows * kQuads / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, c = ((int64_t)(blockIdx.x % col_tiles) * 4 + wave) * (16 * NT) + l16 * NT;
  const unsigned ldx = (unsigned)a.ld_x * 4, ldo = (unsigned)a.ld_out * 4;
  Parts wg[KS][NT], wu[KS][NT];
  float bg[NT], bu[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      wg[s][j] = column_parts((const float*)a.Wg, n, c + j, s * 32 + q * 8, K);
      wu[s][j] = column_parts((const float*)a.Wu, n, c + j, s * 32 + q * 8, K);
    }
    bg[j] = a.bg && c + j < n ? ((const float*)a.bg)[c + j] : 0.f;
    bu[j] = a.bu && c + j < n ? ((const float*)a.bu)[c + j] : 0.f;
  }
  const int64_t blocks = (a.rows + kRows - 1) / kRows;
  f32x4 next[kPer];
  auto fetch = [&](int64_t b) {
    const Buffer in = rows_of(a.x, b * kRows, a.rows, a.ld_x, K, 4);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = t + i * kThreads;
      next[i] = load4(in, e / kQuads * ldx, e % kQuads * 4, K, kVec);
    }
  };
  unsigned at[NT];      // a lane's columns
#pragma unroll
  for (int j = 0; j < NT; ++j) at[j] = c + j < n ? (unsigned)(c + j) * 4 + q * 4 * ldo : kNowhere;
  int64_t b = blockIdx.x / col_tiles;
  if (b < blocks) fetch(b);
  for (; b < blocks; b += splits) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = t + i * kThreads;
      unsigned lo[3], hi[3];
      split(next[i][0], next[i][1], lo);
      split(next[i][2], next[i][3], hi);
#pragma unroll
      for (int p = 0; p < 3; ++p) *(uint2*)&X.v[p][e / kQuads][e % kQuads * 4] = make_uint2(lo[p], hi[p]);
    }
    __syncthreads();
    if (b + splits < blocks) fetch(b + splits);
    const Buffer to = rows_of(a.out, b * kRows, a.rows, a.ld_out, n, 4);
    // the results of a row tile are finished while the products of the next one run
    f32x4 g[2][NT], u[2][NT];
    auto products = [&](int rt, f32x4* gt, f32x4* ut) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        gt[j] = f32x4{bg[j], bg[j], bg[j], bg[j]};
        ut[j] = f32x4{bu[j], bu[j], bu[j], bu[j]};
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Parts xa;
#pragma unroll
        for (int p = 0; p < 3; ++p) xa.p[p] = *(const bf16x8*)&X.v[p][rt * 16 + l16][s * 32 + q * 8];
#pragma unroll
        for (int m = 0; m < 6; ++m)
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            gt[j] = mfma(xa.p[kPairA[m]], wg[s][j].p[kPairB[m]], gt[j]);
            ut[j] = mfma(xa.p[kPairA[m]], wu[s][j].p[kPairB[m]], ut[j]);
          }
      }
    };
    auto finish = [&](int rt, const f32x4* gt, const f32x4* ut) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned row = (rt * 16 + i) * ldo;   // kNowhere + row stays below 2^32: 64 rows are less than 2^31 bytes
        float v[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) v[j] = act_only<kAct>(gt[j][i]) * ut[j][i];
        if constexpr (NT == 2 && kVec) {
          __builtin_amdgcn_raw_buffer_store_b64(u32x2{__builtin_bit_cast(unsigned, v[0]), __builtin_bit_cast(unsigned, v[1])}, to, at[0] + row, 0, kNonTemporal);
        } else {
#pragma unroll
          for (int j = 0; j < NT; ++j) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v[j]), to, at[j] + row, 0, kNonTemporal);
        }
      }
    };
#pragma unroll
    for (int rt = 0; rt < kRows / 16; ++rt) {
      products(rt, g[rt & 1], u[rt & 1]);
      if (rt > 0) finish(rt - 1, g[~rt & 1], u[~rt & 1]);
    }
    finish(kRows / 16 - 1, g[1], u[1]);
  }
}

// ---- the gradients, fp32, up to 128 columns of x --------------------------------------------------------------------------
//
// Two kernels, each of which forms g and u again (a third more products than storing dg and du would need, but those are twice the
// size of gout).  In both a tile of dg and du leaves the registers of the products that made it as an operand of the next ones: a lane holds rows
// (columns) 4 q + i of two tiles, which are taken for the terms 8 q + (0..7) of 32, and the other operand stands in the same order.

// gWg, gWu, gbg, gbu of 16 columns a wave, over the rows blocks of a split; partial sums [split][Wg, Wu: d_in x d_out; bg, bu: d_out]
template <int KS>
struct TurnedParts {   // 64 rows of x in parts, by columns of x; places of a row: 32 (row / 32) + 8 q + (0..7)
  static constexpr int kPitch = kRows + 8;
  __bf16 v[3][KS * 32][kPitch];
};

// the place of rows 4 j .. 4 j + 3 (j < 16) in TurnedParts
__device__ inline int turned_place(int j) { return j / 8 * 32 + j % 4 * 8 + (j % 8) / 4 * 4; }

// waves of a workgroup: eight where its rows in LDS leave room for one workgroup only
template <int KS>
constexpr int kGwWaves = KS > 2 ? 8 : 4;

template <int KS, int kAct, bool kVec>
__global__ void __launch_bounds__(kGwWaves<KS> * 64, 2) k_gated_gw16(GatedArgs a, int col_tiles, int splits, float* part) {
  __shared__ RowParts<KS> X;
  __shared__ TurnedParts<KS> XT;
  // blocks of 4 rows x 4 columns of x; threads without one of their own repeat the last (no lane-conditional code)
  constexpr int kQuads = KS * 8, kBlocks = kRows / 4 * kQuads, kThr = kGwWaves<KS> * 64, kPer = (kBlocks + kThr - 1) / kThr;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, c = ((int64_t)(blockIdx.x % col_tiles) * kGwWaves<KS> + wave) * 16 + l16;
  const unsigned ldx = (unsigned)a.ld_x * 4, ldo = (unsigned)a.ld_gout * 4;
  Parts wg[KS], wu[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    wg[s] = column_parts((const float*)a.Wg, n, c, s * 32 + q * 8, K);
    wu[s] = column_parts((const float*)a.Wu, n, c, s * 32 + q * 8, K);
  }
  const float bg = a.bg && c < n ? ((const float*)a.bg)[c] : 0.f, bu = a.bu && c < n ? ((const float*)a.bu)[c] : 0.f;
  const int64_t blocks = (a.rows + kRows - 1) / kRows;
  f32x4 next[kPer][4];   // 4 rows of 4 columns
  auto fetch = [&](int64_t b) {
    const Buffer in = rows_of(a.x, b * kRows, a.rows, a.ld_x, K, 4);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = t + i * kThr < kBlocks ? t + i * kThr : kBlocks - 1;
#pragma unroll
      for (int j = 0; j < 4; ++j) next[i][j] = load4(in, (e / kQuads * 4 + j) * ldx, e % kQuads * 4, K, kVec);
    }
  };
  const unsigned at = c < n ? (unsigned)c * 4 + q * 4 * ldo : kNowhere;
  f32x4 sg[KS * 2] = {}, su[KS * 2] = {};
  float sbg = 0.f, sbu = 0.f;
  int64_t b = blockIdx.x / col_tiles;
  if (b < blocks) fetch(b);
  for (; b < blocks; b += splits) {
    const Buffer go = rows_of(a.gout, b * kRows, a.rows, a.ld_gout, n, 4);
    float tg[8];   // of gout, 32 rows at a time
    auto fetch_gout = [&](int half) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        tg[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(go, at + (half * 32 + i / 4 * 16 + i % 4) * ldo, 0, kNonTemporal));
    };
    fetch_gout(0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = t + i * kThr < kBlocks ? t + i * kThr : kBlocks - 1, r4 = e / kQuads, k4 = e % kQuads * 4;
      unsigned row[4][2][3], col[2][4][3];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        split(next[i][j][0], next[i][j][1], row[j][0]);
        split(next[i][j][2], next[i][j][3], row[j][1]);
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) *(uint2*)&X.v[p][r4 * 4 + j][k4] = make_uint2(row[j][0][p], row[j][1][p]);
        // columns: halves of the words of two rows
#pragma unroll
        for (int w = 0; w < 2; ++w) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            col[j][w * 2][p] = __builtin_amdgcn_perm(row[2 * j + 1][w][p], row[2 * j][w][p], 0x05040100);
            col[j][w * 2 + 1][p] = __builtin_amdgcn_perm(row[2 * j + 1][w][p], row[2 * j][w][p], 0x07060302);
          }
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) *(uint2*)&XT.v[p][k4 + w][turned_place(r4)] = make_uint2(col[0][w][p], col[1][w][p]);
      }
    }
    __syncthreads();
    if (b + splits < blocks) fetch(b + splits);
#pragma unroll
    for (int half = 0; half < kRows / 32; ++half) {
      float dg[8], du[8];
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        f32x4 g = {bg, bg, bg, bg}, u = {bu, bu, bu, bu};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          Parts xa;
#pragma unroll
          for (int p = 0; p < 3; ++p) xa.p[p] = *(const bf16x8*)&X.v[p][half * 32 + rt * 16 + l16][s * 32 + q * 8];
#pragma unroll
          for (int m = 0; m < 6; ++m) {
            g = mfma(xa.p[kPairA[m]], wg[s].p[kPairB[m]], g);
            u = mfma(xa.p[kPairA[m]], wu[s].p[kPairB[m]], u);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float o = tg[rt * 4 + i];   // zero behind the last row
          float v, d;
          act_both<kAct>(g[i], v, d);
          dg[rt * 4 + i] = o * u[i] * d;
          du[rt * 4 + i] = o * v;
          sbg += dg[rt * 4 + i];
          sbu += du[rt * 4 + i];
        }
      }
      if (half + 1 < kRows / 32) fetch_gout(half + 1);
      const Parts pg = split8(dg), pu = split8(du);
#pragma unroll
      for (int d = 0; d < KS * 2; ++d) {
        Parts xt;
#pragma unroll
        for (int p = 0; p < 3; ++p) xt.p[p] = *(const bf16x8*)&XT.v[p][d * 16 + l16][half * 32 + q * 8];
#pragma unroll
        for (int m = 0; m < 6; ++m) {
          sg[d] = mfma(xt.p[kPairA[m]], pg.p[kPairB[m]], sg[d]);
          su[d] = mfma(xt.p[kPairA[m]], pu.p[kPairB[m]], su[d]);
        }
      }
    }
  }
  if (c >= n) return;
  float* to = part + (int64_t)(blockIdx.x / col_tiles) * 2 * (K + 1) * n + c;
#pragma unroll
  for (int d = 0; d < KS * 2; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = d * 16 + q * 4 + i;
      if (k < K) {
        to[(int64_t)k * n] = sg[d][i];
        to[(int64_t)(K + 1 + k) * n] = su[d][i];
      }
    }
  // the biases' sums of the four quarters of the rows
  sbg += __shfl_xor(sbg, 16);
  sbg += __shfl_xor(sbg, 32);
  sbu += __shfl_xor(sbu, 16);
  sbu += __shfl_xor(sbu, 32);
  if (q == 0) {
    to[(int64_t)K * n] = sbg;
    to[(int64_t)(2 * K + 1) * n] = sbu;
  }
}

// adds up the splits
template <class T>
__global__ void __launch_bounds__(kThreads) k_gated_sums(const T* __restrict__ part, int splits, int64_t K, int64_t n, T* __restrict__ gWg,
                                                     T* __restrict__ gWu, T* __restrict__ gbg, T* __restrict__ gbu) {
  const int64_t size = 2 * (K + 1) * n, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= size) return;
  T v = part[i];
  for (int s = 1; s < splits; ++s) v += part[s * size + i];
  const int64_t row = i / n, c = i % n;
  if (row < K) gWg[i] = v;
  else if (row == K) { if (gbg) gbg[c] = v; }
  else if (row <= 2 * K) gWu[i - (K + 1) * n] = v;
  else if (gbu) gbu[c] = v;
}

// The parts of Wg and Wu as the operands that gx needs, 16 bytes a lane, [32 columns of W][operand][part][lane]:
//   4 KS for g and u again: tile 0, 1 x (g, u) x s: lane: column 16 tile + l16, terms 32 s + 8 q + (0..7) of d_in
//   4 KS for gx: (g, u) x tile of 16 columns of x: lane: column of x 16 d + l16, terms 16 (j / 4) + 4 q + j % 4 of the 32 columns of W
template <int KS>
constexpr int kOperands = 8 * KS;

template <int KS>
__global__ void __launch_bounds__(kThreads) k_gated_operands(GatedArgs a, u32x4* to) {
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, steps = (n + 31) / 32, e = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 64;
  if (e >= steps * kOperands<KS>) return;
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4;
  const int64_t step = e / kOperands<KS>;
  const int op = (int)(e % kOperands<KS>);
  float v[8];
  const float* W = (const float*)(op / (2 * KS) % 2 ? a.Wu : a.Wg);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    int k;
    int64_t c;
    if (op < 4 * KS) {          // order: (g, u), tile, s
      k = op % KS * 32 + q * 8 + j;
      c = step * 32 + op / KS % 2 * 16 + l16;
    } else {                    // order: (g, u), d
      k = op % (2 * KS) * 16 + l16;
      c = step * 32 + j / 4 * 16 + q * 4 + j % 4;
    }
    const bool in = k < K && c < n;
    const float w = W[in ? (int64_t)k * n + c : 0];
    v[j] = in ? w : 0.f;
  }
  const Parts p = split8(v);
#pragma unroll
  for (int i = 0; i < 3; ++i) to[(e * 3 + i) * 64 + lane] = __builtin_bit_cast(u32x4, p.p[i]);
}

// gx of 32 rows a wave (16 from 65 columns of x on, for the registers): the operands of 32 columns of W at a time in LDS for the
// eight waves of a workgroup, all columns one after another
constexpr int kGxWaves = 8;
template <int KS>
constexpr int kGxTiles = KS > 2 ? 1 : 2;

template <int KS, int kAct, bool kVec>
__global__ void __launch_bounds__(kGxWaves * 64, 2) k_gated_gx(GatedArgs a, const u32x4* __restrict__ ops) {
  constexpr int R = kGxTiles<KS>, kOps = kOperands<KS> * 3, kThr = kGxWaves * 64, kPer = (kOps * 64 + kThr - 1) / kThr;
  __shared__ u32x4 W[kOps][64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, steps = (n + 31) / 32, first = (int64_t)blockIdx.x * (kGxWaves * R * 16) + wave * R * 16;
  const unsigned ldx = (unsigned)a.ld_x * 4, ldo = (unsigned)a.ld_gout * 4, ldg = (unsigned)a.ld_gx * 4;
  // x of rows 16 r + l16, terms 32 s + 8 q + (0..7)
  Parts xb[R][KS];
  {
    const Buffer in = rows_of(a.x, first, a.rows, a.ld_x, K, 4);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const f32x4 lo = load4(in, (r * 16 + l16) * ldx, s * 32 + q * 8, K, kVec), hi = load4(in, (r * 16 + l16) * ldx, s * 32 + q * 8 + 4, K, kVec);
        const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        xb[r][s] = split8(v);
      }
  }
  const Buffer go = rows_of(a.gout, first, a.rows, a.ld_gout, n, 4);
  u32x4 next[kPer];
  auto fetch = [&](int64_t step) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (kOps * 64 % kThr == 0 || t + i * kThr < kOps * 64) next[i] = ops[step * kOps * 64 + t + i * kThr];
  };
  f32x4 acc[R][KS * 2] = {};
  fetch(0);
  for (int64_t step = 0; step < steps; ++step) {
    f32x4 tg[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const int64_t c = step * 32 + tile * 16 + q * 4;
        const unsigned row = (r * 16 + l16) * ldo;
        tg[r][tile] = load4(go, row, (int)c, (int)n, kVec);
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (kOps * 64 % kThr == 0 || t + i * kThr < kOps * 64) (&W[0][0])[t + i * kThr] = next[i];
    __syncthreads();
    if (step + 1 < steps) fetch(step + 1);
    float dg[R][8], du[R][8];
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      f32x4 g[R], u[R], bg = {0, 0, 0, 0}, bu = {0, 0, 0, 0};
      if (a.bg) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t c = step * 32 + tile * 16 + q * 4 + i;
          bg[i] = ((const float*)a.bg)[c < n ? c : n - 1];
          bu[i] = ((const float*)a.bu)[c < n ? c : n - 1];
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        g[r] = bg;
        u[r] = bu;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        Parts wg, wu;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          wg.p[p] = __builtin_bit_cast(bf16x8, W[(tile * KS + s) * 3 + p][lane]);
          wu.p[p] = __builtin_bit_cast(bf16x8, W[((2 + tile) * KS + s) * 3 + p][lane]);
        }
#pragma unroll
        for (int m = 0; m < 6; ++m)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            g[r] = mfma(wg.p[kPairA[m]], xb[r][s].p[kPairB[m]], g[r]);
            u[r] = mfma(wu.p[kPairA[m]], xb[r][s].p[kPairB[m]], u[r]);
          }
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float o = tg[r][tile][i];     // zero outside
          float v, d;
          act_both<kAct>(g[r][i], v, d);
          dg[r][tile * 4 + i] = o * u[r][i] * d;
          du[r][tile * 4 + i] = o * v;
        }
    }
    Parts pg[R], pu[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      pg[r] = split8(dg[r]);
      pu[r] = split8(du[r]);
    }
#pragma unroll
    for (int d = 0; d < KS * 2; ++d) {
      Parts wg, wu;
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        wg.p[p] = __builtin_bit_cast(bf16x8, W[(4 * KS + d) * 3 + p][lane]);
        wu.p[p] = __builtin_bit_cast(bf16x8, W[(6 * KS + d) * 3 + p][lane]);
      }
#pragma unroll
      for (int m = 0; m < 6; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][d] = mfma(wg.p[kPairA[m]], pg[r].p[kPairB[m]], acc[r][d]);
#pragma unroll
      for (int m = 0; m < 6; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][d] = mfma(wu.p[kPairA[m]], pu[r].p[kPairB[m]], acc[r][d]);
    }
  }
  const Buffer to = rows_of(a.gx, first, a.rows, a.ld_gx, K, 4);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int d = 0; d < KS * 2; ++d) {
      const int k = d * 16 + q * 4;
      const unsigned row = (r * 16 + l16) * ldg;
      if constexpr (kVec) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[r][d]), to, k < K ? row + k * 4 : kNowhere, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = acc[r][d][i];   // (a bit cast of the element itself takes the first one)
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), to, k + i < K ? row + (k + i) * 4 : kNowhere, 0, 0);
        }
      }
    }
}

// compute units of the current device, asked for once
hipError_t compute_units(int& cus) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  cus = known[dev].load(std::memory_order_relaxed);
  if (cus) return hipSuccess;
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  cus = std::min(cus, 256);   // what the workspace is sized for
  if (e == hipSuccess) known[dev].store(cus, std::memory_order_relaxed);
  return e;
}

template <int KS, int NT, int kAct>
hipError_t launch_fwd(const GatedArgs& a, int cus, hipStream_t st) {
  const int64_t cols = (a.d_out + 64 * NT - 1) / (64 * NT), blocks = (a.rows + kRows - 1) / kRows;
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(blocks, 2 * cus / cols));
  const dim3 grid((unsigned)(cols * splits));
  const bool vec = a.ld_x % 4 == 0 && a.d_in % 4 == 0 && a.ld_out % 2 == 0 && a.d_out % 2 == 0;
  if (vec) k_gated_fwd<KS, NT, kAct, true><<<grid, kThreads, 0, st>>>(a, (int)cols, (int)splits);
  else k_gated_fwd<KS, NT, kAct, false><<<grid, kThreads, 0, st>>>(a, (int)cols, (int)splits);
  return hipGetLastError();
}

template <int kAct>
hipError_t launch_fwd_act(const GatedArgs& a, hipStream_t st) {
  int cus = 0;
  hipError_t e = compute_units(cus);
  if (e != hipSuccess) return e;
  // 32 columns a wave where that leaves every compute unit two workgroups, else 16
  const bool wide = (a.d_out + 127) / 128 * ((a.rows + kRows - 1) / kRows) >= 2 * cus;
  switch ((a.d_in + 31) / 32) {
    case 1: return wide ? launch_fwd<1, 2, kAct>(a, cus, st) : launch_fwd<1, 1, kAct>(a, cus, st);
    case 2: return wide ? launch_fwd<2, 2, kAct>(a, cus, st) : launch_fwd<2, 1, kAct>(a, cus, st);
    case 3: return launch_fwd<3, 1, kAct>(a, cus, st);
    default: return launch_fwd<4, 1, kAct>(a, cus, st);
  }
}

int gw_waves(int64_t K) { return K > 64 ? kGwWaves<4> : kGwWaves<1>; }

// How the rows are split for the weights' gradients: eight waves for each compute unit, but partial sums of at most 64 MiB.
int64_t gw_splits(int64_t rows, int64_t K, int64_t n, int cus) {
  const int64_t wide = 16 * gw_waves(K), cols = (n + wide - 1) / wide, blocks = (rows + kRows - 1) / kRows;
  const int64_t most = std::max<int64_t>(1, ((int64_t)64 << 20) / (2 * (K + 1) * n * 4));
  return std::max<int64_t>(1, std::min({blocks, 8 / gw_waves(K) * cus / cols, most}));
}

size_t operand_bytes(int64_t K, int64_t n) { return (size_t)((n + 31) / 32 * ((K + 31) / 32) * 8 * 3 * 64 * 16); }

template <int KS, int kAct>
hipError_t launch_bwd(const GatedArgs& a, int cus, char* ws, hipStream_t st) {
  const int64_t n = a.d_out, wide = 16 * gw_waves(a.d_in), cols = (n + wide - 1) / wide, splits = gw_splits(a.rows, a.d_in, n, cus);
  u32x4* ops = (u32x4*)ws;
  float* part = (float*)(ws + operand_bytes(a.d_in, n));
  k_gated_operands<KS><<<dim3((unsigned)(((n + 31) / 32 * kOperands<KS> + 3) / 4)), kThreads, 0, st>>>(a, ops);
  constexpr int kGxRows = kGxWaves * kGxTiles<KS> * 16, kGwThreads = kGwWaves<KS> * 64;
  const dim3 gw((unsigned)(cols * splits)), gx((unsigned)((a.rows + kGxRows - 1) / kGxRows));
  const bool vec_x = a.ld_x % 4 == 0 && a.d_in % 4 == 0, vec = vec_x && a.ld_gout % 4 == 0 && n % 4 == 0 && a.ld_gx % 4 == 0;
  if (vec) k_gated_gx<KS, kAct, true><<<gx, kGxWaves * 64, 0, st>>>(a, ops);
  else k_gated_gx<KS, kAct, false><<<gx, kGxWaves * 64, 0, st>>>(a, ops);
  if (vec_x) k_gated_gw16<KS, kAct, true><<<gw, kGwThreads, 0, st>>>(a, (int)cols, (int)splits, part);
  else k_gated_gw16<KS, kAct, false><<<gw, kGwThreads, 0, st>>>(a, (int)cols, (int)splits, part);
  k_gated_sums<float><<<dim3((unsigned)((2 * (a.d_in + 1) * n + kThreads - 1) / kThreads)), kThreads, 0, st>>>(
      part, (int)splits, a.d_in, n, (float*)a.gWg, (float*)a.gWu, (float*)a.gbg, (float*)a.gbu);
  return hipGetLastError();
}

template <int kAct>
hipError_t launch_bwd_act(const GatedArgs& a, char* ws, hipStream_t st) {
  int cus = 0;
  hipError_t e = compute_units(cus);
  if (e != hipSuccess) return e;
  switch ((a.d_in + 31) / 32) {
    case 1: return launch_bwd<1, kAct>(a, cus, ws, st);
    case 2: return launch_bwd<2, kAct>(a, cus, ws, st);
    case 3: return launch_bwd<3, kAct>(a, cus, ws, st);
    default: return launch_bwd<4, kAct>(a, cus, ws, st);
  }
}

hipError_t backward_parts(const GatedArgs& a, char* ws, hipStream_t st) {
  switch (a.act) {
    case CGTP_ACT_NONE: return launch_bwd_act<CGTP_ACT_NONE>(a, ws, st);
    case CGTP_ACT_SILU: return launch_bwd_act<CGTP_ACT_SILU>(a, ws, st);
    case CGTP_ACT_GELU: return launch_bwd_act<CGTP_ACT_GELU>(a, ws, st);
    case CGTP_ACT_SIGMOID: return launch_bwd_act<CGTP_ACT_SIGMOID>(a, ws, st);
    default: return launch_bwd_act<CGTP_ACT_TANH>(a, ws, st);
  }
}

hipError_t forward_parts(const GatedArgs& a, hipStream_t st) {
  switch (a.act) {
    case CGTP_ACT_NONE: return launch_fwd_act<CGTP_ACT_NONE>(a, st);
    case CGTP_ACT_SILU: return launch_fwd_act<CGTP_ACT_SILU>(a, st);
    case CGTP_ACT_GELU: return launch_fwd_act<CGTP_ACT_GELU>(a, st);
    case CGTP_ACT_SIGMOID: return launch_fwd_act<CGTP_ACT_SIGMOID>(a, st);
    default: return launch_fwd_act<CGTP_ACT_TANH>(a, st);
  }
}

constexpr int64_t kPiece = 8192;   // rows whose dg and du stand in the workspace at a time

int64_t tiles(int64_t n) { return (n + kTile - 1) / kTile; }

template <class T, bool kBack>
hipError_t launch_tile(const GatedArgs& a, int64_t row0, int64_t rows, T* dg, T* du, hipStream_t st) {
  const dim3 grid((unsigned)(tiles(rows) * tiles(a.d_out)));
  switch (a.act) {
    case CGTP_ACT_NONE: k_gated_tile<T, CGTP_ACT_NONE, kBack><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, du); break;
    case CGTP_ACT_SILU: k_gated_tile<T, CGTP_ACT_SILU, kBack><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, du); break;
    case CGTP_ACT_GELU: k_gated_tile<T, CGTP_ACT_GELU, kBack><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, du); break;
    case CGTP_ACT_SIGMOID: k_gated_tile<T, CGTP_ACT_SIGMOID, kBack><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, du); break;
    default: k_gated_tile<T, CGTP_ACT_TANH, kBack><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, du); break;
  }
  return hipGetLastError();
}

template <class T>
hipError_t backward(const GatedArgs& a, void* ws, hipStream_t st) {
  T* dg = (T*)ws;
  T* du = dg + std::min(a.rows, kPiece) * a.d_out;
  const int64_t pieces = std::max<int64_t>(1, (a.rows + kPiece - 1) / kPiece);
  for (int64_t p = 0; p < pieces; ++p) {
    const int64_t row0 = p * kPiece, rows = std::min(kPiece, a.rows - row0);
    if (rows > 0) {
      hipError_t e = launch_tile<T, true>(a, row0, rows, dg, du, st);
      if (e != hipSuccess) return e;
      k_gated_gx<T><<<dim3((unsigned)(tiles(rows) * tiles(a.d_in))), kThreads, 0, st>>>(a, row0, rows, dg, du);
    }
    const dim3 grid((unsigned)(tiles(a.d_in) * tiles(a.d_out)));
    k_gated_gw<T><<<grid, kThreads, 0, st>>>(a, row0, rows, dg, (T*)a.gWg, (T*)a.gbg, p == 0);
    k_gated_gw<T><<<grid, kThreads, 0, st>>>(a, row0, rows, du, (T*)a.gWu, (T*)a.gbu, p == 0);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t gated_forward(const GatedArgs& a, hipStream_t st) {
  if (!a.f64 && a.d_in <= kMaxIn) return forward_parts(a, st);
  const int64_t most = (int64_t)65536 * kTile / std::max<int64_t>(1, tiles(a.d_out)) / kTile * kTile;   // rows of a launch
  for (int64_t row0 = 0; row0 < a.rows; row0 += std::max<int64_t>(kTile, most)) {
    const int64_t rows = std::min(a.rows - row0, std::max<int64_t>(kTile, most));
    hipError_t e = a.f64 ? launch_tile<double, false>(a, row0, rows, nullptr, nullptr, st) : launch_tile<float, false>(a, row0, rows, nullptr, nullptr, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t gated_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_out, bool f64) {
  size_t bytes = (size_t)(2 * std::min(rows, kPiece) * d_out * (f64 ? 8 : 4));
  if (!f64 && d_in <= kMaxIn)   // the splits of the largest device, so that the size does not depend on the current one
    bytes = operand_bytes(d_in, d_out) + (size_t)(gw_splits(rows, d_in, d_out, 256) * 2 * (d_in + 1) * d_out * 4);
  return (bytes + 255) / 256 * 256;
}

hipError_t gated_backward(const GatedArgs& a, void* ws, hipStream_t st) {
  if (!a.f64 && a.d_in <= kMaxIn) return backward_parts(a, (char*)ws, st);
  return a.f64 ? backward<double>(a, ws, st) : backward<float>(a, ws, st);
}

}  // namespace cgtp
