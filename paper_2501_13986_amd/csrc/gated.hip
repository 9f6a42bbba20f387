// Gated feed-forward block: out = act(x Wg + bg) * (x Wu + bu), and its gradients.
//
// With g = x Wg + bg, u = x Wu + bu and t = dE/dout:   dg = t u act'(g),  du = t act(g),
//     gx = dg Wg^T + du Wu^T,   gWg = x^T dg,   gWu = x^T du,   gbg = sum dg,   gbu = sum du.
#include <hip/hip_runtime.h>

#include <algorithm>

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
  const int64_t most = (int64_t)65536 * kTile / std::max<int64_t>(1, tiles(a.d_out)) / kTile * kTile;   // rows of a launch
  for (int64_t row0 = 0; row0 < a.rows; row0 += std::max<int64_t>(kTile, most)) {
    const int64_t rows = std::min(a.rows - row0, std::max<int64_t>(kTile, most));
    hipError_t e = a.f64 ? launch_tile<double, false>(a, row0, rows, nullptr, nullptr, st) : launch_tile<float, false>(a, row0, rows, nullptr, nullptr, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

size_t gated_workspace_bytes(int64_t rows, int64_t, int64_t d_out, bool f64) {
  return (size_t)(2 * std::min(rows, kPiece) * d_out * (f64 ? 8 : 4) + 255) / 256 * 256;
}

hipError_t gated_backward(const GatedArgs& a, void* ws, hipStream_t st) { return a.f64 ? backward<double>(a, ws, st) : backward<float>(a, ws, st); }

}  // namespace cgtp
