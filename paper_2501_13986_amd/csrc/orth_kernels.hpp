// Kernels of orthogonalise, for the translation units of its two types (orth_f32.hip, orth_f64.hip).
//
// X = G / (|G| + eps), transposed if G has more rows than columns, so that X is s x l with s <= l; a step is
//     A = X X^T,  B = b A + c A A,  X <- a X + B X.
// A and B are symmetric: tiles on and above the diagonal are formed and written twice.
#pragma once

#include <algorithm>

#include "orth.hpp"
#include "product.hpp"

namespace cgtp {
namespace {

constexpr int kShares = 64;      // partial sums of squares of a matrix, at most

// ---- the start ------------------------------------------------------------------------------------------------------------------

// part [batch][shares]: sums of squares of shares of the rows
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_squares(OrthArgs a, int64_t first, int shares, double* part) {
  __shared__ double sums[kProductThreads / 64];
  const int64_t matrix = first + blockIdx.x / shares, share = blockIdx.x % shares;
  const T* g = (const T*)a.g + matrix * a.stride_g;
  const int64_t from = a.m * share / shares, size = (a.m * (share + 1) / shares - from) * a.n;
  double v = 0;
  for (int64_t i = threadIdx.x; i < size; i += kProductThreads) {
    const double w = (double)g[(from + i / a.n) * a.ld_g + i % a.n];
    v += w * w;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = v;
  __syncthreads();
  if (threadIdx.x == 0) part[matrix * shares + share] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

__device__ inline double scale_of(const double* part, int shares, double eps) {
  double v = 0;
  for (int i = 0; i < shares; ++i) v += part[i];
  return 1.0 / (sqrt(v) + eps);
}

// X, 64 x 64 numbers of G a workgroup; rounded once
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_start(OrthArgs a, int64_t first, int64_t tiles, int shares, const double* part, T* X) {
  __shared__ T tile[64][65];
  const int64_t matrix = first + blockIdx.x / tiles, across = (a.n + 63) / 64, r0 = blockIdx.x % tiles / across * 64, c0 = blockIdx.x % tiles % across * 64;
  const double scale = scale_of(part + matrix * shares, shares, a.eps);
  const T* g = (const T*)a.g + matrix * a.stride_g;
  T* to = X + matrix * a.m * a.n;
  const int x = threadIdx.x % 64;
  if (a.m <= a.n) {
    for (int y = threadIdx.x / 64; y < 64; y += 4)
      if (r0 + y < a.m && c0 + x < a.n) to[(r0 + y) * a.n + c0 + x] = (T)((double)g[(r0 + y) * a.ld_g + c0 + x] * scale);
    return;
  }
  for (int y = threadIdx.x / 64; y < 64; y += 4)
    if (r0 + y < a.m && c0 + x < a.n) tile[y][x] = (T)((double)g[(r0 + y) * a.ld_g + c0 + x] * scale);
  __syncthreads();
  for (int y = threadIdx.x / 64; y < 64; y += 4)
    if (c0 + y < a.n && r0 + x < a.m) to[(c0 + y) * a.m + r0 + x] = tile[x][y];
}

// ---- the products of a step -----------------------------------------------------------------------------------------------------

// tile number -> row and column of tiles, on and above the diagonal
__device__ inline void upper_tile(int t, int& r, int& c) {
  c = (int)((__builtin_sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while (c * (c + 1) / 2 > t) --c;
  while ((c + 1) * (c + 2) / 2 <= t) ++c;
  r = t - c * (c + 1) / 2;
}

// to = alpha Y Y^T (+ beta Y where Y is s x s: it is symmetric itself), Y [s, terms]
template <class T, int kR, bool kWhole>
__global__ void __launch_bounds__(kProductThreads, 2) k_orth_square(int64_t first, int tiles, int s, int terms, const T* Y, T alpha, T beta, T* to) {
  __shared__ Operand<T, kR> R, C;
  const int64_t matrix = first + blockIdx.x / tiles;
  int tr, tc;
  upper_tile(blockIdx.x % tiles, tr, tc);
  const int r0 = tr * kR, c0 = tc * kR;
  Y += matrix * s * terms;
  to += matrix * s * s;
  using Along = AlongTerms<T, kR, kWhole>;
  Along rows, columns;
  const T *pr[Along::kPer], *pc[Along::kPer];
#pragma unroll
  for (int i = 0; i < Along::kPer; ++i) {
    const int r = r0 + Along::row(i), c = c0 + Along::row(i);
    pr[i] = Y + (int64_t)(r < s ? r : 0) * terms;
    pc[i] = Y + (int64_t)(c < s ? c : 0) * terms;
  }
  Results<T, kR, kR> out;
  rows.fetch(pr, 0, terms);
  columns.fetch(pc, 0, terms);
  for (int k0 = 0; k0 < terms; k0 += kStep) {
    __syncthreads();
    rows.put(R);
    columns.put(C);
    __syncthreads();
    if (k0 + kStep < terms) {
      rows.fetch(pr, k0 + kStep, terms);
      columns.fetch(pc, k0 + kStep, terms);
    }
    out.multiply(R, C);
  }
#pragma unroll
  for (int rt = 0; rt < out.RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < out.CT; ++ct) {
      const int r = r0 + out.row(rt), c = c0 + out.column(ct);
      if (r >= s || c >= s) continue;
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = alpha * out.acc[rt][ct][i];
        if (beta != T(0)) v[i] += beta * Y[(int64_t)r * s + (c + i < s ? c + i : c)];
      }
      store_some(to + (int64_t)r * s + c, v, s - c);
      if (tr != tc)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < s) to[(int64_t)(c + i) * s + r] = v[i];
    }
}

// to = alpha X + B X, X [s, l]; kLast: to is the caller's output, transposed where X is
template <class T, int kR, int kC, bool kWhole, bool kLast>
__global__ void __launch_bounds__(kProductThreads, 2) k_orth_apply(int64_t first, int tiles, int s, int l, const T* X, const T* B, T alpha, T* to, int64_t ld, int64_t stride, bool turned) {
  __shared__ Operand<T, kR> R;
  __shared__ Operand<T, kC> C;
  const int64_t matrix = first + blockIdx.x / tiles;
  const int across = (l + kC - 1) / kC, r0 = blockIdx.x % tiles / across * kR, c0 = blockIdx.x % tiles % across * kC;
  X += matrix * s * l;
  B += matrix * s * s;
  to += matrix * stride;
  using Along = AlongTerms<T, kR, kWhole>;
  Along rows;
  AcrossTerms<T, kC, kWhole> columns;
  const T* pr[Along::kPer];
#pragma unroll
  for (int i = 0; i < Along::kPer; ++i) {
    const int r = r0 + Along::row(i);
    pr[i] = B + (int64_t)(r < s ? r : 0) * s;
  }
  auto fetch = [&](int k0) {
    rows.fetch(pr, k0, s);
    const T* p[4];
    bool ok[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = k0 + columns.term() + j;
      ok[j] = k < s;
      p[j] = X + (int64_t)(ok[j] ? k : 0) * l;
    }
    columns.fetch(p, ok, c0, l);
  };
  Results<T, kR, kC> out;
  fetch(0);
  for (int k0 = 0; k0 < s; k0 += kStep) {
    __syncthreads();
    rows.put(R);
    columns.put(C);
    __syncthreads();
    if (k0 + kStep < s) fetch(k0 + kStep);
    out.multiply(R, C);
  }
#pragma unroll
  for (int rt = 0; rt < out.RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < out.CT; ++ct) {
      const int r = r0 + out.row(rt), c = c0 + out.column(ct);
      if (r >= s || c >= l) continue;
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = out.acc[rt][ct][i] + alpha * X[(int64_t)r * l + (c + i < l ? c + i : c)];
      if (kLast && turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < l) to[(c + i) * ld + r] = v[i];
      } else {
        store_some(to + r * ld + c, v, l - c);
      }
    }
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostBlocks = (int64_t)1 << 23;   // workgroups of a launch: 2^32 threads are too many

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// f(first matrix, grid) for `tiles` workgroups a matrix, as many matrices a launch as there may be
template <class F>
hipError_t in_launches(int64_t batch, int64_t tiles, F f) {
  const int64_t most = std::max<int64_t>(1, kMostBlocks / tiles);
  for (int64_t at = 0; at < batch; at += most) {
    f(at, dim3((unsigned)(std::min(most, batch - at) * tiles)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

int shares_of(int64_t m, int64_t n) { return (int)std::min<int64_t>({kShares, m, std::max<int64_t>(1, m * n / 4096)}); }

template <class T>
size_t workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  const int64_t s = std::min(m, n);
  return up(batch * shares_of(m, n) * sizeof(double)) + 2 * up(batch * m * n * sizeof(T)) + 2 * up(batch * s * s * sizeof(T));
}

template <class T, bool kWhole>
hipError_t steps_of(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  const int64_t s = std::min(a.m, a.n), l = std::max(a.m, a.n);
  const int shares = shares_of(a.m, a.n);
  double* part = (double*)ws;
  T* X = (T*)(ws + up(a.batch * shares * sizeof(double)));
  T* other = (T*)((char*)X + up(a.batch * a.m * a.n * sizeof(T)));
  T* A = (T*)((char*)other + up(a.batch * a.m * a.n * sizeof(T)));
  T* B = (T*)((char*)A + up(a.batch * s * s * sizeof(T)));
  hipError_t e = in_launches(a.batch, shares, [&](int64_t first, dim3 grid) { k_orth_squares<T><<<grid, kProductThreads, 0, st>>>(a, first, shares, part); });
  if (e != hipSuccess) return e;
  const int64_t squares = ((a.m + 63) / 64) * ((a.n + 63) / 64);
  e = in_launches(a.batch, squares, [&](int64_t first, dim3 grid) { k_orth_start<T><<<grid, kProductThreads, 0, st>>>(a, first, squares, shares, part, X); });
  constexpr int kR = 64, kC = 64;
  const int64_t side = (s + kR - 1) / kR, upper = side * (side + 1) / 2, all = side * ((l + kC - 1) / kC);
  for (int i = 0; i < steps && e == hipSuccess; ++i) {
    const double* c = coefficients + 3 * i;
    e = in_launches(a.batch, upper, [&](int64_t first, dim3 grid) {
      k_orth_square<T, kR, kWhole><<<grid, kProductThreads, 0, st>>>(first, (int)upper, (int)s, (int)l, X, T(1), T(0), A);
    });
    if (e != hipSuccess) break;
    e = in_launches(a.batch, upper, [&](int64_t first, dim3 grid) {
      k_orth_square<T, kR, kWhole><<<grid, kProductThreads, 0, st>>>(first, (int)upper, (int)s, (int)s, A, (T)c[2], (T)c[1], B);
    });
    if (e != hipSuccess) break;
    e = in_launches(a.batch, all, [&](int64_t first, dim3 grid) {
      if (i + 1 < steps)
        k_orth_apply<T, kR, kC, kWhole, false><<<grid, kProductThreads, 0, st>>>(first, (int)all, (int)s, (int)l, X, B, (T)c[0], other, l, s * l, false);
      else
        k_orth_apply<T, kR, kC, kWhole, true><<<grid, kProductThreads, 0, st>>>(first, (int)all, (int)s, (int)l, X, B, (T)c[0], (T*)a.out, a.ld_out, a.stride_out, a.m > a.n);
    });
    std::swap(X, other);
  }
  return e;
}

template <class T>
hipError_t orthogonalise(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  return a.m % 4 == 0 && a.n % 4 == 0 ? steps_of<T, true>(a, coefficients, steps, ws, st) : steps_of<T, false>(a, coefficients, steps, ws, st);
}

}  // namespace
}  // namespace cgtp
