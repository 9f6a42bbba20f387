// Kernels of orthogonalise, for the translation units of its two types (orth_f32.hip, orth_f64.hip).
//
// X = G / (|G| + eps), transposed if G has more rows than columns, so that X is s x l with s <= l; a step is
//     A = X X^T,  B = b A + c A A,  X <- a X + B X.
// A and B are symmetric: tiles on and above the diagonal are formed and written twice.
#pragma once

#include <algorithm>
#include <type_traits>

#include "orth.hpp"
#include "product.hpp"

namespace cgtp {
namespace {

constexpr int kShares = 256;      // partial sums of squares of a matrix, at most

// ---- the start ------------------------------------------------------------------------------------------------------------------

// part [batch][shares]: sums of squares of shares of the rows
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_squares(OrthArgs a, int64_t first, int shares, double* part) {
  __shared__ double sums[kProductThreads / 64];
  const int64_t matrix = first + blockIdx.x / shares, share = blockIdx.x % shares;
  const T* g = (const T*)a.g + matrix * a.stride_g;
  const int64_t from = a.m * share / shares, end = a.m * (share + 1) / shares;
  // as many lanes side by side as a row has numbers, eight numbers on their way to a thread
  const int wide = a.n >= kProductThreads ? kProductThreads : a.n > 64 ? 128 : a.n > 16 ? 64 : 16, x = threadIdx.x % wide, y = threadIdx.x / wide, high = kProductThreads / wide;
  double v = 0;
  for (int64_t r = from + y; r < end; r += high) {
    const T* p = g + r * a.ld_g;
    int64_t c = x;
    for (; c + 7 * wide < a.n; c += 8 * wide) {
      double w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = (double)p[c + i * wide];
#pragma unroll
      for (int i = 0; i < 8; ++i) v += w[i] * w[i];
    }
    for (; c < a.n; c += wide) v += (double)p[c] * (double)p[c];
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

// ---- up to 128 rows of X --------------------------------------------------------------------------------------------------------
//
// A workgroup has 64 NT columns of X in its registers, a wave 16 NT of them with all their rows: lane: columns NT l16 + j, rows 16 t + 4 q + (0..3).
// A step is X <- a X + A V, V = b X + c A X, so that both products have A (in LDS) on the left and on the right what the wave has: results of the matrix
// instructions are operands of the next ones as they are, with the terms of 32 rows in the order `place`.  Only for A = X X^T does X go through LDS.
// Where the workgroup has all columns, the steps run without leaving it.  Where not, a launch is a step: the workgroups leave their shares of A, which all of the next
// launch add up, and X in the order of their registers.

constexpr int kMostRows = 128;

// the place of row r among 32 terms of results
__device__ inline int place(int r) { return r % 16 / 4 * 8 + r / 16 * 4 + r % 4; }

template <class T, int kS, int NT>
struct Columns {
  using N = Num<T>;
  static constexpr int kTiles = kS / 16, kWide = 64 * NT, kSlices = (kS > kWide ? kS : kWide) / 32;
  using Lds = Operand<T, kS>[kSlices];
  using Gram = Results<T, kS, kS>;
  typename N::Vec x[kTiles][NT];

  static __device__ int lane() { return (int)threadIdx.x & 63; }
  static __device__ int column(int j) { return (int)(threadIdx.x / 64) * (16 * NT) + lane() % 16 * NT + j; }
  static __device__ int row(int t) { return t * 16 + lane() / 16 * 4; }      // the first of four

  // columns c0 .. of the matrix at g (transposed: it has them as rows), as they are; zero outside
  __device__ void load(const T* g, int64_t ld, int s, int l, int c0, bool turned) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int c = c0 + column(j), cc = c < l ? c : 0;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = row(t) + i, rr = r < s ? r : 0;
          const T v = turned ? g[cc * ld + rr] : g[rr * ld + cc];
          x[t][j][i] = c < l && r < s ? v : T(0);
        }
    }
  }
  __device__ void store(T* to, int64_t ld, int s, int l, int c0, bool turned) const {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int c = c0 + column(j);
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = row(t) + i;
          if (c < l && r < s) to[turned ? c * ld + r : r * ld + c] = x[t][j][i];
        }
    }
  }
  // in the order of the registers: kS x kWide numbers a workgroup
  __device__ void keep(T* to) const {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j) *(typename N::Vec*)(to + ((t * NT + j) * kProductThreads + (int)threadIdx.x) * 4) = x[t][j];
  }
  __device__ void take(const T* from) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j) x[t][j] = *(const typename N::Vec*)(from + ((t * NT + j) * kProductThreads + (int)threadIdx.x) * 4);
  }
  // the thread's share of the sum of squares
  __device__ double squares() const {
    double v = 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) v += (double)x[t][j][i] * (double)x[t][j][i];
    return v;
  }
  __device__ void scale(double by) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][j][i] = (T)((double)x[t][j][i] * by);
  }
  // (the share of) A, through LDS
  __device__ void gram(Lds& S, Gram& A) const {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        T v[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) v[j] = x[t][j][i];
        S[column(0) / 32].write_some(row(t) + i, column(0) % 32, v);
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWide / 32; ++k) {
      A.multiply(S[k], S[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
  }
  // A as the left operand of the step's products
  static __device__ void put(Lds& S, const Gram& A) {
#pragma unroll
    for (int rt = 0; rt < Gram::RT; ++rt)
#pragma unroll
      for (int ct = 0; ct < Gram::CT; ++ct) {
        const int c = A.column(ct);
        const T v[4] = {A.acc[rt][ct][0], A.acc[rt][ct][1], A.acc[rt][ct][2], A.acc[rt][ct][3]};
        S[c / 32].write4(A.row(rt), place(c % 32), v);
      }
    __syncthreads();
  }
  // y += A v
  __device__ static void times(const Lds& S, const typename N::Vec (&v)[kTiles][NT], typename N::Vec (&y)[kTiles][NT]) {
    const int l16 = lane() % 16, q = lane() / 16;
    constexpr int kPairs = kTiles / 2;
    typename N::Parts a[2][2], r[NT];
    auto fetch = [&](int i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) a[i % 2][h] = S[i / kPairs].read((i % kPairs * 2 + h) * 16 + column_place<T>(l16), q * 8);
    };
    fetch(0);
#pragma unroll
    for (int i = 0; i < kS / 32 * kPairs; ++i) {
      const int k = i / kPairs, t = i % kPairs * 2;
      if (t == 0)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          T w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = v[2 * k + e / 4][j][e % 4];
          r[j] = N::parts(w);
        }
      if (i + 1 < kS / 32 * kPairs) fetch(i + 1);
      const typename N::Parts &a0 = a[i % 2][0], &a1 = a[i % 2][1];
      if constexpr (NT == 2) N::template mma<4>({&a0, &a0, &a1, &a1}, {&r[0], &r[1], &r[0], &r[1]}, {&y[t][0], &y[t][1], &y[t + 1][0], &y[t + 1][1]});
      else N::template mma<2>({&a0, &a1}, {&r[0], &r[0]}, {&y[t][0], &y[t + 1][0]});
      __builtin_amdgcn_sched_barrier(0);      // else all of A is on its way to registers at once
    }
  }
  // X <- a X + A (b X + c A X), A in LDS
  __device__ void step(const Lds& S, T a, T b, T c) {
    typename N::Vec y[kTiles][NT] = {};
    times(S, x, y);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[t][j][i] = b * x[t][j][i] + c * y[t][j][i];
          x[t][j][i] *= a;
        }
    times(S, y, x);
  }
};

// sum over the workgroup, to all its threads
__device__ inline double sum_of_all(double v, double* sums) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  sums[threadIdx.x / 64] = v;      // all lanes the same
  __syncthreads();
  return (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

struct Schedule {
  double c[64][3];
};

// all steps of a matrix of at most 64 NT columns
template <class T, int kS, int NT>
__global__ void __launch_bounds__(kProductThreads, 1) k_orth_whole(OrthArgs a, int64_t first, int steps, Schedule schedule) {
  using Cols = Columns<T, kS, NT>;
  __shared__ typename Cols::Lds S;
  __shared__ double sums[kProductThreads / 64];
  const int64_t matrix = first + blockIdx.x;
  const bool turned = a.m > a.n;
  const int s = (int)(turned ? a.n : a.m), l = (int)(turned ? a.m : a.n);
  Cols X;
  X.load((const T*)a.g + matrix * a.stride_g, a.ld_g, s, l, 0, turned);
  X.scale(1.0 / (sqrt(sum_of_all(X.squares(), sums)) + a.eps));
  for (int i = 0; i < steps; ++i) {
    typename Cols::Gram A;
    X.gram(S, A);
    Cols::put(S, A);
    X.step(S, (T)schedule.c[i][0], (T)schedule.c[i][1], (T)schedule.c[i][2]);
  }
  X.store((T*)a.out + matrix * a.stride_out, a.ld_out, s, l, 0, turned);
}

// The first share of A [matrix][chunk][kS * kS] and X [matrix][chunk][kS * 64 NT], in the order of the registers
template <class T, int kS, int NT>
__global__ void __launch_bounds__(kProductThreads, 1) k_orth_begin(OrthArgs a, int64_t first, int chunks, int shares, const double* part, T* X_to, T* A_to) {
  using Cols = Columns<T, kS, NT>;
  __shared__ typename Cols::Lds S;
  const int64_t matrix = first + blockIdx.x / chunks, place = matrix * chunks + blockIdx.x % chunks;
  const bool turned = a.m > a.n;
  const int s = (int)(turned ? a.n : a.m), l = (int)(turned ? a.m : a.n);
  Cols X;
  X.load((const T*)a.g + matrix * a.stride_g, a.ld_g, s, l, blockIdx.x % chunks * Cols::kWide, turned);
  X.scale(scale_of(part + matrix * shares, shares, a.eps));
  X.keep(X_to + place * (kS * Cols::kWide));
  typename Cols::Gram A;
  X.gram(S, A);
  A.keep(A_to + place * (kS * kS));
}

// A step.  parts: how many shares of A there are a matrix
template <class T, int kS, int NT, bool kLast>
__global__ void __launch_bounds__(kProductThreads, 1) k_orth_step(OrthArgs a, int64_t first, int chunks, int parts, T c0, T c1, T c2, T* X_at, const T* A_from, T* A_to) {
  using Cols = Columns<T, kS, NT>;
  __shared__ typename Cols::Lds S;
  const int64_t matrix = first + blockIdx.x / chunks, place = matrix * chunks + blockIdx.x % chunks;
  Cols X;
  X.take(X_at + place * (kS * Cols::kWide));
  typename Cols::Gram A;
  A.add_up(A_from + matrix * parts * (kS * kS), parts);
  Cols::put(S, A);
  X.step(S, c0, c1, c2);
  if constexpr (kLast) {
    const bool turned = a.m > a.n;
    const int s = (int)(turned ? a.n : a.m), l = (int)(turned ? a.m : a.n);
    X.store((T*)a.out + matrix * a.stride_out, a.ld_out, s, l, blockIdx.x % chunks * Cols::kWide, turned);
  } else {
    X.keep(X_at + place * (kS * Cols::kWide));
    typename Cols::Gram next;
    X.gram(S, next);
    next.keep(A_to + place * (kS * kS));
  }
}

// to [matrix][size] = sums of from [matrix][parts][size], in their order
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_join(int64_t first, int blocks, int parts, int size, const T* from, T* to) {
  const int64_t matrix = first + blockIdx.x / blocks;
  const int i = blockIdx.x % blocks * kProductThreads + threadIdx.x;
  if (i >= size) return;
  from += matrix * parts * size + i;
  T v[8] = {};
  int p = 0;
  for (; p + 8 <= parts; p += 8)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += from[(int64_t)(p + j) * size];
  for (; p < parts; ++p) v[0] += from[(int64_t)p * size];
  to[matrix * size + i] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
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

// What the columns of X are cut into where it has few rows.  Shares of A are added up by every workgroup of a matrix up to kMostShares of them, by a launch of its own beyond.
constexpr int64_t kMostShares = 32;

struct Few {
  int64_t rows, wide, chunks;      // padded rows, columns of a chunk, chunks
  Few(int64_t m, int64_t n, bool f64) {
    const int64_t s = std::min(m, n), l = std::max(m, n);
    rows = (s + 31) / 32 * 32;
    wide = f64 || l <= 64 ? 64 : 128;
    chunks = (l + wide - 1) / wide;
  }
  size_t x_size() const { return rows * wide * chunks; }      // numbers a matrix
  size_t a_size() const { return rows * rows * chunks; }
  size_t sum_size() const { return chunks > kMostShares ? rows * rows : 0; }
};

template <class T>
size_t workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  const int64_t s = std::min(m, n);
  if (s <= kMostRows) {
    const Few f(m, n, sizeof(T) == 8);
    if (f.chunks == 1) return 0;
    return up(batch * shares_of(m, n) * sizeof(double)) + up(batch * f.x_size() * sizeof(T)) + 2 * up(batch * f.a_size() * sizeof(T)) + up(batch * f.sum_size() * sizeof(T));
  }
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

template <class T, int kS, int NT>
hipError_t few_rows(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  const Few f(a.m, a.n, sizeof(T) == 8);
  if (f.chunks == 1) {
    Schedule schedule = {};
    for (int i = 0; i < 3 * steps; ++i) schedule.c[i / 3][i % 3] = coefficients[i];
    return in_launches(a.batch, 1, [&](int64_t first, dim3 grid) { k_orth_whole<T, kS, NT><<<grid, kProductThreads, 0, st>>>(a, first, steps, schedule); });
  }
  const int shares = shares_of(a.m, a.n), chunks = (int)f.chunks;
  double* part = (double*)ws;
  T* X = (T*)(ws + up(a.batch * shares * sizeof(double)));
  T* A = (T*)((char*)X + up(a.batch * f.x_size() * sizeof(T)));
  T* next = (T*)((char*)A + up(a.batch * f.a_size() * sizeof(T)));
  T* sum = (T*)((char*)next + up(a.batch * f.a_size() * sizeof(T)));
  hipError_t e = in_launches(a.batch, shares, [&](int64_t first, dim3 grid) { k_orth_squares<T><<<grid, kProductThreads, 0, st>>>(a, first, shares, part); });
  if (e != hipSuccess) return e;
  e = in_launches(a.batch, chunks, [&](int64_t first, dim3 grid) { k_orth_begin<T, kS, NT><<<grid, kProductThreads, 0, st>>>(a, first, chunks, shares, part, X, A); });
  for (int i = 0; i < steps && e == hipSuccess; ++i) {
    const double* c = coefficients + 3 * i;
    const T *from = A;
    int parts = chunks;
    if (chunks > kMostShares) {
      constexpr int kBlocks = kS * kS / kProductThreads;
      e = in_launches(a.batch, kBlocks, [&](int64_t first, dim3 grid) { k_orth_join<T><<<grid, kProductThreads, 0, st>>>(first, kBlocks, chunks, kS * kS, A, sum); });
      if (e != hipSuccess) break;
      from = sum;
      parts = 1;
    }
    e = in_launches(a.batch, chunks, [&](int64_t first, dim3 grid) {
      if (i + 1 < steps) k_orth_step<T, kS, NT, false><<<grid, kProductThreads, 0, st>>>(a, first, chunks, parts, (T)c[0], (T)c[1], (T)c[2], X, from, next);
      else k_orth_step<T, kS, NT, true><<<grid, kProductThreads, 0, st>>>(a, first, chunks, parts, (T)c[0], (T)c[1], (T)c[2], X, from, next);
    });
    std::swap(A, next);
  }
  return e;
}

template <class T>
hipError_t orthogonalise(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  if (std::min(a.m, a.n) <= kMostRows) {
    const Few f(a.m, a.n, sizeof(T) == 8);
    auto go = [&](auto rows) {
      constexpr int kS = decltype(rows)::value;
      if constexpr (sizeof(T) == 4)
        if (f.wide == 128) return few_rows<T, kS, 2>(a, coefficients, steps, ws, st);
      return few_rows<T, kS, 1>(a, coefficients, steps, ws, st);
    };
    switch (f.rows) {
      case 32: return go(std::integral_constant<int, 32>());
      case 64: return go(std::integral_constant<int, 64>());
      case 96: return go(std::integral_constant<int, 96>());
      default: return go(std::integral_constant<int, 128>());
    }
  }
  return a.m % 4 == 0 && a.n % 4 == 0 ? steps_of<T, true>(a, coefficients, steps, ws, st) : steps_of<T, false>(a, coefficients, steps, ws, st);
}

}  // namespace
}  // namespace cgtp
