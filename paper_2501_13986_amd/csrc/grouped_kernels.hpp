// Kernels of the products by kind of row, for the translation units of their two types (grouped_f32.hip, grouped_f64.hip).
//
// Positions ptr[g] .. ptr[g+1] - 1 belong to group g; position p is row perm[p] (or p) of x and out, whose components are neighbours in it:
//     out = x W[g] + b[g],   gx = gout W[g]^T,   gW[g] = sum x^T gout,   gb[g] = sum gout.
// "Line" is a component of a position: line = position * comps + component.
// The host does not know ptr: workgroups find their group (find_group), and there are as many of them as any ptr can need.
#pragma once

#include <algorithm>
#include <type_traits>

#include "grouped.hpp"
#include "product.hpp"

namespace cgtp {
namespace {

// ---- positions and groups -----------------------------------------------------------------------------------------------------

__device__ inline int64_t cut(const GroupedArgs& a, int64_t g) {
  const int64_t p = a.ptr[g];
  return p < 0 ? 0 : p > a.rows ? a.rows : p;
}

// Pieces of `of` lines (a power of two) are numbered so that group g's begin at line(ptr[g]) / of + g: a group never needs more numbers than there
// are up to the next one's, and the number alone names the group.  The greatest group whose pieces begin at or before `id`: 64 of them at a time.
__device__ inline int64_t first_piece(const GroupedArgs& a, int64_t g, int64_t comps, int shift) { return (cut(a, g) * comps >> shift) + g; }

__device__ inline int64_t find_group(const GroupedArgs& a, int64_t comps, int shift, int64_t id) {
  int64_t lo = 0, n = a.groups;
  while (n > 1) {
    const int64_t step = (n + 63) / 64, g = lo + (threadIdx.x & 63) * step;
    const bool in = g < lo + n;
    const int64_t key = first_piece(a, in ? g : lo, comps, shift);
    const int found = __popcll(__ballot(in && key <= id));
    const int64_t skip = found > 0 ? (found - 1) * step : 0;
    lo += skip;
    n = n - skip < step ? n - skip : step;
  }
  return lo;
}

// lines -> positions and components, for lines of one workgroup: numbers below 2^16 past a line that is divided once
struct Lines {
  int64_t position;      // of line 0
  unsigned component, comps;
  float inverse;
  __device__ Lines(int64_t first, int64_t comps_) : comps((unsigned)comps_) {
    position = comps == 1 ? first : first / comps_;
    component = (unsigned)(first - position * comps_);
    inverse = 1.f / (float)comps;
  }
  // position (past the first one) and component of line i
  __device__ void of(unsigned i, unsigned& p, unsigned& m) const {
    const unsigned u = component + i;
    p = (unsigned)((float)u * inverse);      // off by one at most
    int r = (int)(u - p * comps);
    p += r < 0 ? -1 : r >= (int)comps ? 1 : 0;
    m = u - p * comps;
  }
};

// ---- lines through buffer descriptors -------------------------------------------------------------------------------------------

template <int kHow, class T>
__device__ inline void store_at(const T (&v)[1], Buffer B, unsigned at) {
  if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v[0]), B, at, 0, kHow);
  else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v[0]), B, at, 0, kHow);
}
template <int kHow>
__device__ inline void store_at(const float (&v)[2], Buffer B, unsigned at) {
  __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{v[0], v[1]}), B, at, 0, kHow);
}

// the row of a position, -1: none
__device__ inline int64_t row_of(const GroupedArgs& a, int64_t p) {
  const int64_t r = a.perm ? a.perm[p] : p;
  return r >= 0 && r < a.rows ? r : -1;
}

// ---- rows times a matrix of at most 128 rows --------------------------------------------------------------------------------------

constexpr int kMostTerms = 128, kMostShift = 10;      // lines of a workgroup

// A wave keeps the parts of its 16 NT columns of the matrix in registers, for up to 2^kMostShift lines of one group, whose parts the workgroup puts into LDS once for its four
// waves, 64 at a time.  Lane: columns NT l16 + j.  out = x W + b, or gx = gout W^T (kBack).
// Lines are reached through buffer descriptors of less than 2^31 bytes: what is not wanted has the offset kNowhere, which is behind them, reads zero and is not
// written, so that no store waits behind a branch (160 710 x 64 -> 2176 fp32: 465 us with branches and 64-bit addresses, 320 in passes, 4.5 TB/s; the writes are the bound
// beside six matrix products for one, pipe busy 45 % of the cycles at 1.6 to 1.8 GHz).  20 000 rows of 3 x 128 -> 128, 89 kinds, through a permutation 23 us, of 7 components
// 41 (3.5 TB/s).  One row 6 us: a chain of loads, group, row, its numbers.  Stores past the caches were no faster.
template <class T, int kIn>
struct StreamLds {
  Operand<T, 64> X[kIn / 32];
  unsigned from[1 << kMostShift], place[1 << kMostShift];      // of the lines in memory and in the results, bytes
};

template <class T, int kIn, int NT, bool kWhole, bool kBack>
__device__ __forceinline__ void stream_lines(const GroupedArgs& a, int64_t first_id, unsigned block, int column_tiles, int shift, StreamLds<T, kIn>& S) {
  using N = Num<T>;
  constexpr int kSlices = kIn / 32, kPer = 2, e = sizeof(T);
  auto &X = S.X;
  auto &from = S.from, &place = S.place;
  const int64_t id = first_id + block / column_tiles, g = find_group(a, a.comps, shift, id), piece = first_piece(a, g, a.comps, shift);
  const int64_t lines_end = cut(a, g + 1) * a.comps, begin = cut(a, g) * a.comps + ((id - piece) << shift);
  if (id < piece || begin >= lines_end) return;
  const int have = (int)(lines_end - begin < 1 << shift ? lines_end - begin : 1 << shift);
  const int K = (int)(kBack ? a.d_out : a.d_in), n = (int)(kBack ? a.d_in : a.d_out);
  const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, c = (int)(block % column_tiles) * (64 * NT) + (threadIdx.x >> 6) * (16 * NT) + l16 * NT;
  const T* W = (const T*)a.W + g * a.d_in * a.d_out;
  const Lines lines(begin, a.comps);
  const int64_t ld = kBack ? a.ld_gout : a.ld_x, ld_to = kBack ? a.ld_gx : a.ld_out, row0 = a.perm ? 0 : lines.position;
  const int64_t span = a.perm ? a.rows : (have + lines.component + a.comps - 1) / a.comps;      // rows that lines may be in
  const Buffer x = buffer_of((const T*)(kBack ? a.gout : a.x) + row0 * ld, ((span - 1) * ld + a.comps * K) * e);
  const Buffer to = buffer_of((T*)(kBack ? a.gx : a.out) + row0 * ld_to, ((span - 1) * ld_to + a.comps * n) * e);
  for (int i = threadIdx.x; i < (have + 63) / 64 * 64; i += kProductThreads) {
    unsigned at, m;
    lines.of(i < have ? i : 0, at, m);
    const int64_t r = row_of(a, lines.position + at) - row0;
    const bool ok = i < have && r >= 0;
    from[i] = ok ? (unsigned)((r * ld + m * (int64_t)K) * e) : kNowhere;
    place[i] = ok ? (unsigned)((r * ld_to + m * (int64_t)n) * e) : kNowhere;
  }
  __syncthreads();
  T next[kSlices][kPer][4];
  const int row = threadIdx.x / 8, term = threadIdx.x % 8 * 4;      // a thread copies four terms of lines row + 32 i
  auto fetch = [&](int line) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const unsigned at = from[line + row + i * 32];
#pragma unroll
      for (int s = 0; s < kSlices; ++s) load_at<kWhole>(x, at, s * 32 + term, K, next[s][i]);
    }
  };
  fetch(0);
  // the matrix: rows behind its end are zero, columns behind it any
  typename N::Parts w[kSlices][NT];
  T bias[NT];
#pragma unroll
  for (int s = 0; s < kSlices; ++s) {
    T v[NT][8];
    if constexpr (kBack) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const T* p = W + (int64_t)(c + j < n ? c + j : 0) * K;
        load_some<T, 4, kWhole>(p, s * 32 + q * 8, K, v[j]);
        load_some<T, 4, kWhole>(p, s * 32 + q * 8 + 4, K, v[j] + 4);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = s * 32 + q * 8 + i;
        T u[NT];
        load_some<T, NT, kWhole>(W + (int64_t)(k < K ? k : 0) * n, c, n, u);
#pragma unroll
        for (int j = 0; j < NT; ++j) v[j][i] = k < K ? u[j] : T(0);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) w[s][j] = N::parts(v[j]);
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) bias[j] = !kBack && a.b ? ((const T*)a.b)[g * n + (c + j < n ? c + j : 0)] : T(0);
  // a lane's columns: of all, or of the first alone where the row ends behind it
  const unsigned at_all = c + NT <= n ? (unsigned)c * e : kNowhere, at_last = c + 1 == n ? (unsigned)c * e : kNowhere;
  typename N::Vec o[2][NT];
  auto products = [&](int rt, typename N::Vec* to) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) to[j][i] = bias[j];
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
      const typename N::Parts xa = X[s].read(rt * 16 + l16, q * 8);
      if constexpr (NT == 2) N::template mma<2>({&xa, &xa}, {&w[s][0], &w[s][1]}, {&to[0], &to[1]});
      else N::template mma<1>({&xa}, {&w[s][0]}, {&to[0]});
    }
  };
  auto finish = [&](int line, const typename N::Vec* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned at = place[line + N::row(q, i)];
      T u[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) u[j] = v[j][i];
      store_at<0>(u, to, plus(at, at_all));
      if constexpr (NT == 2 && !kWhole) store_at<0>({u[0]}, to, plus(at, at_last));
    }
  };
  for (int line = 0; line < have; line += 64) {
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kSlices; ++s)
#pragma unroll
      for (int i = 0; i < kPer; ++i) X[s].write4(row + i * 32, term, next[s][i]);
    __syncthreads();
    if (line + 64 < have) fetch(line + 64);
    if (line + 16 < have) {      // the results of a tile are on their way while the products of the next one run
#pragma unroll
      for (int rt = 0; rt < 4; ++rt) {
        products(rt, o[rt & 1]);
        if (rt > 0) finish(line + rt * 16 - 16, o[~rt & 1]);
      }
      finish(line + 48, o[1]);
    } else {
      products(0, o[0]);
      finish(line, o[0]);
    }
  }
}

template <class T, int kIn, int NT, bool kWhole, bool kBack>
__global__ void __launch_bounds__(kProductThreads, 2) k_grouped_stream(GroupedArgs a, int64_t first_id, int column_tiles, int shift) {
  __shared__ StreamLds<T, kIn> S;
  stream_lines<T, kIn, NT, kWhole, kBack>(a, first_id, on_one_die(blockIdx.x, gridDim.x), column_tiles, shift, S);      // neighbours read the same lines
}

// ---- rows times a matrix ------------------------------------------------------------------------------------------------------

// kR lines x kC columns of out = x W + b (forward) or of gx = gout W^T (kBack), the terms 32 at a time: for more than 128 terms, and where
// lines lie far apart.  160 710 x 2176 -> 64 fp32 340 us (4.2 TB/s; pipe busy 38 % of the cycles, vector instructions, half of them cuts into
// parts, issue in 41 %), 60 710 x 200 -> 800 151 us (129 TFLOP/s), fp64 30 000 x 200 -> 200 76 us (32 TFLOP/s, library 73; LDS conflicts in
// 40 % of its cycles).  kFar: rows lie 2^31 bytes apart or more, or the matrix is as large.
template <class T, int kR, int kC, bool kWhole, bool kBack, bool kFar>
__global__ void __launch_bounds__(kProductThreads, 2) k_grouped_rows(GroupedArgs a, int64_t first_id, int column_tiles) {
  using Rows = AlongTerms<T, kR, kWhole>;
  using Along = AlongTerms<T, kC, kWhole>;
  __shared__ Operand<T, kR> R;
  __shared__ std::conditional_t<kBack, Operand<T, kC>, typename AcrossTerms<T, kC, kWhole>::To> C;
  __shared__ int64_t place[kR];      // of the lines in the results, -1: none
  constexpr int kShift = kR == 128 ? 7 : kR == 64 ? 6 : 5, e = sizeof(T);
  const unsigned block = on_one_die(blockIdx.x, gridDim.x);
  const int64_t id = first_id + block / column_tiles, g = find_group(a, a.comps, kShift, id);
  const int64_t lines_end = cut(a, g + 1) * a.comps, begin = cut(a, g) * a.comps + ((id - first_piece(a, g, a.comps, kShift)) << kShift);
  if (id < first_piece(a, g, a.comps, kShift) || begin >= lines_end) return;
  const int have = (int)(lines_end - begin < kR ? lines_end - begin : kR);
  const int K = (int)(kBack ? a.d_out : a.d_in), n = (int)(kBack ? a.d_in : a.d_out), c0 = (int)(block % column_tiles) * kC;
  const T *x = (const T*)(kBack ? a.gout : a.x), *W = (const T*)a.W + g * a.d_in * a.d_out;
  const int64_t ld = kBack ? a.ld_gout : a.ld_x, ld_to = kBack ? a.ld_gx : a.ld_out;
  const Lines lines(begin, a.comps);
  const int64_t row0 = kFar || a.perm ? 0 : lines.position, span = a.perm ? a.rows : (have + lines.component + a.comps - 1) / a.comps;
  const Buffer bx = buffer_of(x + row0 * ld, kFar ? 0 : ((span - 1) * ld + a.comps * K) * e), bw = buffer_of(W, kFar ? 0 : a.d_in * a.d_out * e);
  const T *p[Rows::kPer], *pw[Along::kPer];
  unsigned at_x[Rows::kPer], at_w[Along::kPer];
#pragma unroll
  for (int i = 0; i < Rows::kPer; ++i) {
    unsigned at, m;
    const int line = Rows::row(i);
    lines.of(line < have ? line : 0, at, m);
    const int64_t r = row_of(a, lines.position + at), from = (r < 0 ? 0 : r - row0) * ld + m * (int64_t)K;
    p[i] = x + from;
    at_x[i] = r < 0 ? kNowhere : (unsigned)(from * e);
    if (threadIdx.x % 8 == 0) place[line] = r < 0 || line >= have ? -1 : r * ld_to + m * (int64_t)n;
  }
  // tiles of half the lines, taken where there are few, fetch two steps ahead (fp64 2503 x 96 x 301 both gradients 37.3 -> 33.7 us); the others have enough waves a unit
  constexpr int kAhead = !kFar && kR < (sizeof(T) == 4 ? 128 : 64) ? 2 : 1;
  Rows rows[2];
  using Across = AcrossTerms<T, kC, kWhole>;
  Across across[2] = {Across(c0, n), Across(c0, n)};
  Along along[2];
  if constexpr (kBack)
#pragma unroll
    for (int i = 0; i < Along::kPer; ++i) {
      const int c = c0 + Along::row(i);
      pw[i] = W + (int64_t)(c < n ? c : 0) * K;
      at_w[i] = c < n ? (unsigned)c * (unsigned)K * e : kNowhere;
    }
  auto fetch = [&](int slot, int k0) {
    if constexpr (kFar) rows[slot].fetch(p, k0, K);
    else rows[slot].fetch(bx, at_x, k0, K);
    if constexpr (kBack) {
      if constexpr (kFar) along[slot].fetch(pw, k0, K);
      else along[slot].fetch(bw, at_w, k0, K);
    } else if constexpr (kFar) {
      const T* q[8];
      bool ok[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = k0 + Across::term() + j;
        ok[j] = k < K;
        q[j] = W + (int64_t)(ok[j] ? k : 0) * n;
      }
      across[slot].fetch(q, ok);
    } else {
      unsigned q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = k0 + Across::term() + j;
        q[j] = k < K ? (unsigned)k * (unsigned)n * e : kNowhere;
      }
      across[slot].fetch(bw, q);
    }
  };
  Results<T, kR, kC> out;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i, i * kStep);
  for (int k0 = 0; k0 < K; k0 += kAhead * kStep) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i > 0 && k0 + i * kStep >= K) break;
      __syncthreads();
      rows[i].put(R);
      if constexpr (kBack) along[i].put(C);
      else across[i].put(C);
      __syncthreads();
      if (kAhead > 1 || k0 + kStep < K) fetch(i, k0 + (i + kAhead) * kStep);
      out.multiply(R, C);
    }
  }
  const T* bias = kBack || !a.b ? nullptr : (const T*)a.b + g * n;
  T* to = (T*)(kBack ? a.gx : a.out);
#pragma unroll
  for (int ct = 0; ct < out.CT; ++ct) {
    const int c = c0 + out.column(ct);
    T add[4] = {};
    if (bias)
#pragma unroll
      for (int i = 0; i < 4; ++i) add[i] = bias[c + i < n ? c + i : 0];
#pragma unroll
    for (int rt = 0; rt < out.RT; ++rt) {
      const int64_t at = place[out.row(rt)];
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = out.acc[rt][ct][i] + add[i];
      if (at >= 0 && c < n) store_some(to + at + c, v, n - c);
    }
  }
}

// ---- the matrices' gradients ----------------------------------------------------------------------------------------------------

// kR x kC numbers of gW[g] (and kC of gb[g]) over the positions of group g in one chunk: chunks are the same for all groups, so that those of a group that has several
// leave their sums at slot 2 chunk + (0: the group began before the chunk, 1: in it).  A group with one chunk, or without rows, is
// written at once.
// The lines' offsets stand in LDS, formed once for all waves (160 710 x 64 x 2176 fp32: 710 us with addresses formed by each thread, 420 to 430
// so and in chunks of 1024; pipe busy 31 % of the cycles, vector instructions 38, LDS 26; the library's rate for its products is 246).
// 20 000 x 7 x 128 x 128: 46 us, 3.1 TB/s of its two inputs, in 330 x 2 workgroups, fewer than three a unit.
constexpr int kTable = 512;      // lines whose offsets stand in LDS at a time

// kFar: rows of x or gout lie 2^31 bytes apart or more, addresses are formed for each.
template <class T, int kR, int kC, bool kFar>
struct WeightsLds {
  typename AcrossTerms<T, kR, false>::To R;
  typename AcrossTerms<T, kC, false>::To C;
  alignas(16) unsigned table[kFar ? 1 : kTable][2];
};

template <class T, int kR, int kC, bool kWhole, bool kFar>
__device__ __forceinline__ void sum_weights(const GroupedArgs& a, int64_t first_id, unsigned block, int shift, int row_tiles, int column_tiles,
                                            T* part, double* part_b, WeightsLds<T, kR, kC, kFar>& S) {
  auto& R = S.R;
  auto& C = S.C;
  auto& table = S.table;
  const int tiles = row_tiles * column_tiles, tile = block % tiles;
  const int64_t id = first_id + block / tiles, g = find_group(a, 1, shift, id), chunk = id - g;
  const int64_t from = cut(a, g), end = cut(a, g + 1), lo = std::max(from, chunk << shift), hi = std::min(end, (chunk + 1) << shift);
  const bool empty = end <= from && chunk == from >> shift;
  if (chunk < from >> shift || (hi <= lo && !empty)) return;
  const int K = (int)a.d_in, n = (int)a.d_out, comps = (int)a.comps, k0 = tile / column_tiles * kR, c0 = tile % column_tiles * kC;
  AcrossTerms<T, kR, kWhole> x(k0, K);
  AcrossTerms<T, kC, kWhole> t(c0, n);
  Results<T, kR, kC> out;
  // gb is summed in fp64 and rounded once: in fp32 each row would round the sum of those before it (root mean square error of 160 710 normal
  // rows 4.5e-7, so 2.5e-8), for 1 % of the time of the kernel
  const bool add_b = a.gb && k0 == 0;
  double sum[kC / 64] = {};
  // the position and component of the wave's first term; all of it is the wave's own
  unsigned position = (unsigned)lo + x.term() / comps;      // below 2^31 but for steps behind the end
  int component = x.term() % comps;
  const unsigned last = (unsigned)hi, rows = (unsigned)a.rows;
  const int skip = kStep / comps, rest = kStep % comps;
  auto fetch = [&]() {
    const T *px[8], *pt[8];
    bool ok[8];
    unsigned p = position;
    int m = component;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned at = p < last ? p : (unsigned)lo;
      unsigned r = at, beyond = 0;
      if (a.perm) {
        const u32x2 w = *(const u32x2*)(a.perm + at);
        r = w[0];
        beyond = w[1];
      }
      ok[j] = p < last && beyond == 0 && r < rows;
      const unsigned row = ok[j] ? r : 0, part_of = ok[j] ? (unsigned)m : 0;      // strides and rows are below 2^31
      px[j] = (const T*)a.x + ((uint64_t)row * (unsigned)a.ld_x + part_of * (unsigned)K);
      pt[j] = (const T*)a.gout + ((uint64_t)row * (unsigned)a.ld_gout + part_of * (unsigned)n);
      const bool next = ++m == comps;
      p += next ? 1 : 0;
      m = next ? 0 : m;
    }
    x.fetch(px, ok);
    t.fetch(pt, ok);
    component += rest;
    const bool next = component >= comps;
    position += skip + (next ? 1 : 0);
    component -= next ? comps : 0;
  };
  const int64_t count = hi > lo ? (hi - lo) * comps : 0;
  auto multiply = [&](bool more, auto fetch_next) {
    __syncthreads();
    x.put(R);
    t.put(C);
    __syncthreads();
    if (add_b)
#pragma unroll
      for (int i = 0; i < kC / 64; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[i] += (double)t.v[j][i];
    if (more) fetch_next();
    out.multiply(R, C);
  };
  if constexpr (kFar) {
    if (count > 0) fetch();
    for (int64_t l = 0; l < count; l += kStep) multiply(l + kStep < count, fetch);
  } else {
    const int64_t row0 = a.perm ? 0 : lo, span = a.perm ? a.rows : hi - lo;
    const Buffer bx = buffer_of((const T*)a.x + row0 * a.ld_x, ((span - 1) * a.ld_x + comps * (int64_t)K) * (int)sizeof(T));
    const Buffer bt = buffer_of((const T*)a.gout + row0 * a.ld_gout, ((span - 1) * a.ld_gout + comps * (int64_t)n) * (int)sizeof(T));
    for (int64_t l0 = 0; l0 < count; l0 += kTable) {
      const int lines = (int)(count - l0 < kTable ? count - l0 : kTable);
      const Lines of(lo * comps + l0, comps);
      __syncthreads();
      for (int i = threadIdx.x; i < (lines + kStep - 1) / kStep * kStep; i += kProductThreads) {
        unsigned at, m;
        of.of(i < lines ? i : 0, at, m);
        const int64_t r = row_of(a, of.position + at) - row0;
        const bool ok = i < lines && r >= 0;
        table[i][0] = ok ? (unsigned)((r * a.ld_x + m * (int64_t)K) * (int)sizeof(T)) : kNowhere;
        table[i][1] = ok ? (unsigned)((r * a.ld_gout + m * (int64_t)n) * (int)sizeof(T)) : kNowhere;
      }
      __syncthreads();
      auto fetch_at = [&](int l) {
        unsigned rx[8], rt[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const u32x4 w = *(const u32x4*)&table[l + x.term() + j][0];
          rx[j] = w[0];
          rt[j] = w[1];
          rx[j + 1] = w[2];
          rt[j + 1] = w[3];
        }
        x.fetch(bx, rx);
        t.fetch(bt, rt);
      };
      fetch_at(0);
      for (int l = 0; l < lines; l += kStep) multiply(l + kStep < lines, [&]() { fetch_at(l + kStep); });
    }
  }
  const bool whole = from >> shift == (end - 1) >> shift || empty;
  const int64_t slot = 2 * chunk + (from >= chunk << shift);
  T* to = whole ? (T*)a.gW + g * a.d_in * a.d_out : part + slot * a.d_in * a.d_out;
#pragma unroll
  for (int rt = 0; rt < out.RT; ++rt)
#pragma unroll
    for (int ct = 0; ct < out.CT; ++ct) {
      const int k = k0 + out.row(rt), c = c0 + out.column(ct);
      T v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = out.acc[rt][ct][i];
      if (k < K && c < n) store_some(to + (int64_t)k * n + c, v, n - c);
    }
  if (!add_b) return;
  // the waves' terms, one after another
  __syncthreads();
  double* sums = (double*)&C;      // [4][kC]
#pragma unroll
  for (int i = 0; i < kC / 64; ++i) sums[x.term() / 8 * kC + t.place() + i] = sum[i];
  __syncthreads();
  for (int c = threadIdx.x; c < kC && c0 + c < n; c += kProductThreads) {
    double v = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) v += sums[j * kC + c];
    if (whole) ((T*)a.gb)[g * a.d_out + c0 + c] = (T)v;
    else part_b[slot * a.d_out + c0 + c] = v;
  }
}

template <class T, int kR, int kC, bool kWhole, bool kFar>
__global__ void __launch_bounds__(kProductThreads, 2) k_grouped_weights(GroupedArgs a, int64_t first_id, int shift, int row_tiles, int column_tiles, T* part, double* part_b) {
  __shared__ WeightsLds<T, kR, kC, kFar> S;
  sum_weights<T, kR, kC, kWhole, kFar>(a, first_id, on_one_die(blockIdx.x, gridDim.x), shift, row_tiles, column_tiles, part, part_b, S);      // neighbours read the same rows
}

// Both gradients of few rows in one launch: the first `split` workgroups form gW, the others gx.
template <class T, int kC, int kIn>
union BackLds {
  WeightsLds<T, 64, kC, false> weights;
  StreamLds<T, kIn> lines;
  __device__ BackLds() {}
};

template <class T, int kC, int kIn, bool kWhole>
__global__ void __launch_bounds__(kProductThreads, 2) k_grouped_back(GroupedArgs a, int split, int chunk_shift, int row_tiles, int column_tiles, T* part, double* part_b, int x_tiles, int shift) {
  __shared__ BackLds<T, kC, kIn> S;
  if ((int)blockIdx.x < split) sum_weights<T, 64, kC, kWhole, false>(a, 0, blockIdx.x, chunk_shift, row_tiles, column_tiles, part, part_b, S.weights);
  else stream_lines<T, kIn, 1, kWhole, true>(a, 0, blockIdx.x - split, x_tiles, shift, S.lines);
}

// Adds up, in a fixed order, the chunks of the groups that have several: of group `at` (of_groups), or of the one that begins in chunk `at` and
// goes on behind it, whichever are fewer.  V numbers of gW a thread (of gb one, its sums are held in fp64); kParts: so many shares of the chunks
// are added up by threads of their own, where a matrix has too few numbers for the latency of its chunks (10 000 x 32 x 64 fp32, 157 chunks:
// 4.1 us in eight shares, 7.0 in one; 160 710 x 64 x 2176 32 and 20).  Addresses are stepped by sums: multiplied out for all eight loads on
// their way they cost 1.4 of 6.4 us (20 000 x 7 x 128 x 128).
template <class T, int V, int kParts>
__global__ void __launch_bounds__(kProductThreads) k_grouped_sums(GroupedArgs a, int64_t first, int shift, int blocks, bool of_groups, const T* part, const double* part_b) {
  const int64_t at = first + blockIdx.x / blocks;
  int64_t lo = at;
  if (!of_groups) {
    const int64_t next = (at + 1) << shift;
    if (next >= a.rows) return;
    // the last group that begins before the next chunk
    lo = 0;
    int64_t n = a.groups;
    while (n > 1) {
      const int64_t step = (n + 63) / 64, g = lo + (threadIdx.x & 63) * step;
      const bool in = g < lo + n;
      const int found = __popcll(__ballot(in && cut(a, in ? g : lo) < next));
      const int64_t skip = found > 0 ? (found - 1) * step : 0;
      lo += skip;
      n = n - skip < step ? n - skip : step;
    }
  }
  const int64_t from = cut(a, lo), end = cut(a, lo + 1), chunk = from >> shift, last = (end - 1) >> shift;
  if (end <= from || last <= chunk || (!of_groups && chunk != at)) return;
  constexpr int kSide = kProductThreads / kParts;
  __shared__ alignas(32) char lds[kProductThreads * std::max(V * sizeof(T), sizeof(double))];
  const int64_t size = a.d_in * a.d_out, many = last - chunk + 1;
  const int lane = threadIdx.x % kSide, share = threadIdx.x / kSide;
  const int64_t from_c = many * share / kParts, end_c = many * (share + 1) / kParts;
  // words of kN numbers from w0 on, of `count` numbers a slot, whose sums are held in S
  auto add_up = [&](auto numbers, const auto* from, int64_t count, int64_t w0, T* to) {
    using S = std::remove_const_t<std::remove_pointer_t<decltype(from)>>;
    constexpr int kN = decltype(numbers)::value;
    typedef S Words __attribute__((ext_vector_type(kN)));
    Words(&sums)[kParts][kSide] = *(Words(*)[kParts][kSide])lds;
    const int64_t words = count / kN, i = (w0 + lane < words ? w0 + lane : words - 1) * kN;
    Words v = {};
    const S* p = from + i + 2 * (chunk + from_c) * count;
#pragma unroll 8
    for (int64_t c = from_c; c < end_c; ++c, p += 2 * count) v += *(const Words*)(p + (c == 0 ? count : 0));
    if constexpr (kParts > 1) {
      __syncthreads();
      sums[share][lane] = v;
      __syncthreads();
      if (share > 0) return;
#pragma unroll
      for (int j = 1; j < kParts; ++j) v += sums[j][lane];
    }
    if (w0 + lane >= words) return;
#pragma unroll
    for (int j = 0; j < kN; ++j) to[i + j] = (T)v[j];
  };
  const int64_t of_w = (size / V + kSide - 1) / kSide, of_b = a.gb ? (a.d_out + kSide - 1) / kSide : 0;
  int64_t w = blockIdx.x % blocks;
  for (; w < of_w; w += blocks) add_up(std::integral_constant<int, V>(), part, size, w * kSide, (T*)a.gW + lo * size);
  for (; w < of_w + of_b; w += blocks) add_up(std::integral_constant<int, 1>(), part_b, a.d_out, (w - of_w) * kSide, (T*)a.gb + lo * a.d_out);
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostBlocks = (int64_t)1 << 23;   // workgroups of a launch: 2^32 threads are too many

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// f(first, blocks) for pieces ids of `tiles` workgroups each, as many a launch as there may be
template <class F>
hipError_t in_launches(int64_t ids, int64_t tiles, F f) {
  const int64_t most = std::max<int64_t>(1, kMostBlocks / tiles);
  for (int64_t at = 0; at < ids; at += most) {
    f(at, dim3((unsigned)(std::min(most, ids - at) * tiles)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// columns of a tile of gW, which is 64 rows high: fp32 with 128 rows, two workgroups a compute unit instead of three, 20 000 x 7 x 128 x 128 49 us for 46, 30 000 x 300 x 300 72 for 60
template <class T>
constexpr int kTile = sizeof(T) == 4 ? 128 : 64;

// lines of a workgroup of k_grouped_stream: fewer where many leave compute units without work
int stream_shift(int64_t lines, int64_t tiles) {
  int shift = kMostShift;
  while (shift > 6 && (lines >> shift) * tiles < 1024) --shift;
  return shift;
}

// f(kIn) for the least of 32, 64, 96, 128 that holds the terms
template <class F>
hipError_t with_terms(int64_t terms, F f) {
  if (terms <= 32) return f(std::integral_constant<int, 32>());
  if (terms <= 64) return f(std::integral_constant<int, 64>());
  if (terms <= 96) return f(std::integral_constant<int, 96>());
  return f(std::integral_constant<int, 128>());
}

template <class T, int kIn, int NT, bool kBack>
hipError_t launch_stream(const GroupedArgs& a, hipStream_t st) {
  const int64_t n = kBack ? a.d_in : a.d_out, tiles = (n + 64 * NT - 1) / (64 * NT), lines = a.rows * a.comps;
  const bool whole = a.d_in % 4 == 0 && a.d_out % 4 == 0;
  const int shift = stream_shift(lines, tiles);
  return in_launches((lines >> shift) + a.groups, tiles, [&](int64_t first, dim3 grid) {
    if (whole) k_grouped_stream<T, kIn, NT, true, kBack><<<grid, kProductThreads, 0, st>>>(a, first, (int)tiles, shift);
    else k_grouped_stream<T, kIn, NT, false, kBack><<<grid, kProductThreads, 0, st>>>(a, first, (int)tiles, shift);
  });
}

template <class T, bool kBack>
hipError_t launch_few_terms(const GroupedArgs& a, hipStream_t st) {
  const int64_t terms = kBack ? a.d_out : a.d_in, n = kBack ? a.d_in : a.d_out;
  return with_terms(terms, [&](auto in) {
    constexpr int kIn = decltype(in)::value;
    if constexpr (sizeof(T) == 4)
      if (n > 64) return launch_stream<T, kIn, 2, kBack>(a, st);
    return launch_stream<T, kIn, 1, kBack>(a, st);
  });
}

// bytes from the first of `rows` rows to the end of the last; descriptors hold less than 2^31
bool in_reach(int64_t rows, int64_t ld, size_t element) { return rows * ld < (int64_t)(((size_t)1 << 31) / element); }

// whether k_grouped_stream serves
template <class T, bool kBack>
bool streams(const GroupedArgs& a) {
  const int64_t rows = a.perm ? a.rows : std::min(a.rows, ((int64_t)1 << kMostShift) / a.comps + 2);
  return (kBack ? a.d_out : a.d_in) <= kMostTerms && in_reach(rows, std::max(kBack ? a.ld_gout : a.ld_x, kBack ? a.ld_gx : a.ld_out), sizeof(T));
}

template <class T, bool kBack>
hipError_t launch_rows(const GroupedArgs& a, hipStream_t st) {
  if (streams<T, kBack>(a)) return launch_few_terms<T, kBack>(a, st);
  const int64_t rows = a.perm ? a.rows : std::min(a.rows, ((int64_t)1 << kMostShift) / a.comps + 2);
  const int64_t n = kBack ? a.d_in : a.d_out, lines = a.rows * a.comps;
  const bool whole = a.d_in % 4 == 0 && a.d_out % 4 == 0, near = in_reach(rows, kBack ? a.ld_gout : a.ld_x, sizeof(T)) && in_reach(a.d_in, a.d_out, sizeof(T));
  const int64_t tiles = (n + 63) / 64;
  auto go = [&](auto tall, auto whole_, auto far) {
    constexpr int kR = decltype(tall)::value;
    return in_launches(lines / kR + a.groups, tiles, [&](int64_t first, dim3 grid) {
      k_grouped_rows<T, kR, 64, decltype(whole_)::value, kBack, decltype(far)::value><<<grid, kProductThreads, 0, st>>>(a, first, (int)tiles);
    });
  };
  // tiles of half the lines where that fills compute units (fp64, 2503 x 301 -> 96, both one step ahead: 17 us for 32; many lines, fp32 160 710 x 2176 -> 64: 343 us, with half 366, with 128
  // columns of twice the registers no faster: 30 000 x 300 -> 300 47 us and 56)
  auto size = [&](auto whole_, auto far) {
    constexpr int kR = sizeof(T) == 4 ? 128 : 64;
    if constexpr (!decltype(far)::value)
      if (lines / kR * tiles < 512) return go(std::integral_constant<int, kR / 2>(), whole_, far);
    return go(std::integral_constant<int, kR>(), whole_, far);
  };
  if (!near) return size(std::false_type(), std::true_type());
  return whole ? size(std::true_type(), std::false_type()) : size(std::false_type(), std::false_type());
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// How the positions are cut for the matrices' gradients
template <class T>
struct Chunks {
  int64_t row_tiles, column_tiles, count, slots;      // chunks, partial sums
  int shift = 20;                                     // positions of a chunk
  Chunks(int64_t rows, int64_t K, int64_t n, int64_t comps) {
    row_tiles = (K + 63) / 64;
    column_tiles = (n + kTile<T> - 1) / kTile<T>;
    // Partial sums are 2 K n numbers of traffic a chunk, its lines K + n each: half as much with `least` lines (20 000 x 7 x 128 x 128, 256 lines: 60 us, with 128 68).
    // Fewer lines where compute units are without work (2503 x 96 x 301: 17 us with 64, 29 with 256).
    auto workgroups = [&]() { return (rows >> shift) * row_tiles * column_tiles; };
    const int64_t least = std::max<int64_t>(256, 4 * K * n / (K + n));
    while (shift > 4 && ((workgroups() < 1600 && comps << (shift - 1) >= least) || (workgroups() < 320 && comps << (shift - 1) >= 64))) --shift;
    count = (rows + ((int64_t)1 << shift) - 1) >> shift;
    slots = count > 1 ? 2 * count : 0;
  }
};

template <class T>
size_t workspace_bytes(int64_t rows, int64_t K, int64_t n, int64_t comps) {
  const Chunks<T> c(rows, K, n, comps);
  return up(c.slots * K * n * sizeof(T)) + up(c.slots * n * sizeof(double));
}

template <class T>
bool weights_near(const GroupedArgs& a, const Chunks<T>& c) {
  return in_reach(a.perm ? a.rows : std::min(a.rows, (int64_t)1 << c.shift), std::max(a.ld_x, a.ld_gout), sizeof(T));
}

template <class T, int kR, int kC>
hipError_t launch_weights(const GroupedArgs& a, const Chunks<T>& c, T* part, double* part_b, hipStream_t st) {
  const bool whole = a.d_in % 4 == 0 && a.d_out % 4 == 0;
  auto go = [&](auto whole, auto far) {
    return in_launches((a.rows >> c.shift) + a.groups, c.row_tiles * c.column_tiles, [&](int64_t first, dim3 grid) {
      k_grouped_weights<T, kR, kC, decltype(whole)::value, decltype(far)::value><<<grid, kProductThreads, 0, st>>>(a, first, c.shift, (int)c.row_tiles, (int)c.column_tiles, part, part_b);
    });
  };
  if (!weights_near<T>(a, c)) return go(std::false_type(), std::true_type());
  return whole ? go(std::true_type(), std::false_type()) : go(std::false_type(), std::false_type());
}

// workgroups up to which both gradients go in one launch: three a compute unit (small molecule 9.7 us a call for 12.4, 2503 x 96 x 100 fp32 13.9 for 17.3, fp64 17.4 for 22.0)
constexpr int64_t kFewBlocks = 768;

template <class T>
hipError_t backward(const GroupedArgs& a, char* ws, hipStream_t st) {
  const int64_t K = a.d_in, n = a.d_out;
  const Chunks<T> c(a.rows, K, n, a.comps);
  T* part = (T*)ws;
  double* part_b = (double*)(ws + up(c.slots * K * n * sizeof(T)));
  const int64_t x_tiles = (K + 63) / 64;
  const int shift = stream_shift(a.rows * a.comps, x_tiles);
  const int64_t for_weights = ((a.rows >> c.shift) + a.groups) * c.row_tiles * c.column_tiles, for_x = ((a.rows * a.comps >> shift) + a.groups) * x_tiles;
  hipError_t e;
  if (for_weights + for_x <= kFewBlocks && streams<T, true>(a) && weights_near<T>(a, c)) {
    e = with_terms(n, [&](auto in) {
      constexpr int kIn = decltype(in)::value, kC = kTile<T>;
      const dim3 grid((unsigned)(for_weights + for_x));
      if (K % 4 == 0 && n % 4 == 0)
        k_grouped_back<T, kC, kIn, true><<<grid, kProductThreads, 0, st>>>(a, (int)for_weights, c.shift, (int)c.row_tiles, (int)c.column_tiles, part, part_b, (int)x_tiles, shift);
      else
        k_grouped_back<T, kC, kIn, false><<<grid, kProductThreads, 0, st>>>(a, (int)for_weights, c.shift, (int)c.row_tiles, (int)c.column_tiles, part, part_b, (int)x_tiles, shift);
      return hipGetLastError();
    });
  } else {
    e = launch_rows<T, true>(a, st);
    if (e == hipSuccess) e = launch_weights<T, 64, kTile<T>>(a, c, part, part_b, st);
  }
  if (e != hipSuccess || c.slots == 0) return e;
  // most chunks have nothing to add up, so that they get few workgroups
  const bool of_groups = a.groups <= c.count - 1, wide = n % 4 == 0 && aligned16(a.gW);
  const int64_t pieces = of_groups ? a.groups : c.count - 1, numbers = K * n / (wide ? 4 : 1), numbers_b = a.gb ? n : 0;
  auto go = [&](auto wide_, auto parts) {
    constexpr int V = decltype(wide_)::value, kParts = decltype(parts)::value, kSide = kProductThreads / kParts;
    const int64_t blocks = std::max<int64_t>(1, std::min((numbers + kSide - 1) / kSide + (numbers_b + kSide - 1) / kSide, std::max<int64_t>(16, 16384 / pieces)));
    return in_launches(pieces, blocks, [&](int64_t first, dim3 grid) {
      k_grouped_sums<T, V, kParts><<<grid, kProductThreads, 0, st>>>(a, first, c.shift, (int)blocks, of_groups, part, part_b);
    });
  };
  using One = std::integral_constant<int, 1>;
  using Four = std::integral_constant<int, 4>;
  using Eight = std::integral_constant<int, 8>;
  // few numbers: the latency of the chunks bounds (20 000 x 128 x 128, 4096 words: 6.4 us in eight shares, 8.9 in one); many: the traffic (28 896 words of fp64 9.7 and 5.0)
  if (numbers <= 8192) return wide ? go(Four(), Eight()) : go(One(), Eight());
  return wide ? go(Four(), One()) : go(One(), One());
}

}  // namespace
}  // namespace cgtp
