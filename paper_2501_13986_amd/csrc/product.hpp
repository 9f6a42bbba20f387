// Products of matrices in memory, a tile of results a workgroup: the parts of 32 terms of both operands in LDS at a time, the next ones on their way to
// registers meanwhile.  For the products by kind of row (grouped_kernels.hpp) and the steps of orthogonalise (orth_kernels.hpp).
//
// The results are kR rows x kC columns, four waves 2 x 2.  The columns are the left operand of the matrix instructions, so that a lane's results are four neighbours
// of one row: row l16 of a tile, columns 4 q + (0..3).
// Nothing here depends on a lane's own condition until results are stored: addresses outside are replaced by ones inside and what they read by zero.
#pragma once

#include "mma.hpp"

namespace cgtp {
namespace {

constexpr int kProductThreads = 256;
constexpr int kStep = 32;      // terms in LDS at a time

// Neighbouring workgroups go to the eight dies in turn: the numbers that make neighbours in work run on one, whose L2 they share.
__device__ inline unsigned on_one_die(unsigned block, unsigned blocks) {
  const unsigned die = block % 8, each = blocks / 8, more = blocks % 8;
  return die * each + (die < more ? die : more) + block / 8;
}

// ---- buffer descriptors: what is behind their range reads as zero and is not written, without a branch

using Buffer = __amdgpu_buffer_rsrc_t;
constexpr unsigned kNowhere = 0x80000000u;      // an offset behind every range

// sums of offsets that stay behind the range where one of them is
__device__ inline unsigned plus(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }

__device__ inline Buffer buffer_of(const void* p, int64_t bytes) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)bytes, 0x00020000); }

// four numbers from column k on of the line at offset `at`, zero behind its end.  kWhole: its width is a multiple of four.
template <bool kWhole, class T>
__device__ inline void load_at(Buffer B, unsigned at, int k, int width, T* v) {
  constexpr int e = sizeof(T);
  const unsigned off = plus(at, k < width ? (unsigned)k * e : kNowhere);
  if constexpr (e == 4) {
    const f32x4 w = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(B, off, 0, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f64x2 w = __builtin_bit_cast(f64x2, __builtin_amdgcn_raw_buffer_load_b128(B, plus(off, h * 16), 0, 0));
      v[2 * h] = w[0];
      v[2 * h + 1] = w[1];
    }
  }
  if constexpr (!kWhole)
#pragma unroll
    for (int i = 1; i < 4; ++i) v[i] = k + i < width ? v[i] : T(0);
}

// which of 16 columns lane l16 of a left operand holds, for results 4 q + i to be neighbours: a lane's results are rows Num::row(q, i) of the instruction
template <class T>
__device__ inline int column_place(int l16) {
  return sizeof(T) == 4 ? l16 : l16 % 4 * 4 + l16 / 4;
}

// V neighbours of a row of `width` numbers from column k on, zero behind its end.  kWhole: width is a multiple of V.
template <class T, int V, bool kWhole>
__device__ inline void load_some(const T* row, int k, int width, T* v) {
  typedef T Words __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  if (kWhole || width >= V) {
    const int at = k <= width - V ? k : width - V;
    const Words w = *(const Words*)(row + at);
    if constexpr (kWhole) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = k < width ? w[i] : T(0);
    } else {      // the row's last ones, moved down
      const int s = k - at;
      T u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] = s & 1 ? (i + 1 < V ? w[i + 1] : T(0)) : w[i];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = s >= V ? T(0) : V > 2 && (s & 2) ? (i + 2 < V ? u[i + 2] : T(0)) : u[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const T w = row[k + i < width ? k + i : 0];
      v[i] = k + i < width ? w : T(0);
    }
  }
}

// kR rows (columns) of 32 terms in LDS.  A wave reads 16 bytes of each of 16 rows, 16 lanes at a time, of two neighbouring quarters (lanes 0-3, 12-15 and 20-27 together, counters
// show): the 16 bytes of a row change places with bits of the row's number so that these find different banks, 256 bytes in all, and so do the lanes that write, 128
// bytes at a time.  They write
//   kWholeRows     rows of 64 bytes one behind the other, or 16 bytes of neighbouring rows
//   kEveryOther    16 bytes of every other row: the odd rows stand behind the even ones (128 rows)
//   kApart         pieces of rows that are four apart: rows are 80 bytes apart
enum Written { kWholeRows, kEveryOther, kApart };
template <class T, int kR, Written kBy = kWholeRows>
struct alignas(16) Operand;
template <int kR, Written kBy>
struct alignas(16) Operand<float, kR, kBy> {
  __bf16 v[3][kR][kBy == kApart ? kStep + 8 : kStep];
  static __device__ int line(int r) { return kBy == kEveryOther ? r >> 1 | (r & 1) << 6 : r; }
  static __device__ int at(int r, int k) {
    const int w = line(r);
    return k ^ (kBy == kApart ? (w >> 2 ^ w >> 3) & 1 : (w >> 1 ^ w >> 6) & 3) * 8;
  }
  __device__ PartsOf<3> read(int r, int k) const {
    PartsOf<3> p;
#pragma unroll
    for (int i = 0; i < 3; ++i) p.w[i] = *(const u32x4*)&v[i][line(r)][at(r, k)];
    return p;
  }
  __device__ void write4(int r, int k, const float* x) {
    unsigned lo[3], hi[3];
    Num<float>::split(x[0], x[1], lo);
    Num<float>::split(x[2], x[3], hi);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(u32x2*)&v[p][line(r)][at(r, k)] = u32x2{lo[p], hi[p]};
  }
  __device__ void write8(int r, int k, const float* x) {
    const PartsOf<3> w = Num<float>::parts(x);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(u32x4*)&v[p][line(r)][at(r, k)] = w.w[p];
  }
  __device__ void write_some(int r, int k, const float (&x)[2]) {
    unsigned w[3];
    Num<float>::split(x[0], x[1], w);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(unsigned*)&v[p][line(r)][at(r, k)] = w[p];
  }
};
template <int kR, Written kBy>
struct alignas(16) Operand<double, kR, kBy> {
  double v[kR][kStep + 2];
  __device__ PartsOf<4> read(int r, int k) const {
    PartsOf<4> p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.w[i] = *(const u32x4*)&v[r][k + 2 * i];
    return p;
  }
  __device__ void write4(int r, int k, const double* x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *(u32x4*)&v[r][k + 2 * h] = __builtin_bit_cast(u32x4, f64x2{x[2 * h], x[2 * h + 1]});
  }
  __device__ void write8(int r, int k, const double* x) {
    write4(r, k, x);
    write4(r, k + 4, x + 4);
  }
  __device__ void write_some(int r, int k, const double (&x)[1]) { v[r][k] = x[0]; }
};

// An operand whose terms are neighbours in memory: a thread has four of them of each of kPer rows
template <class T, int kR, bool kWhole>
struct AlongTerms {
  static constexpr int kPer = kR / 32;
  T v[kPer][4];
  static __device__ int row(int i) { return i * 32 + (int)threadIdx.x / 8; }      // of the thread's i-th
  static __device__ int term() { return (int)threadIdx.x % 8 * 4; }
  // p: the rows in memory, any address inside where there is none (their results are not kept)
  __device__ void fetch(const T* const (&p)[kPer], int k0, int terms) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) load_some<T, 4, kWhole>(p[i], k0 + term(), terms, v[i]);
  }
  // the same through a buffer descriptor, rows at the offsets `at`
  __device__ void fetch(Buffer B, const unsigned (&at)[kPer], int k0, int terms) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) load_at<kWhole>(B, at[i], k0 + term(), terms, v[i]);
  }
  __device__ void put(Operand<T, kR>& to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) to.write4(row(i), term(), v[i]);
  }
};

// An operand whose terms are rows of memory: a wave has eight of them, so that their addresses are the wave's, and a thread kPer neighbours of each
template <class T, int kR, bool kWhole>
struct AcrossTerms {
  static constexpr int kPer = kR / 64;
  using To = Operand<T, kR, kPer == 2 ? kEveryOther : kWholeRows>;
  T v[8][kPer];
  unsigned at[kPer];      // bytes from the start of a row
  static __device__ int place() { return ((int)threadIdx.x & 63) * kPer; }
  static __device__ int term() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) * 8; }
  // places first .. of rows of `width` numbers; those behind the end hold anything: their results are not kept.  kWhole: width is a multiple of kPer.
  __device__ AcrossTerms(int first, int width) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int c = first + place() + i;
      at[i] = (unsigned)(c < width ? c : kWhole ? i : width - 1) * (unsigned)sizeof(T);
    }
  }
  // p: rows of the wave's terms, an address inside where there is none (ok false: zero)
  __device__ void fetch(const T* const (&p)[8], const bool (&ok)[8]) {
    typedef T Words __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
    bool all = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (kWhole) {
        const Words w = *(const Words*)((const char*)p[j] + at[0]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[j][i] = w[i];
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[j][i] = *(const T*)((const char*)p[j] + at[i]);
      }
      all = all && ok[j];
    }
    if (!all) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[j][i] = ok[j] ? v[j][i] : T(0);
    }
  }
  // the same through a buffer descriptor, rows at the offsets `row`: what is behind its range is zero
  __device__ void fetch(Buffer B, const unsigned (&row)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (kWhole && kPer == 2 && sizeof(T) == 4) {
        const f32x2 w = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(B, plus(row[j], at[0]), 0, 0));
        v[j][0] = w[0];
        v[j][1] = w[1];
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if constexpr (sizeof(T) == 4) v[j][i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(B, plus(row[j], at[i]), 0, 0));
          else v[j][i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b64(B, plus(row[j], at[i]), 0, 0));
        }
      }
    }
  }
  __device__ void put(To& to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const T x[8] = {v[0][i], v[1][i], v[2][i], v[3][i], v[4][i], v[5][i], v[6][i], v[7][i]};
      to.write8(place() + i, term(), x);
    }
  }
};

// The results of a workgroup, kUp x kAcross waves
template <class T, int kR, int kC, int kUp = 2, int kAcross = 2>
struct Results {
  using N = Num<T>;
  static constexpr int RT = kR / (16 * kUp), CT = kC / (16 * kAcross), kThreads = 64 * kUp * kAcross;
  typename N::Vec acc[RT][CT] = {};
  static __device__ int lane() { return (int)threadIdx.x & 63; }
  static __device__ int wave() { return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6); }
  static __device__ int first_row() { return wave() / kAcross * (kR / kUp); }
  static __device__ int first_column() { return wave() % kAcross * (kC / kAcross); }
  static __device__ int row(int rt) { return first_row() + rt * 16 + lane() % 16; }
  static __device__ int column(int ct) { return first_column() + ct * 16 + lane() / 16 * 4; }      // the first of four
  // in the order of the registers: kR x kC numbers
  __device__ void keep(T* to) const {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) __builtin_nontemporal_store(acc[rt][ct], (typename N::Vec*)(to + ((rt * CT + ct) * kThreads + (int)threadIdx.x) * 4));
  }
  // the sum of `parts` such times factor(part), in their order; sixteen loads on their way
  template <class F>
  __device__ void add_all(const T* from, int parts, F factor) {
    constexpr int kAtOnce = RT * CT >= 16 ? 1 : 16 / (RT * CT);
    from += (int)threadIdx.x * 4;
    int p = 0;
    for (; p + kAtOnce <= parts; p += kAtOnce) {
      typename N::Vec v[kAtOnce][RT][CT];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) v[j][rt][ct] = *(const typename N::Vec*)(from + (int64_t)(p + j) * (kR * kC) + (rt * CT + ct) * kThreads * 4);
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const T f = factor(p + j);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) acc[rt][ct] += f * v[j][rt][ct];
      }
    }
    for (; p < parts; ++p) {
      const T f = factor(p);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) acc[rt][ct] += f * *(const typename N::Vec*)(from + (int64_t)p * (kR * kC) + (rt * CT + ct) * kThreads * 4);
    }
  }
  // the same of one tile of rows, from a thread's own first number on
  static __device__ void add_up(const T* from, int parts, typename N::Vec (&to)[CT]) {
#pragma unroll 4
    for (int p = 0; p < parts; ++p)
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) to[ct] += *(const typename N::Vec*)(from + (int64_t)p * (kR * kC) + ct * kThreads * 4);
  }
  template <Written kByR, Written kByC>
  __device__ void multiply(const Operand<T, kR, kByR>& R, const Operand<T, kC, kByC>& C) {
    const int l16 = lane() % 16, k = lane() / 16 * 8, r0 = first_row(), c0 = first_column() + column_place<T>(l16);
    typename N::Parts c[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) c[ct] = C.read(c0 + ct * 16, k);
    constexpr int kSide = CT >= 4 || RT < 2 ? 1 : 2;      // rows of tiles side by side: chains of sums in turn; the last of an odd number stands alone
#pragma unroll
    for (int rt = 0; rt < RT; rt += kSide) {
      typename N::Parts r[kSide];
#pragma unroll
      for (int s = 0; s < kSide && rt + s < RT; ++s) r[s] = R.read(r0 + (rt + s) * 16 + l16, k);
      constexpr int kUnits = sizeof(T) == 4 ? 6 : 8;
#pragma unroll
      for (int m = 0; m < kUnits; ++m)
#pragma unroll
        for (int s = 0; s < kSide && rt + s < RT; ++s)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            auto& a = acc[rt + s][ct];
            if constexpr (sizeof(T) == 4)
              a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, c[ct].w[kPairA[m]]), __builtin_bit_cast(bf16x8, r[s].w[kPairB[m]]), a, 0, 0, 0);
            else
              a = __builtin_amdgcn_mfma_f64_16x16x4f64(__builtin_bit_cast(f64x2, c[ct].w[m / 2])[m % 2], __builtin_bit_cast(f64x2, r[s].w[m / 2])[m % 2], a, 0, 0, 0);
          }
    }
  }
};

// the first `have` of four neighbours, at most four
template <class T>
__device__ inline void store_some(T* to, const T* v, int have) {
  typedef T Words __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (have >= 4) {
    *(Words*)to = Words{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < have) to[i] = v[i];
  }
}

}  // namespace
}  // namespace cgtp
