// Kernels of the gated feed-forward block, for the translation units of its two types (gated_f32.hip, gated_f64.hip).
//
// With g = x Wg + bg, u = x Wu + bu, out = act(g) u and t = dE/dout:   dg = t u act'(g),  du = t act(g),
//     gx = dg Wg^T + du Wu^T,   gWg = x^T dg,   gWu = x^T du,   gbg = sum dg,   gbu = sum du.
//
// All products run on the matrix cores, 16 x 16 results from 32 terms at a time.  An operand of them is held in parts: lane l has
// the terms 8 q + (0..7) of row (left operand) or column (right operand) l16, where l16 = l % 16 and q = l / 16.
//   fp32   three bf16 numbers whose sum has the 24 bits of the factor; of the nine products of parts the six largest are formed,
//          the others are below 2^-25 of the product.  Sixteen times the rate of the fp32 matrix instruction, so 2.7 times faster
//          than it with six products.  Sums are held in fp32.
//   fp64   the numbers themselves, eight instructions of four terms.
// A lane's four results are rows Num::row(q, 0..3) of column l16.  Two tiles of them are the parts of another operand with 32 terms,
// in the order Num::term of the tiles' rows, so that dg and du go into their products from the registers that they are formed in;
// the other operand stands in the same order.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "act.hpp"
#include "layer.hpp"

namespace cgtp {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef double f64x2 __attribute__((ext_vector_type(2)));
typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kRows = 64;      // rows of x in LDS at a time
constexpr int kMaxIn = 128;    // columns of x that a wave's registers have room for
constexpr int kNonTemporal = 2;
using Buffer = __amdgpu_buffer_rsrc_t;

template <int kUnits>
struct PartsOf {
  u32x4 w[kUnits];
};

template <class T>
struct Num;

// which parts meet: the smallest products first
constexpr int kPairA[6] = {2, 0, 1, 1, 0, 0}, kPairB[6] = {0, 2, 1, 0, 1, 0};

template <>
struct Num<float> {
  static constexpr int kUnits = 3;
  using Parts = PartsOf<3>;
  using Vec = f32x4;
  static __device__ int row(int q, int i) { return 4 * q + i; }
  // two numbers as three pairs of bf16
  static __device__ void split(float a, float b, unsigned* p) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const unsigned h = __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2));
      p[i] = h;
      if (i == 2) break;
      a -= __builtin_bit_cast(float, h << 16);
      b -= __builtin_bit_cast(float, h & 0xffff0000u);
    }
  }
  static __device__ Parts parts(const float* v) {
    unsigned w[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(v[2 * i], v[2 * i + 1], w[i]);
    Parts r;
#pragma unroll
    for (int i = 0; i < 3; ++i) r.w[i] = u32x4{w[0][i], w[1][i], w[2][i], w[3][i]};
    return r;
  }
  // c[i] += a[i] b[i], the chains of sums in turn
  template <int N>
  static __device__ void mma(const Parts* const (&a)[N], const Parts* const (&b)[N], Vec* const (&c)[N]) {
#pragma unroll
    for (int m = 0; m < 6; ++m)
#pragma unroll
      for (int i = 0; i < N; ++i)
        *c[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i]->w[kPairA[m]]), __builtin_bit_cast(bf16x8, b[i]->w[kPairB[m]]), *c[i], 0, 0, 0);
  }
};

template <>
struct Num<double> {
  static constexpr int kUnits = 4;
  using Parts = PartsOf<4>;
  using Vec = f64x4;
  static __device__ int row(int q, int i) { return 4 * i + q; }
  static __device__ Parts parts(const double* v) {
    Parts r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = __builtin_bit_cast(u32x4, f64x2{v[2 * i], v[2 * i + 1]});
    return r;
  }
  template <int N>
  static __device__ void mma(const Parts* const (&a)[N], const Parts* const (&b)[N], Vec* const (&c)[N]) {
#pragma unroll
    for (int m = 0; m < 8; ++m)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f64x2 u = __builtin_bit_cast(f64x2, a[i]->w[m / 2]), v = __builtin_bit_cast(f64x2, b[i]->w[m / 2]);
        *c[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(u[m % 2], v[m % 2], *c[i], 0, 0, 0);
      }
  }
};

// the place among 32 terms of row r (< 32) of two tiles of results: lane quarter q, number 4 (r / 16) + i
template <class T>
__device__ inline int term(int r) {
  const int t = r / 16, h = r % 16;
  return std::is_same<T, float>::value ? h / 4 * 8 + t * 4 + h % 4 : h % 4 * 8 + t * 4 + h / 4;
}

// ---- rows in memory ---------------------------------------------------------------------------------------------------------
//
// Rows go through buffer descriptors of at most kSpan rows: what lies outside reads as zero and is not written, without a branch.  A
// place inside the descriptor's range that is not wanted gets the offset kNowhere, which is behind every range (row strides are
// below 2^22 numbers, rows at most 2^20: 63 * 2^22 * 8 + 2^20 * 8 < 2^31), and with a row's offset added still below 2^32.

constexpr unsigned kNowhere = 0x80000000u;
constexpr int kSpan = 64;

template <class T>
__device__ inline Buffer rows_of(const void* base, int64_t first, int64_t rows, int64_t ld, int64_t width) {
  const int64_t have = rows - first < kSpan ? rows - first : kSpan;
  const T* p = (const T*)base + (have > 0 ? first * ld : 0);
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, have > 0 ? (int)(((have - 1) * ld + width) * sizeof(T)) : 0, 0x00020000);
}

template <class T>
__device__ inline T load1(Buffer B, unsigned at) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(B, at, 0, 0));
  else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b64(B, at, 0, 0));
}

template <int kHow = kNonTemporal, class T>
__device__ inline void store1(T v, Buffer B, unsigned at) {
  if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), B, at, 0, kHow);
  else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), B, at, 0, kHow);
}

// Four neighbouring numbers of the row that begins at offset `row`, from column k, zero beyond its end (kWhole: the row's width is a multiple of four).
// Buffer accesses of several words need the alignment of one, and are held against the range word by word.
template <bool kWhole, class T>
__device__ inline void load4(Buffer B, unsigned row, int k, int K, T* v) {
  constexpr int e = sizeof(T);
  const unsigned at = k < K ? row + k * e : kNowhere;
  if constexpr (e == 4) {
    const f32x4 w = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(B, at, 0, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = w[i];
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f64x2 w = __builtin_bit_cast(f64x2, __builtin_amdgcn_raw_buffer_load_b128(B, at + h * 16, 0, 0));
      v[2 * h] = w[0];
      v[2 * h + 1] = w[1];
    }
  }
  if constexpr (!kWhole)
#pragma unroll
    for (int i = 1; i < 4; ++i) v[i] = k + i < K ? v[i] : T(0);     // else of the next row, or what lies between rows
}

// the same for writing, fp32
template <bool kWhole>
__device__ inline void store4(f32x4 v, Buffer B, unsigned row, int k, int K) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), B, k + 4 <= K ? row + k * 4 : kNowhere, 0, 0);
  if constexpr (!kWhole)
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const float w = v[i];
      __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, w), B, k + 4 > K && k + i < K ? row + (k + i) * 4 : kNowhere, 0, 0);
    }
}

// `rows` rows of W [.., n] from row k on, at most 128 of them (2^30 bytes); an element's offset in it
template <class T>
__device__ inline Buffer matrix_of(const void* W, int64_t k, int64_t rows, int64_t n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)((const T*)W + k * n), 0, rows > 0 ? (int)(rows * n * sizeof(T)) : 0, 0x00020000);
}

// The parts of column c of the rows of W that a descriptor holds, terms k + (0..7).  Rows behind the last are out of its range.
template <class T>
__device__ inline typename Num<T>::Parts column_parts(Buffer W, int64_t n, int64_t c, int k) {
  T v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = load1<T>(W, c < n ? ((unsigned)(k + j) * (unsigned)n + (unsigned)c) * (unsigned)sizeof(T) : kNowhere);
  return Num<T>::parts(v);
}

template <class T>
__device__ inline T bias_of(const void* b, int64_t c, int64_t n) { return b ? ((const T*)b)[c < n ? c : n - 1] : T(0); }

// kR rows of kC columns in LDS, as operands with the columns as terms.  A wave reads 16 bytes of each of 16 rows: they have to lie on different banks
// (256 bytes in all).  fp32 of 64 columns: the 16 bytes of a row change places by an exclusive or with the row's number, in
// which also the lanes that write 4 x 4 blocks (write_both) find different ones; others: rows are padded by 16 bytes.
template <class T, int kR, int kC>
struct Tile;
template <int kR, int kC>
struct Tile<float, kR, kC> {
  static constexpr bool turned = kC == 64;
  __bf16 v[3][kR][turned ? kC : kC + 8];
  static __device__ int at(int r, int c) {
    if constexpr (kC == 64) return c ^ ((r >> 1 ^ r >> 4 << 2) & 7) * 8;
    else return c;
  }
  __device__ PartsOf<3> read(int r, int c) const {
    PartsOf<3> p;
#pragma unroll
    for (int i = 0; i < 3; ++i) p.w[i] = *(const u32x4*)&v[i][r][at(r, c)];
    return p;
  }
  __device__ void write4(int r, int c, const float* x) {
    unsigned lo[3], hi[3];
    Num<float>::split(x[0], x[1], lo);
    Num<float>::split(x[2], x[3], hi);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(u32x2*)&v[p][r][at(r, c)] = u32x2{lo[p], hi[p]};
  }
};
template <int kR, int kC>
struct Tile<double, kR, kC> {
  double v[kR][kC + 2];
  __device__ PartsOf<4> read(int r, int c) const {
    PartsOf<4> p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.w[i] = *(const u32x4*)&v[r][c + 2 * i];
    return p;
  }
  __device__ void write4(int r, int c, const double* x) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *(u32x4*)&v[r][c + 2 * h] = __builtin_bit_cast(u32x4, f64x2{x[2 * h], x[2 * h + 1]});
  }
};

// Operands with the columns of x as terms, kIn (8, 16 or a multiple of 32) of them.  With 8 or 16 the 32 terms of an fp32 instruction hold four or
// two of the six products of parts side by side (a lane's parts are those of the products that its quarter of the terms is for), so
// that two or three instructions do; fp64 leaves out the empty ones.
template <class T, int kIn>
struct In {
  using N = Num<T>;
  static constexpr bool f32 = sizeof(T) == 4, few = kIn < 32;
  static constexpr int KS = few ? 1 : kIn / 32;                                   // operands a row
  static constexpr int kUnits = !few ? N::kUnits : f32 ? (kIn == 8 ? 2 : 3) : kIn / 8;
  static constexpr int kTerms = few && !f32 ? kIn / 4 : 8;                        // a lane's terms
  static constexpr int kGroup = few && f32 ? kIn / 8 : 4;                         // quarters that hold one product's terms
  static constexpr int DT = (kIn + 15) / 16;                                      // tiles of 16 columns of x
  using Parts = PartsOf<kUnits>;
  static __device__ int first(int s, int q) { return few ? q % kGroup * kTerms : s * 32 + q * 8; }
  // number of the product of parts that unit m of quarter q is for
  static __device__ int pair(int m, int q) { return m * (4 / kGroup) + q / kGroup; }
  // of a lane's terms, for the left or right operand
  static __device__ Parts parts(const T* v, int q, bool left) {
    if constexpr (few && f32) {
      const typename N::Parts w = N::parts(v);
      Parts r;
#pragma unroll
      for (int m = 0; m < kUnits; ++m) {
        const int p = pair(m, q);
        // parts of the six products, two bits each, for the left and the right operand; 3: none
        const int part = (left ? 0xff052 : 0xff118) >> (2 * p) & 3;
        r.w[m] = part == 0 ? w.w[0] : part == 1 ? w.w[1] : part == 2 ? w.w[2] : u32x4{0, 0, 0, 0};
      }
      return r;
    } else if constexpr (few) {
      Parts r;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r.w[i] = __builtin_bit_cast(u32x4, f64x2{v[2 * i], v[2 * i + 1]});
      return r;
    } else {
      return N::parts(v);
    }
  }
  // of a row in LDS, for the left operand
  template <int kR>
  static __device__ Parts read(const Tile<T, kR, kIn>& X, int row, int s, int q) {
    if constexpr (few && f32) {
      Parts r;
#pragma unroll
      for (int m = 0; m < kUnits; ++m) {
        const int part = 0xff052 >> (2 * pair(m, q)) & 3;    // 3: any, the right operand has zeros
        r.w[m] = *(const u32x4*)&X.v[part == 3 ? 0 : part][row][first(0, q)];
      }
      return r;
    } else if constexpr (few) {
      Parts r;
#pragma unroll
      for (int i = 0; i < kUnits; ++i) r.w[i] = *(const u32x4*)&X.v[row][first(0, q) + 2 * i];
      return r;
    } else {
      return X.read(row, first(s, q));
    }
  }
  // of column c of W (all its rows in the descriptor), for the right operand
  static __device__ Parts column(Buffer W, int64_t n, int64_t c, int s, int q) {
    T v[8] = {};
#pragma unroll
    for (int j = 0; j < kTerms; ++j) v[j] = load1<T>(W, c < n ? ((unsigned)(first(s, q) + j) * (unsigned)n + (unsigned)c) * (unsigned)sizeof(T) : kNowhere);
    return parts(v, q, false);
  }
  template <int M>
  static __device__ void mma(const Parts* const (&a)[M], const Parts* const (&b)[M], typename N::Vec* const (&c)[M]) {
    if constexpr (!few) {
      N::template mma<M>(a, b, c);
    } else if constexpr (f32) {
#pragma unroll
      for (int m = 0; m < kUnits; ++m)
#pragma unroll
        for (int i = 0; i < M; ++i)
          *c[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i]->w[m]), __builtin_bit_cast(bf16x8, b[i]->w[m]), *c[i], 0, 0, 0);
    } else {
#pragma unroll
      for (int m = 0; m < kTerms; ++m)
#pragma unroll
        for (int i = 0; i < M; ++i)
          *c[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(__builtin_bit_cast(f64x2, a[i]->w[m / 2])[m % 2], __builtin_bit_cast(f64x2, b[i]->w[m / 2])[m % 2], *c[i], 0, 0, 0);
    }
  }
};

// four rows 4 r4 .. of four columns k4 .. of x into X as they are, and into XT by columns, rows in the order of `term`
template <int KC, int KD>
__device__ inline void write_both(Tile<float, kRows, KC>& X, Tile<float, KD, kRows>& XT, int r4, int k4, float (*x)[4]) {
  unsigned row[4][2][3];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    Num<float>::split(x[j][0], x[j][1], row[j][0]);
    Num<float>::split(x[j][2], x[j][3], row[j][1]);
  }
  const int at = r4 / 8 * 32 + term<float>(r4 % 8 * 4);   // four neighbours
#pragma unroll
  for (int p = 0; p < 3; ++p) {
#pragma unroll
    for (int j = 0; j < 4; ++j) *(u32x2*)&X.v[p][r4 * 4 + j][X.at(r4 * 4 + j, k4)] = u32x2{row[j][0][p], row[j][1][p]};
#pragma unroll
    for (int w = 0; w < 2; ++w) {   // halves of the words of two rows
      const unsigned a = row[0][w][p], b = row[1][w][p], c = row[2][w][p], d = row[3][w][p];
      *(u32x2*)&XT.v[p][k4 + 2 * w][XT.at(k4 + 2 * w, at)] = u32x2{__builtin_amdgcn_perm(b, a, 0x05040100), __builtin_amdgcn_perm(d, c, 0x05040100)};
      *(u32x2*)&XT.v[p][k4 + 2 * w + 1][XT.at(k4 + 2 * w + 1, at)] = u32x2{__builtin_amdgcn_perm(b, a, 0x07060302), __builtin_amdgcn_perm(d, c, 0x07060302)};
    }
  }
}
template <int KC, int KD>
__device__ inline void write_both(Tile<double, kRows, KC>& X, Tile<double, KD, kRows>& XT, int r4, int k4, double (*x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    X.write4(r4 * 4 + j, k4, x[j]);
    const int at = r4 / 8 * 32 + term<double>(r4 % 8 * 4 + j);
#pragma unroll
    for (int w = 0; w < 4; ++w) XT.v[k4 + w][at] = x[j][w];
  }
}

// ---- up to 128 columns of x -------------------------------------------------------------------------------------------------

// A wave keeps the parts of its 16 NT columns of Wg and Wu in registers for the whole call and walks over rows, whose parts the
// workgroup puts into LDS once for its four waves.  Lane: columns NT l16 + j.
// 160 710 x 64 x 2176 fp32 450 to 480 us, 1.12 to 1.19 PFLOP/s of bf16 products (library 1.13) beside 3.1 TB/s of writes: the matrix pipe is busy 59 % of the
// cycles, vector instructions issue in 22 %, at the 1.8 GHz that this load leaves (2.5 GHz where memory is the bound); without the stores 376 us, with half of
// the products 327, so that each has its share and none alone is the bound.  With 8 columns of x bound by the writes: 270 us, 5.2 TB/s.  fp64, 30 011 x 64 x 544:
// 107 us, 39 TFLOP/s (library 72); pipe busy 56 %, vector instructions 17 %, 2.3 GHz.  Two waves per SIMD, for the registers; four with half the columns were no faster.  With the
// instruction of 32 x 32 results 482 us for 457; 16 columns a wave 546 for 472.
template <class T, int kIn, int NT, int kAct, bool kWhole>
__global__ void __launch_bounds__(kThreads, (sizeof(T) == 8 && kIn > 64 ? 1 : 2)) k_gated_fwd(GatedArgs a, int col_tiles, int splits) {
  using N = Num<T>;
  using I = In<T, kIn>;
  __shared__ Tile<T, kRows, kIn> X;
  constexpr int KS = I::KS, kQuads = kIn / 4, kAll = kRows * kQuads, kPer = (kAll + kThreads - 1) / kThreads, e = sizeof(T);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, c = ((int64_t)(blockIdx.x % col_tiles) * 4 + wave) * (16 * NT) + l16 * NT;
  const unsigned ldx = (unsigned)a.ld_x * e, ldo = (unsigned)a.ld_out * e;
  const Buffer Wg = matrix_of<T>(a.Wg, 0, K, n), Wu = matrix_of<T>(a.Wu, 0, K, n);
  typename I::Parts wg[KS][NT], wu[KS][NT];
  T bg[NT], bu[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      wg[s][j] = I::column(Wg, n, c + j, s, q);
      wu[s][j] = I::column(Wu, n, c + j, s, q);
    }
    bg[j] = bias_of<T>(a.bg, c + j, n);
    bu[j] = bias_of<T>(a.bu, c + j, n);
  }
  const int64_t blocks = (a.rows + kRows - 1) / kRows;
  T next[kPer][4];
  auto fetch = [&](int64_t b) {
    const Buffer in = rows_of<T>(a.x, b * kRows, a.rows, a.ld_x, K);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = t + i * kThreads < kAll ? t + i * kThreads : kAll - 1;
      load4<kWhole>(in, at / kQuads * ldx, at % kQuads * 4, K, next[i]);
    }
  };
  // a lane's columns: of all, or of the first alone where the row ends behind it
  const unsigned at = c + NT <= n ? (unsigned)c * e + N::row(q, 0) * ldo : kNowhere, at_last = c + 1 == n ? (unsigned)c * e + N::row(q, 0) * ldo : kNowhere;
  // Whole lines are written past the caches, parts of lines are left to them (160 710 x 64 x 2176, a number between the rows 877 and 522 us, none
  // 482 and 495; fp64, 60 000 x 8 x 544, a number between them 146 and 76 us)
  const bool past = ldo % 64 == 0;
  int64_t b = blockIdx.x / col_tiles;
  if (b < blocks) fetch(b);
  for (; b < blocks; b += splits) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int p = t + i * kThreads;
      if (kAll % kThreads == 0 || __builtin_amdgcn_readfirstlane(p) < kAll) X.write4(p / kQuads, p % kQuads * 4, next[i]);   // whole waves
    }
    __syncthreads();
    if (b + splits < blocks) fetch(b + splits);
    const Buffer to = rows_of<T>(a.out, b * kRows, a.rows, a.ld_out, n);
    // the results of a row tile are finished while the products of the next one run
    typename N::Vec g[2][NT], u[2][NT];
    auto products = [&](int rt, typename N::Vec* gt, typename N::Vec* ut) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          gt[j][i] = bg[j];
          ut[j][i] = bu[j];
        }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const typename I::Parts xa = I::read(X, rt * 16 + l16, s, q);
        if constexpr (NT == 2) I::template mma<4>({&xa, &xa, &xa, &xa}, {&wg[s][0], &wu[s][0], &wg[s][1], &wu[s][1]}, {&gt[0], &ut[0], &gt[1], &ut[1]});
        else I::template mma<2>({&xa, &xa}, {&wg[s][0], &wu[s][0]}, {&gt[0], &ut[0]});
      }
    };
    auto finish = [&](int rt, const typename N::Vec* gt, const typename N::Vec* ut) {
      T v[4][NT];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) v[i][j] = act_only<kAct>(T(gt[j][i])) * T(ut[j][i]);
      auto write = [&](auto how) {
        constexpr int kHow = decltype(how)::value;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned row = (rt * 16 + N::row(0, i)) * ldo;
          if constexpr (NT == 2) {
            __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{v[i][0], v[i][1]}), to, at + row, 0, kHow);
            if constexpr (!kWhole) store1<kHow>(v[i][0], to, at_last + row);
          } else {
            store1<kHow>(v[i][0], to, at + row);
          }
        }
      };
      if (past) write(std::integral_constant<int, kNonTemporal>());
      else write(std::integral_constant<int, 0>());
    };
#pragma unroll
    for (int rt = 0; rt < kRows / 16; ++rt) {
      products(rt, g[rt & 1], u[rt & 1]);
      if (rt > 0) finish(rt - 1, g[~rt & 1], u[~rt & 1]);
    }
    finish(kRows / 16 - 1, g[1], u[1]);
  }
}

// The gradients: two kernels, each of which forms g and u again.  That is a third more products than with dg and du kept in memory,
// but those are twice the size of gout, written once and read twice.  (One kernel that forms both gradients of a share of the columns would need
// neither; its partial sums of gx and what it has to pass through LDS have not been tried.)

// gWg, gWu, gbg, gbu of 16 columns a wave, over the row blocks of a split; partial sums [split][Wg; bg; Wu; bu]
// Products and the vector instructions between them (activation, cuts into parts): 160 710 x 64 x 2176 fp32 1.08 ms under the profiler (with gx 1.89 to 1.94 ms in
// a run of passes, of which 0.3 would do for the bytes), matrix pipe busy 51 % of the cycles, vector instructions 33 %, 1.86 GHz.  Activations of one tile beside the
// products of another: within 1 %.  fp64, 30 011 x 64 x 544: 200 us, pipe busy 61 %, vector instructions 13 %.
// The biases' sums are held like the weights' in the type itself: 16 rows a lane and block one after another, the quarters of the rows, the splits in eight
// chains.
constexpr int kGwWaves = 4;
// whether a wave needs the registers of two: fp64, and from 65 columns of x on (20 011 x 128 x 301, forward and backward 214 us, with two waves that
// keep what does not fit in private memory 230)
template <class T, int kIn>
constexpr bool kGwAlone = kIn > (sizeof(T) == 8 ? 32 : 64);

template <class T, int kIn, int kAct, bool kWhole>
__global__ void __launch_bounds__((kGwWaves * 64), (kGwAlone<T, kIn> ? 1 : 2)) k_gated_gw(GatedArgs a, int col_tiles, int splits, T* part) {
  using N = Num<T>;
  using I = In<T, kIn>;
  constexpr int KS = I::KS, DT = I::DT, e = sizeof(T);
  __shared__ Tile<T, kRows, kIn> X;
  __shared__ Tile<T, DT * 16, kRows> XT;      // with 8 columns of x the other half holds anything: sums that are not kept
  // blocks of 4 rows x 4 columns of x; lanes without one of their own repeat the last, waves without any do nothing
  constexpr int kQuads = kIn / 4, kBlocks = kRows / 4 * kQuads, kThr = kGwWaves * 64, kPer = (kBlocks + kThr - 1) / kThr;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, c = ((int64_t)(blockIdx.x % col_tiles) * kGwWaves + wave) * 16 + l16;
  const unsigned ldx = (unsigned)a.ld_x * e, ldo = (unsigned)a.ld_gout * e;
  const Buffer Wg = matrix_of<T>(a.Wg, 0, K, n), Wu = matrix_of<T>(a.Wu, 0, K, n);
  typename I::Parts wg[KS], wu[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    wg[s] = I::column(Wg, n, c, s, q);
    wu[s] = I::column(Wu, n, c, s, q);
  }
  const T bg = bias_of<T>(a.bg, c, n), bu = bias_of<T>(a.bu, c, n);
  const int64_t blocks = (a.rows + kRows - 1) / kRows;
  // four by four blocks to 16 neighbouring threads: their 8 bytes fall on different banks in X and in XT
  auto block = [&](int i, int& r4, int& k4) {
    const int p = t + i * kThr < kBlocks ? t + i * kThr : kBlocks - 1;
    constexpr int kSide = kQuads < 4 ? kQuads : 4;      // quads side by side
    const int u = p / (4 * kSide);
    r4 = (p & 1) | (u & 1) << 1 | (p >> 1 & 1) << 2 | (u >> 1 & 1) << 3;
    k4 = (p / 4 % kSide + u / 4 * 4) * 4;
  };
  T next[kPer][4][4];
  auto fetch = [&](int64_t b) {
    const Buffer in = rows_of<T>(a.x, b * kRows, a.rows, a.ld_x, K);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      int r4, k4;
      block(i, r4, k4);
#pragma unroll
      for (int j = 0; j < 4; ++j) load4<kWhole>(in, (r4 * 4 + j) * ldx, k4, K, next[i][j]);
    }
  };
  const unsigned at = c < n ? (unsigned)c * e + N::row(q, 0) * ldo : kNowhere;
  typename N::Vec sg[DT] = {}, su[DT] = {};
  T sbg = 0, sbu = 0;
  int64_t b = blockIdx.x / col_tiles;
  if (b < blocks) fetch(b);
  for (; b < blocks; b += splits) {
    const Buffer go = rows_of<T>(a.gout, b * kRows, a.rows, a.ld_gout, n);
    T tg[8];   // of gout, 32 rows at a time
    auto fetch_gout = [&](int half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) tg[i] = load1<T>(go, at + (half * 32 + i / 4 * 16 + N::row(0, i % 4)) * ldo);
    };
    fetch_gout(0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (kBlocks % kThr != 0 && __builtin_amdgcn_readfirstlane(t + i * kThr) >= kBlocks) break;
      int r4, k4;
      block(i, r4, k4);
      write_both(X, XT, r4, k4, next[i]);
    }
    __syncthreads();
    if (b + splits < blocks) fetch(b + splits);
#pragma unroll
    for (int half = 0; half < kRows / 32; ++half) {
      T dg[8], du[8];
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        typename N::Vec g, u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          g[i] = bg;
          u[i] = bu;
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const typename I::Parts xa = I::read(X, half * 32 + rt * 16 + l16, s, q);
          I::template mma<2>({&xa, &xa}, {&wg[s], &wu[s]}, {&g, &u});
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T o = tg[rt * 4 + i];   // zero behind the last row
          T v, d;
          act_both<kAct>(T(g[i]), v, d);
          dg[rt * 4 + i] = o * T(u[i]) * d;
          du[rt * 4 + i] = o * v;
          sbg += dg[rt * 4 + i];
          sbu += du[rt * 4 + i];
        }
      }
      if (half + 1 < kRows / 32) fetch_gout(half + 1);
      const typename N::Parts pg = N::parts(dg), pu = N::parts(du);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const typename N::Parts xt = XT.read(d * 16 + l16, half * 32 + q * 8);
        N::template mma<2>({&xt, &xt}, {&pg, &pu}, {&sg[d], &su[d]});
      }
    }
  }
  // the biases' sums of the four quarters of the rows
  sbg += __shfl_xor(sbg, 16);
  sbg += __shfl_xor(sbg, 32);
  sbu += __shfl_xor(sbu, 16);
  sbu += __shfl_xor(sbu, 32);
  if (c >= n) return;
  T* to = part + (int64_t)(blockIdx.x / col_tiles) * 2 * (K + 1) * n + c;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = d * 16 + N::row(q, i);
      if (k < K) {
        to[(int64_t)k * n] = sg[d][i];
        to[(int64_t)(K + 1 + k) * n] = su[d][i];
      }
    }
  if (q == 0) {
    to[(int64_t)K * n] = sbg;
    to[(int64_t)(2 * K + 1) * n] = sbu;
  }
}

// adds up the splits, in their order: the weights' and biases' gradients, and gx where its sums are split (gx_splits > 1).  4 to 6 us, eight loads in
// flight a thread for the latency of few rows.
template <class T>
__global__ void __launch_bounds__(kThreads) k_gated_sums(GatedArgs a, const T* __restrict__ part, int splits, const T* __restrict__ gx_part, int gx_splits) {
  const int64_t K = a.d_in, n = a.d_out, size = 2 * (K + 1) * n, gx_size = gx_splits > 1 ? a.rows * K : 0;
  auto total = [](const T* p, int m, int64_t of, int64_t i) {
    T v[8] = {};
    int s = 0;
    for (; s + 8 <= m; s += 8)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += p[(s + j) * of + i];
    for (; s < m; ++s) v[0] += p[s * of + i];
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  };
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < size + gx_size; at += (int64_t)gridDim.x * kThreads) {
    if (at < size) {
      const T v = total(part, splits, size, at);
      const int64_t row = at / n, c = at % n;
      if (row < K) ((T*)a.gWg)[at] = v;
      else if (row == K) { if (a.gbg) ((T*)a.gbg)[c] = v; }
      else if (row <= 2 * K) ((T*)a.gWu)[at - (K + 1) * n] = v;
      else if (a.gbu) ((T*)a.gbu)[c] = v;
    } else {
      const int64_t i = at - size;
      ((T*)a.gx)[i / K * a.ld_gx + i % K] = total(gx_part, gx_splits, gx_size, i);
    }
  }
}

// The operands of W that gx needs for 32 of its columns, in units of 16 bytes a lane.  First 4 KS for g and u: (g, u) x tile x s, lane:
// column 16 tile + l16, its terms of d_in; then 2 DT for gx: (g, u) x d, lane: column 16 d + l16 of x, the 32 columns of W in the order of Num::term.
template <class T, int kIn>
struct Operands {
  using N = Num<T>;
  using I = In<T, kIn>;
  static constexpr int kIns = 4 * I::KS, kOuts = 2 * I::DT, kOps = kIns + kOuts, kUnits = kIns * I::kUnits + kOuts * N::kUnits;
  // operand `op` (the wave's) of columns 32 step .., put(unit, value)
  template <class F>
  static __device__ void make(const GatedArgs& a, int64_t step, int op, F put) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, q = lane >> 4, K = (int)a.d_in;
    const int64_t n = a.d_out;
    const bool in = op < kIns;
    const Buffer W = matrix_of<T>((in ? op / (2 * I::KS) : (op - kIns) / I::DT) ? a.Wu : a.Wg, 0, K, n);
    T v[8] = {};
    if (in) {
      const int64_t c = step * 32 + op / I::KS % 2 * 16 + l16;
#pragma unroll
      for (int j = 0; j < I::kTerms; ++j) v[j] = load1<T>(W, c < n ? ((unsigned)(I::first(op % I::KS, q) + j) * (unsigned)n + (unsigned)c) * (unsigned)sizeof(T) : kNowhere);
      const typename I::Parts p = I::parts(v, q, true);
#pragma unroll
      for (int i = 0; i < I::kUnits; ++i) put(op * I::kUnits + i, p.w[i]);
    } else {
      const int k = (op - kIns) % I::DT * 16 + l16;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t c = step * 32 + j / 4 * 16 + N::row(q, j % 4);
        v[j] = load1<T>(W, k < K && c < n ? ((unsigned)k * (unsigned)n + (unsigned)c) * (unsigned)sizeof(T) : kNowhere);
      }
      const typename N::Parts p = N::parts(v);
#pragma unroll
      for (int i = 0; i < N::kUnits; ++i) put(kIns * I::kUnits + (op - kIns) * N::kUnits + i, p.w[i]);
    }
  }
};

// all of them, [32 columns of W][unit][lane]
template <class T, int kIn>
__global__ void __launch_bounds__(kThreads) k_gated_operands(GatedArgs a, u32x4* to) {
  using O = Operands<T, kIn>;
  const int64_t steps = (a.d_out + 31) / 32, e = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (e >= steps * O::kOps) return;
  const int64_t step = e / O::kOps;
  O::make(a, step, (int)(e % O::kOps), [&](int unit, u32x4 v) { to[(step * O::kUnits + unit) * 64 + (threadIdx.x & 63)] = v; });
}

// gx of 16 R rows a wave: the operands of 32 columns of W at a time in LDS for the waves of a workgroup, the columns of a split one after
// another.  160 710 x 64 x 2176 fp32 1.04 ms under the profiler, matrix pipe busy 51 % of the cycles, vector instructions 26 %, 1.84 GHz; fp64, 30 011 x 64 x 544, 223 us,
// pipe busy 51 %, vector instructions 13 %.  20 011 x 128 x 301 fp32 79 us: 157 workgroups on 256 units, pipe busy 20 %, vector instructions 22 %, the rest waits.
// Four waves, so that two workgroups of a compute unit are in different phases (160 710 x 64 x 2176, all of backward 2.01 ms before the
// tiles were without bank conflicts, with eight 2.12); eight in fp32 of more than 64 columns of x, whose operands fill the LDS for one workgroup (50 000 x 128 x 2176 backward 1.40 ms; 1.46 when four took 1.91).  More than one split: partial sums [split][rows][d_in] in part.  ops NULL: the
// workgroups form the operands themselves, which saves a launch where the rows are few.
template <class T, int kIn>
constexpr int kGxWaves = kIn > 64 && sizeof(T) == 4 ? 8 : 4;
template <class T, int kIn>
constexpr int kGxTiles = kIn > 64 || sizeof(T) == 8 ? 1 : 2;   // 2 would not fit the registers

template <class T, int kIn, int kAct, bool kWhole>
__global__ void __launch_bounds__((kGxWaves<T, kIn> * 64), (kIn > 64 && sizeof(T) == 8 ? 1 : 2)) k_gated_gx(GatedArgs a, const u32x4* __restrict__ ops, int splits, T* part) {
  using N = Num<T>;
  using I = In<T, kIn>;
  using O = Operands<T, kIn>;
  constexpr int R = kGxTiles<T, kIn>, KS = I::KS, DT = I::DT, kWaves = kGxWaves<T, kIn>, kPer = (O::kUnits + kWaves - 1) / kWaves, e = sizeof(T);
  __shared__ u32x4 W[O::kUnits][64];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, q = lane >> 4;
  const int K = (int)a.d_in;
  const int64_t n = a.d_out, steps = (n + 31) / 32, first = (int64_t)(blockIdx.x / splits) * (kWaves * R * 16) + wave * R * 16;
  const int64_t from = steps * (blockIdx.x % splits) / splits, end = steps * (blockIdx.x % splits + 1) / splits;
  const unsigned ldx = (unsigned)a.ld_x * e, ldo = (unsigned)a.ld_gout * e;
  auto operand_in = [&](int op) {
    typename I::Parts p;
#pragma unroll
    for (int i = 0; i < I::kUnits; ++i) p.w[i] = W[op * I::kUnits + i][lane];
    return p;
  };
  auto operand_out = [&](int op) {
    typename N::Parts p;
#pragma unroll
    for (int i = 0; i < N::kUnits; ++i) p.w[i] = W[O::kIns * I::kUnits + op * N::kUnits + i][lane];
    return p;
  };
  // x of rows 16 r + l16
  typename I::Parts xb[R][KS];
  {
    const Buffer in = rows_of<T>(a.x, first, a.rows, a.ld_x, K);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        T v[8] = {};
        const int k = I::first(s, q);
        if constexpr (I::kTerms >= 4) {
#pragma unroll
          for (int i = 0; i < I::kTerms; i += 4) load4<kWhole>(in, (r * 16 + l16) * ldx, k + i, K, v + i);
        } else {
#pragma unroll
          for (int i = 0; i < I::kTerms; ++i) v[i] = load1<T>(in, k + i < K ? (r * 16 + l16) * ldx + (k + i) * e : kNowhere);
        }
        xb[r][s] = I::parts(v, q, false);
      }
  }
  const Buffer go = rows_of<T>(a.gout, first, a.rows, a.ld_gout, n);
  u32x4 next[kPer];
  auto fetch = [&](int64_t step) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (O::kUnits % kWaves == 0 || wave + i * kWaves < O::kUnits) next[i] = ops[(step * O::kUnits + wave + i * kWaves) * 64 + lane];
  };
  typename N::Vec acc[R][DT] = {};
  if (ops) fetch(from);
  for (int64_t step = from; step < end; ++step) {
    T tg[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const int c = (int)(step * 32 + tile * 16);
        const unsigned row = (r * 16 + l16) * ldo;
        if constexpr (e == 4) {
          load4<kWhole>(go, row, c + q * 4, (int)n, tg[r] + tile * 4);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) tg[r][tile * 4 + i] = load1<T>(go, c + N::row(q, i) < n ? row + (c + N::row(q, i)) * e : kNowhere);
        }
      }
    __syncthreads();
    if (ops) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (O::kUnits % kWaves == 0 || wave + i * kWaves < O::kUnits) W[wave + i * kWaves][lane] = next[i];
    } else {
      for (int op = wave; op < O::kOps; op += kWaves) O::make(a, step, op, [&](int unit, u32x4 v) { W[unit][lane] = v; });
    }
    __syncthreads();
    if (ops && step + 1 < end) fetch(step + 1);
    T dg[R][8], du[R][8];
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      typename N::Vec g[R], u[R], bg = {0, 0, 0, 0}, bu = {0, 0, 0, 0};
      if (a.bg) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bg[i] = bias_of<T>(a.bg, step * 32 + tile * 16 + N::row(q, i), n);
          bu[i] = bias_of<T>(a.bu, step * 32 + tile * 16 + N::row(q, i), n);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        g[r] = bg;
        u[r] = bu;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const typename I::Parts wg = operand_in(tile * KS + s), wu = operand_in((2 + tile) * KS + s);
        if constexpr (R == 2) I::template mma<4>({&wg, &wu, &wg, &wu}, {&xb[0][s], &xb[0][s], &xb[1][s], &xb[1][s]}, {&g[0], &u[0], &g[1], &u[1]});
        else I::template mma<2>({&wg, &wu}, {&xb[0][s], &xb[0][s]}, {&g[0], &u[0]});
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T o = tg[r][tile * 4 + i];     // zero outside
          T v, d;
          act_both<kAct>(T(g[r][i]), v, d);
          dg[r][tile * 4 + i] = o * T(u[r][i]) * d;
          du[r][tile * 4 + i] = o * v;
        }
    }
    typename N::Parts pg[R], pu[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      pg[r] = N::parts(dg[r]);
      pu[r] = N::parts(du[r]);
    }
    if constexpr (DT == 1) {
      const typename N::Parts w = operand_out(0), v = operand_out(1);
      if constexpr (R == 2) {
        N::template mma<2>({&w, &w}, {&pg[0], &pg[1]}, {&acc[0][0], &acc[1][0]});
        N::template mma<2>({&v, &v}, {&pu[0], &pu[1]}, {&acc[0][0], &acc[1][0]});
      } else {
        N::template mma<1>({&w}, {&pg[0]}, {&acc[0][0]});
        N::template mma<1>({&v}, {&pu[0]}, {&acc[0][0]});
      }
    } else {
#pragma unroll
      for (int d = 0; d + 1 < DT; d += 2) {   // two column tiles in turn
        const typename N::Parts w0 = operand_out(d), w1 = operand_out(d + 1);
        if constexpr (R == 2) N::template mma<4>({&w0, &w1, &w0, &w1}, {&pg[0], &pg[0], &pg[1], &pg[1]}, {&acc[0][d], &acc[0][d + 1], &acc[1][d], &acc[1][d + 1]});
        else N::template mma<2>({&w0, &w1}, {&pg[0], &pg[0]}, {&acc[0][d], &acc[0][d + 1]});
        const typename N::Parts v0 = operand_out(DT + d), v1 = operand_out(DT + d + 1);
        if constexpr (R == 2) N::template mma<4>({&v0, &v1, &v0, &v1}, {&pu[0], &pu[0], &pu[1], &pu[1]}, {&acc[0][d], &acc[0][d + 1], &acc[1][d], &acc[1][d + 1]});
        else N::template mma<2>({&v0, &v1}, {&pu[0], &pu[0]}, {&acc[0][d], &acc[0][d + 1]});
      }
    }
  }
  const unsigned ldg = (unsigned)(splits > 1 ? K : a.ld_gx) * e;
  const Buffer to = splits > 1 ? rows_of<T>(part + (int64_t)(blockIdx.x % splits) * a.rows * K, first, a.rows, K, K) : rows_of<T>(a.gx, first, a.rows, a.ld_gx, K);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const unsigned row = (r * 16 + l16) * ldg;
      if constexpr (e == 4) {
        store4<kWhole>(acc[r][d], to, row, d * 16 + q * 4, K);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = d * 16 + N::row(q, i);
          const T v = acc[r][d][i];   // (a bit cast of the element itself takes the first one)
          store1(v, to, k < K ? row + k * e : kNowhere);
        }
      }
    }
}

// ---- more columns of x ----------------------------------------------------------------------------------------------------------
//
// 128 rows x 64 columns of results a workgroup, 16 columns a wave, the terms 32 at a time: the rows' parts in LDS, the columns' parts formed
// by each wave from memory.  The gradients go through dg and du in the workspace, a piece of the rows at a time, since W
// no longer stays in registers for products that would form g and u again.  Forward and backward of
// 30 000 x 200 x 1000 fp32 1.17 ms (82 TFLOP/s of fp32 products; six bf16 products each at the library's rate would take 0.51), 20 000 x 200 x 500 fp64
// 0.90 ms (35 TFLOP/s, library 72).  Shares of the cycles, matrix pipe and vector instructions: forward 55 and 40 % (each wave forms the parts of its columns
// of W), of a piece dg and du 29 and 21 %, gx 13 and 13 % (one workgroup a unit, bound by its loads), the weights' gradients 24 and 40 %.  One row of 256 to 2176 numbers: 60 us, five launches of few workgroups.

template <class T>
constexpr int kManyRows = sizeof(T) == 4 ? 128 : 64;   // rows of a workgroup, for the registers of their sums
constexpr int64_t kPiece = 8192;   // rows whose dg and du stand in the workspace at a time

// rows first .. of A (ld numbers apart, `width` of them terms), 32 terms from k0 on; each thread copies four at a time
template <class T>
struct ManyRows {
  static constexpr int kPer = kManyRows<T> / 32;
  Tile<T, kManyRows<T>, 32> X;
  __device__ void fetch(const T* A, int64_t first, int64_t rows, int64_t ld, int64_t width, int64_t k0, T (*v)[4]) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const Buffer in = rows_of<T>(A, first + i * 32, rows, ld, width);
      load4<false>(in, threadIdx.x / 8 * (unsigned)(ld * sizeof(T)), (int)k0 + threadIdx.x % 8 * 4, (int)width, v[i]);
    }
  }
  __device__ void put(T (*v)[4]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) X.write4(i * 32 + threadIdx.x / 8, threadIdx.x % 8 * 4, v[i]);
  }
};

// out (kBack: dg and du, [rows][d_out] each) of `rows` rows from row0 on
template <class T, int kAct, bool kBack>
__global__ void __launch_bounds__(kThreads, 2) k_gated_many(GatedArgs a, int64_t row0, int64_t rows, T* dg, T* du) {
  using N = Num<T>;
  constexpr int kTiles = kManyRows<T> / 16, e = sizeof(T);
  __shared__ ManyRows<T> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t n = a.d_out, K = a.d_in, tiles = (n + 63) / 64, first = blockIdx.x / tiles * kManyRows<T>, c = blockIdx.x % tiles * 64 + wave * 16 + l16;
  const T* x = (const T*)a.x + row0 * a.ld_x;
  typename N::Vec g[kTiles] = {}, u[kTiles] = {};
  T next[ManyRows<T>::kPer][4];
  S.fetch(x, first, rows, a.ld_x, K, 0, next);
  for (int64_t k0 = 0; k0 < K; k0 += 32) {
    const int64_t have = K - k0 < 32 ? K - k0 : 32;
    const typename N::Parts wg = column_parts<T>(matrix_of<T>(a.Wg, k0, have, n), n, c, q * 8), wu = column_parts<T>(matrix_of<T>(a.Wu, k0, have, n), n, c, q * 8);
    __syncthreads();
    S.put(next);
    __syncthreads();
    if (k0 + 32 < K) S.fetch(x, first, rows, a.ld_x, K, k0 + 32, next);
#pragma unroll
    for (int rt = 0; rt < kTiles; ++rt) {
      const typename N::Parts xa = S.X.read(rt * 16 + l16, q * 8);
      N::template mma<2>({&xa, &xa}, {&wg, &wu}, {&g[rt], &u[rt]});
    }
  }
  const T bg = bias_of<T>(a.bg, c, n), bu = bias_of<T>(a.bu, c, n);
#pragma unroll
  for (int h = 0; h < kTiles; h += 4) {   // 64 rows
    const int64_t at = first + h * 16;
    const Buffer go = rows_of<T>(kBack ? (const T*)a.gout + row0 * a.ld_gout : nullptr, at, kBack ? rows : 0, a.ld_gout, n);
    const Buffer to = kBack ? rows_of<T>(dg, at, rows, n, n) : rows_of<T>((T*)a.out + row0 * a.ld_out, at, rows, a.ld_out, n);
    const Buffer to_u = rows_of<T>(du, at, kBack ? rows : 0, n, n);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned row = rt * 16 + N::row(q, i), out = (unsigned)(kBack ? n : a.ld_out) * e;
        const T gv = g[h + rt][i] + bg, uv = u[h + rt][i] + bu;
        T v, d;
        act_both<kAct>(gv, v, d);
        if constexpr (kBack) {
          const T o = load1<T>(go, c < n ? row * (unsigned)(a.ld_gout * e) + (unsigned)c * e : kNowhere);
          store1(o * uv * d, to, c < n ? row * out + (unsigned)c * e : kNowhere);
          store1(o * v, to_u, c < n ? row * out + (unsigned)c * e : kNowhere);
        } else {
          store1(v * uv, to, c < n ? row * out + (unsigned)c * e : kNowhere);
        }
      }
  }
}

// gx = dg Wg^T + du Wu^T of a piece of rows: 64 columns of x a workgroup.  More than one split (of the columns of Wg, then Wu): partial sums
// [split][rows][d_in] in part.
template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_gated_many_gx(GatedArgs a, int64_t row0, int64_t rows, const T* dg, const T* du, int splits, T* part) {
  using N = Num<T>;
  constexpr int kTiles = kManyRows<T> / 16, e = sizeof(T);
  __shared__ ManyRows<T> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t n = a.d_out, K = a.d_in, tiles = (K + 63) / 64, block = blockIdx.x / splits, first = block / tiles * kManyRows<T>, k0 = block % tiles * 64;
  const int k = wave * 16 + l16;      // behind k0; rows of W beyond the last are out of the descriptors' range
  const Buffer Wg = matrix_of<T>(a.Wg, k0, K - k0 < 64 ? K - k0 : 64, n), Wu = matrix_of<T>(a.Wu, k0, K - k0 < 64 ? K - k0 : 64, n);
  const int64_t steps = (n + 31) / 32, split = blockIdx.x % splits, from = 2 * steps * split / splits, end = 2 * steps * (split + 1) / splits;
  typename N::Vec acc[kTiles] = {};
  T next[ManyRows<T>::kPer][4];
  S.fetch(from < steps ? dg : du, first, rows, n, n, from % steps * 32, next);
  for (int64_t s = from; s < end; ++s) {
    T v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned c = (unsigned)(s % steps * 32) + q * 8 + j, at = c < n ? ((unsigned)k * (unsigned)n + c) * e : kNowhere;
      v[j] = s < steps ? load1<T>(Wg, at) : load1<T>(Wu, at);
    }
    const typename N::Parts w = N::parts(v);
    __syncthreads();
    S.put(next);
    __syncthreads();
    if (s + 1 < end) S.fetch(s + 1 < steps ? dg : du, first, rows, n, n, (s + 1) % steps * 32, next);
#pragma unroll
    for (int rt = 0; rt < kTiles; rt += 2) {
      const typename N::Parts x0 = S.X.read(rt * 16 + l16, q * 8), x1 = S.X.read(rt * 16 + 16 + l16, q * 8);
      N::template mma<2>({&x0, &x1}, {&w, &w}, {&acc[rt], &acc[rt + 1]});
    }
  }
#pragma unroll
  for (int h = 0; h < kTiles; h += 4) {
    const int64_t ld = splits > 1 ? K : a.ld_gx;
    const Buffer to = rows_of<T>(splits > 1 ? part + split * rows * K : (T*)a.gx + row0 * a.ld_gx, first + h * 16, rows, ld, K);
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const T v = acc[h + rt][i];
        store1(v, to, k0 + k < K ? (rt * 16 + N::row(q, i)) * (unsigned)(ld * e) + (unsigned)(k0 + k) * e : kNowhere);
      }
  }
}

// the weights' gradients of a piece of rows: 64 columns of x by 32 C of W a workgroup, 32 by 16 C a wave, over the 32-row steps of a split;
// partial sums as k_gated_gw leaves them, to which the pieces after the first add
template <class T>
constexpr int kManyCols = sizeof(T) == 4 ? 2 : 1;   // C

template <class T>
__global__ void __launch_bounds__(kThreads, 2) k_gated_many_gw(GatedArgs a, int64_t row0, int64_t rows, const T* dg, const T* du, int splits, T* part, int add) {
  using N = Num<T>;
  constexpr int C = kManyCols<T>, e = sizeof(T);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q = lane >> 4;
  const int64_t n = a.d_out, K = a.d_in, ct = (n + 32 * C - 1) / (32 * C), kt = (K + 63) / 64;
  const int64_t c0 = blockIdx.x % ct * (32 * C) + wave % 2 * (16 * C), k0 = blockIdx.x / ct % kt * 64 + wave / 2 * 32, split = blockIdx.x / (ct * kt);
  const T* x = (const T*)a.x + row0 * a.ld_x;
  typename N::Vec sg[2][C] = {}, su[2][C] = {};
  T bg[C] = {}, bu[C] = {};
  const int64_t steps = (rows + 31) / 32;
  for (int64_t s = split; s < steps; s += splits) {
    const Buffer in = rows_of<T>(x, s * 32, rows, a.ld_x, K), in_g = rows_of<T>(dg, s * 32, rows, n, n), in_u = rows_of<T>(du, s * 32, rows, n, n);
    typename N::Parts xt[2], pg[C], pu[C];
    T v[8];
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const int64_t k = k0 + d * 16 + l16;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = load1<T>(in, k < K ? (q * 8 + j) * (unsigned)(a.ld_x * e) + (unsigned)k * e : kNowhere);
      xt[d] = N::parts(v);
    }
#pragma unroll
    for (int h = 0; h < C; ++h) {
      const int64_t c = c0 + h * 16 + l16;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = load1<T>(in_g, c < n ? (q * 8 + j) * (unsigned)(n * e) + (unsigned)c * e : kNowhere);
        bg[h] += v[j];
      }
      pg[h] = N::parts(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = load1<T>(in_u, c < n ? (q * 8 + j) * (unsigned)(n * e) + (unsigned)c * e : kNowhere);
        bu[h] += v[j];
      }
      pu[h] = N::parts(v);
    }
#pragma unroll
    for (int h = 0; h < C; ++h)
      N::template mma<4>({&xt[0], &xt[0], &xt[1], &xt[1]}, {&pg[h], &pu[h], &pg[h], &pu[h]}, {&sg[0][h], &su[0][h], &sg[1][h], &su[1][h]});
  }
  T* to = part + split * 2 * (K + 1) * n;
#pragma unroll
  for (int h = 0; h < C; ++h) {
    const int64_t c = c0 + h * 16 + l16;
    bg[h] += __shfl_xor(bg[h], 16);
    bg[h] += __shfl_xor(bg[h], 32);
    bu[h] += __shfl_xor(bu[h], 16);
    bu[h] += __shfl_xor(bu[h], 32);
    if (c >= n) continue;
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t k = k0 + d * 16 + N::row(q, i);
        if (k >= K) continue;
        T *g = to + k * n + c, *u = to + (K + 1 + k) * n + c;
        *g = add ? *g + sg[d][h][i] : sg[d][h][i];
        *u = add ? *u + su[d][h][i] : su[d][h][i];
      }
    if (k0 == 0 && q == 0) {
      T *g = to + K * n + c, *u = to + (2 * K + 1) * n + c;
      *g = add ? *g + bg[h] : bg[h];
      *u = add ? *u + bu[h] : bu[h];
    }
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------------------

constexpr int kMostUnits = 256;   // compute units that the workspace is sized for
constexpr int64_t kMostGroups = (int64_t)1 << 22;   // workgroups of a launch: 2^32 threads are too many

// f(kIn) for the least of 8, 16, 32, 64, 96, 128 columns that holds K
template <class F>
auto with_columns(int64_t K, F f) {
  if (K <= 8) return f(std::integral_constant<int, 8>());
  if (K <= 16) return f(std::integral_constant<int, 16>());
  if (K <= 32) return f(std::integral_constant<int, 32>());
  if (K <= 64) return f(std::integral_constant<int, 64>());
  if (K <= 96) return f(std::integral_constant<int, 96>());
  return f(std::integral_constant<int, 128>());
}

// workgroups of four waves that a compute unit has registers for
template <class T, int kIn>
constexpr int kGroups = kIn <= 32 && sizeof(T) == 4 ? 3 : 2;

// How the rows are split for the weights' gradients: as many workgroups as stay on the chip, but partial sums of at most 64 MiB.
template <class T>
int64_t gw_splits(int64_t rows, int64_t K, int64_t n, int cus) {
  const int groups = with_columns(K, [](auto in) { return kGwAlone<T, decltype(in)::value> ? 1 : kGroups<T, decltype(in)::value>; });
  const int64_t wide = 16 * kGwWaves, cols = (n + wide - 1) / wide, blocks = (rows + kRows - 1) / kRows;
  const int64_t most = std::max<int64_t>(1, ((int64_t)64 << 20) / (2 * (K + 1) * n * (int64_t)sizeof(T)));
  return std::max<int64_t>(1, std::min({blocks, groups * cus / cols, most}));
}

// rows of a workgroup of k_gated_gx
template <class T>
int64_t gx_rows(int64_t K) { return with_columns(K, [](auto in) { return kGxWaves<T, decltype(in)::value> * kGxTiles<T, decltype(in)::value> * 16; }); }

// How the columns of W are split for gx.  Few rows: so that every compute unit has work.  More: where the units' shares are uneven, a workgroup more on some
// than on others (40 000 x 128 x 2176, 313 workgroups on 256 units, gradients 1260 us, in three splits 1064; fp64, 20 000 x 64 x 544, 324 and 281).
// That has to save a quarter of the time, or the partial sums cost more than it gives (20 011 x 128 x 301, forward and backward 194 us with loads of
// single words, in three splits, which save a fifth, 214).
template <class T>
int64_t gx_splits(int64_t rows, int64_t K, int64_t n) {
  const int64_t blocks = (rows + gx_rows<T>(K) - 1) / gx_rows<T>(K), room = (K > 64 ? 1 : 2) * kMostUnits, steps = (n + 31) / 32;
  if (blocks <= room / 2) return std::min(steps, room / blocks);
  auto time = [&](int64_t s) { return (blocks * s + kMostUnits - 1) / kMostUnits * ((steps + s - 1) / s); };
  int64_t best = 1;
  for (int64_t s = 2; s <= std::min<int64_t>(steps, 4); ++s)
    if (time(s) < time(best) && 4 * time(s) <= 3 * time(1)) best = s;
  return best;
}
constexpr int64_t kFewBlocks = 4;   // up to this many blocks of rows form the operands of W themselves

template <class T>
size_t operand_bytes(int64_t K, int64_t n) {
  return (size_t)((n + 31) / 32) * with_columns(K, [](auto in) { return Operands<T, decltype(in)::value>::kUnits; }) * 64 * 16;
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// splits of the rows of a piece for k_gated_many_gw
template <class T>
int64_t many_splits(int64_t rows, int64_t K, int64_t n, int cus) {
  constexpr int64_t wide = 32 * kManyCols<T>, element = sizeof(T);
  const int64_t tiles = (n + wide - 1) / wide * ((K + 63) / 64), steps = (std::min(rows, kPiece) + 31) / 32;
  const int64_t most = std::max<int64_t>(1, ((int64_t)64 << 20) / (2 * (K + 1) * n * element));
  return std::max<int64_t>(1, std::min({(steps + 7) / 8, 2 * cus / tiles, most}));
}

// splits of k_gated_many_gx: where one piece of rows leaves compute units without work
template <class T>
int64_t many_gx_splits(int64_t rows, int64_t K, int64_t n, int cus) {
  const int64_t blocks = (rows + kManyRows<T> - 1) / kManyRows<T> * ((K + 63) / 64);
  return rows > kPiece ? 1 : std::max<int64_t>(1, std::min(2 * ((n + 31) / 32), cus / blocks));
}

template <class T>
size_t workspace_bytes(int64_t rows, int64_t K, int64_t n) {
  const size_t e = sizeof(T), part = 2 * (K + 1) * n * e;
  if (K <= kMaxIn) {
    const int64_t gx = gx_splits<T>(rows, K, n);
    return up(operand_bytes<T>(K, n)) + up(gw_splits<T>(rows, K, n, kMostUnits) * part) + (gx > 1 ? up(gx * rows * K * e) : 0);
  }
  const int64_t gx = many_gx_splits<T>(rows, K, n, kMostUnits);
  return 2 * up(std::min(rows, kPiece) * n * e) + up(many_splits<T>(rows, K, n, kMostUnits) * part) + (gx > 1 ? up(gx * rows * K * e) : 0);
}

template <class T, int kIn, int NT, int kAct>
hipError_t launch_fwd(const GatedArgs& a, int cus, hipStream_t st) {
  const int64_t cols = (a.d_out + 64 * NT - 1) / (64 * NT), blocks = (a.rows + kRows - 1) / kRows;
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(blocks, kGroups<T, kIn> * cus / cols));
  const dim3 grid((unsigned)(cols * splits));
  if (a.d_in % 4 == 0 && a.d_out % 2 == 0) k_gated_fwd<T, kIn, NT, kAct, true><<<grid, kThreads, 0, st>>>(a, (int)cols, (int)splits);
  else k_gated_fwd<T, kIn, NT, kAct, false><<<grid, kThreads, 0, st>>>(a, (int)cols, (int)splits);
  return hipGetLastError();
}

template <class T, int kAct>
hipError_t forward_act(const GatedArgs& a, int cus, hipStream_t st) {
  if (a.d_in > kMaxIn) {
    const int64_t tiles = (a.d_out + 63) / 64, most = std::max<int64_t>(1, kMostGroups / tiles) * kManyRows<T>;   // rows of a launch
    for (int64_t r = 0; r < a.rows; r += most) {
      const int64_t rows = std::min(a.rows - r, most);
      k_gated_many<T, kAct, false><<<dim3((unsigned)((rows + kManyRows<T> - 1) / kManyRows<T> * tiles)), kThreads, 0, st>>>(a, r, rows, (T*)nullptr, (T*)nullptr);
    }
    return hipGetLastError();
  }
  // 32 columns a wave where that leaves every compute unit two workgroups, else 16 (fp64 and more columns of x: 16, for the registers)
  const bool wide = sizeof(T) == 4 && (a.d_out + 127) / 128 * ((a.rows + kRows - 1) / kRows) >= 2 * cus;
  return with_columns(a.d_in, [&](auto in) {
    constexpr int kIn = decltype(in)::value;
    if constexpr (sizeof(T) == 4 && kIn <= 64)
      if (wide) return launch_fwd<T, kIn, 2, kAct>(a, cus, st);
    return launch_fwd<T, kIn, 1, kAct>(a, cus, st);
  });
}

template <class T>
hipError_t sum_splits(const GatedArgs& a, const T* part, int64_t splits, const T* gx_part, int64_t gx_splits, hipStream_t st) {
  const int64_t size = 2 * (a.d_in + 1) * a.d_out + (gx_splits > 1 ? a.rows * a.d_in : 0);
  k_gated_sums<T><<<dim3((unsigned)std::min((size + kThreads - 1) / kThreads, kMostGroups)), kThreads, 0, st>>>(a, part, (int)splits, gx_part, (int)gx_splits);
  return hipGetLastError();
}

template <class T, int kIn, int kAct>
hipError_t launch_bwd(const GatedArgs& a, int cus, char* ws, hipStream_t st) {
  const int64_t K = a.d_in, n = a.d_out, wide = 16 * kGwWaves, cols = (n + wide - 1) / wide;
  const int64_t gws = gw_splits<T>(a.rows, K, n, cus), gxs = gx_splits<T>(a.rows, K, n), blocks = (a.rows + gx_rows<T>(K) - 1) / gx_rows<T>(K);
  u32x4* ops = blocks > kFewBlocks ? (u32x4*)ws : nullptr;
  T* part = (T*)(ws + up(operand_bytes<T>(K, n)));
  T* gx_part = (T*)((char*)part + up(gw_splits<T>(a.rows, K, n, kMostUnits) * 2 * (K + 1) * n * sizeof(T)));
  if (ops) k_gated_operands<T, kIn><<<dim3((unsigned)(((n + 31) / 32 * Operands<T, kIn>::kOps + 3) / 4)), kThreads, 0, st>>>(a, ops);
  constexpr int kGxThreads = kGxWaves<T, kIn> * 64, kGwThreads = kGwWaves * 64;
  const dim3 gw((unsigned)(cols * gws));
  const bool whole = K % 4 == 0;
  for (int64_t b = 0; b < blocks; b += kMostGroups) {   // one launch where gxs > 1
    const int64_t r = b * gx_rows<T>(K);
    GatedArgs p = a;
    p.rows = std::min(a.rows - r, kMostGroups * gx_rows<T>(K));
    p.x = (const T*)a.x + r * a.ld_x;
    p.gout = (const T*)a.gout + r * a.ld_gout;
    p.gx = (T*)a.gx + r * a.ld_gx;
    const dim3 gx((unsigned)(std::min(blocks - b, kMostGroups) * gxs));
    if (whole && n % 4 == 0) k_gated_gx<T, kIn, kAct, true><<<gx, kGxThreads, 0, st>>>(p, ops, (int)gxs, gx_part);
    else k_gated_gx<T, kIn, kAct, false><<<gx, kGxThreads, 0, st>>>(p, ops, (int)gxs, gx_part);
  }
  if (whole) k_gated_gw<T, kIn, kAct, true><<<gw, kGwThreads, 0, st>>>(a, (int)cols, (int)gws, part);
  else k_gated_gw<T, kIn, kAct, false><<<gw, kGwThreads, 0, st>>>(a, (int)cols, (int)gws, part);
  return sum_splits<T>(a, part, gws, gx_part, gxs, st);
}

template <class T, int kAct>
hipError_t backward_act(const GatedArgs& a, int cus, char* ws, hipStream_t st) {
  if (a.d_in <= kMaxIn) return with_columns(a.d_in, [&](auto in) { return launch_bwd<T, decltype(in)::value, kAct>(a, cus, ws, st); });
  const int64_t K = a.d_in, n = a.d_out, splits = many_splits<T>(a.rows, K, n, cus);
  const int64_t ct = (n + 63) / 64, kt = (K + 63) / 64, gt = (n + 32 * kManyCols<T> - 1) / (32 * kManyCols<T>);
  T* dg = (T*)ws;
  T* du = (T*)(ws + up(std::min(a.rows, kPiece) * n * sizeof(T)));
  T* part = (T*)((char*)du + up(std::min(a.rows, kPiece) * n * sizeof(T)));
  T* gx_part = (T*)((char*)part + up(many_splits<T>(a.rows, K, n, kMostUnits) * 2 * (K + 1) * n * sizeof(T)));
  const int64_t gxs = many_gx_splits<T>(a.rows, K, n, cus);
  for (int64_t r = 0; r < a.rows; r += kPiece) {
    const int64_t rows = std::min(kPiece, a.rows - r), rb = (rows + kManyRows<T> - 1) / kManyRows<T>;
    k_gated_many<T, kAct, true><<<dim3((unsigned)(rb * ct)), kThreads, 0, st>>>(a, r, rows, dg, du);
    k_gated_many_gx<T><<<dim3((unsigned)(rb * kt * gxs)), kThreads, 0, st>>>(a, r, rows, dg, du, (int)gxs, gx_part);
    k_gated_many_gw<T><<<dim3((unsigned)(gt * kt * splits)), kThreads, 0, st>>>(a, r, rows, dg, du, (int)splits, part, r > 0);
  }
  return sum_splits<T>(a, part, splits, gx_part, gxs, st);
}

template <class T>
hipError_t forward(const GatedArgs& a, int cus, hipStream_t st) {
  switch (a.act) {
    case CGTP_ACT_NONE: return forward_act<T, CGTP_ACT_NONE>(a, cus, st);
    case CGTP_ACT_SILU: return forward_act<T, CGTP_ACT_SILU>(a, cus, st);
    case CGTP_ACT_GELU: return forward_act<T, CGTP_ACT_GELU>(a, cus, st);
    case CGTP_ACT_SIGMOID: return forward_act<T, CGTP_ACT_SIGMOID>(a, cus, st);
    default: return forward_act<T, CGTP_ACT_TANH>(a, cus, st);
  }
}

template <class T>
hipError_t backward(const GatedArgs& a, int cus, char* ws, hipStream_t st) {
  switch (a.act) {
    case CGTP_ACT_NONE: return backward_act<T, CGTP_ACT_NONE>(a, cus, ws, st);
    case CGTP_ACT_SILU: return backward_act<T, CGTP_ACT_SILU>(a, cus, ws, st);
    case CGTP_ACT_GELU: return backward_act<T, CGTP_ACT_GELU>(a, cus, ws, st);
    case CGTP_ACT_SIGMOID: return backward_act<T, CGTP_ACT_SIGMOID>(a, cus, ws, st);
    default: return backward_act<T, CGTP_ACT_TANH>(a, cus, ws, st);
  }
}

}  // namespace
}  // namespace cgtp
