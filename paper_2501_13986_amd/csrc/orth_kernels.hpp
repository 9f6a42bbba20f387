// Kernels of orthogonalise, for the translation units of its two types (orth_f32.hip, orth_f64.hip).
//
// X = G / (|G| + eps), transposed if G has more rows than columns, so that X is s x l with s <= l; a step is
//     A = X X^T,  B = b A + c A A,  X <- a X + B X.
#pragma once

#include <algorithm>
#include <type_traits>

#include "orth.hpp"
#include "product.hpp"

namespace cgtp {
namespace {

constexpr int kShares = 256;      // partial sums of squares of a matrix, at most

// ---- the start ------------------------------------------------------------------------------------------------------------------

// Part of a matrix: the sum of squares of its numbers times `power`, a power of two.  With the power, fp64 numbers of any size serve: unscaled, squares
// of those below 1e-154 are lost and of those above 1e154 overflow.  It costs 0.5 us of a launch for all steps (32 x 32 12.0), 3 of the start of tiles
// (4 of 400 x 400 365); fp32 nothing.
struct Size {
  double squares, power;
};

// The power of two that brings the largest number near one, so that no square overflows or is lost (the squares of fp32 numbers do neither in fp64).  Of zeros the
// greatest, so that they decide nothing beside others; of infinities and NaN any, for their squares tell.
__device__ inline double power_for(double largest) {
  const int e = largest == 0 ? -1000 : __builtin_amdgcn_frexp_exp(largest);
  return __builtin_amdgcn_ldexp(1.0, e < -1000 ? 1000 : e > 1000 ? -1000 : -e);
}

// 1 / (|G| + eps) is power * inverse: numbers are multiplied by one after the other
struct Scale {
  double power, inverse;
  // for numbers that have been multiplied by p
  __device__ double of(double p) const { return power / p * inverse; }
};

// of the parts of a matrix, by all lanes of a wave; none is masked off: those behind the end have the last part again
__device__ inline Scale scale_of(const Size* part, int parts, double eps) {
  const int lane = (int)threadIdx.x & 63;
  auto get = [&](int i) { return part[i + lane < parts ? i + lane : parts - 1]; };
  const Size first = get(0);
  double power = first.power, v = 0;
  for (int i = 64; i < parts; i += 64) power = fmin(power, get(i).power);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) power = fmin(power, __shfl_xor(power, d));
  auto add = [&](int i, const Size& s) {
    const double f = power / s.power, w = s.squares * (f * f);
    v += i + lane < parts ? w : 0.0;
  };
  add(0, first);
  for (int i = 64; i < parts; i += 64) add(i, get(i));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return {power, 1.0 / (sqrt(v) + eps * power)};
}

// part [batch][shares]: of shares of the rows, for matrices of more than 128 rows and columns
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_squares(OrthArgs a, int64_t first, int shares, Size* part) {
  __shared__ double sums[2][kProductThreads / 64];
  const int64_t matrix = first + blockIdx.x / shares, share = blockIdx.x % shares;
  const T* g = (const T*)a.g + matrix * a.stride_g;
  const int64_t from = a.m * share / shares, end = a.m * (share + 1) / shares;
  // rows have more than 128 numbers; eight numbers on their way to a thread
  const int wide = a.n >= kProductThreads ? kProductThreads : 128, x = threadIdx.x % wide, y = threadIdx.x / wide, high = kProductThreads / wide;
  auto each = [&](auto f) {
    for (int64_t r = from + y; r < end; r += high) {
      const T* p = g + r * a.ld_g;
      int64_t c = x;
      for (; c + 7 * wide < a.n; c += 8 * wide) {
        double w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (double)p[c + i * wide];
#pragma unroll
        for (int i = 0; i < 8; ++i) f(w[i]);
      }
      for (; c < a.n; c += wide) f((double)p[c]);
    }
  };
  double power = 1;
  if constexpr (sizeof(T) == 8) {      // the second reading is from the caches
    double most = 0;
    each([&](double w) { most = fmax(most, fabs(w)); });
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmax(most, __shfl_xor(most, d));
    if (threadIdx.x % 64 == 0) sums[0][threadIdx.x / 64] = most;
    __syncthreads();
    power = power_for(fmax(fmax(sums[0][0], sums[0][1]), fmax(sums[0][2], sums[0][3])));
  }
  double v = 0;
  each([&](double w) {
    w *= power;
    v += w * w;
  });
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if (threadIdx.x % 64 == 0) sums[1][threadIdx.x / 64] = v;
  __syncthreads();
  if (threadIdx.x == 0) part[matrix * shares + share] = {(sums[1][0] + sums[1][1]) + (sums[1][2] + sums[1][3]), power};
}

// ---- more rows --------------------------------------------------------------------------------------------------------------------
//
// X, its transpose, A and B stand in memory as operands: in parts, cut once by the kernel that writes them, in blocks of 64 rows x 32 terms, padded with
// zeros.  A product is tiles of kTile x kTile results with the terms in splits, so that there is work for all compute units; sums of splits are left in
// the order of the registers and added up, in their order, by k_orth_finish, which turns the results into operands both ways.  With one split the product does that itself.
// 1152 x 2048 fp32, a step: A 19 us and 6 to finish, B the same, X 31 and 13 (its product 1.05 PFLOP/s of bf16 products, library 1.09, in 432 workgroups on 256 units); operands in fp32, cut by
// each reader, took twice that.  More terms in LDS at a time were no faster, 128 x 64 tiles slower.

constexpr int kBlock = 64;

// numbers [rows, terms] as an operand of products; sizes are those of the padded matrix
template <class T>
struct Stored;
template <>
struct Stored<float> {
  static constexpr int kBytes = 6;
  unsigned short* p;
  int64_t plane;      // from one part to the next
  int ld;             // blocks a row of blocks
  __device__ Stored(void* at, int64_t rows, int64_t terms) : p((unsigned short*)at), plane(rows * terms), ld((int)(terms / kStep)) {}
  __device__ int64_t at(int r, int k) const { return ((int64_t)(r / kBlock) * ld + k / kStep) * (kBlock * kStep) + r % kBlock * kStep + k % kStep; }
  __device__ void write8(int r, int k, const float* x) const {
    const PartsOf<3> w = Num<float>::parts(x);
#pragma unroll
    for (int i = 0; i < 3; ++i) *(u32x4*)(p + i * plane + at(r, k)) = w.w[i];
  }
  // the parts' sum is the number itself
  __device__ void read8(int r, int k, float* x) const {
    u32x4 w[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i] = *(const u32x4*)(p + i * plane + at(r, k));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) v[i] = __builtin_bit_cast(float, j & 1 ? w[i][j / 2] & 0xffff0000u : w[i][j / 2] << 16);
      x[j] = (v[2] + v[1]) + v[0];
    }
  }
};
template <>
struct Stored<double> {
  static constexpr int kBytes = 8;
  double* p;
  int ld;
  __device__ Stored(void* at, int64_t, int64_t terms) : p((double*)at), ld((int)(terms / kStep)) {}
  __device__ int64_t at(int r, int k) const { return ((int64_t)(r / kBlock) * ld + k / kStep) * (kBlock * kStep) + r % kBlock * kStep + k % kStep; }
  __device__ void write8(int r, int k, const double* x) const {
#pragma unroll
    for (int h = 0; h < 8; h += 2) *(f64x2*)(p + at(r, k) + h) = f64x2{x[h], x[h + 1]};
  }
  __device__ void read8(int r, int k, double* x) const {
#pragma unroll
    for (int h = 0; h < 8; h += 2) {
      const f64x2 w = *(const f64x2*)(p + at(r, k) + h);
      x[h] = w[0];
      x[h + 1] = w[1];
    }
  }
};

// kR rows of 32 terms on their way to LDS
template <class T, int kR>
struct Copy;
template <int kR>
struct Copy<float, kR> {
  static constexpr int kPer = 3 * kR / kBlock;
  u32x4 v[kPer];
  __device__ void fetch(const Stored<float>& from, int r0, int k0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      v[i] = *(const u32x4*)(from.p + i / (kR / kBlock) * from.plane + ((int64_t)(r0 / kBlock + i % (kR / kBlock)) * from.ld + k0 / kStep) * (kBlock * kStep) + threadIdx.x * 8);
  }
  __device__ void put(Operand<float, kR>& to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int r = i % (kR / kBlock) * kBlock + (int)threadIdx.x / 4;
      *(u32x4*)&to.v[i / (kR / kBlock)][r][to.at(r, (int)threadIdx.x % 4 * 8)] = v[i];
    }
  }
};
template <int kR>
struct Copy<double, kR> {
  static constexpr int kPer = 4 * kR / kBlock;
  u32x4 v[kPer];
  __device__ void fetch(const Stored<double>& from, int r0, int k0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      v[i] = *(const u32x4*)(from.p + ((int64_t)(r0 / kBlock + i / 4) * from.ld + k0 / kStep) * (kBlock * kStep) + (i % 4 * kProductThreads + threadIdx.x) * 2);
  }
  __device__ void put(Operand<double, kR>& to) const {
#pragma unroll
    for (int i = 0; i < kPer; ++i) *(u32x4*)&to.v[i / 4 * kBlock + i % 4 * 16 + (int)threadIdx.x / 16][(int)threadIdx.x % 16 * 2] = v[i];
  }
};

// X and its transpose, 64 x 64 numbers of G a workgroup; rounded once.  s, l: padded
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_start(OrthArgs a, int64_t first, int tiles, int s, int l, int shares, const Size* part, char* X, char* XT) {
  __shared__ T tile[kBlock][kBlock + 1];
  const int64_t matrix = first + blockIdx.x / tiles, size = (int64_t)s * l * Stored<T>::kBytes;
  const bool turned = a.m > a.n;
  const int across = l / kBlock, r0 = blockIdx.x % tiles / across * kBlock, c0 = blockIdx.x % tiles % across * kBlock;      // of X
  const Scale scale = scale_of(part + matrix * shares, shares, a.eps);
  const T* g = (const T*)a.g + matrix * a.stride_g;
  const Stored<T> to(X + matrix * size, s, l), to_t(XT + matrix * size, l, s);
  const int x = threadIdx.x % kBlock;
  for (int y = threadIdx.x / kBlock; y < kBlock; y += kProductThreads / kBlock) {      // neighbours of G side by side
    const int64_t r = (turned ? c0 : r0) + y, c = (turned ? r0 : c0) + x;
    const T v = r < a.m && c < a.n ? (T)((double)g[r * a.ld_g + c] * scale.power * scale.inverse) : T(0);
    if (turned) tile[x][y] = v;
    else tile[y][x] = v;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kBlock * kBlock / 8; i += kProductThreads) {      // whole blocks one behind the other
    const int y = i / 4 % kBlock, k = i / (4 * kBlock) * kStep + i % 4 * 8;
    T v[8], u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      v[j] = tile[y][k + j];
      u[j] = tile[k + j][y];
    }
    to.write8(r0 + y, c0 + k, v);
    to_t.write8(c0 + y, r0 + k, u);
  }
}

// tile number -> row and column of tiles, on and above the diagonal
__device__ inline void upper_tile(int t, int& r, int& c) {
  c = (int)((__builtin_sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while (c * (c + 1) / 2 > t) --c;
  while ((c + 1) * (c + 2) / 2 <= t) ++c;
  r = t - c * (c + 1) / 2;
}

// A product R C^T [rows, columns]: alpha Y + beta R C^T of it is kept in to (and its transpose in to_t), or in the caller's output.  Symmetric: the tiles on and above the
// diagonal alone, whose transposes are the others.
struct Product {
  char *rows_at, *columns_at, *y, *to, *to_t;
  int rows, columns, terms, tiles, splits;      // padded; tiles a matrix
  double alpha, beta;
  bool symmetric, last;
};

template <class T, int kTile>
union ProductLds {
  struct {
    Operand<T, kTile> R, C;
  } in;
  T out[64][kTile + 1];      // rows of a tile that pass through LDS at a time: 32 of each half
  __device__ ProductLds() {}
};

template <int kTile>
__device__ inline void tile_of(const Product& p, int t, int& tr, int& tc) {
  if (p.symmetric) {
    upper_tile(t, tr, tc);
  } else {
    tr = t / (p.columns / kTile);
    tc = t % (p.columns / kTile);
  }
}

// kRows rows of a tile, whose products (times beta) stand in LDS: the rows from r0 on, and with 64 those that are half a tile behind them
template <class T, int kTile, int kRows>
__device__ inline void finish(const OrthArgs& a, const Product& p, int64_t matrix, int r0, int c0, T (&tile)[kRows][kTile + 1]) {
  const int64_t size = (int64_t)p.rows * p.columns * Stored<T>::kBytes;
  const T alpha = (T)p.alpha;
  auto row = [&](int y) { return r0 + y / 32 * (kTile / 2) + y % 32; };
  __syncthreads();
  const bool add = p.alpha != 0, mirror = !p.symmetric || r0 / kTile != c0 / kTile;
  if (add || !p.last) {
    const Stored<T> y(p.y + matrix * size, p.rows, p.columns), to(p.to + matrix * size, p.rows, p.columns);
    for (int i = threadIdx.x; i < kRows * kTile / 8; i += kProductThreads) {      // rows of 64 bytes one behind the other
      const int r = i / 4 % kRows, k = i / (4 * kRows) * kStep + i % 4 * 8;
      T v[8], u[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = tile[r][k + j];
      if (add) {
        y.read8(row(r), c0 + k, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] += alpha * u[j];
          tile[r][k + j] = v[j];
        }
      }
      if (!p.last) to.write8(row(r), c0 + k, v);
    }
    __syncthreads();
  }
  if (p.last) {
    T* to = (T*)a.out + matrix * a.stride_out;
    if (a.m > a.n) {
      for (int i = threadIdx.x; i < kTile * kRows; i += kProductThreads) {
        const int y = i % kRows, x = i / kRows;
        if (c0 + x < a.m && row(y) < a.n) to[(int64_t)(c0 + x) * a.ld_out + row(y)] = tile[y][x];
      }
    } else {
      for (int i = threadIdx.x; i < kTile * kRows; i += kProductThreads) {
        const int y = i / kTile, x = i % kTile;
        if (row(y) < a.m && c0 + x < a.n) to[(int64_t)row(y) * a.ld_out + c0 + x] = tile[y][x];
      }
    }
  } else if (mirror) {
    const Stored<T> to((p.symmetric ? p.to : p.to_t) + matrix * size, p.columns, p.rows);
    for (int i = threadIdx.x; i < kRows * kTile / 8; i += kProductThreads) {
      const int c = i / 4 % kTile, k = i / (4 * kTile) * 32 + i % 4 * 8;
      T v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = tile[k + j][c];
      to.write8(c0 + c, row(k), v);
    }
  }
}

template <class T, int kTile>
__global__ void __launch_bounds__(kProductThreads, 2) k_orth_product(OrthArgs a, Product p, int64_t first, T* part) {
  __shared__ ProductLds<T, kTile> S;
  const unsigned block = on_one_die(blockIdx.x, gridDim.x);
  const int t = block % p.tiles, split = block / p.tiles % p.splits;
  const int64_t matrix = first + block / p.tiles / p.splits;
  int tr, tc;
  tile_of<kTile>(p, t, tr, tc);
  const Stored<T> left(p.rows_at + matrix * p.rows * p.terms * Stored<T>::kBytes, p.rows, p.terms), right(p.columns_at + matrix * p.columns * p.terms * Stored<T>::kBytes, p.columns, p.terms);
  const int steps = p.terms / kStep, from = steps * split / p.splits, end = steps * (split + 1) / p.splits;
  Results<T, kTile, kTile> out;
  // fp64 fetches two steps ahead, for few waves share a unit (1000 x 1100 736 us, with one 792; fp32 tiles of 64 gain nothing).  What is fetched behind the end is the last step
  // once more: without the condition tiles of 128 need 148 registers, three workgroups a unit, for 191 (2000 x 2000 1078 us for 1171); those of 64 lose (300 x 2000 209 for 201).
  constexpr int kAhead = sizeof(T) == 8 ? 2 : 1;
  Copy<T, kTile> rows[kAhead], columns[kAhead];
  auto fetch = [&](int slot, int k) {
    const int at = (k < end ? k : end - 1) * kStep;
    rows[slot].fetch(left, tr * kTile, at);
    columns[slot].fetch(right, tc * kTile, at);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(i, from + i);
  for (int k = from; k < end; k += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i > 0 && k + i >= end) break;
      __syncthreads();
      rows[i].put(S.in.R);
      columns[i].put(S.in.C);
      __syncthreads();
      if (sizeof(T) == 8 || kTile == 128 || k + 1 < end) fetch(i, k + i + kAhead);
      out.multiply(S.in.R, S.in.C);
    }
  }
  if (p.splits > 1) {
    out.keep(part + ((matrix * p.tiles + t) * p.splits + split) * (kTile * kTile));
    return;
  }
  const T beta = (T)p.beta;
#pragma unroll
  for (int h = 0; h < out.RT / 2; ++h) {
    __syncthreads();
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int ct = 0; ct < out.CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) S.out[out.wave() / 2 * 32 + rt * 16 + out.lane() % 16][out.column(ct) + i] = beta * out.acc[2 * h + rt][ct][i];
    finish<T, kTile, 64>(a, p, matrix, tr * kTile + h * 32, tc * kTile, S.out);
  }
}

// 32 rows of a tile a workgroup
template <class T, int kTile>
__global__ void __launch_bounds__(kProductThreads) k_orth_finish(OrthArgs a, Product p, int64_t first, const T* part) {
  using Out = Results<T, kTile, kTile>;
  constexpr int kStrips = kTile / 32;
  __shared__ T tile[32][kTile + 1];
  const int strip = blockIdx.x % kStrips, t = blockIdx.x / kStrips % p.tiles;
  const int64_t matrix = first + blockIdx.x / kStrips / p.tiles;
  int tr, tc;
  tile_of<kTile>(p, t, tr, tc);
  // of the product's waves the two that have these rows; a thread takes one of two tiles of 16 of them
  const int half = strip / (kStrips / 2), h = strip % (kStrips / 2), rt = threadIdx.x / 128, thread = half * 128 + threadIdx.x % 128, lane = threadIdx.x % 64;
  typename Out::N::Vec acc[Out::CT] = {};
  Out::add_up(part + (matrix * p.tiles + t) * p.splits * (kTile * kTile) + ((2 * h + rt) * Out::CT * Out::kThreads + thread) * 4, p.splits, acc);
  const T beta = (T)p.beta;
#pragma unroll
  for (int ct = 0; ct < Out::CT; ++ct)
#pragma unroll
    for (int i = 0; i < 4; ++i) tile[rt * 16 + lane % 16][thread / 64 % 2 * (kTile / 2) + ct * 16 + lane / 16 * 4 + i] = beta * acc[ct][i];
  finish<T, kTile, 32>(a, p, matrix, tr * kTile + half * (kTile / 2) + h * 32, tc * kTile, tile);
}

// ---- up to 128 rows of X --------------------------------------------------------------------------------------------------------
//
// A workgroup has 16 NT columns of X for each of its kWaves waves in registers, a wave all their rows: lane: columns NT l16 + j, rows 16 t + 4 q + (0..3).
// A step is X <- a X + A V, V = b X + c A X, so that both products have A (in LDS) on the left and on the right what the wave has: results of the matrix
// instructions are operands of the next ones as they are, with the terms of 32 rows in the order `place`.  Only for A = X X^T does X go through LDS.
// Where the workgroup has all columns, the steps run without leaving it.  Where not, a launch is a step: the workgroups leave their shares of A, which all of the next
// launch add up, and X in the order of their registers.
// 89 matrices of 128 x 128 fp32 65 to 70 us on as many units, matrix pipe busy 54 % of their cycles; halves of them on twice the units, a launch a step, 102.  2 of 64 x 2176: 51 us, six
// launches of 5 to 10 us (17 shares of A, 2 us, the products 2 us, launch and end).  64 x 64: 16 us, a chain of 20 barriers.  fp64, 17 of 301 x 96: 132 us, 24 a step on 85
// units, half of it matrix instructions.

constexpr int kMostRows = 128;

// the place of row r among 32 terms of results
__device__ inline int place(int r) { return r % 16 / 4 * 8 + r / 16 * 4 + r % 4; }

// waves a SIMD whose registers are left: two where half of the registers are enough, so that none of their values are moved about
template <class T, int kS, int kWaves>
constexpr int kOrthWaves = kWaves == 8 || sizeof(T) == 4 || kS <= 64 ? 2 : 1;

template <class T, int kS, int NT, int kWaves>
struct Columns {
  using N = Num<T>;
  static constexpr int kTiles = kS / 16, kWide = 16 * NT * kWaves, kSlices = (kS > kWide ? kS : kWide) / 32, kThreads = 64 * kWaves;
  using Lds = Operand<T, kS, kApart>[kSlices];
  // A: 2 x (3 or kWaves / 2) of the waves
  static constexpr int kGramAcross = kS % (kWaves * 8) == 0 ? kWaves / 2 : 3;
  using Gram = Results<T, kS, kS, 2, kGramAcross>;
  static __device__ bool forms_gram() { return kGramAcross * 2 == kWaves || Gram::wave() < kGramAcross * 2; }
  typename N::Vec x[kTiles][NT];

  static __device__ int lane() { return (int)threadIdx.x & 63; }
  static __device__ int column(int j) { return (int)(threadIdx.x / 64) * (16 * NT) + lane() % 16 * NT + j; }
  static __device__ int row(int t) { return t * 16 + lane() / 16 * 4; }      // the first of four

  // columns c0 .. of the matrix at g (transposed: it has them as rows), as they are; zero outside.  Through descriptors of 16 of its rows (strides are below 2^22), so that no
  // lane is masked off.
  __device__ void load(const T* g, int64_t ld, int s, int l, int c0, bool turned) {
    constexpr int e = sizeof(T);
    auto get = [](Buffer B, unsigned at) {
      if constexpr (e == 4) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(B, at, 0, 0));
      else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b64(B, at, 0, 0));
    };
    if (turned) {
      const int first = c0 + Gram::wave() * (16 * NT), have = l - first < 16 * NT ? l - first : 16 * NT;
      const Buffer B = buffer_of(g + (have > 0 ? first : 0) * ld, have > 0 ? ((have - 1) * ld + s) * e : 0);
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = row(t) + i, c = lane() % 16 * NT + j;
            x[t][j][i] = get(B, r < s && c < have ? ((unsigned)c * (unsigned)ld + (unsigned)r) * e : kNowhere);
          }
    } else {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int have = s - t * 16 < 16 ? s - t * 16 : 16;
        const Buffer B = buffer_of(g + (have > 0 ? t * 16 * ld : 0) + c0, have > 0 ? ((have - 1) * ld + l - c0) * e : 0);
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = lane() / 16 * 4 + i;
            x[t][j][i] = get(B, r < have && c0 + column(j) < l ? ((unsigned)r * (unsigned)ld + (unsigned)column(j)) * e : kNowhere);
          }
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
      for (int j = 0; j < NT; ++j) *(typename N::Vec*)(to + ((t * NT + j) * kThreads + (int)threadIdx.x) * 4) = x[t][j];
  }
  __device__ void take(const T* from) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j) x[t][j] = *(const typename N::Vec*)(from + ((t * NT + j) * kThreads + (int)threadIdx.x) * 4);
  }
  // the thread's largest number
  __device__ double largest() const {
    double v = 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) v = fmax(v, fabs((double)x[t][j][i]));
    return v;
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
    if constexpr (NT == 1 && sizeof(T) == 4) {
      // neighbouring lanes change two of their four rows, for pairs of columns in one word
      const bool odd = threadIdx.x & 1;
      const int c = column(0) & ~1;
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float lo = x[t][0][i], hi = x[t][0][i + 2], got = __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, odd ? lo : hi), 0xb1, 0xf, 0xf, true));
          S[c / 32].write_some(row(t) + i + (odd ? 2 : 0), c % 32, {odd ? got : lo, odd ? hi : got});
        }
    } else {
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          T v[NT];
#pragma unroll
          for (int j = 0; j < NT; ++j) v[j] = x[t][j][i];
          S[column(0) / 32].write_some(row(t) + i, column(0) % 32, v);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kWide / 32; ++k) {
      if (forms_gram()) A.multiply(S[k], S[k]);
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
  }
  // A as the left operand of the step's products
  static __device__ void put(Lds& S, const Gram& A) {
    if (forms_gram())
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
  // X <- a X + A (b X + c A X), A in LDS.  The sum of A V starts from zero: from a X, every term's rounding would be one of the whole.
  __device__ void step(const Lds& S, T a, T b, T c) {
    typename N::Vec y[kTiles][NT] = {}, z[kTiles][NT] = {};
    times(S, x, y);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][j][i] = b * x[t][j][i] + c * y[t][j][i];
    times(S, y, z);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][j][i] = a * x[t][j][i] + z[t][j][i];
  }
};

// sum over the workgroup, to all its threads
template <int kWaves>
__device__ inline double sum_of_all(double v, double (&sums)[kWaves]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  sums[threadIdx.x / 64] = v;      // all lanes the same
  __syncthreads();
  v = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) v += sums[i];
  return v;
}

template <int kWaves>
__device__ inline double largest_of_all(double v, double (&most)[kWaves]) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v = fmax(v, __shfl_xor(v, d));
  most[threadIdx.x / 64] = v;      // all lanes the same
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) v = fmax(v, most[i]);
  return v;
}

// X, which is as it was read, is multiplied by a power of two that brings it near one: its size.  fp32: the squares are numbers of fp64 and name the power, so that only `near` asks
// for it; fp64: the largest number does.
template <bool near, int kWaves, class Cols>
__device__ inline Size size_of(Cols& X, double (&sums)[2][kWaves]) {
  if constexpr (sizeof(X.x[0][0][0]) == 8) {
    const double power = power_for(largest_of_all<kWaves>(X.largest(), sums[0]));
    X.scale(power);
    return {sum_of_all<kWaves>(X.squares(), sums[1]), power};
  } else {
    const double squares = sum_of_all<kWaves>(X.squares(), sums[1]), power = near ? power_for(sqrt(squares)) : 1;
    if (near) X.scale(power);
    return {squares * power * power, power};
  }
}

struct Schedule {
  double c[64][3];
};

// all steps of a matrix of at most 16 NT kWaves columns
template <class T, int kS, int NT, int kWaves>
__global__ void __launch_bounds__((64 * kWaves), (kOrthWaves<T, kS, kWaves>)) k_orth_whole(OrthArgs a, int64_t first, int steps, Schedule schedule) {
  using Cols = Columns<T, kS, NT, kWaves>;
  __shared__ typename Cols::Lds S;
  __shared__ double sums[2][kWaves];
  const int64_t matrix = first + blockIdx.x;
  const bool turned = a.m > a.n;
  const int s = (int)(turned ? a.n : a.m), l = (int)(turned ? a.m : a.n);
  Cols X;
  X.load((const T*)a.g + matrix * a.stride_g, a.ld_g, s, l, 0, turned);
  const Size size = size_of<false>(X, sums);
  X.scale(1.0 / (sqrt(size.squares) + a.eps * size.power));
  for (int i = 0; i < steps; ++i) {
    typename Cols::Gram A;
    X.gram(S, A);
    Cols::put(S, A);
    X.step(S, (T)schedule.c[i][0], (T)schedule.c[i][1], (T)schedule.c[i][2]);
  }
  X.store((T*)a.out + matrix * a.stride_out, a.ld_out, s, l, 0, turned);
}

// The start leaves each chunk of X multiplied by the power of two that brings its size near one, so that no product of it overflows or is lost, with its size: that of all of X is known
// when the first step begins, which multiplies X once (as if G were) and the shares of A by the squares.
// The first share of A [matrix][chunk][kS * kS] and X [matrix][chunk][kS * columns], in the order of the registers
template <class T, int kS, int NT, int kWaves>
__global__ void __launch_bounds__((64 * kWaves), (kOrthWaves<T, kS, kWaves>)) k_orth_begin(OrthArgs a, int64_t first, int chunks, Size* chunk, T* X_to, T* A_to) {
  using Cols = Columns<T, kS, NT, kWaves>;
  __shared__ typename Cols::Lds S;
  __shared__ double sums[2][kWaves];
  const int64_t matrix = first + blockIdx.x / chunks, place = matrix * chunks + blockIdx.x % chunks;
  const bool turned = a.m > a.n;
  const int s = (int)(turned ? a.n : a.m), l = (int)(turned ? a.m : a.n);
  Cols X;
  X.load((const T*)a.g + matrix * a.stride_g, a.ld_g, s, l, blockIdx.x % chunks * Cols::kWide, turned);
  const Size size = size_of<true>(X, sums);
  X.keep(X_to + place * (kS * Cols::kWide));
  typename Cols::Gram A;
  X.gram(S, A);
  if (Cols::forms_gram()) A.keep(A_to + place * (kS * kS));
  if (threadIdx.x == 0) chunk[place] = size;
}

// A step.  parts: how many shares of A there are a matrix; chunk: of the first step
template <class T, int kS, int NT, int kWaves, bool kLast>
__global__ void __launch_bounds__((64 * kWaves), (kOrthWaves<T, kS, kWaves>)) k_orth_step(OrthArgs a, int64_t first, int chunks, int parts, T c0, T c1, T c2, const Size* chunk,
                                                                                             T* X_at, const T* A_from, T* A_to) {
  using Cols = Columns<T, kS, NT, kWaves>;
  __shared__ typename Cols::Lds S;
  const int64_t matrix = first + blockIdx.x / chunks, place = matrix * chunks + blockIdx.x % chunks;
  Cols X;
  X.take(X_at + place * (kS * Cols::kWide));
  typename Cols::Gram A;
  A_from += matrix * parts * (kS * kS);
  const Scale scale = chunk ? scale_of(chunk + matrix * chunks, chunks, a.eps) : Scale{1, 1};
  if (chunk) X.scale(scale.of(chunk[place].power));
  if (Cols::forms_gram()) {
    if (chunk && parts == chunks) {
      A.add_all(A_from, parts, [&](int p) {
        const double f = scale.of(chunk[matrix * chunks + p].power);
        return (T)(f * f);
      });
    } else {
      A.add_all(A_from, parts, [](int) { return T(1); });
    }
  }
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
    if (Cols::forms_gram()) next.keep(A_to + place * (kS * kS));
  }
}

// to [matrix][size] = sums of from [matrix][parts][size]; chunk: of the first step.  32 numbers a workgroup (size is a multiple of them), eighths of the parts one after
// another: 157 shares of 32 x 32 numbers 7 us.
template <class T>
__global__ void __launch_bounds__(kProductThreads) k_orth_join(OrthArgs a, int64_t first, int blocks, int parts, int size, const Size* chunk, const T* from, T* to) {
  __shared__ T sums[8][32];
  const int64_t matrix = first + blockIdx.x / blocks;
  const int i = threadIdx.x % 32, group = threadIdx.x / 32, at = blockIdx.x % blocks * 32 + i;
  const Scale scale = chunk ? scale_of(chunk + matrix * parts, parts, a.eps) : Scale{1, 1};
  from += matrix * parts * size + at;
  T v = 0;
#pragma unroll 8
  for (int p = parts * group / 8; p < parts * (group + 1) / 8; ++p) {
    const double f = chunk ? scale.of(chunk[matrix * parts + p].power) : 1;
    v += (T)(f * f) * from[(int64_t)p * size];
  }
  sums[group][i] = v;
  __syncthreads();
  if (group > 0) return;
  v = 0;
#pragma unroll
  for (int g = 0; g < 8; ++g) v += sums[g][i];
  to[matrix * size + at] = v;
}

// ---- launches -------------------------------------------------------------------------------------------------------------------

constexpr int64_t kMostBlocks = (int64_t)1 << 22;   // workgroups of a launch, of up to 512 threads: 2^32 of them are too many

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

// What the columns of X are cut into where it has few rows.  Shares of A are added up by every workgroup of a matrix, beyond kMostShares bytes of them by a launch of its own
// (128 rows, a step: 9 shares, of 64 KiB, 20 us, 24 of them 29, added up before 16 and 5) or many of them (32 rows, 157 shares 17 us, added up before 5 and 7).
constexpr int64_t kMostShares = 640 << 10, kManyShares = 64;

struct Few {
  int64_t rows, wide, chunks;      // padded rows, columns of a chunk, chunks
  bool join;
  Few(int64_t m, int64_t n, bool f64) {
    const int64_t s = std::min(m, n), l = std::max(m, n);
    rows = (s + 31) / 32 * 32;
    wide = f64 || l <= 64 ? 64 : 128;
    chunks = (l + wide - 1) / wide;
    join = chunks * rows * rows * (f64 ? 8 : 4) > kMostShares || chunks > kManyShares;
  }
  size_t x_size() const { return rows * wide * chunks; }      // numbers a matrix
  size_t a_size() const { return rows * rows * chunks; }
  size_t sum_size() const { return join ? rows * rows : 0; }
};

// The products of a step where X has many rows.  Tiles of 128 x 128 read half as much for a product, tiles of 64 x 64 leave less unfilled.  fp32, all steps, X in large tiles and
// in small ones: 700 x 900 275 us and 234, 768 x 2048 310 and 297; A and its square in large and in small ones: 1500 x 1500 581 and 622, 1300 x 1400 515
// and 486.
template <class T>
struct Many {
  int square_tile, x_tile;           // of A and B, of X
  int64_t s, l, square, wide;        // padded sizes, tiles of A (on and above the diagonal) and of X
  int a_splits, b_splits, x_splits;
  Many(int64_t batch, int64_t m, int64_t n) {
    const int64_t s0 = std::min(m, n), l0 = std::max(m, n);
    square_tile = sizeof(T) == 4 && s0 >= 1408 ? 128 : 64;
    x_tile = sizeof(T) == 4 && s0 >= 1024 ? 128 : 64;
    s = (s0 + x_tile - 1) / x_tile * x_tile;
    l = (l0 + x_tile - 1) / x_tile * x_tile;
    square = s / square_tile * (s / square_tile + 1) / 2;
    wide = s / x_tile * (l / x_tile);
    // Splits of the terms, four steps of 32 or more each.  fp32: up to three workgroups of small tiles a compute unit (1152 rows: 27 us a product of A; with two 31) or two of
    // large ones (1152 x 2048 460 us; with three 488).  fp64: by the time of a unit that has the most of them (33 ns a term of a tile, one workgroup alone has two thirds of
    // the rate) and, with several, that of another launch and of the sums at 4.5 TB/s: 1152 x 2048 1134 us, with two workgroups a unit 1219.
    auto splits = [&](int tile, int64_t tiles, int64_t terms) {
      const int64_t all = batch * tiles, most = std::max<int64_t>(1, terms / kStep / 4);
      if constexpr (sizeof(T) == 4) return (int)std::max<int64_t>(1, std::min(most, (tile == 64 ? 768 : 512) / all));
      int best = 1;
      double least = 0;
      for (int n = 1; n <= std::min<int64_t>(most, 32); ++n) {
        const double rounds = std::max(1.5, (double)((all * n + 255) / 256));
        const double time = rounds / n * terms * 0.033 + (n > 1 ? 6 + 2.0 * all * n * tile * tile * sizeof(T) / 4.5e6 : 0);
        if (n == 1 || time < least) {
          least = time;
          best = n;
        }
      }
      return best;
    };
    a_splits = splits(square_tile, square, l);
    b_splits = splits(square_tile, square, s);
    x_splits = splits(x_tile, wide, s);
  }
  int64_t results() const {
    const int64_t a = (int64_t)square_tile * square_tile * square, x = (int64_t)x_tile * x_tile * wide;
    return std::max({a * (a_splits > 1 ? a_splits : 0), a * (b_splits > 1 ? b_splits : 0), x * (x_splits > 1 ? x_splits : 0)});
  }
  size_t x_size() const { return s * l * Stored<T>::kBytes; }
  size_t a_size() const { return s * s * Stored<T>::kBytes; }
};

template <class T>
size_t workspace_bytes(int64_t batch, int64_t m, int64_t n) {
  if (std::min(m, n) <= kMostRows) {
    const Few f(m, n, sizeof(T) == 8);
    if (f.chunks == 1) return 0;
    return up(batch * f.chunks * sizeof(Size)) + up(batch * f.x_size() * sizeof(T)) + 2 * up(batch * f.a_size() * sizeof(T)) + up(batch * f.sum_size() * sizeof(T));
  }
  const Many<T> f(batch, m, n);
  return up(batch * shares_of(m, n) * sizeof(Size)) + 4 * up(batch * f.x_size()) + 2 * up(batch * f.a_size()) + up(batch * f.results() * sizeof(T));
}

template <class T, int kTile>
hipError_t product_of(const OrthArgs& a, const Product& p, T* part, hipStream_t st) {
  hipError_t e = in_launches(a.batch, (int64_t)p.tiles * p.splits, [&](int64_t first, dim3 grid) { k_orth_product<T, kTile><<<grid, kProductThreads, 0, st>>>(a, p, first, part); });
  if (e != hipSuccess || p.splits == 1) return e;
  return in_launches(a.batch, (int64_t)p.tiles * (kTile / 32), [&](int64_t first, dim3 grid) { k_orth_finish<T, kTile><<<grid, kProductThreads, 0, st>>>(a, p, first, part); });
}

template <class T>
hipError_t product(const OrthArgs& a, const Product& p, int tile, T* part, hipStream_t st) {
  if constexpr (sizeof(T) == 4)
    if (tile == 128) return product_of<T, 128>(a, p, part, st);
  return product_of<T, 64>(a, p, part, st);
}

template <class T>
hipError_t many_rows(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  const Many<T> f(a.batch, a.m, a.n);
  const int shares = shares_of(a.m, a.n), s = (int)f.s, l = (int)f.l;
  Size* part = (Size*)ws;
  auto next = [&, at = ws + up(a.batch * shares * sizeof(Size))](size_t bytes) mutable {
    char* p = at;
    at += up(a.batch * bytes);
    return p;
  };
  char *X = next(f.x_size()), *XT = next(f.x_size()), *other = next(f.x_size()), *other_t = next(f.x_size()), *A = next(f.a_size()), *B = next(f.a_size());
  T* sums = (T*)next(f.results() * sizeof(T));
  hipError_t e = in_launches(a.batch, shares, [&](int64_t first, dim3 grid) { k_orth_squares<T><<<grid, kProductThreads, 0, st>>>(a, first, shares, part); });
  if (e != hipSuccess) return e;
  const int64_t blocks = f.s / kBlock * (f.l / kBlock);
  e = in_launches(a.batch, blocks, [&](int64_t first, dim3 grid) { k_orth_start<T><<<grid, kProductThreads, 0, st>>>(a, first, (int)blocks, s, l, shares, part, X, XT); });
  for (int i = 0; i < steps && e == hipSuccess; ++i) {
    const double* c = coefficients + 3 * i;
    e = product<T>(a, {X, X, nullptr, A, nullptr, s, s, l, (int)f.square, f.a_splits, 0, 1, true, false}, f.square_tile, sums, st);
    if (e == hipSuccess) e = product<T>(a, {A, A, A, B, nullptr, s, s, s, (int)f.square, f.b_splits, c[1], c[2], true, false}, f.square_tile, sums, st);
    if (e == hipSuccess) e = product<T>(a, {B, XT, X, other, other_t, s, l, s, (int)f.wide, f.x_splits, c[0], 1, false, i + 1 == steps}, f.x_tile, sums, st);
    std::swap(X, other);
    std::swap(XT, other_t);
  }
  return e;
}

template <class T, int kS, int NT, int kWaves>
hipError_t few_rows(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  const Few f(a.m, a.n, sizeof(T) == 8);
  constexpr int kWide = 16 * NT * kWaves;
  if constexpr (kS <= kWide)      // else there is more than one chunk
    if (f.chunks == 1) {
      Schedule schedule = {};
      for (int i = 0; i < 3 * steps; ++i) schedule.c[i / 3][i % 3] = coefficients[i];
      return in_launches(a.batch, 1, [&](int64_t first, dim3 grid) { k_orth_whole<T, kS, NT, kWaves><<<grid, 64 * kWaves, 0, st>>>(a, first, steps, schedule); });
    }
  if constexpr (sizeof(T) == 4 && kWide == 64) return hipErrorInvalidValue;      // more than 64 columns go by 128
  else {
  const int chunks = (int)f.chunks;
  Size* chunk = (Size*)ws;
  T* X = (T*)(ws + up(a.batch * chunks * sizeof(Size)));
  T* A = (T*)((char*)X + up(a.batch * f.x_size() * sizeof(T)));
  T* next = (T*)((char*)A + up(a.batch * f.a_size() * sizeof(T)));
  T* sum = (T*)((char*)next + up(a.batch * f.a_size() * sizeof(T)));
  hipError_t e = in_launches(a.batch, chunks, [&](int64_t first, dim3 grid) { k_orth_begin<T, kS, NT, kWaves><<<grid, 64 * kWaves, 0, st>>>(a, first, chunks, chunk, X, A); });
  for (int i = 0; i < steps && e == hipSuccess; ++i) {
    const double* c = coefficients + 3 * i;
    const T* from = A;
    const Size* start = i ? nullptr : chunk;
    int parts = chunks;
    if (f.join) {
      constexpr int kBlocks = kS * kS / 32;
      e = in_launches(a.batch, kBlocks, [&](int64_t first, dim3 grid) { k_orth_join<T><<<grid, kProductThreads, 0, st>>>(a, first, kBlocks, chunks, kS * kS, start, A, sum); });
      if (e != hipSuccess) break;
      from = sum;
      parts = 1;
    }
    e = in_launches(a.batch, chunks, [&](int64_t first, dim3 grid) {
      if (i + 1 < steps) k_orth_step<T, kS, NT, kWaves, false><<<grid, 64 * kWaves, 0, st>>>(a, first, chunks, parts, (T)c[0], (T)c[1], (T)c[2], start, X, from, next);
      else k_orth_step<T, kS, NT, kWaves, true><<<grid, 64 * kWaves, 0, st>>>(a, first, chunks, parts, (T)c[0], (T)c[1], (T)c[2], start, X, from, next);
    });
    std::swap(A, next);
  }
  return e;
  }
}

template <class T>
hipError_t orthogonalise(const OrthArgs& a, const double* coefficients, int steps, char* ws, hipStream_t st) {
  if (std::min(a.m, a.n) <= kMostRows) {
    const Few f(a.m, a.n, sizeof(T) == 8);
    auto go = [&](auto rows) {
      constexpr int kS = decltype(rows)::value;
      if constexpr (sizeof(T) == 8) return few_rows<T, kS, 1, 4>(a, coefficients, steps, ws, st);
      // 128 columns: eight waves of 16 each (89 of 128 x 128 74 us, four of 32 each 86), of 32 rows four of 32; there are no more rows than columns
      else if constexpr (kS == 32) return f.wide == 128 ? few_rows<T, kS, 2, 4>(a, coefficients, steps, ws, st) : few_rows<T, kS, 1, 4>(a, coefficients, steps, ws, st);
      else if constexpr (kS == 64) return f.wide == 128 ? few_rows<T, kS, 1, 8>(a, coefficients, steps, ws, st) : few_rows<T, kS, 1, 4>(a, coefficients, steps, ws, st);
      else return few_rows<T, kS, 1, 8>(a, coefficients, steps, ws, st);
    };
    switch (f.rows) {
      case 32: return go(std::integral_constant<int, 32>());
      case 64: return go(std::integral_constant<int, 64>());
      case 96: return go(std::integral_constant<int, 96>());
      default: return go(std::integral_constant<int, 128>());
    }
  }
  return many_rows<T>(a, coefficients, steps, ws, st);
}

}  // namespace
}  // namespace cgtp
