// Kernels of the group normalisation: the segments as constants in front of a text that is the same for all of them.
//
// A unit is one group of one segment, with the group of its gates if it has any: units of a sample depend on nothing of each other.
// With xh = (x - mu) r (mu = 0 unless the segment is 0e), M numbers in a unit of a sample, q = sigmoid(wg xh_g + bg):
//   0e:      y = act(w xh + b)         l = dE/d(w xh + b) = gy act'
//   others:  y = w xh q                l = gy q;  gates: l_g = q (1 - q) sum_m gy w xh
//   gw = sum l xh, gb = sum l, h = w l,  gx = r (h - [0e, gates: mean(h)] - xh mean(h xh))
#include <algorithm>
#include <sstream>

#include "norm.hpp"

namespace cgtp {
namespace {

const char kShared[] = R"HIP(
// All of it is one function: from some size on (32 segments) the compiler would leave calls, whose arguments lie in private memory.
#define ALWAYS __attribute__((always_inline))
#define INLINE __device__ ALWAYS inline
typedef long long i64;
INLINE float fma_(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
INLINE double fma_(double a, double b, double c) { return __builtin_fma(a, b, c); }
// off by |t| half steps where t is negative: at most 0.3 half steps of 1 (as the gated block's, act.hpp, for the same reason)
INLINE float sigmoid_(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t * -1.44269502f)); }
INLINE double sigmoid_(double t) { return 1.0 / (1.0 + exp(-t)); }
INLINE float erfc_(float t) { return erfcf(t); }
INLINE double erfc_(double t) { return erfc(t); }
INLINE float exp_(float t) { return expf(t); }
INLINE double exp_(double t) { return exp(t); }
// 1 - 2 / (1 + exp(2 |t|)), near zero five terms of the series
INLINE float tanh_(float t) {
  const float s = t * t, x = __builtin_fabsf(t);
  const float p = fma_(t * s, fma_(s, fma_(s, fma_(s, 0.0218694885f, -0.0539682540f), 0.133333333f), -0.333333333f), t);
  const float q = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * 2.88539008f));
  return x < 0.25f ? p : __builtin_copysignf(q, t);
}
INLINE double tanh_(double t) { return tanh(t); }
INLINE float sqrt_(float t) { return sqrtf(t); }
INLINE double sqrt_(double t) { return sqrt(t); }

// activation and derivative
INLINE void act_(T t, T& a, T& d) {
  if constexpr (ACT == 0) {
    a = t;
    d = T(1);
  } else if constexpr (ACT == 1) {
    const T q = sigmoid_(t);
    a = t * q;
    d = fma_(a, T(1) - q, q);
  } else if constexpr (ACT == 2) {
    const T p = T(0.5) * erfc_(t * T(-0.70710678118654752440));
    a = t * p;
    d = fma_(t, T(0.39894228040143267794) * exp_(T(-0.5) * t * t), p);
  } else if constexpr (ACT == 3) {
    a = sigmoid_(t);
    d = a * (T(1) - a);
  } else {
    a = tanh_(t);
    d = T(1) - a * a;
  }
}

// column of component m of channel c, counted from the segment's first
template <int s> INLINE int at_(int c, int m) { return IR_MUL ? m * SEG[s].mul + c : c * SEG[s].n + m; }

struct Stat { T mu, r, gmu, gr; };       // of a unit and of its gates
struct Param { T w, b, gw, gb; };        // of a channel and of its gate

template <int s> INLINE Param param_(const T* __restrict__ weight, const T* __restrict__ bias, int c) {
  Param p = {weight[SEG[s].w + c], T(0), T(0), T(0)};
  if constexpr (SEG[s].inv) p.b = bias[SEG[s].b + c];
  if constexpr (SEG[s].gate >= 0) {
    p.gw = weight[SEG[s].gw + c];
    p.gb = bias[SEG[s].gb + c];
  }
  return p;
}

// one channel of one row, its n components in v and its gate in g, normalised: y in place of v
template <int s> INLINE void forward_(T* v, T g, const Stat& S, const Param& p) {
  if constexpr (SEG[s].inv) {
    T d;
    act_(fma_(p.w, (v[0] - S.mu) * S.r, p.b), v[0], d);
  } else {
    T f = S.r * p.w;
    if constexpr (SEG[s].gate >= 0) f *= sigmoid_(fma_(p.gw, (g - S.gmu) * S.gr, p.gb));
#pragma unroll
    for (int m = 0; m < SEG[s].n; ++m) v[m] *= f;
  }
}

// what a channel of a row adds to the sums of the backward pass
struct Sums { T w, b, gw, gb, h, hx, gh, ghx; };

// v, g in: the channel's numbers of x; q: of gy.  Out: v, g as xh, and q, qg as h
template <int s> INLINE Sums backward_(T* v, T& g, T* q, T& qg, const Stat& S, const Param& p) {
  Sums o = {};
  if constexpr (SEG[s].inv) {
    T a, d;
    v[0] = (v[0] - S.mu) * S.r;
    act_(fma_(p.w, v[0], p.b), a, d);
    const T l = q[0] * d;
    o.w = l * v[0];
    o.b = l;
    q[0] = l * p.w;
    o.h = q[0];
    o.hx = q[0] * v[0];
  } else {
    T dot = T(0), f = T(1);
#pragma unroll
    for (int m = 0; m < SEG[s].n; ++m) {
      v[m] *= S.r;
      dot = fma_(q[m], v[m], dot);
    }
    if constexpr (SEG[s].gate >= 0) {
      g = (g - S.gmu) * S.gr;
      f = sigmoid_(fma_(p.gw, g, p.gb));
      const T l = dot * p.w * f * (T(1) - f);
      o.gw = l * g;
      o.gb = l;
      qg = l * p.gw;
      o.gh = qg;
      o.ghx = qg * g;
    }
    o.w = dot * f;
    o.hx = o.w * p.w;
#pragma unroll
    for (int m = 0; m < SEG[s].n; ++m) q[m] *= f * p.w;
  }
  return o;
}

struct Means { T h, hx, gh, ghx; };   // of a unit of a sample

// gx of a channel, from what backward_ left, in place of q and qg
template <int s> INLINE void finish_(const T* v, T g, T* q, T& qg, const Stat& S, const Means& e) {
#pragma unroll
  for (int m = 0; m < SEG[s].n; ++m) q[m] = S.r * (q[m] - (SEG[s].inv ? e.h : T(0)) - v[m] * e.hx);
  if constexpr (SEG[s].gate >= 0) qg = S.gr * (qg - e.gh - g * e.ghx);
}

// rows of sample s, within [0, N]
INLINE void range_(const i64* __restrict__ ptr, i64 s, i64 N, i64& r0, i64& r1) {
  r0 = ptr ? ptr[s] : s;
  r1 = ptr ? ptr[s + 1] : s + 1;
  r0 = r0 < 0 ? 0 : r0 > N ? N : r0;
  r1 = r1 < r0 ? r0 : r1 > N ? N : r1;
}

constexpr int pow2_(int v) { int p = 1; while (p < v) p *= 2; return p; }

// f<s>() for a number s that all lanes share
template <int s, class F> INLINE void with_segment_(int k, F f) {
  if constexpr (s + 1 < NS) {
    if (k != s) return with_segment_<s + 1>(k, f);
  }
  f.template operator()<s>();
}

// sum over the workgroup, the same in every thread; the order is fixed
INLINE double block_sum_(double v, double* lds) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
)HIP";

// ---- a wave's lanes over a segment ----
//
// A lane has V J channels of one group: (j L + li) V + k, li < L its place among the group's L lanes.  A wave takes GP groups and RP rows a step; the
// groups of a segment take PH phases of GP.  All of a segment's words of a step stay in registers.
const char kLanes[] = R"HIP(
// sum over the L lanes of a group, the same in each of them; the order is fixed
template <int ctrl> INLINE float dpp_(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), ctrl, 0xf, 0xf, false)); }
template <int ctrl> INLINE double dpp_(double v) {
  const long long b = __builtin_bit_cast(long long, v);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, ctrl, 0xf, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), ctrl, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (long long)(((unsigned long long)(unsigned)hi << 32) | (unsigned)lo));
}
template <int L, class X> INLINE X lanes_sum_(X v) {
  if constexpr (L > 1) v += dpp_<0xB1>(v);     // neighbour
  if constexpr (L > 2) v += dpp_<0x4E>(v);     // other pair
  if constexpr (L > 4) v += dpp_<0x141>(v);    // the other four, mirrored (within four all are alike by now)
  if constexpr (L > 8) v += dpp_<0x140>(v);
  if constexpr (L > 16) v += __shfl_xor(v, 16);
  if constexpr (L > 32) v += __shfl_xor(v, 32);
  return v;
}

template <int w> struct Wide_ { typedef T type __attribute__((ext_vector_type(w))); };
// w words that are neighbours in memory
template <int w, bool vec> INLINE void get_(const T* p, T* v) {
  if constexpr (vec && w % 4 == 0) {
#pragma unroll
    for (int i = 0; i < w; i += 4) {
      const typename Wide_<4>::type q = *(const typename Wide_<4>::type*)(p + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i + k] = q[k];
    }
  } else if constexpr (vec && w % 2 == 0) {
#pragma unroll
    for (int i = 0; i < w; i += 2) {
      const typename Wide_<2>::type q = *(const typename Wide_<2>::type*)(p + i);
      v[i] = q[0];
      v[i + 1] = q[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < w; ++i) v[i] = p[i];
  }
}
// Results are written past the caches: nothing here reads them again (20 000 rows as above, forward 80 -> 65 us; one graph of them 341 -> 308).  Not where a
// lane's words are neighbours and so many that each instruction writes little of a line (Lane::past): 10 000 rows of 256x3o fp64 in MUL_IR, forward 168 past
// the caches, 72 through them, 20 000 rows of 64x8e fp32 80 and 40, of 512x3o 163 and 117; of 128 channels, l <= 3, 71 and 96.
#define ST(a, b) __builtin_nontemporal_store(b, &(a))
template <int w, bool vec, bool past> INLINE void put_(T* p, const T* v) {
  if constexpr (vec && w % 4 == 0) {
#pragma unroll
    for (int i = 0; i < w; i += 4) { typename Wide_<4>::type q = {v[i], v[i + 1], v[i + 2], v[i + 3]}; ST(*(typename Wide_<4>::type*)(p + i), q); }
  } else if constexpr (vec && w % 2 == 0) {
#pragma unroll
    for (int i = 0; i < w; i += 2) { typename Wide_<2>::type q = {v[i], v[i + 1]}; ST(*(typename Wide_<2>::type*)(p + i), q); }
  } else {
#pragma unroll
    for (int i = 0; i < w; ++i) {
      if constexpr (past) ST(p[i], v[i]);
      else p[i] = v[i];
    }
  }
}

template <int s> struct Lane {
  static constexpr int n = SEG[s].n, V = SEG[s].V, J = SEG[s].J, L = SEG[s].lanes, GP = SEG[s].at_once, RP = SEG[s].rows, cg = SEG[s].mul / G, C = V * J;
  static constexpr bool gated = SEG[s].gate >= 0, inv = SEG[s].inv, vec = SEG[s].vec, full = L * C == cg;
  static constexpr bool past = IR_MUL || n == 1 || (n * sizeof(T) <= 32 && J * n * sizeof(T) <= 192);
  int li, gq, rho, g;       // place in the group, group of the step, row of the step, group
  bool on;                  // lanes that are left over repeat the first row's
  INLINE Lane(int phase) {
    const int lane = threadIdx.x & 63, at = lane / L;
    on = at < GP * RP;
    li = lane % L;
    gq = at % GP;
    rho = on ? at / GP : 0;
    g = phase * GP + gq;
  }
  INLINE bool has(int j) const { return full || (j * L + li) * V < cg; }
  INLINE int channel(int j) const { return g * cg + (full || (j * L + li) * V < cg ? (j * L + li) * V : 0); }
  // words of channels channel(j) + k, component m at v[(j V + k) n + m]; base: the row's first word of the segment
  INLINE void read(const T* base, T* v) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if constexpr (IR_MUL) {
#pragma unroll
        for (int m = 0; m < n; ++m) {
          T w[V];
          get_<V, vec>(base + m * SEG[s].mul + channel(j), w);
#pragma unroll
          for (int k = 0; k < V; ++k) v[(j * V + k) * n + m] = w[k];
        }
      } else {
        get_<V * n, vec>(base + channel(j) * n, v + j * V * n);
      }
    }
  }
  INLINE void write(T* base, const T* v) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (!has(j)) continue;
      if constexpr (IR_MUL) {
#pragma unroll
        for (int m = 0; m < n; ++m) {
          T w[V];
#pragma unroll
          for (int k = 0; k < V; ++k) w[k] = v[(j * V + k) * n + m];
          put_<V, vec, true>(base + m * SEG[s].mul + channel(j), w);
        }
      } else {
        put_<V * n, vec, past>(base + channel(j) * n, v + j * V * n);
      }
    }
  }
  INLINE void read_gates(const T* row, T* g_) const {
    if constexpr (gated) {
#pragma unroll
      for (int j = 0; j < J; ++j) get_<V, vec>(row + SEG[s].gate + channel(j), g_ + j * V);
    }
  }
  INLINE void write_gates(T* row, const T* g_) const {
    if constexpr (gated) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (has(j)) put_<V, vec, true>(row + SEG[s].gate + channel(j), g_ + j * V);
    }
  }
  INLINE void params(const T* __restrict__ weight, const T* __restrict__ bias, Param* p) const {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) p[j * V + k] = param_<s>(weight, bias, channel(j) + k);
  }
  INLINE Stat stat(const T* __restrict__ st) const {
    Stat S = {st[(SEG[s].st * G + g) * 2], st[(SEG[s].st * G + g) * 2 + 1], T(0), T(0)};
    if constexpr (gated) {
      S.gmu = st[(SEG[s].gst * G + g) * 2];
      S.gr = st[(SEG[s].gst * G + g) * 2 + 1];
    }
    return S;
  }
  INLINE void put_stat(T* st, const Stat& S) const {
    st[(SEG[s].st * G + g) * 2] = S.mu;
    st[(SEG[s].st * G + g) * 2 + 1] = S.r;
    if constexpr (gated) {
      st[(SEG[s].gst * G + g) * 2] = S.gmu;
      st[(SEG[s].gst * G + g) * 2 + 1] = S.gr;
    }
  }
  // y of the words in v, in their place
  INLINE void forward(T* v, const T* g_, const Stat& S, const Param* p) const {
#pragma unroll
    for (int c = 0; c < C; ++c) forward_<s>(v + c * n, gated ? g_[c] : T(0), S, p[c]);
  }
  // v, g_: of x, then xh; q: of gy, then h; qg: h of the gates.  Adds to the sums of the channels (a) and of the group (o)
  struct Sum { double w[C], b[C], gw[C], gb[C]; };
  INLINE Sums backward(T* v, T* g_, T* q, T* qg, const Stat& S, const Param* p, bool in, bool add, Sum& a) const {
    Sums o = {};
#pragma unroll
    for (int c = 0; c < C; ++c) {
      T none = T(0), none_q = T(0);
      const Sums t = backward_<s>(v + c * n, gated ? g_[c] : none, q + c * n, gated ? qg[c] : none_q, S, p[c]);
      const bool count = in && has(c / V);
      o.h += count ? t.h : T(0);
      o.hx += count ? t.hx : T(0);
      o.gh += count ? t.gh : T(0);
      o.ghx += count ? t.ghx : T(0);
      if (add) {
        a.w[c] += count ? (double)t.w : 0.0;
        if (inv) a.b[c] += count ? (double)t.b : 0.0;
        if (gated) {
          a.gw[c] += count ? (double)t.gw : 0.0;
          a.gb[c] += count ? (double)t.gb : 0.0;
        }
      }
    }
    return o;
  }
  INLINE void finish(const T* v, const T* g_, T* q, T* qg, const Stat& S, const Means& e) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      T none = T(0);
      finish_<s>(v + c * n, gated ? g_[c] : none, q + c * n, gated ? qg[c] : none, S, e);
    }
  }
  // whether the rows of a step are added by shuffles: they are 64 / RP lanes apart
  static constexpr bool even = (GP * L & (GP * L - 1)) == 0;
  static INLINE double rows_sum(double v) {
    if constexpr (even)
#pragma unroll
      for (int o = GP * L; o < 64; o *= 2) v += __shfl_xor(v, o);
    return v;
  }
  // the workgroup's sums of the channels' gradients, four at a time, one for each wave to add up: into a row of partial sums, or, of the only
  // workgroup of its channels, into gweight and gbias
  // any: whether there is anything in them (the workgroup's)
  INLINE void put_sums(const Sum& a, bool any, double* to, T* gweight, T* gbias, double* lds) const {
    constexpr int kinds = 1 + (inv ? 1 : 0) + (gated ? 2 : 0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    auto put = [&](int i, double t) ALWAYS {
      const int c = i / kinds, k = i % kinds;
      const bool b = inv ? k == 1 : k == 2;
      const int at = (k == 0 ? SEG[s].w : inv ? SEG[s].b : k == 1 ? SEG[s].gw : SEG[s].gb) + channel(c / V) + c % V;
      if (to) to[b ? NW + at : at] = t;
      else (b ? gbias : gweight)[at] = (T)t;
    };
    if (!any) {
      for (int i = wave; i < C * kinds; i += 4)
        if (lane < GP * L && has(i / kinds / V)) put(i, 0.0);
      return;
    }
#pragma unroll
    for (int first = 0; first < C * kinds; first += 4) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (first + i >= C * kinds) break;
        const int c = (first + i) / kinds, k = (first + i) % kinds;
        const double v = k == 0 ? a.w[c] : inv ? a.b[c] : k == 1 ? a.gw[c] : a.gb[c];
        lds[i * 256 + threadIdx.x] = rows_sum(on ? v : 0.0);
      }
      __syncthreads();
      if (first + wave < C * kinds && lane < GP * L && has((first + wave) / kinds / V)) {     // a lane of the step's first row
        double t = 0;
        for (int w = 0; w < 4; ++w)
          for (int r = 0; r < (even ? 1 : RP); ++r) t += lds[wave * 256 + w * 64 + r * GP * L + lane];
        put(first + wave, t);
      }
    }
  }
};

// what a sub-unit (a phase of a segment) is: SUB in the order of their size, the largest first
template <class F> INLINE void with_sub_(int u, F f) { with_segment_<0>(SUB[u].s, f); }
INLINE int sub_() { return blockIdx.x % NSUB; }
INLINE i64 part_() { return blockIdx.x / NSUB; }
)HIP";

// Every row is a sample: a group's numbers of a row are in the registers of its lanes, read once.  Sums in T: trees of at most 64 words a lane
// and six levels.  Bound by memory: 20 000 rows of 128 channels, l <= 3 with gates (359 MB forward, 554 MB backward), IR_MUL forward 65 to 75 us (4.8 to
// 5.5 TB/s, a copy 4.95), MUL_IR forward and backward 207 to 223 us (4.1 to 4.4 TB/s).  Backward keeps the sums of its channels over all its rows in
// registers: as many workgroups as stay on the chip, one row of partial sums each.
const char kRowFwd[] = R"HIP(
struct RowFwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; T* __restrict__ y; T* __restrict__ stats; i64 N; int phase;
  template <int s> INLINE void operator()() const {
    typedef Lane<s> A;
    const A a(phase);
    const i64 waves = (gridDim.x / NSUB) * 4;
    Param p[A::C];
    a.params(weight, bias, p);
    for (i64 base = (part_() * 4 + threadIdx.x / 64) * A::RP; base < N; base += waves * A::RP) {
      const bool in = a.on && base + a.rho < N;
      const i64 r = base + a.rho < N ? base + a.rho : N - 1;
      T v[A::C * A::n], g[A::C];
      a.read(x + r * DX + SEG[s].col, v);
      a.read_gates(x + r * DX, g);
      Stat S = {T(0), T(0), T(0), T(0)};
      auto moments = [&](const T* w, int words, bool centre, T inv_m, T& mu, T& rs) ALWAYS {
        if (centre) {
          T t = T(0);
#pragma unroll
          for (int i = 0; i < words; ++i) t += A::full || a.has(i / (words / A::J)) ? w[i] : T(0);
          mu = lanes_sum_<A::L>(t) * inv_m;
        }
        T t = T(0);
#pragma unroll
        for (int i = 0; i < words; ++i) {
          const T d = w[i] - mu;
          t = fma_(A::full || a.has(i / (words / A::J)) ? d : T(0), d, t);
        }
        rs = T(1) / sqrt_(fma_(lanes_sum_<A::L>(t), inv_m, T(EPS)));
      };
      moments(v, A::C * A::n, A::inv, T(1.0 / (A::cg * A::n)), S.mu, S.r);
      if constexpr (A::gated) moments(g, A::C, true, T(1.0 / A::cg), S.gmu, S.gr);
      a.forward(v, g, S, p);
      if (in) {
        a.write(y + r * DY + SEG[s].ycol, v);
        if (stats && a.li == 0) a.put_stat(stats + r * NST, S);
      }
    }
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_row_fwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                                T* __restrict__ y, T* __restrict__ stats, i64 N) {
  with_sub_(sub_(), RowFwd{x, weight, bias, y, stats, N, SUB[sub_()].phase});
}
)HIP";

const char kRowBwd[] = R"HIP(
struct RowBwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; const T* __restrict__ gy; const T* __restrict__ stats;
  T* __restrict__ gx; double* __restrict__ sums; T* __restrict__ gweight; T* __restrict__ gbias; i64 N; int phase; double* lds;
  template <int s> INLINE void operator()() const {
    typedef Lane<s> A;
    const A a(phase);
    const i64 waves = (gridDim.x / NSUB) * 4;
    Param p[A::C];
    a.params(weight, bias, p);
    typename A::Sum sum = {};
    for (i64 base = (part_() * 4 + threadIdx.x / 64) * A::RP; base < N; base += waves * A::RP) {
      const bool in = a.on && base + a.rho < N;
      const i64 r = base + a.rho < N ? base + a.rho : N - 1;
      T v[A::C * A::n], q[A::C * A::n], g[A::C], qg[A::C];
      a.read(x + r * DX + SEG[s].col, v);
      a.read(gy + r * DY + SEG[s].ycol, q);
      a.read_gates(x + r * DX, g);
      const Stat S = a.stat(stats + r * NST);
      const Sums o = a.backward(v, g, q, qg, S, p, in, true, sum);
      Means e = {T(0), lanes_sum_<A::L>(o.hx) * T(1.0 / (A::cg * A::n)), T(0), T(0)};
      if constexpr (A::inv) e.h = lanes_sum_<A::L>(o.h) * T(1.0 / A::cg);
      if constexpr (A::gated) {
        e.gh = lanes_sum_<A::L>(o.gh) * T(1.0 / A::cg);
        e.ghx = lanes_sum_<A::L>(o.ghx) * T(1.0 / A::cg);
      }
      a.finish(v, g, q, qg, S, e);
      if (in) {
        a.write(gx + r * DX + SEG[s].col, q);
        a.write_gates(gx + r * DX, qg);
      }
    }
    a.put_sums(sum, true, sums ? sums + part_() * (NW + NB) : nullptr, gweight, gbias, lds);
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_row_bwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                                const T* __restrict__ gy, const T* __restrict__ stats, T* __restrict__ gx,
                                                                double* __restrict__ sums, T* __restrict__ gweight, T* __restrict__ gbias, i64 N) {
  __shared__ double lds[1024];
  with_sub_(sub_(), RowBwd{x, weight, bias, gy, stats, gx, sums, gweight, gbias, N, SUB[sub_()].phase, lds});
}
)HIP";

// Samples of any number of rows.  The rows are cut into chunks of D; a workgroup has a sub-unit of a chunk.  A sample of at most R rows (R >= D) belongs to the
// chunk of its first row: its sums are formed and its results written by one workgroup, from registers if it fits one step.  Longer samples take a second
// kernel, which is launched only if N > R: the first leaves the sums of each chunk's share (a chunk has at most two: one that goes on, slot 0, one
// that begins, slot 1), the second adds up the shares of a sample, each workgroup for its groups, and writes the results.  Sums over rows are held
// in 64 bits; those of fp64 are of the distance from one of the group's numbers (shift_), for their variance.
// Bound, with short samples, by the chain of a sample's steps (ptr, rows, sums through LDS, results), which the other workgroups of a unit hide in part: 500
// samples in 12 000 rows of 32 channels, l <= 3, forward 20 to 29 us (2.7 to 1.9 TB/s), backward 36 (2.3); with a sample a wave instead of a workgroup no faster.
// Long ones: by memory, which is read twice (no chip-wide barrier): one sample of 20 000 rows of 128 channels 118 and 199 us, the second kernel going through
// the chunks from the last on, which are still in the caches.
const char kGraphs[] = R"HIP(
INLINE i64 inside_(i64 p, i64 N) { return p < 0 ? 0 : p > N ? N : p; }

// number of i < S with ptr[i] < row (ptr not decreasing), by all 64 lanes of every wave: 64 probes a step
INLINE i64 first_from_(const i64* __restrict__ ptr, i64 S, i64 N, i64 row) {
  const int lane = threadIdx.x & 63;
  i64 lo = 0, hi = S;     // the answer is in [lo, hi]
  while (lo < hi) {
    const i64 step = (hi - lo + 63) / 64, at = lo + lane * step;
    const bool less = at < hi && inside_(ptr[at], N) < row;
    const int c = __popcll(__ballot(less));     // probes 0 .. c - 1 are below
    if (c == 0) return lo;
    const i64 l = lo + (i64)(c - 1) * step + 1, h = lo + (i64)c * step;
    hi = h < hi ? h : hi;
    lo = l;
  }
  return lo;
}

// lane i's number; i is the same in all lanes
INLINE i64 lane_of_(i64 v, int i) {
  const unsigned lo = __builtin_amdgcn_readlane((int)v, i), hi = __builtin_amdgcn_readlane((int)(v >> 32), i);
  return (i64)((unsigned long long)hi << 32 | lo);
}

struct Chunks {
  const i64* __restrict__ ptr;
  i64 N, S, R, D, chunk;
  // f() for each chunk of the workgroup; back: from the last one on
  template <class F> INLINE void all(bool back, F f) {
    const i64 n = N > 0 ? (N + D - 1) / D : 1;
    for (i64 c = part_(); c < n; c += gridDim.x / NSUB) {
      chunk = back ? n - 1 - c : c;
      f();
    }
  }
  // the samples of the chunk: f(sample, first row, end, from, to, slot): the whole of a short one (slot -1), or a long one's rows in this chunk;
  // none(sample, end): neighbours without rows
  template <class F, class E> INLINE void each(F f, E none) const {
    const i64 a = chunk * D, b = a + D < N ? a + D : N;
    const bool last = a + D >= N;
    i64 s = first_from_(ptr, S, N, a), from = -64, p = 0;      // p: a lane's number of ptr, from `from` on
    bool goes_on = s > 0;       // the one before may reach into the chunk
    for (s -= goes_on; s < S; ++s, goes_on = false) {
      if (s - from > 62) {
        const i64 i = s + (threadIdx.x & 63);
        from = s;
        p = inside_(ptr[i < S ? i : S], N);
      }
      const i64 r0 = lane_of_(p, (int)(s - from)), e = lane_of_(p, (int)(s - from) + 1), r1 = e < r0 ? r0 : e;
      const bool is_long = r1 - r0 > R;
      if (goes_on && (!is_long || r1 <= a)) continue;
      if (!goes_on && (r0 < a || (r0 >= b && !(last && r0 == N)))) break;
      if (r1 == r0) {     // those behind it that begin at its row, but for the last, have no rows either
        const i64 next = first_from_(ptr, S, N, r0 + 1) - 1, until = next > s ? next : s + 1;
        none(s, until);
        s = until - 1;
        continue;
      }
      f(s, r0, r1, goes_on ? a : r0, is_long && r1 > b ? b : r1, is_long ? !goes_on : -1);
    }
  }
  // place of a share of a unit's sums
  INLINE i64 share(i64 c, int slot, int s, int g) const { return (((c * 2 + slot) * NS + s) * G + g) * 4; }
  // the sums of all shares of a long sample for the lane's group, by the workgroup: 256 / GP threads a group.  They stay in LDS for the sample's other chunks
  // (`known`): formed for each chunk they are work that grows with the square of the sample's length
  template <class A, int s> INLINE void total(const A& a, const double* __restrict__ part, i64 sample, i64 r0, i64 r1, i64& known, double (&t)[4], double* lds) const {
    if (sample != known) form<A, s>(a, part, r0, r1, lds);
    known = sample;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = lds[a.gq * 4 + i];
  }
  template <class A, int s> INLINE void form(const A& a, const double* __restrict__ part, i64 r0, i64 r1, double* lds) const {
    constexpr int per = A::GP < 256 ? 256 / A::GP : 1;      // threads a group
    const i64 c0 = r0 / D, end = (r1 - 1) / D;
    __syncthreads();
    if ((int)threadIdx.x < per * A::GP) {
      const int gq = threadIdx.x % A::GP, g = a.g - a.gq + gq;
      double v[4] = {};
      for (i64 c = c0 + threadIdx.x / A::GP; c <= end; c += per) {
        const double* p = part + share(c, c == c0, s, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += p[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) lds[threadIdx.x * 4 + i] = v[i];
    }
    __syncthreads();
    // a tree over the threads of a group, in a fixed order
    for (int m = per; m > 1;) {
      const int h = (m + 1) / 2;
      if ((int)threadIdx.x < (m - h) * A::GP)
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[threadIdx.x * 4 + i] += lds[(threadIdx.x + h * A::GP) * 4 + i];
      __syncthreads();
      m = h;
    }
  }
};

// sums of the lanes, rows and waves for each group of the step: four numbers
template <class A> INLINE void group_sums_(const A& a, double (&t)[4], double* lds) {
  constexpr int rows = A::even ? 1 : A::RP;
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = A::rows_sum(lanes_sum_<A::L>(t[i]));
  __syncthreads();
  if (a.on && a.li == 0 && a.rho < rows)
#pragma unroll
    for (int i = 0; i < 4; ++i) lds[(((threadIdx.x / 64) * rows + a.rho) * A::GP + a.gq) * 4 + i] = t[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t[i] = 0;
    for (int k = 0; k < 4 * rows; ++k) t[i] += lds[(k * A::GP + a.gq) * 4 + i];
  }
}

// What the moments are taken about.  fp64: the middle one of three numbers of the group, of the sample's first, middle and last row (about the first one alone, a
// number far from all others loses as many digits of the variance as the sample's size has).  fp32: zero, a square has 48 of the 53 bits that its sum is
// held in.
INLINE double middle_(double a, double b, double c) { return __builtin_fmax(__builtin_fmin(a, b), __builtin_fmin(__builtin_fmax(a, b), c)); }
struct Shift { double x, g; };
template <int s> INLINE Shift shift_(const Lane<s>& a, const T* __restrict__ x, i64 r0, i64 rows) {
  Shift h = {0, 0};
  if (sizeof(T) == 8 && rows > 0) {
    const T *first = x + r0 * DX + a.g * Lane<s>::cg, *mid = first + rows / 2 * DX, *last = first + (rows - 1) * DX;
    if (Lane<s>::inv) h.x = middle_(first[SEG[s].col], mid[SEG[s].col], last[SEG[s].col]);
    if (Lane<s>::gated) h.g = middle_(first[SEG[s].gate], mid[SEG[s].gate], last[SEG[s].gate]);
  }
  return h;
}
template <int s> INLINE void moments_(const Lane<s>& a, const T* v, const T* g, const Shift& h, bool in, double (&t)[4]) {
  typedef Lane<s> A;
#pragma unroll
  for (int c = 0; c < A::C; ++c) {
    const bool count = in && a.has(c / A::V);
#pragma unroll
    for (int m = 0; m < A::n; ++m) {
      const double d = count ? (double)v[c * A::n + m] - h.x : 0.0;
      if (A::inv) t[0] += d;
      t[1] = __builtin_fma(d, d, t[1]);
    }
    if constexpr (A::gated) {
      const double d = count ? (double)g[c] - h.g : 0.0;
      t[2] += d;
      t[3] = __builtin_fma(d, d, t[3]);
    }
  }
}
// 1 / sqrt(var + eps); a variance below zero by rounding is zero, a NaN stays one
INLINE T root_(double var) {
  const T v = (T)((var > 0 || var != var ? var : 0.0) + EPS);
  return T(1) / sqrt_(v);
}
template <int s> INLINE Stat stat_of_(const double (&t)[4], const Shift& h, i64 rows) {
  typedef Lane<s> A;
  const double inv = rows > 0 ? 1.0 / ((double)rows * A::cg) : 1.0, inv_n = inv * (1.0 / A::n);
  const double d = t[0] * inv_n, var = t[1] * inv_n - d * d;
  Stat S = {A::inv ? (T)(rows > 0 ? h.x + d : 0.0) : T(0), root_(var), T(0), T(0)};
  if constexpr (A::gated) {
    const double e = t[2] * inv;
    S.gmu = (T)(rows > 0 ? h.g + e : 0.0);
    S.gr = root_(t[3] * inv - e * e);
  }
  return S;
}

)HIP";

const char kGraphFwd[] = R"HIP(
// kLong: the second kernel
template <bool kLong> struct GraphFwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; T* __restrict__ y; T* __restrict__ stats; double* __restrict__ part;
  Chunks in; int phase; double* lds;
  template <int s> INLINE void operator()() const {
    typedef Lane<s> A;
    const A a(phase);
    Param p[A::C];
    if (!kLong) a.params(weight, bias, p);
    Chunks of = in;
    i64 known = -1;
    of.all(kLong /* what the first kernel read last is still near */, [&]() ALWAYS { of.each([&](i64 sample, i64 r0, i64 r1, i64 from, i64 to, int slot) ALWAYS {
      if (kLong && slot < 0) return;
      if (kLong) a.params(weight, bias, p);     // most workgroups find nothing long
      const i64 first = from + (threadIdx.x / 64) * A::RP;
      i64 base = first;
      T v[A::C * A::n], g[A::C];
      auto fetch = [&]() ALWAYS {
        const i64 r = base + a.rho < to ? base + a.rho : to - 1;
        a.read(x + r * DX + SEG[s].col, v);
        a.read_gates(x + r * DX, g);
      };
      const Shift h = shift_<s>(a, x, r0, r1 - r0);
      double t[4] = {};
      bool held = false;      // the last step's rows are in v, g
      if (kLong) {
        of.template total<A, s>(a, part, sample, r0, r1, known, t, lds);
        if (base < to) base += (to - 1 - base) / (4 * A::RP) * (4 * A::RP);
        else base -= 4 * A::RP;
      } else {
        for (; base < to; base += 4 * A::RP) {
          fetch();
          moments_<s>(a, v, g, h, a.on && base + a.rho < to, t);
        }
        group_sums_(a, t, lds);
        if (slot >= 0) {
          if (threadIdx.x < 64 && a.on && a.rho == 0 && a.li == 0)
            for (int i = 0; i < 4; ++i) part[of.share(of.chunk, slot, s, a.g) + i] = t[i];
          return;
        }
        base -= 4 * A::RP;
        held = true;
      }
      const Stat st = stat_of_<s>(t, h, r1 - r0);
      if (stats && slot != 0 && threadIdx.x < 64 && a.on && a.rho == 0 && a.li == 0) a.put_stat(stats + sample * NST, st);
      for (; base >= first; base -= 4 * A::RP) {
        if (!held) fetch();
        held = false;
        a.forward(v, g, st, p);
        if (a.on && base + a.rho < to) a.write(y + (base + a.rho) * DY + SEG[s].ycol, v);
      }
    }, [&](i64 sample, i64 end) ALWAYS {
      if (kLong || !stats) return;
      const double none[4] = {};
      const Stat st = stat_of_<s>(none, Shift{0, 0}, 0);
      A b = a;
      for (i64 i = threadIdx.x; i < (end - sample) * A::GP; i += 256) {
        b.g = phase * A::GP + (int)(i % A::GP);
        b.put_stat(stats + (sample + i / A::GP) * NST, st);
      }
    }); });
  }
};
#define GRAPH_FWD(name, kLong) \
  extern "C" __global__ void __launch_bounds__(256) name(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias, T* __restrict__ y, \
                                                         T* __restrict__ stats, double* __restrict__ part, const i64* __restrict__ ptr, i64 N, i64 S, i64 R, i64 D) { \
    __shared__ double lds[1024]; \
    with_sub_(sub_(), GraphFwd<kLong>{x, weight, bias, y, stats, part, Chunks{ptr, N, S, R, D, 0}, SUB[sub_()].phase, lds}); \
  }
GRAPH_FWD(cgtp_norm_graph_fwd, false)
GRAPH_FWD(cgtp_norm_long_fwd, true)
)HIP";

const char kGraphBwd[] = R"HIP(
template <int s> INLINE Means means_of_(const double (&t)[4], i64 rows) {
  const double inv = rows > 0 ? 1.0 / ((double)rows * Lane<s>::cg) : 1.0;
  return Means{(T)(t[0] * inv), (T)(t[1] * inv * (1.0 / Lane<s>::n)), (T)(t[2] * inv), (T)(t[3] * inv)};
}
// the parameters' gradients are summed where a row's results are written
template <bool kLong> struct GraphBwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; const T* __restrict__ gy; const T* __restrict__ stats; T* __restrict__ gx;
  double* __restrict__ part; double* __restrict__ sums; T* __restrict__ gweight; T* __restrict__ gbias; Chunks in; int phase; double* lds;
  template <int s> INLINE void operator()() const {
    typedef Lane<s> A;
    const A a(phase);
    Param p[A::C];
    if (!kLong) a.params(weight, bias, p);
    typename A::Sum sum = {};
    bool any = false;
    Chunks of = in;
    i64 known = -1;
    of.all(kLong, [&]() ALWAYS { of.each([&](i64 sample, i64 r0, i64 r1, i64 from, i64 to, int slot) ALWAYS {
      if (kLong && slot < 0) return;
      if (kLong) a.params(weight, bias, p);     // most workgroups find nothing long
      const i64 first = from + (threadIdx.x / 64) * A::RP;
      i64 base = first;
      any = true;
      const Stat st = a.stat(stats + sample * NST);
      T v[A::C * A::n], q[A::C * A::n], g[A::C], qg[A::C];
      auto products = [&](bool add) ALWAYS {
        const i64 r = base + a.rho < to ? base + a.rho : to - 1;
        a.read(x + r * DX + SEG[s].col, v);
        a.read(gy + r * DY + SEG[s].ycol, q);
        a.read_gates(x + r * DX, g);
        return a.backward(v, g, q, qg, st, p, a.on && base + a.rho < to, add, sum);
      };
      double t[4] = {};
      bool held = false;
      if (kLong) {
        of.template total<A, s>(a, part, sample, r0, r1, known, t, lds);
        if (base < to) base += (to - 1 - base) / (4 * A::RP) * (4 * A::RP);
        else base -= 4 * A::RP;
      } else {
        for (; base < to; base += 4 * A::RP) {
          const Sums o = products(slot < 0);
          t[0] += o.h;
          t[1] += o.hx;
          t[2] += o.gh;
          t[3] += o.ghx;
        }
        group_sums_(a, t, lds);
        if (slot >= 0) {
          if (threadIdx.x < 64 && a.on && a.rho == 0 && a.li == 0)
            for (int i = 0; i < 4; ++i) part[of.share(of.chunk, slot, s, a.g) + i] = t[i];
          return;
        }
        base -= 4 * A::RP;
        held = true;
      }
      const Means e = means_of_<s>(t, r1 - r0);
      for (; base >= first; base -= 4 * A::RP) {
        if (!held) products(kLong);
        held = false;
        a.finish(v, g, q, qg, st, e);
        if (a.on && base + a.rho < to) {
          a.write(gx + (base + a.rho) * DX + SEG[s].col, q);
          a.write_gates(gx + (base + a.rho) * DX, qg);
        }
      }
    }, [](i64, i64) ALWAYS {}); });
    a.put_sums(sum, any, sums ? sums + part_() * (NW + NB) : nullptr, gweight, gbias, lds);
  }
};
#define GRAPH_BWD(name, kLong) \
  extern "C" __global__ void __launch_bounds__(256) name(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias, const T* __restrict__ gy, \
                                                         const T* __restrict__ stats, T* __restrict__ gx, double* __restrict__ part, double* __restrict__ sums, \
                                                         T* __restrict__ gweight, T* __restrict__ gbias, const i64* __restrict__ ptr, i64 N, i64 S, i64 R, i64 D) { \
    __shared__ double lds[1024]; \
    with_sub_(sub_(), GraphBwd<kLong>{x, weight, bias, gy, stats, gx, part, sums, gweight, gbias, Chunks{ptr, N, S, R, D, 0}, SUB[sub_()].phase, lds}); \
  }
GRAPH_BWD(cgtp_norm_graph_bwd, false)
GRAPH_BWD(cgtp_norm_long_bwd, true)
)HIP";

// Calls whose kernels above do not fit the registers of a wave: more than 64 words a lane (fp64 32), or code that relocates registers or is refused.  Backward
// holds twice the words of forward and the channels' sums: single groups of 512x0e+512x1o fit both ways in fp32, of 2048x0e forward alone, of 512x3o in
// fp64 neither.  One workgroup for each unit of a sample, whatever its length; the rows are read once for each of mean, variance
// and result.  Rows as samples, 20 000 x 8192x0e fp32: forward 376 us (3.5 TB/s; 49 us and 6.7 for 2048x0e in registers); bound by the loops of one workgroup
// where samples are long: one of 20 000 rows of 2048x0e backward 105 ms (forward in registers 84 us).  All
// lanes make the same steps, those without a row or channel of their own with another's numbers, which do not count: behind a loop that lanes leave at
// different times the compiler has been seen to place vector instructions that none of them executes.
const char kUnits[] = R"HIP(
// a workgroup has one unit of every so many samples (and backward a row of partial sums for all of them)
INLINE int unit_() { return (int)(blockIdx.x % (NS * G)); }
INLINE i64 first_() { return blockIdx.x / (NS * G); }
INLINE i64 apart_() { return gridDim.x / (NS * G); }
)HIP";

const char kUnitFwd[] = R"HIP(
struct UnitFwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; T* __restrict__ y; T* __restrict__ stats;
  i64 N, S; const i64* __restrict__ ptr; int g; double* lds;
  template <int s> INLINE void operator()() const {
    for (i64 sample = first_(); sample < S; sample += apart_()) {
      i64 r0, r1;
      range_(ptr, sample, N, r0, r1);
      one<s>(sample, r0, r1);
    }
  }
  template <int s> INLINE void one(i64 sample, i64 r0, i64 r1) const {
    constexpr int n = SEG[s].n, cg = SEG[s].mul / G, TC = pow2_(cg) < 256 ? pow2_(cg) : 256, TR = 256 / TC;
    constexpr bool gated = SEG[s].gate >= 0, inv = SEG[s].inv;
    const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
    const i64 count = (r1 - r0) * cg;
    double mu = 0, gmu = 0, sq = 0, gsq = 0;
    auto each = [&](auto f) ALWAYS {
#pragma unroll cg <= TC && n <= 3 ? 4 : 1
      for (i64 first = r0; first < r1; first += TR) {
        const i64 r = TR == 1 || first + tr < r1 ? first + tr : r1 - 1;
#pragma unroll 4
        for (int c0 = 0; c0 < cg; c0 += TC) {
          const bool own = cg % TC == 0 || c0 + tc < cg;
          f(r, g * cg + (own ? c0 + tc : cg - 1), own && (TR == 1 || first + tr < r1));
        }
      }
    };
    if (inv || gated) {
      each([&](i64 r, int c, bool in) ALWAYS {
        const T* row = x + r * DX;
        if (inv) mu += in ? (double)row[SEG[s].col + c] : 0.0;
        if (gated) gmu += in ? (double)row[SEG[s].gate + c] : 0.0;
      });
      const double M = count > 0 ? (double)count : 1.0;
      if (inv) mu = block_sum_(mu, lds) / M;
      if (gated) gmu = block_sum_(gmu, lds) / M;
    }
    each([&](i64 r, int c, bool in) ALWAYS {
      const T* row = x + r * DX;
#pragma unroll
      for (int m = 0; m < n; ++m) {
        const double d = in ? (double)row[SEG[s].col + at_<s>(c, m)] - mu : 0.0;
        sq += d * d;
      }
      if (gated) {
        const double d = in ? (double)row[SEG[s].gate + c] - gmu : 0.0;
        gsq += d * d;
      }
    });
    const double M = count > 0 ? (double)count * n : 1.0;
    Stat S = {(T)mu, (T)(1.0 / sqrt(block_sum_(sq, lds) / M + EPS)), T(0), T(0)};
    if (gated) {
      S.gmu = (T)gmu;
      S.gr = (T)(1.0 / sqrt(block_sum_(gsq, lds) / (count > 0 ? (double)count : 1.0) + EPS));
    }
    if (stats && threadIdx.x == 0) {
      T* st = stats + sample * NST;
      st[(SEG[s].st * G + g) * 2] = S.mu;
      st[(SEG[s].st * G + g) * 2 + 1] = S.r;
      if (gated) {
        st[(SEG[s].gst * G + g) * 2] = S.gmu;
        st[(SEG[s].gst * G + g) * 2 + 1] = S.gr;
      }
    }
    each([&](i64 r, int ch, bool in) ALWAYS {
      const T* row = x + r * DX;
      T v[n], gt = gated ? row[SEG[s].gate + ch] : T(0);
#pragma unroll
      for (int m = 0; m < n; ++m) v[m] = row[SEG[s].col + at_<s>(ch, m)];
      forward_<s>(v, gt, S, param_<s>(weight, bias, ch));
      if (!in) return;
#pragma unroll
      for (int m = 0; m < n; ++m) y[r * DY + SEG[s].ycol + at_<s>(ch, m)] = v[m];
    });
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_unit_fwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                            T* __restrict__ y, T* __restrict__ stats, i64 N, i64 S, const i64* __restrict__ ptr) {
  __shared__ double lds[4];
  with_segment_<0>(unit_() / G, UnitFwd{x, weight, bias, y, stats, N, S, ptr, unit_() % G, lds});
}
)HIP";

const char kUnitBwd[] = R"HIP(
struct UnitBwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; const T* __restrict__ gy; const T* __restrict__ stats;
  T* __restrict__ gx; double* __restrict__ row; i64 N, S; const i64* __restrict__ ptr; int g; double* lds; double* cols;
  // sum over the rows' threads of a channel, for channel c < cg: written or added to what the same thread left of the samples before
  template <int TC> INLINE void column(double v, double* to, bool in, bool more) const {
    if constexpr (TC < 256) {
      __syncthreads();
      cols[threadIdx.x] = v;
      __syncthreads();
      v = 0;
      for (int i = 0; i < 256; i += TC) v += cols[threadIdx.x % TC + i];
    }
    if ((int)threadIdx.x < TC && in) *to = more ? *to + v : v;
  }
  template <int s> INLINE void operator()() const {
    for (i64 sample = first_(); sample < S; sample += apart_()) {
      i64 r0, r1;
      range_(ptr, sample, N, r0, r1);
      if (r0 < r1 || sample == first_()) one<s>(sample, r0, r1, sample != first_());
    }
  }
  template <int s> INLINE void one(i64 sample, i64 r0, i64 r1, bool more) const {
    constexpr int n = SEG[s].n, cg = SEG[s].mul / G, TC = pow2_(cg) < 256 ? pow2_(cg) : 256, TR = 256 / TC;
    constexpr bool gated = SEG[s].gate >= 0, inv = SEG[s].inv;
    const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
    const T* st = stats + sample * NST;
    Stat S = {st[(SEG[s].st * G + g) * 2], st[(SEG[s].st * G + g) * 2 + 1], T(0), T(0)};
    if (gated) {
      S.gmu = st[(SEG[s].gst * G + g) * 2];
      S.gr = st[(SEG[s].gst * G + g) * 2 + 1];
    }
    T v[n], q[n], gt = T(0), qg = T(0);
    auto load = [&](i64 r, int ch) ALWAYS {
#pragma unroll
      for (int m = 0; m < n; ++m) {
        v[m] = x[r * DX + SEG[s].col + at_<s>(ch, m)];
        q[m] = gy[r * DY + SEG[s].ycol + at_<s>(ch, m)];
      }
      if (gated) gt = x[r * DX + SEG[s].gate + ch];
    };
    double h = 0, hx = 0, gh = 0, ghx = 0;
    for (int c0 = 0; c0 < cg; c0 += TC) {
      const bool in = c0 + tc < cg;
      const int ch = g * cg + (in ? c0 + tc : cg - 1);
      double w = 0, b = 0, gw = 0, gb = 0;
      const Param p = param_<s>(weight, bias, ch);
#pragma unroll n <= 3 ? 4 : 1
      for (i64 first = r0; first < r1; first += TR) {
        const bool count = in && first + tr < r1;
        load(first + tr < r1 ? first + tr : r1 - 1, ch);
        const Sums o = backward_<s>(v, gt, q, qg, S, p);
        auto add = [count](double& to, T v) ALWAYS { to += count ? (double)v : 0.0; };
        add(w, o.w), add(b, o.b), add(gw, o.gw), add(gb, o.gb);
        add(h, o.h), add(hx, o.hx), add(gh, o.gh), add(ghx, o.ghx);
      }
      column<TC>(w, row + SEG[s].w + ch, in, more);
      if (inv) column<TC>(b, row + NW + SEG[s].b + ch, in, more);
      if (gated) {
        column<TC>(gw, row + SEG[s].gw + ch, in, more);
        column<TC>(gb, row + NW + SEG[s].gb + ch, in, more);
      }
    }
    const double M = r1 > r0 ? (double)(r1 - r0) * cg : 1.0;
    Means e = {T(0), (T)(block_sum_(hx, lds) / (M * n)), T(0), T(0)};
    if (inv) e.h = (T)(block_sum_(h, lds) / M);
    if (gated) {
      e.gh = (T)(block_sum_(gh, lds) / M);
      e.ghx = (T)(block_sum_(ghx, lds) / M);
    }
    for (i64 first = r0; first < r1; first += TR) {
      const i64 r = first + tr < r1 ? first + tr : r1 - 1;
#pragma unroll n <= 3 ? 4 : 1
      for (int c0 = 0; c0 < cg; c0 += TC) {
        const bool in = first + tr < r1 && c0 + tc < cg;
        const int ch = g * cg + (c0 + tc < cg ? c0 + tc : cg - 1);
        load(r, ch);
        backward_<s>(v, gt, q, qg, S, param_<s>(weight, bias, ch));
        finish_<s>(v, gt, q, qg, S, e);
        if (!in) continue;
#pragma unroll
        for (int m = 0; m < n; ++m) gx[r * DX + SEG[s].col + at_<s>(ch, m)] = q[m];
        if (gated) gx[r * DX + SEG[s].gate + ch] = qg;
      }
    }
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_unit_bwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                            const T* __restrict__ gy, const T* __restrict__ stats, T* __restrict__ gx,
                                                            double* __restrict__ part, i64 N, i64 S, const i64* __restrict__ ptr) {
  __shared__ double lds[4], cols[256];
  with_segment_<0>(unit_() / G, UnitBwd{x, weight, bias, gy, stats, gx, part + first_() * (NW + NB), N, S, ptr, unit_() % G, lds, cols});
}
)HIP";

// gweight and gbias from `rows` rows of partial sums: 16 columns a workgroup, 64 threads a column, four loads in flight each: 4 to 5 us, latency
const char kSums[] = R"HIP(
extern "C" __global__ void __launch_bounds__(1024) cgtp_norm_sums(const double* __restrict__ part, i64 rows, T* __restrict__ gweight, T* __restrict__ gbias) {
  __shared__ double lds[1024];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, t = threadIdx.x / 16, cc = c < NW + NB ? c : 0;
  double v[4] = {};
  for (i64 r = t; r < rows; r += 256)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += r + 64 * i < rows ? part[(r + 64 * i) * (NW + NB) + cc] : 0.0;
  lds[threadIdx.x] = (v[0] + v[1]) + (v[2] + v[3]);
  __syncthreads();
#pragma unroll
  for (int h = 512; h >= 16; h /= 2) {
    if ((int)threadIdx.x < h) lds[threadIdx.x] += lds[threadIdx.x + h];
    __syncthreads();
  }
  if (t != 0 || c >= NW + NB) return;
  if (c < NW) gweight[c] = (T)lds[threadIdx.x];
  else gbias[c - NW] = (T)lds[threadIdx.x];
}
)HIP";

}  // namespace

void emit_norm(Norm& N) {
  const bool f64 = N.dtype == CGTP_F64;
  const int most = f64 ? 32 : 64;          // words a lane holds of a row
  bool covered = true;
  struct Sub {
    int s, phase, size;
  };
  std::vector<Sub> subs;
  for (size_t i = 0; i < N.seg.size(); ++i) {
    NormSeg& s = N.seg[i];
    const int cg = s.mul / N.groups;
    // V channels in one piece: everything that is added to a row's start is a multiple of V words
    auto fits = [&](int V) {
      const bool cols = s.col % V == 0 && s.ycol % V == 0 && N.dim_x % V == 0 && N.dim_y % V == 0 && (s.gate < 0 || s.gate % V == 0);
      return cols && cg % V == 0 && V * s.n <= most / 2;
    };
    // In the layout with a channel's components as neighbours one channel a lane: with more, a lane's words are so far apart that the lines of
    // a wave's loads leave the first-level cache between them (20 000 rows of 128 channels, l <= 3, forward and backward 206 us, with two 265, four 363).
    s.V = !N.ir_mul && s.n > 1 ? 1 : fits(4) ? 4 : fits(2) ? 2 : 1;
    s.vec = s.V > 1;
    s.lanes = 1;
    while (s.lanes < 64 && s.lanes * s.V < cg) s.lanes *= 2;
    s.J = (cg + s.lanes * s.V - 1) / (s.lanes * s.V);
    s.at_once = 1;
    for (int g = 1; g <= N.groups; ++g)
      if (N.groups % g == 0 && g * s.lanes <= 64) s.at_once = g;
    s.rows = 64 / (s.at_once * s.lanes);
    s.phases = N.groups / s.at_once;
    if (s.V * s.J * s.n > most || s.phases > 256) covered = false;
    for (int p = 0; covered && p < s.phases; ++p) subs.push_back({(int)i, p, s.at_once * cg * (s.n + (s.gate >= 0))});
  }
  std::stable_sort(subs.begin(), subs.end(), [](const Sub& a, const Sub& b) { return a.size > b.size; });
  N.subs = (int)subs.size();
  std::ostringstream o;
  o.precision(17);
  o << "// group normalisation of irreps rows\ntypedef " << (f64 ? "double" : "float") << " T;\n"
    << "struct Seg { int mul, n, col, ycol; bool inv; int gate, w, b, gw, gb, st, gst, V, J, lanes, at_once, rows; bool vec; };\n"
    << "constexpr int NS = " << N.seg.size() << ", G = " << N.groups << ", ACT = " << N.act << ", DX = " << N.dim_x << ", DY = " << N.dim_y
    << ", NW = " << N.n_w << ", NB = " << N.n_b << ", NST = " << N.n_stat << ", NSUB = " << subs.size() << ";\n"
    << "constexpr bool IR_MUL = " << (N.ir_mul ? "true" : "false") << ";\nconstexpr double EPS = " << N.eps << ";\n"
    << "constexpr Seg SEG[NS] = {\n";
  for (const NormSeg& s : N.seg)
    o << "  {" << s.mul << ", " << s.n << ", " << s.col << ", " << s.ycol << ", " << (s.inv ? "true" : "false") << ", " << s.gate << ", " << s.w
      << ", " << s.b << ", " << s.gw << ", " << s.gb << ", " << s.st << ", " << s.gst << ", " << s.V << ", " << s.J << ", " << s.lanes << ", " << s.at_once
      << ", " << s.rows << ", " << (s.vec ? "true" : "false") << "},\n";
  o << "};\n";
  if (covered) {
    o << "struct Sub { int s, phase; };\n__constant__ constexpr Sub SUB[NSUB] = {";
    for (const Sub& s : subs) o << "{" << s.s << ", " << s.phase << "}, ";
    o << "};\n";
  }
  o << kShared;
  auto kernel = [&o](const char* name, std::initializer_list<const char*> text) {
    Kernel k;
    k.name = name;
    k.source = o.str();
    for (const char* t : text) k.source += t;
    return k;
  };
  N.any[0] = kernel("cgtp_norm_unit_fwd", {kUnits, kUnitFwd});
  N.any[1] = kernel("cgtp_norm_unit_bwd", {kUnits, kUnitBwd, kSums});
  for (NormCall& c : N.call) c.any = !covered;
  if (!covered) return;
  N.call[kRowsForward].code = kernel("cgtp_norm_row_fwd", {kLanes, kRowFwd});
  N.call[kRowsBackward].code = kernel("cgtp_norm_row_bwd", {kLanes, kRowBwd, kSums});
  N.call[kGraphsForward].code = kernel("cgtp_norm_graph_fwd", {kLanes, kGraphs, kGraphFwd});
  N.call[kGraphsBackward].code = kernel("cgtp_norm_graph_bwd", {kLanes, kGraphs, kGraphBwd, kSums});
}

}  // namespace cgtp
