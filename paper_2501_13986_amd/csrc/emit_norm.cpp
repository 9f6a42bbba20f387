// Kernels of the group normalisation: the segments as constants in front of a text that is the same for all of them.
//
// A unit is one group of one segment, with the group of its gates if it has any: units of a sample depend on nothing of each other.
// With xh = (x - mu) r (mu = 0 unless the segment is 0e), M numbers in a unit of a sample, q = sigmoid(wg xh_g + bg):
//   0e:      y = act(w xh + b)         l = dE/d(w xh + b) = gy act'
//   others:  y = w xh q                l = gy q;  gates: l_g = q (1 - q) sum_m gy w xh
//   gw = sum l xh, gb = sum l, h = w l,  gx = r (h - [0e, gates: mean(h)] - xh mean(h xh))
#include <sstream>

#include "norm.hpp"

namespace cgtp {
namespace {

const char kShared[] = R"HIP(
typedef long long i64;
// off by |t| half steps where t is negative: at most 0.3 half steps of 1
__device__ inline float sigmoid_(float t) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(t * -1.44269502f)); }
__device__ inline double sigmoid_(double t) { return 1.0 / (1.0 + exp(-t)); }
__device__ inline float erfc_(float t) { return erfcf(t); }
__device__ inline double erfc_(double t) { return erfc(t); }
__device__ inline float exp_(float t) { return expf(t); }
__device__ inline double exp_(double t) { return exp(t); }
__device__ inline float tanh_(float t) { return tanhf(t); }
__device__ inline double tanh_(double t) { return tanh(t); }
__device__ inline float fma_(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ inline double fma_(double a, double b, double c) { return __builtin_fma(a, b, c); }

// activation and derivative
__device__ inline void act_(T t, T& a, T& d) {
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
template <int s> __device__ inline int at_(int c, int m) { return IR_MUL ? m * SEG[s].mul + c : c * SEG[s].n + m; }

struct Stat { T mu, r, gmu, gr; };       // of a unit and of its gates
struct Param { T w, b, gw, gb; };        // of a channel and of its gate

template <int s> __device__ inline Param param_(const T* __restrict__ weight, const T* __restrict__ bias, int c) {
  Param p = {weight[SEG[s].w + c], T(0), T(0), T(0)};
  if constexpr (SEG[s].inv) p.b = bias[SEG[s].b + c];
  if constexpr (SEG[s].gate >= 0) {
    p.gw = weight[SEG[s].gw + c];
    p.gb = bias[SEG[s].gb + c];
  }
  return p;
}

// one channel of one row, its n components in v and its gate in g, normalised: y in place of v
template <int s> __device__ inline void forward_(T* v, T g, const Stat& S, const Param& p) {
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
template <int s> __device__ inline Sums backward_(T* v, T& g, T* q, T& qg, const Stat& S, const Param& p) {
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
template <int s> __device__ inline void finish_(const T* v, T g, T* q, T& qg, const Stat& S, const Means& e) {
#pragma unroll
  for (int m = 0; m < SEG[s].n; ++m) q[m] = S.r * (q[m] - (SEG[s].inv ? e.h : T(0)) - v[m] * e.hx);
  if constexpr (SEG[s].gate >= 0) qg = S.gr * (qg - e.gh - g * e.ghx);
}

// rows of sample s, within [0, N]
__device__ inline void range_(const i64* __restrict__ ptr, i64 s, i64 N, i64& r0, i64& r1) {
  r0 = ptr ? ptr[s] : s;
  r1 = ptr ? ptr[s + 1] : s + 1;
  r0 = r0 < 0 ? 0 : r0 > N ? N : r0;
  r1 = r1 < r0 ? r0 : r1 > N ? N : r1;
}

constexpr int pow2_(int v) { int p = 1; while (p < v) p *= 2; return p; }

// f<s>() for a number s that all lanes share
template <int s, class F> __device__ inline void with_segment_(int k, F f) {
  if constexpr (s + 1 < NS) {
    if (k != s) return with_segment_<s + 1>(k, f);
  }
  f.template operator()<s>();
}

// sum over the workgroup, the same in every thread; the order is fixed
__device__ inline double block_sum_(double v, double* lds) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}
)HIP";

// One workgroup for each unit of a sample, whatever its length: the rows are read once for each of mean, variance and result.
const char kForward[] = R"HIP(
struct UnitFwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; T* __restrict__ y; T* __restrict__ stats;
  i64 r0, r1, sample; int g; double* lds;
  template <int s> __device__ void operator()() const {
    constexpr int n = SEG[s].n, cg = SEG[s].mul / G, TC = pow2_(cg) < 256 ? pow2_(cg) : 256, TR = 256 / TC;
    constexpr bool gated = SEG[s].gate >= 0, inv = SEG[s].inv;
    const int tc = threadIdx.x % TC, tr = threadIdx.x / TC;
    const i64 count = (r1 - r0) * cg;
    double mu = 0, gmu = 0, sq = 0, gsq = 0;
    auto each = [&](auto f) {
      for (i64 r = r0 + tr; r < r1; r += TR)
        for (int c = tc; c < cg; c += TC) f(x + r * DX, g * cg + c);
    };
    if (inv || gated) {
      each([&](const T* row, int c) {
        if (inv) mu += row[SEG[s].col + c];
        if (gated) gmu += row[SEG[s].gate + c];
      });
      const double M = count > 0 ? (double)count : 1.0;
      if (inv) mu = block_sum_(mu, lds) / M;
      if (gated) gmu = block_sum_(gmu, lds) / M;
    }
    each([&](const T* row, int c) {
#pragma unroll
      for (int m = 0; m < n; ++m) {
        const double d = (double)row[SEG[s].col + at_<s>(c, m)] - mu;
        sq += d * d;
      }
      if (gated) {
        const double d = (double)row[SEG[s].gate + c] - gmu;
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
    for (i64 r = r0 + tr; r < r1; r += TR)
      for (int c = tc; c < cg; c += TC) {
        const T* row = x + r * DX;
        const int ch = g * cg + c;
        T v[n], gt = gated ? row[SEG[s].gate + ch] : T(0);
#pragma unroll
        for (int m = 0; m < n; ++m) v[m] = row[SEG[s].col + at_<s>(ch, m)];
        forward_<s>(v, gt, S, param_<s>(weight, bias, ch));
#pragma unroll
        for (int m = 0; m < n; ++m) y[r * DY + SEG[s].ycol + at_<s>(ch, m)] = v[m];
      }
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_fwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                            T* __restrict__ y, T* __restrict__ stats, i64 N, i64 S, const i64* __restrict__ ptr) {
  __shared__ double lds[4];
  for (i64 u = blockIdx.x; u < S * NS * G; u += gridDim.x) {
    const i64 sample = u / (NS * G);
    const int unit = (int)(u % (NS * G));
    i64 r0, r1;
    range_(ptr, sample, N, r0, r1);
    with_segment_<0>(unit / G, UnitFwd{x, weight, bias, y, stats, r0, r1, sample, unit % G, lds});
  }
}
)HIP";

const char kBackward[] = R"HIP(
struct UnitBwd {
  const T* __restrict__ x; const T* __restrict__ weight; const T* __restrict__ bias; const T* __restrict__ gy; const T* __restrict__ stats;
  T* __restrict__ gx; double* __restrict__ part; i64 r0, r1, sample; int g; double* lds; double* cols;
  // sum over the rows' threads of a channel, into to[] for channel c < cg
  template <int TC> __device__ void column(double v, double* to, bool in) const {
    __syncthreads();
    cols[threadIdx.x] = v;
    __syncthreads();
    if ((int)threadIdx.x < TC && in) {
      double t = 0;
      for (int i = 0; i < 256; i += TC) t += cols[threadIdx.x + i];
      *to = t;
    }
  }
  template <int s> __device__ void operator()() const {
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
    auto load = [&](i64 r, int ch) {
#pragma unroll
      for (int m = 0; m < n; ++m) {
        v[m] = x[r * DX + SEG[s].col + at_<s>(ch, m)];
        q[m] = gy[r * DY + SEG[s].ycol + at_<s>(ch, m)];
      }
      if (gated) gt = x[r * DX + SEG[s].gate + ch];
    };
    double h = 0, hx = 0, gh = 0, ghx = 0;
    for (int c0 = 0; c0 < cg; c0 += TC) {
      const int ch = g * cg + c0 + tc;
      const bool in = c0 + tc < cg;
      double w = 0, b = 0, gw = 0, gb = 0;
      if (in) {
        const Param p = param_<s>(weight, bias, ch);
        for (i64 r = r0 + tr; r < r1; r += TR) {
          load(r, ch);
          const Sums o = backward_<s>(v, gt, q, qg, S, p);
          w += o.w; b += o.b; gw += o.gw; gb += o.gb;
          h += o.h; hx += o.hx; gh += o.gh; ghx += o.ghx;
        }
      }
      double* row = part + sample * (NW + NB);
      column<TC>(w, row + SEG[s].w + ch, in);
      if (inv) column<TC>(b, row + NW + SEG[s].b + ch, in);
      if (gated) {
        column<TC>(gw, row + SEG[s].gw + ch, in);
        column<TC>(gb, row + NW + SEG[s].gb + ch, in);
      }
    }
    const double M = r1 > r0 ? (double)(r1 - r0) * cg : 1.0;
    Means e = {T(0), (T)(block_sum_(hx, lds) / (M * n)), T(0), T(0)};
    if (inv) e.h = (T)(block_sum_(h, lds) / M);
    if (gated) {
      e.gh = (T)(block_sum_(gh, lds) / M);
      e.ghx = (T)(block_sum_(ghx, lds) / M);
    }
    for (i64 r = r0 + tr; r < r1; r += TR)
      for (int c = tc; c < cg; c += TC) {
        const int ch = g * cg + c;
        load(r, ch);
        backward_<s>(v, gt, q, qg, S, param_<s>(weight, bias, ch));
        finish_<s>(v, gt, q, qg, S, e);
#pragma unroll
        for (int m = 0; m < n; ++m) gx[r * DX + SEG[s].col + at_<s>(ch, m)] = q[m];
        if (gated) gx[r * DX + SEG[s].gate + ch] = qg;
      }
  }
};
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_bwd(const T* __restrict__ x, const T* __restrict__ weight, const T* __restrict__ bias,
                                                            const T* __restrict__ gy, const T* __restrict__ stats, T* __restrict__ gx,
                                                            double* __restrict__ part, i64 N, i64 S, const i64* __restrict__ ptr) {
  __shared__ double lds[4], cols[256];
  for (i64 u = blockIdx.x; u < S * NS * G; u += gridDim.x) {
    const i64 sample = u / (NS * G);
    const int unit = (int)(u % (NS * G));
    i64 r0, r1;
    range_(ptr, sample, N, r0, r1);
    with_segment_<0>(unit / G, UnitBwd{x, weight, bias, gy, stats, gx, part, r0, r1, sample, unit % G, lds, cols});
  }
}
)HIP";

// gweight and gbias from `rows` rows of partial sums
const char kSums[] = R"HIP(
extern "C" __global__ void __launch_bounds__(256) cgtp_norm_sums(const double* __restrict__ part, i64 rows, T* __restrict__ gweight, T* __restrict__ gbias) {
  __shared__ double lds[256];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, t = threadIdx.x / 16;
  double v = 0;
  if (c < NW + NB)
    for (i64 r = t; r < rows; r += 16) v += part[r * (NW + NB) + c];
  lds[threadIdx.x] = v;
  __syncthreads();
  if (t != 0 || c >= NW + NB) return;
  for (int i = 1; i < 16; ++i) v += lds[threadIdx.x + 16 * i];
  if (c < NW) gweight[c] = (T)v;
  else gbias[c - NW] = (T)v;
}
)HIP";

}  // namespace

void emit_norm(const Norm& N, Kernel& fwd, Kernel& bwd, Kernel& sums) {
  std::ostringstream o;
  o.precision(17);
  o << "// group normalisation of irreps rows\ntypedef " << (N.dtype == CGTP_F64 ? "double" : "float") << " T;\n"
    << "struct Seg { int mul, n, col, ycol; bool inv; int gate, w, b, gw, gb, st, gst; };\n"
    << "constexpr int NS = " << N.seg.size() << ", G = " << N.groups << ", ACT = " << N.act << ", DX = " << N.dim_x << ", DY = " << N.dim_y
    << ", NW = " << N.n_w << ", NB = " << N.n_b << ", NST = " << N.n_stat << ";\n"
    << "constexpr bool IR_MUL = " << (N.ir_mul ? "true" : "false") << ";\nconstexpr double EPS = " << N.eps << ";\n"
    << "constexpr Seg SEG[NS] = {\n";
  for (const NormSeg& s : N.seg)
    o << "  {" << s.mul << ", " << s.n << ", " << s.col << ", " << s.ycol << ", " << (s.inv ? "true" : "false") << ", " << s.gate << ", " << s.w
      << ", " << s.b << ", " << s.gw << ", " << s.gb << ", " << s.st << ", " << s.gst << "},\n";
  o << "};\n" << kShared;
  const std::string head = o.str();
  auto make = [&](Kernel& k, const char* name, const char* text) {
    k.name = name;
    k.wg = 256;
    k.source = head + text;
  };
  make(fwd, "cgtp_norm_fwd", kForward);
  make(bwd, "cgtp_norm_bwd", kBackward);
  make(sums, "cgtp_norm_sums", kSums);
}

}  // namespace cgtp
