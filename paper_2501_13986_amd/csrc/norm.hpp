// Group normalisation of irreps rows: the handle, and the emitter of its kernels (emit_norm.cpp).
#pragma once

#include "plan.hpp"

namespace cgtp {

struct NormSeg {
  int mul, n;        // channels, components
  int col, ycol;     // first column in x and in y
  bool inv;          // 0e: centred, bias, activation
  int gate;          // first column of its gates, -1: none
  int w, b, gw, gb;  // first weight and bias (b: 0e segments), of the gates as well
  int st, gst;       // its place among the segments of stats, of its gates
};

struct Norm {
  std::vector<NormSeg> seg;
  int groups = 1, act = 0, dtype = 0, device = -1, num_cu = 256;
  bool ir_mul = false;
  double eps = 0;
  int64_t dim_x = 0, dim_y = 0, n_w = 0, n_b = 0, n_stat = 0;   // n_stat: numbers per sample
  Kernel fwd, bwd, sums;
  size_t elt() const { return dtype == CGTP_F64 ? 8 : 4; }
};

void emit_norm(const Norm& N, Kernel& fwd, Kernel& bwd, Kernel& sums);

}  // namespace cgtp
