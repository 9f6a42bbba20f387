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
  // how a wave goes over it: V neighbouring channels a lane, J times, `lanes` lanes a group, `at_once` groups and `rows` rows a step,
  // in phases of groups / at_once; V channels are read and written in one piece where `vec`
  int V, J, lanes, at_once, rows, phases;
  bool vec;
};

// The four calls of a normalisation: every row a sample (ptr NULL), or samples of any number of rows.
enum NormCalls { kRowsForward, kRowsBackward, kGraphsForward, kGraphsBackward, kNormCalls };

struct NormCall {
  Kernel code;                       // kernels with a row's words in registers
  bool any = false;                  // served by the kernels for any size instead: its code relocates registers, or was refused
  hipFunction_t longer = nullptr;    // of long samples
  hipFunction_t sums = nullptr;      // of the parameters' gradients
};

struct Norm {
  std::vector<NormSeg> seg;
  int groups = 1, act = 0, dtype = 0, device = -1, num_cu = 256;
  bool ir_mul = false, loaded = false;
  double eps = 0;
  int64_t dim_x = 0, dim_y = 0, n_w = 0, n_b = 0, n_stat = 0;   // n_stat: numbers per sample
  int subs = 0;             // segments times their phases
  NormCall call[kNormCalls];
  Kernel any[2];            // forward, backward for groups of any size, each row or sample of them
  hipFunction_t any_sums = nullptr;
  size_t elt() const { return dtype == CGTP_F64 ? 8 : 4; }
};

// Fills in how the segments are gone over, and the sources.
void emit_norm(Norm& N);

}  // namespace cgtp
