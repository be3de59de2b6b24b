// Arguments of the attention kernels, shared with their host code (rip_attn.hip).
#pragma once

#include "rip_attn_plan.h"
#include "rip_ops_common.h"

namespace rip {
namespace attn {

constexpr int kMaxStarts = RIP_MAX_INTERVALS - 1;

// Tokens of one side (queries or keys) and where its sequences begin.
struct Side {
  const int32_t* offsets;  // [n_seqs + 1]
  int tokens;
};

struct Args {
  Side q, k;
  int n_seqs;
  int cleaned;        // offsets are in order already (a launch before made them so)
  int heads, group;   // heads of q to a head of k and v
  int pack;           // heads of q that share a tile: the group, or 1
  int dim, causal;
  FastDiv by_pack;
  float scale2, scale;  // scale2 = scale * log2(e)
  int splits;         // of the axis that a workgroup goes over
  int slots;          // tiles of the grid
  const float* lut;   // [heads][lut_size], or NULL
  int lut_size, lut_first;
};

// A matrix of heads side by side.
struct Heads {
  void* p;
  int64_t ld;
};
struct ConstHeads {
  const void* p;
  int64_t ld;
};

// The map from distances to rows of the table, by value.
struct Buckets {
  int n;                           // intervals
  int32_t start[kMaxStarts];       // first distance of intervals 1 ..
  int32_t row[RIP_MAX_INTERVALS];
};

struct Forward {
  Args a;
  ConstHeads q, k, v;
  Heads out, low;
  float* lse;       // [heads][q tokens]
  float* part;      // splits: [splits][heads][q tokens][dim], then their maxima and sums
};
struct Backward {
  Args a;
  ConstHeads q, k, v, out, low, dout;
  Heads dq, dk, dv;
  const float* lse;
  float* delta;     // [heads][q tokens]
  float* part;      // splits: parts of dq, or of dk and dv
  float* bias_part; // [heads][slots * splits][intervals]
  const Buckets* buckets;  // device
};

// The grid of a launch over slots, splits and heads: as many rows as its 32-bit sizes
// need.
inline dim3 grid_of(const Args& p, int heads) {
  const int64_t all = (int64_t)p.slots * p.splits * heads, row = 1 << 20;
  return all <= row ? dim3((uint32_t)all) : dim3((uint32_t)row, (uint32_t)ceil_div(all, row));
}

// Launches by type and width (rip_attn_forward.hip, rip_attn_backward.hip).
int32_t run_forward(Forward& f, int32_t dtype, int width, int waves, void* stream);
struct Plans {
  Plan q, k;
};
int32_t run_backward(Backward& f, const Args& over_q, const Args& over_k, int32_t dtype,
                     const Plans& plan, void* stream);
int32_t run_bias_grad(const Backward& f, int64_t parts, int32_t buckets, int32_t heads,
                      int32_t dtype, void* grad, int64_t ld, int32_t accumulate, void* stream);

}  // namespace attn
}  // namespace rip
