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
  const float* lut;   // the bias by distance, [heads][lut_size], or NULL: made by the workgroup
  int lut_size, lut_first;  // lut_size 0: no bias
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

// The table, and which of its rows a distance reads, by value: what the kernels with a
// bias take behind their other arguments.
struct Buckets {
  const void* table;
  int64_t ld;
  int bf16;
  int n;                           // intervals
  int32_t start[kMaxStarts];       // first distance of intervals 1 ..
  int32_t row[RIP_MAX_INTERVALS];
};
template <typename T>
struct WithBias : T {
  Buckets map;
};
template <typename T, bool BIAS>
struct KernelArgs {
  typedef T type;
};
template <typename T>
struct KernelArgs<T, true> {
  typedef WithBias<T> type;
};

// A bias's value in the log2 domain.  Masks of a type's lowest value hide their keys as
// -inf does: the log-sum of a row of such scores would not hold what tells them apart.
constexpr float kHides = -65536.0f;
__device__ __forceinline__ float bias_at(const Buckets& map, int distance, int head) {
  int row = map.row[0];
  for (int b = 1; b < map.n; ++b) row = distance >= map.start[b - 1] ? map.row[b] : row;
  const int64_t at = row * map.ld + head;
  const float x = map.bf16 ? Elem<RIP_BF16>::load((const uint16_t*)map.table + at) : ((const float*)map.table)[at];
  return x < kHides ? -__builtin_inff() : x * 1.44269504f;
}

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
};

// The grid of a launch over slots, splits and heads: as many rows as its 32-bit sizes
// need.
inline dim3 grid_of(const Args& p, int heads) {
  const int64_t all = (int64_t)p.slots * p.splits * heads, row = 1 << 20;
  return all <= row ? dim3((uint32_t)all) : dim3((uint32_t)row, (uint32_t)ceil_div(all, row));
}

// Launches by type and width (rip_attn_forward.hip, rip_attn_backward.hip).
int32_t run_forward(WithBias<Forward>& f, int32_t dtype, int width, int waves, void* stream);
struct Plans {
  Plan q, k;
};
int32_t run_backward(WithBias<Backward>& f, const Args& over_q, const Args& over_k, int32_t dtype,
                     const Plans& plan, void* stream);
int32_t run_bias_grad(const WithBias<Backward>& f, int64_t parts, int32_t buckets, int32_t heads,
                      int32_t dtype, void* grad, int64_t ld, int32_t accumulate, void* stream);

}  // namespace attn
}  // namespace rip
