// Tile and split of the weight gradient of rip_wgrad.hip.  Plain host code with no HIP
// dependency, so it is tested on its own.
#pragma once

#include <cstdint>

#include "rip_internal.h"

namespace rip {
namespace wgrad {

constexpr int kTokens = 32;  // tokens of a step

// The tiles, by type of dy: rows and columns of grad, workgroups that a compute unit
// holds, and the time (us) of a step of 32 tokens where it holds one and where it
// holds all of them, measured on long products.
struct Shape {
  int n, k, resident;
  double one, all;
};
constexpr Shape kF32Shapes[] = {{128, 128, 1, 0.9, 0.9}, {128, 256, 1, 1.4, 1.4}};
constexpr Shape kBf16Shapes[] = {{128, 128, 2, 0.5, 0.7}, {192, 256, 1, 0.7, 0.7}, {256, 256, 1, 0.75, 0.75}};
constexpr int kUnits = 256;       // compute units
constexpr int64_t kMaxSplits = 64;

struct Plan {
  int shape;
  int tiles_n, tiles_k, splits, part_k;
  int64_t share;
};
// The tile and the number of splits of the least time: rounds of workgroups, each
// with its steps and the time to fill and drain the pipeline (three steps), and
// for split products the parts' way to memory and back and the second launch.
inline Plan make_plan(int32_t dy_dtype, int64_t tokens, int64_t n, int64_t k) {
  const Shape* shapes = dy_dtype == RIP_BF16 ? kBf16Shapes : kF32Shapes;
  const int count = dy_dtype == RIP_BF16 ? 3 : 2;
  const int64_t steps = ceil_div(tokens, kTokens), part_k = ceil_div(k, 4) * 4;
  Plan best{};
  double least = 1e30;
  for (int i = 0; i < count; ++i) {
    const Shape& sh = shapes[i];
    const int64_t tiles_n = ceil_div(n, sh.n), tiles_k = ceil_div(k, sh.k), tiles = tiles_n * tiles_k;
    for (int64_t splits = 1; splits <= kMaxSplits && (splits == 1 || splits * 2 <= steps); ++splits) {
      const int64_t per = ceil_div(steps, splits), groups = tiles * splits;
      const double step = groups <= kUnits ? sh.one : sh.all;
      double us = (double)ceil_div(groups, kUnits * sh.resident) * (per + 3) * step;
      if (splits > 1) us += 4.0 + (double)splits * n * part_k * 8 / 4e6;
      if (us < least) {
        least = us;
        best = Plan{i, (int)tiles_n, (int)tiles_k, (int)splits, (int)part_k, per * kTokens};
      }
    }
  }
  best.splits = tokens > 0 ? (int)ceil_div(tokens, best.share) : 1;
  return best;
}

}  // namespace wgrad
}  // namespace rip
