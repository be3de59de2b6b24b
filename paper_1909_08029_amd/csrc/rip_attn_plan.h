// Widths, workgroups and splits of the attention kernels.  Plain host code with no HIP
// dependency, so it is tested on its own.
#pragma once

#include <algorithm>
#include <cstdint>

#include "rip_internal.h"

namespace rip {
namespace attn {

constexpr int kWidths = 3;
constexpr int kWidth[kWidths] = {64, 128, 256};  // of a head, padded with zeros
constexpr int kWaves = 4;         // of a workgroup; one where queries are few
constexpr int kRows = 32;         // queries (or keys) of a wave
constexpr int kUnits = 256;       // compute units
constexpr int kMaxSplits = 64;
constexpr int kScan = 1024;       // offsets that every workgroup puts in order by itself

// Lengths are the device's; the host knows only how many tokens and sequences.
struct Sizes {
  int64_t q_tokens, k_tokens;
  int n, heads, group, dim;
  bool bias;
};
struct Plan {
  int width, waves, pack, splits;
  int64_t slots;  // tiles of the grid
};

inline int width_of(int dim) {
  for (int i = 0; i < kWidths; ++i)
    if (dim <= kWidth[i]) return kWidth[i];
  return 0;
}
inline int64_t slots_of(int64_t tokens, int pack, int n, int tile) { return tokens * pack / tile + n + 2; }

// Over the queries (forward; dq).  A tile that the queries of a head would not fill
// takes those of all heads that share k and v.
inline Plan over_queries(const Sizes& s, bool one_wave_allowed) {
  Plan p{width_of(s.dim), kWaves, 1, 1, 0};
  const int n = std::max(1, s.n);
  const int64_t q = ceil_div(s.q_tokens, n), k = ceil_div(s.k_tokens, n);  // of a sequence
  if (!s.bias && s.group > 1 && q < kRows * kWaves && s.q_tokens * s.group < (int64_t)1 << 30)
    p.pack = s.group;
  auto units = [&] { return n * ceil_div(q * p.pack, kRows * p.waves) * (s.heads / p.pack); };
  if (one_wave_allowed && units() < kUnits) p.waves = 1;
  const int64_t want = p.waves == 1 ? 4 * kUnits : 2 * kUnits;
  if (units() < want / 2)
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(want, std::max<int64_t>(1, units())),
                                                            k / 128, kMaxSplits}));
  p.slots = slots_of(s.q_tokens, p.pack, s.n, kRows * p.waves);
  return p;
}

// Over the keys (dk and dv).
inline Plan over_keys(const Sizes& s) {
  Plan p{width_of(s.dim), kWaves, 1, 1, 0};
  const int n = std::max(1, s.n);
  const int64_t q = ceil_div(s.q_tokens, n), k = ceil_div(s.k_tokens, n);
  const int64_t units = n * ceil_div(k, kRows * kWaves) * (s.heads / s.group);
  if (units < kUnits)
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(2 * kUnits, std::max<int64_t>(1, units)),
                                                            ceil_div(q, 64) * s.group / 2, kMaxSplits}));
  p.slots = slots_of(s.k_tokens, 1, s.n, kRows * kWaves);
  return p;
}

}  // namespace attn
}  // namespace rip
