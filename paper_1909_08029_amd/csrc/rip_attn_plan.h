// Widths, workgroups and splits of the attention kernels.  Plain host code with no HIP
// dependency, so it is tested on its own.
#pragma once

#include <algorithm>
#include <cstdint>

#include "rip_internal.h"

namespace rip {
namespace attn {

constexpr int kRows = 32;         // queries (or keys) of a wave
constexpr int kMaxSplits = 64;
constexpr int kScan = 1024;       // offsets that every workgroup puts in order by itself

constexpr int kWidths = 4;
constexpr int kWidth[kWidths] = {64, 96, 128, 256};  // of a head, padded with zeros
inline int width_of(int dim) {
  for (int i = 0; i < kWidths; ++i)
    if (dim <= kWidth[i]) return kWidth[i];
  return 0;
}

// Lengths are the device's; the host knows only how many tokens and sequences.
struct Sizes {
  int64_t q_tokens, k_tokens;
  int n, heads, group, dim;
  bool bf16, causal, bias;
  int span;  // of the bias: numbers by distance
};
struct Plan {
  int width, waves, pack, splits;
  int64_t slots;  // tiles of the grid
};

inline int64_t slots_of(int64_t tokens, int pack, int n, int tile) { return tokens * pack / tile + n + 2; }

// The kernels: products of a block of 32 x 32, and time (us) of a block beside them.
struct Kernel {
  int products;
  double softmax;
};
constexpr Kernel kForward = {2, 0.12}, kDq = {3, 0.16}, kDkv = {4, 0.2};

// Time (us) of `units` tiles of `waves` waves (of which `busy` have work) that go over
// `axis` elements each (`share` of them where causal) in `splits` parts: what all 1024
// SIMDs have to do, or one tile's chain, whichever is longer; then the parts' way through
// memory and the launch that adds them (`part`: bytes of a split's parts).
//
// Measured: a block's products take 0.0021 us a column each in bf16 (six times that for
// fp32 as three parts, sixteen times for fp32's own instructions); a tile costs about four
// us before its first block.  Eight waves share a tile's way to LDS (16384 tokens of
// 128 columns: 1089 us for the forward pass, 1306 with four), but two share a SIMD.
// One query each over 200003 keys: 1512 us in one part, 404 in 4, 159 in 32, 164 in 64;
// 2049 tokens of 72 columns in fp32: 150, 76 in 4, 84 in 16.
inline double time_of(const Kernel& k, const Sizes& s, int width, int64_t units, int waves, int busy,
                      int64_t axis, double share, int splits, double part) {
  const double product = (s.bf16 ? 0.0021 : width <= 128 ? 0.0126 : 0.0336) * width;
  const double block = k.products * product + k.softmax;
  const double alone = block * (busy == 8 ? 1.8 : s.bf16 ? 1.1 : 1.25);
  const double blocks = (double)ceil_div(axis, kRows);
  const double all = (double)units * busy * (waves == 8 ? 0.9 : 1.0) *
                     (blocks * share * block + 2.0 * splits) / 1024;
  const double chain = blocks / splits * alone + 4.0;
  return std::max(all, chain) + (splits > 1 ? 5.0 + splits * part / 2e6 : 0.0);
}

// Of all pairs of a query and a key, those that the query sees: its sequence's queries
// are the last of its keys.
inline double share_of(const Sizes& s, int64_t q, int64_t k) {
  return s.causal ? 1.0 - 0.5 * std::min(1.0, (double)q / std::max<int64_t>(1, k)) : 1.0;
}

constexpr int kTrySplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
// A part has 64 elements of the axis or more.  Without a tile there is nothing to join, nor
// a row for the launch that would (a grid of no workgroups is an error).
inline bool may_split(int splits, int64_t axis, int64_t units) {
  return splits == 1 || (units > 0 && splits * 64 <= axis);
}

// Over the queries (forward; dq) with tiles of the given waves.  A tile that the queries
// of a head would not fill takes those of all heads that share k and v.
inline Plan over_queries(const Sizes& s, const Kernel& kernel, const int* waves, int options) {
  Plan best{width_of(s.dim), waves[0], 1, 1, 0};
  const int n = std::max(1, s.n);
  const int64_t q = ceil_div(s.q_tokens, n), k = ceil_div(s.k_tokens, n);  // of a sequence
  if (!s.bias && s.group > 1 && q < kRows * 4 && s.q_tokens * s.group < (int64_t)1 << 30) best.pack = s.group;
  double least = 1e30;
  for (int i = 0; i < options; ++i) {
    // waves without a query wait, and cost nothing; no tile is twice as long as they need
    const int busy = (int)std::min<int64_t>(waves[i], ceil_div(q * best.pack, kRows));
    if (i > 0 && busy <= waves[i] / 2) continue;
    const int64_t units = n * ceil_div(q * best.pack, kRows * waves[i]) * (s.heads / best.pack);
    for (int splits : kTrySplits) {
      if (!may_split(splits, k, units)) break;
      const double us = time_of(kernel, s, best.width, units, waves[i], busy, k, share_of(s, q, k), splits,
                                4.0 * s.q_tokens * s.heads * s.dim);
      if (us < least) least = us, best.waves = waves[i], best.splits = splits;
    }
  }
  best.slots = slots_of(s.q_tokens, best.pack, s.n, kRows * best.waves);
  return best;
}

// Over the keys (dk and dv), each of which goes over the queries of its heads.
inline Plan over_keys(const Sizes& s, int waves) {
  Plan best{width_of(s.dim), waves, 1, 1, 0};
  const int n = std::max(1, s.n);
  const int64_t q = ceil_div(s.q_tokens, n), k = ceil_div(s.k_tokens, n);
  const int64_t units = n * ceil_div(k, kRows * waves) * (s.heads / s.group), axis = ceil_div(q, kRows) * kRows * s.group;
  double least = 1e30;
  for (int splits : kTrySplits) {
    if (!may_split(splits, axis, units)) break;
    const double us = time_of(kDkv, s, best.width, units, waves, waves, axis, share_of(s, q, k), splits,
                              8.0 * s.k_tokens * (s.heads / s.group) * s.dim);
    if (us < least) least = us, best.splits = splits;
  }
  best.slots = slots_of(s.k_tokens, 1, s.n, kRows * waves);
  return best;
}

// Waves of a workgroup.  Eight for 96 and 128 columns, whose registers leave two to a SIMD
// room (with four the forward pass takes them where sequences are short).  Over the keys of
// narrow heads eight where sequences are long (8192 tokens, 16 heads of 64, causal: 608 us
// for the backward pass, 739 with four) and four where they are short (32 sequences: 115
// and 105).
inline Plan plan_forward(const Sizes& s) {
  const int width = width_of(s.dim);
  constexpr int waves[] = {4, 8};
  return over_queries(s, kForward, waves, s.bf16 && (width == 96 || width == 128) ? 2 : 1);
}
// dq sums the bias's gradient by distance in every wave: the LDS of eight waves' sums
// beside the tiles (128 rows of 256 bytes) and the waves' blocks holds spans up to 1468.
constexpr int kSpanOfEight = 1468;
constexpr int dq_waves(bool bf16, int width, int span) {
  return bf16 && width > 64 && width <= 128 && span <= kSpanOfEight ? 8 : 4;
}
inline int dkv_waves(bool bf16, int width, int64_t keys) {
  return bf16 && (width == 64 ? keys >= 512 : width <= 128) ? 8 : 4;
}
inline Plan plan_dq(const Sizes& s) {
  const int waves[] = {dq_waves(s.bf16, width_of(s.dim), s.span)};
  return over_queries(s, kDq, waves, 1);
}
inline Plan plan_dkv(const Sizes& s) {
  return over_keys(s, dkv_waves(s.bf16, width_of(s.dim), ceil_div(s.k_tokens, std::max(1, s.n))));
}

}  // namespace attn
}  // namespace rip
