// Pieces that the attention kernels share (device code of rip_attn_forward.hip and
// rip_attn_backward.hip): where a workgroup's sequence lies, rows on their way to
// LDS, the operands of the matrix instructions, and the bias of a distance.
//
// Layouts.  A matrix instruction computes a 32 x 32 block with 16 products of the
// summed axis: lane l gives eight of row (or column) l % 32, the summed axis' places
// 8 (l / 32) .. + 7, and receives of column l % 32 the 16 rows block_row(r, l / 32).
// Scores are computed with the axis that the next product sums over as rows, so that
// a lane's 16 results, in order, are its operand of that product: the probabilities
// never leave their registers.  The other operand then takes the rows in the same
// order (Columns below).
#pragma once

#include "rip_attn.h"

namespace rip {
namespace attn {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ int block_row(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

// Eight operands of a lane, and a product of 16 steps of the summed axis.
template <int DT>
struct Frag;
template <>
struct Frag<RIP_BF16> {
  bf16x8 x;
  __device__ __forceinline__ void set(u32x4 v) { x = __builtin_bit_cast(bf16x8, v); }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = Elem<RIP_BF16>::pack2(f[2 * j], f[2 * j + 1]);
    set(v);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    Elem<RIP_BF16>::unpack8(__builtin_bit_cast(u32x4, x), f);
  }
};
template <>
struct Frag<RIP_FP32> {
  float x[8];
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f[j];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = x[j];
  }
};
__device__ __forceinline__ f32x16 mma(const Frag<RIP_BF16>& a, const Frag<RIP_BF16>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}
// fp32: eight instructions of two steps each; the order of the summed axis is free.
__device__ __forceinline__ f32x16 mma(const Frag<RIP_FP32>& a, const Frag<RIP_FP32>& b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[j], b.x[j], c, 0, 0, 0);
  return c;
}

// The value of the lane 32 away beside one's own, combined.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---------------------------------------------------------------------------
// Rows in LDS.  A row takes a multiple of 128 bytes, and its 16-byte pieces lie
// turned by swizzle(row): both eight consecutive rows' same piece (row operands) and
// four rows' 32 bytes (transposing reads) fall into different banks.
// ---------------------------------------------------------------------------
__device__ __forceinline__ int swizzle(int row) { return (row & 3) << 1 | (row >> 2 & 1); }

// Swizzles change the lowest three bits of a piece's number alone, and those of a
// lane's rows are the same in every block, so few addresses (bytes) serve all blocks:
// the rest of an address is known when the code is compiled.
template <int DT, int D>
struct Tile;
template <int D>
struct Tile<RIP_BF16, D> {
  typedef uint16_t T;
  static constexpr int kPiece = 8;                    // elements of 16 bytes
  static constexpr int kPitch = D < 64 ? 64 : D;
  static constexpr int kBytes = kPitch * 2;
  uint32_t rows[4], columns[2];
  __device__ __forceinline__ explicit Tile(int lane) {
    const int r = lane % 32, half = lane / 32;
#pragma unroll
    for (int s = 0; s < 4; ++s) rows[s] = r * kBytes + ((2 * s + half) ^ swizzle(r)) * 16;
    // sixteen lanes read four rows of 16 columns and receive a column each
    const int group = lane / 16, in = lane % 16, row = 4 * (group / 2) + in / 4;
#pragma unroll
    for (int c = 0; c < 2; ++c)
      columns[c] = row * kBytes + ((4 * c + group % 2 * 2 + in % 4 / 2) ^ swizzle(row)) * 16 + in % 2 * 8;
  }
  // Operand of row `first` + lane % 32, elements 16 s + 8 half .. (first: of 32)
  __device__ __forceinline__ Frag<RIP_BF16> row(const T* tile, int first, int s) const {
    Frag<RIP_BF16> f;
    f.set(*(const u32x4*)((const char*)tile + first * kBytes + rows[s % 4] + s / 4 * 128));
    return f;
  }
  // Operand of column 32 c + lane % 32 over the 16 rows from `first` (a multiple of
  // 16), in block_row's order: rows first + 4 half .. + 3, then those 8 further.
  __device__ __forceinline__ Frag<RIP_BF16> column(const T* tile, int first, int c) const {
    const char* p = (const char*)tile + first * kBytes + columns[c % 2] + c / 2 * 128;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * kBytes));
    Frag<RIP_BF16> f;
    f.set(__builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7)));
    return f;
  }
};
template <int D>
struct Tile<RIP_FP32, D> {
  typedef float T;
  static constexpr int kPiece = 4;
  static constexpr int kPitch = D < 32 ? 32 : D;
  static constexpr int kBytes = kPitch * 4;
  uint32_t rows[4], columns[4];
  __device__ __forceinline__ explicit Tile(int lane) {
    const int r = lane % 32, half = lane / 32;
#pragma unroll
    for (int s = 0; s < 4; ++s)
      rows[s] = r * kBytes + ((s / 2 * 4 + 2 * half + s % 2) ^ swizzle(r)) * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = 4 * half + j;
      columns[j] = row * kBytes + (lane % 32 / 4 ^ swizzle(row)) * 16 + lane % 4 * 4;
    }
  }
  __device__ __forceinline__ Frag<RIP_FP32> row(const T* tile, int first, int s) const {
    const char* p = (const char*)tile + first * kBytes + s / 2 * 128;
    const f32x4 a = *(const f32x4*)(p + rows[s % 2 * 2]), b = *(const f32x4*)(p + rows[s % 2 * 2 + 1]);
    Frag<RIP_FP32> f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f.x[j] = a[j], f.x[4 + j] = b[j];
    return f;
  }
  __device__ __forceinline__ Frag<RIP_FP32> column(const T* tile, int first, int c) const {
    Frag<RIP_FP32> f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      f.x[j] = *(const float*)((const char*)tile + (first + j / 4 * 8) * kBytes + columns[j % 4] + c * 128);
    return f;
  }
};

// The first n (1 .. 7) of eight elements, then zeros; the others are not read.
template <int DT>
__device__ __forceinline__ void load_tail(const typename Elem<DT>::T* p, int n, float (&f)[kLane]) {
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    const float x = Elem<DT>::load(p + min(j, n - 1));
    f[j] = j < n ? x : 0.0f;
  }
}

// Rows on their way to LDS: ROWS rows of d <= D elements, by THREADS threads, in units
// of eight elements.  Rows of a width that eight does not divide go straight there.
template <int DT, int D, int ROWS, int THREADS>
struct Stage {
  typedef typename Elem<DT>::T T;
  typedef Tile<DT, D> Tl;
  static constexpr int kPerRow = D / kLane, kAtOnce = THREADS / kPerRow;  // rows
  static constexpr int kUnits = ROWS / kAtOnce;
  static constexpr int kWords = DT == RIP_BF16 ? 1 : 2;  // 16 bytes each
  static_assert(THREADS % kPerRow == 0 && ROWS % kAtOnce == 0, "whole rows at once");
  u32x4 x[kUnits][kWords];

  // Rows row .. of the `rows` from `base` on; those past the end and columns past d
  // are zeros.
  __device__ __forceinline__ void load(const T* base, int64_t ld, int row, int rows, int d) {
    if (d % kLane) return;
    const int r = threadIdx.x / kPerRow, c = threadIdx.x % kPerRow * kLane;
    const T* first = base + row * ld;                 // the same in every lane
    const uint32_t at = (uint32_t)r * (uint32_t)ld + c;
    if (row + ROWS <= rows && d == D) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          x[i][w] = *(const u32x4_any*)(first + i * kAtOnce * ld + at + w * Tl::kPiece);
      return;
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
#pragma unroll
      for (int w = 0; w < kWords; ++w) x[i][w] = u32x4{0, 0, 0, 0};
      if (row + r + i * kAtOnce < rows && c < d) {
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          x[i][w] = *(const u32x4_any*)(first + i * kAtOnce * ld + at + w * Tl::kPiece);
      }
    }
  }
  // What load() took; the arguments are the same.
  __device__ __forceinline__ void store(T* tile, const T* base, int64_t ld, int row, int rows, int d) const {
    if (d % kLane) {
#pragma unroll 1
      for (int u = threadIdx.x; u < ROWS * kPerRow; u += THREADS) {
        const int r = u / kPerRow, c = u % kPerRow * kLane;
        float f[kLane] = {};
        if (row + r < rows && c < d) {
          const T* p = base + (row + r) * ld + c;
          if (c + kLane <= d)
            Elem<DT>::load8(p, f);
          else
            load_tail<DT>(p, d - c, f);
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (DT == RIP_BF16)
              v[j] = Elem<RIP_BF16>::pack2(f[2 * j], f[2 * j + 1]);
            else
              v[j] = __float_as_uint(f[4 * w + j]);
          }
          *(u32x4*)((char*)tile + r * Tl::kBytes + ((c / Tl::kPiece + w) ^ swizzle(r)) * 16) = v;
        }
      }
      return;
    }
    const int r = threadIdx.x / kPerRow, piece = threadIdx.x % kPerRow * (kLane / Tl::kPiece);
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int row = r + i * kAtOnce;
#pragma unroll
      for (int w = 0; w < kWords; ++w)
        *(u32x4*)((char*)tile + row * Tl::kBytes + ((piece + w) ^ swizzle(row)) * 16) = x[i][w];
    }
  }
};

// Operands of one row in registers: elements 16 s + 8 half .. for every s.
template <int DT, int D>
__device__ __forceinline__ void load_row(const typename Elem<DT>::T* row, bool valid, int half, int d,
                                         Frag<DT> (&f)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    float x[kLane] = {};
    const int c = 16 * s + 8 * half;
    if (valid && c + kLane <= d) Elem<DT>::load8(row + c, x);
    f[s].set(x);
  }
  if (d % kLane == 0) return;
  const int unit = d / kLane;  // the one that ends inside
  float x[kLane] = {};
  if (valid && half == unit % 2) load_tail<DT>(row + unit * kLane, d % kLane, x);
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
    if (s == unit / 2) {
      float y[kLane];
      f[s].get(y);
#pragma unroll
      for (int j = 0; j < kLane; ++j) y[j] = half == unit % 2 ? x[j] : y[j];
      f[s].set(y);
    }
}

// The 4 consecutive elements that a lane holds of its row: c .. c + 3 below d.
template <int DT>
__device__ __forceinline__ void store4(typename Elem<DT>::T* row, int c, int d, const float (&f)[4]) {
  if (c + 4 <= d) {
    if constexpr (DT == RIP_BF16) {
      typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
      *(u32x2_any*)(row + c) =
          u32x2_any{Elem<DT>::pack2(f[0], f[1]), Elem<DT>::pack2(f[2], f[3])};
    } else {
      *(u32x4_any*)(row + c) = u32x4_any{__float_as_uint(f[0]), __float_as_uint(f[1]),
                                         __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < d) Elem<DT>::store(row + c + j, f[j]);
  }
}

// ---------------------------------------------------------------------------
// A workgroup's sequence.  With T tokens to a tile, sequence e begins at slot
// B[e] / T + e, so that there are slots enough for its tiles whatever the offsets;
// B[0] = 0, then the offsets, cut to 0 .. total and to the largest before them, then
// the total.  Sequences 0 and n + 1 are the tokens that belong to none.
// ---------------------------------------------------------------------------
struct Span {
  int begin, end;
};
struct Place {
  Span here, other;  // tokens of the side that is tiled, and of the other side
  int tile;          // of the sequence; it may lie past its end
};

__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
  for (int o = 32; o >= 1; o /= 2) x = max(x, __shfl_xor(x, o));
  return x;
}

// `here` in tiles of PER elements, `pack` to a token.  Every wave finds it by itself.
template <int PER>
__device__ __forceinline__ Place find(const Args& p, const Side& here, const Side& other, int slot,
                                      int pack) {
  const int lane = threadIdx.x % 64, n = p.n_seqs;
  int e, lo = 0, hi = here.tokens;
  if (p.cleaned) {  // offsets in order: the last e with a slot up to this one
    int a = 0, b = n + 1;
    while (a < b) {
      const int mid = (a + b + 1) / 2;
      if (here.offsets[mid - 1] * pack / PER + mid <= slot)
        a = mid;
      else
        b = mid - 1;
    }
    e = a;
    if (e > 0) lo = here.offsets[e - 1];
    if (e <= n) hi = here.offsets[e];
  } else {
    e = 0;
    int most = 0;
    for (int base = 0; base <= n; base += 64) {
      const int i = base + lane;
      int c = i <= n ? min(max(here.offsets[i], 0), here.tokens) : here.tokens;
      c = max(c, most);
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int up = __shfl_up(c, o);
        if (lane >= o) c = max(c, up);
      }
      const bool before = i <= n && c * pack / PER + i + 1 <= slot;
      const int count = __popcll(__ballot(before));
      e += count;
      if (count > 0) lo = __shfl(c, count - 1);
      if (count < 64) {
        if (base + count <= n) hi = __shfl(c, count);
        break;
      }
      most = __shfl(c, 63);
    }
  }
  Place at{{lo, hi}, {lo, hi}, 0};
  at.tile = slot - (lo * pack / PER + e);
  if (e == 0 || e == n + 1) {
    at.other = {0, 0};
  } else if (other.offsets != here.offsets) {
    if (p.cleaned) {
      at.other = {other.offsets[e - 1], other.offsets[e]};
    } else {
      int a = 0;
      for (int i = lane; i < e; i += 64) a = max(a, min(max(other.offsets[i], 0), other.tokens));
      a = wave_max(a);
      at.other = {a, max(a, min(max(other.offsets[e], 0), other.tokens))};
    }
  }
  // the same in every lane: keep it in scalar registers
  auto uniform = [](int& x) { x = __builtin_amdgcn_readfirstlane(x); };
  uniform(at.here.begin), uniform(at.here.end), uniform(at.other.begin), uniform(at.other.end);
  uniform(at.tile);
  return at;
}

// All of the workgroup's LDS accesses before come before those after; loads from
// memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A workgroup's head (of `heads`), split and slot.  Heads go fastest: workgroups go to
// the eight XCDs, each with an L2 of its own, in turn, so that where 8 divides the
// heads (or they divide 8) a head's rows are read by one (or few) of them; and the
// slots with the most work, which come first, start first whatever their head.
struct Share {
  int head, split, slot;
};
__device__ __forceinline__ bool my_share(const Args& p, int heads, Share* s) {
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, at = id / (uint32_t)heads;
  s->head = id - at * heads;
  s->slot = at / (uint32_t)p.splits;
  s->split = at - s->slot * p.splits;
  return s->slot < p.slots;
}

// ---------------------------------------------------------------------------
// Bias by distance, times log2(e), in LDS: lut[0] holds for every distance (key -
// query) up to first, lut[size - 1] for all from first + size - 1 on.
// ---------------------------------------------------------------------------
struct Bias {
  const float* lut;
  int first, size;
  // Distances from `a` to `b` all have lut[0] (-1) or lut[size - 1] (1); 0: neither.
  __device__ __forceinline__ int uniform(int a, int b) const {
    return b <= first ? -1 : a >= first + size - 1 ? 1 : 0;
  }
  __device__ __forceinline__ float far(int side) const { return lut[side < 0 ? 0 : size - 1]; }
  __device__ __forceinline__ float near(int rel) const {
    return lut[min(max(rel - first, 0), size - 1)];
  }
};
__device__ __forceinline__ void load_lut(const Args& p, int head, float* lut) {
  const float* from = p.lut + (int64_t)head * p.lut_size;
  for (int i = threadIdx.x; i < p.lut_size; i += blockDim.x) lut[i] = from[i];
}

// Scores of a block in the log2 domain with the bias; side: Bias::uniform of the block,
// rel(r): the distance of register r.
template <typename Rel>
__device__ __forceinline__ void add_bias(f32x16& s, float scale2, const Bias& bias, int side, Rel rel) {
  if (side) {
    const float b = bias.far(side);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], scale2, b);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], scale2, bias.near(rel(r)));
  }
}

}  // namespace attn
}  // namespace rip
