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

// How numbers enter the matrix instructions: bf16 as they are; fp32 as three bf16
// numbers whose sum they are (24 bits = 8 + 8 + 8), with the six products of parts that
// reach fp32's last bit, at six times the cost of bf16; or, where those do not fit the
// registers, fp32's own instructions, at sixteen times.
enum { kBf16 = RIP_BF16, kSplit = 2, kFp32 = 3 };
constexpr int storage(int number) { return number == kBf16 ? RIP_BF16 : RIP_FP32; }

// Eight elements as they are loaded, 16 bytes a word (RAW[1] bf16, RAW[2] fp32).
//
// Columns c .. c + 7 of a row of d: where they end past d, the row's last eight are
// loaded instead, and dropped at the front, which leaves zeros at the end (d >= 8).
__device__ __forceinline__ int first_column(int c, int d) { return c < d ? min(c, d - kLane) : 0; }
template <int WORDS>
__device__ __forceinline__ void drop_front(u32x4 (&x)[WORDS], int n) {
  constexpr int N = 4 * WORDS;
  uint32_t w[N];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = x[i / 4][i % 4];
  const int words = WORDS == 1 ? n / 2 : n;
#pragma unroll
  for (int by = N / 2; by >= 1; by /= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = words & by ? (i + by < N ? w[i + by] : 0u) : w[i];
  if (WORDS == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t next = i + 1 < N ? w[i + 1] : 0u;
      w[i] = n & 1 ? w[i] >> 16 | next << 16 : w[i];
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i / 4][i % 4] = w[i];
}
// What columns c .. c + 7 of a row of d are, from what first_column() loaded.
template <int WORDS>
__device__ __forceinline__ void cut_columns(u32x4 (&x)[WORDS], int c, int d, bool row) {
  if (d % kLane) drop_front<WORDS>(x, c < d && c + kLane > d ? c + kLane - d : 0);
#pragma unroll
  for (int w = 0; w < WORDS; ++w) x[w] = row && c < d ? x[w] : u32x4{0, 0, 0, 0};
}

// Eight operands of a lane, and a product of 16 steps of the summed axis.
template <int NT>
struct Frag;
template <>
struct Frag<kBf16> {
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
  __device__ __forceinline__ void set(const u32x4 (&raw)[1]) { set(raw[0]); }
};
template <>
struct Frag<kSplit> {
  bf16x8 x[3];
  // The leading eight bits, cut (so that nothing rounds to an infinity), the next eight
  // rounded, and the rest, which is exact.  An infinity is its first part alone.
  static __device__ __forceinline__ void cut(const float (&f)[8], u32x4 (&part)[3]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float r[2];
      uint32_t lead[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        lead[h] = __float_as_uint(f[2 * j + h]);
        r[h] = f[2 * j + h] - __uint_as_float(lead[h] & 0xffff0000u);
        r[h] = __builtin_isinf(f[2 * j + h]) ? 0.0f : r[h];
      }
      part[0][j] = __builtin_amdgcn_perm(lead[1], lead[0], 0x07060302u);
      const uint32_t next = Elem<RIP_BF16>::pack2(r[0], r[1]);
      part[1][j] = next;
      part[2][j] = Elem<RIP_BF16>::pack2(r[0] - __uint_as_float(next << 16),
                                         r[1] - __uint_as_float(next & 0xffff0000u));
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    u32x4 part[3];
    cut(f, part);
#pragma unroll
    for (int i = 0; i < 3; ++i) x[i] = __builtin_bit_cast(bf16x8, part[i]);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    float a[8], b[8];
    Elem<RIP_BF16>::unpack8(__builtin_bit_cast(u32x4, x[0]), f);
    Elem<RIP_BF16>::unpack8(__builtin_bit_cast(u32x4, x[1]), a);
    Elem<RIP_BF16>::unpack8(__builtin_bit_cast(u32x4, x[2]), b);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] += a[j] + b[j];
  }
  __device__ __forceinline__ void set(const u32x4 (&raw)[2]) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(raw[j / 4][j % 4]);
    set(f);
  }
};
template <>
struct Frag<kFp32> {
  float x[8];
  __device__ __forceinline__ void set(const float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = f[j];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = x[j];
  }
  __device__ __forceinline__ void set(const u32x4 (&raw)[2]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(raw[j / 4][j % 4]);
  }
};
__device__ __forceinline__ f32x16 mma(const Frag<kBf16>& a, const Frag<kBf16>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}
// The smallest products first.
__device__ __forceinline__ f32x16 mma(const Frag<kSplit>& a, const Frag<kSplit>& b, f32x16 c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[0], b.x[2], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[1], b.x[1], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[2], b.x[0], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[0], b.x[1], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[1], b.x[0], c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x[0], b.x[0], c, 0, 0, 0);
}
// Eight instructions of two steps each; the order of the summed axis is free.
__device__ __forceinline__ f32x16 mma(const Frag<kFp32>& a, const Frag<kFp32>& b, f32x16 c) {
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
// A Tile is what the kernels hold in LDS: ROWS rows of D numbers.
constexpr int pitch_of(int d, int bytes) { return (d * bytes + 127) / 128 * 128; }

template <int NT, int D>
struct Tile;
template <int D>
struct Tile<kBf16, D> {
  typedef uint16_t T;
  static constexpr int kBytes = pitch_of(D, 2);   // of a row
  template <int ROWS>
  struct Store {
    __align__(128) char x[ROWS * kBytes];
  };
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
  __device__ __forceinline__ u32x4 row_piece(const char* tile, int first, int s) const {
    return *(const u32x4*)(tile + first * kBytes + rows[s % 4] + s / 4 * 128);
  }
  __device__ __forceinline__ u32x4 column_piece(const char* tile, int first, int c) const {
    const char* p = tile + first * kBytes + columns[c % 2] + c / 2 * 128;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * kBytes));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // Operand of row `first` + lane % 32, elements 16 s + 8 half .. (first: of 32)
  template <int ROWS>
  __device__ __forceinline__ Frag<kBf16> row(const Store<ROWS>& tile, int first, int s) const {
    Frag<kBf16> f;
    f.set(row_piece(tile.x, first, s));
    return f;
  }
  // Operand of column 32 c + lane % 32 over the 16 rows from `first` (a multiple of
  // 16), in block_row's order: rows first + 4 half .. + 3, then those 8 further.
  template <int ROWS>
  __device__ __forceinline__ Frag<kBf16> column(const Store<ROWS>& tile, int first, int c) const {
    Frag<kBf16> f;
    f.set(column_piece(tile.x, first, c));
    return f;
  }
  template <int ROWS>  // eight elements of a row from column 8 `unit` on
  static __device__ __forceinline__ void put(Store<ROWS>& tile, int row, int unit, const u32x4 (&x)[1]) {
    *(u32x4*)(tile.x + row * kBytes + (unit ^ swizzle(row)) * 16) = x[0];
  }
};
template <int D>
struct Tile<kSplit, D> {
  typedef float T;
  typedef Tile<kBf16, D> Part;
  template <int ROWS>
  struct Store {
    typename Part::template Store<ROWS> part[3];
  };
  Part at;
  __device__ __forceinline__ explicit Tile(int lane) : at(lane) {}
  template <int ROWS>
  __device__ __forceinline__ Frag<kSplit> row(const Store<ROWS>& tile, int first, int s) const {
    Frag<kSplit> f;
#pragma unroll
    for (int i = 0; i < 3; ++i) f.x[i] = __builtin_bit_cast(bf16x8, at.row_piece(tile.part[i].x, first, s));
    return f;
  }
  template <int ROWS>
  __device__ __forceinline__ Frag<kSplit> column(const Store<ROWS>& tile, int first, int c) const {
    Frag<kSplit> f;
#pragma unroll
    for (int i = 0; i < 3; ++i)
      f.x[i] = __builtin_bit_cast(bf16x8, at.column_piece(tile.part[i].x, first, c));
    return f;
  }
  template <int ROWS>
  static __device__ __forceinline__ void put(Store<ROWS>& tile, int row, int unit, const u32x4 (&x)[2]) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(x[j / 4][j % 4]);
    u32x4 part[3];
    Frag<kSplit>::cut(f, part);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      *(u32x4*)(tile.part[i].x + row * Part::kBytes + (unit ^ swizzle(row)) * 16) = part[i];
  }
};
template <int D>
struct Tile<kFp32, D> {
  typedef float T;
  static constexpr int kBytes = pitch_of(D, 4);
  template <int ROWS>
  struct Store {
    __align__(128) char x[ROWS * kBytes];
  };
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
  template <int ROWS>
  __device__ __forceinline__ Frag<kFp32> row(const Store<ROWS>& tile, int first, int s) const {
    const char* p = tile.x + first * kBytes + s / 2 * 128;
    const f32x4 a = *(const f32x4*)(p + rows[s % 2 * 2]), b = *(const f32x4*)(p + rows[s % 2 * 2 + 1]);
    Frag<kFp32> f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f.x[j] = a[j], f.x[4 + j] = b[j];
    return f;
  }
  template <int ROWS>
  __device__ __forceinline__ Frag<kFp32> column(const Store<ROWS>& tile, int first, int c) const {
    Frag<kFp32> f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      f.x[j] = *(const float*)(tile.x + (first + j / 4 * 8) * kBytes + columns[j % 4] + c * 128);
    return f;
  }
  template <int ROWS>
  static __device__ __forceinline__ void put(Store<ROWS>& tile, int row, int unit, const u32x4 (&x)[2]) {
#pragma unroll
    for (int w = 0; w < 2; ++w)
      *(u32x4*)(tile.x + row * kBytes + ((2 * unit + w) ^ swizzle(row)) * 16) = x[w];
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

constexpr int two_power(int n) { return n <= 1 ? 1 : 2 * two_power((n + 1) / 2); }

// Rows on their way to LDS: ROWS rows of d <= D elements, by THREADS threads, in units
// of eight elements.  Rows shorter than that go straight there.
template <int NT, int D, int ROWS, int THREADS>
struct Stage {
  typedef Tile<NT, D> Tl;
  typedef typename Tl::T T;
  typedef typename Tl::template Store<ROWS> Store;
  static constexpr int DT = storage(NT);
  static constexpr int kPerRow = two_power(D / kLane);   // threads
  static constexpr int kAtOnce = THREADS / kPerRow;      // rows
  static constexpr int kUnits = ROWS / kAtOnce;
  static constexpr int kWords = DT == RIP_BF16 ? 1 : 2;  // 16 bytes each
  static constexpr int kPiece = 16 / (int)sizeof(T);
  static_assert(THREADS % kPerRow == 0 && ROWS % kAtOnce == 0, "whole rows at once");
  u32x4 x[kUnits][kWords];

  // Rows row .. of the `rows` (at least one) from `base` on.  What lies past the end or past
  // column d is loaded from inside, without a branch, and left out by store().
  __device__ __forceinline__ void load(const T* base, int64_t ld, int row, int rows, int d) {
    if (d < kLane) return;
    const int r = threadIdx.x / kPerRow, c = first_column(threadIdx.x % kPerRow * kLane, d);
    const int from = min(row, rows - 1);              // a tile may lie past the end
    const T* first = base + from * ld;                // the same in every lane
    if (row + ROWS <= rows) {
      const uint32_t at = (uint32_t)r * (uint32_t)ld + c;
#pragma unroll
      for (int i = 0; i < kUnits; ++i)
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          x[i][w] = *(const u32x4_any*)(first + i * kAtOnce * ld + at + w * kPiece);
    } else {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const uint32_t at = (uint32_t)min(r + i * kAtOnce, rows - 1 - from) * (uint32_t)ld + c;
#pragma unroll
        for (int w = 0; w < kWords; ++w) x[i][w] = *(const u32x4_any*)(first + at + w * kPiece);
      }
    }
  }
  // What load() took, with zeros past the end and past column d; the arguments are the
  // same.
  __device__ __forceinline__ void store(Store& tile, const T* base, int64_t ld, int row, int rows, int d) {
    const int r = threadIdx.x / kPerRow, unit = threadIdx.x % kPerRow, c = unit * kLane;
    if (kPerRow * kLane != D && c >= D) return;
    if (d < kLane) {
#pragma unroll 1
      for (int i = 0; i < kUnits; ++i) {
        const int at = row + r + i * kAtOnce;
        float f[kLane] = {};
        if (at < rows && unit == 0) load_tail<DT>(base + at * ld, d, f);
        u32x4 v[kWords];
#pragma unroll
        for (int j = 0; j < kLane; ++j) {
          if constexpr (DT == RIP_FP32)
            v[j / 4][j % 4] = __float_as_uint(f[j]);
          else if (j % 2)
            v[0][j / 2] = Elem<RIP_BF16>::pack2(f[j - 1], f[j]);
        }
        Tl::put(tile, r + i * kAtOnce, unit, v);
      }
      return;
    }
    if (row + ROWS > rows || d != D) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) cut_columns<kWords>(x[i], c, d, row + r + i * kAtOnce < rows);
    }
#pragma unroll
    for (int i = 0; i < kUnits; ++i) Tl::put(tile, r + i * kAtOnce, unit, x[i]);
  }
};

// Operands of one row in registers: elements 16 s + 8 half .. for every s, zeros unless
// `valid` (the row is readable all the same; no load waits behind a branch).
template <int NT, int D>
__device__ __forceinline__ void load_row(const typename Tile<NT, D>::T* row, bool valid, int half, int d,
                                         Frag<NT> (&f)[D / 16]) {
  constexpr int DT = storage(NT), WORDS = DT == RIP_BF16 ? 1 : 2;
  if (d >= kLane) {
    u32x4 raw[D / 16][WORDS];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const auto* p = row + first_column(16 * s + 8 * half, d);
#pragma unroll
      for (int w = 0; w < WORDS; ++w) raw[s][w] = *(const u32x4_any*)(p + 4 * w);
    }
    if (d == D) {
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int w = 0; w < WORDS; ++w) raw[s][w] = valid ? raw[s][w] : u32x4{0, 0, 0, 0};
    } else {
#pragma unroll
      for (int s = 0; s < D / 16; ++s) cut_columns<WORDS>(raw[s], 16 * s + 8 * half, d, valid);
    }
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f[s].set(raw[s]);
  } else {
    float x[kLane] = {};
    if (valid && half == 0) load_tail<DT>(row, d, x);
    f[0].set(x);
#pragma unroll
    for (int s = 1; s < D / 16; ++s) f[s] = Frag<NT>{};
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
  } else if (other.offsets != here.offsets || other.tokens != here.tokens) {
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

// Ends a group of instructions: the compiler orders those of a group, and moves none
// into another.  A group reads the operands of the next one and multiplies its own, so
// that LDS's latency lies beside products; left to itself the compiler reads each
// operand right before its product.
__device__ __forceinline__ void group_end() { __builtin_amdgcn_sched_barrier(0); }

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
// query) up to first, lut[size - 1] for all from first + size - 1 on, and kLutPad
// copies of each beside them, so that a block that lies partly in between needs no look
// at its ends: its distances reach 62 past them.
// ---------------------------------------------------------------------------
constexpr int kLutPad = 64;
struct Bias {
  const float* lut;  // of distance first
  int first, size;
  // Distances from `a` to `b` all have lut[0] (-1) or lut[size - 1] (1); 0: neither.
  __device__ __forceinline__ int uniform(int a, int b) const {
    return b <= first ? -1 : a >= first + size - 1 ? 1 : 0;
  }
  __device__ __forceinline__ float far(int side) const { return lut[side < 0 ? 0 : size - 1]; }
};
// LDS: kLutPad + lut_size + kLutPad numbers from `lut` on.
__device__ __forceinline__ void load_lut(const Args& p, const Buckets& map, int head, float* lut) {
  for (int i = threadIdx.x; i < p.lut_size + 2 * kLutPad; i += blockDim.x) {
    const int at = min(max(i - kLutPad, 0), p.lut_size - 1);
    lut[i] = p.lut ? p.lut[(int64_t)head * p.lut_size + at] : bias_at(map, p.lut_first + at, head);
  }
}
__host__ __device__ constexpr int lut_floats(int lut_size) { return lut_size + 2 * kLutPad; }

// Scores of a block in the log2 domain with the bias; side: Bias::uniform of the block.
// Register r is at distance rel + SIGN * row, row = block_row(r, 0) (rel has the half).
template <int SIGN>
__device__ __forceinline__ void add_bias(f32x16& s, float scale2, const Bias& bias, int side, int rel) {
  if (side) {
    const float b = bias.far(side);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], scale2, b);
  } else {
    // lanes whose query (or key) does not exist repeat the last one's place
    const float* at = bias.lut + (rel - bias.first);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], scale2, at[SIGN * block_row(r, 0)]);
  }
}

}  // namespace attn
}  // namespace rip
