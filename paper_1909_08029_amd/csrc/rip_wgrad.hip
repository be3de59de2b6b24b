// Weight gradient of a linear layer from its input's 8-bit checkpoint (gfx950):
//
//   grad[n][k] = sum_t dy[t][n] * x'[t][k],   x'[t][k] = q * 2^e
//
// A matrix product with both operands laid out along the other axis than the
// sum's.  A checkpoint's values are exact in bf16, so they go into the bf16
// matrix instructions as they are; so does a bf16 dy.  An fp32 dy is cut into
// three bf16 parts (24 bits = 8 + 8 + 8) that add up to it exactly, each with
// products of its own: fp32's accuracy at a third of bf16's rate, several times
// what the fp32 matrix instructions reach.  Sums are fp32.
//
// Bound by the matrix units where the product is large: 16384 tokens, 5504 x 2048,
// bf16, take 351 to 400 us by card and clock, the pack of x (20 us) included (920
// to 1050 TFLOP/s; a product of the same sizes without codes to widen takes the
// vendor's library 416); 8192 x 2048 x 2048 fp32 200 us (345 TFLOP/s, 1030 of bf16
// products).  Small products are bound by the steps of the smallest tile, which leaves
// most of the card idle (257 x 383 x 1000 fp32: 24 workgroups, 14.3 us), narrow layers by
// that and by the parts' way to memory.
//
// A workgroup of four or eight waves computes a tile of grad and goes over its tokens in
// steps of 32.  Rows of dy and of codes come into registers as they lie in
// memory, three steps ahead; the codes widen to bf16 on the way into LDS, which
// holds three steps; and the transposing LDS reads hand each lane eight tokens of
// its column, as the matrix instructions want them.  Where there are few tiles
// the tokens are split; the parts go to the workspace and a second launch adds
// them in order.  Eight waves, two to a SIMD, let one wave's widening run beside the
// other's matrix instructions; four of twice the size ran one after the other (491
// us for the product above).

#include "rip_ckpt_format.h"
#include "rip_wgrad_plan.h"

namespace rip {
namespace {

using namespace wgrad;

constexpr int kReduce = 256; // threads of a workgroup of the second launch
constexpr int kCodes = 16;   // codes that a lane loads at once
constexpr int kStages = 3;   // steps that LDS holds, and that are on their way in registers

// Elements between LDS rows of a tile's `n` columns.  A group of 16 lanes reads 32
// bytes of each of four rows: with rows 64 bytes past a multiple of 128 (or of 256,
// as n is a multiple of 64) the four lie in different banks, and so do the next
// group's beside them.
constexpr int pitch(int n) { return n + 32; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Eight tokens (t .. t+7 by the lane's half of the wave) of column n + lane % 32.
template <int PITCH>
__device__ __forceinline__ bf16x8 read_columns(const uint16_t* tile, int t, int n, int lane) {
  const int group = lane / 16, in = lane % 16;
  const uint16_t* p =
      tile + (t + (group / 2) * 8 + in / 4) * PITCH + n + (group % 2) * 16 + (in % 4) * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * PITCH));
  const s16x8 v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, v);
}

// x as three bf16 numbers that add up to it, each in the high half of a word: the
// leading bits, cut, and what that leaves, twice.  An infinity is the first part
// alone; a NaN's difference from its first part is a NaN whatever that part is.
__device__ __forceinline__ void cut3(float x, uint32_t (&part)[3]) {
  part[0] = __float_as_uint(x);
  float r = x - __uint_as_float(part[0] & 0xffff0000u);
  r = __builtin_isinf(x) ? 0.0f : r;
  part[1] = __float_as_uint(r);
  part[2] = __float_as_uint(r - __uint_as_float(part[1] & 0xffff0000u));
}
// High halves of two words as one, the first below.
__device__ __forceinline__ uint32_t high_halves(uint32_t lo, uint32_t hi) {
  return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}

struct Product {
  int64_t tokens, ld_dy, ld_grad;
  int n, k;          // rows and columns of grad
  int blocks;        // checkpoint blocks of a row
  int tiles_n, tiles_k;
  int64_t share;     // tokens of a split, a multiple of kTokens
  int part_k;        // columns of a split's part in the workspace, a multiple of four
  int accumulate;
};

// The workgroup's tile and split.  Workgroups go to the eight XCDs in turn; each
// XCD, whose workgroups share an L2, takes a run of consecutive places, and places
// run through bands of four tiles along n and all tiles along k, split by split:
// 32 of them read the same tokens of four panels of dy and up to eight of x.
// (16384 x 5504 x 2048 bf16, with four waves to a tile: 528 us in row order, 494 so.)
struct Place {
  int tile_n, tile_k, split;
};
__device__ __forceinline__ Place place(const Product& p) {
  constexpr uint32_t kXcds = 8, kBand = 4;
  const uint32_t all = gridDim.x, xcd = blockIdx.x % kXcds, rest = all % kXcds;
  const uint32_t at = xcd * (all / kXcds) + (xcd < rest ? xcd : rest) + blockIdx.x / kXcds;
  const uint32_t tiles = p.tiles_n * p.tiles_k, split = at / tiles, tile = at - split * tiles;
  const uint32_t band = tile / (kBand * p.tiles_k), in = tile - band * kBand * p.tiles_k;
  const uint32_t width = min(kBand, p.tiles_n - band * kBand);
  return {(int)(band * kBand + in % width), (int)(in / width), (int)split};
}

// A tile of grad for WN x WK waves: each has 32 MN rows (along dy's columns) and
// 32 MK columns (along x's).
template <int DD, int MN_, int MK_, int WN_, int WK_>
struct Tile {
  typedef typename Elem<DD>::T T;
  static constexpr int MN = MN_, MK = MK_, WN = WN_, WK = WK_, kThreads = 64 * WN * WK;
  static constexpr int kParts = DD == RIP_FP32 ? 3 : 1;
  static constexpr int kN = 32 * MN * WN, kK = 32 * MK * WK;
  static constexpr int kPitchN = pitch(kN), kPitchK = pitch(kK);
  // Units of a thread: eight elements of dy, sixteen codes.  Where there are
  // half a round's too few, the last ones are loaded and written twice, alike.
  static constexpr int kYAll = kTokens * kN / kLane, kXAll = kTokens * kK / kCodes;
  static constexpr int kYUnits = (kYAll + kThreads - 1) / kThreads;
  static constexpr int kXUnits = (kXAll + kThreads - 1) / kThreads;
  static constexpr int kYRegs = DD == RIP_FP32 ? 2 : 1;
  static constexpr int kOperands = kParts * MN + MK;  // of 16 tokens
  static_assert(kXAll * 2 % kThreads == 0 && kYAll * 2 % kThreads == 0, "units of a thread");
  template <int ALL>
  static __device__ __forceinline__ int unit(int i) {
    const int u = threadIdx.x + i * kThreads;
    return u - (int)threadIdx.x + kThreads > ALL ? ALL - kThreads / 2 + u % (kThreads / 2) : u;
  }

  struct Shared {
    uint16_t y[kParts][kTokens * kPitchN];
    uint16_t x[kTokens * kPitchK];
  };
  struct Regs {  // a step of one thread on its way to LDS
    u32x4 y[kYUnits][kYRegs];
    u32x4 x[kXUnits];
    uint32_t e[kXUnits];
  };
  struct Offsets {  // bytes of a thread's elements in the 32 rows of a step
    uint32_t y[kYUnits], x[kXUnits], e[kXUnits];
  };
  struct Rows {  // where a step's rows begin
    const char *y, *x, *e;
  };

  // Columns past the last are read as the last ones' neighbours: whatever is there
  // only reaches rows and columns of grad that do not exist.
  static __device__ __forceinline__ Offsets offsets(const Product& p, int n0, int k0) {
    Offsets o;
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      const int u = unit<kYAll>(i);
      const int c = min(n0 + u % (kN / kLane) * kLane, (p.n - 1) / kLane * kLane);
      o.y[i] = ((uint32_t)(u / (kN / kLane)) * (uint32_t)p.ld_dy + c) * (uint32_t)sizeof(T);
    }
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      const int u = unit<kXAll>(i), row = u / (kK / kCodes);
      const int c = min(k0 + u % (kK / kCodes) * kCodes, p.blocks * kCkptBlock - kCodes);
      o.x[i] = (uint32_t)row * (uint32_t)(p.blocks * kCkptBlock) + c;
      o.e[i] = (uint32_t)row * (uint32_t)p.blocks + c / kCkptBlock;
    }
    return o;
  }

  // A step's rows, all of them tokens of the split, sixteen bytes from any column's
  // start inside dy.
  static __device__ __forceinline__ void load(const Offsets& o, const Rows& rows, Regs& r) {
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      r.x[i] = *(const u32x4*)(rows.x + o.x[i]);
      r.e[i] = *(const uint8_t*)(rows.e + o.e[i]);
    }
#pragma unroll
    for (int i = 0; i < kYUnits; ++i)
#pragma unroll
      for (int h = 0; h < kYRegs; ++h) r.y[i][h] = *(const u32x4_any*)(rows.y + o.y[i] + 16 * h);
  }

  // Rows t .. t+31 with those from `end` on and columns past the last as zeros.
  static __device__ __forceinline__ void load_checked(const Product& p, const T* dy,
                                                      const int8_t* codes, const uint8_t* exps,
                                                      int n0, int k0, int64_t t, int64_t end,
                                                      Regs& r) {
    const int width = p.blocks * kCkptBlock;
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      const int u = unit<kYAll>(i), row = u / (kN / kLane);
      const int c = n0 + u % (kN / kLane) * kLane;
      float f[kLane] = {};
      if (t + row < end && c < p.n) load_unit<DD>(dy + (t + row) * p.ld_dy, c, p.n, f);
      if constexpr (DD == RIP_FP32) {
#pragma unroll
        for (int j = 0; j < kLane; ++j) r.y[i][j / 4][j % 4] = __float_as_uint(f[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          r.y[i][0][j] = high_halves(__float_as_uint(f[2 * j]), __float_as_uint(f[2 * j + 1]));
      }
    }
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      const int u = unit<kXAll>(i), row = u / (kK / kCodes);
      const int c = min(k0 + u % (kK / kCodes) * kCodes, width - kCodes);
      r.x[i] = u32x4{0, 0, 0, 0};
      r.e[i] = 0;
      if (t + row < end) {
        r.x[i] = *(const u32x4*)(codes + (t + row) * width + c);
        r.e[i] = exps[(t + row) * p.blocks + c / kCkptBlock];
      }
    }
  }

  // What a step writes to LDS, in items: eight codes widened to bf16, or a unit of
  // dy.  [from, to) are known when the code is compiled.
  static constexpr int kItems = 2 * kXUnits + kYUnits;
  static __device__ __forceinline__ void store(Regs& r, Shared& sh, int from = 0, int to = kItems) {
#pragma unroll
    for (int i = 0; i < 2 * kXUnits; ++i) {
      if (i < from || i >= to) continue;
      // keeps the widening of the codes here, behind the wait for their load,
      // where otherwise it would move up to the load
      if (i % 2 == 0) asm("" : "+v"(r.x[i / 2]), "+v"(r.e[i / 2]));
      const int u = unit<kXAll>(i / 2), row = u / (kK / kCodes);
      const int c = u % (kK / kCodes) * kCodes + i % 2 * kLane;
      float x[kLane];
      const uint32_t codes[2] = {r.x[i / 2][i % 2 * 2], r.x[i / 2][i % 2 * 2 + 1]};
      ckpt_unpack<kLane>(codes, r.e[i / 2], x);
      u32x4 v;  // the values' low halves are zeros
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = high_halves(__float_as_uint(x[2 * j]), __float_as_uint(x[2 * j + 1]));
      *(u32x4*)&sh.x[row * kPitchK + c] = v;
    }
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      if (i + 2 * kXUnits < from || i + 2 * kXUnits >= to) continue;
      const int u = unit<kYAll>(i), row = u / (kN / kLane), c = u % (kN / kLane) * kLane;
      if constexpr (DD == RIP_FP32) {
        asm("" : "+v"(r.y[i][0]), "+v"(r.y[i][1]));
        u32x4 v[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t a[3], b[3];
          cut3(__uint_as_float(r.y[i][j / 2][2 * j % 4]), a);
          cut3(__uint_as_float(r.y[i][j / 2][2 * j % 4 + 1]), b);
#pragma unroll
          for (int q = 0; q < 3; ++q) v[q][j] = high_halves(a[q], b[q]);
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) *(u32x4*)&sh.y[q][row * kPitchN + c] = v[q];
      } else {
        *(u32x4*)&sh.y[0][row * kPitchN + c] = r.y[i][0];
      }
    }
  }

  // Operands of sixteen tokens of a wave's part of the tile: MK of x, then those
  // of dy.
  struct Frags {
    bf16x8 a[kParts][MN], b[MK];
  };
  static __device__ __forceinline__ void read(const Shared& sh, int s, int wn, int wk, int lane,
                                              Frags& f, int from = 0, int to = kOperands) {
#pragma unroll
    for (int j = 0; j < MK; ++j)
      if (j >= from && j < to) f.b[j] = read_columns<kPitchK>(sh.x, s, wk + j * 32, lane);
#pragma unroll
    for (int q = 0; q < kParts; ++q)
#pragma unroll
      for (int i = 0; i < MN; ++i)
        if (MK + q * MN + i >= from && MK + q * MN + i < to)
          f.a[q][i] = read_columns<kPitchN>(sh.y[q], s, wn + i * 32, lane);
  }
  // Row i of part q with all columns: MK matrix instructions.
  static __device__ __forceinline__ void multiply(const Frags& f, int q, int i, f32x16 (&acc)[MN][MK]) {
#pragma unroll
    for (int j = 0; j < MK; ++j)
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[q][i], f.b[j], acc[i][j], 0, 0, 0);
  }
  static __device__ __forceinline__ void multiply(const Frags& f, f32x16 (&acc)[MN][MK]) {
#pragma unroll
    for (int q = 0; q < kParts; ++q)
#pragma unroll
      for (int i = 0; i < MN; ++i) multiply(f, q, i, acc);
  }
};

// All of the workgroup's LDS accesses before come before those after; loads from
// memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Half of a step: the products of the operands in `f`, and beside every MK matrix
// instructions (each keeps its unit busy for 32 cycles) a share of the reads of the
// next operands and of the writes of a later step.  The compiler orders what lies
// between two sched_barriers, and may not gather all reads or all products.
template <typename Tl, int HALF, int C = 0, typename Load>
__device__ __forceinline__ void half(const typename Tl::Frags& f, f32x16 (&acc)[Tl::MN][Tl::MK],
                                     const typename Tl::Shared& from, int at, int wn, int wk,
                                     int lane, typename Tl::Frags& next, typename Tl::Regs& regs,
                                     typename Tl::Shared& to, Load& load) {
  constexpr int MN = Tl::MN, kRows = Tl::kParts * MN, kLast = 2 * kRows - 1;
  if constexpr (C < kRows) {
    constexpr int r0 = C * Tl::kOperands / kRows, r1 = (C + 1) * Tl::kOperands / kRows;
    constexpr int g = HALF * kRows + C;  // the last one starts the loads instead of writing
    constexpr int i0 = g * Tl::kItems / kLast, i1 = g < kLast ? (g + 1) * Tl::kItems / kLast : i0;
    Tl::read(from, at, wn, wk, lane, next, r0, r1);
    if constexpr (g < kLast)
      Tl::store(regs, to, i0, i1);
    else
      load(regs);
    Tl::multiply(f, C / MN, C % MN, acc);
    __builtin_amdgcn_sched_barrier(0);
    half<Tl, HALF, C + 1>(f, acc, from, at, wn, wk, lane, next, regs, to, load);
  }
}

template <typename Tl, int DD, int GD, int RESIDENT, bool PART>
__global__ __launch_bounds__(Tl::kThreads, RESIDENT) void wgrad_kernel(
    Product p, const typename Elem<DD>::T* dy, const int8_t* codes, const uint8_t* exps,
    typename Elem<GD>::T* grad, float* partial) {
  constexpr int MN = Tl::MN, MK = Tl::MK;
  __shared__ __align__(16) typename Tl::Shared sh[kStages];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const Place at = place(p);
  const int n0 = at.tile_n * Tl::kN, k0 = at.tile_k * Tl::kK;
  const int64_t t0 = (int64_t)at.split * p.share;
  const int64_t t1 = t0 + p.share < p.tokens ? t0 + p.share : p.tokens;
  const int wn = wave / Tl::WK * (32 * MN), wk = wave % Tl::WK * (32 * MK);
  const int steps = (int)((t1 - t0 + kTokens - 1) / kTokens);
  // The steps whose loads cannot leave dy are loaded well ahead of their use; the
  // few at the end of the tokens are not.
  const int64_t room = (p.tokens - 1) * p.ld_dy + p.n - (p.n + kLane - 1) / kLane * kLane;
  int whole = 0;
  if (room >= 0) {
    const int64_t rows = min(t1, room / p.ld_dy + 1) - t0;  // row r is safe if r * ld <= room
    whole = rows > 0 ? (int)(rows / kTokens) : 0;
  }
  f32x16 acc[MN][MK] = {};
  // A last step of fewer rows goes first: its loads are on their way together with
  // the first whole steps'.
  typename Tl::Regs tail;
  if (whole < steps)
    Tl::load_checked(p, dy, codes, exps, n0, k0, t0 + (int64_t)whole * kTokens, t1, tail);
  typename Tl::Regs regs[kStages];
  typename Tl::Frags f0, f1;
  auto product = [&](typename Tl::Regs& r) {
    Tl::store(r, sh[0]);
    lds_barrier();
    Tl::read(sh[0], 0, wn, wk, lane, f0);
    Tl::multiply(f0, acc);
    Tl::read(sh[0], 16, wn, wk, lane, f1);
    Tl::multiply(f1, acc);
    lds_barrier();
  };
  if (whole > 0) {
    const typename Tl::Offsets off = Tl::offsets(p, n0, k0);
    const int row_x = p.blocks * kCkptBlock;
    typename Tl::Rows rows = {(const char*)(dy + t0 * p.ld_dy), (const char*)(codes + t0 * row_x),
                              (const char*)(exps + t0 * p.blocks)};
    const int64_t step_y = kTokens * p.ld_dy * (int64_t)sizeof(typename Tl::T);
    int left = whole;  // steps from `rows` on
    auto load = [&](typename Tl::Regs& r) {
      Tl::load(off, rows, r);
      // past the last whole step its rows are loaded once more, and not used
      const int64_t on = left > 1;
      left -= 1;
      rows.y += on * step_y;
      rows.x += on * kTokens * row_x;
      rows.e += on * kTokens * p.blocks;
    };
    // Step s multiplies what lies in LDS stage s, writes step s + 2 to its stage
    // and starts the loads of step s + 5.  Half of a step's operands are read
    // before the barrier that begins it.
    auto step = [&](int now) {
      constexpr auto later = [](int stage, int by) { return (stage + by) % kStages; };
      typename Tl::Regs& r = regs[later(now, 2)];
      typename Tl::Shared& to = sh[later(now, 2)];
      half<Tl, 0>(f0, acc, sh[now], 16, wn, wk, lane, f1, r, to, load);
      half<Tl, 1>(f1, acc, sh[later(now, 1)], 0, wn, wk, lane, f0, r, to, load);
      lds_barrier();
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) load(regs[i]);
    if (whole < steps) product(tail);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      Tl::store(regs[i], sh[i]);
      load(regs[i]);
    }
    lds_barrier();
    Tl::read(sh[0], 0, wn, wk, lane, f0);
    // all loads done: what is on its way here would otherwise be waited for in
    // every round of the loop
    __builtin_amdgcn_s_waitcnt(0);
    for (int s = 0;;) {
      step(0);
      if (++s == whole) break;
      step(1);
      if (++s == whole) break;
      step(2);
      if (++s == whole) break;
    }
  }
  // Steps that cannot be loaded without looking (rows of a few elements, no whole
  // step): one by one.
  for (int s = whole + (whole > 0); s < steps; ++s) {
    if (s > 0) Tl::load_checked(p, dy, codes, exps, n0, k0, t0 + (int64_t)s * kTokens, t1, tail);
    product(tail);
  }
#pragma unroll
  for (int i = 0; i < MN; ++i)
#pragma unroll
    for (int j = 0; j < MK; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = n0 + wn + i * 32 + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
        const int col = k0 + wk + j * 32 + lane % 32;
        if (row >= p.n || col >= p.k) continue;
        if constexpr (PART) {
          partial[((int64_t)at.split * p.n + row) * p.part_k + col] = acc[i][j][r];
        } else {
          typename Elem<GD>::T* g = grad + (int64_t)row * p.ld_grad + col;
          Elem<GD>::store(g, p.accumulate ? Elem<GD>::load(g) + acc[i][j][r] : acc[i][j][r]);
        }
      }
}

// The splits' parts added up: four columns to a thread, a run of the splits to each
// of GROUPS groups of threads, whose sums are then added in order.
template <int GD, int GROUPS>
__global__ __launch_bounds__(kReduce) void reduce_kernel(Product p, const float* partial,
                                                         int splits,
                                                         typename Elem<GD>::T* grad) {
  constexpr int kColumns = kReduce / GROUPS;
  __shared__ float4 sums[GROUPS][kColumns];
  const int in = threadIdx.x % kColumns, group = threadIdx.x / kColumns;
  const int64_t quads = (int64_t)p.n * p.part_k / 4, i = (int64_t)blockIdx.x * kColumns + in;
  float4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (i < quads) {
    const float4* q = (const float4*)partial + i;
    const int to = (group + 1) * splits / GROUPS;
#pragma unroll 8
    for (int s = group * splits / GROUPS; s < to; ++s) {
      const float4 v = q[s * quads];
      sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
  }
  if constexpr (GROUPS > 1) {
    sums[group][in] = sum;
    __syncthreads();
    if (group) return;
    for (int g = 1; g < GROUPS; ++g) {
      const float4 v = sums[g][in];
      sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
    }
  }
  if (i >= quads) return;
  const int per_row = p.part_k / 4, row = (int)(i / per_row), col = (int)(i - (int64_t)row * per_row) * 4;
  typename Elem<GD>::T* g = grad + (int64_t)row * p.ld_grad + col;
  const float f[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < p.k) Elem<GD>::store(g + j, p.accumulate ? Elem<GD>::load(g + j) + f[j] : f[j]);
}

template <int DD, int GD, int MN, int MK, int WN, int WK, int RESIDENT>
int32_t run_tile(Product& p, const Plan& plan, void** args, void* stream) {
  typedef Tile<DD, MN, MK, WN, WK> Tl;
  const void* fn = plan.splits > 1 ? (const void*)wgrad_kernel<Tl, DD, GD, RESIDENT, true>
                                   : (const void*)wgrad_kernel<Tl, DD, GD, RESIDENT, false>;
  return launch(fn, dim3((uint32_t)(plan.tiles_n * plan.tiles_k * plan.splits)),
                dim3(Tl::kThreads), args, 0, stream, "rip_ckpt_wgrad");
}

template <int DD, int GD>
int32_t run(Product& p, const Plan& plan, const void* dy, const int8_t* codes, const uint8_t* exps,
            void* grad, float* partial, void* stream) {
  void* args[] = {&p, &dy, &codes, &exps, &grad, &partial};
  int32_t rc;
  if constexpr (DD == RIP_FP32)
    rc = plan.shape == 0 ? run_tile<DD, GD, 2, 1, 2, 4, 2>(p, plan, args, stream)
                         : run_tile<DD, GD, 2, 2, 2, 4, 2>(p, plan, args, stream);
  else
    rc = plan.shape == 0   ? run_tile<DD, GD, 2, 2, 2, 2, 2>(p, plan, args, stream)
         : plan.shape == 1 ? run_tile<DD, GD, 3, 2, 2, 4, 2>(p, plan, args, stream)
                           : run_tile<DD, GD, 4, 2, 2, 4, 2>(p, plan, args, stream);
  if (rc || plan.splits == 1) return rc;
  int splits = plan.splits;
  void* args2[] = {&p, &partial, &splits, &grad};
  // few columns: several groups of threads share the splits
  const int64_t quads = (int64_t)p.n * p.part_k / 4;
  const bool few = quads < 1 << 17;
  const void* add = few ? (const void*)reduce_kernel<GD, 8> : (const void*)reduce_kernel<GD, 1>;
  return launch(add, dim3((uint32_t)ceil_div(quads, few ? kReduce / 8 : kReduce)), dim3(kReduce),
                args2, 0, stream, "rip_ckpt_wgrad: reduce");
}

int64_t part_bytes(const Plan& plan, int64_t n) {
  return plan.splits > 1 ? plan.splits * n * plan.part_k * 4 : 0;
}

bool sizes_ok(int64_t tokens, int64_t n, int64_t k) {
  return tokens >= 0 && tokens <= RIP_MAX_TOKENS && n >= 1 && n <= RIP_MAX_FEATURES && k >= 1 &&
         k <= RIP_MAX_FEATURES;
}

}  // namespace
}  // namespace rip

using namespace rip;

extern "C" int64_t rip_ckpt_wgrad_workspace(int32_t dy_dtype, int64_t rows,
                                            int64_t out_features, int64_t in_features) {
  if (!known_dtype(dy_dtype) || !sizes_ok(rows, out_features, in_features)) return 0;
  return part_bytes(make_plan(dy_dtype, rows, out_features, in_features), out_features);
}

extern "C" int32_t rip_ckpt_wgrad(const void* dy, int32_t dy_dtype, int64_t ld_dy, int64_t rows,
                                  int64_t out_features, const int8_t* codes, const uint8_t* exps,
                                  int64_t in_features, void* grad, int32_t grad_dtype,
                                  int64_t ld_grad, int32_t accumulate, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  clear_error();
  int32_t rc;
  if (rows < 0 || out_features < 1 || in_features < 1)
    return fail(RIP_E_INVAL, "rip_ckpt_wgrad: %lld rows, %lld x %lld features", (long long)rows,
                (long long)out_features, (long long)in_features);
  if (!sizes_ok(rows, out_features, in_features))
    return fail(RIP_E_UNSUPPORTED, "rip_ckpt_wgrad: %lld rows, %lld x %lld features are above the limit",
                (long long)rows, (long long)out_features, (long long)in_features);
  if ((rc = check_matrix(dy, "dy", dy_dtype, rows, out_features, ld_dy)) ||
      (rc = check_matrix(grad, "grad", grad_dtype, out_features, in_features, ld_grad)))
    return rc;
  if (rows && (!codes || !exps)) return fail(RIP_E_INVAL, "rip_ckpt_wgrad: codes or exps is NULL");
  if (reinterpret_cast<uintptr_t>(codes) % 16)
    return fail(RIP_E_ALIGN, "rip_ckpt_wgrad: codes = %p is not 16-byte aligned", codes);
  if (ld_dy > RIP_MAX_WIDTH)
    return fail(RIP_E_UNSUPPORTED, "rip_ckpt_wgrad: row stride %lld of dy is above the limit",
                (long long)ld_dy);
  const Plan plan = make_plan(dy_dtype, rows, out_features, in_features);
  const int64_t need = part_bytes(plan, out_features);
  if (need && (!workspace || workspace_bytes < need))
    return fail(RIP_E_INVAL, "rip_ckpt_wgrad: workspace of %lld bytes, %lld needed",
                (long long)workspace_bytes, (long long)need);
  if (reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(RIP_E_ALIGN, "rip_ckpt_wgrad: workspace = %p is not 16-byte aligned", workspace);
  const int64_t blocks = ceil_div(in_features, kCkptBlock);
  const int64_t gs = span(grad_dtype, out_features, in_features, ld_grad);
  const int64_t ys = span(dy_dtype, rows, out_features, ld_dy);
  if (overlap(grad, gs, dy, ys) || overlap(grad, gs, codes, rows * blocks * kCkptBlock) ||
      overlap(grad, gs, exps, rows * blocks) || overlap(workspace, need, grad, gs) ||
      overlap(workspace, need, dy, ys) ||
      overlap(workspace, need, codes, rows * blocks * kCkptBlock) ||
      overlap(workspace, need, exps, rows * blocks))
    return fail(RIP_E_OVERLAP, "rip_ckpt_wgrad: grad or workspace overlaps another buffer");
  if (rows == 0 && accumulate) return RIP_OK;
  Product p{rows,
            ld_dy,
            ld_grad,
            (int)out_features,
            (int)in_features,
            (int)blocks,
            plan.tiles_n,
            plan.tiles_k,
            plan.share,
            plan.part_k,
            accumulate};
  float* partial = static_cast<float*>(workspace);
  if (dy_dtype == RIP_FP32)
    return grad_dtype == RIP_FP32
               ? run<RIP_FP32, RIP_FP32>(p, plan, dy, codes, exps, grad, partial, stream)
               : run<RIP_FP32, RIP_BF16>(p, plan, dy, codes, exps, grad, partial, stream);
  return grad_dtype == RIP_FP32
             ? run<RIP_BF16, RIP_FP32>(p, plan, dy, codes, exps, grad, partial, stream)
             : run<RIP_BF16, RIP_BF16>(p, plan, dy, codes, exps, grad, partial, stream);
}
