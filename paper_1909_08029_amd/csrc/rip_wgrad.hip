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
// A workgroup of four waves computes a tile of grad and goes over its tokens in
// steps of 32.  Rows of dy and of codes come into registers as they lie in
// memory, three steps ahead; the codes widen to bf16 on the way into LDS, which
// holds three steps; and the transposing LDS reads hand each lane eight tokens of
// its column, as the matrix instructions want them.  Where there are few tiles
// the tokens are split; the parts go to the workspace and a second launch adds
// them in order.

#include "rip_ckpt_format.h"

namespace rip {
namespace {

constexpr int kTokens = 32;  // tokens of a step
constexpr int kThreads = 256;
constexpr int kCodes = 16;   // codes that a lane loads at once
constexpr int kStages = 4;   // steps that LDS holds
constexpr int kLoads = 2;    // steps that are on their way in registers

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

// x as three bf16 numbers that add up to it: the leading bits, cut, and what
// that leaves, twice.  Infinities and NaNs are the first part alone.
__device__ __forceinline__ void cut3(float x, uint32_t (&part)[3]) {
  const uint32_t b = __float_as_uint(x);
  if ((b & 0x7f800000u) == 0x7f800000u) {
    part[0] = (b >> 16) | ((b & 0x7fffffu) ? 0x40u : 0u);
    part[1] = part[2] = 0;
    return;
  }
  const float r1 = x - __uint_as_float(b & 0xffff0000u);
  const uint32_t b1 = __float_as_uint(r1);
  const float r2 = r1 - __uint_as_float(b1 & 0xffff0000u);
  part[0] = b >> 16;
  part[1] = b1 >> 16;
  part[2] = __float_as_uint(r2) >> 16;
}

struct Product {
  int64_t tokens, ld_dy, ld_grad;
  int n, k;          // rows and columns of grad
  int blocks;        // checkpoint blocks of a row
  int tiles_n, tiles_k;
  int64_t share;     // tokens of a split, a multiple of kTokens
  int accumulate;
};

// A tile of 64 MN rows (along dy's columns) and 64 MK columns (along x's), a
// quarter of it to each wave.
template <int DD, int MN, int MK>
struct Tile {
  typedef typename Elem<DD>::T T;
  static constexpr int kParts = DD == RIP_FP32 ? 3 : 1;
  static constexpr int kN = 64 * MN, kK = 64 * MK;
  static constexpr int kPitchN = pitch(kN), kPitchK = pitch(kK);
  static constexpr int kYUnits = kTokens * kN / kLane / kThreads;   // of eight elements
  static constexpr int kXUnits = kTokens * kK / kCodes / kThreads;  // of sixteen codes
  static constexpr int kYRegs = DD == RIP_FP32 ? 2 : 1;
  static constexpr int kProducts = kParts * MN * MK, kOperands = kParts * MN + MK;  // of 16 tokens

  struct Shared {
    uint16_t y[kParts][kTokens * kPitchN];
    uint16_t x[kTokens * kPitchK];
  };
  struct Regs {  // a step of one thread on its way to LDS
    u32x4 y[kYUnits][kYRegs];
    u32x4 x[kXUnits];
    uint32_t e[kXUnits];
  };
  struct Offsets {  // a thread's elements in the 32 rows of a step
    uint32_t y[kYUnits], x[kXUnits], e[kXUnits];
  };

  // Columns past the last are read as the last ones' neighbours: whatever is there
  // only reaches rows and columns of grad that do not exist.
  static __device__ __forceinline__ Offsets offsets(const Product& p, int n0, int k0) {
    Offsets o;
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      const int u = threadIdx.x + i * kThreads;
      const int c = min(n0 + u % (kN / kLane) * kLane, (p.n - 1) / kLane * kLane);
      o.y[i] = (uint32_t)(u / (kN / kLane)) * (uint32_t)p.ld_dy + c;
    }
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      const int u = threadIdx.x + i * kThreads, row = u / (kK / kCodes);
      const int c = min(k0 + u % (kK / kCodes) * kCodes, p.blocks * kCkptBlock - kCodes);
      o.x[i] = (uint32_t)row * (uint32_t)(p.blocks * kCkptBlock) + c;
      o.e[i] = (uint32_t)row * (uint32_t)p.blocks + c / kCkptBlock;
    }
    return o;
  }

  // Rows t .. t+31, all of them tokens of the split, sixteen bytes from any
  // column's start inside dy.
  static __device__ __forceinline__ void load(const Product& p, const Offsets& o, const T* dy,
                                              const int8_t* codes, const uint8_t* exps, int64_t t,
                                              Regs& r) {
    const T* y = dy + t * p.ld_dy;
    const int8_t* x = codes + t * (p.blocks * kCkptBlock);
    const uint8_t* e = exps + t * p.blocks;
#pragma unroll
    for (int i = 0; i < kYUnits; ++i)
#pragma unroll
      for (int h = 0; h < kYRegs; ++h) r.y[i][h] = *(const u32x4_any*)(y + o.y[i] + 4 * h);
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      r.x[i] = *(const u32x4*)(x + o.x[i]);
      r.e[i] = e[o.e[i]];
    }
  }

  // The same with rows from `end` on and columns past the last as zeros.
  static __device__ __forceinline__ void load_checked(const Product& p, const T* dy,
                                                      const int8_t* codes, const uint8_t* exps,
                                                      int n0, int k0, int64_t t, int64_t end,
                                                      Regs& r) {
    const int width = p.blocks * kCkptBlock;
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      const int u = threadIdx.x + i * kThreads, row = u / (kN / kLane);
      const int c = n0 + u % (kN / kLane) * kLane;
      float f[kLane] = {};
      if (t + row < end && c < p.n) load_unit<DD>(dy + (t + row) * p.ld_dy, c, p.n, f);
      if constexpr (DD == RIP_FP32) {
#pragma unroll
        for (int j = 0; j < kLane; ++j) r.y[i][j / 4][j % 4] = __float_as_uint(f[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          r.y[i][0][j] = __float_as_uint(f[2 * j]) >> 16 | (__float_as_uint(f[2 * j + 1]) & 0xffff0000u);
      }
    }
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      const int u = threadIdx.x + i * kThreads, row = u / (kK / kCodes);
      const int c = min(k0 + u % (kK / kCodes) * kCodes, width - kCodes);
      r.x[i] = u32x4{0, 0, 0, 0};
      r.e[i] = 0;
      if (t + row < end) {
        r.x[i] = *(const u32x4*)(codes + (t + row) * width + c);
        r.e[i] = exps[(t + row) * p.blocks + c / kCkptBlock];
      }
    }
  }

  static __device__ __forceinline__ void store(Regs& r, Shared& sh) {
#pragma unroll
    for (int i = 0; i < kXUnits; ++i) {
      // keeps the widening of the codes here, behind the wait for their load,
      // where otherwise it would move up to the load
      asm("" : "+v"(r.x[i]), "+v"(r.e[i]));
      const int u = threadIdx.x + i * kThreads, row = u / (kK / kCodes), c = u % (kK / kCodes) * kCodes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[kLane];
        ckpt_unpack(make_uint2(r.x[i][2 * h], r.x[i][2 * h + 1]), r.e[i], x);
        u32x4 v;  // the values' low halves are zeros
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[j] = __builtin_amdgcn_perm(__float_as_uint(x[2 * j + 1]), __float_as_uint(x[2 * j]), 0x07060302u);
        *(u32x4*)&sh.x[row * kPitchK + c + h * kLane] = v;
      }
    }
#pragma unroll
    for (int i = 0; i < kYUnits; ++i) {
      const int u = threadIdx.x + i * kThreads, row = u / (kN / kLane), c = u % (kN / kLane) * kLane;
      if constexpr (DD == RIP_FP32) {
        asm("" : "+v"(r.y[i][0]), "+v"(r.y[i][1]));
        u32x4 v[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t a[3], b[3];
          cut3(__uint_as_float(r.y[i][j / 2][2 * j % 4]), a);
          cut3(__uint_as_float(r.y[i][j / 2][2 * j % 4 + 1]), b);
#pragma unroll
          for (int q = 0; q < 3; ++q) v[q][j] = a[q] | b[q] << 16;
        }
#pragma unroll
        for (int q = 0; q < 3; ++q) *(u32x4*)&sh.y[q][row * kPitchN + c] = v[q];
      } else {
        *(u32x4*)&sh.y[0][row * kPitchN + c] = r.y[i][0];
      }
    }
  }

  // Operands of sixteen tokens of a wave's part of the tile.
  struct Frags {
    bf16x8 a[kParts][MN], b[MK];
  };
  static __device__ __forceinline__ void read(const Shared& sh, int s, int wn, int wk, int lane,
                                              Frags& f) {
#pragma unroll
    for (int j = 0; j < MK; ++j) f.b[j] = read_columns<kPitchK>(sh.x, s, wk + j * 32, lane);
#pragma unroll
    for (int q = 0; q < kParts; ++q)
#pragma unroll
      for (int i = 0; i < MN; ++i) f.a[q][i] = read_columns<kPitchN>(sh.y[q], s, wn + i * 32, lane);
  }
  static __device__ __forceinline__ void multiply(const Frags& f, f32x16 (&acc)[MN][MK]) {
#pragma unroll
    for (int q = 0; q < kParts; ++q)
#pragma unroll
      for (int i = 0; i < MN; ++i)
#pragma unroll
        for (int j = 0; j < MK; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.a[q][i], f.b[j], acc[i][j], 0, 0, 0);
  }
};

// All of the workgroup's LDS accesses before come before those after; loads from
// memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Order of a step's instructions: beside each matrix instruction, which keeps its
// unit busy for 32 cycles, an equal share of the LDS reads, of the arithmetic and
// of the rest.
template <typename Tl, int I = 0>
__device__ __forceinline__ void interleave() {
  constexpr int kMfma = 2 * Tl::kProducts, kReads = 4 * Tl::kOperands;
  constexpr int kWrites = Tl::kXUnits * 2 + Tl::kYUnits * Tl::kParts;
  if constexpr (I < kMfma) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix
    constexpr int kRead = (I + 1) * kReads / kMfma - I * kReads / kMfma;
    if constexpr (kRead > 0) __builtin_amdgcn_sched_group_barrier(0x100, kRead, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // vector arithmetic
    constexpr int kWrite = (I + 1) * kWrites / kMfma - I * kWrites / kMfma;
    if constexpr (kWrite > 0) __builtin_amdgcn_sched_group_barrier(0x200, kWrite, 0);
    interleave<Tl, I + 1>();
  }
}

template <int DD, int GD, int MN, int MK, int WAVES, bool PART>
__global__ __launch_bounds__(kThreads, WAVES) void wgrad_kernel(
    Product p, const typename Elem<DD>::T* dy, const int8_t* codes, const uint8_t* exps,
    typename Elem<GD>::T* grad, float* partial) {
  typedef Tile<DD, MN, MK> Tl;
  __shared__ __align__(16) typename Tl::Shared sh[kStages];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int n0 = (int)blockIdx.x % p.tiles_n * Tl::kN, k0 = (int)blockIdx.x / p.tiles_n * Tl::kK;
  const int64_t t0 = (int64_t)blockIdx.y * p.share;
  const int64_t t1 = t0 + p.share < p.tokens ? t0 + p.share : p.tokens;
  const int wn = wave / 2 * (Tl::kN / 2), wk = wave % 2 * (Tl::kK / 2);
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
  if (whole > 0) {
    typename Tl::Regs regs[kLoads];
    typename Tl::Frags f0, f1;
    const typename Tl::Offsets off = Tl::offsets(p, n0, k0);
    auto load = [&](int s, typename Tl::Regs& r) {
      // past the last whole step its rows are loaded once more, and not used
      Tl::load(p, off, dy, codes, exps, t0 + (int64_t)min(s, whole - 1) * kTokens, r);
    };
    // Step s multiplies what lies in LDS stage s, writes step s + 2 to its stage
    // and starts the loads of step s + 4.  Half of a step's operands are read
    // before the barrier that begins it.
    auto step = [&](int s, int now) {
      Tl::read(sh[now], 16, wn, wk, lane, f1);
      Tl::store(regs[now % kLoads], sh[(now + 2) % kStages]);
      load(s + 4, regs[now % kLoads]);
      Tl::multiply(f0, acc);
      Tl::read(sh[(now + 1) % kStages], 0, wn, wk, lane, f0);
      Tl::multiply(f1, acc);
      interleave<Tl>();
      lds_barrier();
    };
    load(0, regs[0]);
    load(1, regs[1]);
    Tl::store(regs[0], sh[0]);
    load(2, regs[0]);
    Tl::store(regs[1], sh[1]);
    load(3, regs[1]);
    lds_barrier();
    Tl::read(sh[0], 0, wn, wk, lane, f0);
    for (int s = 0;;) {
      step(s, 0);
      if (++s == whole) break;
      step(s, 1);
      if (++s == whole) break;
      step(s, 2);
      if (++s == whole) break;
      step(s, 3);
      if (++s == whole) break;
    }
  }
  for (int s = whole; s < steps; ++s) {
    typename Tl::Regs r;
    typename Tl::Frags f;
    Tl::load_checked(p, dy, codes, exps, n0, k0, t0 + (int64_t)s * kTokens, t1, r);
    Tl::store(r, sh[0]);
    lds_barrier();
    Tl::read(sh[0], 0, wn, wk, lane, f);
    Tl::multiply(f, acc);
    Tl::read(sh[0], 16, wn, wk, lane, f);
    Tl::multiply(f, acc);
    lds_barrier();
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
          partial[((int64_t)blockIdx.y * p.n + row) * p.k + col] = acc[i][j][r];
        } else {
          typename Elem<GD>::T* g = grad + (int64_t)row * p.ld_grad + col;
          Elem<GD>::store(g, p.accumulate ? Elem<GD>::load(g) + acc[i][j][r] : acc[i][j][r]);
        }
      }
}

// The splits' parts, added in order.
template <int GD>
__global__ __launch_bounds__(kThreads) void reduce_kernel(Product p, const float* partial,
                                                          int splits,
                                                          typename Elem<GD>::T* grad) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, all = (int64_t)p.n * p.k;
  if (i >= all) return;
  float sum = partial[i];
  for (int s = 1; s < splits; ++s) sum += partial[s * all + i];
  typename Elem<GD>::T* g = grad + i / p.k * p.ld_grad + i % p.k;
  Elem<GD>::store(g, p.accumulate ? Elem<GD>::load(g) + sum : sum);
}

struct Plan {
  bool large;
  int tiles_n, tiles_k, splits;
  int64_t share;
};
Plan make_plan(int32_t dy_dtype, int64_t tokens, int64_t n, int64_t k) {
  Plan best{};
  double least = 1e30;
  for (int large = 0; large < (dy_dtype == RIP_BF16 ? 2 : 1); ++large) {
    const int tn = large ? 192 : 128, tk = large ? 256 : 128;
    const int64_t tiles_n = ceil_div(n, tn), tiles_k = ceil_div(k, tk), tiles = tiles_n * tiles_k;
    const int64_t steps = ceil_div(tokens, kTokens);
    const int slots = large || dy_dtype == RIP_FP32 ? 256 : 512;
    const double step = large ? 0.5 : 0.4;
    for (int64_t splits = 1; splits <= 64 && (splits == 1 || splits * 4 <= steps); ++splits) {
      const int64_t per = ceil_div(steps, splits);
      double us = (double)ceil_div(tiles * splits, slots) * per * step;
      if (splits > 1) us += 4.0 + (double)splits * n * k * 8 / 4e6;
      if (us < least) {
        least = us;
        best = Plan{large != 0, (int)tiles_n, (int)tiles_k, (int)splits, per * kTokens};
      }
    }
  }
  best.splits = tokens > 0 ? (int)ceil_div(tokens, best.share) : 1;
  return best;
}

template <int DD, int GD, int MN, int MK, int WAVES>
const void* kernel_of(bool part) {
  return part ? (const void*)wgrad_kernel<DD, GD, MN, MK, WAVES, true>
              : (const void*)wgrad_kernel<DD, GD, MN, MK, WAVES, false>;
}

template <int DD, int GD>
int32_t run(Product& p, const Plan& plan, const void* dy, const int8_t* codes, const uint8_t* exps,
            void* grad, float* partial, void* stream) {
  void* args[] = {&p, &dy, &codes, &exps, &grad, &partial};
  const void* fn = kernel_of<DD, GD, 2, 2, DD == RIP_FP32 ? 1 : 2>(plan.splits > 1);
  if constexpr (DD == RIP_BF16)
    if (plan.large) fn = kernel_of<DD, GD, 3, 4, 1>(plan.splits > 1);
  int32_t rc = launch(fn, dim3((uint32_t)(plan.tiles_n * plan.tiles_k), (uint32_t)plan.splits),
                      dim3(kThreads), args, 0, stream, "rip_ckpt_wgrad");
  if (rc || plan.splits == 1) return rc;
  int splits = plan.splits;
  void* args2[] = {&p, &partial, &splits, &grad};
  return launch((const void*)reduce_kernel<GD>,
                dim3((uint32_t)ceil_div((int64_t)p.n * p.k, kThreads)), dim3(kThreads), args2, 0,
                stream, "rip_ckpt_wgrad: reduce");
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
  const Plan plan = make_plan(dy_dtype, rows, out_features, in_features);
  return plan.splits > 1 ? plan.splits * out_features * in_features * 4 : 0;
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
  const int64_t need = rip_ckpt_wgrad_workspace(dy_dtype, rows, out_features, in_features);
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
  const Plan plan = make_plan(dy_dtype, rows, out_features, in_features);
  Product p{rows,
            ld_dy,
            ld_grad,
            (int)out_features,
            (int)in_features,
            (int)blocks,
            plan.tiles_n,
            plan.tiles_k,
            plan.share,
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
