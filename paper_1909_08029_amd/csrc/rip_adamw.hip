// AdamW update of many tensors of many replicas in one launch (gfx950), with
// moments in fp32 or in 8 bits:
//
//   g = s * grad;  m = b1 m + (1 - b1) g;  v = b2 v + ((1 - b2) g) g
//   w = w * decay - (rate * m) / (sqrt(v) * root + eps)
//
// One pass over memory: 3 a + 16 bytes an element with moments in fp32 (a: bytes of
// the storage type), 3 a + 4.1 with 8-bit ones.  A lane takes eight consecutive
// elements; the 32 elements that share an exponent are four lanes', which find their
// largest magnitude with two exchanges.
//
// Moments in 8 bits are rounded up or down at random, so that their mean is kept:
// rounded to nearest, a second moment that changes by 0.1% a step would never leave
// a code whose neighbours are 3 to 6% away.  The first moment is a checkpoint
// (rip_ckpt_format.h).  The second needs range rather than steps, as it is a divisor:
// codes of four exponent and four significand bits span 2^19 of the block's largest
// value.  A positive value never becomes zero.
//
// The 16 random bits of a rounding come from a 32-bit finalizer over the element's
// index: the first moment takes the low half, the second the high one.

#include <new>
#include <vector>

#include "rip_ckpt_format.h"
#include "rip_splitmix.h"

namespace rip {
namespace {
// One segment of one replica.
struct Row {
  uint64_t param, grad, m, v, m_exps, v_exps;
  int64_t numel, place;  // place: first element in the packed moments of a replica
};
}  // namespace
}  // namespace rip

struct rip_adamw_state {
  int32_t n = 0, n_seg = 0, dtype = 0, format = 0, device = 0;
  int64_t tiles = 0;   // of one replica
  int64_t packed = 0;  // elements of a replica's segments, each in whole blocks
  void* dmem = nullptr;
  std::vector<rip::Row> host;   // [S][N]
  const void* rows = nullptr;   // device copy of it
  const void* table = nullptr;  // device [tiles] TileAt
};

namespace rip {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads * kLane;  // elements of a workgroup

struct TileAt {
  uint32_t segment, tile;  // tile: of the segment
};

struct Update {
  const Row* rows;
  const TileAt* table;
  int32_t n_rep;
  float b1, c1, b2, c2, eps;      // c = 1 - b
  rip_adamw_scalars s;
  const rip_adamw_scalars* live;  // device; replaces s unless NULL
  uint32_t active[RIP_MAX_REPLICAS / 4];  // a byte each, in words that scalar loads reach
};

// Second moment in 8 bits: code 16 x + y stands for y steps (x = 0) or
// (16 + y) 2^(x - 1), a step being 2^(exp - 127); the largest is 31 * 2^14.
// Shifted to a float's place a code is its value times 2^-130 (x = 0 a subnormal).
// `nan`: bits of a NaN for a block that stands for it, else 0.
__device__ __forceinline__ float second_value(uint32_t codes, int j, int exp, uint32_t nan) {
  const uint32_t at = j < 3 ? codes << (19 - 8 * j) : codes >> 5;
  return __builtin_amdgcn_ldexpf(__uint_as_float((at & 0xffu << 19) | nan), exp + 3);
}
__device__ __forceinline__ uint32_t nan_of(int exp) { return exp == kCkptNan ? 0x7fc00000u : 0; }

// The square root rounded to nearest, for 0 and from kRootLeast on, where the residuals
// below are exact.  The hardware's is within one step; the root lies above the middle
// of y and its neighbour z if x > y z (Tuckerman's test; Agarwal, Cooley, Gustavson,
// Shearer, Slishman and Tuckerman 1986).  (Smaller numbers have to be scaled first, which
// costs as much again: seven of the 88 instructions that an element would take.)
constexpr float kRootLeast = 0x1p-96f;
__device__ __forceinline__ float root_of(float x) {
  const float y = __builtin_amdgcn_sqrtf(x);
  const float down = __uint_as_float(__float_as_uint(y) - 1), up = __uint_as_float(__float_as_uint(y) + 1);
  const float z = __builtin_fmaf(-down, y, x) <= 0.0f ? down : y;
  return __builtin_fmaf(-up, y, x) > 0.0f ? up : z;
}
// Exponent byte of a block whose largest value has the bits `top` (>= 0).
__device__ __forceinline__ uint32_t second_exponent(uint32_t top) {
  // v = f * 2^k, 1 <= f < 2: the largest code reaches 1.9375 * 2^18 steps
  const int e = (int)(top >> 23) - 18 + ((top & 0x7fffffu) > 0x780000u ? 1 : 0);
  return top >= 0x7f800000u ? kCkptNan : (uint32_t)max(1, e);
}
// Code (its low byte) of x >= 0 with 1 / step = inv, rounded up with the probability
// r / 2^16 of a remainder.
__device__ __forceinline__ uint32_t second_code(float x, float inv, uint32_t r) {
  const float t = x * inv;
  const uint32_t low = (uint32_t)__builtin_fmaf((float)r, 0x1p-16f, t);
  const uint32_t high = min((__float_as_uint(t) + (r << 3)) >> 19, (130u << 4) + 255) - (130u << 4);
  return max(t < 16.0f ? low : high, min(__float_as_uint(x), 1u));
}
// The low bytes of four numbers.
__device__ __forceinline__ uint32_t pack4(const uint32_t (&x)[kLane], int j) {
  const uint32_t a = __builtin_amdgcn_perm(x[j + 1], x[j], 0x0c0c0400u);
  const uint32_t b = __builtin_amdgcn_perm(x[j + 3], x[j + 2], 0x0c0c0400u);
  return __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// Finalizer of MurmurHash3 (Appleby), a bijection of 32 bits.
__device__ __forceinline__ uint32_t scramble(uint32_t x) {
  x ^= x >> 16;
  x *= 0x85ebca6bu;
  x ^= x >> 13;
  x *= 0xc2b2ae35u;
  return x ^ (x >> 16);
}

// Largest magnitude (bits) of the 32 elements that four neighbouring lanes hold.
__device__ __forceinline__ uint32_t block_max(const float (&x)[kLane]) {
  static_assert(kCkptBlock == 4 * kLane, "a block is a quad of lanes");
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < kLane; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));  // lane ^ 1
  return max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, true)); // lane ^ 2
}
__device__ __forceinline__ float inverse_step(uint32_t e) {
  return e == kCkptNan ? 0.0f : __uint_as_float((254 - e) << 23);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight elements from c on: weights, gradients and moments as fp32.
struct Unit {
  float w[kLane], g[kLane], m[kLane], v[kLane];
};
template <int DT, bool FULL>
__device__ __forceinline__ void get(uint64_t p, int64_t at, int c, int width, float (&f)[kLane]) {
  const typename Elem<DT>::T* from = (const typename Elem<DT>::T*)p + at;
  if (FULL)
    Elem<DT>::template load8<true>(from + c, f);
  else
    load_unit<DT>(from, c, width, f);
}
template <int DT, bool FULL>
__device__ __forceinline__ void put(uint64_t p, int64_t at, int c, int width, const float (&f)[kLane]) {
  typename Elem<DT>::T* to = (typename Elem<DT>::T*)p + at;
  if (FULL)
    Elem<DT>::store8(to + c, f);
  else
    store_unit<DT>(to, c, width, f);
}
template <int DT, int FORMAT, bool FULL>
__device__ __forceinline__ void load(const Row& row, int64_t at, int width, int c, Unit& u) {
  get<DT, FULL>(row.param, at, c, width, u.w);
  get<DT, FULL>(row.grad, at, c, width, u.g);
  if constexpr (FORMAT == RIP_STATE_FP32) {
    get<RIP_FP32, FULL>(row.m, at, c, width, u.m);
    get<RIP_FP32, FULL>(row.v, at, c, width, u.v);
  } else {
    const u32x2 mc = *(const u32x2*)((const int8_t*)row.m + at + c);
    const u32x2 vc = *(const u32x2*)((const uint8_t*)row.v + at + c);
    const uint32_t codes[2] = {mc[0], mc[1]};
    ckpt_unpack<kLane>(codes, ((const uint8_t*)row.m_exps + at / kCkptBlock)[c / kCkptBlock], u.m);
    const int exp = ((const uint8_t*)row.v_exps + at / kCkptBlock)[c / kCkptBlock];
#pragma unroll
    for (int j = 0; j < kLane; ++j) u.v[j] = second_value(vc[j / 4], j % 4, exp, nan_of(exp));
  }
}

// The weights from the new moments.
template <bool PLAIN>
__device__ __forceinline__ void step(const Update& u, const rip_adamw_scalars& s, Unit& x) {
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    const float root = PLAIN ? root_of(x.v[j]) : __builtin_sqrtf(x.v[j]);
    x.w[j] = x.w[j] * s.decay - (s.rate * x.m[j]) / (root * s.root + u.eps);
  }
}

// Eight elements of a tile; FULL: no segment ends in it.
template <int DT, int FORMAT, bool FULL>
__device__ __forceinline__ void update(const Update& u, const rip_adamw_scalars& s, const Row& row, int rep,
                                       uint32_t segment, int64_t at, int width) {
  const int c = threadIdx.x * kLane;
  if (!FULL && c >= (FORMAT == RIP_STATE_FP32 ? width : (width + kCkptBlock - 1) / kCkptBlock * kCkptBlock))
    return;
  Unit x;
  load<DT, FORMAT, FULL>(row, at, width, c, x);
#pragma unroll
  for (int j = 0; j < kLane; ++j) {
    const float g = s.grad_scale * x.g[j];
    x.m[j] = u.b1 * x.m[j] + u.c1 * g;
    x.v[j] = u.b2 * x.v[j] + (u.c2 * g) * g;
  }
  float least = x.v[0];
#pragma unroll
  for (int j = 1; j < kLane; ++j) least = fminf(least, x.v[j]);
  if (FORMAT == RIP_STATE_8BIT && __all(least >= kRootLeast))
    step<true>(u, s, x);
  else
    step<false>(u, s, x);
  put<DT, FULL>(row.param, at, c, width, x.w);
  if constexpr (FORMAT == RIP_STATE_FP32) {
    put<RIP_FP32, FULL>(row.m, at, c, width, x.m);
    put<RIP_FP32, FULL>(row.v, at, c, width, x.v);
  } else {
    const uint64_t key = fold(fold(s.key[0] | (uint64_t)s.key[1] << 32, (uint64_t)rep), segment);
    const uint32_t seed = (uint32_t)key + (uint32_t)(at >> 32) * 0x9E3779B9u;  // (a tile's)
    const uint32_t i = (uint32_t)at + c;
    const uint32_t me = ckpt_exponent(block_max(x.m)), ve = second_exponent(block_max(x.v));
    const float mi = inverse_step(me), vi = inverse_step(ve);
    uint32_t ms[kLane], vs[kLane];
#pragma unroll
    for (int j = 0; j < kLane; ++j) {
      const uint32_t h = scramble((i + j) ^ seed);
      const float q = floorf(__builtin_fmaf((float)(h & 0xffff), 0x1p-16f, x.m[j] * mi));
      ms[j] = (uint32_t)(int)__builtin_amdgcn_fmed3f(q, -127.0f, 127.0f);
      vs[j] = second_code(x.v[j], vi, h >> 16);
    }
    u32x2 mc = {pack4(ms, 0), pack4(ms, 4)}, vc = {pack4(vs, 0), pack4(vs, 4)};
    if (me == kCkptNan) mc = u32x2{0, 0};
    if (ve == kCkptNan) vc = u32x2{0, 0};
    *(u32x2*)((int8_t*)row.m + at + c) = mc;
    *(u32x2*)((uint8_t*)row.v + at + c) = vc;
    if (threadIdx.x % (kCkptBlock / kLane) == 0) {
      ((uint8_t*)row.m_exps + at / kCkptBlock)[c / kCkptBlock] = (uint8_t)me;
      ((uint8_t*)row.v_exps + at / kCkptBlock)[c / kCkptBlock] = (uint8_t)ve;
    }
  }
}

// A tile of one replica's segment.  Moments in fp32: bound by memory (5.4 TB/s).  In 8
// bits: by instructions, 80 an element, half of them the root and the quotient to the
// last bit, a third the codes (two replicas of 400 M: 1702 us, 4.8 TB/s; 2021 with roots
// scaled always, with branches around each load, and keys made in every lane).
template <int DT, int FORMAT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(Update u) {
  const int rep = u.active[blockIdx.y / 4] >> (8 * (blockIdx.y % 4)) & 0xff;
  const TileAt tile = u.table[blockIdx.x];
  const Row row = u.rows[(int64_t)tile.segment * u.n_rep + rep];
  rip_adamw_scalars s = u.s;
  if (u.live) {  // (word by word: one pointer to both kinds of memory would make them a lane's)
    s.decay = u.live->decay, s.rate = u.live->rate, s.root = u.live->root;
    s.grad_scale = u.live->grad_scale, s.key[0] = u.live->key[0], s.key[1] = u.live->key[1];
  }
  const int64_t at = (int64_t)tile.tile * kTile, left = row.numel - at;
  const int width = left < kTile ? (int)left : kTile;
  // Whole tiles of 8-bit moments load without branches.  With moments in fp32 that is
  // slower: more loads in flight than memory serves well (541 us for four replicas of
  // 25.6 M, 527 with one array's loads after another's).
  if (FORMAT == RIP_STATE_8BIT && width == kTile)
    update<DT, FORMAT, true>(u, s, row, rep, tile.segment, at, width);
  else
    update<DT, FORMAT, false>(u, s, row, rep, tile.segment, at, width);
}

struct Moments {
  const Row* rows;
  const TileAt* table;
  int32_t n_rep;
  int64_t packed;
};

// The values of 8-bit moments, whole blocks of a segment after another.
template <int DT>
__global__ __launch_bounds__(kThreads) void moments_kernel(Moments p, typename Elem<DT>::T* m,
                                                           typename Elem<DT>::T* v) {
  const TileAt tile = p.table[blockIdx.x];
  const Row row = p.rows[(int64_t)tile.segment * p.n_rep + blockIdx.y];
  const int64_t at = (int64_t)tile.tile * kTile, i = at + threadIdx.x * kLane;
  if (i >= (row.numel + kCkptBlock - 1) / kCkptBlock * kCkptBlock) return;
  const u32x2 mc = *(const u32x2*)((const int8_t*)row.m + i);
  const u32x2 vc = *(const u32x2*)((const uint8_t*)row.v + i);
  const uint32_t codes[2] = {mc[0], mc[1]};
  float x[kLane];
  ckpt_unpack<kLane>(codes, ((const uint8_t*)row.m_exps)[i / kCkptBlock], x);
  const int64_t to = blockIdx.y * p.packed + row.place + i;
  Elem<DT>::store8(m + to, x);
  const int exp = ((const uint8_t*)row.v_exps)[i / kCkptBlock];
#pragma unroll
  for (int j = 0; j < kLane; ++j) x[j] = second_value(vc[j / 4], j % 4, exp, nan_of(exp));
  Elem<DT>::store8(v + to, x);
}

int32_t check_device(const rip_adamw_state* s) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail(RIP_E_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  if (dev != s->device)
    return fail(RIP_E_INVAL, "current device %d differs from the handle's device %d", dev, s->device);
  return RIP_OK;
}

int32_t check_aligned(void* const* p, const char* what, int32_t n, int32_t S, const int64_t* numel,
                      int bytes) {
  for (int32_t i = 0; i < n * S; ++i)
    if (numel[i % S] && reinterpret_cast<uintptr_t>(p[i]) % bytes)
      return fail(RIP_E_ALIGN, "%s[%d*S+%d] = %p is not %d-byte aligned", what, i / S, i % S, p[i],
                  bytes);
  return RIP_OK;
}

int32_t create(int32_t n, int32_t S, int32_t dtype, const int64_t* numel, void* const* param,
               void* const* grad, int32_t format, void* const* m, void* const* v,
               void* const* m_exps, void* const* v_exps, rip_adamw_state** out) {
  const bool eight = format == RIP_STATE_8BIT;
  if (!known_dtype(dtype)) return fail(RIP_E_UNSUPPORTED, "unknown dtype %d", dtype);
  if (!eight && format != RIP_STATE_FP32)
    return fail(RIP_E_UNSUPPORTED, "unknown state format %d", format);
  if (n < 1) return fail(RIP_E_INVAL, "n_replicas %d < 1", n);
  if (n > RIP_MAX_REPLICAS)
    return fail(RIP_E_UNSUPPORTED, "n_replicas %d > %d", n, RIP_MAX_REPLICAS);
  if (S < 1 || !numel || !param || !grad || !m || !v || (eight && (!m_exps || !v_exps)))
    return fail(RIP_E_INVAL, "need n_segments >= 1, seg_numel and every buffer of the format");
  std::vector<int64_t> blocks(S), codes(S);
  std::vector<TileAt> table;
  int64_t packed = 0, tiles = 0;
  constexpr int64_t kMostTiles = ((int64_t)1 << 32) / kThreads - 1;  // of a 32-bit grid
  for (int32_t s = 0; s < S; ++s) {
    if (numel[s] < 0) return fail(RIP_E_INVAL, "seg_numel[%d] < 0", s);
    if (numel[s] > kMostTiles * kTile || (tiles += ceil_div(numel[s], kTile)) > kMostTiles)
      return fail(RIP_E_UNSUPPORTED, "more than 2^24 tiles of %d elements in one replica", kTile);
    blocks[s] = ceil_div(numel[s], kCkptBlock);
    codes[s] = blocks[s] * kCkptBlock;
  }
  int32_t rc;
  const BufferKind kinds[] = {{param, "param", true, numel, elem_bytes(dtype)},
                              {grad, "grad", false, numel, elem_bytes(dtype)},
                              {m, "m", true, eight ? codes.data() : numel, eight ? 1 : 4},
                              {v, "v", true, eight ? codes.data() : numel, eight ? 1 : 4},
                              {eight ? m_exps : nullptr, "m_exps", true, blocks.data(), 1},
                              {eight ? v_exps : nullptr, "v_exps", true, blocks.data(), 1}};
  for (const BufferKind& k : kinds) {
    const bool coded = eight && (k.p == m || k.p == v);
    if (k.p && ((rc = check_nonnull(k.p, k.what, n, S, k.numel)) ||
                (rc = check_aligned(k.p, k.what, n, S, k.numel, coded ? 16 : k.esize))))
      return rc;
  }
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return fail(RIP_E_HIP, "hipGetDevice: %s", hipGetErrorString(e));
  if ((rc = check_buffers(kinds, 6, n, S, device))) return rc;

  std::vector<Row> rows((size_t)S * n);
  table.reserve(tiles);
  auto address = [](void* const* p, size_t i) { return p ? reinterpret_cast<uint64_t>(p[i]) : 0; };
  for (int32_t s = 0; s < S; ++s) {
    for (int32_t r = 0; r < n; ++r) {
      const size_t i = (size_t)r * S + s;
      rows[(size_t)s * n + r] = {address(param, i),  address(grad, i),        address(m, i),
                                 address(v, i),      address(kinds[4].p, i),  address(kinds[5].p, i),
                                 numel[s],           packed};
    }
    packed += codes[s];
    for (int64_t t = 0; t < ceil_div(numel[s], kTile); ++t)
      table.push_back({(uint32_t)s, (uint32_t)t});
  }
  const size_t row_bytes = rows.size() * sizeof(Row), table_bytes = table.size() * sizeof(TileAt);
  rip_adamw_state* h = new rip_adamw_state();
  h->host.swap(rows);
  e = hipMalloc(&h->dmem, row_bytes + table_bytes);
  if (e == hipSuccess) e = hipMemcpy(h->dmem, h->host.data(), row_bytes, hipMemcpyHostToDevice);
  if (e == hipSuccess && table_bytes)
    e = hipMemcpy((char*)h->dmem + row_bytes, table.data(), table_bytes, hipMemcpyHostToDevice);
  if (e != hipSuccess) {
    rip_adamw_state_destroy(h);
    return fail(e == hipErrorOutOfMemory ? RIP_E_NOMEM : RIP_E_HIP, "rip_adamw_state_create: %s",
                hipGetErrorString(e));
  }
  h->n = n, h->n_seg = S, h->dtype = dtype, h->format = format, h->device = device;
  h->tiles = tiles, h->packed = packed;
  h->rows = h->dmem;
  h->table = (char*)h->dmem + row_bytes;
  *out = h;
  return RIP_OK;
}

// 0 <= x < 1
bool fraction(double x) { return x >= 0.0 && x < 1.0; }

int32_t scalars_of(const rip_adamw* a, int64_t step, rip_adamw_scalars* out) {
  if (!a || !out) return fail(RIP_E_INVAL, "rip_adamw: NULL argument");
  if (step < 1) return fail(RIP_E_INVAL, "rip_adamw: step %lld < 1", (long long)step);
  if (!fraction(a->beta1) || !fraction(a->beta2) || !((float)a->eps > 0.0f) || !__builtin_isfinite(a->eps) ||
      !__builtin_isfinite(a->lr) || !__builtin_isfinite(a->weight_decay) ||
      !__builtin_isfinite(a->grad_scale))
    return fail(RIP_E_INVAL, "rip_adamw: lr %g, betas %g and %g, eps %g, weight decay %g, grad scale %g",
                a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, a->grad_scale);
  const uint64_t key = fold(a->seed, (uint64_t)step);
  out->decay = (float)(1.0 - a->lr * a->weight_decay);
  out->rate = (float)(a->lr / (1.0 - __builtin_pow(a->beta1, (double)step)));
  out->root = (float)(1.0 / __builtin_sqrt(1.0 - __builtin_pow(a->beta2, (double)step)));
  out->grad_scale = (float)a->grad_scale;
  out->key[0] = (uint32_t)key;
  out->key[1] = (uint32_t)(key >> 32);
  return RIP_OK;
}

}  // namespace
}  // namespace rip

using namespace rip;

extern "C" int32_t rip_adamw_state_create(int32_t n_replicas, int32_t n_segments, int32_t dtype,
                                          const int64_t* seg_numel, void* const* param,
                                          void* const* grad, int32_t format, void* const* m,
                                          void* const* v, void* const* m_exps, void* const* v_exps,
                                          rip_adamw_state** out) {
  clear_error();
  if (!out) return fail(RIP_E_INVAL, "rip_adamw_state_create: out is NULL");
  *out = nullptr;
  try {
    return create(n_replicas, n_segments, dtype, seg_numel, param, grad, format, m, v, m_exps,
                  v_exps, out);
  } catch (const std::bad_alloc&) {
    return fail(RIP_E_NOMEM, "rip_adamw_state_create: out of host memory");
  }
}

extern "C" void rip_adamw_state_destroy(rip_adamw_state* s) {
  if (!s) return;
  if (s->dmem) (void)hipFree(s->dmem);
  delete s;
}

extern "C" int32_t rip_adamw_scalars_at(const rip_adamw* cfg, int64_t step, rip_adamw_scalars* out) {
  clear_error();
  return scalars_of(cfg, step, out);
}

extern "C" int32_t rip_adamw_step(const rip_adamw_state* s, const int32_t* active, int32_t n_active,
                                  const rip_adamw* cfg, int64_t step,
                                  const rip_adamw_scalars* scalars, void* stream) {
  clear_error();
  if (!s || !cfg) return fail(RIP_E_INVAL, "rip_adamw_step: NULL argument");
  if (n_active < 0 || n_active > s->n || (n_active && !active))
    return fail(RIP_E_INVAL, "rip_adamw_step: %d active workers of %d", n_active, s->n);
  Update u{};
  int32_t rc = scalars_of(cfg, step, &u.s);
  if (rc) return rc;
  if (reinterpret_cast<uintptr_t>(scalars) % 4)
    return fail(RIP_E_ALIGN, "rip_adamw_step: scalars = %p is not 4-byte aligned", (const void*)scalars);
  uint8_t seen[RIP_MAX_REPLICAS] = {};
  for (int32_t i = 0; i < n_active; ++i) {
    if (active[i] < 0 || active[i] >= s->n)
      return fail(RIP_E_INVAL, "active id %d out of range", active[i]);
    if (seen[active[i]]) return fail(RIP_E_INVAL, "active id %d listed twice", active[i]);
    seen[active[i]] = 1;
    u.active[i / 4] |= (uint32_t)active[i] << (8 * (i % 4));
  }
  if (!n_active || !s->tiles) return RIP_OK;
  if ((rc = check_device(s))) return rc;
  u.rows = (const Row*)s->rows;
  u.table = (const TileAt*)s->table;
  u.n_rep = s->n;
  u.b1 = (float)cfg->beta1, u.c1 = (float)(1.0 - cfg->beta1);
  u.b2 = (float)cfg->beta2, u.c2 = (float)(1.0 - cfg->beta2);
  u.eps = (float)cfg->eps;
  u.live = scalars;
  const bool eight = s->format == RIP_STATE_8BIT;
  const void* fn = s->dtype == RIP_BF16
                       ? (eight ? (const void*)adamw_kernel<RIP_BF16, RIP_STATE_8BIT>
                                : (const void*)adamw_kernel<RIP_BF16, RIP_STATE_FP32>)
                       : (eight ? (const void*)adamw_kernel<RIP_FP32, RIP_STATE_8BIT>
                                : (const void*)adamw_kernel<RIP_FP32, RIP_STATE_FP32>);
  void* args[] = {&u};
  return launch(fn, dim3((uint32_t)s->tiles, (uint32_t)n_active), dim3(kThreads), args, 0, stream,
                "rip_adamw_step");
}

extern "C" int64_t rip_adamw_packed(const rip_adamw_state* s) { return s ? s->packed : 0; }

extern "C" int32_t rip_adamw_moments(const rip_adamw_state* s, int32_t dtype, void* m, void* v,
                                     void* stream) {
  clear_error();
  if (!s) return fail(RIP_E_INVAL, "rip_adamw_moments: state is NULL");
  if (!known_dtype(dtype)) return fail(RIP_E_UNSUPPORTED, "unknown dtype %d", dtype);
  if (s->format != RIP_STATE_8BIT)
    return fail(RIP_E_UNSUPPORTED, "rip_adamw_moments: the moments are held as values");
  if (!s->tiles) return RIP_OK;
  if (!m || !v) return fail(RIP_E_INVAL, "rip_adamw_moments: m or v is NULL");
  const int bytes = elem_bytes(dtype);
  if (reinterpret_cast<uintptr_t>(m) % bytes || reinterpret_cast<uintptr_t>(v) % bytes)
    return fail(RIP_E_ALIGN, "rip_adamw_moments: m or v is not aligned to its elements");
  const int64_t all = s->n * s->packed * bytes;
  if (overlap(m, all, v, all)) return fail(RIP_E_OVERLAP, "rip_adamw_moments: m overlaps v");
  for (const Row& row : s->host) {
    const int64_t blocks = ceil_div(row.numel, kCkptBlock), a = row.numel * elem_bytes(s->dtype);
    const struct {
      uint64_t p;
      int64_t bytes;
    } held[] = {{row.param, a}, {row.grad, a}, {row.m, blocks * kCkptBlock},
                {row.v, blocks * kCkptBlock}, {row.m_exps, blocks}, {row.v_exps, blocks}};
    for (const auto& h : held)
      if (overlap(m, all, (const void*)h.p, h.bytes) || overlap(v, all, (const void*)h.p, h.bytes))
        return fail(RIP_E_OVERLAP, "rip_adamw_moments: m or v overlaps a registered buffer");
  }
  int32_t rc = check_device(s);
  if (rc) return rc;
  Moments p{(const Row*)s->rows, (const TileAt*)s->table, s->n, s->packed};
  void* args[] = {&p, &m, &v};
  return launch(dtype == RIP_BF16 ? (const void*)moments_kernel<RIP_BF16>
                                  : (const void*)moments_kernel<RIP_FP32>,
                dim3((uint32_t)s->tiles, (uint32_t)s->n), dim3(kThreads), args, 0, stream,
                "rip_adamw_moments");
}
