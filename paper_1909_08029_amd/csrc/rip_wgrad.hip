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
// A workgroup computes a 128 x 128 tile of grad and goes over its tokens in
// steps of 32: rows of dy and of codes come in as they lie in memory, the codes
// widen to bf16 on the way into LDS, and the transposing LDS reads hand each
// lane eight tokens of its column.  Few tiles are split over the tokens; the
// parts go to the workspace and a second launch adds them in order.

#include "rip_ckpt_format.h"

namespace rip {
namespace {

constexpr int kTile = 128;   // rows and columns of grad in a workgroup's tile
constexpr int kTokens = 32;  // tokens of a step
constexpr int kThreads = 256;
constexpr int kPitch = kTile + 16;  // elements between LDS rows: the four rows that
                                    // a group of 16 lanes reads lie in different banks

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Eight tokens (t .. t+7 by the lane's half of the wave) of column n + lane % 32.
__device__ __forceinline__ bf16x8 read_columns(const uint16_t* tile, int t, int n, int lane) {
  const int group = lane / 16, in = lane % 16;
  const uint16_t* p =
      tile + (t + (group / 2) * 8 + in / 4) * kPitch + n + (group % 2) * 16 + (in % 4) * 4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * kPitch));
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
  int tiles_k;       // tiles along k
  int64_t share;     // tokens of a split, a multiple of kTokens
  int accumulate;
};

template <int DD, int GD, bool PART>
__global__ __launch_bounds__(kThreads) void wgrad_kernel(Product p, const typename Elem<DD>::T* dy,
                                                         const int8_t* codes, const uint8_t* exps,
                                                         typename Elem<GD>::T* grad,
                                                         float* partial) {
  constexpr int kParts = DD == RIP_FP32 ? 3 : 1;
  __shared__ __align__(16) uint16_t ys[kParts][kTokens * kPitch];
  __shared__ __align__(16) uint16_t xs[kTokens * kPitch];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int n0 = blockIdx.x / p.tiles_k * kTile, k0 = blockIdx.x % p.tiles_k * kTile;
  const int64_t t0 = (int64_t)blockIdx.y * p.share;
  const int64_t t1 = t0 + p.share < p.tokens ? t0 + p.share : p.tokens;
  const int wn = wave / 2 * 64, wk = wave % 2 * 64;
  f32x16 acc[2][2] = {};
  for (int64_t t = t0; t < t1; t += kTokens) {
#pragma unroll
    for (int i = 0; i < kTokens * kTile / kLane / kThreads; ++i) {
      const int u = tid + i * kThreads, row = u / (kTile / kLane), c = u % (kTile / kLane) * kLane;
      const int64_t tt = t + row;
      float f[kLane] = {};
      if (tt < t1 && n0 + c < p.n) load_unit<DD>(dy + tt * p.ld_dy, n0 + c, p.n, f);
      uint32_t part[kParts][kLane];
#pragma unroll
      for (int j = 0; j < kLane; ++j) {
        if constexpr (kParts == 3) {
          uint32_t q[3];
          cut3(f[j], q);
          part[0][j] = q[0], part[1][j] = q[1], part[2][j] = q[2];
        } else {
          part[0][j] = __float_as_uint(f[j]) >> 16;
        }
      }
#pragma unroll
      for (int q = 0; q < kParts; ++q) {
        u32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = part[q][2 * j] | part[q][2 * j + 1] << 16;
        *(u32x4*)&ys[q][row * kPitch + c] = v;
      }
      // columns past the last block, and tokens past the last, are zeros
      float x[kLane] = {};
      const int block = (k0 + c) / kCkptBlock;
      if (tt < t1 && block < p.blocks) {
        const uint2 code = *(const uint2*)(codes + tt * p.blocks * kCkptBlock + k0 + c);
        ckpt_unpack(code, exps[tt * p.blocks + block], x);
      }
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = __float_as_uint(x[2 * j]) >> 16 | (__float_as_uint(x[2 * j + 1]) & 0xffff0000u);
      *(u32x4*)&xs[row * kPitch + c] = v;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kTokens; s += 16) {
      bf16x8 b[2];
      for (int j = 0; j < 2; ++j) b[j] = read_columns(xs, s, wk + j * 32, lane);
#pragma unroll
      for (int q = 0; q < kParts; ++q)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bf16x8 a = read_columns(ys[q], s, wn + i * 32, lane);
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b[j], acc[i][j], 0, 0, 0);
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
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
  int64_t tiles;
  int splits;
  int64_t share;
};
Plan make_plan(int64_t tokens, int64_t n, int64_t k) {
  Plan p{};
  p.tiles = ceil_div(n, kTile) * ceil_div(k, kTile);
  int64_t splits = 512 / p.tiles;
  const int64_t most = ceil_div(tokens, 8 * kTokens);
  splits = splits > most ? most : splits;
  if (splits < 1) splits = 1;
  p.share = ceil_div(ceil_div(tokens, splits), kTokens) * kTokens;
  p.splits = tokens > 0 ? (int)ceil_div(tokens, p.share) : 1;
  return p;
}

template <int DD, int GD>
int32_t run(Product& p, const Plan& plan, const void* dy, const int8_t* codes, const uint8_t* exps,
            void* grad, float* partial, void* stream) {
  void* args[] = {&p, &dy, &codes, &exps, &grad, &partial};
  const void* fn = plan.splits > 1 ? (const void*)wgrad_kernel<DD, GD, true>
                                   : (const void*)wgrad_kernel<DD, GD, false>;
  int32_t rc = launch(fn, dim3((uint32_t)plan.tiles, (uint32_t)plan.splits), dim3(kThreads), args,
                      0, stream, "rip_ckpt_wgrad");
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
  const Plan plan = make_plan(rows, out_features, in_features);
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
  const Plan plan = make_plan(rows, out_features, in_features);
  Product p{rows,
            ld_dy,
            ld_grad,
            (int)out_features,
            (int)in_features,
            (int)blocks,
            (int)ceil_div(in_features, kTile),
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
