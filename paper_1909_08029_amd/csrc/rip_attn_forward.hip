// Attention's forward pass (gfx950): out_i = sum_j softmax_j(x_ij) v_j in one pass over
// the keys, with the running maximum and sum of each query's scores.
//
// A wave takes 32 queries (a query and a head of it where heads share k and v) whose
// operands stay in registers, and goes over the keys in tiles that the workgroup
// shares in LDS.  Scores are computed as keys x queries: a lane holds one query's
// scores, so the maximum and sum need one exchange with the lane 32 away, and the
// exponentials are the operand of the product with v as they lie.  A maximum that
// grows by less than a factor of 64 (in e^x) stays the reference, which
// leaves the sums within fp32's range and saves rescaling them.
//
// Long sequences are bound by the matrix units and what lies between their
// instructions (16384 causal tokens, 16 heads of 128: 1.2 ms repeated by itself, 1.3 in
// passes with the backward pass, whose clock is lower: 920 and 840 TFLOP/s), single
// queries over long caches by memory (819 MB in 177 to 184 us), short ones by their own
// beginning and end (256 tokens, 64 columns: half of 36 us for 32 x 16 of them).
#include "rip_attn_tile.h"

namespace rip {
namespace attn {
namespace {

// Without a bias, with one, and with one whose gradient will be wanted: that sums ds
// in fp32, and its row sums delta come from out, which must not hold the rounding of
// the exponentials then.  They enter the product as two bf16 numbers (16 bits).
// (A kernel's name holds what its parameters' types depend on: plain numbers, as an
// unnamed type's place is counted differently for the host and the device.)
enum { kPlain, kBias, kExact };

constexpr float kSlack = 6.0f;  // growth of a maximum (log2) that needs no rescaling

template <int NT, int D, int WAVES, int KT, int EU, int MODE, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, EU) void forward_kernel(
    typename KernelArgs<Forward, MODE != 0>::type f) {
  constexpr int DT = storage(NT);
  typedef Tile<NT, D> Tl;
  typedef typename Tl::T T;
  constexpr int KB = KT / 32, QT = kRows * WAVES;
  constexpr bool BIAS = MODE != kPlain, EXACT = MODE == kExact;
  __shared__ typename Tl::template Store<KT> k_tile, v_tile;
  extern __shared__ __align__(16) float lut[];
  const Args& p = f.a;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, half = lane / 32;

  Share my;
  if (!my_share(p, p.heads / p.pack, &my)) return;
  const int hz = my.head, split = my.split;
  // the last tiles of a causal sequence have the most keys and go first
  const Place at = find<QT>(p, p.q, p.k, p.slots - 1 - my.slot, p.pack);
  const int lq = at.here.end - at.here.begin, lk = at.other.end - at.other.begin, shift = lk - lq;
  const int rows = lq * p.pack, w0 = at.tile * QT;
  if (w0 >= rows) return;
  const int head0 = hz * p.pack, kv = head0 / p.group;

  const int wq = w0 + wave * kRows, w = min(wq + lane % 32, rows - 1);
  const int i = p.by_pack.div(w), head = head0 + w - i * p.pack, pos = i + shift;
  const bool valid = wq + lane % 32 < rows;
  const int64_t token = at.here.begin + i;
  const int limit = p.causal ? min(lk, pos + 1) : lk;  // keys below it are seen
  const int least = __builtin_amdgcn_readlane(limit, 0), most = __builtin_amdgcn_readlane(limit, 31);
  int keys = lk;  // that the workgroup goes over
  if (p.causal) keys = max(0, min(lk, (int)p.by_pack.div(min(w0 + QT, rows) - 1) + shift + 1));
  int t = 0, end = keys;
  if (SPLIT) {
    const int share = (((keys + KT - 1) / KT + p.splits - 1) / p.splits) * KT;
    t = min(keys, split * share), end = min(keys, t + share);
  }
  const Bias bias{lut + kLutPad, p.lut_first, p.lut_size};

  const T* k0 = (const T*)f.k.p + at.other.begin * f.k.ld + (int64_t)kv * p.dim;
  const T* v0 = (const T*)f.v.p + at.other.begin * f.v.ld + (int64_t)kv * p.dim;
  const Tl at_lane(lane);

  f32x16 o[D / 32] = {};
  // reference (log2); the sum of this half's keys, and what its last rounding added (Kahan
  // 1965): equal terms all round the same way, so that 100000 plain additions err by 3e-4
  float m = -kInf, l = 0.0f, over = 0.0f;
  Stage<NT, D, KT, 64 * WAVES> ks, vs;
  // (fp32 of 256 columns has no registers for tiles on their way)
  constexpr bool kOnTheWay = NT != kFp32;
  if (kOnTheWay && t < end) {
    ks.load(k0, f.k.ld, t, end, p.dim);
    vs.load(v0, f.v.ld, t, end, p.dim);
  }
  Frag<NT> q[D / 16];
  load_row<NT, D>((const T*)f.q.p + token * f.q.ld + (int64_t)head * p.dim, valid, half, p.dim, q);
  if constexpr (BIAS) load_lut(p, f.map, head0, lut);
  for (; t < end; t += KT) {
    if (!kOnTheWay) {
      ks.load(k0, f.k.ld, t, end, p.dim);
      vs.load(v0, f.v.ld, t, end, p.dim);
    }
    ks.store(k_tile, k0, f.k.ld, t, end, p.dim);
    vs.store(v_tile, v0, f.v.ld, t, end, p.dim);
    lds_barrier();
    if (kOnTheWay && t + KT < end) {
      ks.load(k0, f.k.ld, t + KT, end, p.dim);
      vs.load(v0, f.v.ld, t + KT, end, p.dim);
    }
    if (wq < rows && t < most) {
      f32x16 s[KB] = {};
      Frag<NT> rows[2][KB];
      auto read = [&](int c) {
#pragma unroll
        for (int b = 0; b < KB; ++b) rows[c % 2][b] = at_lane.row(k_tile, b * 32, c);
      };
      read(0);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        if (c + 1 < D / 16) read(c + 1);
#pragma unroll
        for (int b = 0; b < KB; ++b) s[b] = mma(rows[c % 2][b], q[c], s[b]);
        group_end();
      }
      constexpr int kAhead = 2, kColumns = KB * 2 * (D / 32);  // columns on their way; all
      Frag<NT> columns[kAhead];
      auto read_column = [&](int x) {
        columns[x % kAhead] = at_lane.column(v_tile, 16 * (x / (D / 32)), x % (D / 32));
      };
      read_column(0);
      if (BIAS) {
        const int first = __builtin_amdgcn_readlane(pos, 0), last = __builtin_amdgcn_readlane(pos, 31);
#pragma unroll
        for (int b = 0; b < KB; ++b) {
          const int key = t + b * 32;
          add_bias<1>(s[b], p.scale2, bias, bias.uniform(key - last, key + 31 - first),
                      key + 4 * half - pos);
        }
      }
      if (t + KT > least || t + KT > end) {
        const int cut = min(limit, end) - t;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[b][r] = b * 32 + block_row(r, half) < cut ? s[b][r] : -kInf;
      }
      float top = s[0][0];
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
      top = max_halves(BIAS ? top : top * p.scale2);
      if (__any(top > m + kSlack)) {
        const float next = fmaxf(m, top), scale = m == next ? 1.0f : __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= scale, over *= scale;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[c][r] *= scale;
      }
      const float ref = m == -kInf ? 0.0f : m;  // no key seen so far: every exponential is 0
      float sums[4];  // of the tile
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = BIAS ? s[b][r] - ref : __builtin_fmaf(s[b][r], p.scale2, -ref);
          s[b][r] = __builtin_amdgcn_exp2f(x);
          sums[r % 4] = b == 0 && r < 4 ? s[b][r] : sums[r % 4] + s[b][r];
        }
      const float more = ((sums[0] + sums[1]) + (sums[2] + sums[3])) - over, sum = l + more;
      over = (sum - l) - more;
      l = sum;
      // e^x rounded to bf16 (half a step of 2^-8, as out is; their sum is not) so that
      // the product runs at bf16's rate
      Frag<NT> e[KB * 2], rest[EXACT ? KB * 2 : 1];
#pragma unroll
      for (int u = 0; u < KB * 2; ++u) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = s[u / 2][8 * (u % 2) + j];
        e[u].set(x);
        if constexpr (EXACT) {
          float y[8];
          e[u].get(y);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] -= y[j];
          rest[u].set(x);
        }
      }
      read_column(1);
      group_end();
#pragma unroll
      for (int x = 0; x < kColumns; ++x) {
        const int u = x / (D / 32), c = x % (D / 32);
        const Frag<NT> v = columns[x % kAhead];
        if (x + kAhead < kColumns) read_column(x + kAhead);
        o[c] = mma(v, e[u], o[c]);
        if constexpr (EXACT) o[c] = mma(v, rest[u], o[c]);
        group_end();
      }
    }
    lds_barrier();
  }
  if (!valid) return;
  l = add_halves(l - over);
  if constexpr (SPLIT) {
    const int64_t row = ((int64_t)split * p.heads + head) * p.q.tokens + token;
    const int64_t all = (int64_t)p.splits * p.heads * p.q.tokens;
    float* to = f.part + row * p.dim;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float x[4] = {o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]};
        store4<RIP_FP32>(to, c * 32 + block_row(r, half), p.dim, x);
      }
    if (half == 0) {
      f.part[all * p.dim + row] = m;
      f.part[all * (p.dim + 1) + row] = l;
    }
  } else {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    T* out = (T*)f.out.p + token * f.out.ld + (int64_t)head * p.dim;
    T* low = f.low.p ? (T*)f.low.p + token * f.low.ld + (int64_t)head * p.dim : nullptr;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = o[c][r + j] * inv;
        store4<DT>(out, c * 32 + block_row(r, half), p.dim, x);
        if (DT == RIP_BF16 && low) {
#pragma unroll
          for (int j = 0; j < 4; j += 2) {
            const uint32_t b = Elem<RIP_BF16>::pack2(x[j], x[j + 1]);
            x[j] -= __uint_as_float(b << 16), x[j + 1] -= __uint_as_float(b & 0xffff0000u);
          }
          store4<DT>(low, c * 32 + block_row(r, half), p.dim, x);
        }
      }
    if (f.lse && half == 0)
      f.lse[(int64_t)head * p.q.tokens + token] = l == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// The splits of a query and head joined by a workgroup: a lane of each wave has a
// split's weight, and the waves take the splits in turn.
template <int DT>
__global__ __launch_bounds__(256) void join_kernel(Forward f) {
  typedef typename Elem<DT>::T T;
  static_assert(kMaxSplits <= 64, "a lane to a split");
  __shared__ float sums[4][RIP_MAX_HEAD_DIM];
  const Args& p = f.a;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t all = (int64_t)p.heads * p.q.tokens, row = blockIdx.x;
  const float* ms = f.part + all * p.splits * p.dim;
  float m = -kInf, l = 0.0f;
  if (lane < p.splits) {
    m = ms[lane * all + row];
    l = ms[(p.splits + lane) * all + row];
  }
  float top = m;
#pragma unroll
  for (int o = 32; o >= 1; o /= 2) top = fmaxf(top, __shfl_xor(top, o));
  const float weight = __builtin_amdgcn_exp2f(m - (top == -kInf ? 0.0f : top));
  l *= weight;
#pragma unroll
  for (int o = 32; o >= 1; o /= 2) l += __shfl_xor(l, o);
  constexpr int kColumns = RIP_MAX_HEAD_DIM / 64, kAtOnce = 4;  // splits of a wave
  float x[kColumns] = {};
  const float* from = f.part + row * p.dim + lane;
  for (int s0 = wave; s0 < p.splits; s0 += 4 * kAtOnce) {
    float y[kAtOnce][kColumns];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
      for (int c = 0; c < kColumns; ++c)
        y[i][c] = lane + 64 * c < p.dim ? from[min(s0 + 4 * i, p.splits - 1) * all * p.dim + 64 * c] : 0.0f;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float w = __shfl(weight, min(s0 + 4 * i, 63));
      if (s0 + 4 * i < p.splits)
#pragma unroll
        for (int c = 0; c < kColumns; ++c) x[c] += y[i][c] * w;
    }
  }
#pragma unroll
  for (int c = 0; c < kColumns; ++c) sums[wave][lane + 64 * c] = x[c];
  __syncthreads();
  const int c = threadIdx.x;
  const int64_t head = row / p.q.tokens, token = row - head * p.q.tokens;
  if (c < p.dim) {
    const float y = ((sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c])) * (l == 0.0f ? 0.0f : 1.0f / l);
    Elem<DT>::store((T*)f.out.p + token * f.out.ld + head * p.dim + c, y);
    if (DT == RIP_BF16 && f.low.p) {
      const uint32_t b = Elem<RIP_BF16>::pack2(y, y) << 16;
      Elem<DT>::store((T*)f.low.p + token * f.low.ld + head * p.dim + c, y - __uint_as_float(b));
    }
  }
  if (f.lse && c == 0) f.lse[row] = l == 0.0f ? -kInf : (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// Variants: keys of a tile, and waves to a SIMD that the registers have to leave room for
// (three for 64 columns: 8192 tokens, 16 heads, causal 184 us, 212 with two).
template <int NT, int D, int WAVES, int MODE>
const void* variant(bool split) {
  constexpr int keys = (NT == kBf16 && D <= 128) || (NT == kSplit && D <= 64) ? 64 : 32;
  constexpr int units = NT == kBf16 ? (D <= 64 ? 3 : D <= 128 ? 2 : 1) : D <= 96 ? 2 : 1;
  return split ? (const void*)forward_kernel<NT, D, WAVES, keys, units, MODE, true>
               : (const void*)forward_kernel<NT, D, WAVES, keys, units, MODE, false>;
}
template <int NT, int D, int WAVES>
const void* variant(int mode, bool split) {
  if (NT == kBf16 && mode == kExact) return variant<kBf16, D, WAVES, kExact>(split);
  return mode == kPlain ? variant<NT, D, WAVES, kPlain>(split) : variant<NT, D, WAVES, kBias>(split);
}
template <int NT, int D>
const void* variant(int waves, int mode, bool split) {
  if constexpr (NT == kBf16 && (D == 96 || D == 128))
    if (waves == 8) return variant<NT, D, 8>(mode, split);
  return variant<NT, D, 4>(mode, split);
}
const void* kernel_of(int32_t dtype, int width, int waves, int mode, bool split) {
  const bool bf16 = dtype == RIP_BF16;
  switch (width) {
    case 64: return bf16 ? variant<kBf16, 64>(waves, mode, split) : variant<kSplit, 64>(waves, mode, split);
    case 96: return bf16 ? variant<kBf16, 96>(waves, mode, split) : variant<kSplit, 96>(waves, mode, split);
    case 128: return bf16 ? variant<kBf16, 128>(waves, mode, split) : variant<kSplit, 128>(waves, mode, split);
    default: return bf16 ? variant<kBf16, 256>(waves, mode, split) : variant<kFp32, 256>(waves, mode, split);
  }
}

}  // namespace

int32_t run_forward(WithBias<Forward>& f, int32_t dtype, int width, int waves, void* stream) {
  const Args& p = f.a;
  void* args[] = {&f};
  const bool split = p.splits > 1;
  const int mode = !p.lut_size ? kPlain : f.low.p ? kExact : kBias;
  const void* fn = kernel_of(dtype, width, waves, mode, split);
  int32_t rc = launch(fn, grid_of(p, p.heads / p.pack), dim3(64 * waves), args, p.lut_size ? 4 * lut_floats(p.lut_size) : 0, stream, "rip_attn_forward");
  if (rc || !split) return rc;
  return launch(dtype == RIP_BF16 ? (const void*)join_kernel<RIP_BF16> : (const void*)join_kernel<RIP_FP32>,
                dim3((uint32_t)(p.heads * p.q.tokens)), dim3(256), args, 0, stream,
                "rip_attn_forward: join");
}

}  // namespace attn
}  // namespace rip
