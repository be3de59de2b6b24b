// Attention's backward pass (gfx950), which computes the probabilities again from the
// scores and the rows' log-sums:
//
//   p_ij = e^(x_ij - lse_i),  ds_ij = p_ij (dout_i . v_j - delta_i),  delta_i = dout_i . out_i
//   dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i;  dv_j = sum_i p_ij dout_i
//
// Two kernels, each with the sum that it accumulates in registers: one over the keys
// for 32 queries to a wave (dq, delta and the bias's gradient), one over the queries
// for 32 keys to a wave (dk and dv, over all heads that share them).  Seven products
// where one kernel would take five, but no sum is added atomically or goes through
// memory.  16384 causal tokens, 16 heads of 128, four of k and v: 1.6 ms for dq, 2.65
// for dk and dv (1030 and 830 TFLOP/s of the products that they take).
#include "rip_attn_tile.h"

namespace rip {
namespace attn {
namespace {

// A row's log-sum in the log2 domain; +inf, so that every exponential is 0, for a
// query that sees no key.
__device__ __forceinline__ float reference(float lse) {
  return lse == -kInf ? kInf : lse * kLog2e;
}

// Behind the bias's values in LDS: sums by distance of each wave, and a block of each.
// A block's element of key k and query n lies in row (k - n) mod 64, column n; the
// places that no element takes are zeros from the start.  Rows of 36 numbers: a lane's
// writes and the reads of 16 bytes fall into different banks.
constexpr int kBlockPitch = 36, kBlockFloats = 64 * kBlockPitch;
__device__ __host__ constexpr int sums_size(int lut_size) { return lut_size + 2 * 62; }

// Adds a block's ds (32 keys x 32 queries as the matrix instructions leave them, the
// first at distance `rel`) to the sums by distance, a lane to a diagonal.  Only this
// wave touches its sums, so their order is fixed.
__device__ __forceinline__ void add_diagonals(const f32x16& ds, int rel, int first, float* sums,
                                              float* block, int lane) {
  const int n = lane % 32;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    block[((block_row(r, lane / 32) - n) & 63) * kBlockPitch + n] = ds[r];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  const int off = lane - 31;  // key - query within the block
  if (lane < 63) {
    const f32x4* row = (const f32x4*)(block + (off & 63) * kBlockPitch);
    f32x4 sum = row[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) sum += row[i];
    sums[rel + off - first + 62] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  __builtin_amdgcn_wave_barrier();
}

template <int NT, int D, int WAVES, int STEP, int EU, bool BIAS, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, EU) void dq_kernel(
    typename KernelArgs<Backward, BIAS>::type f) {
  constexpr int DT = storage(NT);
  typedef Tile<NT, D> Tl;
  typedef typename Tl::T T;
  constexpr int KT = STEP, KB = KT / 32, QT = kRows * WAVES;
  __shared__ typename Tl::template Store<KT> k_tile, v_tile;
  extern __shared__ __align__(16) float lut[];
  const Args& p = f.a;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, half = lane / 32;

  Share my;
  if (!my_share(p, p.heads / p.pack, &my)) return;
  const int hz = my.head, split = my.split, slot = p.slots - 1 - my.slot;
  const Place at = find<QT>(p, p.q, p.k, slot, p.pack);
  const int lq = at.here.end - at.here.begin, lk = at.other.end - at.other.begin, shift = lk - lq;
  const int rows = lq * p.pack, w0 = at.tile * QT;
  const int head0 = hz * p.pack, kv = head0 / p.group;
  // sums by distance of each wave, then a block of each
  const int pitch = BIAS ? sums_size(p.lut_size) : 0;
  float* const sums = lut + lut_floats(p.lut_size);
  float* const mine = sums + wave * pitch;
  float* const block = sums + WAVES * pitch + wave * kBlockFloats;
  int intervals = 0;
  if constexpr (BIAS) intervals = f.map.n;
  float* const bias_part =
      BIAS ? f.bias_part + ((int64_t)hz * p.slots * p.splits + slot * p.splits + split) * intervals
           : nullptr;
  if (w0 >= rows) {
    if (BIAS)
      for (int b = threadIdx.x; b < intervals; b += 64 * WAVES) bias_part[b] = 0.0f;
    return;
  }

  const int wq = w0 + wave * kRows, w = min(wq + lane % 32, rows - 1);
  const int i = p.by_pack.div(w), head = head0 + w - i * p.pack, pos = i + shift;
  const bool valid = wq + lane % 32 < rows;
  const int64_t token = at.here.begin + i;
  const int limit = p.causal ? min(lk, pos + 1) : lk;
  const int least = __builtin_amdgcn_readlane(limit, 0), most = __builtin_amdgcn_readlane(limit, 31);
  int keys = lk;
  if (p.causal) keys = max(0, min(lk, (int)p.by_pack.div(min(w0 + QT, rows) - 1) + shift + 1));
  int t = 0, end = keys;
  if (SPLIT) {
    const int share = (((keys + KT - 1) / KT + p.splits - 1) / p.splits) * KT;
    t = min(keys, split * share), end = min(keys, t + share);
  }
  const Bias bias{lut + kLutPad, p.lut_first, p.lut_size};
  float below = 0.0f, above = 0.0f;  // ds of blocks all in the first (last) interval
  if constexpr (BIAS) {
    load_lut(p, f.map, head0, lut);
    for (int x = lane; x < pitch; x += 64) mine[x] = 0.0f;
    for (int x = lane; x < kBlockFloats; x += 64) block[x] = 0.0f;
  }

  const T* k0 = (const T*)f.k.p + at.other.begin * f.k.ld + (int64_t)kv * p.dim;
  const T* v0 = (const T*)f.v.p + at.other.begin * f.v.ld + (int64_t)kv * p.dim;
  const Tl at_lane(lane);

  f32x16 dq[D / 32] = {};
  Stage<NT, D, KT, 64 * WAVES> ks, vs;
  constexpr bool kOnTheWay = NT != kFp32;  // as in the forward pass
  if (kOnTheWay && t < end) {
    ks.load(k0, f.k.ld, t, end, p.dim);
    vs.load(v0, f.v.ld, t, end, p.dim);
  }
  Frag<NT> q[D / 16], dout[D / 16];
  load_row<NT, D>((const T*)f.q.p + token * f.q.ld + (int64_t)head * p.dim, valid, half, p.dim, q);
  load_row<NT, D>((const T*)f.dout.p + token * f.dout.ld + (int64_t)head * p.dim, valid, half, p.dim,
                  dout);
  // delta in fp32 from out and what its rounding left
  float delta = 0.0f;
  {
    const int64_t at_head = (int64_t)head * p.dim;
    Frag<NT> out[D / 16], low[D / 16] = {};
    load_row<NT, D>((const T*)f.out.p + token * f.out.ld + at_head, valid, half, p.dim, out);
    if (DT == RIP_BF16 && f.low.p)
      load_row<NT, D>((const T*)f.low.p + token * f.low.ld + at_head, valid, half, p.dim, low);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      float x[kLane], y[kLane], z[kLane];
      out[c].get(x), low[c].get(y), dout[c].get(z);
#pragma unroll
      for (int j = 0; j < kLane; ++j)
        delta = __builtin_fmaf(z[j], DT == RIP_BF16 ? x[j] + y[j] : x[j], delta);
    }
    delta = add_halves(delta);
  }
  const int64_t row = (int64_t)head * p.q.tokens + token;
  const float lse = f.lse[row], ref = valid ? reference(lse) : kInf;
  if (valid && half == 0 && split == 0) f.delta[row] = delta;
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
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        f32x16 s = {}, dp = {};
        struct Rows {
          Frag<NT> k, v;
        } rows[2];
        auto read = [&](int c, Rows& r) {
          r.k = at_lane.row(k_tile, b * 32, c);
          r.v = at_lane.row(v_tile, b * 32, c);
        };
        read(0, rows[0]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          const Rows& r = rows[c % 2];
          if (c + 1 < D / 16) read(c + 1, rows[(c + 1) % 2]);
          s = mma(r.k, q[c], s);
          dp = mma(r.v, dout[c], dp);
          group_end();
        }
        constexpr int kAhead = 2;  // columns on their way
        Frag<NT> columns[kAhead];
        auto read_column = [&](int x) {
          columns[x % kAhead] = at_lane.column(k_tile, b * 32 + 16 * (x / (D / 32)), x % (D / 32));
        };
        read_column(0);
        const int key = t + b * 32;
        int side = 0;
        if (BIAS) {
          side = bias.uniform(key - __builtin_amdgcn_readlane(pos, 31),
                              key + 31 - __builtin_amdgcn_readlane(pos, 0));
          add_bias<1>(s, p.scale2, bias, side, key + 4 * half - pos);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = BIAS ? s[r] - ref : __builtin_fmaf(s[r], p.scale2, -ref);
          s[r] = __builtin_amdgcn_exp2f(x);
        }
        if (key + 32 > least || key + 32 > end) {
          const int cut = min(limit, end) - key;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = block_row(r, half) < cut ? s[r] : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
        if (BIAS) {
          if (side) {
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += s[r];
            if (side < 0)
              below += sum;
            else
              above += sum;
          } else {
            // (queries behind the last have zeros, whatever their diagonal)
            add_diagonals(s, key - (wq + shift), p.lut_first, mine, block, lane);
          }
        }
        // ds rounded to bf16 (half a step of 2^-8, as dq is) for the product
        Frag<NT> e[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = s[8 * u + j];
          e[u].set(x);
        }
        read_column(1);
        group_end();
#pragma unroll
        for (int x = 0; x < 2 * (D / 32); ++x) {
          const Frag<NT> column = columns[x % kAhead];
          if (x + kAhead < 2 * (D / 32)) read_column(x + kAhead);
          dq[x % (D / 32)] = mma(column, e[x / (D / 32)], dq[x % (D / 32)]);
          group_end();
        }
      }
    }
    lds_barrier();
  }
  if (valid) {
    T* to = (T*)f.dq.p + token * f.dq.ld + (int64_t)head * p.dim;
    float* part = SPLIT ? f.part + (((int64_t)split * p.q.tokens + token) * p.heads + head) * p.dim
                        : nullptr;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = dq[c][r + j] * p.scale;
        if (SPLIT)
          store4<RIP_FP32>(part, c * 32 + block_row(r, half), p.dim, x);
        else
          store4<DT>(to, c * 32 + block_row(r, half), p.dim, x);
      }
  }
  if constexpr (BIAS) {
    // sums of an interval's distances over the waves, a wave to an interval
    __syncthreads();
#pragma unroll
    for (int o = 32; o >= 1; o /= 2) below += __shfl_xor(below, o), above += __shfl_xor(above, o);
    if (lane == 0) block[0] = below, block[1] = above;
    __syncthreads();
    const float* const blocks = sums + WAVES * pitch;
    const int x0 = p.lut_first - 62;  // distance of the first sum
    for (int b = wave; b < intervals; b += WAVES) {
      const int from = b == 0 ? x0 : f.map.start[b - 1];
      const int to = b == intervals - 1 ? x0 + pitch : f.map.start[b];
      float sum = 0.0f;
      for (int x = from + lane; x < to; x += 64)
#pragma unroll
        for (int s = 0; s < WAVES; ++s) sum += sums[s * pitch + x - x0];
      if (lane < WAVES) {
        if (b == 0) sum += blocks[lane * kBlockFloats];
        if (b == intervals - 1) sum += blocks[lane * kBlockFloats + 1];
      }
#pragma unroll
      for (int o = 32; o >= 1; o /= 2) sum += __shfl_xor(sum, o);
      if (lane == 0) bias_part[b] = sum;
    }
  }
}

// dk (DK) and dv (DV) of 32 keys to a wave.
template <int NT, int D, int WAVES, int STEP, int EU, bool V_LDS, bool BIAS, bool SPLIT, bool DK, bool DV>
__global__ __launch_bounds__(64 * WAVES, EU) void dkv_kernel(
    typename KernelArgs<Backward, BIAS>::type f) {
  constexpr int DT = storage(NT);
  typedef Tile<NT, D> Tl;
  typedef typename Tl::T T;
  constexpr int QT = STEP, QB = QT / 32, KT = kRows * WAVES;
  __shared__ typename Tl::template Store<QT> q_tile, do_tile;
  __shared__ typename Tl::template Store<QT> v_tile[V_LDS ? KT / QT : 1];
  __shared__ __align__(16) float refs[QT], deltas[QT];
  extern __shared__ __align__(16) float lut[];
  const Args& p = f.a;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, half = lane / 32;

  Share my;
  if (!my_share(p, p.heads / p.group, &my)) return;
  const int kv = my.head, split = my.split;
  // the first keys of a causal sequence have the most queries
  const Place at = find<KT>(p, p.k, p.q, my.slot, 1);
  const int lk = at.here.end - at.here.begin, lq = at.other.end - at.other.begin, shift = lk - lq;
  const int j0 = at.tile * KT;
  if (j0 >= lk) return;
  const int jw = j0 + wave * kRows, j = min(jw + lane % 32, lk - 1);
  const bool valid = jw + lane % 32 < lk;
  const int64_t token = at.here.begin + j;
  // queries from `first` on see the key
  const int first = p.causal ? j - shift : -1;
  const int first_last = __builtin_amdgcn_readlane(first, 31);
  const int first_wave = __builtin_amdgcn_readlane(first, 0);
  const int start = p.causal ? max(0, j0 - shift) / QT * QT : 0;  // of the workgroup
  const int tiles = lq > start ? (lq - start + QT - 1) / QT : 0, steps = tiles * p.group;
  int n = 0, end = steps;  // (head, tile), tile fastest
  if (SPLIT) {
    const int share = (steps + p.splits - 1) / p.splits;
    n = min(steps, split * share), end = min(steps, n + share);
  }
  const Bias bias{lut + kLutPad, p.lut_first, p.lut_size};

  f32x16 dk[DK ? D / 32 : 1] = {}, dv[DV ? D / 32 : 1] = {};

  const T* q0 = (const T*)f.q.p + at.other.begin * f.q.ld + (int64_t)kv * p.group * p.dim;
  const T* do0 = (const T*)f.dout.p + at.other.begin * f.dout.ld + (int64_t)kv * p.group * p.dim;
  const Tl at_lane(lane);
  Stage<NT, D, QT, 64 * WAVES> qs, ds;
  if constexpr (DK && V_LDS) {
    const T* v0 = (const T*)f.v.p + at.here.begin * f.v.ld + (int64_t)kv * p.dim;
#pragma unroll 1
    for (int r = 0; r < KT / QT; ++r) {
      qs.load(v0, f.v.ld, j0 + r * QT, lk, p.dim);
      qs.store(v_tile[r], v0, f.v.ld, j0 + r * QT, lk, p.dim);
    }
  }
  float lse = 0.0f, del = 0.0f;  // of query threadIdx.x of the tile
  auto load = [&](int step) {
    const int g = step / tiles, i0 = start + (step - g * tiles) * QT;
    qs.load(q0 + (int64_t)g * p.dim, f.q.ld, i0, lq, p.dim);
    ds.load(do0 + (int64_t)g * p.dim, f.dout.ld, i0, lq, p.dim);
    const int64_t row = ((int64_t)kv * p.group + g) * p.q.tokens + at.other.begin + min(i0 + (int)threadIdx.x, lq - 1);
    lse = f.lse[row];
    if (DK) del = f.delta[row];
  };
  constexpr bool kOnTheWay = NT != kFp32;
  if (kOnTheWay && n < end) load(n);
  Frag<NT> k[D / 16], v[DK && !V_LDS ? D / 16 : 1];
  load_row<NT, D>((const T*)f.k.p + token * f.k.ld + (int64_t)kv * p.dim, valid, half, p.dim, k);
  if constexpr (DK && !V_LDS)
    load_row<NT, D>((const T*)f.v.p + token * f.v.ld + (int64_t)kv * p.dim, valid, half, p.dim, v);
  int lut_head = -1;
  for (; n < end; ++n) {
    const int g = n / tiles, i0 = start + (n - g * tiles) * QT;
    if (!kOnTheWay) load(n);
    qs.store(q_tile, q0 + (int64_t)g * p.dim, f.q.ld, i0, lq, p.dim);
    ds.store(do_tile, do0 + (int64_t)g * p.dim, f.dout.ld, i0, lq, p.dim);
    if (threadIdx.x < QT) {
      refs[threadIdx.x] = i0 + (int)threadIdx.x < lq ? reference(lse) : kInf;
      deltas[threadIdx.x] = del;
    }
    if constexpr (BIAS) {
      if (lut_head != g) load_lut(p, f.map, kv * p.group + g, lut);
      lut_head = g;
    }
    lds_barrier();
    if (kOnTheWay && n + 1 < end) load(n + 1);
    if (jw < lk && i0 + QT > first_wave) {
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        f32x16 s = {}, dp = {};
        struct Rows {
          Frag<NT> q, dout, v;
        } rows[2];
        auto read = [&](int c, Rows& r) {
          r.q = at_lane.row(q_tile, b * 32, c);
          if constexpr (DK) r.dout = at_lane.row(do_tile, b * 32, c);
          if constexpr (DK && V_LDS) r.v = at_lane.row(v_tile[wave * kRows / QT], wave * kRows % QT, c);
        };
        read(0, rows[0]);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          Rows& r = rows[c % 2];
          if (c + 1 < D / 16) read(c + 1, rows[(c + 1) % 2]);
          s = mma(r.q, k[c], s);
          if constexpr (DK) dp = mma(r.dout, V_LDS ? r.v : v[V_LDS ? 0 : c], dp);
          group_end();
        }
        // the first columns are on their way during the exponentials
        struct Columns {
          Frag<NT> q, dout;
        } columns[2];
        auto read_columns = [&](int x, Columns& r) {
          const int u = x / (D / 32), c = x % (D / 32);
          if constexpr (DV) r.dout = at_lane.column(do_tile, b * 32 + 16 * u, c);
          if constexpr (DK) r.q = at_lane.column(q_tile, b * 32 + 16 * u, c);
        };
        read_columns(0, columns[0]);
        const int ib = i0 + b * 32;
        if (BIAS)
          add_bias<-1>(s, p.scale2, bias,
                       bias.uniform(__builtin_amdgcn_readlane(j, 0) - (ib + 31 + shift),
                                    __builtin_amdgcn_readlane(j, 31) - (ib + shift)),
                       j - (ib + 4 * half + shift));
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4 ref4 = *(const f32x4*)&refs[b * 32 + block_row(r, half)];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const float y = BIAS ? s[r + x] - ref4[x] : __builtin_fmaf(s[r + x], p.scale2, -ref4[x]);
            s[r + x] = __builtin_amdgcn_exp2f(y);
          }
        }
        if (ib < first_last) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = ib + block_row(r, half) < first ? 0.0f : s[r];
        }
        if constexpr (DK) {
#pragma unroll
          for (int r = 0; r < 16; r += 4) {
            const f32x4 del4 = *(const f32x4*)&deltas[b * 32 + block_row(r, half)];
#pragma unroll
            for (int x = 0; x < 4; ++x) dp[r + x] = s[r + x] * (dp[r + x] - del4[x]);
          }
        }
        // p and ds rounded to bf16 (half a step of 2^-8, as dv and dk are)
        Frag<NT> e[2], de[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float x[8], y[8];
#pragma unroll
          for (int z = 0; z < 8; ++z) x[z] = s[8 * u + z], y[z] = dp[8 * u + z];
          e[u].set(x);
          de[u].set(y);
        }
        group_end();
#pragma unroll
        for (int x = 0; x < 2 * (D / 32); ++x) {
          const int u = x / (D / 32), c = x % (D / 32);
          const Columns& r = columns[x % 2];
          if (x + 1 < 2 * (D / 32)) read_columns(x + 1, columns[(x + 1) % 2]);
          if constexpr (DV) dv[c] = mma(r.dout, e[u], dv[c]);
          if constexpr (DK) dk[c] = mma(r.q, de[u], dk[c]);
          group_end();
        }
      }
    }
    lds_barrier();
  }
  if (!valid) return;
  const int kv_heads = p.heads / p.group;
  const int64_t row = ((int64_t)split * p.k.tokens + token) * kv_heads + kv;
  const int64_t all = (int64_t)p.splits * p.k.tokens * kv_heads;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int col = c * 32 + block_row(r, half);
      float x[4];
      if constexpr (DK) {
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = dk[c][r + z] * p.scale;
        if (SPLIT)
          store4<RIP_FP32>(f.part + row * p.dim, col, p.dim, x);
        else
          store4<DT>((T*)f.dk.p + token * f.dk.ld + (int64_t)kv * p.dim, col, p.dim, x);
      }
      if constexpr (DV) {
#pragma unroll
        for (int z = 0; z < 4; ++z) x[z] = dv[c][r + z];
        if (SPLIT)
          store4<RIP_FP32>(f.part + (all + row) * p.dim, col, p.dim, x);
        else
          store4<DT>((T*)f.dv.p + token * f.dv.ld + (int64_t)kv * p.dim, col, p.dim, x);
      }
    }
}

// The splits' parts of `tokens` rows of `width` added in order.
template <int DT>
__global__ __launch_bounds__(256) void add_kernel(const float* part, int splits, int64_t tokens,
                                                  int width, typename Elem<DT>::T* to, int64_t ld) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, all = tokens * width;
  if (i >= all) return;
  float sum = 0.0f;
  for (int s = 0; s < splits; ++s) sum += part[s * all + i];
  const int64_t row = i / width;
  Elem<DT>::store(to + row * ld + (i - row * width), sum);
}

// The bias's gradient: a workgroup adds the parts of one row of the table and one head.
template <int DT>
__global__ __launch_bounds__(256) void bias_kernel(const float* part, Buckets map,
                                                   int64_t parts, typename Elem<DT>::T* grad,
                                                   int64_t ld, int accumulate) {
  __shared__ float sums[4];
  const int row = blockIdx.x, head = blockIdx.y, n = parts ? map.n : 0;
  float sum = 0.0f;
  for (int b = 0; b < n; ++b) {
    if (map.row[b] != row) continue;
    for (int64_t x = threadIdx.x; x < parts; x += 256) sum += part[(head * parts + x) * n + b];
  }
#pragma unroll
  for (int o = 32; o >= 1; o /= 2) sum += __shfl_xor(sum, o);
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  typename Elem<DT>::T* g = grad + (int64_t)row * ld + head;
  Elem<DT>::store(g, accumulate ? Elem<DT>::load(g) + sum : sum);
}

// Variants: rows of a tile of the other axis, and waves to a SIMD that the registers
// have to leave room for.
template <int NT, int D, int WAVES, bool BIAS, bool SPLIT>
const void* dq_of() {
  constexpr int step = NT == kBf16 && D <= 128 && (D > 64 || BIAS) ? 64 : 32;
  // (four waves to a tile of 96 or 128 bf16 columns: their LDS leaves no room for more)
  constexpr int units = D <= 64 || WAVES == 8 ? 2 : 1;
  static_assert(!BIAS || sizeof(typename Tile<NT, D>::template Store<step>) * 2 +
                                 4 * (lut_floats(WAVES == 8 ? kSpanOfEight : RIP_MAX_BIAS_SPAN) +
                                      WAVES * (sums_size(WAVES == 8 ? kSpanOfEight : RIP_MAX_BIAS_SPAN) +
                                               kBlockFloats)) <= 160 * 1024,
                "the LDS holds tiles, the bias and the sums");
  return (const void*)dq_kernel<NT, D, WAVES, step, units, BIAS, SPLIT>;
}
template <int NT, int D>
const void* dq_of(int waves, bool bias, bool split) {
  constexpr int kWaves = dq_waves(NT == kBf16, D, 0);
  if (bias && waves != kWaves)
    return split ? dq_of<NT, D, 4, true, true>() : dq_of<NT, D, 4, true, false>();
  return bias ? (split ? dq_of<NT, D, kWaves, true, true>() : dq_of<NT, D, kWaves, true, false>())
              : (split ? dq_of<NT, D, kWaves, false, true>() : dq_of<NT, D, kWaves, false, false>());
}
template <int NT, int D, int WAVES, bool BIAS, bool SPLIT, bool DK, bool DV>
const void* dkv_of() {
  constexpr int step = NT == kBf16 && D <= 64 ? 64 : 32;
  constexpr int units = D <= (NT == kBf16 ? 128 : 64) ? 2 : 1;
  // the keys' values in LDS where the registers hold too much beside them
  constexpr bool v_lds = (NT == kBf16 && D > 64 && D <= 128) || (NT == kSplit && D != 96);
  return (const void*)dkv_kernel<NT, D, WAVES, step, units, v_lds, BIAS, SPLIT, DK, DV>;
}
template <int NT, int D, int WAVES, bool DK = true, bool DV = true>
const void* dkv_of(bool bias, bool split) {
  return bias ? (split ? dkv_of<NT, D, WAVES, true, true, DK, DV>() : dkv_of<NT, D, WAVES, true, false, DK, DV>())
              : (split ? dkv_of<NT, D, WAVES, false, true, DK, DV>() : dkv_of<NT, D, WAVES, false, false, DK, DV>());
}
template <int DT>
int32_t add(const float* part, int splits, int64_t tokens, int width, Heads to, void* stream) {
  void* args[] = {&part, &splits, &tokens, &width, &to.p, &to.ld};
  return launch((const void*)add_kernel<DT>, dim3((uint32_t)ceil_div(tokens * width, 256)), dim3(256),
                args, 0, stream, "rip_attn_backward: add");
}

template <int DT>
int32_t run(WithBias<Backward>& f, const Args& over_q, const Args& over_k, const Plans& plan, void* stream) {
  int32_t rc;
  const bool bias = over_q.lut_size;
  const int width = plan.q.width;
  {
    f.a = over_q;
    const bool split = f.a.splits > 1;
    constexpr int NT = DT == RIP_BF16 ? kBf16 : kSplit, kWide = DT == RIP_BF16 ? kBf16 : kFp32;
    const int waves = plan.q.waves;
    const void* fn = width == 64    ? dq_of<NT, 64>(waves, bias, split)
                     : width == 96  ? dq_of<NT, 96>(waves, bias, split)
                     : width == 128 ? dq_of<NT, 128>(waves, bias, split)
                                    : dq_of<kWide, 256>(waves, bias, split);
    const size_t lds =
        bias ? 4 * (lut_floats(f.a.lut_size) + plan.q.waves * (sums_size(f.a.lut_size) + kBlockFloats)) : 0;
    void* args[] = {&f};
    if ((rc = launch(fn, grid_of(f.a, f.a.heads / f.a.pack), dim3(64 * plan.q.waves), args, lds, stream, "rip_attn_backward: queries")))
      return rc;
    if (split && (rc = add<DT>(f.part, f.a.splits, f.a.q.tokens, f.a.heads * f.a.dim, f.dq, stream)))
      return rc;
  }
  f.a = over_k;
  const int kv_heads = f.a.heads / f.a.group;
  const bool split = f.a.splits > 1;
  const dim3 grid = grid_of(f.a, kv_heads);
  const size_t lds = bias ? 4 * lut_floats(f.a.lut_size) : 0;
  void* args[] = {&f};
  const char* what = "rip_attn_backward: keys";
  if (width == 256) {
    // dk and dv with the operands of both do not fit the registers: one after the other
    constexpr int kWide = DT == RIP_BF16 ? kBf16 : kFp32;
    if ((rc = launch(dkv_of<kWide, 256, 4, false, true>(bias, split), grid, dim3(64 * plan.k.waves), args,
                     lds, stream, what)) ||
        (rc = launch(dkv_of<kWide, 256, 4, true, false>(bias, split), grid, dim3(64 * plan.k.waves), args,
                     lds, stream, what)))
      return rc;
  } else {
    const void* fn;
    if constexpr (DT == RIP_BF16)
      fn = width == 64 ? (plan.k.waves == 4 ? dkv_of<kBf16, 64, 4>(bias, split) : dkv_of<kBf16, 64, 8>(bias, split))
           : width == 96 ? dkv_of<kBf16, 96, 8>(bias, split)
                         : dkv_of<kBf16, 128, 8>(bias, split);
    else
      fn = width == 64   ? dkv_of<kSplit, 64, 4>(bias, split)
           : width == 96 ? dkv_of<kSplit, 96, 4>(bias, split)
                         : dkv_of<kSplit, 128, 4>(bias, split);
    if ((rc = launch(fn, grid, dim3(64 * plan.k.waves), args, lds, stream, what))) return rc;
  }
  if (!split) return RIP_OK;
  const int cols = kv_heads * f.a.dim;
  if ((rc = add<DT>(f.part, f.a.splits, f.a.k.tokens, cols, f.dk, stream))) return rc;
  return add<DT>(f.part + (int64_t)f.a.splits * f.a.k.tokens * cols, f.a.splits, f.a.k.tokens, cols,
                 f.dv, stream);
}

}  // namespace

int32_t run_backward(WithBias<Backward>& f, const Args& over_q, const Args& over_k, int32_t dtype, const Plans& plan,
                     void* stream) {
  return dtype == RIP_BF16 ? run<RIP_BF16>(f, over_q, over_k, plan, stream)
                           : run<RIP_FP32>(f, over_q, over_k, plan, stream);
}

int32_t run_bias_grad(const WithBias<Backward>& f, int64_t parts, int32_t buckets, int32_t heads, int32_t dtype,
                      void* grad, int64_t ld, int32_t accumulate, void* stream) {
  void* args[] = {(void*)&f.bias_part, (void*)&f.map, &parts, &grad, &ld, &accumulate};
  return launch(dtype == RIP_BF16 ? (const void*)bias_kernel<RIP_BF16> : (const void*)bias_kernel<RIP_FP32>,
                dim3((uint32_t)buckets, (uint32_t)heads), dim3(256), args, 0, stream,
                "rip_attn_backward: bias");
}

}  // namespace attn
}  // namespace rip
