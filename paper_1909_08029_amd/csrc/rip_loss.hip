// Losses over the vocabulary with the gradient of the logits (gfx950): a
// preference loss over pairs of sequences, and a clipped policy loss with a KL
// term.  With x a token's row of logits and y its target,
//
//   logp = x[y] - log sum_v e^x[v]
//   d logp / d x[v] = (v == y) - softmax(x)[v]
//
// and either loss gives each counted token one number, coef = d loss / d logp,
// so the gradient's row is coef * ((v == y) - softmax(x)[v]).
//
//   1. stats   a row's largest logit and the sum of e^(x - largest), in one pass
//              (each lane keeps a running pair); few rows are split over several
//              workgroups, whose pairs the next launch joins; beside them the
//              preference loss's offsets are put in order
//   2. pairs / tokens   log-probabilities, the loss and coef
//   3. grad    one pass over the logits, writing the gradient; rows that do not
//              count are written as zeros without being read
//
// Bound by memory: the preference loss reads the logits twice (coef needs the whole
// pair) and writes the gradient once, 8192 x 50257 bf16, two thirds of it counted:
// stats 91 us (549 MB, 6.0 TB/s), pairs 8, grad 276 (1372 MB, 5.0 TB/s).  The policy
// loss needs no more than the row, which one workgroup takes through all three
// steps: 8192 x 131072 bf16, three quarters counted, 722 us (3.76 GB, 5.2 TB/s).

#include "rip_ops_common.h"

namespace rip {
namespace {

constexpr int kWave = 64;
constexpr int kThreads = 256, kWaves = kThreads / kWave;
// A lane's unit of a row here is sixteen bytes, so that every access of a wave is
// one range whatever the type (fp32 units of 32 bytes, in two accesses of half
// lines: 829 rows of 73856 123 us, 97 so).
template <int DT>
constexpr int kUnit = DT == RIP_BF16 ? 8 : 4;  // elements
constexpr int kStep = kThreads * 8;            // columns of a workgroup that a row is split for
constexpr int kPairThreads = 1024;       // of a pair's workgroup
constexpr int kTotalThreads = 1024;      // of the launch that adds the tokens' losses
constexpr int kHold = 8;                 // units of a row that a lane of the policy loss's
                                         // one-launch form keeps in registers
constexpr float kLowest = -3.402823466e38f;

// A row's largest logit and sum of e^(x - top).  sum == 0 only where every
// logit is -inf (or there is none): then top is the lowest number.
struct Stat {
  float top, sum;
};
// e^x with a relative error of |x| 2^-24 (x is at most 0): its terms in a row's sum are
// e^x of the largest, so that error is at most 0.37 * 2^-24 of the largest for each.
__device__ __forceinline__ float exp_fast(float x) {
  return __builtin_amdgcn_exp2f(x * 1.44269502f);
}
__device__ __forceinline__ Stat join(Stat a, Stat b) {
  const float top = fmaxf(a.top, b.top);
  return {top, a.sum * exp_fast(a.top - top) + b.sum * exp_fast(b.top - top)};
}
template <int N>
__device__ __forceinline__ void add(Stat& s, const float (&f)[N]) {
  float top = s.top;
#pragma unroll
  for (int j = 0; j < N; ++j) top = fmaxf(top, f[j]);
  float sum = s.sum * exp_fast(s.top - top);
#pragma unroll
  for (int j = 0; j < N; ++j) sum += exp_fast(f[j] - top);
  s = {top, sum};
}
// The workgroup's joined pair, in every thread.
template <int WAVES = kWaves>
__device__ __forceinline__ Stat join_block(Stat s, Stat* shared) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) s = join(s, {__shfl_xor(s.top, o), __shfl_xor(s.sum, o)});
  if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = s;
  __syncthreads();
  Stat r = shared[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) r = join(r, shared[w]);
  return r;
}

struct Rows {
  int64_t n, ld;
  int vocab;
  int splits;   // workgroups of a row
  int columns;  // of a workgroup, a multiple of eight
  const void* targets;
  int wide;
};
__device__ __forceinline__ bool counts(const Rows& r, int64_t t, int64_t* target) {
  *target = load_id(r.targets, r.wide, t);
  return *target >= 0 && *target < r.vocab;
}

// A lane's unit as it lies in memory.
template <int DT>
struct Unit {
  u32x4_any a;
  __device__ __forceinline__ void load(const typename Elem<DT>::T* p) { a = *(const u32x4_any*)p; }
  __device__ __forceinline__ void get(float (&f)[kUnit<DT>]) const {
    if constexpr (DT == RIP_BF16) {
      Elem<RIP_BF16>::unpack8(a, f);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(a[j]);
    }
  }
};
template <int DT>
__device__ __forceinline__ void load_elems(const typename Elem<DT>::T* p, float (&f)[kUnit<DT>]) {
  Unit<DT> u;
  u.load(p);
  u.get(f);
}
template <int DT>
__device__ __forceinline__ void store_elems(typename Elem<DT>::T* p, const float (&f)[kUnit<DT>]) {
  if constexpr (DT == RIP_BF16) {
    Elem<RIP_BF16>::store8(p, f);
  } else {
    u32x4_any a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(f[j]);
    store_stream((u32x4_any*)p, a);
  }
}

// Columns [begin, end) of a row as a workgroup walks them: units that
// begin at sixteen-byte boundaries (rows of an odd vocabulary begin anywhere, and
// sixteen bytes across a boundary take twice as long: statistics of 5461 rows of
// 50257 bf16 150 us, 110 so), and fewer than a unit before and after them.
struct Walk {
  int begin, first, units, rest, end;  // units from `first` to `rest`
};
template <int DT>
__device__ __forceinline__ Walk walk(const typename Elem<DT>::T* row, int begin, int end) {
  const int off = (int)(-(uintptr_t)(row + begin) & 15) / (int)sizeof(typename Elem<DT>::T);
  Walk w;
  w.begin = begin;
  w.end = end;
  w.first = min(begin + off, end);
  w.units = (end - w.first) / kUnit<DT>;
  w.rest = w.first + w.units * kUnit<DT>;
  return w;
}
// The columns before the units (edge 0) or after them (edge 1), as a unit filled
// up with -inf.
template <int DT>
__device__ __forceinline__ void load_edge(const typename Elem<DT>::T* row, const Walk& w, int edge,
                                          float (&f)[kUnit<DT>]) {
  const int a = edge ? w.rest : w.begin, b = edge ? w.end : w.first;
#pragma unroll
  for (int j = 0; j < kUnit<DT>; ++j)
    f[j] = a + j < b ? Elem<DT>::load(row + a + j) : -__builtin_huge_valf();
}
template <int DT>
__device__ __forceinline__ void store_edge(typename Elem<DT>::T* row, const Walk& w, int edge,
                                           const float (&f)[kUnit<DT>]) {
  const int a = edge ? w.rest : w.begin, b = edge ? w.end : w.first;
#pragma unroll
  for (int j = 0; j < kUnit<DT>; ++j)
    if (a + j < b) Elem<DT>::store(row + a + j, f[j]);
}

// What the grad launch needs of a token: gradient[v] = scale * e^(x[v] - top),
// plus coef at the target.
struct Token {
  float top, scale, coef;
  int target;
};

// The preference loss's offsets as its pairs take them: within the tokens, and none
// below an earlier one, of whichever pair, so that no two sequences share a token.
// That needs all earlier offsets: one workgroup makes the running maximum, beside
// those that read the logits.
struct Cut {
  const int32_t* offsets;  // as the caller gave them
  int32_t* cut;
  int count;               // 0: no sequences
};
__device__ __forceinline__ void cut_offsets(const Cut& c, int64_t n) {
  constexpr int kEach = 8;  // consecutive offsets of a thread in a round
  __shared__ int32_t tops[2][kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int32_t before = 0;       // the maximum of the rounds before
  for (int i0 = 0, round = 0; i0 < c.count; i0 += kThreads * kEach, ++round) {
    const int i = i0 + (int)threadIdx.x * kEach;
    int32_t o[kEach], top = 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) o[u] = i + u < c.count ? c.offsets[i + u] : 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) top = o[u] = max(top, min(o[u], (int32_t)n));
    for (int s = 1; s < kWave; s <<= 1) {
      const int32_t up = __shfl_up(top, s);
      if (lane >= s) top = max(top, up);
    }
    int32_t mine = __shfl_up(top, 1);  // of the lanes below
    mine = lane ? max(mine, before) : before;
    if (lane == kWave - 1) tops[round % 2][wave] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) {
      const int32_t x = tops[round % 2][w];
      mine = w < wave ? max(mine, x) : mine;
      before = max(before, x);
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      if (i + u < c.count) c.cut[i + u] = max(o[u], mine);
  }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void stats_kernel(Rows r,
                                                         const typename Elem<DT>::T* logits,
                                                         Stat* stat, Token* token, float* logp,
                                                         Cut c) {
  __shared__ Stat shared[kWaves];
  const uint32_t first = c.count > 0;  // a workgroup before those of the rows
  if (blockIdx.x < first) {
    cut_offsets(c, r.n);
    return;
  }
  const uint32_t at = blockIdx.x - first;
  const int64_t t = at / r.splits;
  const int split = at - (uint32_t)t * r.splits;
  if (split == 0 && threadIdx.x == 0) {  // stands for tokens that do not count
    token[t] = {0.0f, 0.0f, 0.0f, -1};
    if (logp) logp[t] = 0.0f;
  }
  int64_t target;
  if (!counts(r, t, &target)) return;
  const int end = min(r.vocab, (split + 1) * r.columns);
  const typename Elem<DT>::T* row = logits + t * r.ld;
  const Walk w = walk<DT>(row, split * r.columns, end);
  const typename Elem<DT>::T* unit = row + w.first;
  Stat s{kLowest, 0.0f};
  int u = threadIdx.x;
  constexpr int kAhead = 32 / kUnit<DT>;
  for (; u + (kAhead - 1) * kThreads < w.units; u += kAhead * kThreads) {
    float f[kAhead][kUnit<DT>];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_elems<DT>(unit + (u + i * kThreads) * kUnit<DT>, f[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) add(s, f[i]);
  }
  float f[kUnit<DT>];
  for (; u < w.units; u += kThreads) {
    load_elems<DT>(unit + u * kUnit<DT>, f);
    add(s, f);
  }
  if (threadIdx.x < 2) {
    load_edge<DT>(row, w, threadIdx.x, f);
    add(s, f);
  }
  s = join_block(s, shared);
  if (threadIdx.x == 0) stat[at] = s;
}

// log-probability of a counted token's target; false where the row has no
// logit above -inf, which leaves the token out.
template <int DT>
__device__ __forceinline__ bool token_logp(const Rows& r, const typename Elem<DT>::T* logits,
                                           const Stat& s, int64_t t, int64_t target, float* logp) {
  if (s.sum == 0.0f) return false;
  *logp = Elem<DT>::load(logits + t * r.ld + target) - s.top - logf(s.sum);
  return true;
}
// A row's pair from those of its splits, by `lanes` consecutive lanes (a power of
// two); each of them gets it.
__device__ __forceinline__ Stat row_stat(const Rows& r, const Stat* stat, int64_t t, int lanes) {
  Stat s{kLowest, 0.0f};
  for (int i = threadIdx.x & (lanes - 1); i < r.splits; i += lanes) s = join(s, stat[t * r.splits + i]);
  for (int o = 1; o < lanes; o <<= 1) s = join(s, {__shfl_xor(s.top, o), __shfl_xor(s.sum, o)});
  return s;
}

template <int WAVES = kWaves>
__device__ __forceinline__ double sum_block(double x, double* shared) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) x += __shfl_xor(x, o);
  __syncthreads();
  if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = x;
  __syncthreads();
  double s = shared[0];
  for (int w = 1; w < WAVES; ++w) s += shared[w];
  return s;
}

__device__ __forceinline__ float log_sigmoid(float z) {
  return fminf(z, 0.0f) - log1pf(expf(-fabsf(z)));
}

// One workgroup a pair, `lanes` threads a token (they join its splits).  The sums
// over a sequence are held in 64 bits: they run to thousands while the loss
// depends on differences of a few.
template <int DT>
__global__ __launch_bounds__(kPairThreads) void pairs_kernel(
    Rows r, const typename Elem<DT>::T* logits, const Stat* stat, const int32_t* cut, int pairs,
    const float* ref, float beta, float smoothing, float grad_scale, int lanes, float* seq_logp,
    Token* token, float* logp, double* pair_loss) {
  __shared__ double shared[2][kPairThreads / kWave];
  const double refs[2] = {ref[2 * blockIdx.x], ref[2 * blockIdx.x + 1]};
  // the pair's tokens, no other pair's
  const int64_t at[3] = {cut[2 * blockIdx.x], cut[2 * blockIdx.x + 1], cut[2 * blockIdx.x + 2]};
  const bool lead = (threadIdx.x & (lanes - 1)) == 0;
  const int64_t begin = at[0] + threadIdx.x / lanes, round = kPairThreads / lanes;
  double chosen = 0.0, rejected = 0.0;
  Token mine = {0.0f, 0.0f, 0.0f, -1};  // of the first round, kept in registers
  for (int64_t t = begin; t < at[2]; t += round) {
    int64_t target;
    if (!counts(r, t, &target)) continue;
    const Stat s = row_stat(r, stat, t, lanes);
    float lp;
    if (!lead || !token_logp<DT>(r, logits, s, t, target, &lp)) continue;
    chosen += t < at[1] ? lp : 0.0f;
    rejected += t < at[1] ? 0.0f : lp;
    if (logp) logp[t] = lp;
    const Token k = {s.top, 1.0f / s.sum, 1.0f, (int)target};
    if (t == begin)
      mine = k;
    else
      token[t] = k;
  }
  double margin[2];
  for (int q = 0; q < 2; ++q) {
    const double all = sum_block<kPairThreads / kWave>(q ? rejected : chosen, shared[q]);
    margin[q] = all - refs[q];
    if (threadIdx.x == 0) seq_logp[2 * blockIdx.x + q] = (float)all;
  }
  const float z = (float)((double)beta * (margin[0] - margin[1]));
  const float good = expf(log_sigmoid(z)), bad = expf(log_sigmoid(-z));
  const float coef =
      grad_scale * beta / (float)pairs * (smoothing * good - (1.0f - smoothing) * bad);
  if (threadIdx.x == 0) {  // a term of weight 0 stays out, also where it is infinite
    double l = 0.0;
    if (smoothing < 1.0f) l -= (1.0 - smoothing) * log_sigmoid(z);
    if (smoothing > 0.0f) l -= (double)smoothing * log_sigmoid(-z);
    pair_loss[blockIdx.x] = l / pairs;
  }
  if (!lead) return;
  for (int64_t t = begin; t < at[2]; t += round) {
    Token k = t == begin ? mine : token[t];
    if (k.target < 0) continue;
    k.coef = t >= at[1] ? -coef : coef;
    k.scale *= -k.coef;
    token[t] = k;
  }
}

struct Policy {
  const float *old_logp, *advantage, *weight, *ref_logp;
  float low, high, kl, grad_scale;
};

// x * a where x may be a number that left fp32: nothing if a is 0, as for any
// number that did not.
__device__ __forceinline__ float times(float x, float a) {
  return a == 0.0f && __builtin_isinf(x) ? 0.0f : x * a;
}

// e^d - d - 1, given m = e^d - 1, within 2^-21 of it: near 0, where policies begin and
// the terms cancel, by its series (as m - d in fp32 it is 0 or off by percents
// below d = 1e-3).
__device__ __forceinline__ float exp_rest(float d, float m) {
  if (fabsf(d) < 0.5f) {  // the next term is below 2^-24 of the sum
    float s = 1.0f / 40320;
    s = __builtin_fmaf(s, d, 1.0f / 5040);
    s = __builtin_fmaf(s, d, 1.0f / 720);
    s = __builtin_fmaf(s, d, 1.0f / 120);
    s = __builtin_fmaf(s, d, 1.0f / 24);
    s = __builtin_fmaf(s, d, 1.0f / 6);
    return d * d * __builtin_fmaf(s, d, 0.5f);
  }
  return __builtin_isinf(m) ? m : m - d;
}

// A counted token's loss and its derivative by logp.  ratio * A is flat where
// the clipped value is the smaller one; a NaN stays on the other branch.  The ratio
// passes fp32 where logp - old_logp is above 88 (a low value in old_logp that marks
// tokens to be left out, say), which no weight or advantage of 0 may turn into NaN.  The KL
// term is added in 64 bits, as the batch is: it may be far smaller than the first.
__device__ __forceinline__ double policy_token(const Policy& p, int64_t t, int64_t n, float lp,
                                               float* coef) {
  const float a = p.advantage[t], w = p.weight ? p.weight[t] : 1.0f / (float)n;
  *coef = 0.0f;
  if (w == 0.0f) return 0.0;
  const float ratio = expf(lp - p.old_logp[t]);
  const float gain = times(ratio, a), bound = times(fminf(fmaxf(ratio, p.low), p.high), a);
  const bool flat = gain > bound;
  double loss = flat ? -bound : -gain;
  float slope = flat ? 0.0f : -gain;
  if (p.ref_logp) {
    const float d = p.ref_logp[t] - lp, m = expm1f(d);
    loss += (double)p.kl * exp_rest(d, m);
    slope -= p.kl * m;
  }
  *coef = times(w * slope, p.grad_scale);
  return w * loss;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void tokens_kernel(Rows r,
                                                          const typename Elem<DT>::T* logits,
                                                          const Stat* stat, Policy p, int lanes,
                                                          Token* token, float* logp,
                                                          double* part_loss) {
  __shared__ double shared[kWaves];
  const int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / lanes;
  double loss = 0.0;
  int64_t target;
  if (t < r.n && counts(r, t, &target)) {
    const Stat s = row_stat(r, stat, t, lanes);
    float lp;
    if ((threadIdx.x & (lanes - 1)) == 0 && token_logp<DT>(r, logits, s, t, target, &lp)) {
      float coef;
      loss = policy_token(p, t, r.n, lp, &coef);
      if (logp) logp[t] = lp;
      token[t] = {s.top, -coef / s.sum, coef, (int)target};
    }
  }
  loss = sum_block(loss, shared);
  if (threadIdx.x == 0) part_loss[blockIdx.x] = loss;
}

// The loss: the sum of `parts` numbers, by one workgroup.
template <int THREADS>
__device__ __forceinline__ void total_loss(const double* part, int parts, float* loss,
                                           double* shared) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += 8 * THREADS) {
    double v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = i + u * THREADS < parts ? part[i + u * THREADS] : 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += v[u];
  }
  sum = sum_block<THREADS / kWave>(sum, shared);
  if (threadIdx.x == 0) *loss = (float)sum;
}
__global__ __launch_bounds__(kTotalThreads) void total_kernel(const double* part, int parts,
                                                              float* loss) {
  __shared__ double shared[kTotalThreads / kWave];
  total_loss<kTotalThreads>(part, parts, loss, shared);
}

// Gradient of a unit from column c on.  The short exponential's error, |x|
// 2^-24, is far below what rounding to bf16 leaves.
template <int DT>
__device__ __forceinline__ void grad_unit(const Token& k, int c, float (&f)[kUnit<DT>]) {
#pragma unroll
  for (int j = 0; j < kUnit<DT>; ++j) {
    const float x = f[j] - k.top;
    f[j] = k.scale * (DT == RIP_BF16 ? exp_fast(x) : exp_acc(x));
  }
  const int hit = k.target - c;
  if (hit >= 0 && hit < kUnit<DT>) {
#pragma unroll
    for (int j = 0; j < kUnit<DT>; ++j)
      if (j == hit) f[j] += k.coef;
  }
}
// A part of a row's gradient by `threads` threads; zeros without a look at the
// logits where the token does not count.
template <int DT>
__device__ __forceinline__ void row_grad(const typename Elem<DT>::T* row, const Walk& w,
                                         const Token& k, typename Elem<DT>::T* out, int thread,
                                         int threads) {
  float f[kUnit<DT>] = {};
  if (k.coef == 0.0f) {
    for (int u = thread; u < w.units; u += threads) store_elems<DT>(out + w.first + u * kUnit<DT>, f);
    if (thread < 2) store_edge<DT>(out, w, thread, f);
    return;
  }
  for (int u = thread; u < w.units; u += threads) {
    const int c = w.first + u * kUnit<DT>;
    load_elems<DT>(row + c, f);
    grad_unit<DT>(k, c, f);
    store_elems<DT>(out + c, f);
  }
  if (thread < 2) {
    load_edge<DT>(row, w, thread, f);
    grad_unit<DT>(k, thread ? w.rest : w.begin, f);
    store_edge<DT>(out, w, thread, f);
  }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void grad_kernel(Rows r,
                                                        const typename Elem<DT>::T* logits,
                                                        const Token* token,
                                                        typename Elem<DT>::T* grad, int64_t ld_grad,
                                                        const double* part, int parts,
                                                        float* loss) {
  __shared__ double shared[kWaves];
  if (blockIdx.x == 0) total_loss<kThreads>(part, parts, loss, shared);
  // from the last row back: those that were read last are still in the caches
  const uint32_t from_end = gridDim.x - 1 - blockIdx.x;
  const int64_t t = from_end / r.splits;
  const int split = from_end - (uint32_t)t * r.splits;
  const int end = min(r.vocab, (split + 1) * r.columns);
  const typename Elem<DT>::T* row = logits + t * r.ld;
  row_grad<DT>(row, walk<DT>(row, split * r.columns, end), token[t], grad + t * ld_grad, threadIdx.x,
               kThreads);
}

// The policy loss of one token in one workgroup, gradient and all: coef needs
// nothing beyond the token's own row.  The first kHold units of a lane stay in
// registers between the two passes; the rest is read again, last first, mostly
// from the caches (8192 rows of 131072 bf16, neither with streaming stores: 1031 us in
// three launches, 780 so; 722 with them).
template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void policy_row_kernel(
    Rows r, const typename Elem<DT>::T* logits, Policy p, float* logp, double* part,
    typename Elem<DT>::T* grad, int64_t ld_grad) {
  __shared__ Stat shared[THREADS / kWave];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const typename Elem<DT>::T* row = logits + t * r.ld;
  const Walk w = walk<DT>(row, 0, r.vocab);
  const typename Elem<DT>::T* unit = row + w.first;
  float f[kUnit<DT>], edge[kUnit<DT>], lp = 0.0f, coef = 0.0f;
  Stat s{kLowest, 0.0f};
  int64_t target;
  double loss = 0.0;
  Unit<DT> held[kHold];
  if (counts(r, t, &target)) {
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (tid + i * THREADS < w.units) held[i].load(unit + (tid + i * THREADS) * kUnit<DT>);
    if (tid < 2) load_edge<DT>(row, w, tid, edge);
    const float hit = Elem<DT>::load(row + target);
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (tid + i * THREADS < w.units) {
        held[i].get(f);
        add(s, f);
      }
    if (tid < 2) add(s, edge);
    int u = tid + kHold * THREADS;
    for (; u + 3 * THREADS < w.units; u += 4 * THREADS) {
      Unit<DT> next[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) next[i].load(unit + (u + i * THREADS) * kUnit<DT>);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        next[i].get(f);
        add(s, f);
      }
    }
    for (; u < w.units; u += THREADS) {
      load_elems<DT>(unit + u * kUnit<DT>, f);
      add(s, f);
    }
    s = join_block<THREADS / kWave>(s, shared);
    if (s.sum != 0.0f) {
      lp = hit - s.top - logf(s.sum);
      loss = policy_token(p, t, r.n, lp, &coef);
    }
  }
  if (tid == 0) {
    part[t] = loss;
    if (logp) logp[t] = lp;
  }
  if (!grad) return;
  typename Elem<DT>::T* out = grad + t * ld_grad;
  const Token k = {s.top, -coef / s.sum, coef, (int)target};
  if (coef == 0.0f) {
    row_grad<DT>(row, w, k, out, tid, THREADS);
    return;
  }
  // in place: each lane overwrites what it alone reads, but for the target's
  // logit, which every lane has read before the join
  if (w.units > tid)
    for (int u = tid + (w.units - 1 - tid) / THREADS * THREADS; u >= tid + kHold * THREADS; u -= THREADS) {
      const int c = w.first + u * kUnit<DT>;
      load_elems<DT>(row + c, f);
      grad_unit<DT>(k, c, f);
      store_elems<DT>(out + c, f);
    }
#pragma unroll
  for (int i = kHold - 1; i >= 0; --i)
    if (tid + i * THREADS < w.units) {
      const int c = w.first + (tid + i * THREADS) * kUnit<DT>;
      held[i].get(f);
      grad_unit<DT>(k, c, f);
      store_elems<DT>(out + c, f);
    }
  if (tid < 2) {
    grad_unit<DT>(k, tid ? w.rest : w.begin, edge);
    store_edge<DT>(out, w, tid, edge);
  }
}

// Workgroups of a row: enough to fill the card where there are few rows, each
// with a round of its threads at least.
Rows make_rows(int64_t n, int64_t vocab, int64_t ld, const void* targets, int32_t id_type) {
  Rows r{n, ld, (int)vocab, 1, 0, targets, id_type == RIP_INT64};
  const int64_t most = ceil_div(vocab, kStep);
  int64_t splits = n > 0 ? 2048 / n : 1;
  splits = splits < 1 ? 1 : splits > most ? most : splits;
  r.columns = (int)(ceil_div(ceil_div(vocab, splits), kLane) * kLane);
  r.splits = (int)ceil_div(vocab, r.columns);
  return r;
}

struct Work {
  Stat* stat;
  Token* token;
  double* part;
  int32_t* cut;
  int64_t bytes;
};
Work make_work(const Rows& r, int64_t parts, int64_t offsets, void* workspace) {
  char* p = static_cast<char*>(workspace);
  Work w{};
  w.stat = (Stat*)p;
  int64_t at = ceil_div(r.n * r.splits * (int64_t)sizeof(Stat), 256) * 256;
  w.token = (Token*)(p + at);
  at += ceil_div(r.n * (int64_t)sizeof(Token), 256) * 256;
  w.part = (double*)(p + at);
  at += (parts + 1) * (int64_t)sizeof(double);
  w.cut = (int32_t*)(p + at);
  w.bytes = at + offsets * (int64_t)sizeof(int32_t);
  return w;
}
// Threads that join the splits of a row.
int join_lanes(const Rows& r) {
  int lanes = 1;
  while (lanes < r.splits && lanes < kWave) lanes *= 2;
  return lanes;
}
// The policy loss takes its one-launch form where the rows fill the card or are
// short: a workgroup a row, of one wave, four or eight, so that a lane has a few
// units of a short row to itself.
// (2^22 rows and more would leave a launch's grid.)
bool one_launch(const Rows& r) {
  return r.n < 1 << 22 && (r.n >= 512 || (r.n > 0 && r.vocab <= 1 << 14));
}
template <int DT>
const void* row_kernel(const Rows& r, int* threads) {
  *threads = r.vocab <= 1 << 11 ? 64 : r.vocab <= 1 << 14 ? 256 : 512;
  return *threads == 64    ? (const void*)policy_row_kernel<DT, 64>
         : *threads == 256 ? (const void*)policy_row_kernel<DT, 256>
                           : (const void*)policy_row_kernel<DT, 512>;
}
int64_t policy_parts(const Rows& r) { return one_launch(r) ? r.n : ceil_div(r.n * join_lanes(r), kThreads); }

// An array of 32-bit numbers that a loss reads or writes; NULL where it has none.
struct Small {
  const void* p;
  int64_t count;
  const char* what;
  bool written;
};
template <int SMALL>
int32_t check_loss(const char* name, const void* logits, int32_t dtype, int64_t ld, int64_t n,
                   int64_t vocab, const void* targets, int32_t id_type, const void* loss,
                   const void* grad, int64_t ld_grad, const void* workspace,
                   int64_t workspace_bytes, int64_t need, const Small (&small)[SMALL]) {
  int32_t rc;
  if (vocab < 1) return fail(RIP_E_INVAL, "%s: vocab %lld < 1", name, (long long)vocab);
  if (vocab > RIP_MAX_WIDTH || n > RIP_MAX_TOKENS)
    return fail(RIP_E_UNSUPPORTED, "%s: %lld tokens of vocabulary %lld are above the limit", name,
                (long long)n, (long long)vocab);
  if ((rc = check_matrix(logits, "logits", dtype, n, vocab, ld))) return rc;
  if (grad && (rc = check_matrix(grad, "grad", dtype, n, vocab, ld_grad))) return rc;
  if (id_type != RIP_INT32 && id_type != RIP_INT64)
    return fail(RIP_E_UNSUPPORTED, "%s: unknown id type %d", name, id_type);
  const int id_bytes = id_type == RIP_INT64 ? 8 : 4;
  if (n && !targets) return fail(RIP_E_INVAL, "%s: targets is NULL", name);
  if (reinterpret_cast<uintptr_t>(targets) % id_bytes)
    return fail(RIP_E_ALIGN, "%s: targets = %p is not aligned to its type", name, targets);
  if (!loss) return fail(RIP_E_INVAL, "%s: loss is NULL", name);
  if (!workspace || workspace_bytes < need)
    return fail(RIP_E_INVAL, "%s: workspace of %lld bytes, %lld needed", name,
                (long long)workspace_bytes, (long long)need);
  if (reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(RIP_E_ALIGN, "%s: workspace = %p is not 16-byte aligned", name, workspace);
  for (const Small& s : small)
    if (reinterpret_cast<uintptr_t>(s.p) % 4)
      return fail(RIP_E_ALIGN, "%s: %s = %p is not 4-byte aligned", name, s.what, s.p);
  // the gradient may be the logits' own matrix
  const bool in_place = grad && grad == logits && ld_grad == ld;
  Range list[4 + SMALL] = {
      {logits, span(dtype, n, vocab, ld), "logits", in_place},
      {grad, grad && !in_place ? span(dtype, n, vocab, ld_grad) : 0, "grad", true},
      {targets, n * id_bytes, "targets", false},
      {workspace, need, "workspace", true}};
  for (int i = 0; i < SMALL; ++i)
    list[4 + i] = {small[i].p, small[i].p ? small[i].count * 4 : 0, small[i].what, small[i].written};
  return check_apart(name, list, 4 + SMALL);
}

template <int DT>
int32_t run_stats(Rows& r, const void* logits, Work& w, float* logp, Cut c, void* stream) {
  const int64_t groups = r.n * r.splits + (c.count > 0);
  if (groups == 0) return RIP_OK;
  void* args[] = {&r, &logits, &w.stat, &w.token, &logp, &c};
  return launch((const void*)stats_kernel<DT>, dim3((uint32_t)groups), dim3(kThreads), args, 0,
                stream, "loss: stats");
}
template <int DT>
int32_t run_grad(Rows& r, const void* logits, Work& w, void* grad, int64_t ld_grad, int parts,
                 float* loss, void* stream) {
  if (!grad || r.n == 0) {
    void* args[] = {&w.part, &parts, &loss};
    return launch((const void*)total_kernel, dim3(1), dim3(kTotalThreads), args, 0, stream,
                  "loss: total");
  }
  void* args[] = {&r, &logits, &w.token, &grad, &ld_grad, &w.part, &parts, &loss};
  return launch((const void*)grad_kernel<DT>, dim3((uint32_t)(r.n * r.splits)), dim3(kThreads),
                args, 0, stream, "loss: grad");
}

template <int DT>
int32_t run_pref(Rows r, const void* logits, const int32_t* offsets, int pairs, const float* ref,
                 float beta, float smoothing, float grad_scale, float* loss, float* seq_logp,
                 float* logp, void* grad, int64_t ld_grad, void* workspace, void* stream) {
  Work w = make_work(r, pairs, 2 * (int64_t)pairs + 1, workspace);
  int32_t rc;
  if ((rc = run_stats<DT>(r, logits, w, logp, Cut{offsets, w.cut, 2 * pairs + 1}, stream))) return rc;
  int lanes = join_lanes(r);
  void* args[] = {&r,          &logits, &w.stat,   &w.cut,   &pairs, &ref,   &beta, &smoothing,
                  &grad_scale, &lanes,  &seq_logp, &w.token, &logp,  &w.part};
  if ((rc = launch((const void*)pairs_kernel<DT>, dim3((uint32_t)pairs), dim3(kPairThreads), args, 0,
                   stream, "rip_pref_loss: pairs")))
    return rc;
  return run_grad<DT>(r, logits, w, grad, ld_grad, pairs, loss, stream);
}

template <int DT>
int32_t run_policy(Rows r, const void* logits, Policy p, float* loss, float* logp, void* grad,
                   int64_t ld_grad, void* workspace, void* stream) {
  int parts = (int)policy_parts(r);
  Work w = make_work(r, parts, 0, workspace);
  int32_t rc;
  if (one_launch(r)) {
    void* args[] = {&r, &logits, &p, &logp, &w.part, &grad, &ld_grad};
    int threads;
    const void* fn = row_kernel<DT>(r, &threads);
    if ((rc = launch(fn, dim3((uint32_t)r.n), dim3(threads), args, 0, stream,
                     "rip_policy_loss: rows")))
      return rc;
    void* total[] = {&w.part, &parts, &loss};
    return launch((const void*)total_kernel, dim3(1), dim3(kTotalThreads), total, 0, stream,
                  "rip_policy_loss: total");
  }
  if ((rc = run_stats<DT>(r, logits, w, logp, Cut{}, stream))) return rc;
  if (r.n) {
    int lanes = join_lanes(r);
    void* args[] = {&r, &logits, &w.stat, &p, &lanes, &w.token, &logp, &w.part};
    if ((rc = launch((const void*)tokens_kernel<DT>, dim3((uint32_t)parts), dim3(kThreads), args, 0,
                     stream, "rip_policy_loss: tokens")))
      return rc;
  }
  return run_grad<DT>(r, logits, w, grad, ld_grad, parts, loss, stream);
}

}  // namespace
}  // namespace rip

using namespace rip;

extern "C" int64_t rip_pref_loss_workspace(int64_t n_tokens, int64_t vocab, int32_t n_pairs) {
  if (n_tokens < 0 || n_tokens > RIP_MAX_TOKENS || vocab < 1 || vocab > RIP_MAX_WIDTH ||
      n_pairs < 0 || n_pairs > RIP_MAX_PAIRS)
    return 0;
  return make_work(make_rows(n_tokens, vocab, vocab, nullptr, 0), n_pairs, 2 * (int64_t)n_pairs + 1,
                   nullptr)
      .bytes;
}
extern "C" int64_t rip_policy_loss_workspace(int64_t n_tokens, int64_t vocab) {
  if (n_tokens < 0 || n_tokens > RIP_MAX_TOKENS || vocab < 1 || vocab > RIP_MAX_WIDTH) return 0;
  const Rows r = make_rows(n_tokens, vocab, vocab, nullptr, 0);
  return make_work(r, policy_parts(r), 0, nullptr).bytes;
}

extern "C" int32_t rip_pref_loss(const void* logits, int32_t dtype, int64_t ld, int64_t n_tokens,
                                 int64_t vocab, const void* targets, int32_t id_type,
                                 const int32_t* seq_offsets, int32_t n_pairs,
                                 const float* ref_logp, float beta, float smoothing,
                                 float grad_scale, float* loss, float* seq_logp, float* logp,
                                 void* grad, int64_t ld_grad, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
  clear_error();
  if (n_pairs < 1) return fail(RIP_E_INVAL, "rip_pref_loss: n_pairs %d < 1", n_pairs);
  if (n_pairs > RIP_MAX_PAIRS)
    return fail(RIP_E_UNSUPPORTED, "rip_pref_loss: n_pairs %d > %d", n_pairs, RIP_MAX_PAIRS);
  int32_t rc;
  if ((rc = check_loss("rip_pref_loss", logits, dtype, ld, n_tokens, vocab, targets, id_type, loss,
                       grad, ld_grad, workspace, workspace_bytes,
                       rip_pref_loss_workspace(n_tokens, vocab, n_pairs),
                       {{seq_offsets, 2 * (int64_t)n_pairs + 1, "seq_offsets", false},
                        {ref_logp, 2 * (int64_t)n_pairs, "ref_logp", false},
                        {loss, 1, "loss", true},
                        {seq_logp, 2 * (int64_t)n_pairs, "seq_logp", true},
                        {logp, n_tokens, "logp", true}})))
    return rc;
  if (!seq_offsets || !ref_logp || !seq_logp)
    return fail(RIP_E_INVAL, "rip_pref_loss: seq_offsets, ref_logp or seq_logp is NULL");
  if (!(smoothing >= 0.0f && smoothing <= 1.0f))
    return fail(RIP_E_INVAL, "rip_pref_loss: smoothing %g is not in 0..1", (double)smoothing);
  if (!(beta == beta) || !(grad_scale == grad_scale))
    return fail(RIP_E_INVAL, "rip_pref_loss: beta or grad_scale is NaN");
  Rows r = make_rows(n_tokens, vocab, ld, targets, id_type);
  return dtype == RIP_FP32
             ? run_pref<RIP_FP32>(r, logits, seq_offsets, n_pairs, ref_logp, beta, smoothing,
                                  grad_scale, loss, seq_logp, logp, grad, ld_grad, workspace, stream)
             : run_pref<RIP_BF16>(r, logits, seq_offsets, n_pairs, ref_logp, beta, smoothing,
                                  grad_scale, loss, seq_logp, logp, grad, ld_grad, workspace,
                                  stream);
}

extern "C" int32_t rip_policy_loss(const void* logits, int32_t dtype, int64_t ld, int64_t n_tokens,
                                   int64_t vocab, const void* targets, int32_t id_type,
                                   const float* old_logp, const float* advantage,
                                   const float* weight, const float* ref_logp, float clip_low,
                                   float clip_high, float kl, float grad_scale, float* loss,
                                   float* logp, void* grad, int64_t ld_grad, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  clear_error();
  int32_t rc;
  if (n_tokens < 0) return fail(RIP_E_INVAL, "rip_policy_loss: n_tokens %lld < 0", (long long)n_tokens);
  if ((rc = check_loss("rip_policy_loss", logits, dtype, ld, n_tokens, vocab, targets, id_type,
                       loss, grad, ld_grad, workspace, workspace_bytes,
                       rip_policy_loss_workspace(n_tokens, vocab),
                       {{old_logp, n_tokens, "old_logp", false},
                        {advantage, n_tokens, "advantage", false},
                        {weight, n_tokens, "weight", false},
                        {ref_logp, n_tokens, "ref_logp", false},
                        {loss, 1, "loss", true},
                        {logp, n_tokens, "logp", true}})))
    return rc;
  if (n_tokens && (!old_logp || !advantage))
    return fail(RIP_E_INVAL, "rip_policy_loss: old_logp or advantage is NULL");
  if (kl != 0.0f && n_tokens && !ref_logp)
    return fail(RIP_E_INVAL, "rip_policy_loss: a KL term needs ref_logp");
  if (!(clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f))
    return fail(RIP_E_INVAL, "rip_policy_loss: clip_low %g is not in 0..1 or clip_high %g < 0",
                (double)clip_low, (double)clip_high);
  if (!(kl == kl) || !(grad_scale == grad_scale))
    return fail(RIP_E_INVAL, "rip_policy_loss: kl or grad_scale is NaN");
  Rows r = make_rows(n_tokens, vocab, ld, targets, id_type);
  Policy p{old_logp,         advantage,         weight, kl != 0.0f ? ref_logp : nullptr,
           1.0f - clip_low, 1.0f + clip_high, kl,     grad_scale};
  return dtype == RIP_FP32 ? run_policy<RIP_FP32>(r, logits, p, loss, logp, grad, ld_grad, workspace, stream)
                           : run_policy<RIP_BF16>(r, logits, p, loss, logp, grad, ld_grad, workspace, stream);
}
