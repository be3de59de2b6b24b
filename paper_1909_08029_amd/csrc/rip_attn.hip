// Host side of attention: argument checks, workspaces and launches, and the small
// kernel that prepares a call (offsets put in order, the bias by distance).
#include "rip_attn.h"

namespace rip {
namespace attn {
namespace {

struct Prepare {
  const int32_t* offsets[2];
  int32_t tokens[2];
  int32_t* cleaned[2];  // or NULL
  int32_t n_seqs, cleans;
  float* lut;
  int32_t lut_size;
  Buckets map;
};

constexpr int kThreads = 1024;

// Workgroups 0 .. cleans-1 make the running maximum of a side's offsets; the others
// write a head's bias by distance.
__global__ __launch_bounds__(kThreads) void prepare_kernel(Prepare p) {
  if ((int)blockIdx.x < p.cleans) {
    __shared__ int tops[kThreads / 64];
    const int side = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int most = 0;
    for (int64_t base = 0; base <= p.n_seqs; base += kThreads) {
      const int64_t i = base + threadIdx.x;
      int c = i <= p.n_seqs ? min(max(p.offsets[side][i], 0), p.tokens[side]) : 0;
      for (int o = 1; o < 64; o *= 2) {
        const int up = __shfl_up(c, o);
        if (lane >= o) c = max(c, up);
      }
      __syncthreads();  // the last round's tops have been read
      if (lane == 63) tops[wave] = c;
      __syncthreads();
      for (int w = 0; w < wave; ++w) c = max(c, tops[w]);
      c = max(c, most);
      if (i <= p.n_seqs) p.cleaned[side][i] = c;
      for (int w = 0; w < kThreads / 64; ++w) most = max(most, tops[w]);
    }
    return;
  }
  const int head = blockIdx.x - p.cleans, first = p.map.n > 1 ? p.map.start[0] - 1 : 0;
  for (int i = threadIdx.x; i < p.lut_size; i += kThreads)
    p.lut[(int64_t)head * p.lut_size + i] = bias_at(p.map, first + i, head);
}

int64_t align16(int64_t bytes) { return ceil_div(bytes, 16) * 16; }

int lut_size(const rip_attn& a) {
  const int n = a.rel->n_intervals;
  return n > 1 ? a.rel->starts[n - 2] - a.rel->starts[0] + 2 : 1;
}

// Whether a launch before makes the bias by distance: where a workgroup would compare a
// lane's distances with more than 16 starts in all (8 of 37 tokens' case: 39.4 us, 44.3
// with the launches; 62 of 8192 tokens in 1024 workgroups: 330 us, 290 with them).
bool lut_before(const rip_attn& a) {
  return a.bias && ceil_div(lut_size(a) + 128, 256) * a.rel->n_intervals > 16;
}
Buckets map_of(const rip_attn& a) {
  Buckets m{};
  if (!a.bias) return m;
  m.table = a.bias, m.ld = a.ld_bias, m.bf16 = a.bias_dtype == RIP_BF16;
  m.n = a.rel->n_intervals;
  for (int b = 0; b < m.n; ++b) {
    m.row[b] = a.rel->rows[b];
    if (b) m.start[b - 1] = a.rel->starts[b - 1];
  }
  return m;
}

// What a call takes of its workspace, in bytes from its start.
struct Layout {
  int64_t cleaned[2] = {-1, -1}, lut = -1, delta = -1, bias_part = -1, part = -1, end = 0;
  void take(int64_t& at, int64_t bytes) {
    at = end;
    end += align16(bytes);
  }
};

// One list for both sides is cut to each side's tokens.
bool two_sided(const rip_attn& a) {
  return a.k_offsets && (a.k_offsets != a.q_offsets || a.k_tokens != a.q_tokens);
}

Sizes sizes_of(const rip_attn& a) {
  return {a.q_tokens, a.k_tokens, a.n_sequences, a.heads, a.heads / a.kv_heads, a.head_dim,
          a.dtype == RIP_BF16, a.causal != 0, a.bias != nullptr, a.bias ? lut_size(a) : 0};
}

Layout layout_of(const rip_attn& a, const Plans& plan, bool backward) {
  Layout l;
  if (a.n_sequences > kScan)
    for (int s = 0; s < (two_sided(a) ? 2 : 1); ++s) l.take(l.cleaned[s], 4 * ((int64_t)a.n_sequences + 1));
  if (lut_before(a)) l.take(l.lut, 4 * (int64_t)a.heads * lut_size(a));
  const int64_t rows = (int64_t)a.heads * a.q_tokens;
  if (!backward) {
    if (plan.q.splits > 1) l.take(l.part, 4 * rows * plan.q.splits * (a.head_dim + 2));
    return l;
  }
  l.take(l.delta, 4 * rows);
  if (a.bias) l.take(l.bias_part, 4 * a.heads * plan.q.slots * plan.q.splits * a.rel->n_intervals);
  const int64_t dq = plan.q.splits > 1 ? plan.q.splits * rows * a.head_dim : 0;
  const int64_t dkv =
      plan.k.splits > 1 ? 2 * plan.k.splits * a.k_tokens * (int64_t)a.kv_heads * a.head_dim : 0;
  if (dq || dkv) l.take(l.part, 4 * (dq > dkv ? dq : dkv));
  return l;
}

int32_t check(const rip_attn* a, const char* name) {
  if (!a) return fail(RIP_E_INVAL, "%s: a is NULL", name);
  if (!known_dtype(a->dtype)) return fail(RIP_E_UNSUPPORTED, "%s: unknown dtype %d", name, a->dtype);
  if (a->heads < 1 || a->kv_heads < 1 || a->head_dim < 1 || a->heads % a->kv_heads || a->q_tokens < 0 ||
      a->k_tokens < 0 || a->n_sequences < 0)
    return fail(RIP_E_INVAL, "%s: %d heads (%d of k and v) of %d, %lld and %lld tokens, %d sequences",
                name, a->heads, a->kv_heads, a->head_dim, (long long)a->q_tokens, (long long)a->k_tokens,
                a->n_sequences);
  if (a->heads > RIP_MAX_HEADS || a->head_dim > RIP_MAX_HEAD_DIM || a->q_tokens > RIP_MAX_TOKENS ||
      a->k_tokens > RIP_MAX_TOKENS || a->n_sequences > RIP_MAX_SEQUENCES)
    return fail(RIP_E_UNSUPPORTED, "%s: %d heads of %d, %lld and %lld tokens, %d sequences are above the limit",
                name, a->heads, a->head_dim, (long long)a->q_tokens, (long long)a->k_tokens, a->n_sequences);
  if (!(a->scale > 0.0f) || !__builtin_isfinite(a->scale) || !__builtin_isfinite(a->scale * 1.44269504f))
    return fail(RIP_E_INVAL, "%s: scale %g", name, (double)a->scale);
  if (!a->k_offsets && a->k_tokens != a->q_tokens)
    return fail(RIP_E_INVAL, "%s: %lld keys for %lld queries with the same offsets", name,
                (long long)a->k_tokens, (long long)a->q_tokens);
  if ((a->q_tokens || a->k_tokens) && !a->q_offsets)
    return fail(RIP_E_INVAL, "%s: q_offsets is NULL", name);
  if (reinterpret_cast<uintptr_t>(a->q_offsets) % 4 || reinterpret_cast<uintptr_t>(a->k_offsets) % 4)
    return fail(RIP_E_ALIGN, "%s: offsets are not 4-byte aligned", name);
  if (!a->bias) return RIP_OK;
  if (!a->rel || a->rel->n_intervals < 1 || !a->rel->rows || (a->rel->n_intervals > 1 && !a->rel->starts) ||
      a->buckets < 1)
    return fail(RIP_E_INVAL, "%s: a bias needs buckets, intervals and their rows", name);
  const int n = a->rel->n_intervals;
  if (n > RIP_MAX_INTERVALS || a->buckets > RIP_MAX_BUCKETS)
    return fail(RIP_E_UNSUPPORTED, "%s: %d intervals, %d buckets are above the limit", name, n, a->buckets);
  for (int b = 0; b < n; ++b)
    if (a->rel->rows[b] < 0 || a->rel->rows[b] >= a->buckets)
      return fail(RIP_E_INVAL, "%s: interval %d has row %d of %d", name, b, a->rel->rows[b], a->buckets);
  for (int b = 1; b < n - 1; ++b)
    if (a->rel->starts[b] <= a->rel->starts[b - 1])
      return fail(RIP_E_INVAL, "%s: the intervals' starts are not strictly ascending", name);
  // both bounds keep distances within 32 bits
  if (n > 1 && ((int64_t)a->rel->starts[n - 2] - a->rel->starts[0] + 2 > RIP_MAX_BIAS_SPAN ||
                a->rel->starts[0] < -(1 << 24) || a->rel->starts[0] > 1 << 24))
    return fail(RIP_E_UNSUPPORTED, "%s: starts from %d to %d are above the limit", name, a->rel->starts[0],
                a->rel->starts[n - 2]);
  return check_matrix(a->bias, "bias", a->bias_dtype, a->buckets, a->heads, a->ld_bias);
}

// A matrix of a call; the kernels count the elements of a tile's rows in 32 bits.
int32_t check_rows(const void* p, const char* what, int32_t dtype, int64_t rows, int64_t width, int64_t ld) {
  const int32_t rc = check_matrix(p, what, dtype, rows, width, ld);
  if (rc) return rc;
  if (rows > 1 && ld > RIP_MAX_WIDTH)
    return fail(RIP_E_UNSUPPORTED, "%s: row stride %lld is above the limit", what, (long long)ld);
  return RIP_OK;
}

// Workgroups are counted in 32 bits.
int32_t check_grid(const Plan& p, int64_t heads, const char* name) {
  if (p.slots * p.splits * heads >= (int64_t)1 << 31)
    return fail(RIP_E_UNSUPPORTED, "%s: %lld tiles of %lld heads are above the limit", name,
                (long long)(p.slots * p.splits), (long long)heads);
  return RIP_OK;
}

Args args_of(const rip_attn& a, const Plan& plan, const Layout& l, char* ws) {
  Args p{};
  p.q = {a.q_offsets, (int)a.q_tokens};
  p.k = {two_sided(a) ? a.k_offsets : a.q_offsets, (int)a.k_tokens};
  if (l.cleaned[0] >= 0) {
    p.q.offsets = (const int32_t*)(ws + l.cleaned[0]);
    p.k.offsets = l.cleaned[1] >= 0 ? (const int32_t*)(ws + l.cleaned[1]) : p.q.offsets;
    p.cleaned = 1;
  }
  p.n_seqs = a.n_sequences;
  p.heads = a.heads, p.group = a.heads / a.kv_heads, p.pack = plan.pack;
  p.dim = a.head_dim, p.causal = a.causal != 0;
  p.by_pack = FastDiv::make((uint32_t)plan.pack);
  p.scale = a.scale, p.scale2 = a.scale * 1.44269504f;
  p.splits = plan.splits, p.slots = (int)plan.slots;
  if (a.bias) {
    if (l.lut >= 0) p.lut = (const float*)(ws + l.lut);
    p.lut_size = lut_size(a);
    p.lut_first = a.rel->n_intervals > 1 ? a.rel->starts[0] - 1 : 0;
  }
  return p;
}

int32_t prepare(const rip_attn& a, const Layout& l, char* ws, void* stream) {
  Prepare p{};
  p.offsets[0] = a.q_offsets, p.offsets[1] = a.k_offsets;
  p.tokens[0] = (int)a.q_tokens, p.tokens[1] = (int)a.k_tokens;
  for (int s = 0; s < 2; ++s)
    if (l.cleaned[s] >= 0) p.cleaned[s] = (int32_t*)(ws + l.cleaned[s]), p.cleans = s + 1;
  p.n_seqs = a.n_sequences;
  if (l.lut >= 0) {
    p.lut = (float*)(ws + l.lut), p.lut_size = lut_size(a);
    p.map = map_of(a);
  }
  const int groups = p.cleans + (l.lut >= 0 ? a.heads : 0);
  if (!groups) return RIP_OK;
  void* args[] = {&p};
  return launch((const void*)prepare_kernel, dim3((uint32_t)groups), dim3(kThreads), args, 0, stream,
                "rip_attn: prepare");
}

int32_t check_workspace(const void* ws, int64_t bytes, int64_t need, const char* name) {
  if (need && (!ws || bytes < need))
    return fail(RIP_E_INVAL, "%s: workspace of %lld bytes, %lld needed", name, (long long)bytes,
                (long long)need);
  if (reinterpret_cast<uintptr_t>(ws) % 16)
    return fail(RIP_E_ALIGN, "%s: workspace = %p is not 16-byte aligned", name, ws);
  return RIP_OK;
}

Plans plans_of(const rip_attn& a, bool backward) {
  const Sizes s = sizes_of(a);
  return {backward ? plan_dq(s) : plan_forward(s), backward ? plan_dkv(s) : Plan{}};
}

// What every call reads besides its matrices.
void add_inputs(Buffers& b, const rip_attn& a) {
  b.in_place = false;
  const int64_t offsets = 4 * ((int64_t)a.n_sequences + 1);
  b.range(a.q_offsets, a.q_offsets ? offsets : 0, "q_offsets", false);
  if (two_sided(a)) b.range(a.k_offsets, offsets, "k_offsets", false);
  if (a.bias) b.matrix(a.bias, a.bias_dtype, a.buckets, a.heads, a.ld_bias, "bias", false);
}

}  // namespace
}  // namespace attn
}  // namespace rip

using namespace rip;
using namespace rip::attn;

extern "C" int64_t rip_attn_forward_workspace(const rip_attn* a) {
  if (check(a, "rip_attn_forward") != RIP_OK) return 0;
  return layout_of(*a, plans_of(*a, false), false).end;
}

extern "C" int32_t rip_attn_forward(const rip_attn* a, const void* q, int64_t ld_q, const void* k,
                                    int64_t ld_k, const void* v, int64_t ld_v, void* out,
                                    int64_t ld_out, float* lse, void* low, int64_t ld_low,
                                    void* workspace, int64_t workspace_bytes, void* stream) {
  const char* name = "rip_attn_forward";
  clear_error();
  int32_t rc = check(a, name);
  if (rc) return rc;
  const int64_t wide = (int64_t)a->heads * a->head_dim, narrow = (int64_t)a->kv_heads * a->head_dim;
  const int32_t t = a->dtype;
  if (t == RIP_FP32) low = nullptr;
  if ((rc = check_rows(q, "q", t, a->q_tokens, wide, ld_q)) ||
      (rc = check_rows(k, "k", t, a->k_tokens, narrow, ld_k)) ||
      (rc = check_rows(v, "v", t, a->k_tokens, narrow, ld_v)) ||
      (rc = check_rows(out, "out", t, a->q_tokens, wide, ld_out)) ||
      (low && (rc = check_rows(low, "low", t, a->q_tokens, wide, ld_low))))
    return rc;
  if (reinterpret_cast<uintptr_t>(lse) % 4)
    return fail(RIP_E_ALIGN, "%s: lse = %p is not 4-byte aligned", name, (const void*)lse);
  const Plans plan = plans_of(*a, false);
  const Layout l = layout_of(*a, plan, false);
  if ((rc = check_grid(plan.q, a->heads / plan.q.pack, name)) ||
      (rc = check_workspace(workspace, workspace_bytes, l.end, name)))
    return rc;
  Buffers b;
  add_inputs(b, *a);
  b.matrix(q, t, a->q_tokens, wide, ld_q, "q", false);
  b.matrix(k, t, a->k_tokens, narrow, ld_k, "k", false);
  b.matrix(v, t, a->k_tokens, narrow, ld_v, "v", false);
  b.matrix(out, t, a->q_tokens, wide, ld_out, "out", true);
  if (low) b.matrix(low, t, a->q_tokens, wide, ld_low, "low", true);
  if (lse) b.range(lse, 4 * a->q_tokens * a->heads, "lse", true);
  b.range(workspace, l.end, "workspace", true);
  if ((rc = b.check())) return rc;
  if (a->q_tokens == 0) return RIP_OK;
  char* ws = static_cast<char*>(workspace);
  if ((rc = prepare(*a, l, ws, stream))) return rc;
  WithBias<Forward> f{};
  f.map = map_of(*a);
  f.a = args_of(*a, plan.q, l, ws);
  f.q = {q, ld_q}, f.k = {k, ld_k}, f.v = {v, ld_v};
  f.out = {out, ld_out}, f.low = {low, ld_low};
  f.lse = lse;
  f.part = l.part >= 0 ? (float*)(ws + l.part) : nullptr;
  return run_forward(f, t, plan.q.width, plan.q.waves, stream);
}

extern "C" int64_t rip_attn_backward_workspace(const rip_attn* a) {
  if (check(a, "rip_attn_backward") != RIP_OK) return 0;
  return layout_of(*a, plans_of(*a, true), true).end;
}

extern "C" int32_t rip_attn_backward(const rip_attn* a, const void* q, int64_t ld_q, const void* k,
                                     int64_t ld_k, const void* v, int64_t ld_v, const void* out,
                                     int64_t ld_out, const float* lse, const void* low, int64_t ld_low,
                                     const void* dout, int64_t ld_dout, void* dq, int64_t ld_dq, void* dk,
                                     int64_t ld_dk, void* dv, int64_t ld_dv, void* dbias,
                                     int32_t dbias_dtype, int64_t ld_dbias, int32_t accumulate,
                                     void* workspace, int64_t workspace_bytes, void* stream) {
  const char* name = "rip_attn_backward";
  clear_error();
  int32_t rc = check(a, name);
  if (rc) return rc;
  const int64_t wide = (int64_t)a->heads * a->head_dim, narrow = (int64_t)a->kv_heads * a->head_dim;
  const int32_t t = a->dtype;
  if (t == RIP_FP32) low = nullptr;
  if ((rc = check_rows(q, "q", t, a->q_tokens, wide, ld_q)) ||
      (rc = check_rows(k, "k", t, a->k_tokens, narrow, ld_k)) ||
      (rc = check_rows(v, "v", t, a->k_tokens, narrow, ld_v)) ||
      (rc = check_rows(out, "out", t, a->q_tokens, wide, ld_out)) ||
      (rc = check_rows(dout, "dout", t, a->q_tokens, wide, ld_dout)) ||
      (low && (rc = check_rows(low, "low", t, a->q_tokens, wide, ld_low))) ||
      (rc = check_rows(dq, "dq", t, a->q_tokens, wide, ld_dq)) ||
      (rc = check_rows(dk, "dk", t, a->k_tokens, narrow, ld_dk)) ||
      (rc = check_rows(dv, "dv", t, a->k_tokens, narrow, ld_dv)))
    return rc;
  if (dbias && !a->bias) return fail(RIP_E_INVAL, "%s: dbias without a bias", name);
  if (dbias && (rc = check_matrix(dbias, "dbias", dbias_dtype, a->buckets, a->heads, ld_dbias))) return rc;
  if (a->q_tokens && !lse) return fail(RIP_E_INVAL, "%s: lse is NULL", name);
  if (reinterpret_cast<uintptr_t>(lse) % 4)
    return fail(RIP_E_ALIGN, "%s: lse = %p is not 4-byte aligned", name, (const void*)lse);
  const Plans plan = plans_of(*a, true);
  const Layout l = layout_of(*a, plan, true);
  if ((rc = check_grid(plan.q, a->heads / plan.q.pack, name)) ||
      (rc = check_grid(plan.k, a->kv_heads, name)) ||
      (rc = check_workspace(workspace, workspace_bytes, l.end, name)))
    return rc;
  Buffers b;
  add_inputs(b, *a);
  b.matrix(q, t, a->q_tokens, wide, ld_q, "q", false);
  b.matrix(k, t, a->k_tokens, narrow, ld_k, "k", false);
  b.matrix(v, t, a->k_tokens, narrow, ld_v, "v", false);
  b.matrix(out, t, a->q_tokens, wide, ld_out, "out", false);
  b.matrix(dout, t, a->q_tokens, wide, ld_dout, "dout", false);
  if (low) b.matrix(low, t, a->q_tokens, wide, ld_low, "low", false);
  if (lse) b.range(lse, 4 * a->q_tokens * a->heads, "lse", false);
  b.matrix(dq, t, a->q_tokens, wide, ld_dq, "dq", true);
  b.matrix(dk, t, a->k_tokens, narrow, ld_dk, "dk", true);
  b.matrix(dv, t, a->k_tokens, narrow, ld_dv, "dv", true);
  if (dbias) b.matrix(dbias, dbias_dtype, a->buckets, a->heads, ld_dbias, "dbias", true);
  b.range(workspace, l.end, "workspace", true);
  if ((rc = b.check())) return rc;
  WithBias<Backward> f{};
  f.map = map_of(*a);
  if (a->q_tokens == 0 && a->k_tokens == 0)
    return !dbias || accumulate
               ? RIP_OK
               : run_bias_grad(f, 0, a->buckets, a->heads, dbias_dtype, dbias, ld_dbias, 0, stream);
  char* ws = static_cast<char*>(workspace);
  if ((rc = prepare(*a, l, ws, stream))) return rc;
  f.q = {q, ld_q}, f.k = {k, ld_k}, f.v = {v, ld_v};
  f.out = {out, ld_out}, f.low = {low, ld_low}, f.dout = {dout, ld_dout};
  f.dq = {dq, ld_dq}, f.dk = {dk, ld_dk}, f.dv = {dv, ld_dv};
  f.lse = lse;
  f.delta = (float*)(ws + l.delta);
  f.part = l.part >= 0 ? (float*)(ws + l.part) : nullptr;
  if (a->bias) f.bias_part = (float*)(ws + l.bias_part);
  if ((rc = run_backward(f, args_of(*a, plan.q, l, ws), args_of(*a, plan.k, l, ws), t, plan, stream)) ||
      !dbias)
    return rc;
  return run_bias_grad(f, plan.q.slots * plan.q.splits, a->buckets, a->heads, dbias_dtype, dbias, ld_dbias,
                       accumulate, stream);
}
