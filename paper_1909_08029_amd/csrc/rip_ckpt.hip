// Activations kept as 8-bit checkpoints, and the gated unit that uses them
// (gfx950).
//
//   pack, unpack   x -> (codes, exponents) -> x'
//   forward        h = silu(gate) * up, gate and up packed in the same pass
//   backward       from gate' and up' as the checkpoints hold them,
//                  s = 1 / (1 + e^-gate'):
//                  dgate = dh * up' * s * (1 + gate' * (1 - s))
//                  dup   = dh * gate' * s
//                  and, if asked for, h' = gate' * s * up' packed anew: the
//                  checkpoint of the next layer's input, which need not be kept
//
// Each is one pass over its data, bound by memory.  A lane handles sixteen bytes of
// a row, eight columns of bf16 or four of fp32, so that every access of a wave is
// one range (fp32 with eight columns a lane: 116 us for the backward pass of 8192 x
// 5504, 94 so), and four or eight lanes a block, whose largest magnitude takes
// two or three exchanges between them.  The codes of a row fill whole blocks
// (zeros past the last column), so they are always stored and read whole.  16384 x 5504
// bf16: pack 44 us (6.2 TB/s), unpack 40, forward 112 (734 MB, 6.6 TB/s), backward
// 109; a width of 5503, whose rows begin anywhere, takes 1.1 to 1.25 times that.

#include "rip_ckpt_format.h"

namespace rip {
namespace {

constexpr int kBlockThreads = 256;

template <int DT>
constexpr int kCols = DT == RIP_BF16 ? 8 : 4;  // columns of a lane
template <int DT>
constexpr int kLanes = kCkptBlock / kCols<DT>;  // lanes of a block

// A matrix's blocks as the kernels index them: a lane each for its units.
struct Shape {
  uint32_t units;
  FastDiv per_row;
  int width;
  uint32_t blocks;  // of all rows
};

// Columns c .. c + kCols - 1 of a row; zero past its end, nothing read there.
template <int DT, bool STREAM = false>
__device__ __forceinline__ void load_cols(const typename Elem<DT>::T* row, int c, int width,
                                          float (&f)[kCols<DT>]) {
  if constexpr (DT == RIP_BF16) {
    load_unit<DT, STREAM>(row, c, width, f);
  } else if (c + 4 <= width) {
    const u32x4 a = STREAM ? load_stream((const u32x4_any*)(row + c)) : *(const u32x4_any*)(row + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(a[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = c + j < width ? row[c + j] : 0.0f;
  }
}
template <int DT>
__device__ __forceinline__ void store_cols(typename Elem<DT>::T* row, int c, int width,
                                           const float (&f)[kCols<DT>]) {
  if constexpr (DT == RIP_BF16) {
    store_unit<DT>(row, c, width, f);
  } else if (c + 4 <= width) {
    u32x4_any a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = __float_as_uint(f[j]);
    store_stream((u32x4_any*)(row + c), a);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < width) row[c + j] = f[j];
  }
}

struct Ckpt {
  int8_t* codes;
  uint8_t* exps;
};

struct Place {
  int64_t row;
  int col;     // first column of the lane
  int64_t code;  // byte offset of its codes
  int64_t exp;   // index of its block's exponent
  bool lead;   // first lane of the block
};
template <int DT>
__device__ __forceinline__ Place place(const Shape& s, uint32_t unit) {
  Place p;
  const uint32_t row = s.per_row.div(unit), in = unit - row * s.per_row.d;
  p.row = row;
  p.col = (int)in * kCols<DT>;
  p.code = (int64_t)unit * kCols<DT>;
  p.exp = unit / kLanes<DT>;
  p.lead = in % kLanes<DT> == 0;
  return p;
}

template <int DT>
__device__ __forceinline__ void store_ckpt(const Ckpt& c, const Place& p,
                                           const float (&x)[kCols<DT>]) {
  uint32_t codes[kCols<DT> / 4];
  const uint32_t e = ckpt_pack<kCols<DT>>(x, codes);
  if constexpr (DT == RIP_BF16)
    *(uint2*)(c.codes + p.code) = make_uint2(codes[0], codes[1]);
  else
    *(uint32_t*)(c.codes + p.code) = codes[0];
  if (p.lead) c.exps[p.exp] = (uint8_t)e;
}
template <int DT>
__device__ __forceinline__ void load_ckpt(const Ckpt& c, const Place& p, float (&x)[kCols<DT>]) {
  uint32_t codes[kCols<DT> / 4];
  if constexpr (DT == RIP_BF16) {
    const uint2 v = *(const uint2*)(c.codes + p.code);
    codes[0] = v.x, codes[1] = v.y;
  } else {
    codes[0] = *(const uint32_t*)(c.codes + p.code);
  }
  ckpt_unpack<kCols<DT>>(codes, c.exps[p.exp], x);
}

// 1 / (1 + e^-x), from e^-|x|, which neither overflows nor loses the small
// results; one step of Newton's method after the hardware's reciprocal.
__device__ __forceinline__ float sigmoid(float x) {
  const float e = exp_acc(-fabsf(x)), d = 1.0f + e;
  const float r = __builtin_amdgcn_rcpf(d);
  const float y = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
  return x < 0.0f ? e * y : y;
}

// The lanes of a block take every branch together: units are whole blocks, and so
// are the lanes past them.
template <int DT>
__global__ __launch_bounds__(kBlockThreads) void pack_kernel(Shape s, const typename Elem<DT>::T* x,
                                                             int64_t ld, Ckpt out) {
  const uint32_t unit = blockIdx.x * kBlockThreads + threadIdx.x;
  if (unit >= s.units) return;
  const Place p = place<DT>(s, unit);
  float f[kCols<DT>];
  load_cols<DT>(x + p.row * ld, p.col, s.width, f);
  store_ckpt<DT>(out, p, f);
}

template <int DT>
__global__ __launch_bounds__(kBlockThreads) void unpack_kernel(Shape s, Ckpt in,
                                                               typename Elem<DT>::T* x,
                                                               int64_t ld) {
  const uint32_t unit = blockIdx.x * kBlockThreads + threadIdx.x;
  if (unit >= s.units) return;
  const Place p = place<DT>(s, unit);
  float f[kCols<DT>];
  load_ckpt<DT>(in, p, f);
  store_cols<DT>(x + p.row * ld, p.col, s.width, f);
}

// STREAM: the inputs are read past the caches.
template <int DT, bool STREAM>
__global__ __launch_bounds__(kBlockThreads) void gate_forward_kernel(
    Shape s, const typename Elem<DT>::T* gate, int64_t ld_gate, const typename Elem<DT>::T* up,
    int64_t ld_up, typename Elem<DT>::T* h, int64_t ld_h, Ckpt gate8, Ckpt up8) {
  const uint32_t unit = blockIdx.x * kBlockThreads + threadIdx.x;
  if (unit >= s.units) return;
  const Place p = place<DT>(s, unit);
  float g[kCols<DT>], u[kCols<DT>];
  load_cols<DT, STREAM>(gate + p.row * ld_gate, p.col, s.width, g);
  load_cols<DT, STREAM>(up + p.row * ld_up, p.col, s.width, u);
  store_ckpt<DT>(gate8, p, g);
  store_ckpt<DT>(up8, p, u);
#pragma unroll
  for (int j = 0; j < kCols<DT>; ++j) g[j] = g[j] * sigmoid(g[j]) * u[j];
  store_cols<DT>(h + p.row * ld_h, p.col, s.width, g);
}

template <int DT, bool AGAIN, bool STREAM>
__global__ __launch_bounds__(kBlockThreads) void gate_backward_kernel(
    Shape s, const typename Elem<DT>::T* dh, int64_t ld_dh, Ckpt gate8, Ckpt up8,
    typename Elem<DT>::T* dgate, int64_t ld_dgate, typename Elem<DT>::T* dup, int64_t ld_dup,
    Ckpt h8) {
  const uint32_t unit = blockIdx.x * kBlockThreads + threadIdx.x;
  if (unit >= s.units) return;
  const Place p = place<DT>(s, unit);
  float d[kCols<DT>], g[kCols<DT>], u[kCols<DT>];
  load_cols<DT, STREAM>(dh + p.row * ld_dh, p.col, s.width, d);
  load_ckpt<DT>(gate8, p, g);
  load_ckpt<DT>(up8, p, u);
  float a[kCols<DT>], h[kCols<DT>];
#pragma unroll
  for (int j = 0; j < kCols<DT>; ++j) {
    const float sg = sigmoid(g[j]);
    const float silu = g[j] * sg;
    // dh and up' meet last: their product alone may pass fp32 where dgate does not
    a[j] = d[j] * (sg * (1.0f + g[j] * (1.0f - sg))) * u[j];
    h[j] = silu * u[j];
    d[j] *= silu;
  }
  store_cols<DT>(dgate + p.row * ld_dgate, p.col, s.width, a);
  store_cols<DT>(dup + p.row * ld_dup, p.col, s.width, d);
  if (AGAIN) store_ckpt<DT>(h8, p, h);
}

int32_t make_shape(int32_t dtype, int64_t rows, int64_t width, Shape* out) {
  if (!known_dtype(dtype)) return fail(RIP_E_UNSUPPORTED, "unknown dtype %d", dtype);
  if (rows < 0 || width < 1)
    return fail(RIP_E_INVAL, "%lld rows of width %lld", (long long)rows, (long long)width);
  const int64_t blocks = ceil_div(width, kCkptBlock);
  const int lanes = dtype == RIP_BF16 ? kLanes<RIP_BF16> : kLanes<RIP_FP32>;
  if (rows > RIP_MAX_TOKENS || width > RIP_MAX_WIDTH ||
      rows * blocks * kLanes<RIP_FP32> >= (int64_t)1 << 31)
    return fail(RIP_E_UNSUPPORTED, "%lld rows of width %lld are above the limit", (long long)rows,
                (long long)width);
  out->units = (uint32_t)(rows * blocks * lanes);
  out->per_row = FastDiv::make((uint32_t)(blocks * lanes));
  out->width = (int)width;
  out->blocks = (uint32_t)(rows * blocks);
  return RIP_OK;
}

template <int DT>
const void* backward_of(bool again, bool past) {
  return again ? (past ? (const void*)gate_backward_kernel<DT, true, true>
                       : (const void*)gate_backward_kernel<DT, true, false>)
               : (past ? (const void*)gate_backward_kernel<DT, false, true>
                       : (const void*)gate_backward_kernel<DT, false, false>);
}

// Inputs that the memory-side cache cannot hold are read past it (16384 x 5504 bf16
// forward 113 us against 119, backward 107 against 117); smaller ones may lie in it
// from the launch that made them (8192 x 1024: 13 against 15 past it).
bool stream_inputs(int32_t dtype, int64_t rows, int64_t width, int inputs) {
  return rows * width * elem_bytes(dtype) * inputs > kCacheBytes;
}

int64_t code_bytes(const Shape& s) { return (int64_t)s.blocks * kCkptBlock; }
int64_t exp_bytes(const Shape& s) { return s.blocks; }

int32_t check_ckpt(const void* codes, const void* exps, const char* what, const Shape& s) {
  if (s.units && (!codes || !exps)) return fail(RIP_E_INVAL, "%s: codes or exps is NULL", what);
  if (reinterpret_cast<uintptr_t>(codes) % 16)
    return fail(RIP_E_ALIGN, "%s: codes = %p is not 16-byte aligned", what, codes);
  return RIP_OK;
}

int32_t run(const void* fn, const Shape& s, void** args, void* stream, const char* what) {
  if (s.units == 0) return RIP_OK;
  return launch(fn, dim3((uint32_t)ceil_div(s.units, kBlockThreads)), dim3(kBlockThreads), args, 0,
                stream, what);
}

}  // namespace
}  // namespace rip

using namespace rip;

extern "C" int32_t rip_ckpt_pack(const void* x, int32_t dtype, int64_t ld, int64_t rows,
                                 int64_t width, int8_t* codes, uint8_t* exps, void* stream) {
  clear_error();
  int32_t rc;
  Shape s;
  if ((rc = make_shape(dtype, rows, width, &s)) || (rc = check_matrix(x, "x", dtype, rows, width, ld)) ||
      (rc = check_ckpt(codes, exps, "out", s)))
    return rc;
  Buffers b;
  b.matrix(x, dtype, rows, width, ld, "x", false);
  b.range(codes, code_bytes(s), "codes", true);
  b.range(exps, exp_bytes(s), "exps", true);
  if ((rc = b.check())) return rc;
  Ckpt out{codes, exps};
  void* args[] = {&s, &x, &ld, &out};
  return run(dtype == RIP_FP32 ? (const void*)pack_kernel<RIP_FP32>
                               : (const void*)pack_kernel<RIP_BF16>,
             s, args, stream, "rip_ckpt_pack");
}

extern "C" int32_t rip_ckpt_unpack(const int8_t* codes, const uint8_t* exps, int64_t rows,
                                   int64_t width, void* x, int32_t dtype, int64_t ld,
                                   void* stream) {
  clear_error();
  int32_t rc;
  Shape s;
  if ((rc = make_shape(dtype, rows, width, &s)) || (rc = check_matrix(x, "x", dtype, rows, width, ld)) ||
      (rc = check_ckpt(codes, exps, "in", s)))
    return rc;
  Buffers b;
  b.matrix(x, dtype, rows, width, ld, "x", true);
  b.range(codes, code_bytes(s), "codes", false);
  b.range(exps, exp_bytes(s), "exps", false);
  if ((rc = b.check())) return rc;
  Ckpt in{const_cast<int8_t*>(codes), const_cast<uint8_t*>(exps)};
  void* args[] = {&s, &in, &x, &ld};
  return run(dtype == RIP_FP32 ? (const void*)unpack_kernel<RIP_FP32>
                               : (const void*)unpack_kernel<RIP_BF16>,
             s, args, stream, "rip_ckpt_unpack");
}

extern "C" int32_t rip_gate_forward(const void* gate, int64_t ld_gate, const void* up,
                                    int64_t ld_up, int32_t dtype, int64_t rows, int64_t width,
                                    void* h, int64_t ld_h, int8_t* gate_codes, uint8_t* gate_exps,
                                    int8_t* up_codes, uint8_t* up_exps, void* stream) {
  clear_error();
  int32_t rc;
  Shape s;
  if ((rc = make_shape(dtype, rows, width, &s)) ||
      (rc = check_matrix(gate, "gate", dtype, rows, width, ld_gate)) ||
      (rc = check_matrix(up, "up", dtype, rows, width, ld_up)) ||
      (rc = check_matrix(h, "h", dtype, rows, width, ld_h)) ||
      (rc = check_ckpt(gate_codes, gate_exps, "gate checkpoint", s)) ||
      (rc = check_ckpt(up_codes, up_exps, "up checkpoint", s)))
    return rc;
  Buffers b;
  b.matrix(gate, dtype, rows, width, ld_gate, "gate", false);
  b.matrix(up, dtype, rows, width, ld_up, "up", false);
  b.matrix(h, dtype, rows, width, ld_h, "h", true);
  b.range(gate_codes, code_bytes(s), "gate codes", true);
  b.range(gate_exps, exp_bytes(s), "gate exps", true);
  b.range(up_codes, code_bytes(s), "up codes", true);
  b.range(up_exps, exp_bytes(s), "up exps", true);
  if ((rc = b.check())) return rc;
  Ckpt g8{gate_codes, gate_exps}, u8{up_codes, up_exps};
  void* args[] = {&s, &gate, &ld_gate, &up, &ld_up, &h, &ld_h, &g8, &u8};
  const bool past = stream_inputs(dtype, rows, width, 2);
  const void* fn = dtype == RIP_FP32 ? (past ? (const void*)gate_forward_kernel<RIP_FP32, true>
                                             : (const void*)gate_forward_kernel<RIP_FP32, false>)
                                     : (past ? (const void*)gate_forward_kernel<RIP_BF16, true>
                                             : (const void*)gate_forward_kernel<RIP_BF16, false>);
  return run(fn, s, args, stream, "rip_gate_forward");
}

extern "C" int32_t rip_gate_backward(const void* dh, int64_t ld_dh, int32_t dtype,
                                     const int8_t* gate_codes, const uint8_t* gate_exps,
                                     const int8_t* up_codes, const uint8_t* up_exps, int64_t rows,
                                     int64_t width, void* dgate, int64_t ld_dgate, void* dup,
                                     int64_t ld_dup, int8_t* h_codes, uint8_t* h_exps,
                                     void* stream) {
  clear_error();
  int32_t rc;
  Shape s;
  if ((rc = make_shape(dtype, rows, width, &s)) ||
      (rc = check_matrix(dh, "dh", dtype, rows, width, ld_dh)) ||
      (rc = check_matrix(dgate, "dgate", dtype, rows, width, ld_dgate)) ||
      (rc = check_matrix(dup, "dup", dtype, rows, width, ld_dup)) ||
      (rc = check_ckpt(gate_codes, gate_exps, "gate checkpoint", s)) ||
      (rc = check_ckpt(up_codes, up_exps, "up checkpoint", s)))
    return rc;
  const bool again = h_codes || h_exps;
  if (again && (rc = check_ckpt(h_codes, h_exps, "h checkpoint", s))) return rc;
  Buffers b;
  b.matrix(dh, dtype, rows, width, ld_dh, "dh", false);
  b.matrix(dgate, dtype, rows, width, ld_dgate, "dgate", true);
  b.matrix(dup, dtype, rows, width, ld_dup, "dup", true);
  b.range(gate_codes, code_bytes(s), "gate codes", false);
  b.range(gate_exps, exp_bytes(s), "gate exps", false);
  b.range(up_codes, code_bytes(s), "up codes", false);
  b.range(up_exps, exp_bytes(s), "up exps", false);
  if (again) {
    b.range(h_codes, code_bytes(s), "h codes", true);
    b.range(h_exps, exp_bytes(s), "h exps", true);
  }
  if ((rc = b.check())) return rc;
  Ckpt g8{const_cast<int8_t*>(gate_codes), const_cast<uint8_t*>(gate_exps)};
  Ckpt u8{const_cast<int8_t*>(up_codes), const_cast<uint8_t*>(up_exps)};
  Ckpt h8{h_codes, h_exps};
  void* args[] = {&s, &dh, &ld_dh, &g8, &u8, &dgate, &ld_dgate, &dup, &ld_dup, &h8};
  const bool past = stream_inputs(dtype, rows, width, 2);  // dh, and at most as much again
  const void* fn = dtype == RIP_FP32 ? backward_of<RIP_FP32>(again, past)
                                     : backward_of<RIP_BF16>(again, past);
  return run(fn, s, args, stream, "rip_gate_backward");
}
