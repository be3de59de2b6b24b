// Device and host helpers shared by the operators that fill gradient buffers
// (rip_embed.hip, rip_ckpt.hip, rip_wgrad.hip, rip_loss.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "rip_internal.h"

namespace rip {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Sixteen bytes at any address that an element may have: rows of odd length
// start anywhere, and gfx950 loads and stores 16 bytes at any alignment.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int64_t kCacheBytes = (int64_t)256 << 20;  // what the memory-side cache holds

// Sixteen bytes past the caches (non-temporal), for data of which a launch writes
// or reads more than a cache holds, once: the gated unit of 16384 x 5504 bf16 took
// 251 us without, 242 with such stores, 218 with such loads too; the policy loss
// of 8192 x 131072 bf16 840 and 777 with such stores.  Not where a lane's 32 bytes are
// two accesses and each covers half of every cache line (eight fp32 columns): an
// embedding and its gradient in fp32 took 1.7 times as long so.
__device__ __forceinline__ void store_stream(u32x4_any* p, u32x4_any v) {
  __builtin_nontemporal_store(v, p);
}
__device__ __forceinline__ u32x4 load_stream(const u32x4_any* p) {
  return __builtin_nontemporal_load(p);
}

// Eight consecutive elements are what one lane handles of a row: 16 bytes of
// bf16, 32 of fp32.
constexpr int kLane = 8;

template <int DT>
struct Elem;  // storage type of RIP_FP32 / RIP_BF16
template <>
struct Elem<RIP_FP32> {
  typedef float T;
  static __device__ __forceinline__ float load(const T* p) { return *p; }
  static __device__ __forceinline__ void store(T* p, float x) { *p = x; }
  template <bool STREAM = false>
  static __device__ __forceinline__ void load8(const T* p, float (&f)[kLane]) {
    const u32x4_any a = *(const u32x4_any*)p, b = *(const u32x4_any*)(p + 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[j] = __uint_as_float(a[j]);
      f[4 + j] = __uint_as_float(b[j]);
    }
  }
  static __device__ __forceinline__ void store8(T* p, const float (&f)[kLane]) {
    u32x4_any a, b;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = __float_as_uint(f[j]);
      b[j] = __float_as_uint(f[4 + j]);
    }
    *(u32x4_any*)p = a;
    *(u32x4_any*)(p + 4) = b;
  }
};
template <>
struct Elem<RIP_BF16> {
  typedef uint16_t T;
  static __device__ __forceinline__ float load(const T* p) {
    return __uint_as_float((uint32_t)*p << 16);
  }
  // fp32 -> bf16, to nearest even, with the hardware's conversion
  static __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f32x2 f = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
  }
  static __device__ __forceinline__ void store(T* p, float x) { *p = (uint16_t)pack2(x, x); }
  static __device__ __forceinline__ void unpack8(u32x4 a, float (&f)[kLane]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = __uint_as_float(a[j] << 16);
      f[2 * j + 1] = __uint_as_float(a[j] & 0xffff0000u);
    }
  }
  template <bool STREAM = false>
  static __device__ __forceinline__ void load8(const T* p, float (&f)[kLane]) {
    const u32x4 a = STREAM ? load_stream((const u32x4_any*)p) : *(const u32x4_any*)p;
    unpack8(a, f);
  }
  static __device__ __forceinline__ void store8(T* p, const float (&f)[kLane]) {
    u32x4_any a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = pack2(f[2 * j], f[2 * j + 1]);
    store_stream((u32x4_any*)p, a);
  }
};

// Elements c .. c+7 of a row of `width`; zero past its end, nothing read there.
template <int DT, bool STREAM = false>
__device__ __forceinline__ void load_unit(const typename Elem<DT>::T* row, int c, int width,
                                          float (&f)[kLane]) {
  if (c + kLane <= width) {
    Elem<DT>::template load8<STREAM>(row + c, f);
  } else {
#pragma unroll
    for (int j = 0; j < kLane; ++j) f[j] = c + j < width ? Elem<DT>::load(row + c + j) : 0.0f;
  }
}
template <int DT>
__device__ __forceinline__ void store_unit(typename Elem<DT>::T* row, int c, int width,
                                           const float (&f)[kLane]) {
  if (c + kLane <= width) {
    Elem<DT>::store8(row + c, f);
  } else {
#pragma unroll
    for (int j = 0; j < kLane; ++j)
      if (c + j < width) Elem<DT>::store(row + c + j, f[j]);
  }
}

// A token id as 64 bits; ids are int32 (wide = 0) or int64.
__device__ __forceinline__ int64_t load_id(const void* ids, int wide, int64_t i) {
  return wide ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
}

// e^x within two units in the last place: x * log2(e) in two parts, so that the
// rounding of the product does not grow with |x|.  -inf gives 0, NaN stays NaN;
// x is at most 88 wherever this is called.
__device__ __forceinline__ float exp_acc(float x) {
  const float kL2e = 1.44269502f, kL2eLo = 1.92596299e-8f;
  const float t = x * kL2e;
  const float lo = __builtin_fmaf(x, kL2eLo, __builtin_fmaf(x, kL2e, -t));
  const float p = __builtin_amdgcn_exp2f(t);
  // below the smallest result the correction would be 0 * inf for x = -inf
  return x < -104.0f ? 0.0f : __builtin_fmaf(p, lo * 0.693147182f, p);
}

// Division of a 32-bit number by a fixed divisor with one high product and a
// shift, for n < 2^31 (the divisor's reciprocal rounded up to 33 bits).
struct FastDiv {
  uint32_t d, mul, shift;
  static FastDiv make(uint32_t d) {
    FastDiv f{d, 0, 0};
    while (f.shift < 31 && (1u << f.shift) < d) ++f.shift;
    f.mul = (uint32_t)(((((uint64_t)1 << f.shift) - d) << 32) / d + 1);
    return f;
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return (__umulhi(n, mul) + n) >> shift;
  }
};

inline int elem_bytes(int32_t dtype) { return dtype == RIP_BF16 ? 2 : 4; }
inline bool known_dtype(int32_t dtype) { return dtype == RIP_FP32 || dtype == RIP_BF16; }

// A launch's own status (not an earlier sticky error).
inline int32_t launch(const void* fn, dim3 grid, dim3 block, void** args, size_t lds,
                      void* stream, const char* what) {
  const hipError_t e = hipLaunchKernel(fn, grid, block, args, lds, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(RIP_E_HIP, "%s: %s", what, hipGetErrorString(e));
  return RIP_OK;
}

// A matrix argument: not NULL unless empty, rows no shorter than their width,
// and its base at an element's boundary.
int32_t check_matrix(const void* p, const char* what, int32_t dtype, int64_t rows, int64_t width,
                     int64_t ld);
// [a, a+na) and [b, b+nb) share a byte.
inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}
// One of a call's buffers; RIP_E_OVERLAP where one that is written shares a byte with
// another.
struct Range {
  const void* p;
  int64_t bytes;
  const char* what;
  bool written;
};
inline int32_t check_apart(const char* name, const Range* list, int count) {
  for (int i = 0; i < count; ++i)
    for (int j = 0; j < i; ++j)
      if ((list[i].written || list[j].written) &&
          overlap(list[i].p, list[i].bytes, list[j].p, list[j].bytes))
        return fail(RIP_E_OVERLAP, "%s: %s overlaps %s", name, list[i].what, list[j].what);
  return RIP_OK;
}
// Bytes from a matrix's first element to the end of its last.
inline int64_t span(int32_t dtype, int64_t rows, int64_t width, int64_t ld) {
  return rows < 1 || width < 1 ? 0 : ((rows - 1) * ld + width) * elem_bytes(dtype);
}

}  // namespace rip
