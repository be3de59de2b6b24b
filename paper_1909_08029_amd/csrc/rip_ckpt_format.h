// The 8-bit checkpoint format: how a block of 32 values becomes 32 integers and
// one exponent, and back (device code shared by rip_ckpt.hip and rip_wgrad.hip).
//
// A block's step is the smallest power of two 2^e, -126 <= e <= 121, for which its
// largest magnitude is at most 127 steps (or 2^121, where there is none: the few
// fp32 numbers beyond are cut to 127 steps, as 2^122 would round them to 2^128).
// A power of two instead of a free
// scale costs at most one of the eight bits and buys two things: the value
// q * 2^e has at most seven significant bits, so it is exact in bf16 and goes
// into the matrix cores as it is, and packing is exact up to the one rounding
// of x / 2^e, the same on every machine.
#pragma once

#include "rip_ops_common.h"

namespace rip {

constexpr int kCkptBlock = 32;                 // columns of a block
constexpr uint32_t kCkptMax = 121 + 127;       // largest exponent byte of a finite block
constexpr uint32_t kCkptNan = 255;             // exponent byte of a block with an inf or NaN

// Exponent byte (e + 127, 1..248) of a block whose largest magnitude has the
// bits `top`; kCkptNan if that is an infinity or a NaN.
__device__ __forceinline__ uint32_t ckpt_exponent(uint32_t top) {
  // |x| = m * 2^k, 1 <= m < 2: 127 steps of 2^(k-6) reach 1.984375 * 2^k
  const int e = (int)(top >> 23) - 6 + ((top & 0x7fffffu) > 0x7e0000u ? 1 : 0);
  return top >= 0x7f800000u ? kCkptNan : (uint32_t)max(1, min(e, (int)kCkptMax));
}

// Exponent byte and codes (four to a word) of the lane's N values; the 32 / N lanes
// of a block are consecutive and all active.
template <int N>
__device__ __forceinline__ uint32_t ckpt_pack(const float (&x)[N], uint32_t (&codes)[N / 4]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < kCkptBlock / N; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  const uint32_t e = ckpt_exponent(top);
  // x / 2^e + 1.5 * 2^23, rounded once to nearest even: its low byte is q
  const float inv = e == kCkptNan ? 0.0f : __uint_as_float((254 - e) << 23);
  uint32_t q[N];
#pragma unroll
  for (int j = 0; j < N; ++j)
    q[j] = __float_as_uint(__builtin_fmaf(x[j], inv, 12582912.0f)) & 0xff;
  if (e == kCkptMax) {  // the one step that a magnitude may exceed
#pragma unroll
    for (int j = 0; j < N; ++j)
      q[j] = (uint32_t)(int)fminf(fmaxf(rintf(x[j] * inv), -127.0f), 127.0f) & 0xff;
  }
#pragma unroll
  for (int j = 0; j < N; j += 4)
    codes[j / 4] = e == kCkptNan ? 0 : q[j] | q[j + 1] << 8 | q[j + 2] << 16 | q[j + 3] << 24;
  return e;
}

// 2^e, NaN for a block that held an inf or a NaN (its codes are zeros).
__device__ __forceinline__ float ckpt_step(uint32_t e) {
  return __uint_as_float(e == kCkptNan ? 0x7fc00000u : e << 23);
}

// Byte j of a word as a signed integer, widened to fp32 (one instruction, which
// picks the byte itself; written so that the compiler finds it).
__device__ __forceinline__ float widen(uint32_t w, int j) {
  return (float)((int)(w << (24 - 8 * j)) >> 24);
}

template <int N>
__device__ __forceinline__ void ckpt_unpack(const uint32_t (&codes)[N / 4], uint32_t e,
                                            float (&x)[N]) {
  const float step = ckpt_step(e);
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = widen(codes[j / 4], j % 4) * step;
}

}  // namespace rip
