// The 8-bit token cache's element format and device helpers (qcache.hip, qattn.hip).
//
// A row's keys and values are e4m3 numbers times the scale of their block of 64 rows and
// key-value head.  Scales are powers of two: they change no mantissa, so dequantising to
// bfloat16 is exact (3 stored mantissa bits) and rounding a held code again under a larger
// scale loses bits only where the code falls among the subnormals.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "fc_internal.h"
#include "gemm_dev.h"

namespace fc {
namespace {

constexpr int kQBlock = FC_QCACHE_BLOCK;   // rows that share a scale
constexpr float kQTop = 448.f;             // largest e4m3 number
constexpr int kQLowExp = -100;             // smallest scale 2^-100: 1 / scale stays finite

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Smallest power of two s >= 2^-100 with amax <= 448 s (448 = 1.75 * 2^8; amax finite, >= 0).
__device__ __forceinline__ float scale_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return pow2f(max(e, kQLowExp));
}
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;   // infinities and NaN set no scale
}
// To the range of e4m3; a NaN stays one.
__device__ __forceinline__ float clamp_top(float x) {
  return fabsf(x) > kQTop ? copysignf(kQTop, x) : x;
}
// Four values (already divided by their scale) as e4m3 codes, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_top(a), clamp_top(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_top(c), clamp_top(d), w, true);
}
__device__ __forceinline__ float4 unpack_e4m3(uint32_t w) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return make_float4(a[0], a[1], b[0], b[1]);
}
// Codes under another scale: ratio = old scale / new scale (a power of two).
__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float ratio) {
  const float4 x = unpack_e4m3(w);
  return pack_e4m3(x.x * ratio, x.y * ratio, x.z * ratio, x.w * ratio);
}

// Rows held and rows new of item b (the same in every lane), clamped so that no value makes a
// kernel leave its buffers.
__device__ __forceinline__ int q_held(const int32_t *len, int b, int cap) {
  return __builtin_amdgcn_readfirstlane(min(max(len[b], 0), cap));
}
__device__ __forceinline__ int q_new(const int32_t *n_new, int b, int n, int held, int cap) {
  return min(n_new ? __builtin_amdgcn_readfirstlane(min(max(n_new[b], 0), n)) : n, cap - held);
}

// Numbers that no kernel of the launch writes, at an index that all lanes share: read by the scalar
// unit, whose loads no wait for vector loads in flight touches.
typedef const __attribute__((address_space(4))) float *uniform_floats;
__device__ __forceinline__ uniform_floats as_uniform(const float *p) {
  return (uniform_floats)(uintptr_t)p;
}

// Quotients i / d for 0 <= i < 2^30 and 1 <= d <= 2^30: mulhi(4 i, magic) >> s with s = ceil(log2 d) and
// magic = ceil(2^(30 + s) / d) < 2^32.  e = magic d - 2^(30 + s) < d <= 2^s, so i magic / 2^(30 + s)
// exceeds i / d by i e / (d 2^(30 + s)) < 1 / d: not enough to reach the next integer.
struct Quot {
  uint32_t magic;
  int shift;
  __device__ __forceinline__ int operator()(int i) const {
    return (int)(__umulhi((uint32_t)i << 2, magic) >> shift);
  }
};
inline Quot quot_by(int d) {
  int s = 0;
  while ((1L << s) < d) ++s;
  return Quot{(uint32_t)(((1UL << (30 + s)) + d - 1) / d), s};
}

}  // namespace
}  // namespace fc
