// Groups of values as whole numbers with a scale: the arithmetic that the 4-bit weights and the cache share.
//
//   scale = bf16(max |w| over the group / Q), Q = 2^(bits - 1) - 1, rounded once to nearest even; 0 below 2^-126
//   code  = the whole number nearest to w / scale, ties to even; 0 where the scale is 0
//   value = code * scale
//
// The scale has 8 significant bits because the codes are chosen against the rounded scale (so its rounding costs nothing) and
// because w - code * scale and scale / 2 are then exact in fp32: whether a code is the nearest one is decided exactly, by a
// compare, although the first guess comes from a product with a rounded reciprocal. max / scale is at most Q / (1 - 2^-8), i.e.
// 7.03 and 127.4981, so codes stay within +-Q without a clamp. A group that holds Inf or NaN gets a scale of NaN (and codes of 0).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lc_common.cuh"

namespace lc {

constexpr uint32_t kScaleNaN = 0x7FC00000u;  // as the upper half of an fp32

template <int type>
struct TypeOf;
template <>
struct TypeOf<LC_TYPE_F32> { using T = float; };
template <>
struct TypeOf<LC_TYPE_BF16> { using T = __nv_bfloat16; };
template <>
struct TypeOf<LC_TYPE_F16> { using T = __half; };

inline uint32_t type_bytes(int type) { return type == LC_TYPE_F32 ? 4 : 2; }
inline bool type_ok(int type) { return type == LC_TYPE_F32 || type == LC_TYPE_BF16 || type == LC_TYPE_F16; }
inline bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_float(float v, float& x) { x = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16& x) { x = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half& x) { x = __float2half_rn(v); }

// Eight neighbouring values of a row as fp32, zeros from `valid` on. Where all are there and the address allows it, by loads of 16 bytes.
template <class T>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8]) {
  if (valid >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    uint4 raw[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? to_float(p[i]) : 0.0f;
  }
}

template <class T>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8]) {
  if (valid >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    uint4 raw[sizeof(T) / 2];
    T* e = reinterpret_cast<T*>(raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) from_float(v[i], e[i]);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = raw[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < valid) from_float(v[i], p[i]);
  }
}

// The largest magnitude of eight values as fp32 bits: as whole numbers these order like the magnitudes, with Inf and NaN above.
__device__ __forceinline__ uint32_t max_bits8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return m;
}

// The maximum over the `lanes` neighbouring lanes (a power of two, aligned) that hold a group. All 32 lanes take part.
__device__ __forceinline__ uint32_t max_over_lanes(uint32_t m, int lanes) {
  for (int d = 1; d < lanes; d <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  return m;
}

// bf16(max / top), as fp32 bits, from the maximum's bits. The fp32 quotient rounds a second time only if it lies exactly between
// two bf16 numbers; the sign of its remainder (exact, by one multiply-add) then tells on which side the true quotient is.
__device__ __forceinline__ uint32_t group_scale(uint32_t max_bits, float top) {
  if (max_bits >= 0x7F800000u) return kScaleNaN;
  const float most = __uint_as_float(max_bits), q = __fdiv_rn(most, top);
  const uint32_t u = __float_as_uint(q);
  uint32_t s = u + 0x7FFFu + ((u >> 16) & 1u);
  if ((u & 0xFFFFu) == 0x8000u) {
    const float rest = __fmaf_rn(-q, top, most);
    if (rest != 0.0f) s = rest > 0.0f ? u + 0x8000u : u;
  }
  s &= 0xFFFF0000u;
  return s < 0x00800000u ? 0u : s;
}

// The codes of eight values, as two's complement whole numbers. (x + 1.5 * 2^23 rounds x to a whole number, ties to even, and
// holds it in its low bits.)
__device__ __forceinline__ void codes8(const float (&v)[8], uint32_t scale_bits, int (&q)[8]) {
  if (scale_bits == 0u || scale_bits == kScaleNaN) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = 0;
    return;
  }
  const float s = __uint_as_float(scale_bits), inv = __frcp_rn(s), half = 0.5f * s, magic = 12582912.0f;
  float far = 0.0f, rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = __fmaf_rn(v[i], inv, magic);
    q[i] = (int)(__float_as_uint(t) - __float_as_uint(magic));
    rest[i] = __fmaf_rn(-(t - magic), s, v[i]);
    far = fmaxf(far, fabsf(rest[i]));
  }
  if (far >= half) {  // a guess on the wrong side of a border, or a value on one
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float r = fabsf(rest[i]);
      if (r > half || (r == half && (q[i] & 1))) q[i] += rest[i] > 0.0f ? 1 : -1;
    }
  }
}

// Eight codes in a row of 4 bits: value e at bit 4 * (e / 2) + 16 * (e % 2), offset by 8, so that a mask takes two neighbours out
// as the two halves of a word. In 8 bits: one byte after the other, offset by 128.
__device__ __forceinline__ uint32_t pack4(const int (&q)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) w |= ((uint32_t)(q[e] + 8) & 15u) << (4 * (e / 2) + 16 * (e % 2));
  return w;
}
__device__ __forceinline__ uint2 pack8(const int (&q)[8]) {
  uint2 w = make_uint2(0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w.x |= ((uint32_t)(q[e] + 128) & 255u) << (8 * e);
    w.y |= ((uint32_t)(q[e + 4] + 128) & 255u) << (8 * e);
  }
  return w;
}

// code * scale, exact in fp32. 2^23 + n holds n in its low bits.
__device__ __forceinline__ void values_of4(uint32_t w, float s, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = (__uint_as_float(((w >> (4 * (e / 2) + 16 * (e % 2))) & 15u) | 0x4B000000u) - 8388616.0f) * s;
}
__device__ __forceinline__ void values_of8(uint2 w, float s, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = (__uint_as_float(__byte_perm(e < 4 ? w.x : w.y, 0x4B000000u, 0x7540 | (e & 3))) - 8388736.0f) * s;
}

// n / d by a multiplication, for n < 2^31 and 1 <= d < 2^31 (a division by a number known only at run time takes some twenty
// instructions, as much as the rest of the index arithmetic of a row).
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t d_) : d(d_), mul(0), shift(0) {
    while ((1ull << shift) < d) ++shift;
    mul = (uint32_t)(((1ull << (31 + shift)) + d - 1) / d);  // < 2^32, since 2^shift < 2 d
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> (31 + shift)); }
};

}  // namespace lc
