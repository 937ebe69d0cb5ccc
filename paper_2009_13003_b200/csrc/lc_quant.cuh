// Groups of values as whole numbers with a scale: the arithmetic that the 4-bit weights and the cache share.
//
//   scale = bf16(max |w| over the group / Q), Q = 2^(bits - 1) - 1, rounded once to nearest even; 0 below 2^-126
//   code  = the whole number nearest to w / scale, ties to even; 0 where the scale is 0
//   value = code * scale
//
// The scale has 8 significant bits because the codes are chosen against the rounded scale (so its rounding costs nothing) and
// because w - code * scale and scale / 2 are then exact in fp32: whether a code is the nearest one is decided exactly, by a
// compare, although the first guess comes from a product with a reciprocal. max / scale is at most Q / (1 - 2^-8), i.e.
// 7.03 and 127.4981, so codes stay within +-Q without a clamp. A group that holds Inf or NaN gets a scale of NaN (and codes of 0).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include <type_traits>

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

// Eight neighbouring values of a row as fp32, zeros from `valid` on: by the widest loads that the address allows (rows of heads of 100
// values in 16 bits begin on 8 bytes).
// kWhole: the caller knows that all are there, on 16 bytes.
template <bool kWhole = false, class T>
__device__ __forceinline__ void load8(const T* p, int valid, float* v) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (kWhole || (valid >= 8 && (at & 15) == 0)) {
    uint4 raw[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
    return;
  }
  if constexpr (!kWhole) {
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      if (sizeof(T) == 2 && valid >= h + 4 && (at & 7) == 0) {
        const uint2 raw = __ldg(reinterpret_cast<const uint2*>(p + h));
        const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[h + i] = to_float(e[i]);
      } else if (sizeof(T) == 2 && valid >= h + 4) {  // pairs on 4 bytes, and what is left at the ends
        const int odd = (at & 2) / 2;
        const uint32_t a = __ldg(reinterpret_cast<const uint32_t*>(p + h + odd));
        const T* e = reinterpret_cast<const T*>(&a);
        if (odd) {
          v[h] = to_float(p[h]);
          v[h + 1] = to_float(e[0]);
          v[h + 2] = to_float(e[1]);
          v[h + 3] = to_float(p[h + 3]);
        } else {
          const uint32_t b = __ldg(reinterpret_cast<const uint32_t*>(p + h + 2));
          const T* f = reinterpret_cast<const T*>(&b);
          v[h] = to_float(e[0]);
          v[h + 1] = to_float(e[1]);
          v[h + 2] = to_float(f[0]);
          v[h + 3] = to_float(f[1]);
        }
      } else {
#pragma unroll
        for (int i = h; i < h + 4; ++i) v[i] = i < valid ? to_float(p[i]) : 0.0f;
      }
    }
  }
}

// A value read into the type T, rounded to nearest. bf16: numbers beyond the largest are the largest, not Inf; the scale of a group with
// the largest may be rounded up past it (to 1.0078125 * 2^121 in 8 bits, 1.140625 * 2^125 in 4).
__device__ __forceinline__ void read_as(float v, float& x) { x = v; }
__device__ __forceinline__ void read_as(float v, __half& x) { x = __float2half_rn(v); }
__device__ __forceinline__ void read_as(float v, __nv_bfloat16& x) {
  unsigned short h;
  asm("cvt.rn.satfinite.bf16.f32 %0, %1;" : "=h"(h) : "f"(v));
  x = __ushort_as_bfloat16(h);
}
template <class T>
__device__ __forceinline__ uint32_t read_two(float a, float b) {
  uint32_t r;
  if constexpr (std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  else asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// `n` neighbouring values the other way, 16 bytes of them where all are there. The lanes of a warp hold neighbouring runs, so that a store
// of theirs is one run of bytes: with 32 bytes a lane and two stores of every other 16, memory pays for both halves of each 32 (0.4 GB of
// fp32 from 4 bits: 99 us; so 75).
template <class T>
constexpr int kRun = 16 / sizeof(T);
template <bool kWhole = false, class T>
__device__ __forceinline__ void store_run(T* p, int valid, const float* v) {
  constexpr int n = kRun<T>;
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (kWhole || (valid >= n && (at & 15) == 0)) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint4*>(p) = make_uint4(read_two<T>(v[0], v[1]), read_two<T>(v[2], v[3]), read_two<T>(v[4], v[5]), read_two<T>(v[6], v[7]));
    else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
  if constexpr (!kWhole) {
#pragma unroll
    for (int h = 0; h < n; h += 4) {
      if (sizeof(T) == 2 && valid >= h + 4 && (at & 7) == 0) {
        uint2 raw;
        T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
        for (int i = 0; i < 4; ++i) read_as(v[h + i], e[i]);
        *reinterpret_cast<uint2*>(p + h) = raw;
      } else if (sizeof(T) == 2 && valid >= h + 4) {
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) read_as(v[h + i], e[i]);
        uint32_t w[2];
        memcpy(w, e, sizeof w);
        if (at & 2) {
          p[h] = e[0];
          *reinterpret_cast<uint32_t*>(p + h + 1) = __byte_perm(w[0], w[1], 0x5432);
          p[h + 3] = e[3];
        } else {
          reinterpret_cast<uint32_t*>(p + h)[0] = w[0];
          reinterpret_cast<uint32_t*>(p + h)[1] = w[1];
        }
      } else {
#pragma unroll
        for (int i = h; i < h + 4; ++i)
          if (i < valid) read_as(v[i], p[i]);
      }
    }
  }
}

// The larger of two magnitudes; NaN if one is.
__device__ __forceinline__ float max_magnitude(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
  return m;
}

// 16 whole values on 16 bytes as fp32, and the largest magnitude of them. Of 16-bit values, two at a time: without their signs their
// patterns order like the magnitudes, Inf and NaN last.
template <class T>
__device__ __forceinline__ float load16(const T* p, float (&v)[16]) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[8], most = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 x = __ldg(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      most = __vmaxu2(most, w[i] & 0x7FFF7FFFu);
      const T* e = reinterpret_cast<const T*>(&w[i]);
      v[2 * i] = to_float(e[0]);
      v[2 * i + 1] = to_float(e[1]);
    }
    const unsigned short m = (unsigned short)max(most & 0xFFFFu, most >> 16);
    return to_float(reinterpret_cast<const T&>(m));
  } else {
    load8<true>(p, 8, v);
    load8<true>(p + 8, 8, v + 8);
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max_magnitude(m, v[i]);
    return m;
  }
}

// The largest magnitude over the `lanes` neighbouring lanes (a power of two, aligned) that hold a group. All lanes of the warp
// take part that have not left it: rows share a warp whole groups of lanes each, and the lanes of a row leave together.
__device__ __forceinline__ float max_over_lanes(float m, int lanes) {
  for (int d = 1; d < lanes; d <<= 1) m = max_magnitude(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  return m;
}

// bf16(most / Q), as fp32 bits. From a quotient that is right to a few units in fp32's last place, cut to bf16: the next bf16 number is the
// nearer one if most lies beyond Q times the middle between the two, or on it and the lower one is odd. That product has 16 bits, so
// the compare is exact (and it holds also where the cut is one number off).
template <int kBits>
__device__ __forceinline__ uint32_t group_scale(float most) {
  constexpr float kTop = (1 << (kBits - 1)) - 1;
  if (!(most < __uint_as_float(0x7F800000u))) return kScaleNaN;
  const uint32_t low = __float_as_uint(most * (1.0f / kTop)) & 0xFFFF0000u;
  const float beyond = __fmaf_rn(-__uint_as_float(low | 0x8000u), kTop, most);
  const uint32_t s = beyond > 0.0f || (beyond == 0.0f && (low & 0x10000u)) ? low + 0x10000u : low;
  return s < 0x00800000u ? 0u : s;
}

// Two fp32 numbers in one instruction.
using Two = unsigned long long;
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split_two(Two r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ Two add_two(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Two mul_two(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The codes of `n` values of type T, each plus 2^(bits - 1) in the low bits of a float's pattern (x + 1.5 * 2^23 rounds x to a whole number,
// ties to even, and holds it there). With at most 11 bits in a value and 8 in the scale, a quotient is a tie or far from one, and one
// step of refinement makes it the nearest fp32 number, which a tie is itself (also where the scale is next to 2^-126 and the remainder is rounded
// to 2^-149: all numbers of both types at all scales of the lowest binades are tested). An fp32 value can be anywhere: its code is a guess
// that the exact remainder confirms, or, hardly ever, moves by one.
template <class T, int kBits, int n>
__device__ __forceinline__ void codes(const float (&v)[n], uint32_t scale_bits, float (&t)[n]) {
  constexpr float kMagic = 12582912.0f + (1 << (kBits - 1));
  if (scale_bits == 0u || scale_bits == kScaleNaN) {
#pragma unroll
    for (int i = 0; i < n; ++i) t[i] = kMagic;
    return;
  }
  const float s = __uint_as_float(scale_bits), half = 0.5f * s;
  float inv, far = 0.0f;
  asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(s));
  const Two inv2 = two(inv, inv), minus_s = two(-s, -s), magic = two(kMagic, kMagic);
#pragma unroll
  for (int i = 0; i < n; i += 2) {
    const Two x = two(v[i], v[i + 1]);
    if constexpr (sizeof(T) == 2) {
      const Two q = mul_two(x, inv2);
      split_two(add_two(fma_two(fma_two(q, minus_s, x), inv2, q), magic), t[i], t[i + 1]);
    } else {
      const Two c = fma_two(x, inv2, magic);
      float a, b;
      split_two(fma_two(add_two(c, two(-kMagic, -kMagic)), minus_s, x), a, b);
      far = fmaxf(far, fmaxf(fabsf(a), fabsf(b)));
      split_two(c, t[i], t[i + 1]);
    }
  }
  if (sizeof(T) == 4 && far >= half) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float rest = __fmaf_rn(kMagic - t[i], s, v[i]), r = fabsf(rest);
      if (r > half || (r == half && (__float_as_uint(t[i]) & 1u))) t[i] += rest > 0.0f ? 1.0f : -1.0f;
    }
  }
}

// Two neighbouring codes as the halves of a word, and four pairs of 4 bits as one: a mask takes a pair out again. Pair p of eight values
// in a row is values 2 p and 2 p + 1.
__device__ __forceinline__ uint32_t pair_of(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410); }
__device__ __forceinline__ uint32_t pack_pairs(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return a + (b << 4) + (c << 8) + (d << 12); }
__device__ __forceinline__ uint32_t pack4(const float* t) {
  return pack_pairs(pair_of(t[0], t[1]), pair_of(t[2], t[3]), pair_of(t[4], t[5]), pair_of(t[6], t[7]));
}
// Four codes of 8 bits, one byte after the other.
__device__ __forceinline__ uint32_t pack_bytes(const float* t) {
  const uint32_t a = __byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040), b = __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040);
  return __byte_perm(a, b, 0x5410);
}
__device__ __forceinline__ uint2 pack8(const float* t) { return make_uint2(pack_bytes(t), pack_bytes(t + 4)); }

// What the codes in the low bits of n[] stand for, in fp32: exact. (2^23 + n holds n in its low bits.)
template <int kBits, int count>
__device__ __forceinline__ void values_of(const uint32_t (&n)[count], float scale, float* v) {
  constexpr float kOffset = -(8388608.0f + (1 << (kBits - 1)));
#pragma unroll
  for (int e = 0; e < count; e += 2) {
    const Two x = two(__uint_as_float(n[e] | 0x4B000000u), __uint_as_float(n[e + 1] | 0x4B000000u));
    split_two(mul_two(add_two(x, two(kOffset, kOffset)), two(scale, scale)), v[e], v[e + 1]);
  }
}
// Reading into fp16 from 8 bits: the scale of a group whose largest magnitude is 65504 or next to it was rounded up to 516, and 127 * 516 =
// 65532 rounds to Inf. Such values read as 65504: what was a number of fp16 when it was written stays one. (A larger scale comes from
// a value beyond fp16, a smaller one stays within it, and so does 7 * 9344, from 4 bits. For bf16 see read_as.)
template <class T, int kBits, int count>
__device__ __forceinline__ void keep_in_type(float scale, float (&v)[count]) {
  if constexpr (std::is_same<T, __half>::value && kBits == 8) {
    if (scale != 516.0f) return;
#pragma unroll
    for (int e = 0; e < count; ++e) v[e] = fminf(fmaxf(v[e], -65504.0f), 65504.0f);
  }
}
// The first `count` values of eight in a row of a cache.
template <int kBits, int count>
__device__ __forceinline__ void values_in_row(uint2 w, float scale, float* v) {
  uint32_t n[count];
#pragma unroll
  for (int e = 0; e < count; ++e) n[e] = kBits == 4 ? (w.x >> (4 * (e / 2) + 16 * (e % 2))) & 15u : __byte_perm(e < 4 ? w.x : w.y, 0, 0x4440 | (e & 3));
  values_of<kBits>(n, scale, v);
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
