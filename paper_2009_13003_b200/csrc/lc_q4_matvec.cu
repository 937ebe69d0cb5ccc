// Products of 4-bit weights with the vectors of a few tokens:
//   out[t, r] = sum over groups G of scale[r, G] * (sum over c in G of code[r, c] * x[t, c]).
//
// The weights are read once and bound the product up to some 16 tokens; the multiplications go to the tensor cores (m16n8k16:
// 16 rows, 8 tokens, 16 columns), which take the codes as exact 16-bit numbers and add up in fp32. A group's scale meets the group's
// sum in fp32, not the codes: code * scale needs 11 bits, more than bf16 has. An fp32 vector takes three columns of the product: its
// values cut into three bf16 numbers, 8 bits each, whose sum they are, so that nothing of them is lost (but what lies below 2^-133).
#include "lc_q4.cuh"

namespace lc {
namespace {

constexpr uint32_t kWarps = 8;
constexpr uint32_t kAhead = 4;       // steps of weights that a warp has in flight: 4 KB
constexpr uint32_t kRedStride = 20;  // floats from one column of a tile's sums to the next: the lanes of a store meet in no bank

struct MatvecArgs {
  const uint8_t* q4;
  const void* x;
  void* out;
  uint64_t x_stride, out_stride;
  Q4Layout L;
  uint32_t tokens, per_pass;  // vectors in all, and of one pass (blockIdx.y)
  int out_type;
  uint32_t chunk_steps;       // steps whose part of x is in shared memory at a time
};

__device__ __forceinline__ uint4 load_weights(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

template <class M>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The eight codes of a word as four pairs of 16-bit numbers. A code n + 8 in the low bits of 128 (bf16) or 1024 (fp16), less 136 or
// 1032; the fp16 mantissa also holds a code four bits up, which a multiplication by 1/16 brings down.
template <class M>
__device__ __forceinline__ void operands(uint32_t w, uint32_t (&a)[4]);
template <>
__device__ __forceinline__ void operands<__nv_bfloat16>(uint32_t w, uint32_t (&a)[4]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t u = ((w >> (4 * p)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 d = __hsub2(reinterpret_cast<const __nv_bfloat162&>(u), __nv_bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308)));
    a[p] = reinterpret_cast<const uint32_t&>(d);
  }
}
template <>
__device__ __forceinline__ void operands<__half>(uint32_t w, uint32_t (&a)[4]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t v = p < 2 ? w : w >> 8;
    const uint32_t u = (v & (p & 1 ? 0x00F000F0u : 0x000F000Fu)) | 0x64006400u;
    const __half2 h = reinterpret_cast<const __half2&>(u);
    const __half2 d = p & 1 ? __hfma2(h, __half2(__ushort_as_half(0x2C00), __ushort_as_half(0x2C00)), __half2(__ushort_as_half(0xD480), __ushort_as_half(0xD480)))
                            : __hsub2(h, __half2(__ushort_as_half(0x6408), __ushort_as_half(0x6408)));
    a[p] = reinterpret_cast<const uint32_t&>(d);
  }
}

// The three bf16 numbers of an fp32: the upper half of its bits, that of the exact rest, and what is then left (8 bits at most).
// Inf and NaN are their own first part (a NaN stays one: its lower bits may be all that tells it from Inf).
__device__ __forceinline__ void three_parts(float x, uint32_t (&part)[3]) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7F800000u) == 0x7F800000u) {
    part[0] = (u >> 16) | ((u & 0x007FFFFFu) ? 0x40u : 0u);
    part[1] = part[2] = 0;
    return;
  }
  part[0] = u >> 16;
  const float r1 = x - __uint_as_float(u & 0xFFFF0000u);
  part[1] = __float_as_uint(r1) >> 16;
  const float r2 = r1 - __uint_as_float(__float_as_uint(r1) & 0xFFFF0000u);
  part[2] = __float_as_uint(r2) >> 16;
}

// x of the steps [begin, end) into shared memory: 16 bytes (8 columns of one token) at ((unit * columns + column) * 4 + t) * 16,
// unit: 32 columns of the matrix, t: the quarter of them that lanes 4 r + t multiply. Zeros behind the matrix's last column.
template <class X, class M>
__device__ __forceinline__ void stage_x(const MatvecArgs& A, uint32_t first, uint32_t count, uint32_t columns, uint32_t begin, uint32_t end, uint4* xs) {
  const uint32_t units = (end - begin) * 4;
  for (uint32_t i = threadIdx.x; i < units * count * 4; i += kWarps * 32) {
    const uint32_t t = i & 3u, token = (i >> 2) % count, unit = (i >> 2) / count;
    const uint32_t col = begin * kQ4StepCols + unit * 32 + 8 * t;
    const int valid = col >= A.L.cols ? 0 : (int)min(8u, A.L.cols - col);
    const X* p = static_cast<const X*>(A.x) + (uint64_t)(first + token) * A.x_stride + col;
    if constexpr (sizeof(X) == 4) {
      float v[8];
      load8(p, valid, v);
      uint32_t part[8][3];
#pragma unroll
      for (int e = 0; e < 8; ++e) three_parts(v[e], part[e]);
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        uint4 o;
        o.x = part[0][k] | part[1][k] << 16;
        o.y = part[2][k] | part[3][k] << 16;
        o.z = part[4][k] | part[5][k] << 16;
        o.w = part[6][k] | part[7][k] << 16;
        xs[(unit * columns + 3 * token + k) * 4 + t] = o;
      }
    } else {
      uint4 o = make_uint4(0, 0, 0, 0);
      if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        o = __ldg(reinterpret_cast<const uint4*>(p));
      } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
        uint32_t e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = k < valid ? h[k] : 0u;
        o = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
      }
      xs[(unit * columns + token) * 4 + t] = o;
    }
  }
}

template <int G>
struct Step {  // a warp's part of 16 rows and 128 columns
  uint4 w[2];
  uint32_t s[kQ4StepCols / G];
};

template <class X, class M, int NT, int G>
__global__ void __launch_bounds__(kWarps * 32) matvec_kernel(MatvecArgs A) {
  extern __shared__ uint4 smem[];
  constexpr uint32_t kParts = sizeof(X) == 4 ? 3 : 1;
  float* red = reinterpret_cast<float*>(smem);
  uint4* xs = smem + kWarps * 8 * NT * kRedStride / 4;

  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, t = lane & 3;
  const uint32_t tile = blockIdx.x, first = blockIdx.y * A.per_pass;
  const uint32_t count = min(A.per_pass, A.tokens - first), columns = count * kParts;
  const uint8_t* weights = A.q4 + (uint64_t)tile * A.L.steps * kQ4StepBytes + lane * 16;
  const uint32_t* scales = reinterpret_cast<const uint32_t*>(A.q4 + A.L.scales_off) + (uint64_t)tile * A.L.groups * 8 + r;

  auto load = [&](Step<G>& d, uint32_t step) {
    const uint8_t* p = weights + (uint64_t)step * kQ4StepBytes;
    d.w[0] = load_weights(p);
    d.w[1] = load_weights(p + 512);
#pragma unroll
    for (int i = 0; i < (int)kQ4StepCols / G; ++i) d.s[i] = __ldg(scales + (step * (kQ4StepCols / G) + i) * 8);
  };

  float sum[NT][4] = {};
  for (uint32_t begin = 0; begin < A.L.steps; begin += A.chunk_steps) {
    const uint32_t end = min(A.L.steps, begin + A.chunk_steps);
    Step<G> ring[kAhead];
#pragma unroll
    for (uint32_t d = 0; d < kAhead; ++d)
      if (begin + warp + d * kWarps < end) load(ring[d], begin + warp + d * kWarps);
    __syncthreads();
    stage_x<X, M>(A, first, count, columns, begin, end, xs);
    __syncthreads();
    for (uint32_t s0 = begin + warp; s0 < end; s0 += kAhead * kWarps) {
#pragma unroll
      for (uint32_t d = 0; d < kAhead; ++d) {
        const uint32_t step = s0 + d * kWarps;
        if (step < end) {
          float part[NT][4] = {};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t w0 = u & 1 ? ring[d].w[u >> 1].z : ring[d].w[u >> 1].x, w1 = u & 1 ? ring[d].w[u >> 1].w : ring[d].w[u >> 1].y;
            uint32_t a0[4], a1[4];
            operands<M>(w0, a0);
            operands<M>(w1, a1);
            const uint4* xu = xs + ((step - begin) * 4 + u) * columns * 4;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              uint4 b = make_uint4(0, 0, 0, 0);
              if (8 * n + r < columns) b = xu[(8 * n + r) * 4 + t];
              mma<M>(part[n], a0, b.x, b.y);
              mma<M>(part[n], a1, b.z, b.w);
            }
            if (((u + 1) * 32) % G == 0) {
              const uint32_t s = ring[d].s[u * 32 / G];
              const float s_lo = __uint_as_float(s << 16), s_hi = __uint_as_float(s & 0xFFFF0000u);
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                sum[n][0] += s_lo * part[n][0];
                sum[n][1] += s_lo * part[n][1];
                sum[n][2] += s_hi * part[n][2];
                sum[n][3] += s_hi * part[n][3];
                part[n][0] = part[n][1] = part[n][2] = part[n][3] = 0.0f;
              }
            }
          }
          if (step + kAhead * kWarps < end) load(ring[d], step + kAhead * kWarps);
        }
      }
    }
  }

  // the warps' sums, added up in their order
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float* o = red + (warp * 8 * NT + 8 * n + 2 * t) * kRedStride + r;
    o[0] = sum[n][0];
    o[kRedStride] = sum[n][1];
    o[8] = sum[n][2];
    o[kRedStride + 8] = sum[n][3];
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < count * kQ4TileRows; i += kWarps * 32) {
    const uint32_t token = i / kQ4TileRows, row = tile * kQ4TileRows + i % kQ4TileRows;
    if (row >= A.L.rows) continue;
    float y = 0.0f;
#pragma unroll
    for (int k = (int)kParts - 1; k >= 0; --k) {  // the smallest part first
      const float* p = red + (token * kParts + k) * kRedStride + i % kQ4TileRows;
      float v = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < kWarps; ++w) v += p[w * 8 * NT * kRedStride];
      y += v;
    }
    const uint64_t at = (uint64_t)(first + token) * A.out_stride + row;
    if (sizeof(X) == 2 && A.out_type) from_float(y, static_cast<X*>(A.out)[at]);
    else static_cast<float*>(A.out)[at] = y;
  }
}

template <class X, class M, int NT, int G>
cudaError_t launch(MatvecArgs A, uint32_t passes, uint32_t columns, cudaStream_t cs) {
  const size_t red = kWarps * 8 * NT * kRedStride * 4;
  A.chunk_steps = 65536 / (columns * kQ4StepCols * 2);
  if (A.chunk_steps > A.L.steps) A.chunk_steps = A.L.steps ? A.L.steps : 1;
  const size_t smem = red + (size_t)A.chunk_steps * columns * kQ4StepCols * 2;
  static bool raised[kMaxDevices];
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (!raised[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(matvec_kernel<X, M, NT, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)red + 65536);
    if (e != cudaSuccess) return e;
    raised[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(A.L.tiles, passes);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = cs;
  return cudaLaunchKernelEx(&cfg, matvec_kernel<X, M, NT, G>, A);
}

template <class X, class M, int NT>
cudaError_t launch_group(const MatvecArgs& A, uint32_t passes, uint32_t columns, cudaStream_t cs) {
  if (A.L.group == 32) return launch<X, M, NT, 32>(A, passes, columns, cs);
  if (A.L.group == 64) return launch<X, M, NT, 64>(A, passes, columns, cs);
  return launch<X, M, NT, 128>(A, passes, columns, cs);
}

template <class X, class M>
cudaError_t launch_columns(MatvecArgs A, cudaStream_t cs) {
  constexpr uint32_t kParts = sizeof(X) == 4 ? 3 : 1, kMost = 64 / kParts;
  const uint32_t passes = (A.tokens + kMost - 1) / kMost;
  A.per_pass = (A.tokens + passes - 1) / passes;
  const uint32_t columns = A.per_pass * kParts;
  if (columns <= 8) return launch_group<X, M, 1>(A, passes, columns, cs);
  if (columns <= 16) return launch_group<X, M, 2>(A, passes, columns, cs);
  if (columns <= 32) return launch_group<X, M, 4>(A, passes, columns, cs);
  return launch_group<X, M, 8>(A, passes, columns, cs);
}

}  // namespace

cudaError_t launch_q4_matvec(const Q4Layout& L, const uint8_t* q4, const void* x, int type, uint32_t tokens, uint64_t x_stride, void* out, int out_type,
                             uint64_t out_stride, cudaStream_t cs) {
  MatvecArgs A = {};
  A.q4 = q4;
  A.x = x;
  A.out = out;
  A.x_stride = x_stride;
  A.out_stride = out_stride;
  A.L = L;
  A.tokens = tokens;
  A.out_type = out_type;
  if (type == LC_TYPE_F32) return launch_columns<float, __nv_bfloat16>(A, cs);
  if (type == LC_TYPE_BF16) return launch_columns<__nv_bfloat16, __nv_bfloat16>(A, cs);
  return launch_columns<__half, __half>(A, cs);
}

}  // namespace lc
