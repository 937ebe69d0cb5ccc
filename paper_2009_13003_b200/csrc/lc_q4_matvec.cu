// Products of 4-bit weights with the vectors of a few tokens:
//   out[t, r] = sum over groups G of scale[r, G] * (sum over c in G of code[r, c] * x[t, c]).
//
// The weights are read once. The multiplications go to the tensor cores (m16n8k16: 16 rows, 8 tokens, 16 columns), which multiply
// 16-bit numbers exactly and add up in fp32. A group's scale meets the group's sum in fp32, not the codes: code * scale needs 11
// bits, more than bf16 has. An fp32 vector takes three columns of the product: its values cut into three bf16 numbers, 8 bits
// each, whose sum they are, so that nothing of them is lost.
//
// The operands are the codes themselves, signed: a large x under a code of 0 then adds nothing and costs the rest of its group no bits. (With
// code + 8 as operands, which saves an instruction a pair, and 8 times the group's sum of x taken off afterwards, a weight of 7 beside 2^30
// on a zero came out as 0.) They are made of 4-bit codes in as few instructions as can be. In a float's lowest 8 (bf16) or 11 (fp16) bits
// a whole number N stands for N * 2^-133 or N * 2^-24 (subnormal numbers, and the first binade above them, which goes on in the same
// steps): with n = code + 8, a mask takes two n's out of a word for a row r, and the same mask four bits up two 16 n's for row r + 8.
// One fused multiplication then brings a pair into the normal range and takes off 8. One shift, four masks and four multiplications for
// eight codes, exact; a row's sums are in units of kUnit until they are done. A 16-bit x enters as it is; an fp32 one is multiplied by 2^24
// when it is staged, so that its smallest part is a normal bf16 number. Where a sum comes out as Inf or NaN (x holds one, or values of 2^96
// and more, or a result is that large), the warp takes that vector's 16 sums again by plain multiplications (slow_sums).
//
// Measured, the kernel alone over weights that the L2 does not hold: 28672 x 8192 (121 MB) with one bf16 vector 31 us, 3.9 TB/s (with
// code + 8 29 us); with 16 52 us, with 32 92 us; 50257 x 2048 with 16 22 us; 4096 x 25088 with 4 fp32 vectors 28 us; 2048 x 2048 with one
// 3.3 us.
#include <type_traits>

#include "lc_q4.cuh"
#include "../../include/lc_debug.h"

namespace lc {
namespace {

constexpr uint32_t kMaxSplit = 8;       // CTAs of a cluster that share a tile's columns
constexpr uint32_t kSharedPerSM = 227 * 1024;

struct MatvecArgs {
  const uint8_t* q4;
  const void* x;
  void* out;
  uint64_t x_stride, out_stride;
  Q4Layout L;
  uint32_t tokens, per_pass;  // vectors in all, and of one pass (blockIdx.y)
  int out_type;
  uint32_t ways;              // warps of a CTA that share a block of rows
  uint32_t direct;            // 1 if a warp's sums are the results: nothing to add up
  uint32_t stages;            // steps in the ring of a warp
  uint32_t aligned;           // 1 if every vector begins on a 16-byte boundary
  uint32_t slice;             // steps of a CTA: all of them, or its share in the cluster
  uint32_t chunk;             // steps whose part of x is in shared memory at a time
  uint32_t rounds;            // blocks of rows that a group of warps goes through, at most
  FastDiv by_count;           // vectors of a whole pass
};

template <class M>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same, from zero.
template <class M>
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_first<__nv_bfloat16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
template <>
__device__ __forceinline__ void mma_first<__half>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}

// Codes as numbers of type M, in units of 1 / kUnit (row r) and 16 / kUnit (row r + 8): kTimes takes a pair of subnormal numbers there, kMinus
// (a row each) then takes off 8 units. kUp: what an fp32 vector is multiplied by.
template <class M>
struct Unit;
template <>
struct Unit<__nv_bfloat16> {
  static constexpr uint32_t kTimes = 0x7F007F00u, kMinus[2] = {0xBE00BE00u, 0xC000C000u};  // 2^127, -2^-3, -2
  static constexpr float kUnit = 0x1p6f, kUp = 0x1p24f;
};
template <>
struct Unit<__half> {
  static constexpr uint32_t kTimes = 0x78007800u, kMinus[2] = {0xA400A400u, 0xB400B400u};  // 2^15, -2^-6, -2^-2
  static constexpr float kUnit = 0x1p9f;
};
template <class M>
__device__ __forceinline__ uint32_t code_pair(uint32_t tiny, uint32_t minus) {
  uint32_t d;
  if constexpr (std::is_same<M, __half>::value) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(tiny), "r"(Unit<M>::kTimes), "r"(minus));
  else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(tiny), "r"(Unit<M>::kTimes), "r"(minus));
  return d;
}
// The eight codes of a word as four pairs: of row r, of row r + 8, and so for two more columns.
template <class M>
__device__ __forceinline__ void operands(uint32_t w, uint32_t (&a)[4]) {
  a[0] = code_pair<M>(w & 0x000F000Fu, Unit<M>::kMinus[0]);
  a[1] = code_pair<M>(w & 0x00F000F0u, Unit<M>::kMinus[1]);
  w >>= 8;
  a[2] = code_pair<M>(w & 0x000F000Fu, Unit<M>::kMinus[0]);
  a[3] = code_pair<M>(w & 0x00F000F0u, Unit<M>::kMinus[1]);
}

// Eight values of a vector from column `col` on, as they are in memory; zeros behind the last column.
template <class X>
__device__ __forceinline__ void load_piece(const MatvecArgs& A, uint32_t token, uint32_t col, bool there, uint32_t (&raw)[2 * sizeof(X)]) {
  const int valid = !there || col >= A.L.cols ? 0 : (int)min(8u, A.L.cols - col);
  const X* p = static_cast<const X*>(A.x) + (uint64_t)token * A.x_stride + col;
  if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int k = 0; k < (int)sizeof(X) / 2; ++k) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + k);
      raw[4 * k] = v.x, raw[4 * k + 1] = v.y, raw[4 * k + 2] = v.z, raw[4 * k + 3] = v.w;
    }
  } else if constexpr (sizeof(X) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k) raw[k] = k < valid ? __ldg(reinterpret_cast<const uint32_t*>(p) + k) : 0u;
  } else {
    const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) raw[k] = (2 * k < valid ? __ldg(h + 2 * k) : 0u) | (uint32_t)(2 * k + 1 < valid ? __ldg(h + 2 * k + 1) : 0u) << 16;
  }
}

// A piece into shared memory as columns of the product: one, or `stride` apart the three parts of fp32, which are the upper half of its
// bits, that of the exact rest, and what is then left (8 bits at most).
template <class X>
__device__ __forceinline__ void store_piece(const uint32_t (&raw)[2 * sizeof(X)], uint4* to, uint32_t stride) {
  if constexpr (sizeof(X) == 4) {
    uint32_t part[3][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = __uint_as_float(raw[e]) * Unit<__nv_bfloat16>::kUp;
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        part[k][e] = __float_as_uint(v);
        v -= __uint_as_float(part[k][e] & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __byte_perm(part[k][2 * e], part[k][2 * e + 1], 0x7632);
      to[k * stride] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    to[0] = make_uint4(raw[0], raw[1], raw[2], raw[3]);
  }
}

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }
// Waits for all but the latest `left` (at most 4) groups of copies.
__device__ __forceinline__ void copies_wait(uint32_t left) {
  if (left >= 4) copies_wait<4>();
  else if (left == 3) copies_wait<3>();
  else if (left == 2) copies_wait<2>();
  else if (left == 1) copies_wait<1>();
  else copies_wait<0>();
}


// x of the steps [begin, end) into shared memory, one column of the product behind the other: `stride` 16-byte pieces, an odd
// number of units (32 columns of the matrix, four pieces) of which lanes 4 r + t multiply piece t, so that eight columns lie in
// eight different parts of the banks. Zeros behind the matrix's last column. Where the vectors are aligned, a thread first copies its
// pieces as they are (an fp32 piece to where its first two parts will be), all of them on their way at once, and then changes
// them in place; those of 16 bits stay as they are. (The code is short rather than unrolled: in a small product it runs once, and reading it
// from memory takes as long as the loads; with four pieces a turn 2048 x 2048 took 4.9 us, with one 4.1.)
template <class X>
__device__ __forceinline__ void stage_x(const MatvecArgs& A, uint32_t first, uint32_t count, uint32_t begin, uint32_t end, uint32_t stride, uint4* xs, bool copy) {
  constexpr int kParts = sizeof(X) == 4 ? 3 : 1;
  const uint32_t t = threadIdx.x & 3u, step = blockDim.x / 4;
#pragma unroll 1
  for (uint32_t i = threadIdx.x >> 2; i < (end - begin) * 4 * count; i += step) {
    const uint32_t unit = count == A.by_count.d ? A.by_count.div(i) : i / count, token = i - unit * count, col = (begin * 4 + unit) * 32 + 8 * t;
    uint4* to = xs + token * kParts * stride + unit * 4 + t;
    const bool whole = A.aligned && col + 8 <= A.L.cols;
    if (copy) {
      if (!whole) continue;
      const X* from = static_cast<const X*>(A.x) + (uint64_t)(first + token) * A.x_stride + col;
#pragma unroll
      for (int k = 0; k < (int)sizeof(X) / 2; ++k) copy16(shared_address(to + k * stride), reinterpret_cast<const uint4*>(from) + k);
      continue;
    }
    if (whole && sizeof(X) == 2) continue;
    uint32_t raw[2 * sizeof(X)];
    if (whole) {
#pragma unroll
      for (int k = 0; k < (int)sizeof(X) / 2; ++k) {
        const uint4 v = to[k * stride];
        raw[4 * k] = v.x, raw[4 * k + 1] = v.y, raw[4 * k + 2] = v.z, raw[4 * k + 3] = v.w;
      }
    } else {
      load_piece<X>(A, first + token, col, true, raw);
    }
    store_piece<X>(raw, to, stride);
  }
}

// A warp's sums for one vector and rows r and r + 8 of a tile by plain multiplications, in all four lanes of r: what the definition
// says for Inf, NaN and large values.
template <class X>
__device__ __noinline__ float2 slow_sums(const MatvecArgs& A, uint32_t tile, uint32_t token, uint32_t begin, uint32_t end) {
  const uint32_t lane = threadIdx.x & 31, r = lane >> 2, t = lane & 3;
  const X* x = static_cast<const X*>(A.x) + (uint64_t)token * A.x_stride;
  float2 y = make_float2(0.0f, 0.0f);
  for (uint32_t step = begin; step < end; step += A.ways) {
    for (uint32_t h = 0; h < 4; ++h) {
      const uint2 w = __ldg(reinterpret_cast<const uint2*>(A.q4 + ((uint64_t)tile * A.L.steps + step) * kQ4StepBytes + (h / 2) * 512 + lane * 16 + (h & 1) * 8));
      const uint32_t col = step * kQ4StepCols + h * 32 + 8 * t;
      const uint32_t s = __ldg(reinterpret_cast<const uint32_t*>(A.q4 + A.L.scales_off) + ((uint64_t)tile * A.L.groups + col / A.L.group) * 8 + r);
      float2 p = make_float2(0.0f, 0.0f);
      for (uint32_t e = 0; e < 8; ++e) {
        if (col + e >= A.L.cols) break;
        const float v = to_float(x[col + e]);
        const uint32_t n = (e < 4 ? w.x : w.y) >> (16 * (e & 1) + 8 * ((e >> 1) & 1));
        p.x += (float)((int)(n & 15u) - 8) * v;
        p.y += (float)((int)((n >> 4) & 15u) - 8) * v;
      }
      y.x += __uint_as_float(s << 16) * p.x;
      y.y += __uint_as_float(s & 0xFFFF0000u) * p.y;
    }
  }
  __syncwarp();
#pragma unroll
  for (int d = 1; d < 4; d *= 2) {
    y.x += __shfl_xor_sync(0xFFFFFFFFu, y.x, d);
    y.y += __shfl_xor_sync(0xFFFFFFFFu, y.y, d);
  }
  return y;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_in_cluster(float* mine, uint32_t rank, float v) {
  asm volatile("{ .reg .u32 a; mapa.shared::cluster.u32 a, %0, %1; st.shared::cluster.f32 [a], %2; }" ::"r"(shared_address(mine)), "r"(rank), "f"(v) : "memory");
}

// Shared memory: the warps' rings, their sums, what the cluster's CTAs send each other, x.
template <int NT, int MT, int G>
struct Shared {
  static constexpr uint32_t kGroups = kQ4StepCols / G, kSlot = kQ4StepBytes + kGroups * 32, kStage = MT * kSlot;  // codes and scales of a step
  static constexpr uint32_t kRows = MT * kQ4TileRows, kRedStride = kRows + 4;  // floats from column to column: the lanes of a store meet in no bank
  static __host__ __device__ __forceinline__ uint32_t part_tokens(uint32_t per_pass, uint32_t split) { return split > 1 ? (per_pass + split - 1) / split : 0; }
  static __host__ __device__ __forceinline__ uint32_t red(bool direct, uint32_t warps, uint32_t columns) { return direct ? 0 : warps * columns * kRedStride * 4; }
  static __host__ __device__ __forceinline__ uint32_t part(uint32_t groups, uint32_t split, uint32_t per_pass) {  // [2][groups][split][part_tokens][kRows] floats
    return 2 * groups * split * part_tokens(per_pass, split) * kRows * 4;
  }
  static __host__ __device__ __forceinline__ uint64_t x(uint32_t columns, uint32_t steps) { return (uint64_t)columns * (steps * 256 + 64); }
};
constexpr uint32_t kMostWarps = 16;  // on an SM, by their registers

// The `ways` warps of a group share a block of MT tiles of 16 rows: they deal its steps (128 columns) among themselves, each with a ring
// of steps in flight in shared memory that goes on from one block to the next. x is staged once, if the slice's part of it fits.
// kSplit: the CTAs of a cluster have a slice of the columns each.
template <class X, class M, int NT, int MT, int G, bool kSplit>
__global__ void __launch_bounds__(kMostWarps * 32, 1) matvec_kernel(const __grid_constant__ MatvecArgs A) {
  extern __shared__ uint4 smem[];
  using S = Shared<NT, MT, G>;
  constexpr uint32_t kParts = sizeof(X) == 4 ? 3 : 1, kGroups = S::kGroups, kRows = S::kRows, kRedStride = S::kRedStride;
  constexpr uint32_t kSlot = S::kSlot, kStage = S::kStage;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, r = lane >> 2, t = lane & 3;
  const uint32_t way = warp & (A.ways - 1), groups = warps / A.ways, group = warp / A.ways;
  uint32_t split = 1, rank = 0;
  if constexpr (kSplit) {
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    cluster_arrive();  // the others' shared memory may be written once they have begun
  }
  const uint32_t first = blockIdx.y * A.per_pass, count = min(A.per_pass, A.tokens - first), columns = count * kParts;
  const uint32_t slice = min(rank * A.slice, A.L.steps), slice_end = min(slice + A.slice, A.L.steps);
  const uint32_t clusters = gridDim.x / split, slots = clusters * groups, blocks = (A.L.tiles + MT - 1) / MT;
  uint32_t block = group * clusters + blockIdx.x / split;

  uint8_t* base = reinterpret_cast<uint8_t*>(smem);
  const uint32_t ring_bytes = A.stages * kStage;
  uint8_t* ring = base + warp * ring_bytes;
  float* red = reinterpret_cast<float*>(base + warps * ring_bytes);
  const uint32_t part_tokens = S::part_tokens(A.per_pass, split), red_columns = A.per_pass * kParts;
  float* part = red + S::red(A.direct, warps, red_columns) / 4;
  uint4* xs = reinterpret_cast<uint4*>(part + S::part(groups, split, A.per_pass) / 4);
  const uint32_t x_stride = A.chunk * 16 + 4;
  const bool resident = A.chunk >= A.slice;
  if (resident && A.aligned) stage_x<X>(A, first, count, slice, slice_end, x_stride, xs, true);
  copies_end();

  // the next step to ask for: where it is, and how many there are left of this block and in all
  const uint32_t turns = slice + way < slice_end ? (slice_end - slice - way + A.ways - 1) / A.ways : 0;
  uint32_t left = block < blocks ? ((blocks - block + slots - 1) / slots) * turns : 0, left_block = turns, ask_slot = 0;
  const uint8_t* codes = A.q4 + ((uint64_t)block * MT * A.L.steps + slice + way) * kQ4StepBytes + lane * 16;
  const uint8_t* scales = A.q4 + A.L.scales_off + (((uint64_t)block * MT * A.L.groups + (slice + way) * kGroups + t) * 8 + r) * 4;
  const uint64_t tile_codes = (uint64_t)A.L.steps * kQ4StepBytes, tile_scales = (uint64_t)A.L.groups * 32;
  const uint64_t next_block = MT * slots * tile_codes - (uint64_t)turns * A.ways * kQ4StepBytes;
  const uint64_t next_block_scales = MT * slots * tile_scales - (uint64_t)turns * A.ways * kGroups * 32;
  const uint32_t ring_at = shared_address(ring) + lane * 16, ring_scales = shared_address(ring) + kQ4StepBytes + (t * 8 + r) * 4;
  uint32_t ask_tiles = A.L.tiles - block * MT;  // of this block, if it is the matrix's last
  auto ask_next = [&]() {
    if (left != 0) {
#pragma unroll
      for (uint32_t m = 0; m < MT; ++m) {
        if (m > 0 && ask_tiles <= m) break;  // the last block may be half a one
        const uint32_t to = ask_slot + m * kSlot;
        copy16(ring_at + to, codes + m * tile_codes);
        copy16(ring_at + to + 512, codes + m * tile_codes + 512);
        if (t < kGroups) copy4(ring_scales + to, scales + m * tile_scales);
      }
      --left;
      codes += A.ways * kQ4StepBytes;
      scales += A.ways * kGroups * 32;
      if (--left_block == 0) {
        left_block = turns;
        codes += next_block;
        scales += next_block_scales;
        ask_tiles -= MT * slots;
      }
      ask_slot = ask_slot + kStage == ring_bytes ? 0 : ask_slot + kStage;
    }
    copies_end();
  };
  for (uint32_t i = 1; i < A.stages; ++i) ask_next();

  if constexpr (kSplit) {
    __syncwarp();
    cluster_wait();
  }
  const uint4* column[NT];  // this lane's column of each eight; column 0 for those that are not there, whose sums nobody takes
#pragma unroll
  for (int n = 0; n < NT; ++n) column[n] = xs + (8 * n + r < columns ? 8 * n + r : 0) * x_stride + t;

  uint32_t slot = 0;
  for (uint32_t round = 0; round < A.rounds; ++round, block += slots) {
    const bool there = block < blocks;
    float* mine = red + warp * red_columns * kRedStride;
    auto put = [&](uint32_t token, uint32_t row, float y) {
      row += block * kRows;
      if (row >= A.L.rows) return;
      const uint64_t at = (uint64_t)(first + token) * A.out_stride + row;
      if (sizeof(X) == 2 && A.out_type) from_float(y, static_cast<X*>(A.out)[at]);
      else static_cast<float*>(A.out)[at] = y;
    };
    Two sum[MT][NT][2] = {};  // of rows r and r + 8, two columns each
    for (uint32_t begin = slice; begin < slice_end; begin += A.chunk) {
      const uint32_t end = min(slice_end, begin + A.chunk);
      if (!resident || round == 0) {
        if (!resident) {
          __syncthreads();
          if (A.aligned) stage_x<X>(A, first, count, begin, end, x_stride, xs, true);
          copies_end();
          copies_wait<0>();
        } else {
          copies_wait(A.stages - 1);
        }
        if (kParts > 1 || !A.aligned || A.L.cols % kQ4StepCols != 0) stage_x<X>(A, first, count, begin, end, x_stride, xs, false);
        __syncthreads();
      }
      if (!there) continue;
#pragma unroll 1
      for (uint32_t step = begin + way; step < end; step += A.ways) {
        copies_wait(A.stages - 2);
        __syncwarp();  // the scales of a row are copied by its four lanes; and all lanes have left the slot asked for now
        ask_next();
        const uint8_t* w = ring + slot;
        slot = slot + kStage == ring_bytes ? 0 : slot + kStage;
        float acc[MT][NT][4];
        const uint32_t at = (step - begin) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 v[MT];
#pragma unroll
          for (int m = 0; m < MT; ++m) v[m] = *reinterpret_cast<const uint4*>(w + m * kSlot + h * 512 + lane * 16);
#pragma unroll
          for (int u = 2 * h; u < 2 * h + 2; ++u) {
            const bool begins = u * 32 % G == 0, ends = (u + 1) * 32 % G == 0;  // a group
            uint32_t a[MT][2][4];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              operands<M>(u & 1 ? v[m].z : v[m].x, a[m][0]);
              operands<M>(u & 1 ? v[m].w : v[m].y, a[m][1]);
            }
            constexpr int kSide = NT < 2 ? 1 : 2;  // eights of columns at a time: products that do not wait for each other
#pragma unroll
            for (int n0 = 0; n0 < NT; n0 += kSide) {
              uint4 b[kSide];
#pragma unroll
              for (int i = 0; i < kSide; ++i) b[i] = column[n0 + i][at + u * 4];
#pragma unroll
              for (int i = 0; i < kSide; ++i) {
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                  if (begins) mma_first<M>(acc[m][n0 + i], a[m][0], b[i].x, b[i].y);
                  else mma<M>(acc[m][n0 + i], a[m][0], b[i].x, b[i].y);
                }
              }
#pragma unroll
              for (int i = 0; i < kSide; ++i) {
#pragma unroll
                for (int m = 0; m < MT; ++m) mma<M>(acc[m][n0 + i], a[m][1], b[i].z, b[i].w);
              }
            }
            if (ends) {
#pragma unroll
              for (int m = 0; m < MT; ++m) {
                const uint32_t s = *reinterpret_cast<const uint32_t*>(w + m * kSlot + kQ4StepBytes + (u * 32 / G * 8 + r) * 4);
                const float s_lo = __uint_as_float(s << 16), s_hi = __uint_as_float(s & 0xFFFF0000u);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                  sum[m][n][0] = fma_two(two(s_lo, s_lo), two(acc[m][n][0], acc[m][n][1]), sum[m][n][0]);
                  sum[m][n][1] = fma_two(two(s_hi, s_hi), two(acc[m][n][2], acc[m][n][3]), sum[m][n][1]);
                }
              }
            }
          }
        }
      }
    }
    if (there) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        if (m > 0 && block * MT + m >= A.L.tiles) break;
        constexpr float kLow = kParts == 1 ? Unit<M>::kUnit : Unit<M>::kUnit / Unit<__nv_bfloat16>::kUp;  // row r + 8: a sixteenth
        float y[NT][4];
        uint32_t bad = 0;  // bit 2 n + i: a sum of column 8 n + 2 t + i is Inf or NaN
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            split_two(mul_two(sum[m][n][i / 2], i == 0 ? two(kLow, kLow) : two(kLow / 16, kLow / 16)), y[n][i], y[n][i + 1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) bad |= fabsf(y[n][i + k]) < __uint_as_float(0x7F800000u) ? 0u : 1u << (2 * n + k);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t col = 8 * n + 2 * t + (i & 1), row = m * 16 + r + 8 * (i >> 1);
            if (col >= columns) continue;
            if (kParts == 1 && A.direct) put(col, row, y[n][i]);
            else mine[col * kRedStride + row] = y[n][i];
          }
        }
        if (!__any_sync(0xFFFFFFFFu, bad != 0)) continue;
        for (int d = 4; d < 32; d *= 2) bad |= __shfl_xor_sync(0xFFFFFFFFu, bad, d);
        for (uint32_t token = 0; token < count; ++token) {  // those vectors alone: the others keep their sums
          uint32_t again = 0;
          for (uint32_t col = token * kParts; col < (token + 1) * kParts; ++col) again |= __shfl_sync(0xFFFFFFFFu, bad, (col & 7) / 2) >> (2 * (col / 8) + (col & 1)) & 1u;
          if (!again) continue;
          const float2 z = slow_sums<X>(A, block * MT + m, first + token, slice + way, slice_end);  // behind a __syncwarp: after the stores above
          const uint32_t row = m * 16 + r;
          if (kParts == 1 && A.direct) {
            if (t == 0) put(token, row, z.x), put(token, row + 8, z.y);
          } else if (t < kParts) {
            mine[(token * kParts + t) * kRedStride + row] = t == 0 ? z.x : 0.0f;
            mine[(token * kParts + t) * kRedStride + row + 8] = t == 0 ? z.y : 0.0f;
          }
        }
      }
    }

    // the warps' sums, added up in their order, then those of the cluster's CTAs
    if (kParts == 1 && A.direct) continue;
    auto group_barrier = [&]() {
      if (A.ways == 1) __syncwarp();
      else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(A.ways * 32) : "memory");
    };
    group_barrier();
    if (there) {
      const uint32_t row = lane % kRows;  // the lanes of a warp take as many vectors side by side as they are times the rows
      for (uint32_t token = (way * 32 + lane) / kRows; token < count; token += A.ways * 32 / kRows) {
        float y = 0.0f;
#pragma unroll
        for (int k = (int)kParts - 1; k >= 0; --k) {  // the smallest part first
          const float* p = red + (group * A.ways * red_columns + token * kParts + k) * kRedStride + row;
          float v = 0.0f;
          for (uint32_t w = 0; w < A.ways; ++w, p += red_columns * kRedStride) v += *p;
          y += v;
        }
        if constexpr (kSplit) store_in_cluster(part + ((((round & 1) * groups + group) * split + rank) * part_tokens + token / split) * kRows + row, (token + round) % split, y);
        else put(token, row, y);
      }
    }
    if constexpr (kSplit) {
      __syncwarp();
      cluster_arrive();  // also ends the reads of `red`
      cluster_wait();
      if (there) {
        for (uint32_t i = way * 32 + lane; i < part_tokens * kRows; i += A.ways * 32) {
          const uint32_t token = i / kRows * split + (rank + split - round % split) % split, row = i % kRows;
          if (token >= count) continue;
          float y = 0.0f;
          for (uint32_t s = 0; s < split; ++s) y += part[(((round & 1) * groups + group) * split + s) * part_tokens * kRows + i];
          put(token, row, y);
        }
        __syncwarp();
      }
    } else {
      group_barrier();
    }
  }
  copies_wait<0>();
}

uint32_t ctas_per_sm(uint32_t warps, uint32_t smem) { return warps * 2 <= kMostWarps && smem <= kSharedPerSM / 2 - 1024 ? 2 : 1; }

template <class X, class M, int NT, int MT, int G, bool kSplit>
cudaError_t launch_split(MatvecArgs A, uint32_t blocks, uint32_t passes, uint32_t split, uint32_t warps, uint32_t smem, uint32_t sms, cudaStream_t cs) {
  const auto kernel = matvec_kernel<X, M, NT, MT, G, kSplit>;
  static bool raised[kMaxDevices];
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  cudaError_t e;
  if (!raised[dev]) {
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedPerSM)) != cudaSuccess) return e;
    raised[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(split, passes);
  cfg.blockDim = dim3(warps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = cs;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = split;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  int fit = (int)(sms * ctas_per_sm(warps, smem));  // clusters that the device holds at once
  if (kSplit) {
    cfg.numAttrs = 1;
    if ((e = cudaOccupancyMaxActiveClusters(&fit, kernel, &cfg)) != cudaSuccess) return e;  // 0.2 us
    if (fit < 1) return cudaErrorInvalidConfiguration;
  }
  const uint32_t groups = warps / A.ways, fill = (blocks + groups - 1) / groups;
  const uint32_t clusters = (uint32_t)fit < fill ? (uint32_t)fit : fill;
  A.rounds = (blocks + clusters * groups - 1) / (clusters * groups);
  cfg.gridDim.x = clusters * split;
  return cudaLaunchKernelEx(&cfg, kernel, A);
}

// How a product is laid out over the device.
struct Plan {
  uint32_t mt, ways, split, warps, stages, slice, chunk, direct, smem;
};

// The areas of Shared, and 4 bytes for each group and column of the product that stay free behind them.
uint64_t plan_bytes(const Plan& p, uint32_t nt, uint32_t group, uint32_t per_pass, uint32_t parts, uint32_t steps) {
  const uint32_t columns = per_pass * parts, rows = p.mt * kQ4TileRows, groups = kQ4StepCols / group;
  const uint32_t stage = p.mt * (kQ4StepBytes + groups * 32), part_tokens = p.split > 1 ? (per_pass + p.split - 1) / p.split : 0;
  return (uint64_t)p.warps * p.stages * stage + (p.direct ? 0 : (uint64_t)p.warps * columns * (rows + 4) * 4) +
         (uint64_t)2 * (p.warps / p.ways) * p.split * part_tokens * rows * 4 + (uint64_t)steps * groups * 8 * nt * 4 + (uint64_t)columns * (steps * 256 + 64);
}

// About how many cycles a layout takes: a step takes a warp `alone` cycles and an SM with all its warps `busy`; every CTA stages x; the
// sums of a round of blocks are added up behind it. The numbers were fitted to 37 shapes of 1 to 40 vectors in up to 64 layouts each,
// with a loop that made its operands in fewer instructions. What the rule takes is now 5.6 % slower than the fastest of them (geometric mean; 17 %
// at most, but for x of over 16 vectors 33 %), and 6.4 % over 30 other shapes (19 % at most). Numbers fitted anew to both came to 5 to 6 %
// over shapes that they had not seen.
constexpr uint32_t kStepAlone[2][3] = {{825, 1130, 1750}, {1270, 1800, 3000}}, kStepBusy[2][3] = {{71, 110, 200}, {130, 190, 390}};
uint64_t plan_cycles(const Plan& p, uint32_t nt_log, uint32_t tiles, uint32_t per_pass, uint32_t parts, uint32_t sms) {
  const uint32_t per_sm = ctas_per_sm(p.warps, p.smem);
  // clusters of 2, 4 and 8 on 148 SMs with one CTA each: 74, 33 and 15
  const uint32_t clusters = sms * per_sm * (p.split <= 2 ? 148 / p.split : p.split == 4 ? 33 : 15) / 148;
  const uint32_t groups = p.warps / p.ways, rows = p.mt * kQ4TileRows, blocks = (tiles + p.mt - 1) / p.mt, slots = (clusters ? clusters : 1) * groups;
  const uint32_t steps = (p.slice + p.ways - 1) / p.ways, alone = kStepAlone[p.mt - 1][nt_log], busy = kStepBusy[p.mt - 1][nt_log];
  const uint32_t sums = 300 + per_pass * rows * (20 + 6 * p.ways * parts) / (32 * p.ways) + (p.split == 1 ? 0 : p.split == 2 ? 1160 : p.split == 4 ? 1400 : 2000);
  auto round = [&](uint32_t used) {  // blocks of a round
    const uint32_t warps = (uint32_t)(((uint64_t)used * p.ways * p.split + sms - 1) / sms), all = p.warps * per_sm;
    const uint32_t together = (warps < all ? warps : all) * busy;
    return (uint64_t)steps * (together > alone ? together : alone) + sums;
  };
  // 32 pieces of x at a time; what does not fit comes again with every round, but then enough of it is on its way
  const bool resident = p.chunk >= p.slice;
  const uint64_t staged = (uint64_t)(resident ? per_sm : blocks / slots + 1) * (p.slice * (uint64_t)per_pass / 2) * (parts == 3 ? 90 : resident ? 50 : 20);
  return staged + (p.split > 1 ? 950 : 0) + blocks / slots * round(slots) + (blocks % slots ? round(blocks % slots) : 0);
}

Plan plan_pass(uint32_t nt_log, const Q4Layout& L, uint32_t per_pass, uint32_t parts, uint32_t sms, uint64_t& least) {
  const uint32_t nt = 1u << nt_log;
  Plan best = {};
  least = ~0ull;
  for (uint32_t mt = nt_log == 2 ? 2 : 1; mt <= 2; ++mt) {
    const uint32_t blocks = (L.tiles + mt - 1) / mt;
    if (mt == 2 && L.tiles <= sms && best.smem) break;  // too few tiles to put two together
    for (uint32_t split = 1; split <= kMaxSplit; split *= 2) {
      if (split > 1 && L.steps < 8 * split && best.smem && best.chunk >= best.slice) break;  // too few columns to share
      for (uint32_t ways = 1; ways <= 8; ways *= 2) {
        const uint32_t slice = L.steps ? (L.steps + split - 1) / split : 1, shared = blocks * ways * split;  // warps that there is work for
        if (ways > 1 && (slice < ways || shared / 2 > sms * kMostWarps * 2)) break;  // nothing to share, or no need to
        if (shared < sms && ways < 8 && slice >= 2 * ways) continue;
        Plan p = {mt, ways, split, shared > sms * 8 ? 16u : 8u, mt == 1 ? 6u : 3u, slice, 0, ways == 1 && split == 1 && parts == 1, 0};
        p.chunk = p.slice;
        uint64_t bytes = plan_bytes(p, nt, L.group, per_pass, parts, p.chunk);
        if (bytes > kSharedPerSM) {
          p.warps = 8;
          if (mt == 1) p.stages = 4;
          if ((bytes = plan_bytes(p, nt, L.group, per_pass, parts, p.chunk)) > kSharedPerSM) {  // x in parts: whole turns of the warps
            const uint64_t fixed = plan_bytes(p, nt, L.group, per_pass, parts, 0), step = plan_bytes(p, nt, L.group, per_pass, parts, 1) - fixed;
            p.chunk = fixed >= kSharedPerSM ? 0 : (uint32_t)((kSharedPerSM - fixed) / step) / ways * ways;
            if (p.chunk == 0) continue;
            bytes = plan_bytes(p, nt, L.group, per_pass, parts, p.chunk);
          }
        }
        p.smem = (uint32_t)bytes;
        const uint64_t cycles = plan_cycles(p, nt_log, L.tiles, per_pass, parts, sms);
        if (cycles < least) least = cycles, best = p;
      }
    }
  }
  return best;
}

// Of a product's vectors: how many go in a pass, and the logarithm of the eights of columns that it then has. A pass of 32 columns reads the
// weights half as often, but has x and sums for fewer warps: 50257 x 2048 with 32 vectors 66 us, in passes of 16 41; 500 x 9000 with 64 16 and
// 29 us. So make_plan takes the width whose passes take fewer cycles: over 39 shapes that the rule was not made on 3 % off the faster of the two
// (33 % at most), where 32 columns always are 13 % off and 16 are 8 %.
uint32_t tokens_per_pass(uint32_t tokens, uint32_t parts, uint32_t columns) {
  const uint32_t most = columns / parts, passes = (tokens + most - 1) / most;
  return (tokens + passes - 1) / passes;
}
uint32_t eights_log(uint32_t columns) { return columns <= 8 ? 0 : columns <= 16 ? 1 : 2; }
constexpr uint32_t kMostTokens = 1u << 18;  // of a launch: 52429 passes of 5 fp32 vectors, where a grid has 65535 rows

Plan make_plan(const Q4Layout& L, uint32_t tokens, uint32_t parts, uint32_t sms, uint32_t& per_pass, uint32_t& nt_log) {
  Plan best = {};
  uint64_t least = ~0ull;
  for (uint32_t columns = tokens * parts <= 16 ? 16 : 32; columns >= 16; columns /= 2) {
    const uint32_t per = tokens_per_pass(tokens, parts, columns), log = eights_log(per * parts);
    uint64_t cycles;
    const Plan p = plan_pass(log, L, per, parts, sms, cycles);
    if (p.smem == 0) continue;
    // passes that do not fill the device run side by side
    const uint64_t slots = p.warps / p.ways, blocks = (L.tiles + p.mt - 1) / p.mt, room = (uint64_t)sms * ctas_per_sm(p.warps, p.smem);
    const uint64_t wanted = (blocks + slots - 1) / slots * p.split, used = wanted < room ? wanted : room, passes = (tokens + per - 1) / per;
    const uint64_t all = cycles * ((passes * used + room - 1) / room);
    if (all < least) least = all, best = p, per_pass = per, nt_log = log;
  }
  return best;
}

template <class X, class M, int NT, int MT, int G>
cudaError_t launch(const MatvecArgs& A, const Plan& p, uint32_t passes, uint32_t sms, cudaStream_t cs) {
  const uint32_t blocks = (A.L.tiles + MT - 1) / MT;
  return p.split > 1 ? launch_split<X, M, NT, MT, G, true>(A, blocks, passes, p.split, p.warps, p.smem, sms, cs)
                     : launch_split<X, M, NT, MT, G, false>(A, blocks, passes, 1, p.warps, p.smem, sms, cs);
}

template <class X, class M, int NT, int MT>
cudaError_t launch_group(const MatvecArgs& A, const Plan& p, uint32_t passes, uint32_t sms, cudaStream_t cs) {
  if (A.L.group == 32) return launch<X, M, NT, MT, 32>(A, p, passes, sms, cs);
  if (A.L.group == 64) return launch<X, M, NT, MT, 64>(A, p, passes, sms, cs);
  return launch<X, M, NT, MT, 128>(A, p, passes, sms, cs);
}

template <class X, class M>
cudaError_t launch_columns(MatvecArgs A, cudaStream_t cs) {
  constexpr uint32_t kParts = sizeof(X) == 4 ? 3 : 1;
  A.aligned = (reinterpret_cast<uintptr_t>(A.x) & 15) == 0 && (A.tokens == 1 || A.x_stride % (16 / sizeof(X)) == 0);
  static int count[kMaxDevices];  // SMs
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (count[dev] == 0) {
    int n = 0;
    const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    count[dev] = n;
  }
  const uint32_t sms = (uint32_t)count[dev];
  uint32_t nt_log = 0;
  const Plan p = make_plan(A.L, A.tokens, kParts, sms, A.per_pass, nt_log);
  if (p.smem == 0) return cudaErrorInvalidConfiguration;
  const uint32_t passes = (A.tokens + A.per_pass - 1) / A.per_pass;
  A.by_count = FastDiv(A.per_pass);
  A.ways = p.ways;
  A.direct = p.direct;
  A.stages = p.stages;
  A.slice = p.slice;
  A.chunk = p.chunk;
  if (nt_log == 0) return p.mt == 2 ? launch_group<X, M, 1, 2>(A, p, passes, sms, cs) : launch_group<X, M, 1, 1>(A, p, passes, sms, cs);
  if (nt_log == 1) return p.mt == 2 ? launch_group<X, M, 2, 2>(A, p, passes, sms, cs) : launch_group<X, M, 2, 1>(A, p, passes, sms, cs);
  return launch_group<X, M, 4, 2>(A, p, passes, sms, cs);
}

}  // namespace

cudaError_t launch_q4_matvec(const Q4Layout& L, const uint8_t* q4, const void* x, int type, uint32_t tokens, uint64_t x_stride, void* out, int out_type,
                             uint64_t out_stride, cudaStream_t cs) {
  MatvecArgs A = {};
  A.q4 = q4;
  A.x_stride = x_stride;
  A.out_stride = out_stride;
  A.L = L;
  A.out_type = out_type;
  for (uint32_t first = 0; first < tokens; first += kMostTokens) {
    A.x = static_cast<const uint8_t*>(x) + first * x_stride * type_bytes(type);
    A.out = static_cast<uint8_t*>(out) + first * out_stride * type_bytes(out_type);
    A.tokens = tokens - first < kMostTokens ? tokens - first : kMostTokens;
    const cudaError_t e = type == LC_TYPE_F32    ? launch_columns<float, __nv_bfloat16>(A, cs)
                          : type == LC_TYPE_BF16 ? launch_columns<__nv_bfloat16, __nv_bfloat16>(A, cs)
                                                 : launch_columns<__half, __half>(A, cs);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace lc

// Declared in include/lc_debug.h: how a product is laid out, for the test of its bounds.
extern "C" int lc_debug_q4_plan(uint64_t rows, uint64_t cols, int group, int type, uint32_t tokens, uint32_t sms, uint32_t* plan) {
  using namespace lc;
  if (!plan || !group_ok(group) || !type_ok(type) || tokens == 0 || sms == 0 || rows == 0 || rows >= (1ull << 31) || cols >= (1ull << 31) - kQ4StepCols)
    return LC_ERR_ARG;
  uint32_t per_pass = 0, nt_log = 0;
  const Plan p = make_plan(q4_layout(rows, cols, group), tokens < kMostTokens ? tokens : kMostTokens, type == LC_TYPE_F32 ? 3 : 1, sms, per_pass, nt_log);
  const uint32_t values[LC_Q4_PLAN_WORDS] = {per_pass, 1u << nt_log, p.mt, p.ways, p.split, p.warps, p.stages, p.slice, p.chunk, p.direct, p.smem};
  for (int i = 0; i < LC_Q4_PLAN_WORDS; ++i) plan[i] = values[i];
  return LC_OK;
}
