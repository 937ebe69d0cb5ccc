// Attention of new tokens to what a quantised cache holds, read where it lies.
//
//   t(i, p) = scale * q_i . k_p, capped: cap * tanh(t / cap), less slope * |i - p|
//   out_i   = sum over the p that i sees of exp(t(i, p)) v_p / sum of exp(t(i, p)), or 0 if it sees none
//
// in one pass over the keys, with a running maximum and sum of each query (a block of keys whose scores exceed the maximum so far scales
// what there is down by exp of the difference). Work is (sequence, block of queries of one head of the cache, tile of 128 or 64 keys); all tiles of a call
// are dealt out evenly, so that one long sequence keeps all SMs busy like many short ones. A CTA's first and last block may be shared with
// its neighbours: those go to the workspace as sums with their maxima, and a second launch joins them in a fixed order.
//
// A warp holds 32 or 16 keys of a tile and multiplies codes, not values: keys are the rows of the product (m16n8k16), 8 queries its columns, and
// the values' product is transposed the same way, so that a code becomes an operand once for 8 ... 32 queries. The codes become
// bf16 numbers by a mask and one fused multiplication for two of them, exactly: in a bf16 number's lowest 8 bits a whole number N stands
// for N * 2^-133 (subnormals, and the first binade above, in the same steps). Queries of more than 8 bits enter as the bf16 parts that they
// are the sum of: fp16 two, fp32 three. A group's scale meets the key's sums in fp32, and the value's scale the probability ahead of its
// rounding to as many parts; so nothing of the cache is rounded, and a scale's magnitude, NaN in a key that a query does not
// see, or a type's range cost nothing (up to sums of values beyond fp32's range). Probabilities of bf16 queries have 8 bits, of fp16 16, of fp32 24; sums are fp32.
#pragma once

#include "lc_attend.cuh"

namespace lc {
namespace {

constexpr uint32_t kWarps = 4, kThreads = 32 * kWarps;
// Products of 16 keys that a warp has at a time: two, where registers and shared memory allow it, since what a step costs beyond its products is then paid half as
// often (a maximum over eight lanes for each query, the places of its keys, waits).
template <int NB, int NT>
constexpr int kProducts = NB <= 4 && NT <= 2 ? 2 : 1;
template <int NB, int NT>
constexpr uint32_t kTileKeys = 16 * kProducts<NB, NT> * kWarps;  // of a CTA's step: the unit in which keys are dealt out
constexpr float kUnit = 64.0f;  // operands are codes / kUnit
constexpr float kSlack = 8.0f;  // a maximum is raised once the scores exceed it by a factor of 2^kSlack: sums are fp32 and have room for that

template <int kParts>
struct Query;
template <>
struct Query<1> { using T = __nv_bfloat16; };
template <>
struct Query<2> { using T = __half; };
template <>
struct Query<3> { using T = float; };

__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two whole numbers below 256 in the halves' low bits (kHigh: 16 times as large, from the four bits above), less 2^(bits - 1), as bf16 numbers / kUnit.
template <int kBits, bool kHigh>
__device__ __forceinline__ uint32_t operand(uint32_t pair) {
  constexpr uint32_t times = kHigh ? 0x7D007D00u : 0x7F007F00u, minus = kBits == 4 ? 0xBE00BE00u : 0xC000C000u;  // 2^123, 2^127; -2^-3, -2
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(pair), "r"(times), "r"(minus));
  return d;
}
__device__ __forceinline__ uint32_t two_bf16(float low, float high) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(high), "f"(low));
  return r;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ float bf16_float(unsigned short x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_scales(uint32_t to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Which of a tile's 16 keys a row of the product is: bytes of 8-bit codes then lie in different banks both for the keys' operands (lanes of
// neighbouring rows) and for the values' (lanes of every second row).
template <int kBits>
__device__ __forceinline__ uint32_t key_of(uint32_t row) { return kBits == 8 ? row ^ ((row >> 2) & 1) : row; }

// Shared memory of a CTA, in bytes. The rings of the warps and, once a block is done, the sums that the warps add up share their place.
template <int kBits, int NB, int NT, int kParts>
struct Shape {
  static constexpr int M = kProducts<NB, NT>;
  static constexpr uint32_t kKeys = 16 * M, kTile = kTileKeys<NB, NT>;  // of a warp's step, of the CTA's
  static constexpr uint32_t kBlockBytes = 32 * kBits / 8;  // of 32 codes
  // Rows of 128 bytes and more lie as they are, their 16 bytes swapped among each other by the key (place_in), shorter ones 16 (4 bits) or 32 (8 bits) times an
  // odd number of bytes apart: see key_of.
  static constexpr bool kSwapped = NB * kBlockBytes >= 128;
  static constexpr uint32_t kPitch = kSwapped ? NB * kBlockBytes : kBits == 4 ? (NB * kBlockBytes / 16 | 1) * 16 : (NB * kBlockBytes / 32 | 1) * 32;
  static constexpr uint32_t kScaleWords = NB / 2 + 1;  // of a key's row of scales, which may begin in the middle of a word
  static constexpr uint32_t kScales = 2 * kKeys * kPitch;        // where a stage's scales begin: a row's words, the keys' then the values'
  static constexpr uint32_t kParity = kScales + 2 * kKeys * 4 * kScaleWords;  // which of them begin in the middle of a word: a bit for each key, and each value
  static constexpr uint32_t kStage = (kParity + 16 + 255) / 256 * 256;
  static constexpr uint32_t kStages = 2;  // CTAs on an SM bring more than stages: with three, a CTA less fits
  static constexpr uint32_t kColumns = 8 * NT;
  static constexpr uint32_t kQueryPitch = (NB * 64 / 64 | 1) * 64;  // an odd number of times 64 bytes: four lanes' 16 bytes of two neighbouring columns fill all banks
  static constexpr uint32_t kQueries = (kParts * kColumns * kQueryPitch + 255) / 256 * 256;
  static constexpr uint32_t kSumPitch = NB * 32 + 4;  // floats
  static constexpr uint32_t kRing = kWarps * kStages * kStage, kSums = kWarps * kColumns * kSumPitch * 4;
  static constexpr uint32_t kWhole = kQueries + (kRing > kSums ? kRing : kSums);
  static constexpr uint32_t kPart = kColumns * (NB * 32 + 2);  // floats of a partial result
};

// How the tiles of a call are dealt out: `share` of them to each CTA, one behind the other. (Or, if sequences are so short that joining costs more than it
// gains, whole blocks: kWholeRoom.)
__device__ __forceinline__ uint64_t share_of(uint64_t tiles, uint32_t ctas, bool whole) {
  const uint64_t share = (tiles + ctas - 1) / ctas;
  return share < 2 && !whole ? 2 : share;
}
constexpr uint64_t kWholeRoom = 512;

// kWide: 4 bits, groups of 64 values or more: a word of eight values may be dealt to products of 64 rows.
template <int kBits, int NB, int NT, int kParts, bool kWide>
struct Kernel {
  using S = Shape<kBits, NB, NT, kParts>;
  using T = typename Query<kParts>::T;
  static constexpr int M = S::M;
  static constexpr uint32_t kKeys = S::kKeys, kTile = S::kTile;

  // The block's queries as bf16 parts, row by row; zeros behind the last value and the last query.
  static __device__ __forceinline__ void load_queries(const AttendArgs& A, const Sequence& q, uint32_t head, uint32_t block, uint8_t* smem) {
    constexpr uint32_t kPairs = NB * 16;
    for (uint32_t i = threadIdx.x; i < S::kColumns * kPairs; i += kThreads) {
      const uint32_t column = i / kPairs, d = 2 * (i - column * kPairs), r = block * S::kColumns + column;
      const uint32_t token = A.by_shared.div(r), lane_head = r - token * A.shared;
      float v[2] = {0.0f, 0.0f};
      if (token < q.rows) {
        const T* p = static_cast<const T*>(A.q) + (uint64_t)(q.row + token) * A.q_row + (uint64_t)(head * A.shared + lane_head) * A.q_head + d;
        if (d < A.dim) v[0] = to_float(p[0]);
        if (d + 1 < A.dim) v[1] = to_float(p[1]);
      }
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        // the upper half of a float's bits, then that of the exact rest
        *reinterpret_cast<uint32_t*>(smem + (k * S::kColumns + column) * S::kQueryPitch + d * 2) = __byte_perm(__float_as_uint(v[0]), __float_as_uint(v[1]), 0x7632);
        v[0] -= __uint_as_float(__float_as_uint(v[0]) & 0xFFFF0000u);
        v[1] -= __uint_as_float(__float_as_uint(v[1]) & 0xFFFF0000u);
      }
    }
  }

  // Where a byte of a key's row is in a stage (of the keys, or of the values).
  static __device__ __forceinline__ uint32_t place_in(uint32_t key, uint32_t byte) {
    return key * S::kPitch + (S::kSwapped ? byte ^ ((key & 3) << 5 | (key & 4) << 2) : byte);
  }
  // The same a block of 32 values further on: rows begin on multiples of 256 bytes, or of 128 if they are no longer.
  static __device__ __forceinline__ uint32_t block_on(uint32_t at, uint32_t block) { return S::kSwapped ? at ^ block * S::kBlockBytes : at + block * S::kBlockBytes; }
  static __device__ __forceinline__ uint32_t word_at(uint32_t at) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
  }
  static __device__ __forceinline__ uint2 words_at(uint32_t at) {
    uint2 x;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at) : "memory");
    return x;
  }
  // The keys and values of a step's keys on their way into a stage: lane `key` (of 16 keys, also lane 16 + key) holds where that key's row is (`place`, slot *
  // heads + head) and whether it is there. Lanes share rows, `pieces` lanes a row.
  template <int kPiece, class P>
  static __device__ __forceinline__ void copy_rows(const AttendArgs& A, P place, uint32_t there, uint8_t* stage) {
    const uint32_t lane = threadIdx.x & 31, pieces = A.by_pieces.d;
    if ((pieces & (pieces - 1)) == 0 && pieces * M >= 2 && pieces <= 16) {  // a power of two: the piece is the same in all turns, and planes have turns of their own
      const uint32_t log = __ffs(pieces) - 1, piece = lane & (pieces - 1), step = 32 >> log, half = pieces * M / 2;
      uint32_t row = lane >> log;
      const uint32_t to = shared_address(stage);
      const uint8_t* codes = A.codes + piece * kPiece;
#pragma unroll 4
      for (uint32_t i = 0; i < pieces * M; ++i, row += step) {
        if (i == half) codes += A.plane_codes;
        const P at = __shfl_sync(0xFFFFFFFFu, place, row % kKeys);
        if (there >> (row % kKeys) & 1) copy_async<kPiece>(to + place_in(row, piece * kPiece), codes + (uint64_t)at * A.row_bytes);
      }
    } else {
      for (uint32_t i = lane; i < 2 * kKeys * pieces; i += 32) {
        const uint32_t row = A.by_pieces.div(i), piece = i - row * pieces;
        const P at = __shfl_sync(0xFFFFFFFFu, place, row % kKeys);
        if (there >> (row % kKeys) & 1)
          copy_async<kPiece>(shared_address(stage) + place_in(row, piece * kPiece), A.codes + (row / kKeys) * A.plane_codes + (uint64_t)at * A.row_bytes + piece * kPiece);
      }
    }
  }
  template <class P>
  static __device__ __forceinline__ void issue_rows(const AttendArgs& A, P place, int64_t slot, uint8_t* stage) {
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t there = __ballot_sync(0xFFFFFFFFu, slot >= 0);
    const uint32_t piece = A.row_bytes & (0u - A.row_bytes);  // the largest power of two that divides the rows
    if (piece >= 16) copy_rows<16>(A, place, there, stage);
    else if (piece == 8) copy_rows<8>(A, place, there, stage);
    else copy_rows<4>(A, place, there, stage);
    // scales: the words that a row's numbers lie in, which begin in the middle of one where groups are odd in number
#pragma unroll
    for (uint32_t x = 0; x < (uint32_t)M; ++x) {  // a lane's key and its value one after the other, or, of 16 keys, one of them
      const uint32_t plane = M == 2 ? x : lane >> 4, to = shared_address(stage + S::kScales) + (plane * kKeys + lane % kKeys) * 4 * S::kScaleWords;
      const uint64_t at = plane * A.plane_scales + (uint64_t)place * A.groups, word = at / 2;
      const uint32_t* from = reinterpret_cast<const uint32_t*>(A.scales) + word;
      if (slot >= 0) {
        if (A.groups & 1) {
#pragma unroll
          for (uint32_t w = 0; w < S::kScaleWords; ++w)
            if (w * 2 < ((uint32_t)at & 1) + A.groups) copy_scales(to + 4 * w, from + w, (word + w) * 2 + 1 < A.scale_count ? 4 : 2);
        } else {
#pragma unroll
          for (uint32_t w = 0; w < S::kScaleWords - 1; ++w)
            if (w * 2 < A.groups) copy_async<4>(to + 4 * w, from + w);
        }
      } else if (slot == -2) {  // a page that does not exist: its keys count as zeros
        for (uint32_t w = 0; w < S::kScaleWords; ++w) asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + 4 * w), "r"(0) : "memory");
      }
      if (A.groups & 1) {
        const uint32_t odd = __ballot_sync(0xFFFFFFFFu, at & 1);
        uint32_t* to_odd = reinterpret_cast<uint32_t*>(stage + S::kParity);
        if (lane == 0 && M == 2) to_odd[x] = odd;
        if (lane == 0 && M == 1) to_odd[0] = odd & 0xFFFFu, to_odd[1] = odd >> 16;
      }
    }
  }
  static __device__ __forceinline__ void issue(const AttendArgs& A, int64_t slot, uint32_t head, uint8_t* stage) {
    if (A.near) issue_rows<uint32_t>(A, (uint32_t)slot * A.heads + head, slot, stage);
    else issue_rows<unsigned long long>(A, (unsigned long long)slot * A.heads + head, slot, stage);
  }
  // The slot of a key; -1 behind the sequence's end, -2 if its page does not exist.
  static __device__ __forceinline__ int64_t slot_of(const AttendArgs& A, const Sequence& q, uint32_t s, uint32_t key) {
    if (key >= q.length) return -1;
    const uint32_t page = A.by_page.div(key);
    const int32_t number = __ldg(A.table + s * A.table_stride + page);
    const int64_t slot = (int64_t)number * A.by_page.d + (key - page * A.by_page.d);
    return number < 0 || slot >= (int64_t)A.slots ? -2 : slot;
  }

  static __device__ __forceinline__ void run(const AttendArgs& A) {
    extern __shared__ __align__(256) uint8_t smem[];
    __shared__ unsigned long long scan[kWarps], found_base;
    __shared__ uint32_t found;
    __shared__ float maxima[kWarps][S::kColumns], sums[kWarps][S::kColumns];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t words = (A.dim + 31) / 32;  // blocks of 32 values that are there
    const uint32_t value_blocks = kWide ? (words + 1) & ~1u : words;
    const float factor = kUnit * A.scale * kLog2e;
    const Cap cap(A.cap);
    begin_next();

    // all tiles of the call, and where this CTA's begin
    unsigned long long all = 0;
    for (uint32_t s = threadIdx.x; s < A.sequences; s += kThreads) {
      const Sequence q = sequence_of<kTile>(A, s, blockIdx.x == 0);
      all += (unsigned long long)blocks_of(A, q, S::kColumns) * A.heads * (A.whole ? q.tiles > 0 : q.tiles);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
    if (lane == 0) scan[warp] = all;
    __syncthreads();
    all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) all += scan[w];
    const unsigned long long share = share_of(all, gridDim.x, A.whole), from = blockIdx.x * share, to = min(from + share, all);
    if (blockIdx.x == 0 || from < all) {
      unsigned long long base = 0;
      for (uint32_t s0 = 0; s0 < A.sequences; s0 += kThreads) {
        const uint32_t s = s0 + threadIdx.x;
        unsigned long long mine = 0;
        if (s < A.sequences) {
          const Sequence q = sequence_of<kTile>(A, s, false);
          mine = (unsigned long long)blocks_of(A, q, S::kColumns) * A.heads * (A.whole ? q.tiles > 0 : q.tiles);
        }
        unsigned long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned long long x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
          if (lane >= (uint32_t)d) upto += x;
        }
        __syncthreads();
        if (lane == 31) scan[warp] = upto;
        __syncthreads();
        unsigned long long ahead = base + upto - mine;
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) {
          if (w < warp) ahead += scan[w];
          base += scan[w];
        }
        if (blockIdx.x == 0 && s < A.sequences) A.flat[s] = ahead;  // for the launch that joins
        if (from >= ahead && from < ahead + mine) {
          found = s;
          found_base = ahead;
        }
        if (blockIdx.x != 0 && base > from) break;
      }
      if (blockIdx.x == 0 && threadIdx.x == 0) A.flat[A.sequences] = all;
    }
    __syncthreads();
    if (from >= to) return;

    uint32_t s = found;
    Sequence q = sequence_of<kTile>(A, s, false);
    uint64_t rest = from - found_base;
    uint32_t blocks = blocks_of(A, q, S::kColumns);
    uint32_t item = A.whole ? (uint32_t)rest : (uint32_t)(rest / q.tiles), j0 = A.whole ? 0 : (uint32_t)(rest - (uint64_t)item * q.tiles);  // item: block * heads + head
    uint8_t* ring = smem + S::kQueries + warp * S::kStages * S::kStage;
    float* const red = reinterpret_cast<float*>(smem + S::kQueries);

    for (unsigned long long at = from; at < to;) {
      const uint32_t j1 = A.whole ? q.tiles : (uint32_t)min((unsigned long long)q.tiles, j0 + (to - at));
      const uint32_t block = item / A.heads, head = item - block * A.heads;
      load_queries(A, q, head, block, smem);
      // the columns of this thread: positions, slopes; the block's first and last position
      uint32_t position[2 * NT];
      float slope[2 * NT];
#pragma unroll
      for (int c = 0; c < 2 * NT; ++c) {
        const uint32_t r = block * S::kColumns + (c / 2) * 8 + 2 * t + (c & 1), token = min(A.by_shared.div(r), q.rows - 1), h = r - A.by_shared.div(r) * A.shared;
        position[c] = q.first + token;
        slope[c] = A.slopes ? A.slopes[head * A.shared + h] * kLog2e : 0.0f;
      }
      const int used = NT == 1 ? 1 : (int)min((uint32_t)NT, (q.rows * A.shared - block * S::kColumns + 7) / 8);  // eights of columns that hold queries
      const uint32_t low = q.first + A.by_shared.div(block * S::kColumns);
      const uint32_t high = q.first + min(A.by_shared.div(block * S::kColumns + S::kColumns - 1), q.rows - 1);
      // of the tiles j0 ... j1 - 1, those that some query of the block sees: some of the prefix's and some behind
      const uint32_t n0 = min(j1, q.ahead) - min(j0, q.ahead);
      const uint32_t seen0 = max(first_seen(A, low) / kTile, q.from) - q.from + q.ahead, seen1 = max(high / kTile + 1, q.from) - q.from + q.ahead;
      const uint32_t b0 = max(j0, seen0), b1 = min(j1, seen1), n = n0 + (b1 > b0 ? b1 - b0 : 0);
      auto key0 = [&](uint32_t i) {  // first key of this warp in the i-th of those tiles
        const uint32_t j = i < n0 ? min(j0, q.ahead) + i : b0 + i - n0;
        return (j < q.ahead ? j : q.from + j - q.ahead) * kTile + warp * kKeys;
      };

      float o[NB][2][NT][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][h][c][e] = 0.0f;
#pragma unroll
      for (int c = 0; c < NT; ++c) m[c][0] = m[c][1] = -INFINITY, l[c][0] = l[c][1] = 0.0f;

      // the ring: the slots of the next tile's keys are looked up while this one's copies start
      int64_t slot = n > 0 ? slot_of(A, q, s, key0(0) + lane % kKeys) : -1;
      __syncthreads();  // the queries are there, and the sums of the block before are read
#pragma unroll
      for (uint32_t i = 0; i < S::kStages - 1; ++i) {
        if (i < n) {
          if (slot == -2 && A.status) set_status(A.status, LC_ERR_INDEX);
          issue(A, slot, head, ring + i * S::kStage);
          slot = i + 1 < n ? slot_of(A, q, s, key0(i + 1) + lane % kKeys) : -1;
        }
        copies_end();
      }
      uint32_t stage_at = 0;
      for (uint32_t i = 0; i < n; ++i) {
        copies_wait<(int)S::kStages - 2>();
        __syncwarp();
        {
          const uint32_t next = i + S::kStages - 1;
          if (next < n) {
            if (slot == -2 && A.status) set_status(A.status, LC_ERR_INDEX);
            issue(A, slot, head, ring + (stage_at == 0 ? S::kStages - 1 : stage_at - 1) * S::kStage);
            slot = next + 1 < n ? slot_of(A, q, s, key0(next + 1) + lane % kKeys) : -1;
          }
          copies_end();
        }
        const uint8_t* stage = ring + stage_at * S::kStage;
        stage_at = stage_at + 1 == S::kStages ? 0 : stage_at + 1;
        const uint32_t key = key0(i);

        // ---- scores: codes times queries, a group at a time
        float score[M][NT][4] = {};
        const uint32_t row = key_of<kBits>(g);  // of the first product; its other key is row + 8
        const uint2 odd = A.groups & 1 ? *reinterpret_cast<const uint2*>(stage + S::kParity) : make_uint2(0, 0);
        // where the scales of this lane's keys begin, and of their values
        const unsigned short* const scales = reinterpret_cast<const unsigned short*>(stage + S::kScales);
        const unsigned short *key_scales[M][2], *value_scales[M][2];
#pragma unroll
        for (int x = 0; x < M; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t k = row + 16 * x + 8 * h;
            key_scales[x][h] = scales + k * (2 * S::kScaleWords) + (odd.x >> k & 1);
            value_scales[x][h] = scales + (kKeys + k) * (2 * S::kScaleWords) + (odd.y >> k & 1);
          }
        const uint32_t key_at = shared_address(stage) + place_in(row, t * kBits);  // of its first key: eight values a lane of four
        float part[M][NT][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if ((uint32_t)b >= words) break;
          uint32_t a[M][2][4];
#pragma unroll
          for (int x = 0; x < M; ++x) {
            const uint32_t p = block_on(key_at + 16 * x * S::kPitch, b), r = p + 8 * S::kPitch;
            uint32_t (&a0)[4] = a[x][0];
            uint32_t (&a1)[4] = a[x][1];
            if constexpr (kBits == 4) {
              const uint32_t u = word_at(p), v = word_at(r);
              a0[0] = operand<4, false>(u & 0x000F000Fu), a0[1] = operand<4, false>(v & 0x000F000Fu);
              a0[2] = operand<4, true>(u & 0x00F000F0u), a0[3] = operand<4, true>(v & 0x00F000F0u);
              a1[0] = operand<4, false>(u >> 8 & 0x000F000Fu), a1[1] = operand<4, false>(v >> 8 & 0x000F000Fu);
              a1[2] = operand<4, true>(u >> 8 & 0x00F000F0u), a1[3] = operand<4, true>(v >> 8 & 0x00F000F0u);
            } else {
              const uint2 u = words_at(p), v = words_at(r);
              a0[0] = operand<8, false>(__byte_perm(u.x, 0, 0x4140)), a0[1] = operand<8, false>(__byte_perm(v.x, 0, 0x4140));
              a0[2] = operand<8, false>(__byte_perm(u.x, 0, 0x4342)), a0[3] = operand<8, false>(__byte_perm(v.x, 0, 0x4342));
              a1[0] = operand<8, false>(__byte_perm(u.y, 0, 0x4140)), a1[1] = operand<8, false>(__byte_perm(v.y, 0, 0x4140));
              a1[2] = operand<8, false>(__byte_perm(u.y, 0, 0x4342)), a1[3] = operand<8, false>(__byte_perm(v.y, 0, 0x4342));
            }
          }
          const bool begins = (b & (A.per_group - 1)) == 0, ends = ((b + 1) & (A.per_group - 1)) == 0 || (uint32_t)b + 1 == words;
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            if (c >= used) break;
            if (begins) {
#pragma unroll
              for (int x = 0; x < M; ++x) part[x][c][0] = part[x][c][1] = part[x][c][2] = part[x][c][3] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
              const uint4 w = *reinterpret_cast<const uint4*>(smem + (k * S::kColumns + c * 8 + g) * S::kQueryPitch + b * 64 + t * 16);
#pragma unroll
              for (int x = 0; x < M; ++x) {
                mma_bf16(part[x][c], a[x][0], w.x, w.y);
                mma_bf16(part[x][c], a[x][1], w.z, w.w);
              }
            }
          }
          if (ends) {
#pragma unroll
            for (int x = 0; x < M; ++x) {
              const float sa = bf16_float(*key_scales[x][0]++), sb = bf16_float(*key_scales[x][1]++);
#pragma unroll
              for (int c = 0; c < NT; ++c) {
                if (c >= used) break;
                score[x][c][0] = fmaf(part[x][c][0], sa, score[x][c][0]);
                score[x][c][1] = fmaf(part[x][c][1], sa, score[x][c][1]);
                score[x][c][2] = fmaf(part[x][c][2], sb, score[x][c][2]);
                score[x][c][3] = fmaf(part[x][c][3], sb, score[x][c][3]);
              }
            }
          }
        }

        // ---- the running maximum and sum, base 2
        const bool full = key + kKeys - 1 <= low && (A.window == 0 || high - key < A.window);
        uint32_t seen = 0xFFFFFFFFu;  // a bit for each score
        bool higher = false;
        float top[NT][2];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          if (c >= used) break;
#pragma unroll
          for (int x = 0; x < M; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t at_key = key + row + 16 * x + 8 * (e / 2), p = position[2 * c + (e & 1)];
              float y = score[x][c][e] * factor;
              if (A.cap > 0.0f) y = cap(y);
              if (A.slopes) y = fmaf(-slope[2 * c + (e & 1)], fabsf((float)(int32_t)(p - at_key)), y);
              if (!full) {
                const bool visible = (at_key <= p && (A.window == 0 || p - at_key < A.window)) || at_key < q.prefix;
                if (!visible) {
                  y = -INFINITY;
                  seen &= ~(1u << (4 * (x * NT + c) + e));
                }
              }
              score[x][c][e] = y;
            }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float z = fmaxf(score[0][c][h], score[0][c][h + 2]);
            if constexpr (M == 2) z = fmaxf(z, fmaxf(score[M - 1][c][h], score[M - 1][c][h + 2]));
            z = fmaxf(z, __shfl_xor_sync(0xFFFFFFFFu, z, 4));
            z = fmaxf(z, __shfl_xor_sync(0xFFFFFFFFu, z, 8));
            z = fmaxf(z, __shfl_xor_sync(0xFFFFFFFFu, z, 16));
            top[c][h] = z;
            higher |= z > m[c][h] + kSlack;
          }
        }
        if (__any_sync(0xFFFFFFFFu, higher)) {
#pragma unroll
          for (int c = 0; c < NT; ++c) {
            if (c >= used) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              // by its own scores alone, so that a query's bits do not depend on those beside it
              const float now = top[c][h] > m[c][h] + kSlack ? top[c][h] : m[c][h], down = now == m[c][h] ? 1.0f : exp2_fast(m[c][h] - now);
              m[c][h] = now;
              l[c][h] *= down;
#pragma unroll
              for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int x = 0; x < 2; ++x) o[b][x][c][h] *= down, o[b][x][c][h + 2] *= down;
            }
          }
        }
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          if (c >= used) break;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float base = m[c][h] == -INFINITY ? 0.0f : m[c][h];
#pragma unroll
            for (int x = 0; x < M; ++x) {
              score[x][c][h] = exp2_fast(score[x][c][h] - base);
              score[x][c][h + 2] = exp2_fast(score[x][c][h + 2] - base);
              l[c][h] += score[x][c][h] + score[x][c][h + 2];
            }
          }
        }

        // ---- probabilities, with the values' scales, times codes
        uint32_t prob[M][NT][kParts][2];
        // where this lane's part of two neighbouring keys' values is; of 4 bits a word of eight values, dealt to products of 64 rows, or two lanes share one
        const uint32_t part_of = kBits == 8 || kWide ? g * 4 : g / 2 * 4, values_at = shared_address(stage) + kKeys * S::kPitch;
        const uint32_t value_a = values_at + place_in(key_of<kBits>(2 * t), part_of), value_b = values_at + place_in(key_of<kBits>(2 * t + 1), part_of);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          if ((uint32_t)b >= value_blocks) break;
          if ((b & (A.per_group - 1)) == 0) {
#pragma unroll
            for (int x = 0; x < M; ++x) {
              const float sa = bf16_float(*value_scales[x][0]++), sb = bf16_float(*value_scales[x][1]++);
#pragma unroll
              for (int c = 0; c < NT; ++c) {
                if (c >= used) break;
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = score[x][c][e] * (e < 2 ? sa : sb);
                if (!full) {  // what is not seen is 0, whatever its scale is
#pragma unroll
                  for (int e = 0; e < 4; ++e) p[e] = seen >> (4 * (x * NT + c) + e) & 1 ? p[e] : 0.0f;
                }
#pragma unroll
                for (int k = 0; k < kParts; ++k) {
                  const uint32_t u = two_bf16(p[0], p[1]), v = two_bf16(p[2], p[3]);
                  prob[x][c][k][0] = transposed(u);
                  prob[x][c][k][1] = transposed(v);
                  p[0] -= __uint_as_float(u << 16), p[1] -= __uint_as_float(u & 0xFFFF0000u);
                  p[2] -= __uint_as_float(v << 16), p[3] -= __uint_as_float(v & 0xFFFF0000u);
                }
              }
            }
          }
#pragma unroll
          for (int x = 0; x < M; ++x) {
            uint32_t a0[4], a1[4];
            const uint32_t on = kWide ? b & ~1 : b, p = block_on(value_a + 16 * x * S::kPitch, on), r = block_on(value_b + 16 * x * S::kPitch, on);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // keys 2 t, 2 t + 1, and 8 behind
              if constexpr (kBits == 4) {
                const uint32_t shift = kWide ? 8 * (b & 1) : 8 * (g & 1), u = word_at(p + 8 * h * S::kPitch), v = word_at(r + 8 * h * S::kPitch);
                const uint32_t even = __byte_perm(u, v, 0x5410) >> shift, odds = __byte_perm(u, v, 0x7632) >> shift;
                a0[2 * h] = operand<4, false>(even & 0x000F000Fu), a0[2 * h + 1] = operand<4, false>(odds & 0x000F000Fu);
                a1[2 * h] = operand<4, true>(even & 0x00F000F0u), a1[2 * h + 1] = operand<4, true>(odds & 0x00F000F0u);
              } else {
                const uint32_t u = word_at(p + 8 * h * S::kPitch), v = word_at(r + 8 * h * S::kPitch);
                const uint32_t even = __byte_perm(u, v, 0x6420), odds = __byte_perm(u, v, 0x7531);
                a0[2 * h] = operand<8, false>(even & 0x00FF00FFu), a0[2 * h + 1] = operand<8, false>(odds & 0x00FF00FFu);
                a1[2 * h] = operand<8, false>(__byte_perm(even, 0, 0x4341)), a1[2 * h + 1] = operand<8, false>(__byte_perm(odds, 0, 0x4341));
              }
            }
#pragma unroll
            for (int c = 0; c < NT; ++c) {
              if (c >= used) break;
#pragma unroll
              for (int k = 0; k < kParts; ++k) {
                mma_bf16(o[b][0][c], a0, prob[x][c][k][0], prob[x][c][k][1]);
                mma_bf16(o[b][1][c], a1, prob[x][c][k][0], prob[x][c][k][1]);
              }
            }
          }
        }
      }

      // ---- the warps' sums, brought to one maximum, added up in their order
      asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[c][h] += __shfl_xor_sync(0xFFFFFFFFu, l[c][h], d);
          if (g == 0) maxima[warp][8 * c + 2 * t + h] = m[c][h];
        }
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t column = 8 * c + 2 * t + h;
          float most = maxima[0][column];
#pragma unroll
          for (uint32_t w = 1; w < kWarps; ++w) most = fmaxf(most, maxima[w][column]);
          const float down = m[c][h] == most ? 1.0f : exp2_fast(m[c][h] - most);
          if (g == 0) sums[warp][column] = l[c][h] * down;
          float* to_sum = red + (warp * S::kColumns + column) * S::kSumPitch;
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            if ((uint32_t)b >= value_blocks) break;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                uint32_t d;
                if (kBits == 8) d = b * 32 + g * 4 + 2 * x + e;
                else if (kWide) d = (b >> 1) * 64 + g * 8 + 4 * (b & 1) + 2 * x + e;
                else d = b * 32 + g * 4 + 2 * x + e;
                to_sum[d] = o[b][x][c][h + 2 * e] * down;
              }
          }
        }
      __syncthreads();
      const bool whole = j0 == 0 && j1 == q.tiles;
      float* part_out = A.parts + (2ull * blockIdx.x + (at == from ? 0 : 1)) * S::kPart;
      for (uint32_t x = threadIdx.x; x < S::kColumns * NB * 32; x += kThreads) {
        const uint32_t column = x / (NB * 32), d = x - column * (NB * 32);
        const uint32_t r = block * S::kColumns + column, token = A.by_shared.div(r);
        if (d >= A.dim || token >= q.rows) continue;
        float v = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) v += red[(w * S::kColumns + column) * S::kSumPitch + d];
        if (whole) {
          float sum = 0.0f;
#pragma unroll
          for (uint32_t w = 0; w < kWarps; ++w) sum += sums[w][column];
          from_float(v * (kUnit / sum), static_cast<T*>(A.out)[(uint64_t)(q.row + token) * A.out_row + (uint64_t)(head * A.shared + (r - token * A.shared)) * A.out_head + d]);
        } else {
          part_out[x] = v;
        }
      }
      if (!whole && threadIdx.x < S::kColumns) {
        float most = maxima[0][threadIdx.x], sum = 0.0f;
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) most = fmaxf(most, maxima[w][threadIdx.x]), sum += sums[w][threadIdx.x];
        part_out[S::kColumns * NB * 32 + threadIdx.x] = most;
        part_out[S::kColumns * (NB * 32 + 1) + threadIdx.x] = sum;
      }

      at += A.whole ? 1 : j1 - j0;
      j0 = 0;
      if (at < to && ++item == blocks * A.heads) {
        item = 0;
        do {
          q = sequence_of<kTile>(A, ++s, false);
        } while (q.rows == 0);
        blocks = blocks_of(A, q, S::kColumns);
      }
      __syncthreads();  // the queries' place and the sums are free
    }
  }
};

// CTAs on an SM: as many as shared memory has room for, and registers.
template <int kBits, int NB, int NT, int kParts>
constexpr int kPerSm = NB * NT <= 4 ? 4 : NB * NT <= 8 ? 3 : 2;

template <int kBits, int NB, int NT, int kParts, bool kWide>
__global__ void __launch_bounds__(kThreads, (kPerSm<kBits, NB, NT, kParts>)) attend_rows_kernel(AttendArgs A) {
  Kernel<kBits, NB, NT, kParts, kWide>::run(A);
  wait_previous();  // so that what joins both kernels' parts waits for both
}

// Joins the parts of the blocks that CTAs share. CTA c looks at the border between the shares of CTAs c and c + 1: if that is the first one that
// cuts a block, the block is its own. A warp takes a query: its lanes the parts' maxima and sums, then the values, four each.
template <int NB, int NT, class T>
__global__ void __launch_bounds__(256 * NT) join_kernel(AttendArgs A, uint32_t ctas) {
  constexpr uint32_t kColumns = 8 * NT, kPart = kColumns * (NB * 32 + 2);
  wait_previous();
  const uint32_t lane = threadIdx.x & 31, column = threadIdx.x >> 5;
  const unsigned long long all = A.flat[A.sequences], share = share_of(all, ctas, false), border = (blockIdx.x + 1) * share;
  if (border >= all) return;
  uint32_t lo = 0, count = A.sequences;  // the last sequence that begins at or ahead of the border, among `count`
  while (count > 1) {
    const uint32_t step = (count + 31) / 32, at = lane * step;
    const uint32_t found = __popc(__ballot_sync(0xFFFFFFFFu, at < count && A.flat[lo + at] <= border)) - 1;
    lo += found * step;
    count = min(step, count - found * step);
  }
  const Sequence q = sequence_of<kTileKeys<NB, NT>>(A, lo, false);
  const unsigned long long rest = border - A.flat[lo];
  const uint32_t item = (uint32_t)(rest / q.tiles), j = (uint32_t)(rest - (unsigned long long)item * q.tiles);
  const unsigned long long begin = border - j, end = begin + q.tiles;
  if (j == 0 || begin + share < border) return;
  const uint32_t block = item / A.heads, head = item - block * A.heads, r = block * kColumns + column, token = A.by_shared.div(r);
  if (token >= q.rows) return;
  const uint32_t first = blockIdx.x, last = (uint32_t)((end - 1) / share);
  auto part_of = [&](uint32_t cta) { return A.parts + (2ull * cta + (begin <= cta * share ? 0 : 1)) * kPart; };
  float most = -INFINITY, sum = 0.0f;
  for (uint32_t c = first + lane; c <= last; c += 32) most = fmaxf(most, part_of(c)[kColumns * NB * 32 + column]);
#pragma unroll
  for (int d = 16; d; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
  constexpr uint32_t kTurns = (NB * 32 + 127) / 128;
  float4 v[kTurns] = {};
  for (uint32_t c0 = first; c0 <= last; c0 += 32) {
    float down = 0.0f;
    if (c0 + lane <= last) {
      const float* p = part_of(c0 + lane) + kColumns * NB * 32 + column;
      down = p[0] == most ? 1.0f : exp2_fast(p[0] - most);
      sum += p[kColumns] * down;
    }
    const uint32_t here = min(32u, last - c0 + 1);
#pragma unroll 4
    for (uint32_t i = 0; i < here; ++i) {
      const float f = __shfl_sync(0xFFFFFFFFu, down, i);
      const float4* p = reinterpret_cast<const float4*>(part_of(c0 + i) + column * (NB * 32));
#pragma unroll
      for (uint32_t k = 0; k < kTurns; ++k)
        if (NB * 32 % 128 == 0 || lane < NB * 8) {
          const float4 x = p[k * 32 + lane];
          v[k].x = fmaf(x.x, f, v[k].x), v[k].y = fmaf(x.y, f, v[k].y), v[k].z = fmaf(x.z, f, v[k].z), v[k].w = fmaf(x.w, f, v[k].w);
        }
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
  T* out = static_cast<T*>(A.out) + (uint64_t)(q.row + token) * A.out_row + (uint64_t)(head * A.shared + (r - token * A.shared)) * A.out_head;
  const float factor = kUnit / sum;
#pragma unroll
  for (uint32_t k = 0; k < kTurns; ++k) {
    const float x[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t d = k * 128 + lane * 4 + e;
      if (d < A.dim) from_float(x[e] * factor, out[d]);
    }
  }
}

template <int kBits, int NB, int NT, int kParts, bool kWide>
cudaError_t launch(const AttendArgs& args, bool overlap, cudaStream_t cs) {
  AttendArgs a = args;
  using S = Shape<kBits, NB, NT, kParts>;
  constexpr int per_sm = kPerSm<kBits, NB, NT, kParts>;
  static int sms[kMaxDevices] = {};  // by device ordinal: 0 not looked at yet
  static int fit[kMaxDevices] = {};  // CTAs on an SM
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  auto kernel = attend_rows_kernel<kBits, NB, NT, kParts, kWide>;
  if (!sms[dev]) {
    int n = 0, k = 0;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kWhole);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, kernel, kThreads, S::kWhole);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    if (k < 1) return cudaErrorLaunchOutOfResources;
    fit[dev] = k < per_sm ? k : per_sm;
    sms[dev] = n;
  }
  // no more CTAs than there can be work for
  const uint64_t blocks = ((uint64_t)a.rows * a.shared / S::kColumns + (a.rows < a.sequences ? a.rows : a.sequences)) * a.heads;
  uint64_t ctas = (uint64_t)sms[dev] * fit[dev];
  if (ctas > kMaxParts) ctas = kMaxParts;
  const uint64_t most = args.room <= kWholeRoom ? blocks : (blocks * ((a.room + S::kTile - 1) / S::kTile + 1) + 1) / 2;
  if (ctas > most) ctas = most;
  a.whole = args.room <= kWholeRoom;
  cudaError_t e = launch_kernel(overlap, kernel, (unsigned)ctas, kThreads, S::kWhole, cs, a);
  if (e == cudaSuccess && ctas > 1 && !a.whole) e = launch_kernel(true, join_kernel<NB, NT, typename Query<kParts>::T>, (unsigned)ctas - 1, 256 * NT, 0, cs, a, (uint32_t)ctas);
  return e;
}

template <int kBits, int NB, int kParts, bool kWide>
cudaError_t launch_columns(const AttendArgs& a, bool overlap, cudaStream_t cs) {
  const uint64_t columns = (uint64_t)a.longest * a.shared;
  if (columns <= 8) return launch<kBits, NB, 1, kParts, kWide>(a, overlap, cs);
  if constexpr (NB == 8) return launch<kBits, NB, 2, kParts, kWide>(a, overlap, cs);
  else {
    if (columns <= 16) return launch<kBits, NB, 2, kParts, kWide>(a, overlap, cs);
    return launch<kBits, NB, 4, kParts, kWide>(a, overlap, cs);
  }
}
template <int kBits, int NB, int kParts>
cudaError_t launch_wide(const AttendArgs& a, bool overlap, cudaStream_t cs) {
  if constexpr (kBits == 4)
    if (a.per_group > 1) return launch_columns<kBits, NB, kParts, true>(a, overlap, cs);
  return launch_columns<kBits, NB, kParts, false>(a, overlap, cs);
}
template <int kBits, int kParts>
cudaError_t launch_dim(const AttendArgs& a, bool overlap, cudaStream_t cs) {
  return a.dim <= 64 ? launch_wide<kBits, 2, kParts>(a, overlap, cs) : a.dim <= 128 ? launch_wide<kBits, 4, kParts>(a, overlap, cs) : launch_wide<kBits, 8, kParts>(a, overlap, cs);
}
constexpr uint64_t kLargestPart = 4ull * (Shape<8, 8, 2, 1>::kPart > Shape<8, 4, 4, 1>::kPart ? Shape<8, 8, 2, 1>::kPart : Shape<8, 4, 4, 1>::kPart);
static_assert(kLargestPart <= kPartBytes, "room for a part in the workspace");

}  // namespace
}  // namespace lc
