// Attention over a quantised cache: what its kernels share.
#pragma once

#include "lc_quant.cuh"

namespace lc {

constexpr uint32_t kAttendDim = 256;   // longest rows
constexpr uint32_t kMaxParts = 592;    // CTAs that share a call's tiles, at most: four on each of 148 SMs
constexpr uint32_t kMaxColumns = 32;   // queries of a block

struct AttendArgs {
  const uint8_t* codes;         // of the keys; the values' lie plane_codes bytes behind
  const unsigned short* scales; // likewise, plane_scales numbers behind
  uint64_t plane_codes, plane_scales, scale_count;  // scale_count: of all planes
  uint64_t slots;
  uint32_t heads, dim, row_bytes, groups, per_group;  // per_group: blocks of 32 values
  const void* q;
  void* out;
  uint64_t q_row, q_head, out_row, out_head;
  const int32_t* table;
  uint64_t table_stride, room;  // room: positions that a row of the table has pages for
  const int32_t *begin, *first, *prefix;
  const float* slopes;
  uint32_t sequences, rows, shortest, longest;  // a kernel takes the sequences of shortest ... longest rows
  uint32_t most;                                // no sequence of the call has more rows
  uint32_t shared, window;
  uint32_t near;   // slot * heads + head is below 2^32
  uint32_t whole;  // few rows: blocks are dealt out whole, not by their tiles, and nothing is joined
  float scale, cap;
  int32_t* status;
  float* parts;                 // partial results of the CTAs' first and last blocks
  unsigned long long* flat;     // [sequences + 1] first tile of each sequence among all
  FastDiv by_page, by_shared, by_pieces;
};

// A sequence of a call: its rows, positions, and the tiles of keys that its rows see. The tiles of its prefix come first, then those from the first
// row's window to the last row; where the two meet none is there twice.
struct Sequence {
  uint32_t row, rows;          // its first row, and their number: 0 if it has none, or none that the kernel takes
  uint32_t first, length;      // position of the first row; keys
  uint32_t prefix, ahead;      // keys that all rows see, tiles of those
  uint32_t from, tiles;        // first tile behind those of the prefix; tiles in all
};
__device__ __forceinline__ uint32_t first_seen(const AttendArgs& A, uint32_t position) {  // ignoring the prefix
  return A.window && position >= A.window ? position - A.window + 1 : 0;
}
// kTile: keys of a tile.
template <uint32_t kTile>
__device__ __forceinline__ Sequence sequence_of(const AttendArgs& A, uint32_t s, bool report) {
  Sequence q = {};
  const int64_t begin = A.begin[s], n = (int64_t)A.begin[s + 1] - begin;
  const int64_t first = A.first ? A.first[s] : 0;
  if (n <= 0) return q;
  if (begin < 0 || begin + n > (int64_t)A.rows || n > (int64_t)A.most || first < 0 || first + n > (int64_t)A.room) {
    if (report && A.status) set_status(A.status, LC_ERR_INDEX);
    return q;
  }
  if (n < (int64_t)A.shortest || n > (int64_t)A.longest) return q;
  q.row = (uint32_t)begin;
  q.rows = (uint32_t)n;
  q.first = (uint32_t)first;
  q.length = (uint32_t)(first + n);
  const int32_t prefix = A.prefix ? A.prefix[s] : 0;
  q.prefix = prefix <= 0 ? 0 : min((uint32_t)prefix, q.length);
  q.ahead = (q.prefix + kTile - 1) / kTile;
  q.from = max(q.ahead, first_seen(A, q.first) / kTile);
  q.tiles = q.ahead + max((q.length + kTile - 1) / kTile, q.from) - q.from;
  return q;
}
__device__ __forceinline__ uint32_t blocks_of(const AttendArgs& A, const Sequence& q, uint32_t columns) {
  return (uint32_t)(((uint64_t)q.rows * A.shared + columns - 1) / columns);
}

// 2^x, 1 / x and the like as the hardware approximates them (relative error about 2^-22).
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// Scores and the cap in units of base 2: cap * tanh(z / cap) of z. Where x = z / cap is small, the series x - x^3 / 3 + 2 x^5 / 15 - 17 x^7 / 315 + 62 x^9 / 2835 (what it
// leaves out is below 2^-26 of x), elsewhere cap - 2 cap / (1 + e^2x), which is off by some 2^-22 of the cap: everywhere by no more than 2^-20 of the result.
// (That form alone would lose small scores in the rounding of a large cap.)
struct Cap {
  float in, out;  // 2 x log2(e) = z * in; out: the cap
  static constexpr float kSmall = 0.72f;  // of |2 x log2(e)|: |x| < 0.2496
  __device__ __forceinline__ explicit Cap(float cap) : in(2.0f / cap), out(cap * kLog2e) {}
  // The series in a^2, a = 2 x log2(e), i.e. x^2 = (ln(2) / 2)^2 a^2: what follows its leading 1, over a^2.
  static constexpr float kUnit = 0.1201132535f, k1 = -kUnit / 3, k2 = 2 * kUnit * kUnit / 15, k3 = -17 * kUnit * kUnit * kUnit / 315, k4 = 62 * kUnit * kUnit * kUnit * kUnit / 2835;
  __device__ __forceinline__ float operator()(float z) const {
    const float a = z * in, b = a * a, series = b * fmaf(fmaf(fmaf(k4, b, k3), b, k2), b, k1);
    return fabsf(a) < kSmall ? fmaf(z, series, z) : large(z);
  }
  __device__ __forceinline__ float large(float z) const { return fmaf(-2.0f * out, reciprocal(1.0f + exp2_fast(z * in)), out); }
  // Two of them that are known to be small.
  __device__ __forceinline__ Two small(Two z) const {
    const Two a = mul_two(z, two(in, in)), b = mul_two(a, a);
    const Two series = mul_two(b, fma_two(fma_two(fma_two(two(k4, k4), b, two(k3, k3)), b, two(k2, k2)), b, two(k1, k1)));
    return fma_two(z, series, z);
  }
};

constexpr uint64_t kPartBytes = 4ull * (kMaxColumns * 128 + 2 * kMaxColumns);  // of a partial result: 32 queries of 128 values, or 16 of 256

constexpr uint32_t kTileCtas = 160;     // CTAs of the kernel for many rows, at most: one on each SM
constexpr uint32_t kTileRows = 256;     // queries of its blocks
constexpr uint32_t kTileDim = 128;      // longest rows that it takes
constexpr uint64_t kTilePartBytes = 4ull * kTileRows * (kTileDim + 2);

// The kernel for sequences of many rows (lc_attend_tiles.cu), for queries of bf16 or fp16, and what joins its parts, behind it and other launches of the call.
cudaError_t launch_attend_tiles(const AttendArgs& a, int bits, int type, cudaStream_t cs);
cudaError_t launch_join_tiles(const AttendArgs& a, int type, cudaStream_t cs);
// The kernel for few rows (lc_attend_rows.cuh) and what joins its parts. overlap: behind a launch of the same call.
cudaError_t launch_attend_bf16(const AttendArgs& a, int bits, bool overlap, cudaStream_t cs);
cudaError_t launch_attend_f16(const AttendArgs& a, int bits, bool overlap, cudaStream_t cs);
cudaError_t launch_attend_f32(const AttendArgs& a, int bits, bool overlap, cudaStream_t cs);

}  // namespace lc
