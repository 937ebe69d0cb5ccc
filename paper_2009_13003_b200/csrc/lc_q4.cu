// 4-bit weights: a matrix into groups of 4-bit codes with scales, and back into numbers.
#include "lc_q4.cuh"

namespace lc {
namespace {

constexpr int kThreads = 256;

// A thread takes eight columns of rows r and r + 8 of a tile, which is where the two words that hold them meet; the group / 8 lanes
// of a group sit side by side, so that a group's maximum is a few shuffles and a row is read in whole lines. The next lanes take the
// next r: together they write whole blocks. One pass, bound by memory: 4.5 (fp32) or 2.5 bytes a weight.
template <class T>
__global__ void __launch_bounds__(kThreads) q4_quantize_kernel(const T* __restrict__ w, uint64_t row_stride, Q4Layout L, uint8_t* __restrict__ q4,
                                                               int32_t* status, FastDiv by_groups) {
  const uint32_t lanes = L.group / 8;
  const uint64_t item = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / lanes;  // (tile, group, r)
  const uint32_t lane = threadIdx.x & (lanes - 1);
  const uint32_t r = (uint32_t)item & 7u;
  const uint32_t tg = (uint32_t)(item >> 3);
  const bool inside = (item >> 3) < (uint64_t)L.tiles * L.groups;  // all lanes stay for the shuffles
  const uint32_t tile = inside ? by_groups.div(tg) : 0, g = tg - tile * L.groups;
  const uint32_t col = g * L.group + 8 * lane;
  const int valid = !inside || col >= L.cols ? 0 : (int)min(8u, L.cols - col);
  uint32_t scale[2];
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint64_t row = (uint64_t)tile * kQ4TileRows + r + 8 * h;
    load8(w + row * row_stride + col, row < L.rows ? valid : 0, v[h]);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) scale[h] = group_scale(max_over_lanes(max_bits8(v[h]), (int)lanes), 7.0f);
  if (!inside) return;
  int q[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) codes8(v[h], scale[h], q[h]);
  uint32_t word[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t x = 0;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int* s = &q[p & 1][4 * j + 2 * (p >> 1)];
      x |= ((uint32_t)(s[0] + 8) & 15u) << (4 * p) | ((uint32_t)(s[1] + 8) & 15u) << (16 + 4 * p);
    }
    word[j] = x;
  }
  const uint32_t block = col / 64, half = (col / 32) & 1, t = (col / 8) & 3;
  uint8_t* at = q4 + ((uint64_t)tile * L.steps * 2 + block) * 512 + (r * 4 + t) * 16 + half * 8;
  *reinterpret_cast<uint2*>(at) = make_uint2(word[0], word[1]);
  if (lane == 0) {
    reinterpret_cast<uint32_t*>(q4 + L.scales_off)[((uint64_t)tile * L.groups + g) * 8 + r] = (scale[0] >> 16) | (scale[1] & 0xFFFF0000u);
    if (scale[0] == kScaleNaN || scale[1] == kScaleNaN) set_status(status, LC_ERR_NONFINITE);
  }
}

// The same threads the other way round.
template <class T>
__global__ void __launch_bounds__(kThreads) q4_read_kernel(const uint8_t* __restrict__ q4, Q4Layout L, T* __restrict__ out, uint64_t row_stride,
                                                           FastDiv by_groups) {
  const uint32_t lanes = L.group / 8;
  const uint64_t item = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / lanes;
  const uint32_t r = (uint32_t)item & 7u;
  const uint32_t tg = (uint32_t)(item >> 3);
  if ((item >> 3) >= (uint64_t)L.tiles * L.groups) return;
  const uint32_t tile = by_groups.div(tg), g = tg - tile * L.groups;
  const uint32_t col = g * L.group + 8 * (threadIdx.x & (lanes - 1));
  if (col >= L.cols) return;
  const int valid = (int)min(8u, L.cols - col);
  const uint32_t block = col / 64, half = (col / 32) & 1, t = (col / 8) & 3;
  const uint8_t* at = q4 + ((uint64_t)tile * L.steps * 2 + block) * 512 + (r * 4 + t) * 16 + half * 8;
  const uint2 w = __ldg(reinterpret_cast<const uint2*>(at));
  const uint32_t s = __ldg(reinterpret_cast<const uint32_t*>(q4 + L.scales_off) + ((uint64_t)tile * L.groups + g) * 8 + r);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint64_t row = (uint64_t)tile * kQ4TileRows + r + 8 * h;
    const float scale = __uint_as_float(h ? s & 0xFFFF0000u : s << 16);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int bit = 16 * (e & 1) + 4 * (h + 2 * ((e >> 1) & 1));
      v[e] = (__uint_as_float((((e < 4 ? w.x : w.y) >> bit) & 15u) | 0x4B000000u) - 8388616.0f) * scale;
    }
    if (row < L.rows) store8(out + row * row_stride + col, valid, v);
  }
}

uint64_t blocks_for(const Q4Layout& L) { return ((uint64_t)L.tiles * L.groups * L.group + kThreads - 1) / kThreads; }  // 8 r, group / 8 lanes

}  // namespace

cudaError_t launch_q4_quantize(const Q4Layout& L, const void* w, int type, uint64_t row_stride, uint8_t* q4, int32_t* status, cudaStream_t cs) {
  const uint64_t blocks = blocks_for(L);
  if (blocks == 0) return cudaSuccess;
  const FastDiv by_groups(L.groups);
  if (type == LC_TYPE_F32)
    return launch_kernel(false, q4_quantize_kernel<float>, (unsigned)blocks, kThreads, 0, cs, static_cast<const float*>(w), row_stride, L, q4, status, by_groups);
  if (type == LC_TYPE_BF16)
    return launch_kernel(false, q4_quantize_kernel<__nv_bfloat16>, (unsigned)blocks, kThreads, 0, cs, static_cast<const __nv_bfloat16*>(w), row_stride, L, q4,
                         status, by_groups);
  return launch_kernel(false, q4_quantize_kernel<__half>, (unsigned)blocks, kThreads, 0, cs, static_cast<const __half*>(w), row_stride, L, q4, status, by_groups);
}

cudaError_t launch_q4_read(const Q4Layout& L, const uint8_t* q4, void* out, int type, uint64_t row_stride, cudaStream_t cs) {
  const uint64_t blocks = blocks_for(L);
  if (blocks == 0) return cudaSuccess;
  const FastDiv by_groups(L.groups);
  if (type == LC_TYPE_F32)
    return launch_kernel(false, q4_read_kernel<float>, (unsigned)blocks, kThreads, 0, cs, q4, L, static_cast<float*>(out), row_stride, by_groups);
  if (type == LC_TYPE_BF16)
    return launch_kernel(false, q4_read_kernel<__nv_bfloat16>, (unsigned)blocks, kThreads, 0, cs, q4, L, static_cast<__nv_bfloat16*>(out), row_stride, by_groups);
  return launch_kernel(false, q4_read_kernel<__half>, (unsigned)blocks, kThreads, 0, cs, q4, L, static_cast<__half*>(out), row_stride, by_groups);
}

}  // namespace lc

using namespace lc;

namespace {

// Limits that keep a matrix's index arithmetic in range: tiles * groups < 2^31, and so a grid of fewer than 2^31 blocks.
bool q4_shape_ok(uint64_t rows, uint64_t cols, int group) {
  if (!group_ok(group) || rows >= (1ull << 31) || cols >= (1ull << 31) - kQ4StepCols) return false;
  const Q4Layout L = q4_layout(rows, cols, group);
  return (uint64_t)L.tiles * L.groups < (1ull << 31) / 8;
}

int check_q4(const void* q4, uint64_t q4_bytes, uint64_t rows, uint64_t cols, int group) {
  if (!q4_shape_ok(rows, cols, group)) return LC_ERR_ARG;
  if (rows == 0 || cols == 0) return LC_OK;
  if (!q4 || !aligned_to(q4, 256)) return LC_ERR_ARG;
  return q4_bytes < q4_layout(rows, cols, group).total ? LC_ERR_CAPACITY : LC_OK;
}

// A matrix of rows * cols values in the caller's memory.
int check_matrix(const void* p, int type, uint64_t rows, uint64_t cols, uint64_t row_stride) {
  if (!type_ok(type)) return LC_ERR_ARG;
  if (rows == 0 || cols == 0) return LC_OK;
  if (!p || !aligned_to(p, type_bytes(type)) || (rows > 1 && row_stride < cols)) return LC_ERR_ARG;
  return row_stride >= (1ull << 40) ? LC_ERR_ARG : LC_OK;
}

int quantize_impl(const void* w, int type, uint64_t rows, uint64_t cols, uint64_t row_stride, int group, void* q4, uint64_t q4_bytes, void* workspace,
                  cudaStream_t cs) {
  const Q4Layout L = q4_layout(rows, cols, group);
  return launch_q4_quantize(L, w, type, row_stride, static_cast<uint8_t*>(q4), &static_cast<Control*>(workspace)->status, cs) == cudaSuccess ? LC_OK
                                                                                                                                             : LC_ERR_CUDA;
}

}  // namespace

extern "C" {

uint64_t lc_q4_bytes(uint64_t rows, uint64_t cols, int group) { return q4_shape_ok(rows, cols, group) ? q4_layout(rows, cols, group).total : 0; }

int lc_q4_quantize(const void* w, int type, uint64_t rows, uint64_t cols, uint64_t row_stride, int group, void* q4, uint64_t q4_bytes, void* workspace,
                   uint64_t workspace_bytes, lc_cuda_stream_t cs) {
  int rc = check_q4(q4, q4_bytes, rows, cols, group);
  if (rc == LC_OK) rc = check_matrix(w, type, rows, cols, row_stride);
  if (rc != LC_OK) return rc;
  if (!workspace || !aligned_to(workspace, 256)) return LC_ERR_ARG;
  if (workspace_bytes < lc_workspace_bytes(0)) return LC_ERR_CAPACITY;
  if (cudaMemsetAsync(workspace, 0, sizeof(int32_t), cs) != cudaSuccess) return LC_ERR_CUDA;
  return quantize_impl(w, type, rows, cols, row_stride, group, q4, q4_bytes, workspace, cs);
}

int lc_recover_q4(const float* base, const void* const* streams, const uint64_t* stream_bytes, int k, uint64_t rows, uint64_t cols, int group, void* q4,
                  uint64_t q4_bytes, float* scratch, void* workspace, uint64_t workspace_bytes, lc_cuda_stream_t cs) {
  int rc = check_q4(q4, q4_bytes, rows, cols, group);
  if (rc != LC_OK) return rc;
  if (rows * cols >= (1ull << 32)) return LC_ERR_ARG;
  if ((rc = lc_recover(base, streams, stream_bytes, k, rows * cols, scratch, workspace, workspace_bytes, cs)) != LC_OK) return rc;
  return quantize_impl(scratch, LC_TYPE_F32, rows, cols, cols, group, q4, q4_bytes, workspace, cs);
}

int lc_q4_read(const void* q4, uint64_t q4_bytes, uint64_t rows, uint64_t cols, int group, void* out, int type, uint64_t row_stride, lc_cuda_stream_t cs) {
  int rc = check_q4(q4, q4_bytes, rows, cols, group);
  if (rc == LC_OK) rc = check_matrix(out, type, rows, cols, row_stride);
  if (rc != LC_OK) return rc;
  return launch_q4_read(q4_layout(rows, cols, group), static_cast<const uint8_t*>(q4), out, type, row_stride, cs) == cudaSuccess ? LC_OK : LC_ERR_CUDA;
}

int lc_q4_matvec(const void* q4, uint64_t q4_bytes, uint64_t rows, uint64_t cols, int group, const void* x, int type, uint64_t tokens, uint64_t x_stride,
                 void* out, int out_type, uint64_t out_stride, lc_cuda_stream_t cs) {
  int rc = check_q4(q4, q4_bytes, rows, cols, group);
  if (rc == LC_OK) rc = check_matrix(x, type, tokens, cols, tokens > 1 && x_stride == 0 ? cols : x_stride);  // one vector for all tokens is fine
  if (rc == LC_OK) rc = check_matrix(out, out_type, tokens, rows, out_stride);
  if (rc != LC_OK) return rc;
  if ((out_type != type && out_type != LC_TYPE_F32) || tokens > LC_Q4_MAX_TOKENS) return LC_ERR_ARG;
  if (tokens == 0 || rows == 0) return LC_OK;
  return launch_q4_matvec(q4_layout(rows, cols, group), static_cast<const uint8_t*>(q4), x, type, (uint32_t)tokens, x_stride, out, out_type, out_stride,
                          cs) == cudaSuccess
             ? LC_OK
             : LC_ERR_CUDA;
}

}  // extern "C"
