// 4-bit weights: a matrix into groups of 4-bit codes with scales, and back into numbers.
#include "lc_q4.cuh"

namespace lc {
namespace {

constexpr int kThreads = 256;

// A thread takes columns 8 t ... 8 t + 7 of both halves of a block of 64, of rows r and r + 8 of a tile: what 16 bytes of a lane's words
// hold. The 4 lanes t (with groups of 128, those of two blocks) have a group's maximum by a few shuffles; the next lanes take the next
// r, so that a warp writes whole blocks. One pass, bound by memory: 4.5 bytes a weight from fp32 (4096 x 25088: 70 us, the copy rate),
// 2.5 from 16 bits, where the instructions of the codes weigh as much.
template <class T, int G>
__global__ void __launch_bounds__(kThreads) q4_quantize_kernel(const T* __restrict__ w, uint64_t row_stride, Q4Layout L, uint8_t* __restrict__ q4,
                                                               int32_t* status, FastDiv by_spans) {
  constexpr uint32_t kSpan = G == 128 ? 128 : 64, kLanes = kSpan / 16, kScales = G == 32 ? 2 : 1;  // columns, lanes and scales a row has here
  const uint64_t item = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;                  // (tile, span, r)
  const uint32_t lane = threadIdx.x & (kLanes - 1), r = (uint32_t)item & 7u;
  const bool inside = (item >> 3) < (uint64_t)L.tiles * by_spans.d;  // all lanes stay for the shuffles
  const uint32_t tile = inside ? by_spans.div((uint32_t)(item >> 3)) : 0, span = inside ? (uint32_t)(item >> 3) - tile * by_spans.d : 0;
  const uint32_t col = span * kSpan + (lane >> 2) * 64 + (lane & 3) * 8;
  float v[2][2][8];  // row, half
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint64_t row = (uint64_t)tile * kQ4TileRows + r + 8 * h;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t c = col + 32 * u;
      load8(w + row * row_stride + c, !inside || row >= L.rows || c >= L.cols ? 0 : (int)min(8u, L.cols - c), v[h][u]);
    }
  }
  uint32_t scale[2][kScales];
  float most[2][kScales];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float m[2] = {0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) m[u % kScales] = max_magnitude(m[u % kScales], v[h][u][i]);
    }
#pragma unroll
    for (uint32_t k = 0; k < kScales; ++k) most[h][k] = max_over_lanes(m[k], kLanes);
  }
  if constexpr (kScales == 2) {  // four scales and four lanes: one each
    const uint32_t mine = group_scale<4>(lane & 2 ? (lane & 1 ? most[1][1] : most[1][0]) : (lane & 1 ? most[0][1] : most[0][0]));
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[i >> 1][i & 1] = __shfl_sync(0xFFFFFFFFu, mine, i, 4);
  } else {
    scale[0][0] = group_scale<4>(most[0][0]);
    scale[1][0] = group_scale<4>(most[1][0]);
  }
  if (!inside) return;
  uint32_t word[2][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float t[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) codes<T, 4>(v[h][u], scale[h][u % kScales], t[h]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float *a = t[0] + 4 * j, *b = t[1] + 4 * j;
      word[u][j] = pack_pairs(pair_of(a[0], a[1]), pair_of(b[0], b[1]), pair_of(a[2], a[3]), pair_of(b[2], b[3]));
    }
  }
  *reinterpret_cast<uint4*>(q4 + ((uint64_t)tile * L.steps * 2 + col / 64) * 512 + (r * 4 + (lane & 3)) * 16) = make_uint4(word[0][0], word[0][1], word[1][0], word[1][1]);
  if (lane == 0) {
#pragma unroll
    for (uint32_t k = 0; k < kScales; ++k) {
      reinterpret_cast<uint32_t*>(q4 + L.scales_off)[((uint64_t)tile * L.groups + span * kScales + k) * 8 + r] = (scale[0][k] >> 16) | (scale[1][k] & 0xFFFF0000u);
      if (scale[0][k] == kScaleNaN || scale[1][k] == kScaleNaN) set_status(status, LC_ERR_NONFINITE);
    }
  }
}

// The other way round: rows r and r + 8 of a block of 64 columns, in both halves of it 16 bytes of the output a lane, so that the lanes of
// a row write whole runs: 4 lanes for a 16-bit output, 8 for fp32 (half the words each). Bound by memory: 4096 x 25088 to fp32 75 us, the
// bytes take 71; 8192 x 8192 to fp16 29 us and 26.
template <class T>
__global__ void __launch_bounds__(kThreads) q4_read_kernel(const uint8_t* __restrict__ q4, Q4Layout L, T* __restrict__ out, uint64_t row_stride,
                                                           FastDiv by_blocks) {
  constexpr uint32_t n = kRun<T>, kLanes = 32 / n;
  const uint64_t item = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes;  // (tile, block, r)
  if ((item >> 3) >= (uint64_t)L.tiles * by_blocks.d) return;
  const uint32_t lane = threadIdx.x & (kLanes - 1), r = (uint32_t)item & 7u, tile = by_blocks.div((uint32_t)(item >> 3)), block = (uint32_t)(item >> 3) - tile * by_blocks.d;
  const uint8_t* at = q4 + ((uint64_t)tile * L.steps * 2 + block) * 512 + r * 64;
  uint2 w[2];  // of a half: the words of n columns
  if constexpr (n == 8) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(at) + lane);
    w[0] = make_uint2(x.x, x.y);
    w[1] = make_uint2(x.z, x.w);
  } else {
    const uint32_t* x = reinterpret_cast<const uint32_t*>(at) + (lane >> 1) * 4 + (lane & 1);
    w[0].x = __ldg(x);
    w[1].x = __ldg(x + 2);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const uint32_t c = block * 64 + 32 * u, s = __ldg(reinterpret_cast<const uint32_t*>(q4 + L.scales_off) + ((uint64_t)tile * L.groups + c / L.group) * 8 + r);
    const uint32_t col = c + lane * n;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t row = (uint64_t)tile * kQ4TileRows + r + 8 * h;
      const float scale = __uint_as_float(h ? s & 0xFFFF0000u : s << 16);
      uint32_t codes[n];
#pragma unroll
      for (uint32_t e = 0; e < n; ++e) codes[e] = ((e < 4 ? w[u].x : w[u].y) >> (16 * (e & 1) + 4 * (h + 2 * ((e >> 1) & 1)))) & 15u;
      float v[n];
      values_of<4>(codes, scale, v);
      keep_in_type<T, 4>(scale, v);
      if (row < L.rows && col < L.cols) store_run(out + row * row_stride + col, (int)min(n, L.cols - col), v);
    }
  }
}

// Threads for a tile's spans of `columns`, eight rows r each
unsigned grid_of(const Q4Layout& L, uint32_t spans, uint32_t lanes) { return (unsigned)(((uint64_t)L.tiles * spans * 8 * lanes + kThreads - 1) / kThreads); }

template <class T>
cudaError_t quantize(const Q4Layout& L, const void* w, uint64_t row_stride, uint8_t* q4, int32_t* status, cudaStream_t cs) {
  const auto kernel = L.group == 32 ? q4_quantize_kernel<T, 32> : L.group == 64 ? q4_quantize_kernel<T, 64> : q4_quantize_kernel<T, 128>;
  const uint32_t spans = L.group == 128 ? L.steps : 2 * L.steps, lanes = L.group == 128 ? 8 : 4;
  return launch_kernel(false, kernel, grid_of(L, spans, lanes), kThreads, 0, cs, static_cast<const T*>(w), row_stride, L, q4, status, FastDiv(spans));
}
template <class T>
cudaError_t read(const Q4Layout& L, const uint8_t* q4, void* out, uint64_t row_stride, cudaStream_t cs) {
  return launch_kernel(false, q4_read_kernel<T>, grid_of(L, 2 * L.steps, 32 / kRun<T>), kThreads, 0, cs, q4, L, static_cast<T*>(out), row_stride, FastDiv(2 * L.steps));
}

}  // namespace

cudaError_t launch_q4_quantize(const Q4Layout& L, const void* w, int type, uint64_t row_stride, uint8_t* q4, int32_t* status, cudaStream_t cs) {
  if (L.tiles == 0 || L.steps == 0) return cudaSuccess;
  if (type == LC_TYPE_F32) return quantize<float>(L, w, row_stride, q4, status, cs);
  if (type == LC_TYPE_BF16) return quantize<__nv_bfloat16>(L, w, row_stride, q4, status, cs);
  return quantize<__half>(L, w, row_stride, q4, status, cs);
}

cudaError_t launch_q4_read(const Q4Layout& L, const uint8_t* q4, void* out, int type, uint64_t row_stride, cudaStream_t cs) {
  if (L.tiles == 0 || L.steps == 0) return cudaSuccess;
  if (type == LC_TYPE_F32) return read<float>(L, q4, out, row_stride, cs);
  if (type == LC_TYPE_BF16) return read<__nv_bfloat16>(L, q4, out, row_stride, cs);
  return read<__half>(L, q4, out, row_stride, cs);
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
