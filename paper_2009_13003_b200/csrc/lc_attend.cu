// The entry points of attention to a quantised cache: what they refuse, and which kernel a call goes to.
#include "lc_attend.cuh"

namespace lc {
namespace {

uint64_t flat_bytes(uint64_t sequences) { return (8 * (sequences + 1) + 255) / 256 * 256; }

// Queries of a sequence for one head of the cache up to which the kernel for few rows takes it. The other one multiplies blocks of 256, full or not. 24 sequences of up to 8192
// keys, 8 heads in 8 bits (in 4), 20, 32, 64 queries for each, few rows / many, us: dim 128 301 / 212, 332 / 212, 634 / 212 (255 / 210, 292 / 210, 559 / 208); dim 64 156 / 198, 173 / 196,
// 315 / 194 (151 / 197, 169 / 195, 309 / 194). One limit for both dims: that of dim 128.
constexpr uint32_t kFewQueries = 16;

constexpr float kLargest = 1e30f;  // of scale and cap: what is made of them stays in fp32's range

// A cache that can be attended to, whatever the number of its slots.
bool shape_ok(const lc_cache* cache) {
  if (!cache || cache->planes != 2 || cache->dim > kAttendDim) return false;
  lc_cache one = *cache;
  one.slots = 1;
  return lc_cache_code_bytes(&one) > 0;
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" {

uint64_t lc_cache_attend_bytes(const lc_cache* cache, uint32_t sequences) {
  return shape_ok(cache) && sequences < (1u << 31) ? 2 * flat_bytes(sequences) + 2 * (kMaxParts * kPartBytes + kTileCtas * kTilePartBytes) : 0;
}

int lc_cache_attend(const lc_cache* cache, const lc_rows* q, const lc_rows* out, int type, uint64_t rows, const lc_attend* how, void* workspace,
                    uint64_t workspace_bytes, int32_t* status, lc_cuda_stream_t cs) {
  if (!q || !out || !how || !type_ok(type)) return LC_ERR_ARG;
  if (!shape_ok(cache) || (cache->slots > 0 && lc_cache_code_bytes(cache) == 0)) return LC_ERR_ARG;
  if (how->heads < 1 || how->heads > 65536 || how->heads % cache->heads || rows >= (1ull << 31) || rows * how->heads >= (1ull << 30)) return LC_ERR_ARG;
  if (how->page < 1 || how->page >= (1u << 31) || how->sequences >= (1u << 31) || how->table_stride >= (1ull << 32) ||
      (how->sequences > 1 && how->table_stride < how->width) || how->window >= (1u << 31))
    return LC_ERR_ARG;
  if (!(how->scale >= -kLargest && how->scale <= kLargest) || !(how->cap >= 0.0f && how->cap <= kLargest)) return LC_ERR_ARG;
  if (rows == 0 || how->sequences == 0) return LC_OK;
  const lc_rows* both[2] = {q, out};
  for (const lc_rows* r : both)
    if (!r->data || !aligned_to(r->data, type_bytes(type)) || r->row_stride >= (1ull << 33) || r->head_stride >= (1ull << 40)) return LC_ERR_ARG;
  const uint64_t n = rows, h = how->heads, dim = cache->dim;
  const bool by_row = (h == 1 || out->head_stride >= dim) && (n == 1 || out->row_stride >= (h - 1) * out->head_stride + dim);
  const bool by_head = (n == 1 || out->row_stride >= dim) && (h == 1 || out->head_stride >= (n - 1) * out->row_stride + dim);
  if (!by_row && !by_head) return LC_ERR_ARG;
  if (cache->slots > 0 && (!cache->codes || !cache->scales || !aligned_to(cache->codes, 16) || !aligned_to(cache->scales, 4))) return LC_ERR_ARG;
  if ((how->width > 0 && !how->table) || !how->begin || !aligned_to(how->table, 4) || !aligned_to(how->begin, 4) || !aligned_to(how->first, 4) ||
      !aligned_to(how->prefix, 4) || !aligned_to(how->slopes, 4) || !aligned_to(status, 4))
    return LC_ERR_ARG;
  if (!workspace || !aligned_to(workspace, 256)) return LC_ERR_ARG;
  if (workspace_bytes < lc_cache_attend_bytes(cache, how->sequences)) return LC_ERR_CAPACITY;

  AttendArgs a = {};
  a.codes = static_cast<const uint8_t*>(cache->codes);
  a.scales = static_cast<const unsigned short*>(cache->scales);
  a.heads = cache->heads;
  a.dim = cache->dim;
  a.row_bytes = (cache->dim + 7) / 8 * cache->bits;
  a.groups = (cache->dim + cache->group - 1) / cache->group;
  a.per_group = cache->group / 32;
  a.slots = cache->slots;
  a.plane_codes = cache->slots * cache->heads * a.row_bytes;
  a.plane_scales = cache->slots * cache->heads * a.groups;
  a.scale_count = 2 * a.plane_scales;
  a.q = q->data;
  a.out = out->data;
  a.q_row = q->row_stride, a.q_head = q->head_stride;
  a.out_row = out->row_stride, a.out_head = out->head_stride;
  a.table = how->table;
  a.table_stride = how->table_stride;
  const uint64_t room = (uint64_t)how->width * how->page;
  a.room = room < 0x7FFFFFFFull ? room : 0x7FFFFFFFull;
  a.begin = how->begin;
  a.first = how->first;
  a.prefix = how->prefix;
  a.slopes = how->slopes;
  a.sequences = how->sequences;
  a.rows = (uint32_t)rows;
  a.most = how->longest && how->longest < rows ? how->longest : (uint32_t)rows;
  a.shortest = 1;
  a.longest = a.most;
  a.shared = how->heads / cache->heads;
  a.window = how->window;
  a.near = cache->slots < 0xFFFFFFFFull / cache->heads;
  a.scale = how->scale;
  a.cap = how->cap > 0.0f && how->cap < 1.0f / kLargest ? 1.0f / kLargest : how->cap;  // below that scores are 0 all the same
  a.status = status;
  a.flat = static_cast<unsigned long long*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 2 * flat_bytes(how->sequences));
  a.by_page = FastDiv(how->page);
  a.by_shared = FastDiv(a.shared);
  const uint32_t piece = a.row_bytes & (0u - a.row_bytes);
  a.by_pieces = FastDiv(a.row_bytes / (piece > 16 ? 16 : piece));
  const int bits = (int)cache->bits;
  cudaError_t e = cudaSuccess;
  const bool tiles = type != LC_TYPE_F32 && a.dim <= kTileDim && a.near && (uint64_t)a.most * a.shared > kFewQueries;
  // The long sequences first: the short ones then fill the SMs as those end.
  AttendArgs b = a;
  if (tiles) {
    a.longest = kFewQueries / a.shared;
    b.shortest = a.longest + 1;
    b.flat = reinterpret_cast<unsigned long long*>(reinterpret_cast<uint8_t*>(a.flat) + flat_bytes(how->sequences));
    b.parts = a.parts + 2 * kMaxParts * kPartBytes / 4;
    if (cache->slots == 0) b.codes = static_cast<const uint8_t*>(workspace);  // nothing is read there, but the address is formed
    e = launch_attend_tiles(b, bits, type, cs);
  }
  if (e == cudaSuccess && a.longest > 0)
    e = type == LC_TYPE_BF16 ? launch_attend_bf16(a, bits, tiles, cs) : type == LC_TYPE_F16 ? launch_attend_f16(a, bits, tiles, cs) : launch_attend_f32(a, bits, tiles, cs);
  if (tiles && e == cudaSuccess) e = launch_join_tiles(b, type, cs);
  return e == cudaSuccess ? LC_OK : LC_ERR_CUDA;
}

}  // extern "C"
