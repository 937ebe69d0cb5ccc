// A cache of keys and values in 8 or 4 bits: rows quantised as they are written, and read back by slots or through a table of pages.
#include "lc_quant.cuh"

namespace lc {
namespace {

constexpr int kThreads = 256;

struct CacheArgs {
  uint8_t* codes;
  unsigned short* scales;
  uint64_t slots;
  uint32_t heads, dim, groups, lanes, row_bytes, bits;  // groups per row of dim values; lanes: of 8 values, per group
  FastDiv by_row, by_groups;                            // items (head, group) per row; groups per head
};

struct Rows {  // the caller's rows of one plane
  uint8_t* data;
  uint64_t row_stride, head_stride;  // in values
};
struct Planes {
  Rows plane[2];
};

// Where the rows of a call are in the cache: a slot for each, or sequences in pages.
struct Places {
  const int64_t* slots;
  const int32_t* table;  // [sequences][table_stride]: pages
  uint64_t table_stride;
  const int32_t* begin;  // [sequences + 1]: a sequence's first row
  const int32_t* first;  // position of a sequence's first row in it; null: 0
  uint32_t sequences, width;
  FastDiv by_page;
};

// The slot of a row, or -1 for one that has none. bad: it names a place that does not exist.
template <bool kPages>
__device__ __forceinline__ int64_t slot_of(const Places& P, uint32_t row, uint64_t slots, bool& bad) {
  int64_t slot;
  if constexpr (kPages) {
    // the last sequence that begins at or ahead of the row: empty ones share their begin with the next
    uint32_t lo = 0, hi = P.sequences;
    while (lo < hi) {
      const uint32_t mid = (lo + hi) / 2;
      if ((int64_t)__ldg(P.begin + mid + 1) <= (int64_t)row) lo = mid + 1;
      else hi = mid;
    }
    if (lo >= P.sequences) return -1;  // behind the last sequence
    const int64_t begin = __ldg(P.begin + lo);
    const int64_t at = (int64_t)row - begin + (P.first ? (int64_t)__ldg(P.first + lo) : 0);
    if (begin > (int64_t)row || at < 0 || at >= (int64_t)P.width * P.by_page.d || at >= (1ll << 31)) {
      bad = begin <= (int64_t)row;
      return -1;
    }
    const uint32_t page = P.by_page.div((uint32_t)at);
    const int64_t number = __ldg(P.table + lo * P.table_stride + page);
    if (number < 0) {
      bad = true;
      return -1;
    }
    slot = number * P.by_page.d + (at - (int64_t)page * P.by_page.d);
  } else {
    slot = __ldg(P.slots + row);
    if (slot == -1) return -1;
  }
  if (slot < 0 || slot >= (int64_t)slots) {
    bad = true;
    return -1;
  }
  return slot;
}

// group / 8 lanes hold a group, eight values each; one pass over the rows, bound by memory.
template <class T>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheArgs C, Planes src, Places P, uint32_t items, int32_t* status) {
  const uint32_t item = (uint32_t)(((uint64_t)blockIdx.x * kThreads + threadIdx.x) / C.lanes);
  const uint32_t lane = threadIdx.x & (C.lanes - 1);
  const bool inside = item < items;
  const uint32_t row = inside ? C.by_row.div(item) : 0, hg = inside ? item - row * C.by_row.d : 0;
  const uint32_t head = C.by_groups.div(hg), g = hg - head * C.groups;
  bool bad = false;
  const int64_t slot = inside ? slot_of<false>(P, row, C.slots, bad) : -1;
  if (bad && status) set_status(status, LC_ERR_INDEX);
  const uint32_t at = (g * C.lanes + lane) * 8;
  const int valid = slot < 0 || at >= C.dim ? 0 : (int)min(8u, C.dim - at);
  const Rows& R = src.plane[blockIdx.y];
  float v[8];
  load8(reinterpret_cast<const T*>(R.data) + row * R.row_stride + head * R.head_stride + at, valid, v);
  const uint32_t scale = group_scale(max_over_lanes(max_bits8(v), (int)C.lanes), C.bits == 4 ? 7.0f : 127.0f);
  if (valid == 0) return;
  int q[8];
  codes8(v, scale, q);
  const uint64_t place = (blockIdx.y * C.slots + (uint64_t)slot) * C.heads + head;
  uint8_t* o = C.codes + place * C.row_bytes + at * C.bits / 8;
  if (C.bits == 4) *reinterpret_cast<uint32_t*>(o) = pack4(q);
  else *reinterpret_cast<uint2*>(o) = pack8(q);
  if (lane == 0) C.scales[place * C.groups + g] = (unsigned short)(scale >> 16);
}

template <class T, bool kPages>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(CacheArgs C, Planes out, Places P, uint32_t items, int32_t* status) {
  const uint32_t item = (uint32_t)(((uint64_t)blockIdx.x * kThreads + threadIdx.x) / C.lanes);
  if (item >= items) return;
  const uint32_t lane = threadIdx.x & (C.lanes - 1);
  const uint32_t row = C.by_row.div(item), hg = item - row * C.by_row.d;
  const uint32_t head = C.by_groups.div(hg), g = hg - head * C.groups;
  bool bad = false;
  const int64_t slot = slot_of<kPages>(P, row, C.slots, bad);
  if (bad && status) set_status(status, LC_ERR_INDEX);
  const uint32_t at = (g * C.lanes + lane) * 8;
  if (slot < 0 || at >= C.dim) return;
  const uint64_t place = (blockIdx.y * C.slots + (uint64_t)slot) * C.heads + head;
  const uint8_t* p = C.codes + place * C.row_bytes + at * C.bits / 8;
  const float scale = __uint_as_float((uint32_t)C.scales[place * C.groups + g] << 16);
  float v[8];
  if (C.bits == 4) values_of4(*reinterpret_cast<const uint32_t*>(p), scale, v);
  else values_of8(*reinterpret_cast<const uint2*>(p), scale, v);
  const Rows& R = out.plane[blockIdx.y];
  store8(reinterpret_cast<T*>(R.data) + row * R.row_stride + head * R.head_stride + at, (int)min(8u, C.dim - at), v);
}

bool cache_ok(const lc_cache* c) {
  return c && (c->bits == 4 || c->bits == 8) && group_ok((int)c->group) && (c->planes == 1 || c->planes == 2) && c->heads >= 1 && c->heads <= 65536 &&
         c->dim >= 1 && c->dim <= 65536 && c->slots < (1ull << 40);
}

uint32_t row_bytes(const lc_cache* c) { return (c->dim + 7) / 8 * c->bits; }
uint32_t row_groups(const lc_cache* c) { return (c->dim + c->group - 1) / c->group; }

CacheArgs cache_args(const lc_cache* c) {
  CacheArgs a = {};
  a.codes = static_cast<uint8_t*>(c->codes);
  a.scales = static_cast<unsigned short*>(c->scales);
  a.slots = c->slots;
  a.heads = c->heads;
  a.dim = c->dim;
  a.bits = c->bits;
  a.row_bytes = row_bytes(c);
  a.groups = row_groups(c);
  a.lanes = c->group / 8;
  a.by_row = FastDiv(a.heads * a.groups);
  a.by_groups = FastDiv(a.groups);
  return a;
}

// The rows of a call: every plane's pointer and strides. written: no two rows may share memory.
int check_rows(const lc_cache* c, const lc_rows* rows, int type, uint64_t n, bool written) {
  if (!cache_ok(c) || !type_ok(type) || !rows) return LC_ERR_ARG;
  if ((uint64_t)c->heads * row_groups(c) >= (1ull << 31)) return LC_ERR_ARG;
  if (n == 0) return LC_OK;
  if (n >= (1ull << 31) || n * c->heads * row_groups(c) >= (1ull << 31)) return LC_ERR_ARG;
  if (c->slots > 0 && (!c->codes || !c->scales || !aligned_to(c->codes, 16) || !aligned_to(c->scales, 2))) return LC_ERR_ARG;
  for (uint32_t i = 0; i < c->planes; ++i) {
    const lc_rows& r = rows[i];
    if (!r.data || !aligned_to(r.data, type_bytes(type)) || r.row_stride >= (1ull << 33) || r.head_stride >= (1ull << 40)) return LC_ERR_ARG;
    const bool by_row = (c->heads == 1 || r.head_stride >= c->dim) && (n == 1 || r.row_stride >= (c->heads - 1) * r.head_stride + c->dim);
    const bool by_head = (n == 1 || r.row_stride >= c->dim) && (c->heads == 1 || r.head_stride >= (n - 1) * r.row_stride + c->dim);
    if (written && !by_row && !by_head) return LC_ERR_ARG;
  }
  return LC_OK;
}

Planes planes_of(const lc_cache* c, const lc_rows* rows) {
  Planes p = {};
  for (uint32_t i = 0; i < c->planes; ++i) p.plane[i] = Rows{static_cast<uint8_t*>(rows[i].data), rows[i].row_stride, rows[i].head_stride};
  return p;
}

int launch_rows(void (*kernel)(CacheArgs, Planes, Places, uint32_t, int32_t*), const lc_cache* c, const lc_rows* rows, const Places& places, uint64_t n,
                int32_t* status, cudaStream_t cs) {
  const CacheArgs a = cache_args(c);
  const uint32_t items = (uint32_t)n * a.by_row.d;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((uint64_t)items * a.lanes + kThreads - 1) / kThreads), c->planes);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = cs;
  return cudaLaunchKernelEx(&cfg, kernel, a, planes_of(c, rows), places, items, status) == cudaSuccess ? LC_OK : LC_ERR_CUDA;
}

template <bool kPages>
int read_impl(const lc_cache* c, const lc_rows* out, int type, const Places& places, uint64_t n, int32_t* status, cudaStream_t cs) {
  auto kernel = type == LC_TYPE_F32    ? cache_read_kernel<float, kPages>
                : type == LC_TYPE_BF16 ? cache_read_kernel<__nv_bfloat16, kPages>
                                       : cache_read_kernel<__half, kPages>;
  return launch_rows(kernel, c, out, places, n, status, cs);
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" {

uint64_t lc_cache_code_bytes(const lc_cache* cache) { return cache_ok(cache) ? cache->planes * cache->slots * cache->heads * row_bytes(cache) : 0; }
uint64_t lc_cache_scale_bytes(const lc_cache* cache) { return cache_ok(cache) ? cache->planes * cache->slots * cache->heads * row_groups(cache) * 2 : 0; }

int lc_cache_write(const lc_cache* cache, const lc_rows* src, int type, uint64_t rows, const int64_t* slots, int32_t* status, lc_cuda_stream_t cs) {
  const int rc = check_rows(cache, src, type, rows, false);
  if (rc != LC_OK || rows == 0) return rc;
  if (!slots || !aligned_to(slots, 8) || !aligned_to(status, 4)) return LC_ERR_ARG;
  Places places = {};
  places.slots = slots;
  places.by_page = FastDiv(1);
  auto kernel = type == LC_TYPE_F32 ? cache_write_kernel<float> : type == LC_TYPE_BF16 ? cache_write_kernel<__nv_bfloat16> : cache_write_kernel<__half>;
  return launch_rows(kernel, cache, src, places, rows, status, cs);
}

int lc_cache_read(const lc_cache* cache, const lc_rows* out, int type, uint64_t rows, const int64_t* slots, int32_t* status, lc_cuda_stream_t cs) {
  const int rc = check_rows(cache, out, type, rows, true);
  if (rc != LC_OK || rows == 0) return rc;
  if (!slots || !aligned_to(slots, 8) || !aligned_to(status, 4)) return LC_ERR_ARG;
  Places places = {};
  places.slots = slots;
  places.by_page = FastDiv(1);
  return read_impl<false>(cache, out, type, places, rows, status, cs);
}

int lc_cache_read_pages(const lc_cache* cache, const lc_rows* out, int type, uint64_t rows, const int32_t* table, uint64_t table_stride, uint32_t width,
                        uint32_t page, const int32_t* begin, const int32_t* first, uint32_t sequences, int32_t* status, lc_cuda_stream_t cs) {
  const int rc = check_rows(cache, out, type, rows, true);
  if (rc != LC_OK) return rc;
  if (page < 1 || page >= (1u << 31) || sequences >= (1u << 31) || table_stride >= (1ull << 32) || (sequences > 1 && table_stride < width)) return LC_ERR_ARG;
  if (rows == 0 || sequences == 0) return LC_OK;
  if ((width > 0 && !table) || !begin || !aligned_to(table, 4) || !aligned_to(begin, 4) || !aligned_to(first, 4) || !aligned_to(status, 4)) return LC_ERR_ARG;
  Places places = {};
  places.table = table;
  places.table_stride = table_stride;
  places.width = width;
  places.begin = begin;
  places.first = first;
  places.sequences = sequences;
  places.by_page = FastDiv(page);
  return read_impl<true>(cache, out, type, places, rows, status, cs);
}

}  // extern "C"
