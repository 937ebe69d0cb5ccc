// A cache of keys and values in 8 or 4 bits: rows quantised as they are written, and read back by slots or through a table of pages.
#include "lc_quant.cuh"

namespace lc {
namespace {

constexpr int kThreads = 256;

struct CacheArgs {
  uint8_t* codes;
  unsigned short* scales;
  uint64_t slots;
  uint32_t heads, dim, groups, row_bytes;  // groups per row of dim values
  uint32_t per_plane, per_row;                        // lanes: of a plane's row, of all planes'
  uint32_t width_log;                                 // of the lanes of a warp that a row gets: less than all, if they are enough
  FastDiv by_head, by_warps;                          // lanes of a head, warps that share a row
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

// A warp takes a row (with few rows several share one; short rows share a warp): its place is looked up once for all planes and heads. group / 16 lanes hold
// a group, 16 values each: neighbouring ones where they are quantised; where they are read, runs of 16 bytes of the output, so that
// the lanes' runs follow each other. One pass over the rows; from and to 16 bits the instructions of the codes weigh as much as the bytes
// (reading 131072 rows of 8 x 128 from 4 bits to bf16, twice: 116 us; with one run of 8 values a lane, and so twice the index arithmetic, 177).
struct Lane {
  uint32_t plane, head, part;  // part: which of the head's lanes
};
__device__ __forceinline__ Lane lane_of(const CacheArgs& C, uint32_t j) {
  Lane l;
  l.plane = j >= C.per_plane;
  const uint32_t v = j - (l.plane ? C.per_plane : 0);
  l.head = C.by_head.div(v);
  l.part = v - l.head * C.by_head.d;
  return l;
}

// 131072 rows of 8 x 128, keys and values: bf16 to 4 bits 160 us (the bytes take 104; 238 instructions for 16 values a lane), fp32 to 8
// bits 212 (206). With registers for six CTAs an SM 154 and 219: what is spilled costs as much as the warps bring.
// kWhole: dim is a multiple of 16, and so are the addresses of all heads' rows (in bytes): nothing is cut off and nothing to be looked at a lane.
template <class T, int G, int kBits, bool kWhole>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheArgs C, Planes src, Places P, uint32_t rows, int32_t* status) {
  constexpr int kLanes = G / 16;
  const uint32_t warp = (uint32_t)(((uint64_t)blockIdx.x * kThreads + threadIdx.x) >> 5), width = 1u << C.width_log;
  const uint32_t lane = threadIdx.x & (width - 1), share = C.by_warps.div(warp), row = (share << (5 - C.width_log)) + ((threadIdx.x & 31) >> C.width_log);
  if (row >= rows) return;  // a row's lanes together
  bool bad = false;
  const int64_t slot = slot_of<false>(P, row, C.slots, bad);
  if (bad && status && lane == 0) set_status(status, LC_ERR_INDEX);
  if (slot < 0) return;
  for (uint32_t j0 = (warp - share * C.by_warps.d) * 32; j0 < C.per_row; j0 += C.by_warps.d * 32) {
    const bool inside = j0 + lane < C.per_row;
    const Lane l = lane_of(C, inside ? j0 + lane : 0);
    const uint32_t at = l.part * 16;
    const Rows R = l.plane ? src.plane[1] : src.plane[0];
    const T* p = reinterpret_cast<const T*>(R.data) + row * R.row_stride + l.head * R.head_stride + at;
    const int valid = inside ? (int)C.dim - (int)at : 0;
    float v[16] = {}, m = 0.0f;
    if constexpr (kWhole) {
      if (valid > 0) m = load16(p, v);
    } else {
      load8(p, valid, v);
      load8(p + 8, valid - 8, v + 8);
#pragma unroll
      for (int i = 0; i < 16; ++i) m = max_magnitude(m, v[i]);
    }
    const uint32_t scale = group_scale<kBits>(max_over_lanes(m, kLanes));
    if (valid <= 0) continue;
    float t[16];
    codes<T, kBits>(v, scale, t);
    const uint64_t place = (l.plane * C.slots + (uint64_t)slot) * C.heads + l.head;
    uint8_t* o = C.codes + place * C.row_bytes + at * kBits / 8;
    if constexpr (kBits == 4) {
      const uint32_t a = pack4(t), b = pack4(t + 8);
      if (kWhole || (valid > 8 && (reinterpret_cast<uintptr_t>(o) & 7) == 0)) {
        *reinterpret_cast<uint2*>(o) = make_uint2(a, b);
      } else {
        *reinterpret_cast<uint32_t*>(o) = a;
        if (valid > 8) *reinterpret_cast<uint32_t*>(o + 4) = b;
      }
    } else {
      const uint2 a = pack8(t), b = pack8(t + 8);
      if (kWhole || (valid > 8 && (reinterpret_cast<uintptr_t>(o) & 15) == 0)) {
        *reinterpret_cast<uint4*>(o) = make_uint4(a.x, a.y, b.x, b.y);
      } else {
        *reinterpret_cast<uint2*>(o) = a;
        if (valid > 8) *reinterpret_cast<uint2*>(o + 8) = b;
      }
    }
    if ((lane & (kLanes - 1)) == 0) C.scales[place * C.groups + at / G] = (unsigned short)(scale >> 16);
  }
}

// Four values' codes of 4 bits, of a word that holds eight: the first four are in its bytes 0 and 2, the others in 1 and 3.
__device__ __forceinline__ uint32_t half_word(const uint8_t* p, uint32_t at) {
  return *reinterpret_cast<const uint32_t*>(p - (at & 4) / 2) >> ((at & 4) * 2);
}

template <class T, int G, int kBits, bool kPages, bool kWhole>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(CacheArgs C, Planes out, Places P, uint32_t rows, int32_t* status) {
  constexpr uint32_t kLanes = G / 16, n = kRun<T>, kRuns = 16 / n;
  const uint32_t warp = (uint32_t)(((uint64_t)blockIdx.x * kThreads + threadIdx.x) >> 5), width = 1u << C.width_log;
  const uint32_t lane = threadIdx.x & (width - 1), share = C.by_warps.div(warp), row = (share << (5 - C.width_log)) + ((threadIdx.x & 31) >> C.width_log);
  if (row >= rows) return;
  bool bad = false;
  const int64_t slot = slot_of<kPages>(P, row, C.slots, bad);
  if (bad && status && lane == 0) set_status(status, LC_ERR_INDEX);
  if (slot < 0) return;
  for (uint32_t j = (warp - share * C.by_warps.d) * 32 + lane; j < C.per_row; j += C.by_warps.d * 32) {
    const Lane l = lane_of(C, j);
    const uint32_t group = l.part / kLanes, at = group * G + (l.part & (kLanes - 1)) * n;  // of the first run
    const uint64_t place = (l.plane * C.slots + (uint64_t)slot) * C.heads + l.head;
    const uint8_t* p = C.codes + place * C.row_bytes + at * kBits / 8;
    const bool whole = kWhole && (group + 1) * G <= C.dim;  // the row's last group may be short
    uint2 w[kRuns];
#pragma unroll
    for (uint32_t k = 0; k < kRuns; ++k) {
      constexpr uint32_t kStep = kLanes * n * kBits / 8;
      w[k] = make_uint2(0, 0);
      if (!whole && at + k * kLanes * n >= C.dim) continue;
      if constexpr (n * kBits == 16) w[k].x = half_word(p + k * kStep, at);
      else if constexpr (n * kBits == 32) w[k].x = *reinterpret_cast<const uint32_t*>(p + k * kStep);
      else w[k] = *reinterpret_cast<const uint2*>(p + k * kStep);
    }
    const float scale = __uint_as_float((uint32_t)C.scales[place * C.groups + group] << 16);
    const Rows R = l.plane ? out.plane[1] : out.plane[0];
    T* o = reinterpret_cast<T*>(R.data) + row * R.row_stride + l.head * R.head_stride + at;
#pragma unroll
    for (uint32_t k = 0; k < kRuns; ++k) {
      const uint32_t first = at + k * kLanes * n;
      if (!whole && first >= C.dim) continue;
      float v[n];
      values_in_row<kBits, n>(w[k], scale, v);
      keep_in_type<T, kBits>(scale, v);
      store_run<kWhole>(o + k * kLanes * n, (int)min(n, C.dim - first), v);
    }
  }
}

uint32_t row_bytes(const lc_cache* c) { return (c->dim + 7) / 8 * c->bits; }
// Codes of less than 2^62 bytes (scales take no more): every size and offset fits 64 bits.
bool cache_ok(const lc_cache* c) {
  return c && (c->bits == 4 || c->bits == 8) && group_ok((int)c->group) && (c->planes == 1 || c->planes == 2) && c->heads >= 1 && c->heads <= 65536 &&
         c->dim >= 1 && c->dim <= 65536 && (uint64_t)c->heads * c->dim < (1ull << 31) && c->slots < (1ull << 40) &&
         c->slots <= ((1ull << 62) - 1) / ((uint64_t)c->planes * c->heads * row_bytes(c));
}

uint32_t row_groups(const lc_cache* c) { return (c->dim + c->group - 1) / c->group; }

CacheArgs cache_args(const lc_cache* c, uint64_t rows) {
  const uint32_t lanes = row_groups(c) * (c->group / 16);  // of a head
  CacheArgs a = {};
  a.codes = static_cast<uint8_t*>(c->codes);
  a.scales = static_cast<unsigned short*>(c->scales);
  a.slots = c->slots;
  a.heads = c->heads;
  a.dim = c->dim;
  a.row_bytes = row_bytes(c);
  a.groups = row_groups(c);
  a.per_plane = c->heads * lanes;
  a.per_row = a.per_plane * c->planes;
  a.by_head = FastDiv(lanes);
  // with few rows several warps share one, so that some thousands of them have work
  const uint64_t turns = ((uint64_t)a.per_row + 31) / 32, wanted = (4096 + rows - 1) / rows;
  a.by_warps = FastDiv((uint32_t)(wanted < turns ? wanted : turns));
  while ((1u << a.width_log) < a.per_row && a.width_log < 5) ++a.width_log;
  return a;
}

// The rows of a call: every plane's pointer and strides. written: no two rows may share memory.
int check_rows(const lc_cache* c, const lc_rows* rows, int type, uint64_t n, bool written) {
  if (!cache_ok(c) || !type_ok(type) || !rows) return LC_ERR_ARG;
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

using Kernel = void (*)(CacheArgs, Planes, Places, uint32_t, int32_t*);

int launch_rows(Kernel kernel, const lc_cache* c, const lc_rows* rows, const Places& places, uint64_t n, int32_t* status, cudaStream_t cs) {
  const CacheArgs a = cache_args(c, n);
  const uint64_t shares = (n + (32 >> a.width_log) - 1) >> (5 - a.width_log);
  const unsigned grid = (unsigned)((shares * a.by_warps.d * 32 + kThreads - 1) / kThreads);
  return launch_kernel(false, kernel, grid, kThreads, 0, cs, a, planes_of(c, rows), places, (uint32_t)n, status) == cudaSuccess ? LC_OK : LC_ERR_CUDA;
}

template <class T, int G, bool kWhole>
Kernel write_kernel(int bits) { return bits == 4 ? cache_write_kernel<T, G, 4, kWhole> : cache_write_kernel<T, G, 8, kWhole>; }
template <class T, bool kWhole>
Kernel write_kernel(int group, int bits) {
  return group == 32 ? write_kernel<T, 32, kWhole>(bits) : group == 64 ? write_kernel<T, 64, kWhole>(bits) : write_kernel<T, 128, kWhole>(bits);
}
template <class T, int G, bool kPages, bool kWhole>
Kernel read_kernel(int bits) { return bits == 4 ? cache_read_kernel<T, G, 4, kPages, kWhole> : cache_read_kernel<T, G, 8, kPages, kWhole>; }
template <class T, bool kPages, bool kWhole>
Kernel read_kernel(int group, int bits) {
  return group == 32 ? read_kernel<T, 32, kPages, kWhole>(bits) : group == 64 ? read_kernel<T, 64, kPages, kWhole>(bits) : read_kernel<T, 128, kPages, kWhole>(bits);
}

// Whether all rows of a call are whole runs of 16 values on 16 bytes.
bool whole_rows(const lc_cache* c, const lc_rows* rows, int type) {
  const uint64_t run = 16 / type_bytes(type);
  bool whole = c->dim % 16 == 0;
  for (uint32_t i = 0; i < c->planes; ++i) whole &= aligned_to(rows[i].data, 16) && rows[i].row_stride % run == 0 && rows[i].head_stride % run == 0;
  return whole;
}

template <bool kPages>
int read_impl(const lc_cache* c, const lc_rows* out, int type, const Places& places, uint64_t n, int32_t* status, cudaStream_t cs) {
  const int group = (int)c->group, bits = (int)c->bits;
  Kernel kernel;
  if (whole_rows(c, out, type))
    kernel = type == LC_TYPE_F32    ? read_kernel<float, kPages, true>(group, bits)
             : type == LC_TYPE_BF16 ? read_kernel<__nv_bfloat16, kPages, true>(group, bits)
                                    : read_kernel<__half, kPages, true>(group, bits);
  else
    kernel = type == LC_TYPE_F32    ? read_kernel<float, kPages, false>(group, bits)
             : type == LC_TYPE_BF16 ? read_kernel<__nv_bfloat16, kPages, false>(group, bits)
                                    : read_kernel<__half, kPages, false>(group, bits);
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
  const int group = (int)cache->group, bits = (int)cache->bits;
  Kernel kernel;
  if (whole_rows(cache, src, type))
    kernel = type == LC_TYPE_F32    ? write_kernel<float, true>(group, bits)
             : type == LC_TYPE_BF16 ? write_kernel<__nv_bfloat16, true>(group, bits)
                                    : write_kernel<__half, true>(group, bits);
  else
    kernel = type == LC_TYPE_F32    ? write_kernel<float, false>(group, bits)
             : type == LC_TYPE_BF16 ? write_kernel<__nv_bfloat16, false>(group, bits)
                                    : write_kernel<__half, false>(group, bits);
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
