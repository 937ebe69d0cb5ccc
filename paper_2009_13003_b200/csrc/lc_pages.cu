// The plan of a step: where each sequence's new rows begin, the pages that it gets, and the slot of every row.
#include "lc_quant.cuh"

namespace lc {
namespace {

constexpr uint32_t kPlanThreads = 512, kPlanCtas = 8;  // CTAs: a portable cluster
constexpr uint32_t kPlanHere = 4096;                   // rows whose slots the first launch writes itself
constexpr uint32_t kSearch = 4096;                     // sequences whose beginnings fit into shared memory
constexpr uint32_t kSlotThreads = 256, kSlotRows = 4;  // rows of a thread

struct PlanArgs {
  int32_t* table;
  uint64_t table_stride;
  const int32_t* held;
  int32_t* spare;
  const int32_t* count;
  const int32_t* tokens;
  int32_t *begin, *first;
  int64_t* slots;
  int32_t *held_after, *count_after, *status;
  uint64_t room;  // positions that a sequence's row of the table has pages for
  uint32_t sequences, pages, rows;
  FastDiv by_page;
};

// The CTAs of the cluster meet, and see what the others wrote ahead of it. One alone needs less.
__device__ __forceinline__ void cluster_meet() {
  if (gridDim.x == 1) {
    __syncthreads();
    return;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t pages_of(const FastDiv& by_page, int32_t positions) {  // of 0 <= positions
  return positions ? by_page.div((uint32_t)positions - 1) + 1 : 0;
}

// What sequences ask for: rows, pages that they get, pages that they give back.
struct Ask {
  uint64_t rows, wants, gives;
};
__device__ __forceinline__ Ask operator+(Ask a, Ask b) { return Ask{a.rows + b.rows, a.wants + b.wants, a.gives + b.gives}; }

// A sequence of a plan that holds: what it asks for, its position ahead of the step.
__device__ __forceinline__ Ask ask(const PlanArgs& A, int32_t held, int32_t tokens, int32_t& first) {
  first = tokens < 0 ? 0 : held;
  if (tokens < 0) return Ask{0, 0, pages_of(A.by_page, held)};
  return Ask{(uint64_t)tokens, pages_of(A.by_page, held + tokens) - pages_of(A.by_page, held), 0};
}

// The slot of a row. begins, firsts: where the sequences begin, and at which position, in shared memory where that fits.
__device__ __forceinline__ void write_slot(const PlanArgs& A, const int32_t* begins, const int32_t* firsts, uint32_t row) {
  uint32_t lo = 0, hi = A.sequences;
  while (lo < hi) {
    const uint32_t mid = (lo + hi) / 2;
    if ((uint32_t)begins[mid + 1] <= row) lo = mid + 1;
    else hi = mid;
  }
  int64_t slot = -1;
  if (lo < A.sequences) {
    const uint32_t at = (uint32_t)firsts[lo] + (row - (uint32_t)begins[lo]), page = A.by_page.div(at);
    const int32_t number = A.table[lo * A.table_stride + page];
    if (number >= 0 && (uint32_t)number < A.pages) slot = (int64_t)number * A.by_page.d + (at - page * A.by_page.d);
    else if (A.status) set_status(A.status, LC_ERR_INDEX);
  }
  A.slots[row] = slot;
}

// f(lane of the sequence, page of it) for n pages of each lane's sequence, a page a lane: sequences of a few pages and of many take their turns side by side.
template <class F>
__device__ __forceinline__ void for_pages(uint32_t n, F f) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t upto = n;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= (uint32_t)d) upto += x;
  }
  const uint32_t all = __shfl_sync(0xFFFFFFFFu, upto, 31);
#pragma unroll 4
  for (uint32_t base = 0; base < all; base += 32) {
    uint32_t owner = 0;  // the first lane whose pages end behind this one
#pragma unroll
    for (uint32_t step = 16; step; step >>= 1)
      if (__shfl_sync(0xFFFFFFFFu, upto, owner + step - 1) <= base + lane) owner += step;
    const uint32_t before = __shfl_sync(0xFFFFFFFFu, upto - n, owner);
    f(owner, base + lane - before, base + lane < all);
  }
}

// One cluster. Every thread takes a strip of neighbouring sequences; the threads' sums are added up within the CTA, the CTAs' read from each
// other's shared memory, so that each knows what those ahead of it ask for, and all know whether the step fits, before anything is
// written. Three meetings of the cluster: all have read the books (which may be written in place); pages given back are in the list;
// pages taken off it are in the table. Latency bounds it (a few loads one behind the other, and the meetings).
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(PlanArgs A) {
  __shared__ Ask warps[kPlanThreads / 32];
  __shared__ Ask mine;
  __shared__ uint32_t faults;
  __shared__ int32_t begins[kPlanThreads + 1], firsts[kPlanThreads];  // of one CTA alone
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, all = gridDim.x * kPlanThreads, me = blockIdx.x * kPlanThreads + threadIdx.x;
  const uint32_t strip = (A.sequences + all - 1) / all;
  const uint32_t from = (uint32_t)min((uint64_t)me * strip, (uint64_t)A.sequences), to = (uint32_t)min((uint64_t)from + strip, (uint64_t)A.sequences);
  begin_next();
  if (threadIdx.x == 0) faults = 0;
  __syncthreads();

  const int32_t count = *A.count;
  Ask sum = {0, 0, 0};
  uint32_t bad = 0;  // 1: the books are wrong, 2: no room
  int32_t held = 0, tokens = 0, first = 0, after = 0;  // of a strip of one sequence all the way
  for (uint32_t s = from; s < to; ++s) {
    held = A.held[s], tokens = A.tokens[s];
    if (held < 0 || (uint64_t)held > A.room) bad |= 1;
    else if (tokens > 0 && (uint64_t)held + (uint64_t)tokens > A.room) bad |= 2;
    else sum = sum + ask(A, held, tokens, first);
  }
  if (bad) atomicOr(&faults, bad);
  Ask ahead = sum;  // of this thread's strip and those before it in the warp
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const Ask x = {__shfl_up_sync(0xFFFFFFFFu, ahead.rows, d), __shfl_up_sync(0xFFFFFFFFu, ahead.wants, d), __shfl_up_sync(0xFFFFFFFFu, ahead.gives, d)};
    if (lane >= (uint32_t)d) ahead = ahead + x;
  }
  if (lane == 31) warps[warp] = ahead;
  ahead = Ask{ahead.rows - sum.rows, ahead.wants - sum.wants, ahead.gives - sum.gives};
  __syncthreads();
  Ask cta = {0, 0, 0};
  for (uint32_t w = 0; w < kPlanThreads / 32; ++w) {
    if (w == warp) ahead = ahead + cta;
    cta = cta + warps[w];
  }
  if (threadIdx.x == 0) mine = cta;
  cluster_meet();

  Ask whole = {0, 0, 0};
  uint32_t fault = 0;
  for (uint32_t c = 0; c < gridDim.x; ++c) {
    Ask x;
    uint32_t f, at = (uint32_t)__cvta_generic_to_shared(&mine), flag = (uint32_t)__cvta_generic_to_shared(&faults);
    asm volatile("{ .reg .u32 a; mapa.shared::cluster.u32 a, %3, %4; ld.shared::cluster.u64 %0, [a]; ld.shared::cluster.u64 %1, [a + 8]; ld.shared::cluster.u64 %2, [a + 16]; }"
                 : "=l"(x.rows), "=l"(x.wants), "=l"(x.gives)
                 : "r"(at), "r"(c)
                 : "memory");
    asm volatile("{ .reg .u32 a; mapa.shared::cluster.u32 a, %1, %2; ld.shared::cluster.u32 %0, [a]; }" : "=r"(f) : "r"(flag), "r"(c) : "memory");
    if (c == blockIdx.x) ahead = ahead + whole;
    whole = whole + x;
    fault |= f;
  }
  if (count < 0 || (uint64_t)count + whole.gives > A.pages) fault |= 1;
  else if (whole.wants > (uint64_t)count + whole.gives || whole.rows > A.rows) fault |= 2;
  const uint32_t top = (uint32_t)count + (uint32_t)whole.gives;  // pages in the list once all are back
  const bool ok = fault == 0, here = gridDim.x == 1 && strip <= 1;
  if (me == 0) {
    if (!ok && A.status) set_status(A.status, fault & 1 ? LC_ERR_INDEX : LC_ERR_CAPACITY);
    *A.count_after = ok ? (int32_t)(top - (uint32_t)whole.wants) : count;
    A.begin[A.sequences] = ok ? (int32_t)whole.rows : 0;
    if (here) begins[A.sequences] = ok ? (int32_t)whole.rows : 0;
  }

  // a warp's sequences: books by its lanes, pages of one sequence after the other by all of them
  const Ask start = ahead;
  for (uint32_t k = 0; k < strip; ++k) {
    const uint32_t s = from + k;
    const bool there = s < to;
    Ask x = {0, 0, 0};
    if (there) {
      if (strip > 1) held = A.held[s], tokens = A.tokens[s];
      first = held;
      if (ok) x = ask(A, held, tokens, first);
      after = first + (int32_t)x.rows;
      const int32_t begin = ok ? (int32_t)ahead.rows : 0;
      A.begin[s] = begin;
      A.first[s] = first;
      A.held_after[s] = after;
      if (here) begins[s] = begin, firsts[s] = first;
    }
    const uint32_t behind = (uint32_t)count + (uint32_t)ahead.gives;
    if (__any_sync(0xFFFFFFFFu, x.gives > 0))
      for_pages((uint32_t)x.gives, [&](uint32_t owner, uint32_t i, bool is) {
        const uint32_t seq = __shfl_sync(0xFFFFFFFFu, s, owner), to_list = __shfl_sync(0xFFFFFFFFu, behind, owner);
        if (is) A.spare[to_list + i] = A.table[seq * A.table_stride + i];
      });
    ahead = ahead + x;
  }
  cluster_meet();
  if (ok) {
    uint32_t wants = (uint32_t)start.wants;
    for (uint32_t k = 0; k < strip; ++k) {
      const uint32_t s = from + k;
      uint32_t has = 0, n = 0;
      if (s < to) {
        if (strip > 1) first = A.first[s], after = A.held_after[s];
        has = pages_of(A.by_page, first);
        n = pages_of(A.by_page, after) - has;
      }
      if (__any_sync(0xFFFFFFFFu, n > 0))
        for_pages(n, [&](uint32_t owner, uint32_t i, bool is) {
          const uint32_t seq = __shfl_sync(0xFFFFFFFFu, s, owner), j = __shfl_sync(0xFFFFFFFFu, has, owner), last = top - 1 - __shfl_sync(0xFFFFFFFFu, wants, owner);
          if (is) A.table[seq * A.table_stride + j + i] = A.spare[last - i];
        });
      wants += n;
    }
  }
  if (A.rows > kPlanHere) return;
  cluster_meet();
  for (uint32_t row = me; row < A.rows; row += all) write_slot(A, here ? begins : A.begin, here ? firsts : A.first, row);
}

// The slots of a larger batch, a second launch over all SMs.
__global__ void __launch_bounds__(kSlotThreads) slots_kernel(PlanArgs A) {
  __shared__ int32_t begins[kSearch + 1];
  wait_previous();
  const bool here = A.sequences <= kSearch;
  if (here) {
    for (uint32_t i = threadIdx.x; i <= A.sequences; i += kSlotThreads) begins[i] = A.begin[i];
    __syncthreads();
  }
#pragma unroll
  for (uint32_t k = 0; k < kSlotRows; ++k) {
    const uint64_t row = ((uint64_t)blockIdx.x * kSlotRows + k) * kSlotThreads + threadIdx.x;
    if (row < A.rows) write_slot(A, here ? begins : A.begin, A.first, (uint32_t)row);
  }
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" int lc_cache_plan(const lc_pages* pages, const int32_t* tokens, uint32_t sequences, uint64_t rows, int32_t* begin, int32_t* first, int64_t* slots,
                             int32_t* held_after, int32_t* count_after, int32_t* status, lc_cuda_stream_t cs) {
  if (!pages || pages->page < 1 || pages->page >= (1u << 31) || pages->pages >= (1u << 31) || sequences >= (1u << 31) || rows >= (1ull << 31) ||
      pages->table_stride >= (1ull << 32) || (sequences > 1 && pages->table_stride < pages->width))
    return LC_ERR_ARG;
  if (!pages->count || !count_after || !begin || !aligned_to(pages->table, 4) || !aligned_to(pages->held, 4) || !aligned_to(pages->spare, 4) ||
      !aligned_to(pages->count, 4) || !aligned_to(tokens, 4) || !aligned_to(begin, 4) || !aligned_to(first, 4) || !aligned_to(slots, 8) ||
      !aligned_to(held_after, 4) || !aligned_to(count_after, 4) || !aligned_to(status, 4))
    return LC_ERR_ARG;
  if (sequences > 0 && (!tokens || !first || !pages->held || !held_after || (pages->width > 0 && !pages->table))) return LC_ERR_ARG;
  if ((rows > 0 && !slots) || (pages->pages > 0 && !pages->spare)) return LC_ERR_ARG;
  PlanArgs a = {};
  a.table = pages->table;
  a.table_stride = pages->table_stride;
  a.held = pages->held;
  a.spare = pages->spare;
  a.count = pages->count;
  a.tokens = tokens;
  a.begin = begin;
  a.first = first;
  a.slots = slots;
  a.held_after = held_after;
  a.count_after = count_after;
  a.status = status;
  const uint64_t room = (uint64_t)pages->width * pages->page;
  a.room = room < 0x7FFFFFFFull ? room : 0x7FFFFFFFull;
  a.sequences = sequences;
  a.pages = pages->pages;
  a.rows = (uint32_t)rows;
  a.by_page = FastDiv(pages->page);

  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sequences > kPlanThreads ? kPlanCtas : 1);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.stream = cs;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cfg.gridDim.x;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, plan_kernel, a) != cudaSuccess) return LC_ERR_CUDA;
  if (rows > kPlanHere && launch_kernel(true, slots_kernel, (unsigned)((rows + kSlotThreads * kSlotRows - 1) / (kSlotThreads * kSlotRows)), kSlotThreads, 0, cs, a) != cudaSuccess)
    return LC_ERR_CUDA;
  return LC_OK;
}
