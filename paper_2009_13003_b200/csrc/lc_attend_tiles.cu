// Attention to a quantised cache for sequences of many new rows: the products on the tensor cores' own memory (tcgen05).
//
// A CTA takes blocks of 256 queries of one head of the cache (its tokens, times the heads that share it) as two tiles of 128, and goes through the keys
// 128 at a time with a running maximum and sum of each query. Its warps have one task each: four read the keys' codes and four the values', turn them into
// numbers and store them as operands (both in one layout, rows of 64 values with the 128-byte swizzle: keys are read along a row, values across);
// two warps look up where the next tiles' keys lie, and their scales;
// a thread for each tile issues its products; a warpgroup for each tile takes the scores out of tensor memory, a query a thread, and puts the probabilities back
// there, over the scores, as the first operand of the product with the values. Scores go to the warps 64 keys at a time: while one half of a tile is with
// them, the products of the other half, and of the other tile, run.
// The sums of the values stay in tensor memory; they are scaled down only where a score exceeds the maximum so far by more than a factor of 2^kSlack.
//
// All products are of fp16 numbers, 11 bits, also for bf16 queries: a query's row is multiplied by the power of two that takes its largest value to [1, 2) (what
// that loses lies 2^-25 below it), keys are in units of the power of two in the largest scale of 16 neighbours, values in units of that of the block's
// values so far; where it rises the sums are scaled down. So no magnitude of them is out of the type, and what a code stands for is rounded once, to 11 bits. Where scales
// differ by more than 2^14 that would not hold, and a key that a row does not see would take bits from those that it sees: there each key has a unit of its own, and what that lacks goes
// to its score and, for its values, to its probability. (Such tiles go through a loop of their own; looking for them costs 2 %: chunks 639 -> 646 us, a prompt 888 -> 902.)
// Probabilities are held 2^7 times as large, up to 2^(7 + kSlack): next to its smallest numbers the type has few bits. (With keys, values and
// probabilities of bf16, 2 x 1024 rows behind up to 16384 keys took 602 us instead of 638, and the error was 0.0049 of the result instead of 0.0017, the result's own rounding.)
// A value of NaN enters as 0, or rows that do not see it would get 0 * NaN; rows that do get their NaN at the end.
//
// Blocks differ in how many keys they see. Each weighs about as many as it does and a block's own cost; a CTA gets an equal share of the weight, and
// of a block that it shares with its neighbours the tiles in proportion. Those parts are joined by a second launch, in a fixed order.
#include "lc_attend.cuh"

namespace lc {
namespace {

constexpr uint32_t kRows = 128, kKeys = 128, kHalf = 64;  // of a tile of queries, of keys, of the keys that are between products and warps at a time
constexpr uint32_t kSoftmaxWarps = 8, kReadWarps = 4;   // kReadWarps each for keys and for values, then two that issue and two that look up
constexpr uint32_t kThreads = 32 * (kSoftmaxWarps + 2 * kReadWarps + 4), kReaders = 32 * kReadWarps;
// Registers of a thread: as launched, and what each warpgroup then has (together no more than before).
constexpr uint32_t kRegsAtLaunch = 96, kRegsSoftmax = 144, kRegsReader = 64, kRegsIssue = 64;
static_assert(2 * kRegsSoftmax + 2 * kRegsReader + kRegsIssue <= 5 * kRegsAtLaunch && kThreads == 5 * 128, "registers of five warpgroups");
constexpr uint32_t kStages = 3;                         // halves of a tile of keys, and of values, as operands
constexpr uint32_t kAhead = 3;                          // halves whose codes are on their way
constexpr uint32_t kFound = 4;                          // tiles whose keys have been looked up
constexpr uint32_t kMemo = 8;                           // tiles whose units are kept: the scores of a tile are done before the keys of the seventh behind it are looked up (blocks have a tile or more)
constexpr float kSlack = 8.0f;
constexpr long long kWaitCycles = 4ll << 30;            // how long a barrier is waited for before the kernel gives up: some two seconds
// Up to this cap the form for large scores is taken for all of them: it is off by 2^-22 of the cap, which moves a weight by no more than 2^-16, and they have 11 bits here. (2 x
// 1024 rows behind up to 16384 keys, cap 3: 1031 us; with both forms and a choice for each score 1577. Where scores are far below their cap: the series alone, 890.)
constexpr float kPlainCap = 64.0f;
constexpr uint32_t kBlockCost = 320;                    // what a block costs beyond its keys, in keys: fitted to a prompt of 8192 (with 192 its first CTA took twice as long as the others)

// ---- barriers and tensor memory -----------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Waits for the end of the barrier's phase of that parity. False, and `dead` set for all, if it does not come within some seconds.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile uint32_t* dead) {
  long long since = 0;
  for (;;) {
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    if (done) return true;
    const long long now = clock64();
    if (since == 0) since = now;
    if (now - since > kWaitCycles) *dead = 1;
    if (*dead) return false;
  }
}
// The same for a warp as a whole: its threads go on together or not at all.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* dead) { return __all_sync(0xFFFFFFFFu, barrier_wait(bar, parity, dead)); }
// Whether all of a warpgroup's threads say so: they go on together or not at all.
__device__ __forceinline__ bool together(uint32_t barrier, bool good) {
  uint32_t all;
  asm volatile("{ .reg .pred p, r; setp.ne.b32 p, %3, 0; barrier.cta.red.and.pred r, %1, %2, p; selp.u32 %0, 1, 0, r; }" : "=r"(all) : "r"(barrier), "n"(kRows), "r"((uint32_t)good) : "memory");
  return all;
}
__device__ __forceinline__ void order_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void order_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit_to(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// An operand in rows of 128 bytes, swizzled, in groups of eight rows, 1024 bytes apart: the lower half of its descriptor, with `lead` bytes from one run of
// 64 values to the next where it is read across the rows (an address further on is a larger number), and the upper half.
__device__ __forceinline__ uint32_t operand_at(uint32_t address, uint32_t lead) { return (address >> 4 & 0x3FFF) | lead >> 4 << 16; }
constexpr uint32_t kOperandKind = 1024 >> 4 | 1u << 14 | 2u << 29;
// d (tensor memory) = or += a * b; a in shared or tensor memory. One thread issues all of a CTA's products, beside busy warps: few instructions each.
__device__ __forceinline__ void product(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 a, b; mov.b64 a, {%1, %5}; mov.b64 b, {%2, %5}; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p; }" ::"r"(d), "r"(a),
               "r"(b), "r"(what), "r"((uint32_t)add), "r"(kOperandKind)
               : "memory");
}
__device__ __forceinline__ void product_of_tensor(uint32_t d, uint32_t a, uint32_t b, uint32_t what, bool add) {
  asm volatile("{ .reg .pred p; .reg .b64 b; mov.b64 b, {%2, %5}; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p; }" ::"r"(d), "r"(a), "r"(b), "r"(what),
               "r"((uint32_t)add), "r"(kOperandKind)
               : "memory");
}
__device__ __forceinline__ bool one_lane() {
  uint32_t yes;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(yes));
  return yes;
}
// The product's shape and types: fp16 operands, fp32 sums, m = 128.
__device__ __forceinline__ uint32_t product_kind(uint32_t n, bool across) { return 1u << 4 | (uint32_t)across << 16 | (n >> 3) << 17 | (kRows >> 4) << 24; }

// 16, 32 or 64 columns of the 32 lanes of a warp, a lane a thread. tensor_loaded: the numbers are there; they go through it, so that nothing that uses them
// is moved ahead of it. The load of 16 waits itself.
__device__ __forceinline__ void tensor_load(uint32_t at, uint32_t (&x)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;"
               : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tensor_load(uint32_t at, float (&x)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
               : "r"(at));
}
__device__ __forceinline__ void tensor_load(uint32_t at, float (&x)[64]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]), "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]), "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]), "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31]), "=f"(x[32]), "=f"(x[33]), "=f"(x[34]), "=f"(x[35]), "=f"(x[36]), "=f"(x[37]), "=f"(x[38]), "=f"(x[39]), "=f"(x[40]), "=f"(x[41]), "=f"(x[42]), "=f"(x[43]), "=f"(x[44]), "=f"(x[45]), "=f"(x[46]), "=f"(x[47]), "=f"(x[48]), "=f"(x[49]), "=f"(x[50]), "=f"(x[51]), "=f"(x[52]), "=f"(x[53]), "=f"(x[54]), "=f"(x[55]), "=f"(x[56]), "=f"(x[57]), "=f"(x[58]), "=f"(x[59]), "=f"(x[60]), "=f"(x[61]), "=f"(x[62]), "=f"(x[63])
               : "r"(at));
}
template <int n>
__device__ __forceinline__ void tensor_loaded(float (&x)[n]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < n; ++i) asm volatile("" : "+f"(x[i]));
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&x)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(at)
               : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&x)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]), "r"(x[21]), "r"(x[22]), "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]), "r"(x[31]), "r"(at)
               : "memory");
}
__device__ __forceinline__ void tensor_store(uint32_t at, const uint32_t (&x)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(at)
               : "memory");
}
__device__ __forceinline__ void tensor_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// What generic stores have put into shared memory is there for the products that follow.
__device__ __forceinline__ void order_for_products() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <bool kBf16>
__device__ __forceinline__ uint32_t rounded(float low, float high) {
  uint32_t r;
  if constexpr (kBf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(high), "f"(low));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(high), "f"(low));
  return r;
}

// 16 columns of sums times a number.
__device__ __forceinline__ void scale_sums(uint32_t at, float down) {
  uint32_t x[16];
  tensor_load(at, x);
#pragma unroll
  for (uint32_t e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * down);
  tensor_store(at, x);
}
// The bits of the first n of 32.
__device__ __forceinline__ uint32_t bits_below(int32_t n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ float max_of(float a, float b, float c) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}

// ---- what weighs how much -----------------------------------------------------------------------------------------
// The blocks of a sequence weigh prefix + min(base + step * b, most), each once for every head of the cache; see above.
struct Weights {
  uint64_t base, most;
  uint32_t step, prefix, blocks, crossing;  // crossing: blocks ahead of it weigh less than `most`
};
__device__ __forceinline__ Weights weights_of(const AttendArgs& A, const Sequence& q) {
  Weights w;
  w.blocks = blocks_of(A, q, kTileRows);
  w.step = A.shared < kTileRows ? kTileRows / A.shared : 1;
  w.base = (uint64_t)q.first + w.step + kKeys / 2 + kBlockCost;
  w.prefix = A.window ? q.prefix : 0;
  w.most = A.window ? (uint64_t)A.window + w.step + kKeys + kBlockCost : 1ull << 62;
  w.crossing = w.most <= w.base ? 0 : (uint32_t)min((uint64_t)w.blocks, (w.most - w.base + w.step - 1) / w.step);
  return w;
}
__device__ __forceinline__ uint64_t weight_of(const Weights& w, uint32_t b) { return w.prefix + (b < w.crossing ? w.base + (uint64_t)w.step * b : w.most); }
__device__ __forceinline__ uint64_t weight_ahead(const Weights& w, uint32_t b) {  // of the blocks ahead of b
  const uint64_t n = min(b, w.crossing);
  return (uint64_t)w.prefix * b + n * w.base + w.step * (n * (n - 1) / 2) + (b > w.crossing ? (b - w.crossing) * w.most : 0);
}
// A block that some weight falls into.
struct Place {
  uint32_t block, head;
  uint64_t offset, weight;  // within the block; the block's
};
__device__ __forceinline__ Place place_of(const AttendArgs& A, const Weights& w, uint64_t rest) {
  uint32_t lo = 0, hi = w.blocks;  // the last block at or ahead of it
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (weight_ahead(w, mid) * A.heads <= rest) lo = mid;
    else hi = mid;
  }
  Place p;
  p.block = lo;
  p.weight = weight_of(w, lo);
  rest -= weight_ahead(w, lo) * A.heads;
  p.head = (uint32_t)(rest / p.weight);
  p.offset = rest - p.head * p.weight;
  return p;
}
// The tiles of keys that a block sees, numbered from 0: those of the prefix, then the others.
struct Tiles {
  uint32_t low, high;    // positions of its first and last query
  uint32_t ahead, from, count;
  __device__ __forceinline__ uint32_t key(uint32_t j) const { return (j < ahead ? j : from + j - ahead) * kKeys; }
};
__device__ __forceinline__ Tiles tiles_of(const AttendArgs& A, const Sequence& q, uint32_t block) {
  Tiles t;
  t.low = q.first + A.by_shared.div(block * kTileRows);
  t.high = q.first + min(A.by_shared.div(block * kTileRows + kTileRows - 1), q.rows - 1);
  t.ahead = q.ahead;
  t.from = max(q.ahead, first_seen(A, t.low) / kKeys);
  t.count = q.ahead + max(t.high / kKeys + 1, t.from) - t.from;
  return t;
}
__device__ __forceinline__ uint32_t tile_at(uint64_t offset, uint32_t tiles, uint64_t weight) {
  return offset == 0 ? 0 : offset >= weight ? tiles : (uint32_t)(offset * tiles / weight);
}
__device__ __forceinline__ uint64_t share_of(uint64_t all, uint32_t ctas) { return max((all + ctas - 1) / ctas, (uint64_t)(2 * kKeys)); }

// A CTA's way through its share: the blocks of which it has tiles, and which tiles.
struct Walk {
  Sequence q;
  Weights w;
  Place place;
  Tiles tiles;
  uint32_t s, block, head, j0, n;
  bool first;  // the block lies at the share's beginning, perhaps the CTA ahead has a part of it
  uint64_t at, from, to;
  __device__ __forceinline__ Walk(const AttendArgs& A, uint32_t sequence, uint64_t rest, uint64_t from_, uint64_t to_) : s(sequence), at(from_), from(from_), to(to_) {
    q = sequence_of<kKeys>(A, s, false);
    w = weights_of(A, q);
    place = place_of(A, w, rest);
  }
  __device__ __forceinline__ bool next(const AttendArgs& A) {
    while (at < to) {
      if (place.offset == place.weight) step(A);
      const uint64_t upto = min(to - at + place.offset, place.weight);
      block = place.block, head = place.head;
      tiles = tiles_of(A, q, block);
      j0 = tile_at(place.offset, tiles.count, place.weight);
      n = tile_at(upto, tiles.count, place.weight) - j0;
      first = at == from;
      at += upto - place.offset;
      place.offset = upto;
      if (n > 0) return true;
    }
    return false;
  }
  __device__ __forceinline__ void step(const AttendArgs& A) {
    place.offset = 0;
    if (++place.head == A.heads) {
      place.head = 0;
      if (++place.block == w.blocks) {
        do {
          q = sequence_of<kKeys>(A, ++s, false);
        } while (q.rows == 0);
        w = weights_of(A, q);
        place.block = 0;
      }
      place.weight = weight_of(w, place.block);
    }
  }
};

// ---- the kernel ---------------------------------------------------------------------------------------------------
template <int kBits, uint32_t DP>
struct Layout {
  static constexpr uint32_t kRuns = DP / 64;                         // of 64 values
  static constexpr uint32_t kQueries = kRuns * kRows * 128;          // bytes of a tile of queries
  static constexpr uint32_t kOperand = kRuns * kHalf * 128;          // of half a tile of keys or values
  static constexpr uint32_t kRow = DP * kBits / 8, kCodes = kHalf * kRow;  // of a key's codes, of half a tile's, on their way
  static constexpr uint32_t kOperandsAt = 2 * kQueries, kCodesAt = kOperandsAt + 2 * kStages * kOperand;
  static constexpr uint32_t kWhole = kCodesAt + 2 * kAhead * kCodes + 1024;
  static constexpr uint32_t kScoresAt = 0, kSumsAt = 2 * kKeys;      // columns of tensor memory; the second tile's kKeys and DP columns behind
};

constexpr uint32_t kNone = ~0u;  // a key without a place
struct Shared {
  unsigned long long full_k[kStages], empty_k[kStages], full_v[kStages], empty_v[kStages], found_full[2][kFound], found_empty[2][kFound], queries[2], scores[2][2], weights[2][2], sums[2][2];  // barriers
  unsigned long long scan[kThreads / 32], found_base;
  uint32_t found, tensor, dead;
  uint2 scales[2][kFound][kKeys];          // for the readers of keys and of values: a key's scales in fp16, two in a word
  uint32_t places[2][kFound][kKeys];       // slot * heads + head, which is below 2^32 in this kernel; kNone
  // The powers of two that 16 keys each are in units of, and that a tile's values are in units of; below 0 where each key, or each key's values, is in units of a power
  // of its own, whose exponents (of fp32) then stand beside.
  float units[kMemo][kKeys / 16], value_units[kMemo];
  alignas(16) uint8_t exponents[2][kMemo][kKeys];
  float query_units[kTileRows];
  uint32_t broken[kMemo][kTileRows / 8];   // for the queries of a block, four bits each: groups of which they see a value that is no number
};

static_assert(sizeof(Shared) + Layout<8, 128>::kWhole <= 232448, "a CTA's shared memory");

// kCap, kBias: scores are capped, lowered by distance.
template <int kBits, uint32_t DP, bool kBf16, bool kCap, bool kBias>
struct Kernel {
  using L = Layout<kBits, DP>;
  using T = typename TypeOf<kBf16 ? LC_TYPE_BF16 : LC_TYPE_F16>::T;
  static constexpr float kLift = 7.0f;
  static constexpr uint32_t kParts = L::kRow / 16, kUnits = kParts / 2;  // pieces of 16 bytes of a row's codes, at most; of half a tile that a reader takes

  // A tile of a block's queries as an operand, by the warpgroup that takes its scores. A negative scale goes to their signs. All of a thread's loads are on their
  // way at once.
  static __device__ __forceinline__ void load_queries(const AttendArgs& A, const Sequence& q, uint32_t first, uint32_t head, uint32_t thread, uint8_t* to, float* units) {
    const uint32_t flip = A.scale < 0.0f ? 0x80008000u : 0u, c = thread % (DP / 8);
    constexpr uint32_t kRowsAtOnce = kRows / (DP / 8);  // rows that the threads take together
    const unsigned short* const from = static_cast<const unsigned short*>(A.q) + (uint64_t)(head * A.shared) * A.q_head + c * 8;
    auto row_at = [&](uint32_t i) { return i * kRowsAtOnce + thread / (DP / 8); };
    auto put = [&](uint32_t row, uint4 x) {
      uint32_t w[4] = {x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip};
      if constexpr (kBf16) {
        // the row's largest exponent, over the lanes that hold it
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) most = __vmaxu2(most, w[e] & 0x7F807F80u);
        most = max(most & 0xFFFFu, most >> 16) >> 7;
#pragma unroll
        for (uint32_t d = DP / 16; d; d >>= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
        most = most == 255 ? 127 : min(max(most, 1u), 253u);  // of Inf and NaN: as they are
        const float down = __uint_as_float((254 - most) << 23);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = rounded<false>(__uint_as_float(w[e] << 16) * down, __uint_as_float(w[e] & 0xFFFF0000u) * down);
        if (c == 0) units[row] = __uint_as_float(most << 23);
      }
      *reinterpret_cast<uint4*>(to + (c / 8) * (kRows * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    };
    if (A.dim % 8 == 0 && ((reinterpret_cast<uintptr_t>(A.q) / 2 | A.q_row | A.q_head) & 7) == 0) {
      uint4 x[DP / 8];
#pragma unroll
      for (uint32_t i = 0; i < DP / 8; ++i) {
        const uint32_t r = first + row_at(i), token = A.by_shared.div(r);
        x[i] = make_uint4(0, 0, 0, 0);
        if (token < q.rows && c * 8 < A.dim) x[i] = __ldg(reinterpret_cast<const uint4*>(from + (uint64_t)(q.row + token) * A.q_row + (uint64_t)(r - token * A.shared) * A.q_head));
      }
#pragma unroll
      for (uint32_t i = 0; i < DP / 8; ++i) put(row_at(i), x[i]);
    } else {
#pragma unroll 1
      for (uint32_t i = 0; i < DP / 8; ++i) {
        const uint32_t r = first + row_at(i), token = A.by_shared.div(r);
        const unsigned short* p = from + (uint64_t)(q.row + token) * A.q_row + (uint64_t)(r - token * A.shared) * A.q_head;
        unsigned short x[8];
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) {
          x[e] = 0;
          if (token < q.rows && c * 8 + e < A.dim) x[e] = __ldg(p + e);
        }
        put(row_at(i), make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16));
      }
    }
  }

  // A reader takes one piece of 16 bytes of kUnits keys' codes of half a tile, kStep apart, which come by asynchronous copies, kAhead halves ahead, to places of
  // its own. Lanes are dealt to pieces and keys so that eight lanes in a row store to different banks: 8 bits, four pieces of two neighbouring keys
  // (their runs of eight values are every other one, which the swizzle puts into the even and the odd places), 4 bits, two pieces of four.
  static constexpr uint32_t kStep = 32 / kParts, kRuns = 16 / kBits;  // kRuns: of eight values in a piece
  static_assert(kStep * kUnits == 16, "a warp's keys of a half");
  struct Reader {
    uint32_t key, group;     // first key of a half; group of the piece
    uint32_t left;           // words of the row from the piece on
    uint32_t at[kRuns];      // where its runs go for the first key
    uint32_t copies;         // where its copies go
    const uint8_t* codes;
  };
  static __device__ __forceinline__ Reader reader_of(const AttendArgs& A, uint32_t set, uint32_t warp, uint32_t lane, uint32_t copies) {
    Reader r;
    uint32_t part, row;
    if (kBits == 8) part = kParts == 8 ? (lane & 3) | (lane >> 1 & 4) : lane & 3, row = kParts == 8 ? (lane >> 2 & 1) | (lane >> 3 & 2) : lane >> 2;
    else part = kParts == 4 ? (lane & 1) | (lane >> 2 & 2) : lane & 1, row = kParts == 4 ? (lane >> 1 & 3) | (lane >> 2 & 4) : lane >> 1;
    r.key = warp * 16 + row;
    r.left = part * 16 < A.row_bytes ? (A.row_bytes - part * 16) / 4 : 0;
    r.group = r.left ? part / (A.per_group * (kBits == 8 ? 2 : 1)) : 0;
    r.copies = copies + (warp * 32 + lane) * 16;
    r.codes = A.codes + (set ? A.plane_codes : 0) + (r.left ? part * 16 : 0);
#pragma unroll
    for (uint32_t k = 0; k < kRuns; ++k) {
      const uint32_t n = part * kRuns + k;
      r.at[k] = (n / 8) * (kHalf * 128) + r.key * 128 + (((n & 7) ^ (r.key & 7)) << 4);
    }
    return r;
  }
  // Starts the copies of a half into slot `slot`; places: of its keys. Nothing is read for keys without a place.
  static __device__ __forceinline__ void copy_half(const AttendArgs& A, const uint32_t* places, uint32_t slot, const Reader& r) {
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
      const uint32_t place = places[r.key + i * kStep], to = r.copies + slot * L::kCodes + i * (kReaders * 16);
      const bool there = place != kNone && r.left > 0;
      const uint8_t* p = r.codes + (uint64_t)(there ? place : 0) * A.row_bytes;
      if ((A.row_bytes & 15) == 0) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(p), "r"(there ? 16 : 0) : "memory");
      } else {
#pragma unroll
        for (uint32_t w = 0; w < 4; ++w)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * w), "l"(p + (w < r.left ? 4 * w : 0)), "r"(there && w < r.left ? 4 : 0) : "memory");
      }
    }
  }
  static __device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // Four pairs of fp16 numbers from eight codes; scale: twice. In the lowest bits of 1024 a whole number is itself, or 16 times as large, and one exact operation
  // for two of them brings them to where they belong.
  static __device__ __forceinline__ uint4 numbers(uint32_t a, uint32_t b, uint32_t scale) {
    uint32_t r[4];
    if constexpr (kBits == 4) {
      const uint32_t x[4] = {(a & 0x000F000Fu) | 0x64006400u, (a & 0x00F000F0u) | 0x64006400u, (a >> 8 & 0x000F000Fu) | 0x64006400u, (a >> 8 & 0x00F000F0u) | 0x64006400u};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e % 2 == 0) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[e]) : "r"(x[e]), "r"(0xE408E408u));              // - 1032
        else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[e]) : "r"(x[e]), "r"(0x2C002C00u), "r"(0xD480D480u));  // / 16 - 72
      }
    } else {
      const uint32_t x[4] = {__byte_perm(a, 0x64646464u, 0x4140), __byte_perm(a, 0x64646464u, 0x4342), __byte_perm(b, 0x64646464u, 0x4140), __byte_perm(b, 0x64646464u, 0x4342)};
#pragma unroll
      for (int e = 0; e < 4; ++e) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r[e]) : "r"(x[e]), "r"(0xE480E480u));  // - 1152
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r[e]) : "r"(r[e]), "r"(scale));
    return make_uint4(r[0], r[1], r[2], r[3]);
  }
  // A half's pieces as operands. scales: of its keys.
  static __device__ __forceinline__ void store_numbers(const uint2* scales, uint32_t slot, const Reader& r, uint32_t operand) {
    if (r.left == 0) return;
    const uint32_t* pairs = reinterpret_cast<const uint32_t*>(scales + r.key) + r.group / 2;
#pragma unroll
    for (uint32_t i = 0; i < kUnits; ++i) {
      const uint32_t scale = __byte_perm(pairs[i * kStep * 2], 0, r.group & 1 ? 0x3232 : 0x1010);
      uint32_t w[4];
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(r.copies + slot * L::kCodes + i * (kReaders * 16)) : "memory");
#pragma unroll
      for (uint32_t k = 0; k < kRuns; ++k) {
        const uint4 y = kBits == 8 ? numbers(w[2 * k], w[2 * k + 1], scale) : numbers(w[k], 0, scale);
        // kStep 4: every second key's places are the others of the swizzle's upper bit (its row's number differs by 4)
        const uint32_t at = operand + (kStep == 4 && (i & 1) ? r.at[k] ^ 64u : r.at[k]) + i * (kStep * 128);
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w) : "memory");
      }
    }
  }
  // Where a key lies, in two steps: the page's number as the table has it, and what follows from it.
  static __device__ __forceinline__ int32_t page_of(const AttendArgs& A, const Sequence& q, uint32_t s, uint32_t key) {
    return key < q.length ? __ldg(A.table + s * A.table_stride + A.by_page.div(key)) : 0;
  }
  static __device__ __forceinline__ uint32_t place_of_key(const AttendArgs& A, const Sequence& q, uint32_t head, uint32_t key, int32_t number) {
    if (key >= q.length) return kNone;
    const int64_t slot = (int64_t)number * A.by_page.d + (key - A.by_page.div(key) * A.by_page.d);
    if (number < 0 || slot >= (int64_t)A.slots) {
      if (A.status) set_status(A.status, LC_ERR_INDEX);
      return kNone;
    }
    return (uint32_t)slot * A.heads + head;
  }

  // Notes which queries of the walk's block see values of a tile that are no numbers, and in which groups. broken: of a lane's keys first + lane + 32 k, four bits
  // each.
  static __device__ __forceinline__ void note_broken(const AttendArgs& A, const Walk& walk, uint32_t broken, uint32_t first, uint32_t lane, uint32_t* noted) {
#pragma unroll 1
    for (uint32_t k = 0; k < kKeys / 32; ++k) {
      const uint32_t groups = broken >> (4 * k) & 15;
#pragma unroll 1
      for (uint32_t those = __ballot_sync(0xFFFFFFFFu, groups); those; those &= those - 1) {
        const uint32_t owner = __ffs(those) - 1, its = __shfl_sync(0xFFFFFFFFu, groups, owner), key = first + 32 * k + owner;
#pragma unroll 1
        for (uint32_t row = lane; row < kTileRows; row += 32) {
          const uint32_t position = walk.q.first + min(A.by_shared.div(walk.block * kTileRows + row), walk.q.rows - 1);
          if ((key <= position && (A.window == 0 || position - key < A.window)) || key < walk.q.prefix) atomicOr(noted + row / 8, its << (row % 8 * 4));
        }
        __syncwarp();
      }
    }
  }

  static __device__ __forceinline__ void run(const AttendArgs& A) {
    extern __shared__ uint8_t raw[];
    __shared__ Shared S;
    uint8_t* const smem = raw + (1024 - (shared_address(raw) & 1023)) % 1024;
    uint8_t* const queries = smem;
    uint8_t* const keys = smem + L::kOperandsAt;
    uint8_t* const values = keys + kStages * L::kOperand;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    begin_next();

    if (threadIdx.x == 0) {
      S.dead = 0;
      for (uint32_t i = 0; i < kStages; ++i) {
        barrier_init(shared_address(&S.full_k[i]), kReaders);
        barrier_init(shared_address(&S.empty_k[i]), 2);
        barrier_init(shared_address(&S.full_v[i]), kReaders);
        barrier_init(shared_address(&S.empty_v[i]), 2);
      }
      for (uint32_t i = 0; i < 2 * kFound; ++i) {
        barrier_init(shared_address(&S.found_full[i / kFound][i % kFound]), 1);
        barrier_init(shared_address(&S.found_empty[i / kFound][i % kFound]), kReadWarps);
      }
      for (uint32_t t = 0; t < 2; ++t) {
        barrier_init(shared_address(&S.queries[t]), kRows);
        for (uint32_t h = 0; h < 2; ++h) {
          barrier_init(shared_address(&S.scores[t][h]), 1);
          barrier_init(shared_address(&S.weights[t][h]), kRows);
          barrier_init(shared_address(&S.sums[t][h]), 1);
        }
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }

    if (threadIdx.x < kMemo * (kTileRows / 8)) S.broken[threadIdx.x / (kTileRows / 8)][threadIdx.x % (kTileRows / 8)] = 0;

    // this CTA's share of the weight
    unsigned long long all = 0;
    for (uint32_t s = threadIdx.x; s < A.sequences; s += kThreads) {
      const Sequence q = sequence_of<kKeys>(A, s, blockIdx.x == 0);
      if (q.rows) {
        const Weights w = weights_of(A, q);
        all += weight_ahead(w, w.blocks) * A.heads;
      }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, d);
    if (lane == 0) S.scan[warp] = all;
    __syncthreads();
    all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32; ++w) all += S.scan[w];
    const unsigned long long share = share_of(all, gridDim.x), from = blockIdx.x * share, to = min(from + share, all);
    if (blockIdx.x == 0 || from < all) {
      unsigned long long base = 0;
      for (uint32_t s0 = 0; s0 < A.sequences; s0 += kThreads) {
        const uint32_t s = s0 + threadIdx.x;
        unsigned long long mine = 0;
        if (s < A.sequences) {
          const Sequence q = sequence_of<kKeys>(A, s, false);
          if (q.rows) {
            const Weights w = weights_of(A, q);
            mine = weight_ahead(w, w.blocks) * A.heads;
          }
        }
        unsigned long long upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const unsigned long long x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
          if (lane >= (uint32_t)d) upto += x;
        }
        __syncthreads();
        if (lane == 31) S.scan[warp] = upto;
        __syncthreads();
        unsigned long long ahead = base + upto - mine;
#pragma unroll
        for (uint32_t w = 0; w < kThreads / 32; ++w) {
          if (w < warp) ahead += S.scan[w];
          base += S.scan[w];
        }
        if (blockIdx.x == 0 && s < A.sequences) A.flat[s] = ahead;  // for the launch that joins
        if (from >= ahead && from < ahead + mine) {
          S.found = s;
          S.found_base = ahead;
        }
        if (blockIdx.x != 0 && base > from) break;
      }
      if (blockIdx.x == 0 && threadIdx.x == 0) A.flat[A.sequences] = all;
    }
    __syncthreads();
    if (from >= to) return;
    if (warp == kSoftmaxWarps + 2 * kReadWarps) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&S.tensor)), "n"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
      order_before();
    }

    __syncthreads();
    order_after();
    const uint32_t tensor = S.tensor;
    volatile uint32_t* dead = &S.dead;
    Walk walk(A, S.found, from - S.found_base, from, to);
    uint32_t done = 0;  // tiles of keys so far: what the barriers' phases go by

    if (warp < kSoftmaxWarps) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
      bool good = true;
      for (uint32_t blocks = 0; good && walk.next(A); ++blocks) {
        const Sequence& q = walk.q;
        const Tiles& tiles = walk.tiles;
        const uint32_t block = walk.block, head = walk.head, j0 = walk.j0, n = walk.n;
        // ---- scores to probabilities: a query a thread
        const uint32_t t = warp / 4, row = threadIdx.x % kRows, r = block * kTileRows + t * kRows + row, token = A.by_shared.div(r), in_group = r - token * A.shared;
        const uint32_t lanes = tensor + ((warp & 3) * 32 << 16), scores = lanes + L::kScoresAt + t * kKeys, sums = lanes + L::kSumsAt + t * DP;
        const uint32_t position = q.first + min(token, q.rows - 1);
        const float slope = kBias ? A.slopes[head * A.shared + in_group] * kLog2e : 0.0f;
        const Cap cap(kCap ? A.cap : 1.0f);
        // positions of this warp's first and last query
        const uint32_t low = __shfl_sync(0xFFFFFFFFu, position, 0), high = __shfl_sync(0xFFFFFFFFu, position, 31);
        float m = -INFINITY;
        Two l = two(0.0f, 0.0f);
        load_queries(A, q, block * kTileRows + t * kRows, head, row, queries + t * L::kQueries, S.query_units + t * kRows);
        float own = fabsf(A.scale) * kLog2e;  // what the row's scores are multiplied by
        if constexpr (kBf16) {
          asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + t), "n"(kRows) : "memory");
          own *= S.query_units[t * kRows + row];
        }
        float value_unit = 1.0f;  // of the sums; by_exponent: its exponent as it stands in fp32, then no whole number
        bool by_exponent = false;
        order_for_products();
        order_before();  // the sums of the block before are read
        barrier_arrive(shared_address(&S.queries[t]));
        good = false;  // all tiles are through
        uint32_t i = 0;
        bool apart = false;
        for (; i < 2 * n; ++i) {
          const uint32_t number = done + i / 2, half = i & 1, key = tiles.key(j0 + i / 2) + half * kHalf, at = scores + half * kHalf;
          if (!warp_wait(shared_address(&S.scores[t][half]), number & 1, dead)) break;
          // What is looked up of a tile's values (their unit) comes another way than its scores. Behind a block's first tile it is there: scores of a half wait for the
          // values of the second half ahead of it, which are stored once the tile after theirs has been looked up. For the first tile its values are waited for; they
          // are not replaced before this warp's probabilities have met them.
          if (i == 0 && !warp_wait(shared_address(&S.full_v[2 * done % kStages]), 2 * done / kStages & 1, dead)) break;
          order_after();
          float y[kHalf];
          tensor_load(at, y);
          const float tile_unit = S.value_units[number % kMemo], first_unit = S.units[number % kMemo][half * 4];
          if (fminf(tile_unit, first_unit) < 0.0f) {
            tensor_loaded(y);
            apart = true;
            break;
          }
          float factor[kHalf / 16];  // of 16 keys each; not 0, or a key that is not seen, -Inf, times that would be no number
#pragma unroll
          for (uint32_t c = 0; c < kHalf / 16; ++c) factor[c] = fmaxf(own * S.units[number % kMemo][half * 4 + c], 1e-37f);
          const bool full = key + kHalf - 1 <= low && (A.window == 0 || high - key < A.window);
          tensor_loaded(y);
          if constexpr (kCap || kBias) {
#pragma unroll
            for (uint32_t e = 0; e < kHalf; ++e) y[e] *= factor[e / 16];
            if constexpr (kCap) {
              if (A.cap <= kPlainCap) {
#pragma unroll
                for (uint32_t e = 0; e < kHalf; ++e) y[e] = cap.large(y[e]);
              } else {
                float most = 0.0f;
#pragma unroll
                for (uint32_t e = 0; e < kHalf; ++e) most = fmaxf(most, fabsf(y[e]));
                if (__all_sync(0xFFFFFFFFu, most * cap.in < Cap::kSmall)) {  // the same numbers as below
#pragma unroll
                  for (uint32_t e = 0; e < kHalf; e += 2) split_two(cap.small(two(y[e], y[e + 1])), y[e], y[e + 1]);
                } else {
#pragma unroll
                  for (uint32_t e = 0; e < kHalf; ++e) y[e] = cap(y[e]);
                }
              }
            }
            if constexpr (kBias) {
              const float away = (float)(int32_t)(position - key);
#pragma unroll
              for (uint32_t e = 0; e < kHalf; ++e) y[e] = fmaf(-slope, fabsf(away - (float)e), y[e]);
            }
          }
          if (!full) {
            // of these keys a query sees those from `begin` on and ahead of `end`, and those ahead of `prefix`
            const int32_t end = (int32_t)(position - key) + 1, begin = A.window ? end - (int32_t)A.window : 0, prefix = (int32_t)(q.prefix - key);
#pragma unroll
            for (uint32_t c = 0; c < kHalf; c += 32) {
              const uint32_t seen = (bits_below(end - (int32_t)c) & ~bits_below(begin - (int32_t)c)) | bits_below(prefix - (int32_t)c);
#pragma unroll
              for (uint32_t e = 0; e < 32; ++e) y[c + e] = seen >> e & 1 ? y[c + e] : -INFINITY;
            }
          }
          float top = -INFINITY;
#pragma unroll
          for (uint32_t c = 0; c < kHalf; c += 16) {
            float x = fmaxf(y[c], y[c + 1]);
#pragma unroll
            for (uint32_t e = 2; e < 16; e += 2) x = max_of(x, y[c + e], y[c + e + 1]);
            top = fmaxf(top, kCap || kBias ? x : __fmul_rn(x, factor[c / 16]));  // grows with the product
          }
          const bool rises = top > m + kSlack;
          if (__any_sync(0xFFFFFFFFu, rises) || tile_unit != value_unit) {
            const float now = rises ? top : m, down = rises ? exp2_fast(m - now) : 1.0f, sums_down = down * (value_unit / tile_unit);
            value_unit = tile_unit;
            if (i > 0) {
              // the product before (the one before that has ended, or these scores would not be there)
              if (!warp_wait(shared_address(&S.sums[t][1 - half]), (done + (i - 1) / 2) & 1, dead)) break;
              order_after();
#pragma unroll 1
              for (uint32_t d = 0; d < DP; d += 16) scale_sums(sums + d, sums_down);
            }
            m = now;
            l = mul_two(l, two(down, down));
          }
          const float base = (m == -INFINITY ? 0.0f : m) - kLift;
          if (kCap || kBias || fabsf(m) > 0x1p20f) {
            // Of large scores the product is rounded like the maximum was, which then weighs 1: fused, what rounding took from that is 2^-24 of it and no small
            // exponent.
#pragma unroll
            for (uint32_t e = 0; e < kHalf; ++e) y[e] = (kCap || kBias ? y[e] : __fmul_rn(y[e], factor[e / 16])) - base;
          } else {
#pragma unroll
            for (uint32_t e = 0; e < kHalf; e += 2) split_two(fma_two(two(y[e], y[e + 1]), two(factor[e / 16], factor[e / 16]), two(-base, -base)), y[e], y[e + 1]);
          }
          uint32_t p[kHalf / 2];
#pragma unroll
          for (uint32_t e = 0; e < kHalf; e += 2) {
            y[e] = exp2_fast(y[e]), y[e + 1] = exp2_fast(y[e + 1]);
            l = add_two(l, two(y[e], y[e + 1]));
            p[e / 2] = rounded<false>(y[e], y[e + 1]);
          }
          __syncwarp();
          tensor_store(at, p);
          tensor_stored();
          order_before();
          barrier_arrive(shared_address(&S.weights[t][half]));
          good = i + 1 == 2 * n;
        }
        // From the first tile on whose keys, or their values, have units of their own (see the warps that look them up): the same with fewer registers, 16 scores at a time, each
        // read as often as it is needed. A value's power of two goes to its probability: with m and e_k the base and the exponents, sums are of 2^(y_k - m + e_k - d), and in units
        // of 2^d, where d grows with the largest that the query has seen. (A loop of its own: as a way through the one above it took that 6 % of its time.)
        if (apart) {
          for (; i < 2 * n; ++i) {
            const uint32_t number = done + i / 2, half = i & 1, key = tiles.key(j0 + i / 2) + half * kHalf, at = scores + half * kHalf, memo = number % kMemo;
            if (!warp_wait(shared_address(&S.scores[t][half]), number & 1, dead)) break;
            order_after();
            const float tile_unit = S.value_units[memo];
            const bool keys_apart = S.units[memo][0] < 0.0f, values_apart = tile_unit < 0.0f;
            auto scores_of = [&](uint32_t c, float (&y)[16]) {  // 16 of them from c on
              uint32_t x[16];
              tensor_load(at + c, x);
              const int32_t end = (int32_t)(position - key - c) + 1, begin = A.window ? end - (int32_t)A.window : 0, prefix = (int32_t)(q.prefix - key - c);
              const uint32_t seen = (bits_below(end) & ~bits_below(begin)) | bits_below(prefix);
              const float away = (float)(int32_t)(position - key - c);
#pragma unroll
              for (uint32_t e = 0; e < 16; ++e) {
                const float unit = keys_apart ? __uint_as_float((uint32_t)S.exponents[0][memo][half * kHalf + c + e] << 23) : S.units[memo][half * 4 + c / 16];
                y[e] = __fmul_rn(__uint_as_float(x[e]), own * unit);
                if constexpr (kCap) y[e] = A.cap <= kPlainCap ? cap.large(y[e]) : cap(y[e]);
                if constexpr (kBias) y[e] = fmaf(-slope, fabsf(away - (float)e), y[e]);
                if (!(seen >> e & 1)) y[e] = -INFINITY;
              }
            };
            auto exponent_of = [&](uint32_t k) { return (float)(values_apart ? (uint32_t)S.exponents[1][memo][half * kHalf + k] : __float_as_uint(tile_unit) >> 23); };
            float y[16], now = m;
#pragma unroll 1
            for (uint32_t c = 0; c < kHalf; c += 16) {
              scores_of(c, y);
#pragma unroll
              for (uint32_t e = 0; e < 16; ++e) now = fmaxf(now, y[e]);
            }
            const float base = now == -INFINITY ? 0.0f : now, down = m == now ? 1.0f : exp2_fast(m - now);
            const float before = m == -INFINITY ? -1e4f : (by_exponent ? value_unit : (float)(__float_as_uint(value_unit) >> 23)) + (m - now);
            float d = values_apart ? before : exponent_of(0);
            if (values_apart) {
#pragma unroll 1
              for (uint32_t c = 0; c < kHalf; c += 16) {
                scores_of(c, y);
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e) d = fmaxf(d, y[e] - base + exponent_of(c + e));
              }
            }
            const float sums_down = exp2_fast(before - d);
            if (i > 0 && __any_sync(0xFFFFFFFFu, sums_down != 1.0f)) {
              if (!warp_wait(shared_address(&S.sums[t][1 - half]), (done + (i - 1) / 2) & 1, dead)) break;
              order_after();
#pragma unroll 1
              for (uint32_t c = 0; c < DP; c += 16) scale_sums(sums + c, sums_down);
            }
            m = now;
            l = mul_two(l, two(down, down));
            by_exponent = values_apart;
            value_unit = values_apart ? d : tile_unit;
#pragma unroll 1
            for (uint32_t c = 0; c < kHalf; c += 16) {
              scores_of(c, y);
              uint32_t p[8];
#pragma unroll
              for (uint32_t e = 0; e < 16; e += 2) {
                y[e] -= base, y[e + 1] -= base;
                l = add_two(l, two(exp2_fast(y[e] + kLift), exp2_fast(y[e + 1] + kLift)));
                p[e / 2] = rounded<false>(exp2_fast(y[e] + (exponent_of(c + e) - d + kLift)), exp2_fast(y[e + 1] + (exponent_of(c + e + 1) - d + kLift)));
              }
              __syncwarp();
              tensor_store(at + c / 2, p);  // over scores that have been read
            }
            tensor_stored();
            order_before();
            barrier_arrive(shared_address(&S.weights[t][half]));
            good = i + 1 == 2 * n;
          }
        }
        for (uint32_t h = 0; h < 2; ++h) good = good && warp_wait(shared_address(&S.sums[t][h]), (done + n - 1) & 1, dead);
        if (good) {
          order_after();
          // noted by the warp that looks up values, ahead of those that the sums have waited for
          uint32_t* const noted = &S.broken[blocks % kMemo][(t * kRows + row) / 8];
          const uint32_t broken = *noted >> (row % 8 * 4) & 15;
          __syncwarp();
          if (row % 8 == 0) *noted = 0;
          const bool whole = j0 == 0 && n == tiles.count, there = token < q.rows;
          float* part = A.parts + (2ull * blockIdx.x + (walk.first ? 0 : 1)) * (kTilePartBytes / 4);
          T* out = static_cast<T*>(A.out) + (uint64_t)(q.row + min(token, q.rows - 1)) * A.out_row + (uint64_t)(head * A.shared + in_group) * A.out_head;
          const bool aligned = ((reinterpret_cast<uintptr_t>(A.out) / 2 | A.out_row | A.out_head) & 7) == 0;
          float sum, other;
          split_two(l, sum, other);
          sum += other;
          if (by_exponent) value_unit = exp2_fast(value_unit - 127.0f);
          // A part is a mean too, that of the keys that it has: its sums may be beyond fp32. (Its queries may see none of them. Of a whole block's a sum is 0 only if all scores are -Inf.)
          const float over = !whole && sum == 0.0f ? 0.0f : value_unit / sum;
          const uint32_t shift = 5 + (A.per_group > 1) + (A.per_group > 2);  // values of a group
#pragma unroll 1
          for (uint32_t c = 0; c < A.dim; c += 32) {
            float x[32];
            tensor_load(sums + c, x);
            tensor_loaded(x);
#pragma unroll
            for (uint32_t e = 0; e < 32; ++e) x[e] *= over;
            if (broken >> (c >> shift) & 1) {
#pragma unroll
              for (uint32_t e = 0; e < 32; ++e) x[e] = __uint_as_float(0x7FFFFFFFu);
            }
            if (there && whole) {
#pragma unroll
              for (uint32_t e = 0; e < 32; e += 8) {
                const uint32_t w[4] = {rounded<kBf16>(x[e], x[e + 1]), rounded<kBf16>(x[e + 2], x[e + 3]), rounded<kBf16>(x[e + 4], x[e + 5]), rounded<kBf16>(x[e + 6], x[e + 7])};
                if (aligned && c + e + 8 <= A.dim) {
                  *reinterpret_cast<uint4*>(out + c + e) = make_uint4(w[0], w[1], w[2], w[3]);
                } else {
#pragma unroll
                  for (uint32_t k = 0; k < 8; ++k)
                    if (c + e + k < A.dim) reinterpret_cast<unsigned short*>(out)[c + e + k] = (unsigned short)(w[k / 2] >> (16 * (k & 1)));
                }
              }
            } else if (there) {
#pragma unroll
              for (uint32_t e = 0; e < 32; e += 4)
                *reinterpret_cast<float4*>(part + ((c + e) / 4 * kTileRows + t * kRows + row) * 4) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
            }
            __syncwarp();
          }
          if (!whole) {
            part[kTileRows * kTileDim + t * kRows + row] = m;
            part[kTileRows * (kTileDim + 1) + t * kRows + row] = sum;
          }
        }
        done += n;
        good = together(1 + t, good);
      }
    } else if (warp < kSoftmaxWarps + 2 * kReadWarps) {
      // ---- codes to operands
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsReader));
      const uint32_t set = (warp - kSoftmaxWarps) / kReadWarps, mine = (warp - kSoftmaxWarps) % kReadWarps;  // set: 0 keys, 1 values
      const uint32_t operands = shared_address(set ? values : keys);
      unsigned long long* const full = set ? S.full_v : S.full_k;
      unsigned long long* const empty = set ? S.empty_v : S.empty_k;
      const Reader R = reader_of(A, set, mine, lane, shared_address(smem) + L::kCodesAt + set * kAhead * L::kCodes);
      uint32_t stage = 0, turn = 0;  // of the operands
      bool good = true;
      while (good && walk.next(A)) {
        const uint32_t n = walk.n;
        auto found = [&](uint32_t tile) {  // of the block: waits until its keys have been looked up
          const uint32_t x = done + tile;
          return warp_wait(shared_address(&S.found_full[set][x % kFound]), x / kFound & 1, dead);
        };
        auto places = [&](uint32_t half) { return S.places[set][(done + half / 2) % kFound] + (half & 1) * kHalf; };
        uint32_t slot = 0;
        good = found(0);
        if (!good) break;
        copy_half(A, places(0), 0, R);
        copies_end();
        copy_half(A, places(1), 1, R);
        copies_end();
        if (n > 1) {
          good = found(1);
          if (!good) break;
          copy_half(A, places(2), 2, R);
        }
        copies_end();
        for (uint32_t i = 0; i < 2 * n; ++i) {
          if (turn > 0) good = warp_wait(shared_address(&empty[stage]), (turn - 1) & 1, dead);
          if (!good) break;
          asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
          store_numbers(S.scales[set][(done + i / 2) % kFound] + (i & 1) * kHalf, slot, R, operands + stage * L::kOperand);
          order_for_products();
          barrier_arrive(shared_address(&full[stage]));
          if (i + kAhead < 2 * n) {
            if (i & 1) good = found((i + kAhead) / 2);
            if (!good) break;
            copy_half(A, places(i + kAhead), slot, R);
          }
          copies_end();
          if (i & 1) {
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&S.found_empty[set][(done + i / 2) % kFound]));
          }
          slot = slot + 1 == kAhead ? 0 : slot + 1;
          if (++stage == kStages) stage = 0, ++turn;
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        done += n;
      }
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
      if (warp < kSoftmaxWarps + 2 * kReadWarps + 2) {
        // ---- the products, a warp for each tile of queries: the warp as a whole goes through the keys, with numbers that the compiler knows to be the same for all
        // lanes; one lane issues
        const uint32_t all_lanes = 0xFFFFFFFFu, at_tensor = __shfl_sync(all_lanes, tensor, 0), t = __shfl_sync(all_lanes, warp, 0) - (kSoftmaxWarps + 2 * kReadWarps);
        const uint32_t steps = (A.dim + 15) / 16, scores_kind = product_kind(kHalf, false), sums_kind = product_kind(steps * 16, true);
        const uint32_t query_at = operand_at(shared_address(queries) + t * L::kQueries, 16), key_at = operand_at(shared_address(keys), 16), value_at = operand_at(shared_address(values), kHalf * 128);
        const uint32_t scores_at = at_tensor + L::kScoresAt + t * kKeys, sums_at = at_tensor + L::kSumsAt + t * DP;
        auto multiply_keys = [&](uint32_t half, uint32_t stage) {
          const uint32_t b = key_at + stage * (L::kOperand >> 4), d = scores_at + half * kHalf;
#pragma unroll
          for (uint32_t x = 0; x < DP / 16; ++x)
            if (x < steps) product(d, query_at + ((x / 4) * (kRows * 128) + (x % 4) * 32 >> 4), b + ((x / 4) * (kHalf * 128) + (x % 4) * 32 >> 4), scores_kind, x > 0);
          commit_to(shared_address(&S.scores[t][half]));
          commit_to(shared_address(&S.empty_k[stage]));
        };
        bool good = true;
        uint32_t k_stage = 0, k_turn = 0, v_stage = 0, v_turn = 0;
        auto wait_keys = [&] { return warp_wait(shared_address(&S.full_k[k_stage]), k_turn & 1, dead); };
        auto next_keys = [&] { if (++k_stage == kStages) k_stage = 0, ++k_turn; };
        for (uint32_t count = 0; good && walk.next(A); ++count) {
          const uint32_t n = __shfl_sync(all_lanes, walk.n, 0);
          good = warp_wait(shared_address(&S.queries[t]), count & 1, dead);
          for (uint32_t half = 0; half < 2 && good; ++half) {
            good = wait_keys();
            if (!good) break;
            order_after();
            if (one_lane()) multiply_keys(half, k_stage);
            __syncwarp();
            next_keys();
          }
          for (uint32_t i = 0; i < 2 * n && good; ++i) {
            const uint32_t half = i & 1;
            const bool more = i + 2 < 2 * n;
            good = (!more || wait_keys()) && warp_wait(shared_address(&S.full_v[v_stage]), v_turn & 1, dead) && warp_wait(shared_address(&S.weights[t][half]), (done + i / 2) & 1, dead);
            if (!good) break;
            order_after();
            if (one_lane()) {
              const uint32_t a = scores_at + half * kHalf, b = value_at + v_stage * (L::kOperand >> 4);
#pragma unroll
              for (uint32_t x = 0; x < kHalf / 16; ++x) product_of_tensor(sums_at, a + x * 8, b + (x * 2048 >> 4), sums_kind, i > 0 || x > 0);
              commit_to(shared_address(&S.sums[t][half]));
              commit_to(shared_address(&S.empty_v[v_stage]));
              if (more) multiply_keys(half, k_stage);
            }
            __syncwarp();
            if (more) next_keys();
            if (++v_stage == kStages) v_stage = 0, ++v_turn;
          }
          done += n;
        }
      } else {
        // ---- where keys lie, and their scales: a warp for the readers of keys, one for those of values
        const uint32_t set = warp - (kSoftmaxWarps + 2 * kReadWarps + 2);
        const unsigned short* const scales = A.scales + (set ? A.plane_scales : 0);
        uint32_t value_unit = 0;  // the upper half of a float, 0 while there are only zeros
        bool good = true, apart = false;
        for (uint32_t blocks = 0; good && walk.next(A); ++blocks) {
          for (uint32_t i = 0; i < walk.n; ++i) {
            const uint32_t x = done + i, slot = x % kFound;
            if (x >= kFound) good = warp_wait(shared_address(&S.found_empty[set][slot]), (x / kFound - 1) & 1, dead);
            if (!good) break;
            const uint32_t key = walk.tiles.key(walk.j0 + i) + lane;
            int32_t page[kKeys / 32];
            uint32_t place[kKeys / 32], all_scales[kKeys / 32][4] = {};  // a key without a place counts as zeros
#pragma unroll
            for (uint32_t k = 0; k < kKeys / 32; ++k) page[k] = page_of(A, walk.q, walk.s, key + 32 * k);
#pragma unroll
            for (uint32_t k = 0; k < kKeys / 32; ++k) place[k] = place_of_key(A, walk.q, walk.head, key + 32 * k, page[k]);
#pragma unroll
            for (uint32_t k = 0; k < kKeys / 32; ++k)
#pragma unroll
              for (uint32_t g = 0; g < 4; ++g)
                if (place[k] != kNone && g < A.groups) all_scales[k][g] = __ldg(scales + (uint64_t)place[k] * A.groups + g);
            // the largest exponents, of a key, and of 16 keys or of the tile, among scales that are numbers; values that are not count as 0
            constexpr uint32_t kExponent = 0x7F80u;
            const bool more = A.groups > 2;
            uint32_t own[kKeys / 32], several[kKeys / 32], most = 0, least = ~0u;  // least: of the scales less 1, so that a 0 does not count
#pragma unroll
            for (uint32_t k = 0; k < kKeys / 32; ++k) {
              own[k] = max(all_scales[k][0], all_scales[k][1]);
              least = min(least, min(all_scales[k][0] - 1, all_scales[k][1] - 1));
              if (more) {
                own[k] = max(own[k], max(all_scales[k][2], all_scales[k][3]));
                least = min(least, min(all_scales[k][2] - 1, all_scales[k][3] - 1));
              }
              most = max(most, own[k]);
            }
            if (__any_sync(0xFFFFFFFFu, most >= kExponent)) {  // some are no numbers, or below 0
              uint32_t broken = 0;  // four bits for each key's groups
              most = 0;
#pragma unroll
              for (uint32_t k = 0; k < kKeys / 32; ++k) {
                own[k] = 0;
#pragma unroll
                for (uint32_t g = 0; g < 4; ++g) {
                  const bool number = (all_scales[k][g] & kExponent) != kExponent;
                  if (set && !number) all_scales[k][g] = 0, broken |= 1u << (4 * k + g);
                  own[k] = max(own[k], number ? all_scales[k][g] & kExponent : 0u);
                }
                most = max(most, own[k]);
              }
              if (set) note_broken(A, walk, broken, key - lane, lane, S.broken[blocks % kMemo]);
            }
            auto in_range = [](uint32_t x) { return min(max(x & kExponent, 0x0100u), 0x7E00u); };
            // A unit for several keys will do while every scale is above 2^-14 of it: in fp16 it keeps its bits then, and its products with codes 11 (and sums do not lose
            // theirs where the unit rises). Else each key has its own, or what one row sees would cost another row bits of what it sees.
            constexpr uint32_t kTogether = 14 << 7;
            if (set) {
              most = __reduce_max_sync(0xFFFFFFFFu, most) & kExponent;
              apart = i > 0 && (apart || (value_unit > 0 && most > value_unit + kTogether));  // for the rest of the block
              value_unit = i == 0 ? most : max(value_unit, most);
              most = in_range(value_unit);
#pragma unroll
              for (uint32_t k = 0; k < kKeys / 32; ++k) several[k] = most;
            } else {
              apart = false;
              uint32_t two[2] = {own[0] | own[1] << 16, own[2] | own[3] << 16};
#pragma unroll
              for (int d = 8; d; d >>= 1) two[0] = __vmaxu2(two[0], __shfl_xor_sync(0xFFFFFFFFu, two[0], d)), two[1] = __vmaxu2(two[1], __shfl_xor_sync(0xFFFFFFFFu, two[1], d));
#pragma unroll
              for (uint32_t k = 0; k < kKeys / 32; ++k) several[k] = in_range(two[k / 2] >> (16 * (k & 1)));
              most = max(max(several[0], several[1]), max(several[2], several[3]));
            }
            apart = __any_sync(0xFFFFFFFFu, apart || (least < kExponent && least + kTogether < most));
            if (apart) {
#pragma unroll
              for (uint32_t k = 0; k < kKeys / 32; ++k) {
                several[k] = in_range(own[k]);
                S.exponents[set][x % kMemo][lane + 32 * k] = (uint8_t)(several[k] >> 7);
              }
            }
            if (set) {
              if (lane == 0) S.value_units[x % kMemo] = apart ? -1.0f : __uint_as_float(most << 16);
            } else if (lane % 16 == 0) {
#pragma unroll
              for (uint32_t k = 0; k < kKeys / 32; ++k) S.units[x % kMemo][2 * k + lane / 16] = apart ? -1.0f : __uint_as_float(several[k] << 16);
            }
#pragma unroll
            for (uint32_t k = 0; k < kKeys / 32; ++k) {
              const float down = __uint_as_float((0x7F00u - several[k]) << 16);
              float y[4] = {};
#pragma unroll
              for (uint32_t g = 0; g < 4; ++g)
                if (g < 2 || more) y[g] = __uint_as_float(all_scales[k][g] << 16) * down;
              S.scales[set][slot][lane + 32 * k] = make_uint2(rounded<false>(y[0], y[1]), rounded<false>(y[2], y[3]));
              S.places[set][slot][lane + 32 * k] = place[k];
            }
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&S.found_full[set][slot]));
          }
          done += walk.n;
        }
      }
    }
    order_before();
    __syncthreads();
    if (S.dead) {  // copies and products on their way have ended long before this
      if (threadIdx.x == 0 && A.status) set_status(A.status, LC_ERR_TIMEOUT);
      for (const long long since = clock64(); clock64() - since < (1 << 22);) {}
    }
    if (warp == kSoftmaxWarps + 2 * kReadWarps) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(S.tensor), "n"(512) : "memory");
  }
};

template <int kBits, uint32_t DP, bool kBf16, bool kCap, bool kBias>
__global__ void __launch_bounds__(kThreads, 1) attend_tiles_kernel(AttendArgs A) {
  Kernel<kBits, DP, kBf16, kCap, kBias>::run(A);
}

// Joins the parts of the blocks that CTAs share (see join_kernel of lc_attend_rows.cuh): a query a thread, blockIdx.y a run of 16 values.
template <bool kBf16>
__global__ void __launch_bounds__(kTileRows) join_tiles_kernel(AttendArgs A, uint32_t ctas) {
  using T = typename TypeOf<kBf16 ? LC_TYPE_BF16 : LC_TYPE_F16>::T;
  __shared__ uint32_t found;
  wait_previous();
  const unsigned long long all = A.flat[A.sequences], share = share_of(all, ctas), border = (blockIdx.x + 1) * share;
  if (border >= all) return;
  if (threadIdx.x < 32) {
    uint32_t lo = 0, count = A.sequences;
    while (count > 1) {
      const uint32_t step = (count + 31) / 32, at = threadIdx.x * step;
      const uint32_t n = __popc(__ballot_sync(0xFFFFFFFFu, at < count && A.flat[lo + at] <= border)) - 1;
      lo += n * step;
      count = min(step, count - n * step);
    }
    if (threadIdx.x == 0) found = lo;
  }
  __syncthreads();
  const uint32_t s = found;
  const Sequence q = sequence_of<kKeys>(A, s, false);
  const Weights W = weights_of(A, q);
  const Place P = place_of(A, W, border - A.flat[s]);
  const unsigned long long begin = border - P.offset, end = begin + P.weight;
  if (P.offset == 0 || begin + share < border) return;
  const uint32_t first = blockIdx.x, last = (uint32_t)((end - 1) / share), r = P.block * kTileRows + threadIdx.x, token = A.by_shared.div(r);
  if (token >= q.rows) return;
  const Tiles tiles = tiles_of(A, q, P.block);
  auto part_of = [&](uint32_t cta) -> const float* {  // null: no tile of the block is that CTA's
    const unsigned long long from = cta * share, to = from + share;
    const uint32_t j0 = from > begin ? tile_at(from - begin, tiles.count, P.weight) : 0, j1 = to < end ? tile_at(to - begin, tiles.count, P.weight) : tiles.count;
    return j0 == j1 || (j0 == 0 && j1 == tiles.count) ? nullptr : A.parts + (2ull * cta + (begin <= from ? 0 : 1)) * (kTilePartBytes / 4);
  };
  float most = -INFINITY, sum = 0.0f, v[16] = {};  // v: the mean over the parts so far
  uint32_t parts = 0;
  const uint32_t d0 = blockIdx.y * 16;
  for (uint32_t c = first; c <= last; ++c) {
    const float* p = part_of(c);
    if (!p) continue;
    const float m = p[kTileRows * kTileDim + threadIdx.x], l = p[kTileRows * (kTileDim + 1) + threadIdx.x], now = fmaxf(most, m);
    float4 x[4];
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) x[e] = d0 + 4 * e < A.dim ? *reinterpret_cast<const float4*>(p + ((d0 / 4 + e) * kTileRows + threadIdx.x) * 4) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float old = most == now ? sum : sum * exp2_fast(most - now), added = m == now ? l : l * exp2_fast(m - now);
    sum = old + added;
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum, keeps = old * over, here = added * over;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      v[4 * e] = v[4 * e] * keeps + x[e].x * here, v[4 * e + 1] = v[4 * e + 1] * keeps + x[e].y * here;
      v[4 * e + 2] = v[4 * e + 2] * keeps + x[e].z * here, v[4 * e + 3] = v[4 * e + 3] * keeps + x[e].w * here;
    }
    most = now;
    ++parts;
  }
  if (parts == 0) return;  // one CTA has had them all
  if (sum == 0.0f) {  // all scores are -Inf
#pragma unroll
    for (uint32_t e = 0; e < 16; ++e) v[e] = __uint_as_float(0x7FFFFFFFu);
  }
  T* out = static_cast<T*>(A.out) + (uint64_t)(q.row + token) * A.out_row + (uint64_t)(P.head * A.shared + (r - token * A.shared)) * A.out_head + d0;
  if (d0 + 16 <= A.dim && (reinterpret_cast<uintptr_t>(out) & 15) == 0) {
#pragma unroll
    for (uint32_t e = 0; e < 16; e += 8)
      *reinterpret_cast<uint4*>(out + e) = make_uint4(rounded<kBf16>(v[e], v[e + 1]), rounded<kBf16>(v[e + 2], v[e + 3]), rounded<kBf16>(v[e + 4], v[e + 5]), rounded<kBf16>(v[e + 6], v[e + 7]));
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 16; ++e)
      if (d0 + e < A.dim) from_float(v[e], out[e]);
  }
}

// CTAs of the kernel: one on each SM.
cudaError_t tile_ctas(uint32_t& ctas) {
  static int sms[kMaxDevices] = {};  // by device ordinal: 0 not looked at yet
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  if (!sms[dev]) {
    int n = 0;
    const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    sms[dev] = n;
  }
  ctas = (uint32_t)sms[dev] < kTileCtas ? (uint32_t)sms[dev] : kTileCtas;
  return cudaSuccess;
}

template <int kBits, uint32_t DP, bool kBf16, bool kCap, bool kBias>
cudaError_t launch(const AttendArgs& a, cudaStream_t cs) {
  static bool ready[kMaxDevices] = {};  // by device ordinal: the kernel may have its shared memory
  const int dev = current_device_index();
  if (dev < 0) return cudaErrorInvalidDevice;
  auto kernel = attend_tiles_kernel<kBits, DP, kBf16, kCap, kBias>;
  if (!ready[dev]) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Layout<kBits, DP>::kWhole);
    if (e != cudaSuccess) return e;
    ready[dev] = true;
  }
  uint32_t ctas = 0;
  const cudaError_t e = tile_ctas(ctas);
  return e != cudaSuccess ? e : launch_kernel(false, kernel, ctas, kThreads, Layout<kBits, DP>::kWhole, cs, a);
}
template <int kBits, bool kBf16, bool kCap, bool kBias>
cudaError_t launch_dim(const AttendArgs& a, cudaStream_t cs) {
  return a.dim <= 64 ? launch<kBits, 64, kBf16, kCap, kBias>(a, cs) : launch<kBits, 128, kBf16, kCap, kBias>(a, cs);
}
template <int kBits, bool kBf16>
cudaError_t launch_scores(const AttendArgs& a, cudaStream_t cs) {
  if (a.cap > 0.0f) return a.slopes ? launch_dim<kBits, kBf16, true, true>(a, cs) : launch_dim<kBits, kBf16, true, false>(a, cs);
  return a.slopes ? launch_dim<kBits, kBf16, false, true>(a, cs) : launch_dim<kBits, kBf16, false, false>(a, cs);
}

}  // namespace

cudaError_t launch_attend_tiles(const AttendArgs& a, int bits, int type, cudaStream_t cs) {
  if (type == LC_TYPE_BF16) return bits == 4 ? launch_scores<4, true>(a, cs) : launch_scores<8, true>(a, cs);
  return bits == 4 ? launch_scores<4, false>(a, cs) : launch_scores<8, false>(a, cs);
}

cudaError_t launch_join_tiles(const AttendArgs& a, int type, cudaStream_t cs) {
  uint32_t ctas = 0;
  const cudaError_t e = tile_ctas(ctas);
  if (e != cudaSuccess || ctas < 2) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas - 1, (a.dim + 15) / 16);
  cfg.blockDim = dim3(kTileRows);
  cfg.stream = cs;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return type == LC_TYPE_BF16 ? cudaLaunchKernelEx(&cfg, join_tiles_kernel<true>, a, ctas) : cudaLaunchKernelEx(&cfg, join_tiles_kernel<false>, a, ctas);
}

}  // namespace lc
