// kv_rows.cuh -- attention of many query rows over the same keys and values of the paged cache: the new tokens of
// prompts (p2p_kv_attend_prompt) and the shared part of rows that begin with the same pages (p2p_kv_attend_shared).
//
// For a query row and the tokens t that it sees: x_t = scale * q . k_t, m = max x_t, z = sum exp(x_t - m), out = sum
// exp(x_t - m) v_t / z, lse = m + ln z.  Rows are (token, query head of one kv head) pairs, numbered with the heads
// inside the tokens; a unit is one or two tiles of up to 128 consecutive ones of one sequence (or group) and kv head,
// with the tokens that any of them sees, kBt at a time.  (Where queries come by boxes, a row tile is as many whole
// tokens as fit 128 rows.)
//
// Both products are the tensor cores' (tcgen05): S = Q K^T with Q and K in shared memory, O += P V with P in tensor
// memory and V in shared memory as it lies in the pages, tokens by values, which the second product takes as its
// transposed operand. S, P (in the place of S) and O stay in tensor memory; a thread owns a row, so maxima and sums
// need no shuffles.  Two tiles of 128 rows take turns: while one's logits go through exp, the tensor cores work on the
// other's.  exp(x - m) takes for m a maximum that lags the running one by at most 2^kLag (see Type), so that O is
// rarely rescaled.  P is rounded to the values' type (beside 8-bit ones to f16), as the tensor cores take both operands
// in 16 bits: each term is off by half a step at most, 2^-8 of it in bf16 and 2^-11 in f16, to either side; z is summed
// from what was not rounded.  Maxima, sums, S, O and parts have 32 bits.
//
// A CTA of the persistent grid takes an equal, contiguous share of all units' steps (a step: kBt tokens); a unit that
// several CTAs share goes to scratch in parts, which a launch after this one joins in their order (kv_join.cu), so
// results do not depend on timing.  A unit with one row tile alone lets both tiles take its steps by turns, each with
// sums of its own, as one tile's chain of products and exp leaves the tensor cores idle (191 sequences of 1 to 9 new
// tokens, 1,000 seen: 375 us, and one tile at a time 408).
//
// Warps: softmax (four a row tile), copies (four), one each for the products and the schedule, and two helpers, which
// bring the queries and look for infinities and NaN among the values of tokens that not all rows see: 0 * NaN is NaN,
// so such values are taken out before the product and added to the rows that do see them at the end.  Pages of whole
// eights of tokens come by the tensor memory accelerator, a box of tokens of one page and head at a time, turned as the
// products read them; others by cp.async, 16 bytes a lane (an instruction for 512 bytes instead of some kilobytes: the
// copy warps then need 3,500 cycles for a step of 128 tokens of 128 values, more than the products and exp).  8-bit
// values are widened to f16 on their way through a warp's registers, as queries of 16 bits have to meet values of their
// own type.
//
// Long prompts are bound by the tensor cores and the chain behind them: 4,096 tokens after 12,288, 40 / 8 heads of 128
// in f16, 1.2e12 operations in 784 to 850 us on one GB300 (1.41 to 1.53 PFLOP/s, 73 to 80% of what cuBLAS reaches in a
// burst; the tensor pipe is 68% active): a step's S and P V take 2,048 cycles at the rate of the tensor cores, and the
// 3,100 that they take are a tile's products (1,024), its exp (1,500: 512 of the exponential units, the rest loads of
// tensor memory, the maximum, rounding and the way back) and the waits between them.  Short ones are bound by what a
// unit costs beside its steps: 1.5 to 2 us of its queries' way in and its results' way out, and 5 to 10 us of the launch
// before the first step (the schedule, cold code).  Registers: 184 a thread for softmax, where a step's logits stay, 72
// for the others, which spill more with 56 (of the kernels for heads of up to 128, 32 to 112 bytes a thread are spilled,
// none beyond).
#pragma once
#include "kv_math.cuh"
#include "kv_values.cuh"

namespace p2p {
namespace {

template <int KIND, int DP>
struct RowsShape {
  static constexpr int kTiles = DP <= 128 ? 2 : 1;     // row tiles of a unit
  static constexpr int kBt = DP <= 128 ? 128 : 64;     // tokens of a step
  static constexpr int kBtLog = DP <= 128 ? 7 : 6;
  static constexpr int kChunks = DP / 64;              // of 64 values: 128 bytes, a swizzled row
  static constexpr int kQTile = 128 * DP * 2;
  static constexpr int kStage = kBt * DP * 2;          // keys or values of a step, 16 bits each
  static constexpr int kRaw = KIND == P2P_KV_E4M3 ? kBt * DP : 0;  // the same in 8 bits, on its way
  static constexpr int kRaws = 4;                      // two of keys, two of values
  static constexpr int kMisc = 2048;
  static constexpr int kFit = (232448 - 1024 - kMisc - kTiles * kQTile - kRaws * kRaw) / kStage;
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static_assert(kStages >= 3, "keys and values of a step, and the next on their way");
  static constexpr int kBytes = 1024 + kMisc + kTiles * kQTile + kRaws * kRaw + kStages * kStage;
  static constexpr int kSoft = 4 * kTiles;             // softmax warps
  static constexpr int kThreads = (kSoft + 8) * 32;
  static constexpr int kOCol = kTiles * kBt;           // columns of tensor memory: S of the tiles, then O of them
  static_assert(kOCol + kTiles * DP <= 512);
};

constexpr int kSplitSteps = 4;  // from which on
constexpr int kRing = 4;  // units that the schedule is ahead
struct RowsUnit {
  int64_t row;       // of q: the unit's first
  int32_t rows;      // 0: no more units
  int32_t g0;        // the first row's head among its kv head's
  int32_t h, seq;
  int32_t pos;       // prompts: position of the first row's token
  int32_t begin, end;        // tokens that any row sees
  int32_t all_begin, all_end;  // tokens that every row sees, or none
  int32_t j0, j1;            // steps of this piece
  int32_t t0[2], t1[2];      // of them, those of each row tile
  int32_t parts, part, c0;   // of the unit, where it is shared: this piece's number and the first one's CTA
  int32_t split;             // 1: both row tiles have the same rows, and every other step
};
// The q-th stage of a unit's n steps, keys or values of one: K0, V0, K1, V1, .., or, where the row tiles take turns
// with the steps, K0, K1, V0, K2, V1, .., as the products need them.
struct RowsStage {
  int32_t step;
  bool values;
};
__device__ __forceinline__ RowsStage rows_stage(int32_t q, int32_t n, bool split) {
  if (!split) return {q >> 1, (q & 1) != 0};
  const bool values = q == 2 * n - 1 || (q > 0 && !(q & 1));
  return {q == 2 * n - 1 ? n - 1 : values ? q / 2 - 1 : (q + 1) / 2, values};
}
struct RowsShared {
  uint64_t full[8], empty[8], q_full[2], s_full[2], p_full[2], o_full[2], unit_full[kRing], unit_empty[kRing],
      checked[8], q_empty[2], q_raw[2], pair, pair_done, drain, done, raw[4][4];
  RowsUnit unit[kRing];
  uint32_t sums[16];
  int32_t tmem, dead;
  int32_t signs;             // of work: not negative; changes with every stage, and within add_poison_of
  int32_t poison[kRing];     // whether values were taken out of the unit's steps
  float pair_top[128], pair_sum[128];  // of the second tile's rows, where both have the same
};
static_assert(sizeof(RowsShared) <= 2048);

__device__ __forceinline__ void bar_init(const uint64_t& bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_of(&bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(const uint64_t& bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_of(&bar)) : "memory");
}
// Whether a phase is over; the thread may sleep for up to 10 ms.
__device__ __forceinline__ bool bar_try(const uint64_t& bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.b32 %0, 1, 0, p; }"
               : "=r"(ok)
               : "r"(smem_of(&bar)), "r"(parity), "r"(10000000)
               : "memory");
  return ok;
}
// Waits for a phase; false where the watch (bar_watch) gave up meanwhile.  Of a warp's lanes some may go on and others
// not.  (Every wait has this in place, so it is small: with a limit of its own in each, 191 sequences of 1 to 9 new
// tokens take 429 us, not 377.)
__device__ __forceinline__ bool bar_wait_lane(const uint64_t& bar, uint32_t parity, RowsShared& sh) {
  while (!bar_try(bar, parity))
    if (*(volatile int32_t*)&sh.dead) return false;
  return true;
}
// The same for a whole warp, whose lanes go on or give up together: what follows takes all of them.
__device__ __forceinline__ bool bar_wait(const uint64_t& bar, uint32_t parity, RowsShared& sh) {
  while (!__all_sync(~0u, bar_try(bar, parity)))
    if (__any_sync(~0u, *(volatile int32_t*)&sh.dead)) return false;
  return true;
}
// The same for the one warp that watches while it waits: where it sees no sign of work in the CTA for as long as the
// call has patience (which should never be), all give up, and the kernel ends and reports it.
__device__ __forceinline__ bool bar_watch(const uint64_t& bar, uint32_t parity, RowsShared& sh, long long patience) {
  long long from = clock64();
  int32_t signs = -1;
  while (!__all_sync(~0u, bar_try(bar, parity))) {
    const int32_t now = *(volatile int32_t*)&sh.signs;
    if (now != signs) signs = now, from = clock64();
    if (__any_sync(~0u, clock64() - from > patience)) {
      *(volatile int32_t*)&sh.dead = 1;
      return false;
    }
  }
  return true;
}
// What is still on its way when a kernel gives up, waited for with a limit (a phase may never come).
__device__ __forceinline__ void bar_drain(const uint64_t& bar, uint32_t parity) {
  const long long from = clock64();
  for (uint32_t ok = 0; !ok && clock64() - from < 1 << 22;)
    asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.b32 %0, 1, 0, p; }"
                 : "=r"(ok)
                 : "r"(smem_of(&bar)), "r"(parity)
                 : "memory");
}
// The next phase also takes so many bytes of copies.
__device__ __forceinline__ void bar_expect(const uint64_t& bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_of(&bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* map, int32_t x, int32_t token, int32_t head,
    int32_t page,
                                         int32_t layer, const uint64_t& bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, "
               "%6}], [%7];" ::"r"(to), "l"(map), "r"(x), "r"(token), "r"(head), "r"(page), "r"(layer),
                   "r"(smem_of(&bar))
               : "memory");
}
__device__ __forceinline__ void copy_query_box(uint32_t to, const CUtensorMap* map, int32_t x, int32_t head,
    int32_t row,
                                               const uint64_t& bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, 0, %3, %4}], "
               "[%5];" ::"r"(to), "l"(map), "r"(x), "r"(head), "r"(row), "r"(smem_of(&bar))
               : "memory");
}
__device__ __forceinline__ void async_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// (The products' warp runs together and one of its threads issues: operands stay in uniform registers that way.)
__device__ __forceinline__ uint32_t elected() {
  uint32_t x;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.b32 %0, 1, 0, p; }" : "=r"(x));
  return x;
}
__device__ __forceinline__ void mma_done(const uint64_t& bar, uint32_t one) {
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %1, 0;\n"
               "@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(smem_of(&bar)),
                   "r"(one)
               : "memory");
}
// A matrix in shared memory, rows of 128 bytes turned within eights of them; lead: bytes between chunks of 64 values,
// for an operand whose rows are the product's k.
__device__ __forceinline__ uint64_t matrix(uint32_t at, uint32_t lead) {
  return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, uint32_t add, uint32_t one) {
  asm volatile("{ .reg .pred p, q; setp.ne.b32 p, %4, 0; setp.ne.b32 q, %5, 0;\n"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b), "r"(what),
                   "r"(add), "r"(one)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, uint32_t add, uint32_t one) {
  asm volatile("{ .reg .pred p, q; setp.ne.b32 p, %4, 0; setp.ne.b32 q, %5, 0;\n"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b), "r"(what),
                   "r"(add), "r"(one)
               : "memory");
}
#define P2P_R8(r, o) "=r"((r)[o]), "=r"((r)[o + 1]), "=r"((r)[o + 2]), "=r"((r)[o + 3]), "=r"((r)[o + 4]), "=r"((r)[o + 5]), \
                     "=r"((r)[o + 6]), "=r"((r)[o + 7])
#define P2P_I8(r, o) "r"((r)[o]), "r"((r)[o + 1]), "r"((r)[o + 2]), "r"((r)[o + 3]), "r"((r)[o + 4]), "r"((r)[o + 5]), \
                     "r"((r)[o + 6]), "r"((r)[o + 7])
// 32 columns of the warp's 32 rows, a row a lane.
__device__ __forceinline__ void tmem_load(uint32_t* r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : P2P_R8(r, 0), P2P_R8(r, 8), P2P_R8(r, 16), P2P_R8(r, 24)
               : "r"(at)
               : "memory");
}
// The same for 16 columns.
__device__ __forceinline__ void tmem_load16(uint32_t* r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
               "[%16];"
               : P2P_R8(r, 0), P2P_R8(r, 8)
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16};" ::"r"(at),
               P2P_I8(r, 0), P2P_I8(r, 8)
               : "memory");
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ float2 parts_of(uint64_t x) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(x));
  return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t x;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
  return x;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t x;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
  return x;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float x;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(x) : "f"(a), "f"(b), "f"(c));
  return x;
}

// An item of the call: a sequence with its new tokens, or a group with what it shares.  Its tiles of rows follow one
// another for each kv head in turn.  (Rows are counted in 31 bits and costs in 32: the host sees to both.)
struct RowsItem {
  int64_t row0;             // its first row of q
  int32_t members, tiles;   // tokens (rows of the group), and tiles of them times the heads of a kv head
  int32_t seq, pos;         // pos: the first token's position; of a group: where the last row's window begins
  int32_t shared, first;    // of a group: tokens first .. shared - 1 are seen
};
// broken: set where offsets descend or leave the batch.  (No item is then taken: rows that several items name would be
// counted beyond what the host allows for.)
template <class S>
__device__ __forceinline__ RowsItem rows_item(const KvView& c, const KvRowsCall& a, int32_t i, int32_t* err,
                                              bool& broken) {
  RowsItem r = {0, 0, 0, 0, 0, 0, 0};
  if (a.spans) {
    const int4 span = a.spans[i];
    if (span.x == 0) return r;  // (nothing is shared, or the groups do not hold)
    const int32_t r0 = a.groups[i], r1 = a.groups[i + 1], shared = shared_tokens(c, span, r1 - r0);
    if (shared == 0) return r;
    r = {r0, r1 - r0, 0, a.seq ? a.seq[r0] : r0, span.z, shared, span.y};
  } else {
    const int64_t o0 = a.offsets[i], o1 = a.offsets[i + 1];
    const int32_t seq = a.seq ? a.seq[i] : i;
    int32_t bad = o0 < 0 || o1 < o0 || o1 > a.n_tokens ? KV_BAD_OFFSETS : 0;
    broken |= bad != 0;
    if (!bad && o1 > o0) {
      const int32_t len = (uint32_t)seq < (uint32_t)c.n_seqs ? length_of(c, seq) : -2;
      if (len == -2)
        bad = KV_BAD_SEQ;
      else if (len < o1 - o0)
        bad = KV_BAD_COUNT;
      else
        r = {o0, (int32_t)(o1 - o0), 0, seq, len - (int32_t)(o1 - o0), 0, 0};
    }
    if (bad && err) atomicOr(err, bad);
  }
  const uint32_t unit = S::kTiles * a.tile_rows;
  r.tiles = (r.members * a.group + unit - 1) / unit;
  return r;
}
__device__ __forceinline__ int32_t window_begin(const KvRowsCall& a, int32_t end) {
  return a.window && end > a.window ? end - a.window : 0;
}
// Tokens that rows of an item's members (tokens) t0 to t1 see: any of the rows, and each of them.
struct RowsSpan {
  int32_t begin, end, all_begin, all_end;
};
__device__ __forceinline__ RowsSpan rows_span(const KvRowsCall& a, const RowsItem& it, int32_t t0, int32_t t1) {
  if (a.spans) return {it.first, it.shared, it.pos, it.shared};
  const int32_t e0 = it.pos + t0 + 1, e1 = it.pos + t1 + 1;
  return {window_begin(a, e0), e1, window_begin(a, e1), e0};
}
template <class S>
__device__ __forceinline__ RowsCost rows_cost(const KvRowsCall& a, const RowsItem& it) {
  return a.spans ? RowsCost::of_prefix(it.first, it.shared, a.count, S::kBtLog)
                 : RowsCost::of_prompt(it.pos, a.window, a.count, S::kBtLog);
}
// Values d .. d + 15 of a row's result: o, times f.  (Whole sectors where that is to be had, as the lanes' rows are
// apart.)
__device__ __forceinline__ void put(const KvView& c, const KvRowsCall& a, int64_t row, int32_t head, int32_t d,
    const float* o, float f) {
  const bool half = d + 8 >= c.dim;  // (head_dim is a multiple of 8)
  if (a.pre) {
    uint32_t b[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) b[k] = __float_as_uint(o[k] * f);
    float* const to = a.pre + (row * a.heads + head) * c.dim + d;
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), P2P_I8(b, 0) : "memory");
    if (!half) asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 8), P2P_I8(b, 8)
        : "memory");
    return;
  }
  uint16_t* const out = (uint16_t*)a.out + row * a.out_row + head * a.out_head + d;
  uint32_t b[8];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    b[k] = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(o[2 * k] * f, o[2 * k + 1] * f)
        : pack<P2P_KV_F16>(o[2 * k] * f, o[2 * k + 1] * f);
  if (a.out32 && !half) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out), P2P_I8(b, 0) : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < 8 || !half) out[k] = (uint16_t)(b[k / 2] >> (k & 1) * 16);
  }
}
// Whether every row sees all of step j's tokens.  (Its end may be 2^31, which 32 bits do not hold.)
template <int BT>
__device__ __forceinline__ bool seen_by_all(int32_t j, int32_t all_begin, int32_t all_end) {
  return j * BT >= all_begin && all_end - j * BT >= BT;
}
// Infinities and NaN that were taken out of the values of `every` step from j0 to j1 (of those that not all rows see):
// added to the sums of the rows that see them, tokens begin .. end - 1.  By a warp, whose 32 rows of sums are at o_at.
// Rarely needed, so it is small, not fast.
template <int KIND, int BT>
__device__ __forceinline__ void add_poison_of(const KvView& c, const KvRowsCall& a, const RowsUnit& u, uint32_t o_at,
    int32_t j0, int32_t j1,
                                              int32_t every, int32_t begin, int32_t end, int32_t& signs) {
  const int lane = threadIdx.x & 31;
  constexpr int kValues = KIND == P2P_KV_E4M3 ? 16 : 8;  // of a piece
#pragma unroll 1
  for (int32_t j = j0; j < j1; j += every) {
    if (seen_by_all<BT>(j, u.all_begin, u.all_end)) continue;
    const int32_t last = j * BT + min(BT, u.end - j * BT);
#pragma unroll 1
    for (int32_t p = max(u.begin, j * BT); p < last; ++p) {
      if (lane == 0) *(volatile int32_t*)&signs = p;  // (the next token's number is another)
      const uint32_t e = c.by_page.div(p);
      const int32_t page = row_of(c, u.seq)[e];
      if ((uint32_t)page >= (uint32_t)c.n_pages) continue;
      const char* const at = c.v + a.layer * c.layer_stride + page * c.page_stride +
          (p - (int32_t)e * c.page) * c.token_stride + u.h * c.head_stride;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (lane < c.row16) v = *(const uint4*)(at + lane * 16);
      const uint32_t b[4] = {v.x, v.y, v.z, v.w};
      bool bad = false;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        bad |= KIND == P2P_KV_E4M3 ? (((b[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0
                                   : (((b[k] & (KIND == P2P_KV_BF16 ? 0x7f807f80u : 0x7c007c00u)) +
                                       (KIND == P2P_KV_BF16 ? 0x00800080u : 0x04000400u)) & 0x80008000u) != 0;
#pragma unroll 1
      for (uint32_t pieces = __ballot_sync(~0u, bad); pieces; pieces &= pieces - 1) {
        const int piece = __ffs(pieces) - 1;
#pragma unroll 1
        for (int k = 0; k < kValues; ++k) {
          const char* const one = at + piece * 16 + k * (16 / kValues);
          const float f = KIND == P2P_KV_E4M3   ? __half2float(__nv_cvt_fp8_to_halfraw(*(const uint8_t*)one, __NV_E4M3))
                          : KIND == P2P_KV_BF16 ? __bfloat162float(*(const __nv_bfloat16*)one)
                                                : __half2float(*(const __half*)one);
          if (fabsf(f) < INFINITY) continue;
          uint32_t o;
          asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(o) : "r"(o_at + piece * kValues + k)
              : "memory");
          tmem_loaded();
          if (p >= begin && p < end) o = __float_as_uint(__uint_as_float(o) + f);
          asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(o_at + piece * kValues + k), "r"(o)
              : "memory");
          tmem_stored();
        }
      }
    }
  }
}

template <int KIND, int DP>
__global__ void __launch_bounds__(RowsShape<KIND, DP>::kThreads, 1)
    rows_kernel(KvView c, const __grid_constant__ KvMaps maps, const __grid_constant__ CUtensorMap q_map, KvRowsCall a,
                KvAttendScratch w) {
  using S = RowsShape<KIND, DP>;
  constexpr int kTiles = S::kTiles, kBt = S::kBt, kStages = S::kStages;
  extern __shared__ char room_[];
  char* const room = room_ + ((1024 - (smem_of(room_) & 1023)) & 1023);
  char* const q_room = room;
  char* const stages = q_room + kTiles * S::kQTile;
  char* const raws = stages + kStages * S::kStage;
  RowsShared& sh = *(RowsShared*)(raws + S::kRaws * S::kRaw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // Whether queries are multiplied as they are (see change_queries).
  const bool direct = KIND != P2P_KV_E4M3 && a.scale >= 0.f;
  // (Nothing so far touches memory: it runs beside the end of the kernel before.)
  if (threadIdx.x == 0) {
    for (int i = 0; i < 8; ++i) bar_init(sh.full[i], KIND != P2P_KV_E4M3 && maps.rows ? 4 : 128),
        bar_init(sh.empty[i], 3), bar_init(sh.checked[i], 2);
    for (int i = 0; i < 2; ++i) bar_init(sh.q_full[i], !direct ? 4 : a.boxes ? 2 : 64),
        bar_init(sh.q_raw[i], a.boxes ? 2 : 64), bar_init(sh.q_empty[i], 1), bar_init(sh.s_full[i], 1),
            bar_init(sh.p_full[i], 4), bar_init(sh.o_full[i], 1);
    for (int i = 0; i < kRing; ++i) bar_init(sh.unit_full[i], 1), bar_init(sh.unit_empty[i], S::kSoft + 7),
        sh.poison[i] = 0;
    for (int i = 0; i < 16; ++i) bar_init(sh.raw[i / 4][i & 3], 1);
    bar_init(sh.pair, 4);
    bar_init(sh.pair_done, 4);
    bar_init(sh.drain, 1);
    bar_init(sh.done, S::kSoft + 7);
    sh.dead = 0, sh.signs = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == S::kSoft + 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(&sh.tmem))
        : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    before_sync();
  }
  begin_kernel();

  // ---- what all items count for: a warp sums consecutive ones, 32 at a time.  (Code that runs once costs its way from
  // memory, a microsecond every few hundred instructions: this and the schedule are kept short.)
  constexpr int kAll = S::kThreads / 32;
  const int32_t per_warp = ((a.n + kAll - 1) / kAll + 31) & ~31;
  uint32_t sum_of = 0;
  // (The schedule's warp has the first items, and keeps them.)
  const int turn = warp >= S::kSoft + 5 ? warp - (S::kSoft + 5) : warp + 3;
  RowsItem own = {};
  uint32_t own_cost = 0;
  bool broken = false;
#pragma unroll 1
  for (int32_t i = turn * per_warp + lane; i < min(a.n, (turn + 1) * per_warp); i += 32) {
    own = rows_item<S>(c, a, i, blockIdx.x == 0 ? w.err : nullptr, broken);
    own_cost = own.tiles ? rows_cost<S>(a, own).of(own.tiles) : 0;
    sum_of += c.heads * own_cost;
  }
  sum_of = __reduce_add_sync(~0u, sum_of);
  broken = __any_sync(~0u, broken);  // (~0 in the place of a sum, which is less)
  if (lane == 0) sh.sums[turn] = broken ? ~0u : sum_of;
  __syncthreads();
  after_sync();
  const uint32_t of_warp = lane < kAll ? sh.sums[lane] : 0,
      total = __any_sync(~0u, of_warp == ~0u) ? 0 : __reduce_add_sync(~0u, of_warp);
  // (Shares of kRowsSet at least, so that no two begin at the same step inside a unit.  One prompt of 540 tokens, 14 / 2
  // heads of 64: 14.8 us, and with shares of four at least 16.5, of eight 20.7.)
  const uint32_t ctas = min(gridDim.x, max(1u, total / kRowsSet));
  if (total == 0 || blockIdx.x >= ctas) {
    if (threadIdx.x == 0) w.joins[blockIdx.x].parts = 0;
    if (warp == S::kSoft + 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh.tmem));
    return;
  }
  const uint32_t tmem = sh.tmem;
  const int32_t dim16 = (c.dim + 15) / 16 * 16, chunks = (dim16 + 63) / 64;  // (of 64 values, all of which are filled)
  int32_t ring = 0;          // the unit's place, and the phase of its barriers
  uint32_t ring_phase = 0;
  const auto next_unit = [&]() {
    if (++ring == kRing) ring = 0, ring_phase ^= 1;
  };

  if (warp < S::kSoft) {
    // ================================ softmax: a thread a row
    if (kTiles == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    const int tile = warp / 4, r = (warp & 3) * 32 + lane;  // of the row tile
    // (tensor memory's lanes 32 * (warp % 4) .., from bit 16 on)
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;
    const uint32_t s_at = tmem + lanes + tile * kBt, o_at = tmem + lanes + S::kOCol + tile * DP;
    char* const q_tile = q_room + tile * S::kQTile;
    uint32_t s_phase = 0, o_phase = 0;
    float mul = 0.f;  // logit (in log2) of a sum of products
    // (0 times a masked -infinity would be NaN.  The least number instead makes of the largest sum 2^-21; NaN stays NaN.)
    const auto not_zero = [](float x) { return x == 0.f ? 0x1p-149f : x; };
    // Where row x of the unit's tile is.
    const auto row_of_q = [&](const RowsUnit& u, int x, int64_t& row, int32_t& head) {
      const uint32_t y = u.g0 + (u.split ? 0 : tile * a.tile_rows) + x, t = a.by_group.div(y);
      row = u.row + t;
      head = u.h * a.group + (int32_t)(y - t * a.group);
    };
    // Queries that are not multiplied as they are: a negative scale changes their signs, as exp's maximum is the
    // products', and beside 8-bit keys bf16 ones become f16.  A thread has its row.
    uint32_t raw_phase = 0;
    const auto change_queries = [&](const RowsUnit& u) {
      if (!bar_wait(sh.q_raw[tile], raw_phase, sh)) return false;
      raw_phase ^= 1;
      float unit = fabsf(a.scale) * kLog2e;
      bool minus = a.scale < 0.f;
      if (KIND == P2P_KV_E4M3) {
        const float k_scale = c.k_scale[a.layer * c.heads + u.h];
        unit *= fabsf(k_scale), minus ^= k_scale < 0.f;
      }
      const uint32_t flip = minus ? 0x80008000u : 0;
      const auto piece_at = [&](int k) { return (uint4*)(q_tile + k / 8 * (128 * 128) + r * 128 +
          ((k & 7) ^ (r & 7)) * 16); };
      const bool narrow = KIND == P2P_KV_E4M3 && a.type == P2P_KV_BF16;
      float down = 1.f;
      if (narrow) {
        // In f16, scaled by a power of two so that the row's largest is in [2^14, 2^15): exact but for what is below
        // 2^-28 of it. (Magnitudes compare as their bits do.)
        uint32_t m = 0;
#pragma unroll 4
        for (int k = 0; k < dim16 / 8; ++k) {
          const uint4 v = *piece_at(k);
          m = __vmaxu2(m, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu),
              __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
        }
        const float largest = __uint_as_float(max(m << 16, m & 0xffff0000u));
        // (Of 0, an infinity or NaN: as they are.)
        const int e = largest > 0.f && largest < INFINITY ? max((int)(__float_as_uint(largest) >> 23) - 127, -112) - 14
            : 0;
        down = __uint_as_float((127 - e) << 23), unit *= __uint_as_float((127 + e) << 23);
      }
      mul = not_zero(unit);
      if (narrow || flip) {
#pragma unroll 4
        for (int k = 0; k < dim16 / 8; ++k) {
          const uint4 v = *piece_at(k);
          uint32_t b[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (narrow) {
              const float2 y = two_halves(b[i], P2P_KV_BF16);
              b[i] = pack<P2P_KV_F16>(y.x * down, y.y * down);
            }
            b[i] ^= flip;
          }
          *piece_at(k) = make_uint4(b[0], b[1], b[2], b[3]);
        }
        async_fence();
      }
      __syncwarp();
      if (lane == 0) bar_arrive(sh.q_full[tile]);
      return true;
    };
    const auto run = [&]() {
      int32_t now = -1;  // the unit whose results are to be put away
      bool some = false, valid = false;
      float top = 0.f;
      uint64_t sum = 0;
      int64_t row = 0;
      int32_t head = 0, begin = 0, end = 0, from = 0, to = 0;
      uint32_t pair_phase = 0;
#pragma unroll 1
      for (;;) {
        if (!bar_wait(sh.unit_full[ring], ring_phase, sh)) return;
        const bool more = sh.unit[ring].rows > 0;

        // ---- the last unit's results
        if (some) {
          const RowsUnit& u = sh.unit[now];
          if (to > from) {
            if (!bar_wait(sh.o_full[tile], o_phase, sh)) return;
            o_phase ^= 1;
            after_sync();
            if (sh.poison[now])
              add_poison_of<KIND, kBt>(c, a, u, o_at, from, to, u.split ? 2 : 1, valid ? begin : INT32_MAX, end, sh.signs);
          }
          const float2 z2 = parts_of(sum);
          float z = z2.x + z2.y, fade = 1.f, fade2 = 0.f;  // of this tile's sums, and of the second's
          const bool paired = kTiles == 2 && u.split && u.t1[1] > u.t0[1];
          if (paired) {
            if (tile == 1) {  // the first tile's warps take over
              sh.pair_top[r] = top, sh.pair_sum[r] = z;
              before_sync();
              __syncwarp();
              if (lane == 0) bar_arrive(sh.pair);
              if (!bar_wait(sh.pair_done, pair_phase, sh)) return;
              pair_phase ^= 1;
              after_sync();
              valid = false;
            } else {
              if (!bar_wait(sh.pair, pair_phase, sh)) return;
              pair_phase ^= 1;
              after_sync();
              const float other = sh.pair_top[r], high = fmaxf(top, other), ref = high == -INFINITY ? 0.f : high;
              fade = exp2_fast(top - ref), fade2 = exp2_fast(other - ref);
              z = z * fade + sh.pair_sum[r] * fade2;
              top = high;
            }
          }
          const float v_scale = KIND == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + u.h] : 1.f;
          float* const part = w.parts + rows_part(u.c0 + u.part, u.part == 0, kTiles, tile, DP);
          const bool keep = u.parts > 1 && !(paired && tile == 1);
          float f = 0.f;
          if (keep) {
            part[DP * 128 + r] = top, part[(DP + 1) * 128 + r] = z;
          } else if (valid) {
            // (A part without a finite logit counts for nothing; a row has a token at least, and is then NaN.)
            f = z == 0.f && a.pre ? 0.f : v_scale / z;
            if (a.pre)
              a.pre_sum[row * a.heads + head] = make_float2(top, z);
            else if (a.lse)
              a.lse[row * a.heads + head] = z == 0.f ? -INFINITY : log_sum<KIND>(top, z);
          }
#pragma unroll 1
          for (int32_t d = 0; d < dim16 && !(paired && tile == 1); d += 32) {
            float o[32] = {};
            if (to > from) {
              tmem_load((uint32_t*)o, o_at + d);
              if (paired && tile == 0) {
                uint32_t o2[32];
                tmem_load(o2, o_at + DP + d);
                tmem_loaded();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = o[i] * fade + __uint_as_float(o2[i]) * fade2;
              }
              tmem_loaded();
            }
            if (keep) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (d + 4 * i < dim16) ((float4*)part)[r + (d / 4 + i) * 128] = make_float4(o[4 * i], o[4 * i + 1],
                    o[4 * i + 2], o[4 * i + 3]);
            } else if (valid) {
              put(c, a, row, head, d, o, f);
              if (d + 16 < dim16) put(c, a, row, head, d + 16, o + 16, f);
            }
          }
          if (paired && tile == 0) {
            before_sync();
            __syncwarp();
            if (lane == 0) bar_arrive(sh.pair_done);
          }
        }
        // (Loads of tensor memory are done before the next products may write there: P of this unit is announced
        // later.)
        before_sync();
        __syncwarp();
        if (now >= 0 && lane == 0) bar_arrive(sh.unit_empty[now]);
        if (!more) return;

        // ---- this unit's steps
        now = ring;
        next_unit();
        const RowsUnit& u = sh.unit[now];
        const int32_t every = u.split ? 2 : 1;
        some = u.split ? u.t1[tile] > u.t0[tile] : u.rows > tile * a.tile_rows;
        valid = some && r < a.tile_rows && (u.split ? 0 : tile * a.tile_rows) + r < u.rows;
        from = u.t0[tile], to = u.t1[tile];
        top = -INFINITY, sum = 0;
        begin = 0, end = INT32_MAX;  // (rows past the last one mask nothing)
        if (valid) {
          row_of_q(u, r, row, head);
          if (a.spans) {
            end = u.end;
            if (a.window) begin = window_begin(a, length_of(c, a.seq ? a.seq[row] : (int32_t)row));
          } else {
            end = u.pos + (int32_t)(row - u.row) + 1;
            begin = window_begin(a, end);
          }
        }
        if (direct)
          mul = not_zero(a.scale * kLog2e);
        else if (to > from && !change_queries(u))
          return;
        const float unit_mul = mul;
#pragma unroll 1
        for (int32_t j = from; j < to; j += every) {
          if (!bar_wait(sh.s_full[tile], s_phase, sh)) return;
          s_phase ^= 1;
          after_sync();
          uint32_t x[kBt];
#pragma unroll
          for (int k = 0; k < kBt / 32; ++k) tmem_load(x + 32 * k, s_at + 32 * k);
          tmem_loaded();
          const int32_t t0 = j * kBt, lo = begin - t0, hi = end - t0;  // seen: lo .. hi - 1
          if (__any_sync(~0u, lo > 0 || hi < kBt)) {
#pragma unroll
            for (int k = 0; k < kBt / 32; ++k) {
              const int32_t l = min(max(lo - 32 * k, 0), 32), m = min(max(hi - 32 * k, 0), 32);
              const uint32_t seen = (m >= 32 ? ~0u : (1u << m) - 1) & (l >= 32 ? 0u : ~0u << l);
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(seen >> i & 1)) x[32 * k + i] = 0xff800000u;
            }
          }
          float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < kBt; i += 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = max3(t[k], __uint_as_float(x[i + 2 * k]),
                __uint_as_float(x[i + 2 * k + 1]));
          const float most = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) * unit_mul;
          // (Rows past the last one, whatever they are, have no say: results would depend on it.)
          if (__any_sync(~0u, valid && most > top + (Type<KIND>::kUp + Type<KIND>::kLag))) {
            const float next = fmaxf(most - Type<KIND>::kUp, top), fade = next == -INFINITY ? 1.f
                : exp2_fast(top - next);
            top = next;
            const float2 z = parts_of(sum);
            sum = pair_of(z.x * fade, z.y * fade);
            if (j > from) {
#pragma unroll 1
              for (int32_t d = 0; d < dim16; d += 16) {
                uint32_t o[16];
                tmem_load16(o, o_at + d);
                tmem_loaded();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * fade);
                tmem_store16(o_at + d, o);
              }
            }
          }
          const float less = top == -INFINITY ? 0.f : -top;
          const uint64_t by = pair_of(unit_mul, unit_mul), plus = pair_of(less, less);
          uint64_t sum2 = 0;
#pragma unroll
          for (int k = 0; k < kBt / 32; ++k) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int y = 32 * k + 2 * i;
              const float2 f = parts_of(fma2(pair_of(__uint_as_float(x[y]), __uint_as_float(x[y + 1])), by, plus));
              const float e0 = exp2_fast(f.x), e1 = exp2_fast(f.y);
              if (i & 1)
                sum2 = add2(sum2, pair_of(e0, e1));
              else
                sum = add2(sum, pair_of(e0, e1));
              p[i] = pack<KIND>(e0, e1);
            }
            tmem_store16(s_at + 16 * k, p);
          }
          sum = add2(sum, sum2);
          tmem_stored();
          before_sync();
          __syncwarp();
          if (lane == 0) bar_arrive(sh.p_full[tile]);
        }
      }
    };
    run();
  } else if (warp < S::kSoft + 4) {
    // ================================ copies: a warp has a quarter of a step's tokens
    if (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    constexpr int kOwn = kBt / 4;
    const int own0 = (warp - S::kSoft) * kOwn;
    const int64_t across = c.v - c.k;
    int32_t stage = 0;
    uint32_t phase = 1;   // (of `empty`: a fresh barrier's last phase counts as done)
    uint32_t raw_phase = 0;
    const auto run = [&]() {
#pragma unroll 1
      for (;;) {
        if (!bar_wait(sh.unit_full[ring], ring_phase, sh)) return;
        const RowsUnit& u = sh.unit[ring];
        if (u.rows == 0) return;
        const int32_t j0 = u.j0, n = u.j1 - j0, begin = u.begin, end = u.end;
        const bool split = u.split;
        const char* const base = c.k + a.layer * c.layer_stride + u.h * c.head_stride;
        const int32_t* const pages = row_of(c, u.seq);
        // A lane has a box of tokens of each step (a token, without maps): its first, and the page that it lies in, -1:
        // it is not needed.
        const int32_t size = maps.rows ? maps.rows : 1, boxes = kOwn / size;
        // (of a step past the last one: any number)
        const auto token_of = [&](int32_t step) {
          return (int32_t)((uint32_t)(j0 + step) * kBt + own0 + lane * size);
        };
        const auto find = [&](int32_t step) {
          const int32_t t = token_of(step);
          if (lane >= boxes || step >= n || t >= end || t + size <= begin) return -1;
          const int32_t page = pages[c.by_page.div(t)];
          return (uint32_t)page < (uint32_t)c.n_pages ? page : INT32_MAX;  // INT32_MAX: none such
        };
        int32_t before = -1, page = -1, next = find(0);
        if (KIND == P2P_KV_E4M3 && maps.rows) {
          // In 8 bits into room of the warp's own by the tensor memory accelerator, two steps ahead; widened from
          // there.
          constexpr int kLanes = DP == 64 ? 4 : DP == 128 ? 8 : 16, kAtOnce = 32 / kLanes;
          const int piece = lane % kLanes;
          char* const raw = raws + (warp - S::kSoft) * (S::kRaw / 4);
          const int size_log = __ffs(size) - 1;
          // Steps by turns into two places each of keys and of values; a lane keeps its box's pages of four steps.
          const auto fetch = [&](int32_t step, int32_t from, int v) {
            const bool there = step < n && from >= 0 && from != INT32_MAX;
            if (step < n && from == INT32_MAX) atomicOr(w.err, KV_BAD_PAGE);
            const uint32_t which = __ballot_sync(~0u, there);
            if (step < n) {
              const int slot = 2 * v + (step & 1);
              if (lane == 0) bar_expect(sh.raw[warp - S::kSoft][slot], __popc(which) * size * c.dim);
              __syncwarp();
              const int32_t t = token_of(step);
              if (there)
                copy_box(smem_of(raw) + slot * S::kRaw + lane * size * c.dim, v ? &maps.v : &maps.k, 0,
                         t - (int32_t)c.by_page.div(t) * c.page, u.h, from, a.layer, sh.raw[warp - S::kSoft][slot]);
            }
          };
          int32_t p0 = next, p1 = find(1), p2 = find(2), p3 = find(3);
          const auto page_of = [&](int32_t step) { return step & 2 ? (step & 1 ? p3 : p2) : step & 1 ? p1 : p0; };
#pragma unroll
          for (int k = 0; k < 2; ++k) fetch(k, page_of(k), 0), fetch(k, page_of(k), 1);
#pragma unroll 1
          for (int32_t q = 0; q < 2 * n; ++q) {
            const RowsStage it = rows_stage(q, n, split);
            const int v = it.values, step = it.step, slot = 2 * v + (step & 1);
            const int32_t his = page_of(step);
            const uint32_t here = __ballot_sync(~0u, his >= 0 && his != INT32_MAX);
            if (!bar_wait(sh.raw[warp - S::kSoft][slot], raw_phase >> slot & 1, sh) ||
                !bar_wait(sh.empty[stage], phase, sh)) return;
            raw_phase ^= 1u << slot;
            // The warp's tokens that are there.
            const int32_t t = (j0 + step) * kBt + own0 + lane;
            const uint32_t rows = __ballot_sync(~0u, lane < kOwn && t >= begin && t < end &&
                (here >> (lane >> size_log) & 1));
            char* const to = stages + stage * S::kStage + (piece / 4) * (kBt * 128) + own0 * 128;
            const char* const his_raw = raw + slot * S::kRaw + piece * 16;
            if (piece < 4 * chunks) {
#pragma unroll
              for (int x = 0; x < kOwn; x += kAtOnce) {
                const int row = x + lane / kLanes;
                uint4 y = *(const uint4*)(his_raw + row * c.dim);
                if (piece >= c.row16 || !(rows >> row & 1)) y = make_uint4(0, 0, 0, 0);
                *(uint4*)(to + row * 128 + ((2 * piece & 7) ^ (row & 7)) * 16) =
                    make_uint4(widen(y.x), widen_high(y.x), widen(y.y), widen_high(y.y));
                *(uint4*)(to + row * 128 + (((2 * piece & 7) + 1) ^ (row & 7)) * 16) =
                    make_uint4(widen(y.z), widen_high(y.z), widen(y.w), widen_high(y.w));
              }
            }
            async_fence();
            bar_arrive(sh.full[stage]);
            if (++stage == kStages) stage = 0, phase ^= 1;
            __syncwarp();
            fetch(step + 2, page_of(step + 2), v);
            if (v) {  // (the values come last: the step's page is not needed any more)
              const int32_t later = find(step + 4);
              p0 = (step & 3) == 0 ? later : p0, p1 = (step & 3) == 1 ? later : p1;
              p2 = (step & 3) == 2 ? later : p2, p3 = (step & 3) == 3 ? later : p3;
            }
          }
        } else {
#pragma unroll 1
          for (int32_t q = 0; q < 2 * n; ++q) {
            const RowsStage it = rows_stage(q, n, split);
            const int v = it.values, step = it.step;
            if (!v) before = page, page = next, next = find(step + 1);
            const int32_t from = v && split && step < n - 1 ? before : page, t = token_of(step);
            const bool there = from >= 0 && from != INT32_MAX;
            if (from == INT32_MAX) atomicOr(w.err, KV_BAD_PAGE);
            const int32_t in_page = there ? t - (int32_t)c.by_page.div(t) * c.page : 0;
            const uint32_t holes = __ballot_sync(~0u, from == INT32_MAX);
            const uint32_t bytes = __popc(__ballot_sync(~0u, there)) * size * 128 * chunks;
            char* const to = stages + stage * S::kStage;
            if (!bar_wait(sh.empty[stage], phase, sh)) return;
            if (KIND != P2P_KV_E4M3 && maps.rows) {
              // By the tensor memory accelerator; zeros in the place of pages that are out of range.
              for (uint32_t left = holes; left; left &= left - 1) {
                const int first = (own0 + (__ffs(left) - 1) * size) * 128;
                for (int y = lane; y < size * chunks * 8; y += 32)
                  *(uint4*)(to + y / (size * 8) * (kBt * 128) + first + y % (size * 8) * 16) = make_uint4(0, 0, 0, 0);
              }
              if (holes) async_fence();
              __syncwarp();
              if (lane == 0) bar_expect(sh.full[stage], bytes);
              __syncwarp();
              if (there)
#pragma unroll
                for (int x = 0; x < S::kChunks; ++x)
                  if (x < chunks) copy_box(smem_of(to) + x * (kBt * 128) + (own0 + lane * size) * 128, v ? &maps.v
                      : &maps.k, x * 64, in_page, u.h, from,
                           a.layer, sh.full[stage]);
            } else {
              const int64_t at = there && t >= begin ? (v ? across : 0) + from * c.page_stride +
                  (int64_t)in_page * c.token_stride : -1;
              const bool some = there && t >= begin;
              if (KIND != P2P_KV_E4M3) {
                constexpr int kLanes = DP == 64 ? 8 : DP == 128 ? 16 : 32, kAtOnce = 32 / kLanes;
                const int piece = lane % kLanes;
                const uint32_t rows_there = __ballot_sync(~0u, some), tile_at = smem_of(to) + (piece / 8) * (kBt * 128);
                // (Places four at a time: one by one, each copy waits for its exchange.)
#pragma unroll 1
                for (int x0 = 0; x0 < kOwn; x0 += 4 * kAtOnce) {
                  int64_t o[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) o[k] = __shfl_sync(~0u, at, (x0 + k * kAtOnce + lane / kLanes) & 31);
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    const int row = x0 + k * kAtOnce + lane / kLanes, in_tile = own0 + row;
                    const bool in = row < kOwn && (rows_there >> row & 1) && piece < c.row16;
                    const char* const his = in ? base + o[k] + piece * 16 : c.k;
                    if (piece < 8 * chunks && row < kOwn) copy16(tile_at + in_tile * 128 +
                        ((piece & 7) ^ (in_tile & 7)) * 16, his, in);
                  }
                }
                // (Arrives when the thread's copies have; whoever reads them through another path fences after it has
                // waited.)
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_of(&sh.full[stage]))
                    : "memory");
              } else {
                // 16 values a piece; widened on the way.
                constexpr int kLanes = DP == 64 ? 4 : DP == 128 ? 8 : 16, kAtOnce = 32 / kLanes;
                const int piece = lane % kLanes;
                const uint32_t rows_there = __ballot_sync(~0u, some);
                uint4 b[kOwn / kAtOnce];
#pragma unroll
                for (int x = 0; x < kOwn; x += kAtOnce) {
                  const int row = x + lane / kLanes;
                  const int64_t o = __shfl_sync(~0u, at, row);
                  b[x / kAtOnce] = make_uint4(0, 0, 0, 0);
                  if ((rows_there >> row & 1) && piece < c.row16) b[x / kAtOnce] =
                      __ldcg((const uint4*)(base + o + piece * 16));
                }
                char* const tile_at = to + (piece / 4) * (kBt * 128);
#pragma unroll
                for (int x = 0; x < kOwn; x += kAtOnce) {
                  const int row = own0 + x + lane / kLanes;
                  const uint4 y = b[x / kAtOnce];
                  if (piece < 4 * chunks) {
                    *(uint4*)(tile_at + row * 128 + ((2 * piece & 7) ^ (row & 7)) * 16) =
                        make_uint4(widen(y.x), widen_high(y.x), widen(y.y), widen_high(y.y));
                    *(uint4*)(tile_at + row * 128 + (((2 * piece & 7) + 1) ^ (row & 7)) * 16) =
                        make_uint4(widen(y.z), widen_high(y.z), widen(y.w), widen_high(y.w));
                  }
                }
                async_fence();
                bar_arrive(sh.full[stage]);
              }
            }
            if (++stage == kStages) stage = 0, phase ^= 1;
          }
        }
        __syncwarp();
        if (lane == 0) bar_arrive(sh.unit_empty[ring]);
        next_unit();
      }
    };
    run();
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (*(volatile int32_t*)&sh.dead) {  // (copies that are still on their way)
      for (int i = 0; i < kStages; ++i) bar_drain(sh.full[i], i < stage ? phase ^ 1 : phase);
      for (int v = 0; v < 4; ++v) bar_drain(sh.raw[warp - S::kSoft][v], raw_phase >> v & 1);
    }
  } else if (warp == S::kSoft + 4) {
    // ================================ products
    if (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    {
      const uint32_t one = elected();
      const uint32_t type = KIND == P2P_KV_BF16 ? 1u : 0u;
      const uint32_t what = 1u << 4 | type << 7 | type << 10 | 8u << 24;  // sums in 32 bits, 128 rows
      const uint32_t qk = what | (uint32_t)(kBt / 8) << 17, pv = what | 1u << 16 | (uint32_t)(dim16 / 8) << 17;
      const uint32_t q_at = smem_of(q_room), stage_at = smem_of(stages);
      int32_t stage = 0;
      uint32_t phase = 0, q_phase[2] = {0, 0}, p_phase = 0;
      const auto next_stage = [&]() {
        if (++stage == kStages) stage = 0, phase ^= 1;
      };
      const auto logits = [&](int tile, int at_stage, bool last) {
        const uint64_t q0 = matrix(q_at + tile * S::kQTile, 16), k0 = matrix(stage_at + at_stage * S::kStage, 16);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          if (k * 16 < dim16)
            mma_ss(tmem + tile * kBt, q0 + ((k / 4) * (128 * 128) + (k & 3) * 32) / 16,
                   k0 + ((k / 4) * (kBt * 128) + (k & 3) * 32) / 16, qk, k > 0, one);
        mma_done(sh.s_full[tile], one);
        if (last) mma_done(sh.q_empty[tile], one);
      };
      int32_t all_begin = 0, all_end = 0;
      // The values of step j, at the current stage.
      const auto values_there = [&](int32_t j) {
        if (!bar_wait_lane(sh.full[stage], phase, sh)) return false;
        if (!seen_by_all<kBt>(j, all_begin, all_end) && !bar_wait_lane(sh.checked[stage], phase, sh)) return false;
        async_fence();
        return true;
      };
      const auto add_values = [&](int tile, int at_stage, bool add, bool last) {
        if (!bar_wait_lane(sh.p_full[tile], p_phase >> tile & 1, sh)) return false;
        p_phase ^= 1u << tile;
        after_sync();
        const uint64_t v0 = matrix(stage_at + at_stage * S::kStage, kBt * 128);
#pragma unroll
        for (int k = 0; k < kBt / 16; ++k)
          mma_ts(tmem + S::kOCol + tile * DP, tmem + tile * kBt + 8 * k, v0 + k * (2048 / 16), pv, add || k > 0, one);
        if (last) mma_done(sh.o_full[tile], one);
        return true;
      };
      // (Its lanes wait each for itself, without a vote: nothing here needs them all, and the one that issues drains at
      // the end.)
      const auto run = [&]() {
        for (;;) {
          if (!bar_wait_lane(sh.unit_full[ring], ring_phase, sh)) return;
          const RowsUnit& u = sh.unit[ring];
          if (u.rows == 0) return;
          const int32_t j0 = u.j0, j1 = u.j1;
          const bool split = u.split;
          all_begin = u.all_begin, all_end = u.all_end;
          int32_t t0[2], t1[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) t0[i] = u.t0[i], t1[i] = u.t1[i];
#pragma unroll
          for (int i = 0; i < kTiles; ++i)
            if (t1[i] > t0[i]) {
              if (!bar_wait_lane(sh.q_full[i], q_phase[i], sh)) return;
              q_phase[i] ^= 1;
              async_fence();
            }
          if (one) bar_arrive(sh.unit_empty[ring]);
          next_unit();
          if (!bar_wait_lane(sh.full[stage], phase, sh)) return;
          async_fence();
          if (!split) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
              if (j0 >= t0[i] && j0 < t1[i]) logits(i, stage, j0 + 1 == t1[i]);
            mma_done(sh.empty[stage], one);
            next_stage();
#pragma unroll 1
            for (int32_t j = j0; j < j1; ++j) {
              if (!values_there(j)) return;
              const int v_stage = stage;
              next_stage();
              bool keys = j + 1 == j1;  // the next step's are there (or there are none)
#pragma unroll
              for (int i = 0; i < kTiles; ++i) {
                if (j >= t0[i] && j < t1[i] && !add_values(i, v_stage, j > t0[i], j + 1 == t1[i])) return;
                if (j + 1 < j1 && j + 1 >= t0[i] && j + 1 < t1[i]) {
                  if (!keys) {
                    if (!bar_wait_lane(sh.full[stage], phase, sh)) return;
                    async_fence();
                    keys = true;
                  }
                  logits(i, stage, j + 2 == t1[i]);
                }
              }
              mma_done(sh.empty[v_stage], one);
              if (j + 1 < j1) {
                if (!keys && !bar_wait_lane(sh.full[stage], phase, sh)) return;
                mma_done(sh.empty[stage], one);
                next_stage();
              }
            }
          } else if (kTiles == 2) {
            // The tiles take turns with the steps.
            const int32_t n = j1 - j0;
            logits(0, stage, n <= 2);
            mma_done(sh.empty[stage], one);
            next_stage();
            if (n > 1) {
              if (!bar_wait_lane(sh.full[stage], phase, sh)) return;
              async_fence();
              logits(1, stage, n <= 3);
              mma_done(sh.empty[stage], one);
              next_stage();
            }
#pragma unroll 1
            for (int32_t x = 0; x < n; ++x) {
              const int i = x & 1;
              if (!values_there(j0 + x) || !add_values(i, stage, x > 1, x + 2 >= n)) return;
              mma_done(sh.empty[stage], one);
              next_stage();
              if (x + 2 < n) {
                if (!bar_wait_lane(sh.full[stage], phase, sh)) return;
                async_fence();
                logits(i, stage, x + 4 >= n);
                mma_done(sh.empty[stage], one);
                next_stage();
              }
            }
          }
        }
      };
      run();
      mma_done(sh.drain, one);
      bar_drain(sh.drain, 0);
    }
    __syncwarp();
  } else if (warp == S::kSoft + 5) {
    // ================================ schedule: the units of this CTA's share
    if (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const long long patience = a.patience < 0 ? -a.patience : a.patience;
    const auto emit = [&](const RowsUnit& u) {
      if (!bar_watch(sh.unit_empty[ring], ring_phase ^ 1, sh, patience)) return false;
      if (lane == 0) {
        sh.unit[ring] = u;
        sh.poison[ring] = 0;
        bar_arrive(sh.unit_full[ring]);
      }
      __syncwarp();
      next_unit();
      return true;
    };
    // floor(total * k / ctas) for this CTA and the next.
    const uint32_t whole = total / ctas, rest = total - whole * ctas;
    const uint32_t x0 = whole * blockIdx.x + rest * blockIdx.x / ctas, x1 = whole * (blockIdx.x + 1) +
        rest * (blockIdx.x + 1) / ctas;
    // The first row's member (token) and head move by these from tile to tile, and to a tile's second half.
    const int32_t unit = kTiles * a.tile_rows, tile_t = a.by_group.div(unit), tile_g = unit - tile_t * a.group;
    const int32_t half_t = a.by_group.div(a.tile_rows), half_g = a.tile_rows - half_t * a.group;
    // The warp that summed the item where the share begins, and where its items begin.
    uint32_t x = of_warp;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t y = __shfl_up_sync(~0u, x, d);
      if (lane >= d) x += y;
    }
    const int from = __ffs(__ballot_sync(~0u, x0 < x)) - 1;
    x = __shfl_sync(~0u, x - of_warp, from);
    bool alive = true, found = false;
    KvJoin join = {};  // the unit that the next CTA goes on with
    // 32 items at a time, a lane each.
#pragma unroll 1
    for (int32_t i0 = from * per_warp; alive && x < x1 && i0 < a.n; i0 += 32) {
      if (i0 > 0 || per_warp > 32) {  // (else they are still there)
        own = {}, own_cost = 0;
        bool unused = false;
        if (i0 + lane < a.n) own = rows_item<S>(c, a, i0 + lane, nullptr, unused);
        if (own.tiles) own_cost = rows_cost<S>(a, own).of(own.tiles);
      }
#pragma unroll 1
      for (uint32_t some = __ballot_sync(~0u, own.tiles > 0); some && alive && x < x1; some &= some - 1) {
        const int l = __ffs(some) - 1;
        const uint32_t all = __shfl_sync(~0u, own_cost, l);
        if (!found && x0 - x >= c.heads * all) {
          x += c.heads * all;
          continue;
        }
        RowsItem it;
        it.row0 = __shfl_sync(~0u, own.row0, l);
        it.members = __shfl_sync(~0u, own.members, l), it.tiles = __shfl_sync(~0u, own.tiles, l);
        it.seq = __shfl_sync(~0u, own.seq, l), it.pos = __shfl_sync(~0u, own.pos, l);
        it.shared = __shfl_sync(~0u, own.shared, l), it.first = __shfl_sync(~0u, own.first, l);
        const RowsCost costs = rows_cost<S>(a, it);
        int32_t h = 0, j = 0;
        uint32_t cost = 0;
        if (!found) {  // the head and tile where the share begins
          found = true;
          uint32_t in = x0 - x;
          h = (int32_t)(in / all);
          in -= h * all;
          int32_t past = it.tiles;
#pragma unroll 1
          while (past - j > 1) {
            const int32_t mid = j + ((past - j) >> 1);
            const uint32_t y = costs.of(mid);
            if (y <= in)
              j = mid, cost = y;
            else
              past = mid;
          }
        }
        const uint32_t x_next = x + c.heads * all;
        x += h * all + cost;
        int32_t t = a.by_group.div(j * unit), g0 = j * unit - t * a.group;
#pragma unroll 1
        while (alive && x < x1) {
          const uint32_t cost1 = costs.of(j + 1), width = cost1 - cost;
          const int32_t rows = min(unit, it.members * a.group - j * unit);
          // The next tile's first row, and the second half's.
          int32_t t_next = t + tile_t, g_next = g0 + tile_g, t_half = t + half_t, g_half = g0 + half_g;
          if (g_next >= a.group) g_next -= a.group, ++t_next;
          if (g_half >= a.group) g_half -= a.group, ++t_half;
          const int32_t t_last = min(g_next ? t_next : t_next - 1, it.members - 1);
          const RowsSpan span = rows_span(a, it, t, t_last);
          const int32_t j0 = span.begin >> S::kBtLog, n = ((span.end - 1) >> S::kBtLog) + 1 - j0;
          // A share that begins at x + kRowsSet + 1 .. x + inside - 1 begins within the unit, at this step of it:
          const uint32_t inside = min(width, (uint32_t)((n - 1) >> a.count.shift) + 1 + kRowsSet);
          const auto step = [&](uint32_t y) {
            return y <= x + kRowsSet ? 0 : y - x >= inside ? n : (int32_t)((y - x - kRowsSet) << a.count.shift);
          };
          const int32_t s0 = step(x0), s1 = step(x1);
          if (s1 > s0) {
            RowsUnit u;
            u.row = it.row0 + t;
            u.g0 = g0;
            u.rows = rows;
            u.h = h;
            u.seq = it.seq;
            u.pos = it.pos + t;
            u.begin = span.begin, u.end = span.end, u.all_begin = span.all_begin, u.all_end = span.all_end;
            u.j0 = j0 + s0, u.j1 = j0 + s1;
            u.t0[0] = u.t1[0] = u.t0[1] = u.t1[1] = u.j0;
            {
              const RowsSpan its = rows_span(a, it, t, rows <= a.tile_rows ? t_last : g_half ? t_half : t_half - 1);
              u.t0[0] = max(u.j0, its.begin >> S::kBtLog);
              u.t1[0] = max(u.t0[0], min(u.j1, ((its.end - 1) >> S::kBtLog) + 1));
            }
            if (kTiles == 2 && rows > a.tile_rows) {
              const RowsSpan its = rows_span(a, it, t_half, t_last);
              u.t0[1] = max(u.j0, its.begin >> S::kBtLog);
              u.t1[1] = max(u.t0[1], min(u.j1, ((its.end - 1) >> S::kBtLog) + 1));
            }
            u.split = 0;
            if (kTiles == 2 && rows <= a.tile_rows && s1 - s0 >= kSplitSteps) {
              u.split = 1;
              u.t0[0] = u.j0, u.t0[1] = u.j0 + 1;
              u.t1[0] = u.t1[1] = u.j1;
            }
            u.parts = 1, u.part = 0, u.c0 = blockIdx.x;
            if (s1 - s0 < n) {
              // The first shares that begin within the unit, and after it, by a lane each: the first k with total * k
              // >= y * ctas.
              const uint32_t y = x + (lane & 1 ? inside : kRowsSet + 1);
              uint32_t k = (uint32_t)__fdividef((float)y * (float)ctas, (float)total);
              k = k > 1 ? k - 1 : 0;
              while ((uint64_t)k * total < (uint64_t)y * ctas) ++k;
              const uint32_t first = __shfl_sync(~0u, k, 0), end = __shfl_sync(~0u, k, 1);
              u.c0 = (int32_t)first - 1;
              u.parts = (int32_t)(end - first) + 1;
              u.part = blockIdx.x - u.c0;
              if (u.part == 0) join = {u.row, u.rows, u.g0, u.h, u.parts};
            }
            alive = emit(u);
          }
          x += width;
          cost = cost1;
          t = t_next, g0 = g_next;
          if (++j < it.tiles) continue;
          j = 0, cost = 0, t = 0, g0 = 0;
          if (++h == c.heads) break;
        }
        if (x < x1) x = x_next;
      }
    }
    if (lane == 0) w.joins[blockIdx.x] = join;
    if (alive && a.patience >= 0) {  // (else the others wait for a word that never comes: see p2p_kv_set_patience)
      RowsUnit u = {};
      alive = emit(u);
    }
    if (alive) bar_watch(sh.done, 0, sh, patience);
  } else {
    // ================================ infinities and NaN among values that not all rows see
    if (kTiles == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    const int mine = (warp - S::kSoft - 6) * 32 + lane;
    int32_t stage = 0;
    uint32_t phase = 0, q_phase = 3;  // (of fresh barriers: the last phases count as done)
    const auto run = [&]() {
      for (;;) {
        if (!bar_wait(sh.unit_full[ring], ring_phase, sh)) return;
        const RowsUnit& u = sh.unit[ring];
        if (u.rows == 0) return;
        // The unit's queries, when the products with the last one's are done.
#pragma unroll 1
        for (int i = 0; i < kTiles; ++i) {
          if (u.t1[i] <= u.t0[i]) continue;
          if (!bar_wait(sh.q_empty[i], q_phase >> i & 1, sh)) return;
          q_phase ^= 1u << i;
          const uint64_t& there = direct ? sh.q_full[i] : sh.q_raw[i];
          const int first = u.split ? 0 : i * a.tile_rows;
          char* const to = q_room + i * S::kQTile;
          // (Where one helper brings all, the other arrives as well, so that neither misses a phase of q_empty.)
          if (a.boxes) {  // whole tokens
            if (mine == 32) bar_arrive(there);
            if (mine == 0) {
              bar_expect(there, a.tile_rows * 128 * chunks);
              for (int x = 0; x < chunks; ++x)
                copy_query_box(smem_of(to) + x * (128 * 128), &q_map, x * 64, u.h,
                    (int32_t)(u.row + a.by_group.div(first)), there);
            }
            continue;
          }
          // From anywhere, a piece of 16 bytes a thread.
          const int pieces = dim16 / 8;
#pragma unroll 1
          for (int y = mine; y < 128 * pieces; y += 64) {
            const int x = y / pieces, piece = y - x * pieces;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (first + x < u.rows && x < a.tile_rows && piece * 8 < c.dim) {
              const uint32_t z = u.g0 + first + x, t = a.by_group.div(z);
              const uint16_t* const f =
                  (const uint16_t*)a.q + (u.row + t) * a.q_row +
                      (u.h * a.group + (int32_t)(z - t * a.group)) * a.q_head + piece * 8;
              v = make_uint4(f[0] | f[1] << 16, f[2] | f[3] << 16, f[4] | f[5] << 16, f[6] | f[7] << 16);
            }
            *(uint4*)(to + piece / 8 * (128 * 128) + x * 128 + ((piece & 7) ^ (x & 7)) * 16) = v;
          }
          async_fence();
          bar_arrive(there);
        }
        const int32_t n = u.j1 - u.j0;
#pragma unroll 1
        for (int32_t q = 0; q < 2 * n; ++q) {
          const RowsStage it = rows_stage(q, n, u.split);
          const int32_t j = u.j0 + it.step;
          if (!bar_wait(sh.full[stage], phase, sh)) return;
          if (it.values && !seen_by_all<kBt>(j, u.all_begin, u.all_end)) {
            // An exponent of all ones carries into the sign's place.
            constexpr uint32_t kExponent = KIND == P2P_KV_BF16 ? 0x7f807f80u : 0x7c007c00u, kOne = KIND == P2P_KV_BF16
                ? 0x00800080u : 0x04000400u;
            char* const tile = stages + stage * S::kStage;
            // the rows that are somebody's
            const int32_t first = max(u.begin - j * kBt, 0), end = min(u.end - j * kBt, kBt);
            for (int x = mine; x < (kBt - (end - first)) * 8; x += 64) {  // (the others hold whatever lay there)
              const int row = x / 8 < first ? x / 8 : x / 8 - first + end;
              for (int k = 0; k < S::kChunks; ++k) *(uint4*)(tile + k * (kBt * 128) + row * 128 + (x & 7) * 16) =
                  make_uint4(0, 0, 0, 0);
            }
            uint32_t ends = 0;
#pragma unroll 1
            for (int k = 0; k * 64 < dim16; ++k)
#pragma unroll 4
              for (int x = mine; x < kBt * 8; x += 64) {
                const uint4 v = *(const uint4*)(tile + k * (kBt * 128) + x * 16);
                const uint32_t some = ((v.x & kExponent) + kOne) | ((v.y & kExponent) + kOne) | ((v.z & kExponent) +
                    kOne) |
                                      ((v.w & kExponent) + kOne);
                const int row = x >> 3;
                if (row >= first && row < end) ends |= some;
              }
            bool found = false;
            if (ends & 0x80008000u) {
              for (int k = 0; k * 64 < dim16; ++k)
                for (int x = mine; x < kBt * 8; x += 64) {
                  const int row = x >> 3;
                  if (row < first || row >= end) continue;
                  uint4* const p = (uint4*)(tile + k * (kBt * 128) + x * 16);
                  const uint4 v = *p;
                  uint32_t b[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                  for (int y = 0; y < 4; ++y) {
                    const uint32_t bad = ((b[y] & kExponent) + kOne) & 0x80008000u;
                    b[y] &= ~((bad >> 15) * 0xffffu);
                  }
                  *p = make_uint4(b[0], b[1], b[2], b[3]);
                }
              found = true;
            }
            if (found) sh.poison[ring] = 1;
            async_fence();
          }
          __syncwarp();
          // (A stage is free when the products and both helpers are done with it: one that fell a turn behind would take
          // phases for one another.)
          if (lane == 0) bar_arrive(sh.checked[stage]), bar_arrive(sh.empty[stage]), ++*(volatile int32_t*)&sh.signs;
          if (++stage == kStages) stage = 0, phase ^= 1;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(sh.unit_empty[ring]);
        next_unit();
      }
    };
    run();
    if (*(volatile int32_t*)&sh.dead)  // (queries that are still on their way)
      for (int i = 0; i < kTiles; ++i) bar_drain(direct ? sh.q_full[i] : sh.q_raw[i], q_phase >> i & 1);
  }
  __syncwarp();
  if (warp != S::kSoft + 5 && lane == 0) bar_arrive(sh.done);
  __syncthreads();
  if (sh.dead && threadIdx.x == 0) atomicOr(w.err, KV_STUCK);
  if (warp == S::kSoft + 4)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// With a = NULL the kernel is only made ready for launches.
template <int KIND, int DP>
cudaError_t launch_rows(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w, int num_sms,
    cudaStream_t st) {
  using S = RowsShape<KIND, DP>;
  const auto kernel = rows_kernel<KIND, DP>;
  if (!a) {
    cudaFuncAttributes got;
    cudaError_t e = cudaFuncGetAttributes(&got, kernel);
    // (The softmax warps take 56 registers a thread more, which the others give back: of 128 that each starts with.)
    if (e == cudaSuccess && S::kTiles == 2 && got.numRegs != 128) e = cudaErrorInvalidDeviceFunction;
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
  }
  return launch_early(kernel, dim3(num_sms), S::kThreads, S::kBytes, st, c, m, a->q_map ? *a->q_map : m.k, *a, w);
}
template <int KIND>
cudaError_t launch_rows_dim(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w,
    int num_sms,
                            cudaStream_t st) {
  return c.dim <= 64    ? launch_rows<KIND, 64>(c, m, a, w, num_sms, st)
         : c.dim <= 128 ? launch_rows<KIND, 128>(c, m, a, w, num_sms, st)
         : c.dim <= 192 ? launch_rows<KIND, 192>(c, m, a, w, num_sms, st)
                        : launch_rows<KIND, 256>(c, m, a, w, num_sms, st);
}

}  // namespace
}  // namespace p2p
