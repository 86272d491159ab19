// kv_attend.cuh -- attention of one new token a sequence over the paged key-value cache (p2p_kv_attend).
//
// For a query head and the tokens t that it sees: x_t = scale * q . k_t, m = max x_t, z = sum exp(x_t - m), out = sum
// exp(x_t - m) v_t / z, lse = m + ln z; without a token, out = 0 and lse = -inf.
//
// Keys and values are read once, and that is what bounds it: with g query heads a kv head, 4 g dim operations go with
// 4 dim bytes, g a byte (2 g with 8 bits), where the GPU has 277 operations of its tensor cores for a byte of memory.
// Measured on one GB300 (device time in a graph; copy bandwidth 6.8 TB/s): 32 sequences of 4,352 to 33,792 tokens, 40
// / 8 heads of 128 f16 values, 1.88 GB in 282 us (98%); one sequence of 131,071 tokens, 32 / 8 heads, 0.54 GB in 86 us
// (92%); 256 sequences of 128 to 4,224 tokens in 8 bits, 64 / 8 heads, 0.62 GB in 104 us (88%: there the widening of
// the values and the ends of the rows weigh); one of 540 tokens 7.6 us, a chain of a launch, four loads, a tile and
// the join.
//
// The work is cut into units of 64 or 128 tokens (2^kTileLog) of a (sequence, kv head, block of its query heads), or,
// where that pays (SIDE), of 2^side times fewer tokens of 2^side neighbouring kv heads, numbered in that order, and
// every CTA takes an equal, contiguous range of them: one long sequence fills the GPU as a batch does.  A range's
// parts of a unit row that it shares with other CTAs go to scratch (maximum, sum, unnormalised out), and the CTA that
// finishes such a row last joins its parts, in their order: results do not depend on timing.  (The start of a unit row
// counts as kOver units more, for what its end costs: with 1 instead of 3, the 256 sequences in 8 bits take 115 us.)
//
// Each warp streams 16 or 32 tokens at a time through shared memory of its own, up to seven tiles ahead (cp.async, 16
// bytes a lane, 16-byte pieces turned so that ldmatrix meets no bank twice), with no barrier between warps inside a
// unit row; the copies run on into the next unit row while this one's parts are joined.  Where pages are whole
// sixteens of tokens, a lane looks up the page of a whole tile ahead, for 32 tiles at once; else each token's is
// looked up two tiles ahead.  Sixteen tokens are multiplied transposed: S^T [tokens, heads] = K Q^T and O^T [dim,
// heads] += V^T P^T, so that eight query heads fill a product's n and the tokens (or values) its m of 16.  P^T goes
// from the first product's layout to the second's by two 8 x 8 transposes of registers.  exp(x - m) takes for m not
// the running maximum but one that lags it by at most a factor of 2^8 (2^3 for f16 and 8 bits), so that a tile's
// maximum is only reduced, and O rescaled, where it goes past that.  P is rounded to the values' type (f16 for 8 bits)
// for its product; sums, maxima and O are held in 32 bits.  Of f16, whose range is small, P takes the upper end (kUp):
// what is 2^26 times smaller than a warp's largest keeps all 11 bits, what is 2^37 times smaller is lost, 2^-37 of the
// largest a token at most.  (P <= 1 loses bits from 2^-14 on and everything below 2^-25, and then, where one token
// that is far ahead has values near zero, what the result consists of.)
//
// The products are warp-wide ones (mma): 9% of the tensor cores' time at the copy bandwidth (8 bits: 18%), and their
// operands come out of shared memory by ldmatrix in any row size.  The tensor memory path (tcgen05) would free issue
// slots that 16-bit values do not need and that 8-bit values, which have to be widened beside 16-bit queries, could
// not use it for.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "kv.h"

// (No load here goes past the coherent path, as __ldg or const __restrict__ would have it: the kernel before may
// still be writing when this one starts, see launch_early.)

namespace p2p {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kOver = 3;                // units that a unit row counts for beyond its own
constexpr int kJoin = 16;               // parts of a unit row that are read together
// Heads side by side (see SIDE), with so many units a CTA at least.  Where heads share lines of memory, with so many
// parts of a unit row at most, as joining that many more heads' parts takes longer than the lines save: 4 rows with 8
// heads of 192 8-bit values 50 us, not 24; 21 of 20,000 tokens with 4 of 96 16-bit values 86 and 74 (29 parts); 40 of
// 1,000 with 24 of 80 60, not 86.  Elsewhere, with so many units a row's head on average at most (kOver of them for
// starting it), as there are fewer unit rows to start and finish: 2,000 sequences of 1 to 200 tokens (half below 15)
// with 8 heads of 128 and 4 query heads to each take 78 us, with one head at a time 137, and 122 in the kernel without
// SIDE; in 8 bits 81, 168 and 158.  More query heads gain less, as parts grow with them: 1,000 of 1 to 500 (5 units)
// with 4 heads of 128 and 4, 8 or 16 query heads to each 41, 50 and 75, not 50, 56 and 80 (without SIDE 46, 50 and
// 71); 512 of 1 to 800 (5.6 units) with 8 of 256 and 4 or 8 96 and 140, not 120 and 136 (112 and 119).  Beyond, the
// parts cost as much or more: 512 of 1 to 1,200 with 8 of 256 and 8 171, not 153 (138).
constexpr int kSideUnits = 32, kSideParts = 16, kSideShort = 6;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// kUp: exp(x - m) is taken times 2^kUp (m is held less kUp, in log2).  kLag: how far (log2) a logit may pass the
// maximum in use.  P is at most 2^(kUp + kLag), which f16 has to hold.
template <int KIND>
struct Type;
template <>
struct Type<P2P_KV_BF16> {
  static constexpr float kUp = 0.f, kLag = 8.f;
};
template <>
struct Type<P2P_KV_F16> {
  static constexpr float kUp = 12.f, kLag = 3.f;
};
template <>
struct Type<P2P_KV_E4M3> {
  static constexpr float kUp = 12.f, kLag = 3.f;
};

// Sizes of the kernel for values of KIND, head_dim padded to DP, NB blocks of eight query heads.
template <int KIND, int DP, int NB>
struct Shape {
  static constexpr int kRowBytes = DP * attend_value_size(KIND);
  static constexpr int kPieces = kRowBytes / 16;               // 16-byte pieces of a row
  static_assert(kPieces % 2 == 0, "a tile's pieces are whole turns of the warp");
  // Tokens that a warp takes at a time: 32 of small 8-bit rows, where a turn of the loop costs much beside the bytes
  // it takes (256 sequences of 8-bit values of 64: 83 us with 16, 65 with 32).  Of 16-bit values of 64, 131,071
  // tokens take 49.3 and 47.9 us, but 512 sequences of 10 to 300 tokens 13.6 and 14.8: there smaller tiles fit rows
  // better.
  static constexpr int kRows = attend_rows(KIND, DP);
  static constexpr int kTileLog = kRows == 32 ? 7 : 6;         // (log2) that a CTA takes at a time, of one head
  static_assert(kWarps * kRows == 1 << kTileLog);
  static constexpr int kArray = kRows * kRowBytes;             // keys (or values) of a warp's tile
  static constexpr int kStage = 2 * kArray;
  static constexpr int kCtas = attend_ctas(KIND, DP, NB);
  static constexpr int kSumPitch = (DP + 31) / 32 * 32;        // of a head's sums, which lie in the room of a tile
  static_assert(8 * kSumPitch * 4 <= kStage);
  static constexpr int kFit = (232448 / kCtas - 1024 - 512) / kWarps / kStage;
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static constexpr int kRoom = kStages * kStage;               // a warp's tiles
  static constexpr int kBytes = kRoom * kWarps;                // of a CTA
  static constexpr int kHeads = 8 * NB;
  static_assert(kStages >= 2, "a tile on its way");
};

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void load4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void load4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// c [16, 8] += a [16, 16] b [16, 8]
template <int KIND>
__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  if (KIND == P2P_KV_BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ int32_t add_acq_rel(int32_t* p, int32_t x) {
  int32_t y;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(y) : "l"(p), "r"(x) : "memory");
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// ln of a sum of exp that was taken relative to t (in log2): near the largest term, where log2 is small.
template <int KIND>
__device__ __forceinline__ float log_sum(float t, float z) {
  constexpr float kUp = Type<KIND>::kUp, kDown = 1.f / (1 << (int)kUp);
  return (t + kUp + __log2f(z * kDown)) * kLn2;
}
template <int KIND>
__device__ __forceinline__ uint32_t pack(float a, float b) {
  if (KIND == P2P_KV_BF16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *(const uint32_t*)&x;
  }
  const __half2 x = __floats2half2_rn(a, b);
  return *(const uint32_t*)&x;
}
// Two 8-bit values (the low half of x) as two of 16.
__device__ __forceinline__ uint32_t widen(uint32_t x) {
  uint32_t y;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t widen_high(uint32_t x) {
  uint32_t y;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float2 two_halves(uint32_t x, int32_t type) {
  return type == P2P_KV_BF16 ? __bfloat1622float2(*(const __nv_bfloat162*)&x) : __half22float2(*(const __half2*)&x);
}
// Values d .. d + 3 of a head's result, times f; zero: 0 in their place.
__device__ __forceinline__ void store4(const KvView& c, const KvQuery& a, int32_t i, int32_t head, int32_t d, float4 v,
                                       float f, bool zero) {
  if (d >= c.dim) return;  // (dim is a multiple of 8)
  if (zero) v = make_float4(0.f, 0.f, 0.f, 0.f), f = 0.f;
  const uint32_t x = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(v.x * f, v.y * f) : pack<P2P_KV_F16>(v.x * f, v.y * f);
  const uint32_t y = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(v.z * f, v.w * f) : pack<P2P_KV_F16>(v.z * f, v.w * f);
  uint16_t* to = (uint16_t*)a.out + i * a.out_row + head * a.out_head + d;
  if (a.out_fours) {
    *(uint2*)to = make_uint2(x, y);
  } else {
    to[0] = (uint16_t)x, to[1] = (uint16_t)(x >> 16);
    to[2] = (uint16_t)y, to[3] = (uint16_t)(y >> 16);
  }
}

// Byte offset in a warp's tile of piece `piece` of row `row`: the pieces of eight rows that ldmatrix reads together lie
// in different banks (a turn by 1, 2 or all 3 low bits, as the rows' distance leaves them together).
template <int PIECES>
__device__ __forceinline__ uint32_t place(int row, int piece) {
  const int turn = PIECES % 8 == 0 ? row & 7 : PIECES % 4 == 0 ? (row >> 1) & 3 : (row >> 2) & 1;
  return (uint32_t)(row * PIECES + (piece ^ turn)) * 16;
}

// A row of the batch: it sees tokens begin .. end of its sequence; tiles are counted from `from`.
struct Row {
  int32_t seq, from, begin, end;
  // Units of 1 << tile_log tokens (one without any).
  __device__ __forceinline__ int32_t tiles(int32_t tile_log) const {
    return end > begin ? ((end - from - 1) >> tile_log) + 1 : 1;
  }
};
template <bool WHOLE>
__device__ __forceinline__ Row row_at(const KvView& c, const KvQuery& a, int32_t i, int32_t* err) {
  const bool there = i < a.n;
  const int32_t seq = there && a.seq ? a.seq[i] : there ? i : 0;
  const bool known = (uint32_t)seq < (uint32_t)c.n_seqs;
  const int32_t len = there && known ? c.length[seq] : 0;
  const bool fits = len >= 0 && len <= c.max_pages * c.page;
  if (err && !(known && fits)) atomicOr(err, known ? KV_BAD_COUNT : KV_BAD_SEQ);
  Row r = {known ? seq : 0, 0, 0, fits ? len : 0};
  r.begin = a.window && r.end > a.window ? r.end - a.window : 0;
  r.from = WHOLE ? r.begin / 16 * 16 : r.begin;
  return r;
}

struct Shared {
  int64_t sums[2][kWarps];
  int64_t before;  // units of the rows before `row` (over the kv heads and blocks of one)
  int32_t row, last, side;
  float top[kWarps][8], sum[kWarps][8];  // of the warps' parts, by head of a block
};

static_assert(sizeof(Shared) <= 512, "Shape counts on it");

// A place in a CTA's range: tile t of nt of the unit row (row i, kv head h, block of its query heads).
struct Cursor {
  Row row, next;
  int32_t i, h, block, t, nt;  // (h: the first of the unit's kv heads)
  int64_t left;  // units of the range from here on; none: at its end
  // k tiles on, none past the unit row's end.
  template <bool WHOLE>
  __device__ __forceinline__ void advance(int32_t k, const KvView& c, const KvQuery& a, int32_t blocks, int32_t side,
                                          int32_t tile_log) {
    t += k;
    left -= k;
    if (t < nt) return;
    t = 0;
    left -= kOver;
    if (++block < blocks) return;
    block = 0;
    h += 1 << side;
    if (h < c.heads) return;
    h = 0;
    ++i;
    row = next;
    nt = row.tiles(tile_log);
    next = row_at<WHOLE>(c, a, i + 1, nullptr);
  }
};

// SIDE: the warps of a CTA take 1 << c.side neighbouring kv heads where that pays (see kSideUnits), else one.  WHOLE:
// pages are whole sixteens of tokens, and tiles are counted from one: 16 tokens lie in one page, evenly apart.
template <int KIND, int DP, int NB, bool SIDE, bool WHOLE>
__global__ void __launch_bounds__(kThreads, Shape<KIND, DP, NB>::kCtas)
    attend_kernel(KvView c, KvQuery a, KvAttendScratch w) {
  using S = Shape<KIND, DP, NB>;
  constexpr int PIECES = S::kPieces, KSTEPS = DP / 16;
  extern __shared__ __align__(128) char room[];
  __shared__ Shared sh;
  begin_kernel();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tiles_at = smem_of(room + warp * S::kRoom);
  const int32_t group = a.heads / c.heads, blocks = (group + S::kHeads - 1) / S::kHeads;

  // ---- this CTA's range of the units: a thread sums those of consecutive rows, the CTA scans the threads' sums.
  const int32_t each = (a.n + kThreads - 1) / kThreads, r0 = threadIdx.x * each;
  int64_t mine[SIDE + 1] = {};  // with the heads side by side, and, last, without
  for (int32_t i0 = r0; i0 < r0 + each && i0 < a.n; i0 += 4) {
    Row r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      r[k] = row_at<WHOLE>(c, a, i0 + k < r0 + each ? i0 + k : a.n, blockIdx.x == 0 ? w.err : nullptr);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i0 + k < r0 + each && i0 + k < a.n) {
        mine[SIDE] += r[k].tiles(S::kTileLog) + kOver;
        if (SIDE) mine[0] += r[k].tiles(S::kTileLog - c.side) + kOver;
      }
  }
  int64_t scan[SIDE + 1], before = 0, all = 0;
#pragma unroll
  for (int x = 0; x <= SIDE; ++x) {
    scan[x] = mine[x];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(~0u, scan[x], d);
      if (lane >= d) scan[x] += y;
    }
    if (lane == 31) sh.sums[x][warp] = scan[x];
  }
  __syncthreads();
  int32_t side = 0;
  if (SIDE) {
    // (By one thread: where each decides for itself, the registers spill, up to 1 KB, and 256 sequences with 8 heads of
    // 96 8-bit values take 147 us, not 107.)
    if (threadIdx.x == 0) {
      int64_t units = 0;
#pragma unroll
      for (int k = 0; k < kWarps; ++k) units += sh.sums[SIDE][k];
      const int64_t grid = gridDim.x, unit_rows = (int64_t)a.n * (c.heads >> c.side) * blocks;
      const bool fit = c.lines ? unit_rows * kSideParts >= grid : units <= (int64_t)kSideShort * a.n;
      sh.side = fit && units * c.heads * blocks >= kSideUnits * grid ? c.side : 0;
    }
    __syncthreads();
    side = sh.side;
    if (side == 0) mine[0] = mine[SIDE], scan[0] = scan[SIDE];
  }
  const int32_t per_row = (c.heads >> side) * blocks;  // unit rows of a row
  // the warp's kv head and tokens of a unit
  const int32_t part_of_side = warp & ((1 << side) - 1), rank = warp >> side;
  const int32_t tile_log = S::kTileLog - side;
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    const int64_t of_warp = SIDE && side == 0 ? sh.sums[SIDE][k] : sh.sums[0][k];
    before += k < warp ? of_warp : 0;
    all += of_warp;
  }
  const int64_t total = all * per_row;
  // Two units a CTA at least: fewer parts to join (one sequence of 3,000 tokens with 8 kv heads: 11.0 us with one,
  // 10.0 with two).
  const int64_t ctas = max((int64_t)1, min((int64_t)gridDim.x, total / 2));
  if (blockIdx.x >= ctas) return;
  const int64_t x0 = total * blockIdx.x / ctas, x_end = total * (blockIdx.x + 1) / ctas;
  before += scan[0] - mine[0];
  const int64_t at = x0 / per_row;
  if (at >= before && at < before + mine[0]) {
    int32_t i = r0;
    for (;; ++i) {
      const int32_t t = row_at<WHOLE>(c, a, i, nullptr).tiles(tile_log) + kOver;
      if (at < before + t) break;
      before += t;
    }
    sh.row = i;
    sh.before = before;
  }
  __syncthreads();
  Cursor here;  // what is computed
  here.i = sh.row;
  here.row = row_at<WHOLE>(c, a, here.i, nullptr);
  here.next = row_at<WHOLE>(c, a, here.i + 1, nullptr);
  here.nt = here.row.tiles(tile_log);
  {
    const int64_t in = x0 - sh.before * per_row;
    const int32_t units = here.nt + kOver, pair = (int32_t)(in / units), u = (int32_t)(in % units);
    here.h = pair / blocks << side;
    here.block = pair % blocks;
    here.t = u > kOver ? u - kOver : 0;
    here.left = x_end - x0 - (u < kOver ? kOver - u : 0);
  }

  // ---- copies of the warp's tiles, in the order of the range.
  Cursor ahead = here;  // what is copied next, or, token by token, looked up next
  int32_t to_slot = 0;
  const auto next_slot = [&]() {
    const uint32_t to = tiles_at + to_slot * S::kStage;
    to_slot = to_slot + 1 < S::kStages ? to_slot + 1 : 0;
    return to;
  };
  const int64_t across = c.v - c.k, layer_at = (int64_t)a.layer * c.layer_stride + part_of_side * c.head_stride;
  // WHOLE: lane l has where the sixteens of tile near_t + l of row near_i lie (< 0: none); the kv heads of a row
  // share them.
  constexpr int SIXTEENS = S::kRows / 16;
  int64_t near[SIXTEENS];
  int32_t near_i = -1, near_t = 0;
  const auto step_whole = [&]() {
    if (ahead.left > 0) {
      if (ahead.i != near_i || (uint32_t)(ahead.t - near_t) >= 32u) {
        near_i = ahead.i, near_t = ahead.t;
#pragma unroll
        for (int m = 0; m < SIXTEENS; ++m) {
          const int64_t t = (int64_t)ahead.row.from + ((int64_t)(near_t + lane) << tile_log) + rank * S::kRows + 16 * m;
          near[m] = -1;
          if (t < ahead.row.end) {
            const uint32_t e = c.by_page.div((uint32_t)t);
            const int32_t page = c.table[(int64_t)ahead.row.seq * c.max_pages + e];
            if ((uint32_t)page < (uint32_t)c.n_pages)
              near[m] = page * c.page_stride + (int64_t)((uint32_t)t - e * (uint32_t)c.page) * c.token_stride;
            else
              atomicOr(w.err, KV_BAD_PAGE);
          }
        }
      }
      const uint32_t to = next_slot();
      const int64_t t0 = (int64_t)ahead.row.from + ((int64_t)ahead.t << tile_log) + rank * S::kRows;
      // rows lo .. lo + n - 1
      const int32_t lo = (int32_t)max(ahead.row.begin - t0, (int64_t)0);
      const int32_t n = (int32_t)(min(ahead.row.end - t0, (int64_t)S::kRows) - lo);
#pragma unroll
      for (int m = 0; m < SIXTEENS; ++m) {
        const int64_t o = __shfl_sync(~0u, near[m], ahead.t - near_t);
        const char* const base = c.k + (layer_at + ahead.h * c.head_stride + o);
#pragma unroll
        for (int y = 0; y < PIECES / 2; ++y) {  // the lane's y-th piece is the (lane + 32 y)-th of sixteen tokens'
          const int z = lane + 32 * y, r = z / PIECES, piece = z % PIECES;
          const bool in = o >= 0 && piece < c.row16 && 16 * m + r >= lo && 16 * m + r < lo + n;
          const char* from = in ? base + (r * c.token_stride + piece * 16) : c.k;
          const uint32_t d = to + m * 16 * S::kRowBytes + place<PIECES>(r, piece);
          copy16(d, from, in);
          copy16(d + S::kArray, from + across, in);
        }
      }
      ahead.advance<WHOLE>(1, c, a, blocks, side, tile_log);
    }
    commit();
  };
  // Otherwise a lane looks up a token: its page, and where it lies but for that (page < 0: no token), two tiles ahead.
  struct Token {
    int32_t page;
    int64_t at;
  };
  const auto look_up = [&]() {
    Token k = {-1, 0};
    if (ahead.left > 0) {
      const int64_t t = (int64_t)ahead.row.from + ((int64_t)ahead.t << tile_log) + rank * S::kRows +
          (lane & (S::kRows - 1));
      if (t < ahead.row.end) {
        const uint32_t e = c.by_page.div((uint32_t)t);
        k.page = c.table[(int64_t)ahead.row.seq * c.max_pages + e];
        k.at = layer_at + ahead.h * c.head_stride + (int64_t)((uint32_t)t - e * (uint32_t)c.page) * c.token_stride;
        if (k.page < 0) k.page = INT32_MAX;
      }
      ahead.advance<WHOLE>(1, c, a, blocks, side, tile_log);
    }
    return k;
  };
  Token soon = {-1, 0}, later = {-1, 0};
  const auto step = [&]() {
    if constexpr (WHOLE) {
      step_whole();
    } else {
      int64_t offset = -1;
      if (soon.page >= 0) {
        if (soon.page < c.n_pages)
          offset = soon.at + soon.page * c.page_stride;
        else
          atomicOr(w.err, KV_BAD_PAGE);
      }
      const uint32_t to = next_slot();
#pragma unroll
      for (int y = 0; y < S::kRows * PIECES / 32; ++y) {
        const int z = lane + 32 * y, r = z / PIECES, piece = z % PIECES;
        const int64_t o = __shfl_sync(~0u, offset, r);
        const bool in = o >= 0 && piece < c.row16;
        const char* from = c.k + (in ? o + piece * 16 : 0);
        const uint32_t d = to + place<PIECES>(r, piece);
        copy16(d, from, in);
        copy16(d + S::kArray, from + across, in);
      }
      commit();
      soon = later;
      later = look_up();
    }
  };
  if constexpr (!WHOLE) {
    soon = look_up();
    later = look_up();
  }

  // ---- the queries, as the second operand of the first product: lane holds head lane / 4 of each block of eight.
  // (With 8-bit values a piece of 16 is 16 of the product's k, in the order that their bytes come to a lane.)
  uint32_t q[KSTEPS][NB][2];
  float mul[NB][2];  // logit (in log2) of a sum, for the heads 2 * (lane % 4) + {0, 1} of a block
  const auto load_queries = [&](const Cursor& u) {
    const int32_t head0 = (u.h + part_of_side) * group + u.block * S::kHeads,
        heads = min(group - u.block * S::kHeads, S::kHeads);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int32_t head = b * 8 + lane / 4;
      const uint16_t* from = (const uint16_t*)a.q + u.i * a.q_row + (head0 + head) * a.q_head;
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int d = KIND == P2P_KV_E4M3 ? 16 * k + 4 * (lane % 4) + 2 * y : 16 * k + 8 * y + 2 * (lane % 4);
          uint32_t v = 0;
          if (head < heads && d < c.dim)
            v = a.q_pairs ? *(const uint32_t*)(from + d) : from[d] | (uint32_t)from[d + 1] << 16;
          q[k][b][y] = v;
        }
    }
  };
  const auto use_queries = [&](const Cursor& u) {
    float unit = a.scale * kLog2e * (KIND == P2P_KV_E4M3 ? c.k_scale[a.layer * c.heads + u.h + part_of_side] : 1.f);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float mine = unit;
      if (KIND == P2P_KV_E4M3) {
        // The queries in f16, scaled by a power of two so that a row's largest is in [2^14, 2^15): exact but for what
        // is below 2^-28 of it.  (In [1, 2) it would be 2^-14, and the upper half of f16's range of no use; sums of 256
        // products with up to 448 are far from the end of 32 bits either way.)
        float largest = 0.f;
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 v = two_halves(q[k][b][y], a.type);
            largest = fmaxf(largest, fmaxf(fabsf(v.x), fabsf(v.y)));
          }
        largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 1));
        largest = fmaxf(largest, __shfl_xor_sync(~0u, largest, 2));
        const int e = largest > 0.f && largest < INFINITY ? max(ilogbf(largest), -112) - 14 : 0;
        const float down = ldexpf(1.f, -e);
        mine = ldexpf(unit, e);
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 v = two_halves(q[k][b][y], a.type);
            q[k][b][y] = pack<KIND>(v.x * down, v.y * down);
          }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y) mul[b][y] = __shfl_sync(~0u, mine, 4 * (2 * (lane % 4) + y));
    }
  };

  load_queries(here);
#pragma unroll 1
  for (int j = 0; j < S::kStages - 1; ++j) step();
  int32_t slot = 0;

  while (here.left > 0) {
    use_queries(here);
    const Cursor u = here;  // the unit row, from its tile u.t on
    const int32_t count = (int32_t)(u.nt - u.t < u.left ? u.nt - u.t : u.left);
    const uint32_t first = (uint32_t)u.row.from + ((uint32_t)u.t << tile_log) + rank * S::kRows;
    float o[KSTEPS][NB][4], top[NB][2], sum[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      top[b][0] = top[b][1] = -INFINITY;
      sum[b][0] = sum[b][1] = 0.f;
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) o[k][b][0] = o[k][b][1] = o[k][b][2] = o[k][b][3] = 0.f;
    }

#pragma unroll 1
    for (int32_t j = 0; j < count; ++j) {
      wait<S::kStages - 2>();
      __syncwarp();  // every lane's pieces of tile j are there, and every lane is done with tile j - 1
      step();
      const uint32_t keys = tiles_at + slot * S::kStage, values = keys + S::kArray;
      slot = slot + 1 < S::kStages ? slot + 1 : 0;

      constexpr int MB = S::kRows / 16;
      float s[MB][NB][4] = {};  // of each sixteen: tokens lane / 4 (+ 8 in 2, 3), heads 2 * (lane % 4) + {0, 1}
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const uint32_t keys16 = keys + m * 16 * S::kRowBytes;
        if (KIND == P2P_KV_E4M3) {
#pragma unroll
          for (int k = 0; k < KSTEPS; k += 2) {
            uint32_t r[4];  // tokens 0-7 and 8-15 of piece k, then of piece k + 1
            load4(r, keys16 + place<PIECES>((lane & 7) + (lane >> 3 & 1) * 8, k + (lane >> 4)));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint32_t f[4] = {widen(r[2 * y]), widen(r[2 * y + 1]), widen_high(r[2 * y]),
                                     widen_high(r[2 * y + 1])};
#pragma unroll
              for (int b = 0; b < NB; ++b) multiply<KIND>(s[m][b], f, q[k + y][b]);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k) {
            uint32_t f[4];
            load4(f, keys16 + place<PIECES>((lane & 7) + (lane >> 3 & 1) * 8, 2 * k + (lane >> 4)));
#pragma unroll
            for (int b = 0; b < NB; ++b) multiply<KIND>(s[m][b], f, q[k][b]);
          }
        }
      }
      // The tile's tokens that are seen, if not all, and those before them that are not.
      const int32_t left = (int32_t)((uint32_t)u.row.end - (first + ((uint32_t)j << tile_log)));
      bool past = false;
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int y = 0; y < 4; ++y) s[m][b][y] *= mul[b][y & 1];
      const int32_t lead = WHOLE ? u.row.begin - (int32_t)(first + ((uint32_t)j << tile_log)) : 0;
      if (left < S::kRows || lead > 0) {
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              if (const int r = 16 * m + lane / 4 + (y >> 1) * 8; r >= left || r < lead) s[m][b][y] = -INFINITY;
      }
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int y = 0; y < 4; ++y) past |= s[m][b][y] > top[b][y & 1] + (Type<KIND>::kUp + Type<KIND>::kLag);
      if (__any_sync(~0u, past)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float t = fmaxf(s[0][b][y], s[0][b][y + 2]);
#pragma unroll
            for (int m = 1; m < MB; ++m) t = fmaxf(t, fmaxf(s[m][b][y], s[m][b][y + 2]));
            t = fmaxf(t, __shfl_xor_sync(~0u, t, 4));
            t = fmaxf(t, __shfl_xor_sync(~0u, t, 8));
            t = fmaxf(t, __shfl_xor_sync(~0u, t, 16));
            t = fmaxf(t - Type<KIND>::kUp, top[b][y]);
            const float fade = t == -INFINITY ? 1.f : exp2_fast(top[b][y] - t);
            top[b][y] = t;
            sum[b][y] *= fade;
#pragma unroll
            for (int k = 0; k < KSTEPS; ++k) {
              o[k][b][y] *= fade;
              o[k][b][y + 2] *= fade;
            }
          }
      }
      uint32_t p[MB][NB][2];
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float from = top[b][y & 1];
            s[m][b][y] = exp2_fast(s[m][b][y] - (from == -INFINITY ? 0.f : from));
            sum[b][y & 1] += s[m][b][y];
          }
          p[m][b][0] = transpose8(pack<KIND>(s[m][b][0], s[m][b][1]));
          p[m][b][1] = transpose8(pack<KIND>(s[m][b][2], s[m][b][3]));
        }
#pragma unroll
      for (int m = 0; m < MB; ++m) {
        const uint32_t values16 = values + m * 16 * S::kRowBytes;
        if (KIND == P2P_KV_E4M3) {
#pragma unroll
          for (int k = 0; k < KSTEPS; k += 2) {
            uint32_t r[4];  // tokens 0-7 and 8-15 of piece k, then of piece k + 1
            load4t(r, values16 + place<PIECES>((lane & 7) + (lane >> 3 & 1) * 8, k + (lane >> 4)));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              // A lane's register: values 2 * (lane / 4) + {0, 1} of one token, then of the next; the product's rows
              // 0-7 are the even values, 8-15 the odd ones.
              const uint32_t lo = __byte_perm(r[2 * y], 0, 0x3120), hi = __byte_perm(r[2 * y + 1], 0, 0x3120);
              const uint32_t f[4] = {widen(lo), widen_high(lo), widen(hi), widen_high(hi)};
#pragma unroll
              for (int b = 0; b < NB; ++b) multiply<KIND>(o[k + y][b], f, p[m][b]);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < KSTEPS; ++k) {
            uint32_t f[4];
            load4t(f, values16 + place<PIECES>((lane & 7) + (lane >> 4) * 8, 2 * k + (lane >> 3 & 1)));
#pragma unroll
            for (int b = 0; b < NB; ++b) multiply<KIND>(o[k][b], f, p[m][b]);
          }
        }
      }
    }
    // (the last tile's room: it is not filled before the next step)
    float* const sums = (float*)(room + warp * S::kRoom + (slot ? slot - 1 : S::kStages - 1) * S::kStage);
    here.advance<WHOLE>(count, c, a, blocks, side, tile_log);
    if (here.left > 0) load_queries(here);  // (on their way while this unit row's parts are joined)

    __syncwarp();  // every lane is done with the last tile

    // ---- the four warps' parts, eight heads at a time through shared memory: [head][dim], turned by the head so that
    // neither side's accesses meet a bank twice (within 32 values, which the pitch is a multiple of).
    const int32_t head0 = u.h * group + u.block * S::kHeads, heads = min(group - u.block * S::kHeads, S::kHeads);
    const bool whole = u.t == 0 && count == u.nt, empty = u.row.end <= u.row.begin;
    const int64_t unit0 = x_end - u.left - u.t;  // where the unit row's first tile stands among all units
    // A part: the sums [kv head of the unit][query head][dim], then the maxima, then the sums of exp.
    const int32_t part_heads = S::kHeads << side;
    const int64_t part_size = (int64_t)part_heads * (DP + 2);
    float* const part = w.parts + (blockIdx.x * 4 + (u.t == 0)) * part_size;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b * 8 >= heads) break;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int head = 2 * (lane % 4) + y;
        float z = sum[b][y];
        z += __shfl_xor_sync(~0u, z, 4);
        z += __shfl_xor_sync(~0u, z, 8);
        z += __shfl_xor_sync(~0u, z, 16);
        if (lane < 4) sh.top[warp][head] = top[b][y], sh.sum[warp][head] = z;
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k) {
          const int d = KIND == P2P_KV_E4M3 ? 16 * k + 2 * (lane / 4) : 16 * k + lane / 4;
          sums[head * S::kSumPitch + (d ^ head * 4)] = o[k][b][y];
          sums[head * S::kSumPitch + ((d + (KIND == P2P_KV_E4M3 ? 1 : 8)) ^ head * 4)] = o[k][b][y + 2];
        }
      }
      __syncthreads();
      // (only the block's heads: with 32 on 8 of 128, 2,000 sequences of 1 to 40 tokens take 58 us, with all 8 68)
      for (int y = threadIdx.x; y < min(8, heads - b * 8) * (DP / 4) << side; y += kThreads) {
        const int own = y / (DP / 4), beside = own & ((1 << side) - 1), head = own >> side, d = y % (DP / 4) * 4;
        const int h8 = b * 8 + head;
        float t = -INFINITY, z = 0.f;
#pragma unroll
        for (int k = 0; k < kWarps; ++k)  // the warps that had this kv head
          if ((k & ((1 << side) - 1)) == beside) t = fmaxf(t, sh.top[k][head]);
        const float ref = t == -INFINITY ? 0.f : t;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < kWarps; ++k)
          if ((k & ((1 << side) - 1)) == beside) {
            const float fade = exp2_fast(sh.top[k][head] - ref);
            const float* const his = sums + (k - warp) * (S::kRoom / 4);
            const float4 f = *(const float4*)(his + head * S::kSumPitch + (d ^ head * 4));
            z += fade * sh.sum[k][head];
            v.x += fade * f.x, v.y += fade * f.y, v.z += fade * f.z, v.w += fade * f.w;
          }
        if (!whole) {
          const int at = beside * S::kHeads + h8;
          *(float4*)(part + at * DP + d) = v;
          if (d == 0) part[part_heads * DP + at] = t, part[part_heads * (DP + 1) + at] = z;
        } else {
          const int32_t q_head = head0 + beside * group + h8;
          const float v_scale = KIND == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + u.h + beside] : 1.f;
          store4(c, a, u.i, q_head, d, v, __fdividef(v_scale, z), empty);
          if (d == 0 && a.lse) a.lse[(int64_t)u.i * a.heads + q_head] = empty ? -INFINITY : log_sum<KIND>(t, z);
        }
      }
      if (whole || b + 1 < NB) __syncthreads();  // the sums' room is free again
    }
    if (whole) continue;

    // The CTA that brings the last part of the unit row joins them; where there are many, that of each `bunch` of
    // them joins those, and the one that brings the last of the results joins these.  Each thread has four values of
    // a head, over the parts in their order, kJoin of which are on their way at a time, or, where there are few parts,
    // 4 of 4 such values (34 short rows with 16 heads of 192 values to a kv head 13.7 us, not 16.6); with few values,
    // groups of threads take every so many parts, and the first group puts theirs together.
    const int32_t c0 = (int32_t)(((unit0 + 1) * ctas - 1) / total), c1 = (int32_t)(((unit0 + u.nt) * ctas - 1) / total);
    const int32_t parts = c1 - c0 + 1, all4 = (heads << side) * (DP / 4), turns = (all4 + kThreads - 1) / kThreads;
    const int32_t teams = max(1, kThreads / all4);
    int32_t bunch = parts;
    if (parts * turns > 4 * kJoin * teams) {
      bunch = kJoin * teams;
      while (bunch * bunch < parts) bunch += kJoin * teams;
    }
    int32_t first_part = (blockIdx.x - c0) / bunch * bunch, members = min(bunch, parts - first_part);
    for (int32_t level = 0;; ++level) {
      // Part k lies with its CTA: the first CTA's is its range's last unit row, the others' their first.
      const auto part_of = [&](int32_t k) { return w.parts + ((c0 + k) * 4 + (k == 0) + 2 * level) * part_size; };
      const int32_t apart = level ? bunch : 1;
      // (The count is read and raised after the barrier, in acquire and release order for all of the CTA's accesses.)
      __syncthreads();
      if (threadIdx.x == 0) {
        int32_t* const arrived = w.arrived + (c0 + first_part) * 4 + (first_part == 0) + 2 * level;
        sh.last = add_acq_rel(arrived, 1) == members - 1;
        if (sh.last) *arrived = 0;  // for the next launch
      }
      __syncthreads();
      if (!sh.last) break;
      const bool done = level == 1 || members == parts;
      float* const joined = w.parts + ((c0 + first_part) * 4 + (first_part == 0) + 2) * part_size;
      // AT parts at a time, of ITEMS fours of values.
      const auto join = [&](auto at_a_time, auto values) {
        constexpr int AT = decltype(at_a_time)::value, ITEMS = decltype(values)::value;
        for (int y0 = 0; y0 < all4; y0 += ITEMS * kThreads) {
          const int y1 = teams > 1 ? (int)threadIdx.x % all4 : y0 + (int)threadIdx.x;
          const int team = teams > 1 ? (int)threadIdx.x / all4 : 0;
          float t[ITEMS], z[ITEMS];
          float4 v[ITEMS];
          int at[ITEMS], d[ITEMS];  // where each lies in a part; at < 0: nowhere
#pragma unroll
          for (int i = 0; i < ITEMS; ++i) {
            const int y = y1 + i * kThreads, own = y / (DP / 4), beside = own / heads;
            t[i] = -INFINITY, z[i] = 0.f, v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            at[i] = y < all4 && team < teams ? beside * S::kHeads + (own - beside * heads) : -1;
            d[i] = y % (DP / 4) * 4;
          }
          for (int32_t k0 = team; k0 < members; k0 += teams * AT) {
            float pt[ITEMS][AT], pz[ITEMS][AT];
            float4 pv[ITEMS][AT];
#pragma unroll
            for (int j = 0; j < AT; ++j) {
              const int32_t k = k0 + j * teams;
              const float* const p = part_of(first_part + min(k, members - 1) * apart);
#pragma unroll
              for (int i = 0; i < ITEMS; ++i) {
                pt[i][j] = -INFINITY, pz[i][j] = 0.f, pv[i][j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < members && at[i] >= 0) {
                  pt[i][j] = __ldcg(p + part_heads * DP + at[i]);
                  pz[i][j] = __ldcg(p + part_heads * (DP + 1) + at[i]);
                  pv[i][j] = __ldcg((const float4*)(p + at[i] * DP + d[i]));
                }
              }
            }
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
              float top1 = t[i];
#pragma unroll
              for (int j = 0; j < AT; ++j) top1 = fmaxf(top1, pt[i][j]);
              const float ref = top1 == -INFINITY ? 0.f : top1;
              float fade = exp2_fast(t[i] - ref);
              t[i] = top1;
              z[i] *= fade, v[i].x *= fade, v[i].y *= fade, v[i].z *= fade, v[i].w *= fade;
#pragma unroll
              for (int j = 0; j < AT; ++j) {
                fade = exp2_fast(pt[i][j] - ref);
                z[i] += fade * pz[i][j];
                v[i].x += fade * pv[i][j].x, v[i].y += fade * pv[i][j].y;
                v[i].z += fade * pv[i][j].z, v[i].w += fade * pv[i][j].w;
              }
            }
          }
          if (ITEMS == 1 && teams > 1) {
            const auto of_thread = [&](int x) { return sums + ((x >> 5) - warp) * (S::kRoom / 4) + (x & 31) * 8; };
            float* const mine = of_thread(threadIdx.x);
            mine[0] = t[0], mine[1] = z[0];
            *(float4*)(mine + 4) = v[0];
            __syncthreads();
            if (team == 0) {
              float top1 = t[0];
              for (int k = 1; k < teams; ++k) top1 = fmaxf(top1, of_thread(threadIdx.x + k * all4)[0]);
              const float ref = top1 == -INFINITY ? 0.f : top1;
              float fade = exp2_fast(t[0] - ref);
              t[0] = top1;
              z[0] *= fade, v[0].x *= fade, v[0].y *= fade, v[0].z *= fade, v[0].w *= fade;
              for (int k = 1; k < teams; ++k) {
                const float* p = of_thread(threadIdx.x + k * all4);
                fade = exp2_fast(p[0] - ref);
                z[0] += fade * p[1], v[0].x += fade * p[4], v[0].y += fade * p[5], v[0].z += fade * p[6],
                    v[0].w += fade * p[7];
              }
            }
          }
#pragma unroll
          for (int i = 0; i < ITEMS; ++i) {
            if (at[i] < 0 || team != 0) continue;
            if (done) {
              const int beside = at[i] / S::kHeads;
              const int32_t q_head = head0 + beside * group + at[i] % S::kHeads;
              const float v_scale = KIND == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + u.h + beside] : 1.f;
              store4(c, a, u.i, q_head, d[i], v[i], __fdividef(v_scale, z[i]), false);
              if (d[i] == 0 && a.lse) a.lse[(int64_t)u.i * a.heads + q_head] = log_sum<KIND>(t[i], z[i]);
            } else {
              *(float4*)(joined + at[i] * DP + d[i]) = v[i];
              if (d[i] == 0) joined[part_heads * DP + at[i]] = t[i], joined[part_heads * (DP + 1) + at[i]] = z[i];
            }
          }
        }
      };
      using std::integral_constant;
      if (members <= 4 && turns > 1)
        join(integral_constant<int, 4>(), integral_constant<int, 4>());
      else
        join(integral_constant<int, kJoin>(), integral_constant<int, 1>());
      if (done) break;
      first_part = 0;
      members = (parts + bunch - 1) / bunch;
    }
    __syncthreads();
  }
  wait<0>();  // (of copies past the end of the range, of nothing, into room that is given back now)
}

// With q = NULL the kernel is only made ready for launches.
template <int KIND, int DP, int NB, bool SIDE, bool WHOLE>
cudaError_t launch(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms, cudaStream_t st) {
  using S = Shape<KIND, DP, NB>;
  const auto kernel = attend_kernel<KIND, DP, NB, SIDE, WHOLE>;
  if (!q) return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kBytes);
  // As many CTAs as are resident together (by shared memory: 227 KB an SM, of which each CTA takes 1 KB for the
  // system).
  static_assert(S::kCtas <= KvAttendScratch::kCtasPerSm, "the scratch is for so many");
  return launch_early(kernel, dim3(S::kCtas * num_sms), kThreads, S::kBytes, st, c, *q, w);
}

// (Pages of 16 tokens taken token by token, as others are: 64 ragged 10.7 us, not 9.7, 256 sequences in 8 bits 109,
// not 104.)
template <int KIND, int DP, int NB, bool SIDE>
cudaError_t launch_pages(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms, cudaStream_t st) {
  return c.page % 16 == 0 ? launch<KIND, DP, NB, SIDE, true>(c, q, w, num_sms, st)
                          : launch<KIND, DP, NB, SIDE, false>(c, q, w, num_sms, st);
}

// Blocks of 8, 16 or 32 query heads: the fewest that hold a kv head's, as each block reads the keys and values again
// (on the 32 long sequences 40 heads on 8 take 282 us with blocks of 16 and 523 with 8; 128 heads of 256 values on 8
// 551 and 1,061; 256 heads on 8 301 with blocks of 32 and 539 with 16).  Blocks of 32 beyond 128 values, or beside
// 8-bit values, do not fit the registers (256 heads on 8 over the 8-bit case 286 us, and 234 with blocks of 16).
template <int KIND, int DP, bool SIDE>
cudaError_t launch_heads(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms, cudaStream_t st) {
  const int blocks = q ? attend_blocks(KIND, DP, q->heads / c.heads) : 0;
  cudaError_t e = cudaSuccess;
  if (!q || blocks == 1) e = launch_pages<KIND, DP, 1, SIDE>(c, q, w, num_sms, st);
  if (e == cudaSuccess && (!q || blocks == 2)) e = launch_pages<KIND, DP, 2, SIDE>(c, q, w, num_sms, st);
  if constexpr (attend_blocks(KIND, DP, 32) == 4)
    if (e == cudaSuccess && (!q || blocks == 4)) e = launch_pages<KIND, DP, 4, SIDE>(c, q, w, num_sms, st);
  return e;
}

template <int KIND, bool SIDE>
cudaError_t launch_dim(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms, cudaStream_t st) {
  switch (attend_dim(KIND, c.dim)) {
    case 64: return launch_heads<KIND, 64, SIDE>(c, q, w, num_sms, st);
    case 80: return launch_heads<KIND, attend_dim(KIND, 80), SIDE>(c, q, w, num_sms, st);
    case 96: return launch_heads<KIND, 96, SIDE>(c, q, w, num_sms, st);
    case 128: return launch_heads<KIND, 128, SIDE>(c, q, w, num_sms, st);
    case 192: return launch_heads<KIND, 192, SIDE>(c, q, w, num_sms, st);
    default: return launch_heads<KIND, 256, SIDE>(c, q, w, num_sms, st);
  }
}

}  // namespace
}  // namespace p2p
