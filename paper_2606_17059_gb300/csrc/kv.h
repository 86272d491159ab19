// kv.h -- the paged key-value cache (p2p_kv_* of p2p_router.h): what its host code and its kernels share.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "kv_rows_cost.h"
#include "p2p_router.h"

namespace p2p {

// Division of x < 2^31 by a fixed 1 <= d < 2^31: floor(x / d) = (x * mul) >> shift with shift = 31 + ceil(log2 d) and
// mul = ceil(2^shift / d) = (2^shift + e) / d, 0 <= e < d.  The product over 2^shift is x / d + (x * e / 2^shift) /
// d; as x * e < 2^shift, that is less than 1 / d above x / d, which does not reach the next whole number.
struct FastDiv {
  uint32_t d = 1, shift = 31;
  uint64_t mul = 1ull << 31;
  FastDiv() = default;
  explicit FastDiv(uint32_t n) : d(n) {
    uint32_t l = 0;
    while ((1ull << l) < n) ++l;
    shift = 31 + l;
    mul = ((1ull << shift) + n - 1) / n;
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t x) const { return (uint32_t)((x * mul) >> shift); }
  __host__ __device__ __forceinline__ uint32_t ceil(uint32_t x) const { return x ? div(x - 1) + 1 : 0; }
};

// The cache's kernels are launched so that one may start while the one before it on the stream still runs; each waits
// for that one's end before its first access to memory (begin_kernel) and lets the next start at once.  A short
// call's launch is hidden that way.
template <class... P, class... A>
cudaError_t launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t shared, cudaStream_t st,
                         const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = shared;
  cfg.stream = st;
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}
#ifdef __CUDACC__
__device__ __forceinline__ void begin_kernel() {
  asm volatile("griddepcontrol.launch_dependents;\n griddepcontrol.wait;" ::: "memory");
}
#endif

// The cache as the kernels see it; strides in bytes.
struct KvView {
  char *k, *v;
  const float *k_scale, *v_scale;
  int32_t *table, *length, *refs;
  int32_t n_layers, n_pages, page, heads, dim, type, n_seqs, max_pages;
  int64_t layer_stride, page_stride, token_stride, head_stride;
  FastDiv by_page;
  int32_t row16;  // 16-byte pieces of a head's values of one token
  int32_t side;   // log2 of the kv heads that a unit of the attention may take side by side
  bool lines;     // whether heads share lines of memory (see shares_lines in kv_cache.cpp)
};

// Bits of the device error word.
enum { KV_BAD_SEQ = 1, KV_BAD_COUNT = 2, KV_NO_PAGES = 4, KV_BAD_PAGE = 8, KV_SHARED = 16, KV_BAD_OFFSETS = 32,
    KV_STUCK = 64 };

struct __align__(16) KvJob {  // copy the first `tokens` tokens of page `from` to page `to`, in every layer
  int32_t from, to, tokens, pad_;
};

// Device words and scratch of the calls that change the page tables.
struct KvScratch {
  int32_t* err;    // error bits since the last p2p_kv_sync
  int32_t* halt;   // 1 since a call on the tables failed: later ones, and writes, change nothing until p2p_kv_sync
  int32_t* njobs;
  int32_t* live;   // pages in use, as a compaction found them
  int32_t* claim;  // [n_seqs], zero between calls: a sequence named twice in one call
  int32_t* start;  // [n_seqs + 1]: where a sequence's page entries start among the call's
  int32_t* first;  // [n_seqs]: its first entry concerned
  int32_t* cut;    // [n_seqs]: > 0: the tokens of its shared last page that it takes along into a page of its own
  int32_t* list;   // [n_pages]: compaction: a moved page's new number
  KvJob* jobs;     // [max(n_seqs, n_pages)]
};

cudaError_t prepare_kv_pages();  // makes the kernels ready for launches (at creation)
cudaError_t launch_kv_extend(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* count,
                             int num_sms, cudaStream_t st);
cudaError_t launch_kv_trim(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* to,
                           cudaStream_t st);
cudaError_t launch_kv_fork(const KvView& c, const KvScratch& s, int32_t n, const int32_t* src, const int32_t* dst,
                           const int32_t* tokens, cudaStream_t st);
cudaError_t launch_kv_compact(const KvView& c, const KvScratch& s, int num_sms, cudaStream_t st, int* launches);
// Keys and values to write; strides in elements.
struct KvRows {
  const void *k, *v;
  int64_t layer_stride, token_stride, head_stride;
  int32_t type;
};
cudaError_t launch_kv_write(const KvView& c, const KvScratch& s, int32_t layer, int32_t n_layers, int32_t n,
                            const int32_t* seq, const int64_t* offsets, int64_t n_tokens, const KvRows& rows,
                            int num_sms, cudaStream_t st);
// out (zeroed by the launch): pages in use, pages shared, the highest page in use + 1, tokens held.
cudaError_t launch_kv_stats(const KvView& c, unsigned long long* out, int num_sms, cudaStream_t st);

// Queries, keys and values of new tokens to norm, rotate and write (kv_rotate.cu); strides in elements.
struct KvTurn {
  const void *q, *k, *v;
  void* out;  // of the queries
  int64_t q_token, q_head, out_token, out_head, token, head;
  const uint64_t* turns;
  const float *q_weight, *k_weight;
  float amplitude, eps;
  int32_t heads, type, rot;
  bool pairs;
};
cudaError_t launch_kv_turn(const KvView& c, const KvScratch& s, const KvTurn& a, int32_t layer, int32_t n,
                           const int32_t* seq, const int64_t* offsets, int64_t n_tokens, int num_sms, cudaStream_t st);

// One token of each of n sequences (kv_attend.cuh).
struct KvQuery {
  const void* q;
  void* out;
  float* lse;
  const int32_t* seq;  // NULL: sequences 0 .. n-1
  int64_t q_row, q_head, out_row, out_head;  // strides in elements
  int32_t n, heads, type, window, layer;
  float scale;
  // Whether rows of q may be read by twos, and those of out written by fours, of their values.
  bool q_pairs, out_fours;
  // Row i is taken from token skip[i] on (NULL: all of it), and where that is not 0, put together with the result of
  // those before: pre [row][head][value], and their maximum (in log2, as it is held: see Type) and sum of exp, pre_sum
  // [row][head].
  const int32_t* skip;
  const float* pre;
  const float2* pre_sum;
};
// The attention's kernel for values of a type, head_dim and `group` query heads a kv head: head_dim as it is padded,
// blocks of eight query heads taken together, and CTAs resident on an SM.
constexpr int attend_value_size(int type) { return type == P2P_KV_E4M3 ? 1 : 2; }
constexpr int attend_dim(int type, int dim) {
  // (80 values of 8 bits are five 16-byte pieces, not whole turns of a warp)
  return dim <= 64    ? 64
         : dim <= 80 && type != P2P_KV_E4M3 ? 80
         : dim <= 96  ? 96
         : dim <= 128 ? 128
         : dim <= 192 ? 192
                      : 256;
}
constexpr int attend_blocks(int type, int dp, int group) {
  return group <= 8 ? 1 : group <= 16 || dp > 128 || type == P2P_KV_E4M3 ? 2 : 4;
}
// Tokens that a warp takes at a time (see Shape in kv_attend.cuh).
constexpr int attend_rows(int type, int dp) { return type == P2P_KV_E4M3 && dp <= 128 ? 32 : 16; }
// Three where three have room for more than two tiles a warp and registers enough (168 a thread), one where two have
// not.
constexpr int attend_ctas(int type, int dp, int blocks) {
  const int row = dp * attend_value_size(type);
  return attend_rows(type, dp) * row <= 3 * 1024 && dp * blocks <= 256 ? 3 : row <= 256 ? 2 : 1;
}

// Rows (of a sequence and kv head) a CTA, of two an SM at least, from which the attention's kernel that may take heads
// together is used where they do not share lines: only the device knows how long they are.  Below, it is mostly the
// slower one: 512 sequences of 1 to 800 tokens with 4 heads of 256 16-bit values 84 us, not 66 (of 1 to 40 40, not
// 45), 608 of 1 to 300 with 4 of 64 22.4, not 20.9.  Above, short rows gain up to 2x (see kSideShort), those of some
// hundred tokens lose up to 18% (608 of 1 to 800 with 4 of 256 90, not 77; 2,000 of them 236, not 225) and long ones
// 1% (512 of 1,000 to 4,000 with 8 of 128 657, not 653).
constexpr int kSideRows = 7;
struct KvJoin {        // a unit of kv_rows.cuh that CTA c0 begins and others go on with
  int64_t row;         // its first row
  int32_t rows, g0, h, parts;  // parts: 0 where there is none
};
// Parts of rows that several CTAs share, four a CTA (see the kernel), and how many have arrived (zero between
// launches).
struct KvAttendScratch {
  static constexpr int kCtasPerSm = 3;
  float* parts;      // [the more of kv_attend_parts() and kv_rows_parts()]
  int32_t* arrived;  // [4 * kCtasPerSm * SMs]
  KvJoin* joins;     // [SMs]: of each CTA of kv_rows.cuh
  int32_t* err;
};
// Floats of `parts`: for the blocks of query heads that take most, each part with the sums, maximum and sum of exp of
// up to 4 kv heads.
inline size_t kv_attend_parts(const KvView& c, int num_sms) {
  const int dp = attend_dim(c.type, c.dim);
  size_t most = 0;
  for (const int group : {8, 16, 32}) {
    const int blocks = attend_blocks(c.type, dp, group);
    most = std::max(most, (size_t)4 * attend_ctas(c.type, dp, blocks) * num_sms * (8 * blocks << c.side) * (dp + 2));
  }
  return most;
}
// With q = NULL they launch nothing, but make the cache's kernels ready for launches (at creation).
cudaError_t launch_kv_attend_bf16(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                  cudaStream_t st);
cudaError_t launch_kv_attend_bf16_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                        cudaStream_t st);
cudaError_t launch_kv_attend_bf16_side(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                       cudaStream_t st);
cudaError_t launch_kv_attend_bf16_side_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                             cudaStream_t st);
cudaError_t launch_kv_attend_f16(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                 cudaStream_t st);
cudaError_t launch_kv_attend_f16_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                       cudaStream_t st);
cudaError_t launch_kv_attend_f16_side(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                      cudaStream_t st);
cudaError_t launch_kv_attend_f16_side_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                            cudaStream_t st);
cudaError_t launch_kv_attend_e4m3(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                  cudaStream_t st);
cudaError_t launch_kv_attend_e4m3_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                        cudaStream_t st);
cudaError_t launch_kv_attend_e4m3_side(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                       cudaStream_t st);
cudaError_t launch_kv_attend_e4m3_side_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                             cudaStream_t st);


// What the rows of each group share, into spans[n_groups] (x: leading entries that are the same; y, z: the first and
// the last token that a row's window begins with), and the tokens of each row that its group works off, into skip[n]:
// none, if that saves the reading of fewer than `least` tokens, a group of m rows counted as m - kTogether (0: any).
cudaError_t launch_kv_share(const KvView& c, int32_t* err, int32_t n, const int32_t* seq, int32_t n_groups,
                            const int32_t* groups, int32_t window, int64_t least, int32_t* skip, int4* spans,
                            cudaStream_t st);
// Reports groups that do not ascend or leave the batch.
cudaError_t launch_kv_groups(int32_t* err, int32_t n, int32_t n_groups, const int32_t* groups, cudaStream_t st);
// Fewer shared tokens than these are read by each row for itself.
constexpr int kSharedTokens = 64;
// What a group's rows cost together, in rows that are read alone.
constexpr int kTogether = 4;

// Many query rows over the same keys and values (kv_rows.cuh): the last offsets[i + 1] - offsets[i] tokens of each of n
// sequences, or, with spans, what each of n groups of rows shares.  Strides in elements.
struct KvRowsCall {
  const void* q;
  void* out;
  float* lse;
  const int32_t* seq;  // of a sequence, or of a row; NULL: its own number
  const int64_t* offsets;
  const int32_t* groups;    // [n + 1]
  const int4* spans;        // [n]: see launch_kv_share
  float* pre;               // where results go, in 32 bits, [row][head][value] (NULL: to out and lse)
  float2* pre_sum;          // and their maxima and sums of exp, [row][head]
  int64_t n_tokens, q_row, q_head, out_row, out_head;
  int32_t n, heads, group, type, window, layer;  // group: query heads a kv head
  FastDiv by_group;
  RowsScale count;   // how work is counted
  int64_t patience;  // clock cycles without a sign of work after which the kernel gives up; negative: it is made to
  float scale;
  bool boxes, out32;      // whether queries come by boxes of whole tokens, and rows of out lie on 32-byte boundaries
  int32_t tile_rows;      // rows of a row tile: 128, or as many whole tokens as fit them
  const CUtensorMap* q_map;  // (host)
};
// The pages as tensors [layer][page][head][token][value] for copies of `rows` tokens of one head and page at a time,
// 16-bit values 64 at a time (128 bytes, turned as the tensor cores want them), 8-bit ones whole rows; rows 0: not to
// be had (pages that are not whole eights of tokens).
struct KvMaps {
  CUtensorMap k, v;
  int32_t rows;
};
// Where the part of CTA `cta` of a unit that it begins (else: goes on with) lies among the parts, in floats: for each
// row tile of 128 rows [fours of values][row][4], then maxima and sums.
__host__ __device__ inline int64_t rows_part(int32_t cta, bool begins, int32_t tiles, int32_t tile, int32_t dp) {
  return (int64_t)((2 * cta + begins) * tiles + tile) * 128 * (dp + 2);
}
// Joins the parts of units that several CTAs of the launch before shared.
cudaError_t launch_kv_join(const KvView& c, const KvRowsCall& a, const KvAttendScratch& w, int num_sms,
    cudaStream_t st);
// Floats of KvAttendScratch::parts: two parts a CTA, of 256 or (head_dim above 128) 128 rows.
inline size_t kv_rows_parts(const KvView& c, int num_sms) {
  const int dp = (c.dim + 63) / 64 * 64;
  return (size_t)2 * num_sms * (dp <= 128 ? 256 : 128) * (dp + 2);
}
// With a = NULL they launch nothing, but make the cache's kernel ready for launches (at creation).
cudaError_t launch_kv_rows_bf16(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w,
    int num_sms,
                                cudaStream_t st);
cudaError_t launch_kv_rows_f16(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w,
    int num_sms,
                               cudaStream_t st);
cudaError_t launch_kv_rows_e4m3(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w,
    int num_sms,
                                cudaStream_t st);

}  // namespace p2p
