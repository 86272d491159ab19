// kv_values.cuh -- what the kernels that write to the paged key-value cache share: where a batch's tokens go, and
// values of 8 bits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv.h"

// (No load here goes past the coherent path, as __ldg or const __restrict__ would have it: the kernel before may
// still be writing when this one starts, see launch_early.)
namespace p2p {
namespace {

// A length as the table can hold it, or -1.
__device__ __forceinline__ int32_t length_of(const KvView& c, int32_t seq) {
  const int32_t n = c.length[seq];
  return n >= 0 && n <= c.max_pages * c.page ? n : -1;
}
__device__ __forceinline__ int32_t* row_of(const KvView& c, int32_t seq) {
  return c.table + (int64_t)seq * c.max_pages;
}

// The last item that starts at or before token t (items without tokens share a start): every lane gets it.
template <class T>
__device__ __forceinline__ int32_t find_item(const T* offsets, int32_t n, int64_t t) {
  const int lane = threadIdx.x & 31;
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {  // 32 probes a round
    const int32_t step = (hi - lo + 31) / 32, at = lo + step * lane;
    const uint32_t m = __ballot_sync(~0u, at < hi && offsets[at] <= t);
    if (!m) return lo;
    const int32_t k = 31 - __clz(m);
    lo = lo + step * k;
    hi = min(hi, lo + step);
  }
  return lo;
}

// Tokens that a group of rows works off together, from what launch_kv_share found: x entries that are the same, tokens
// from y on seen by some row.
__device__ __forceinline__ int32_t shared_tokens(const KvView& c, int4 span, int32_t members) {
  const int32_t tokens = span.x * c.page;
  return members > 1 && tokens - span.y >= kSharedTokens ? tokens : 0;
}

// By all threads of a CTA: reports offsets that do not ascend or leave the batch.
__device__ __forceinline__ void check_offsets(const int64_t* offsets, int32_t n, int64_t n_tokens, int32_t* err) {
  for (int32_t i = threadIdx.x; i < n; i += blockDim.x)
    if (offsets[i] < 0 || offsets[i + 1] < offsets[i] || offsets[i + 1] > n_tokens) atomicOr(err, KV_BAD_OFFSETS);
}

// By a whole warp: where token t0 + lane of the batch goes, in bytes within a layer, and (pos) its position in its
// sequence; -1: it is not written, and reported if it should be.
__device__ __forceinline__ int64_t place_of(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq,
                                            const int64_t* offsets, int64_t n_tokens, int64_t t0, int32_t halt,
                                            int32_t& pos) {
  const int64_t t = t0 + (threadIdx.x & 31);
  int32_t lo = find_item(offsets, n, t0), hi = min(n, find_item(offsets, n, t0 + 31) + 1);
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (offsets[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  int64_t at = -1;
  pos = 0;
  const int64_t o0 = offsets[lo], o1 = offsets[lo + 1];
  if (!halt && o0 >= 0 && o0 <= t && t < o1 && o1 <= n_tokens) {  // (else it belongs to no sequence)
    const int32_t q = seq[lo], len = (uint32_t)q < (uint32_t)c.n_seqs ? length_of(c, q) : 0;
    int32_t bad = 0;
    if ((uint32_t)q >= (uint32_t)c.n_seqs) {
      bad = KV_BAD_SEQ;
    } else if (o1 - o0 > len) {
      bad = KV_BAD_COUNT;
    } else {
      pos = len - (int32_t)(o1 - t);
      const int32_t e = (int32_t)c.by_page.div(pos), page = row_of(c, q)[e];
      const int32_t refs = (uint32_t)page < (uint32_t)c.n_pages ? c.refs[page] : 0;
      if (refs != 1)
        bad = refs > 1 ? KV_SHARED : KV_BAD_PAGE;
      else
        at = page * c.page_stride + (pos - e * c.page) * c.token_stride;
    }
    if (bad) atomicOr(s.err, bad);
  }
  return at;
}

// If the quotient rounded to 32 bits is a tie (its 19 lowest bits are zero) and the quotient is not: one step to its
// side, as its exact remainder tells (of which nothing vanishes or overflows).  For scales of an extreme size.
__device__ __forceinline__ float divide_extreme(float x, float scale) {
  const float z = __fdiv_rn(x, scale), up = fabsf(scale) < 1.f ? 0x1p100f : 1.f, r = fmaf(-z, scale * up, x * up);
  int32_t b = __float_as_int(z);
  if ((b & 0x7ffff) == 0 && (r < 0.f || r > 0.f)) b += (r < 0.f) == (x < 0.f) ? 1 : -1;
  return __int_as_float(b);
}
template <bool BF16>
__device__ __forceinline__ float2 two_values(uint32_t x) {
  return BF16 ? __bfloat1622float2(*(const __nv_bfloat162*)&x) : __half22float2(*(const __half2*)&x);
}
// Two values to 8 bits each, the first in the low ones.
__device__ __forceinline__ uint32_t narrow(float2 v) {
  return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}

}  // namespace
}  // namespace p2p
