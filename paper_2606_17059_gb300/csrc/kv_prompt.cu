// kv_prompt.cu -- attention of several new tokens a sequence over the paged key-value cache (p2p_kv_attend_prompt).
//
// The new token at position p of its sequence sees tokens max(0, p + 1 - window) .. p: x_t = scale * q . k_t, m = max x_t,
// z = sum exp(x_t - m), out = sum exp(x_t - m) v_t / z, lse = m + ln z.  A warp takes one query head of one token and
// goes through its tokens one by one, with the maximum and the sum as they run.
#include "kv_values.cuh"

namespace p2p {
namespace {

constexpr int kRowThreads = 128, kMost = 8;  // values of a lane: head_dim is at most 256

template <int TYPE>
__device__ __forceinline__ float number(const void* p, int64_t i) {
  if (TYPE == P2P_KV_BF16) return __bfloat162float(((const __nv_bfloat16*)p)[i]);
  if (TYPE == P2P_KV_F16) return __half2float(((const __half*)p)[i]);
  return __half2float(__nv_cvt_fp8_to_halfraw(((const __nv_fp8_storage_t*)p)[i], __NV_E4M3));
}

template <int KIND, int IN>
__global__ void __launch_bounds__(kRowThreads) prompt_kernel(KvView c, KvPrompt a, int32_t* err) {
  begin_kernel();
  if (blockIdx.x == 0) check_offsets(a.offsets, a.n, a.n_tokens, err);
  const int lane = threadIdx.x & 31;
  const int64_t rows = a.n_tokens * a.heads, all = (int64_t)gridDim.x * (kRowThreads / 32);
  for (int64_t r = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5); r < rows; r += all) {
    const int64_t t = r / a.heads;
    const int32_t head = (int32_t)(r - t * a.heads), h = head / (a.heads / c.heads);
    const int32_t i = find_item(a.offsets, a.n, t);
    const int64_t o0 = a.offsets[i], o1 = a.offsets[i + 1];
    if (o0 < 0 || t < o0 || t >= o1 || o1 > a.n_tokens) continue;
    const int32_t seq = a.seq ? a.seq[i] : i;
    if ((uint32_t)seq >= (uint32_t)c.n_seqs) {
      atomicOr(err, KV_BAD_SEQ);
      continue;
    }
    const int32_t len = length_of(c, seq);
    if (len < o1 - o0) {
      atomicOr(err, KV_BAD_COUNT);
      continue;
    }
    const int32_t end = len - (int32_t)(o1 - t) + 1, begin = a.window && end > a.window ? end - a.window : 0;
    float q[kMost], o[kMost] = {}, top = -INFINITY, z = 0.f;
#pragma unroll
    for (int m = 0; m < kMost; ++m)
      q[m] = lane + 32 * m < c.dim ? number<IN>(a.q, t * a.q_token + head * a.q_head + lane + 32 * m) : 0.f;
    const float unit = a.scale * (KIND == P2P_KV_E4M3 ? c.k_scale[a.layer * c.heads + h] : 1.f);
    for (int32_t p = begin; p < end; ++p) {
      const uint32_t e = c.by_page.div(p);
      const int32_t page = row_of(c, seq)[e];
      if ((uint32_t)page >= (uint32_t)c.n_pages) atomicOr(err, KV_BAD_PAGE);
      const bool there = (uint32_t)page < (uint32_t)c.n_pages;
      const int64_t at = a.layer * c.layer_stride + page * c.page_stride + (p - e * c.page) * c.token_stride + h * c.head_stride;
      float x = 0.f;
#pragma unroll
      for (int m = 0; m < kMost; ++m)
        if (there && lane + 32 * m < c.dim) x = fmaf(q[m], number<KIND>(c.k + at, lane + 32 * m), x);
#pragma unroll
      for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
      x *= unit;
      const float now = fmaxf(top, x), fade = now == -INFINITY ? 1.f : expf(top - now), y = now == -INFINITY ? 1.f : expf(x - now);
      top = now;
      z = z * fade + y;
#pragma unroll
      for (int m = 0; m < kMost; ++m)
        o[m] = o[m] * fade + (there && lane + 32 * m < c.dim ? y * number<KIND>(c.v + at, lane + 32 * m) : 0.f);
    }
    const float f = (KIND == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + h] : 1.f) / z;
#pragma unroll
    for (int m = 0; m < kMost; ++m) {
      if (lane + 32 * m >= c.dim) continue;
      const int64_t to = t * a.out_token + head * a.out_head + lane + 32 * m;
      if (IN == P2P_KV_BF16)
        ((__nv_bfloat16*)a.out)[to] = __float2bfloat16(o[m] * f);
      else
        ((__half*)a.out)[to] = __float2half(o[m] * f);
    }
    if (lane == 0 && a.lse) a.lse[t * a.heads + head] = top + logf(z);
  }
}

}  // namespace

cudaError_t launch_kv_prompt(const KvView& c, const KvPrompt& a, int32_t* err, int num_sms, cudaStream_t st) {
  const auto kernel = c.type == P2P_KV_BF16  ? prompt_kernel<P2P_KV_BF16, P2P_KV_BF16>
                      : c.type == P2P_KV_F16 ? prompt_kernel<P2P_KV_F16, P2P_KV_F16>
                      : a.type == P2P_KV_BF16 ? prompt_kernel<P2P_KV_E4M3, P2P_KV_BF16>
                                              : prompt_kernel<P2P_KV_E4M3, P2P_KV_F16>;
  return launch_early(kernel, dim3(16 * num_sms), kRowThreads, 0, st, c, a, err);
}

}  // namespace p2p
