// kv_attend.cu -- attention of one new token a sequence over the paged key-value cache (p2p_kv_attend).
//
// For a query head and the tokens t that it sees: x_t = scale * q . k_t, m = max x_t, z = sum exp(x_t - m), out = sum
// exp(x_t - m) v_t / z, lse = m + ln z; without a token, out = 0 and lse = -inf.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv.h"

namespace p2p {
namespace {

constexpr int kWarps = 8, kPer = 8;  // values of a head's row that a lane holds (head_dim <= 256)

__device__ __forceinline__ float value(const char* row, int32_t i, int32_t type) {
  if (type == P2P_KV_BF16) return __bfloat162float(((const __nv_bfloat16*)row)[i]);
  if (type == P2P_KV_F16) return __half2float(((const __half*)row)[i]);
  __nv_fp8_e4m3 x;
  x.__x = ((const uint8_t*)row)[i];
  return float(x);
}

// A CTA takes a (sequence, query head); its warps take tokens in turn, a running maximum and sum each.
__global__ void __launch_bounds__(kWarps * 32) attend_kernel(KvView c, KvQuery a, int32_t* err) {
  const int32_t i = blockIdx.x / a.heads, head = blockIdx.x % a.heads, h = head / (a.heads / c.heads);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int32_t s = a.seq ? a.seq[i] : i;
  int32_t len = 0;
  if ((uint32_t)s >= (uint32_t)c.n_seqs) {
    if (threadIdx.x == 0) atomicOr(err, KV_BAD_SEQ);
  } else {
    len = c.length[s];
    if (len < 0 || len > c.max_pages * c.page) {
      if (threadIdx.x == 0) atomicOr(err, KV_BAD_COUNT);
      len = 0;
    }
  }
  const int32_t begin = a.window && len > a.window ? len - a.window : 0;
  const int64_t layer = (int64_t)a.layer * c.layer_stride + h * c.head_stride;
  const float k_scale = (c.k_scale ? c.k_scale[a.layer * c.heads + h] : 1.f) * a.scale;
  const float v_scale = c.v_scale ? c.v_scale[a.layer * c.heads + h] : 1.f;
  float q[kPer], o[kPer] = {}, m = -INFINITY, z = 0.f;
  for (int j = 0; j < kPer; ++j) {
    const int32_t x = lane + 32 * j;
    q[j] = x < c.dim ? value((const char*)a.q + (i * a.q_row + head * a.q_head) * 2, x, a.type) : 0.f;
  }
  for (int32_t t = begin + warp; t < len; t += kWarps) {
    const int32_t e = (int32_t)c.by_page.div(t), page = c.table[(int64_t)s * c.max_pages + e];
    if ((uint32_t)page >= (uint32_t)c.n_pages) {
      if (lane == 0) atomicOr(err, KV_BAD_PAGE);
      continue;
    }
    const int64_t at = layer + page * c.page_stride + (t - e * c.page) * c.token_stride;
    float x = 0.f;
    for (int j = 0; j < kPer; ++j)
      if (lane + 32 * j < c.dim) x += q[j] * value(c.k + at, lane + 32 * j, c.type);
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    x *= k_scale;
    const float top = fmaxf(m, x), base = top == -INFINITY ? 0.f : top, fade = __expf(m - base), p = __expf(x - base);
    z = z * fade + p;
    for (int j = 0; j < kPer; ++j)
      if (lane + 32 * j < c.dim) o[j] = o[j] * fade + p * value(c.v + at, lane + 32 * j, c.type);
    m = top;
  }
  __shared__ float sm[kWarps], sz[kWarps], so[kWarps][kPer * 32];
  if (lane == 0) sm[warp] = m, sz[warp] = z;
  for (int j = 0; j < kPer; ++j) so[warp][lane + 32 * j] = o[j];
  __syncthreads();
  float top = -INFINITY, sum = 0.f, w[kWarps];
  for (int k = 0; k < kWarps; ++k) top = fmaxf(top, sm[k]);
  const float base = top == -INFINITY ? 0.f : top;
  for (int k = 0; k < kWarps; ++k) sum += sz[k] * (w[k] = __expf(sm[k] - base));
  for (int32_t x = threadIdx.x; x < c.dim; x += kWarps * 32) {
    float y = 0.f;
    for (int k = 0; k < kWarps; ++k) y += w[k] * so[k][x];
    y = len > begin ? y / sum * v_scale : 0.f;
    const int64_t to = i * a.out_row + head * a.out_head + x;
    if (a.type == P2P_KV_BF16)
      ((__nv_bfloat16*)a.out)[to] = __float2bfloat16(y);
    else
      ((__half*)a.out)[to] = __float2half(y);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[(int64_t)i * a.heads + head] = len > begin ? top + logf(sum) : -INFINITY;
}

}  // namespace

cudaError_t launch_kv_attend(const KvView& c, const KvQuery& q, int32_t* err, int num_sms, cudaStream_t st) {
  (void)num_sms;
  if ((int64_t)q.n * q.heads > INT32_MAX) return cudaErrorInvalidValue;
  attend_kernel<<<q.n * q.heads, kWarps * 32, 0, st>>>(c, q, err);
  return cudaGetLastError();
}

}  // namespace p2p
