// kv_join.cu -- the parts of units that several CTAs of kv_rows.cuh shared, put together: with each part's maximum m_k (in log2),
// sum z_k and unnormalised result o_k, out = sum 2^(m_k - m) o_k / sum 2^(m_k - m) z_k, m = max m_k, in the parts' order.
//
// A launch of its own, as its few loads in a row then run on all SMs at once: by the CTAs that brought the last parts, 40 of 128 x
// 128 values and 5 parts each took 22 us at the end of the launch.  A warp has four rows and 32 values of them, so that loads are
// of 64 bytes a row and stores too.
#include "kv_math.cuh"

namespace p2p {
namespace {

constexpr int kThreads = 128, kRowsOfWarp = 4, kMostCtas = 1024;

__global__ void __launch_bounds__(kThreads)
    join_kernel(KvView c, KvRowsCall a, KvAttendScratch w, int32_t ctas, int32_t dp, int32_t tiles) {
  __shared__ int32_t units[kMostCtas];
  __shared__ int32_t count;
  begin_kernel();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // The units that there are, in the same order in every CTA.
  if (warp == 0) {
    int32_t n = 0;
    for (int i0 = 0; i0 < ctas; i0 += 32) {
      const bool some = i0 + lane < ctas && w.joins[i0 + lane].parts > 0;
      const uint32_t m = __ballot_sync(~0u, some);
      if (some) units[n + __popc(m & ((1u << lane) - 1))] = i0 + lane;
      n += __popc(m);
    }
    if (lane == 0) count = n;
  }
  __syncthreads();
  // (The maximum is held less 2^kUp, see Type.)
  const float up = c.type == P2P_KV_BF16 ? Type<P2P_KV_BF16>::kUp : Type<P2P_KV_F16>::kUp;
  const int columns = (c.dim + 31) / 32, each = tiles * (128 / kRowsOfWarp) * columns;  // of a unit
  for (int y = blockIdx.x * (kThreads / 32) + warp; y < count * each; y += gridDim.x * (kThreads / 32)) {
    const int c0 = units[y / each], x = y % (each / tiles), tile = y % each / (each / tiles);
    const KvJoin u = w.joins[c0];
    const float v_scale = c.type == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + u.h] : 1.f;
    const auto part_of = [&](int32_t k) { return w.parts + rows_part(c0 + k, k == 0, tiles, tile, dp); };
    const int r = x / columns * kRowsOfWarp + lane / 8, d = x % columns * 32 + lane % 8 * 4;
    if (r >= a.tile_rows || tile * a.tile_rows + r >= u.rows || d >= c.dim) continue;
    float m = -INFINITY, z = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = 8;
    for (int32_t k0 = 0; k0 < u.parts; k0 += kAhead) {
      float pm[kAhead], pz[kAhead];
      float4 po[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float* const p = part_of(min(k0 + k, u.parts - 1));
        pm[k] = __ldcg(p + dp * 128 + r), pz[k] = __ldcg(p + (dp + 1) * 128 + r);
        po[k] = __ldcg((const float4*)p + d / 4 * 128 + r);
        if (k0 + k >= u.parts) pm[k] = -INFINITY;
      }
      float most = m;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) most = fmaxf(most, pm[k]);
      const float ref = most == -INFINITY ? 0.f : most;
      float fade = exp2_fast(m - ref);
      m = most;
      z *= fade, o.x *= fade, o.y *= fade, o.z *= fade, o.w *= fade;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k0 + k >= u.parts) break;
        fade = exp2_fast(pm[k] - ref);
        z = fmaf(pz[k], fade, z);
        o.x = fmaf(po[k].x, fade, o.x), o.y = fmaf(po[k].y, fade, o.y);
        o.z = fmaf(po[k].z, fade, o.z), o.w = fmaf(po[k].w, fade, o.w);
      }
    }
    const uint32_t at = u.g0 + tile * a.tile_rows + r, t = a.by_group.div(at);
    const int64_t row = u.row + t;
    const int32_t head = u.h * a.group + (int32_t)(at - t * a.group);
    const float f = z > 0.f || z != z ? v_scale / z : 0.f;
    if (d == 0)
      if (float* const lse = a.pre ? a.pre_lse : a.lse)
        lse[row * a.heads + head] = z == 0.f ? -INFINITY : (m + up + __log2f(z * exp2f(-up))) * kLn2;
    o.x *= f, o.y *= f, o.z *= f, o.w *= f;
    if (a.pre) {
      *(float4*)(a.pre + (row * a.heads + head) * c.dim + d) = o;
      continue;
    }
    const uint32_t b0 = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(o.x, o.y) : pack<P2P_KV_F16>(o.x, o.y);
    const uint32_t b1 = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(o.z, o.w) : pack<P2P_KV_F16>(o.z, o.w);
    uint16_t* const to = (uint16_t*)a.out + row * a.out_row + head * a.out_head + d;
    if (a.out32) {
      *(uint2*)to = make_uint2(b0, b1);
    } else {
      to[0] = (uint16_t)b0, to[1] = (uint16_t)(b0 >> 16);
      to[2] = (uint16_t)b1, to[3] = (uint16_t)(b1 >> 16);
    }
  }
}

}  // namespace

cudaError_t launch_kv_join(const KvView& c, const KvRowsCall& a, const KvAttendScratch& w, int num_sms, cudaStream_t st) {
  const int dp = (c.dim + 63) / 64 * 64, tiles = dp <= 128 ? 2 : 1;
  if (num_sms > kMostCtas) return cudaErrorInvalidConfiguration;
  return launch_early(join_kernel, dim3(8 * num_sms), kThreads, 0, st, c, a, w, (int32_t)num_sms, (int32_t)dp, (int32_t)tiles);
}

}  // namespace p2p
