// kv_join.cu -- the parts of units that several CTAs of kv_rows.cuh shared, put together: with each part's maximum m_k
// (in log2), sum z_k and unnormalised result o_k, out = sum 2^(m_k - m) o_k / sum 2^(m_k - m) z_k, m = max m_k, in the
// parts' order.
//
// A launch of its own, as its few loads in a row then run on all SMs at once: by the CTAs that brought the last parts, 40
// tiles of 128 x 128 values and 5 parts each took 22 us at the end of the launch, and take 6 here.  A warp has four rows
// and up to 128 values of them, so that up to 16 loads of a lane are on their way together.  7 to 18 us under ncu (cold),
// in a graph behind kv_rows.cuh less: a chain of loads (a unit's parts, their maxima, their rows).
#include "kv_math.cuh"

namespace p2p {
namespace {

constexpr int kThreads = 256, kRowsOfWarp = 4, kMostCtas = 1024;

// COLUMNS: thirty-twos of a row's values that a warp takes at a time, all of whose loads are on their way together.
template <int COLUMNS>
__global__ void __launch_bounds__(kThreads)
    join_kernel(KvView c, KvRowsCall a, KvAttendScratch w, int32_t ctas, int32_t dp, int32_t tiles) {
  __shared__ int32_t units[kMostCtas], of_warp[kThreads / 32];
  begin_kernel();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // The units that there are, in the same order in every CTA.
  int32_t count = 0;
  for (int i0 = 0; i0 < ctas; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const bool some = i < ctas && w.joins[i].parts > 0;
    const uint32_t m = __ballot_sync(~0u, some);
    __syncthreads();  // of_warp has been read
    if (lane == 0) of_warp[warp] = __popc(m);
    __syncthreads();
    int32_t before = count;
#pragma unroll
    for (int k = 0; k < kThreads / 32; ++k) {
      if (k < warp) before += of_warp[k];
      count += of_warp[k];
    }
    if (some) units[before + __popc(m & ((1u << lane) - 1))] = i;
  }
  __syncthreads();
  // (The maximum is held less 2^kUp, see Type.)
  const float up = c.type == P2P_KV_BF16 ? Type<P2P_KV_BF16>::kUp : Type<P2P_KV_F16>::kUp;
  const int columns = (c.dim + 32 * COLUMNS - 1) / (32 * COLUMNS), of_tile = 128 / kRowsOfWarp * columns;
  for (int y = blockIdx.x * (kThreads / 32) + warp; y < count * tiles * of_tile; y += gridDim.x * (kThreads / 32)) {
    const int x = y % of_tile, tile = y / of_tile % tiles, c0 = units[y / (of_tile * tiles)];
    const KvJoin u = w.joins[c0];
    const auto part_of = [&](int32_t k) { return w.parts + rows_part(c0 + k, k == 0, tiles, tile, dp); };
    const int r = x / columns * kRowsOfWarp + lane / 8, d0 = x % columns * (32 * COLUMNS) + lane % 8 * 4;
    if (r >= a.tile_rows || tile * a.tile_rows + r >= u.rows) continue;
    float m = -INFINITY, z = 0.f;
    float4 o[COLUMNS];
#pragma unroll
    for (int i = 0; i < COLUMNS; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kAhead = COLUMNS == 4 ? 3 : 4;
    for (int32_t k0 = 0; k0 < u.parts; k0 += kAhead) {
      float pm[kAhead], pz[kAhead];
      float4 po[kAhead][COLUMNS];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float* const p = part_of(min(k0 + k, u.parts - 1));
        pm[k] = __ldcg(p + dp * 128 + r), pz[k] = __ldcg(p + (dp + 1) * 128 + r);
#pragma unroll
        for (int i = 0; i < COLUMNS; ++i)
          po[k][i] = k0 + k < u.parts && d0 + 32 * i < c.dim ? __ldcg((const float4*)p + (d0 / 4 + 8 * i) * 128 + r)
                                                             : make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + k >= u.parts) pm[k] = -INFINITY, pz[k] = 0.f;
      }
      float most = m;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) most = fmaxf(most, pm[k]);
      const float ref = most == -INFINITY ? 0.f : most;
      float fade = exp2_fast(m - ref);
      m = most;
      z *= fade;
#pragma unroll
      for (int i = 0; i < COLUMNS; ++i) o[i].x *= fade, o[i].y *= fade, o[i].z *= fade, o[i].w *= fade;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        fade = exp2_fast(pm[k] - ref);
        z = fmaf(pz[k], fade, z);
#pragma unroll
        for (int i = 0; i < COLUMNS; ++i) {
          o[i].x = fmaf(po[k][i].x, fade, o[i].x), o[i].y = fmaf(po[k][i].y, fade, o[i].y);
          o[i].z = fmaf(po[k][i].z, fade, o[i].z), o[i].w = fmaf(po[k][i].w, fade, o[i].w);
        }
      }
    }
    const uint32_t at = u.g0 + tile * a.tile_rows + r, t = a.by_group.div(at);
    const int64_t row = u.row + t;
    const int32_t head = u.h * a.group + (int32_t)(at - t * a.group);
    const float v_scale = c.type == P2P_KV_E4M3 ? c.v_scale[a.layer * c.heads + u.h] : 1.f;
    const float f = z == 0.f && a.pre ? 0.f : v_scale / z;  // (as in kv_rows.cuh)
    if (d0 == 0 && a.pre) a.pre_sum[row * a.heads + head] = make_float2(m, z);
    if (d0 == 0 && !a.pre && a.lse)
      a.lse[row * a.heads + head] = z == 0.f ? -INFINITY : (m + up + __log2f(z * exp2f(-up))) * kLn2;
#pragma unroll
    for (int i = 0; i < COLUMNS; ++i) {
      const int d = d0 + 32 * i;
      if (d >= c.dim) continue;
      const float4 v = make_float4(o[i].x * f, o[i].y * f, o[i].z * f, o[i].w * f);
      if (a.pre) {
        *(float4*)(a.pre + (row * a.heads + head) * c.dim + d) = v;
        continue;
      }
      const uint32_t b0 = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(v.x, v.y) : pack<P2P_KV_F16>(v.x, v.y);
      const uint32_t b1 = a.type == P2P_KV_BF16 ? pack<P2P_KV_BF16>(v.z, v.w) : pack<P2P_KV_F16>(v.z, v.w);
      uint16_t* const to = (uint16_t*)a.out + row * a.out_row + head * a.out_head + d;
      if (a.out32) {
        *(uint2*)to = make_uint2(b0, b1);
      } else {
        to[0] = (uint16_t)b0, to[1] = (uint16_t)(b0 >> 16);
        to[2] = (uint16_t)b1, to[3] = (uint16_t)(b1 >> 16);
      }
    }
  }
}

}  // namespace

cudaError_t launch_kv_join(const KvView& c, const KvRowsCall& a, const KvAttendScratch& w, int num_sms,
                           cudaStream_t st) {
  const int dp = (c.dim + 63) / 64 * 64, tiles = dp <= 128 ? 2 : 1;
  if (num_sms > kMostCtas) return cudaErrorInvalidConfiguration;
  return launch_early(dp == 64 ? join_kernel<2> : join_kernel<4>, dim3(4 * num_sms), kThreads, 0, st, c, a, w,
                      (int32_t)num_sms, (int32_t)dp, (int32_t)tiles);
}

}  // namespace p2p
