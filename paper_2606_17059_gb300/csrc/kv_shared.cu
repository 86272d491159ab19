// kv_shared.cu -- what the rows of a group share (p2p_kv_attend_shared): the leading page entries that are the same in
// all of them.
//
// One cluster of eight CTAs: a warp compares a row's entries with those of its group's first row, 256 at a time, and the
// group keeps the least; then, if that saves enough, every row learns how many of its tokens are left to the group.
// Bound by the chain of loads behind a row (its group, sequence, length, entries) and three meetings, not by the bytes:
// under ncu (cold) 8.5 us for 64 rows of 64 entries, 10.5 for 200 of 512.
#include <cooperative_groups.h>

#include "kv_values.cuh"

namespace p2p {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 1024, kCluster = 8, kAhead = 8;

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    share_kernel(KvView c, int32_t* err, int32_t n, const int32_t* seq, int32_t n_groups, const int32_t* groups,
                 int32_t window, int64_t least, int32_t* skip, int4* spans) {
  __shared__ unsigned long long saved;  // (two's complement: groups of few rows count below 0)
  begin_kernel();
  if (threadIdx.x == 0) saved = 0;
  cg::cluster_group cluster = cg::this_cluster();
  const int lane = threadIdx.x & 31, rank = (int)cluster.block_rank();
  const int32_t me = rank * kThreads + threadIdx.x, all = kCluster * kThreads;
  int32_t bad = 0;
  for (int32_t g = threadIdx.x; g < n_groups; g += kThreads)
    bad |= groups[g] < 0 || groups[g + 1] < groups[g] || groups[g + 1] > n;
  bad = __syncthreads_or(bad);
  if (bad && me == 0) atomicOr(err, KV_BAD_OFFSETS);
  for (int32_t g = me; g < n_groups; g += all) spans[g] = make_int4(bad ? 0 : INT32_MAX, INT32_MAX, 0, 0);
  for (int32_t i = me; i < n; i += all) skip[i] = 0;
  if (bad || n_groups == 0) return;  // (every CTA finds the same)
  __threadfence();
  cluster.sync();
  const auto length = [&](int32_t s) { return (uint32_t)s < (uint32_t)c.n_seqs ? max(length_of(c, s), 0) : 0; };
  for (int32_t i = me / 32; i < n; i += all / 32) {
    const int32_t g = find_item(groups, n_groups, i), r0 = groups[g];
    if (i < r0 || i >= groups[g + 1]) continue;
    const int32_t s = seq ? seq[i] : i, s0 = seq ? seq[r0] : r0, len = length(s), len0 = length(s0);
    int32_t same = (int32_t)c.by_page.div(min(len, len0));
    if (s != s0 && same > 0) {
      const int32_t *mine = row_of(c, s), *his = row_of(c, s0);
      for (int32_t e0 = 0; e0 < same; e0 += 32 * kAhead) {
        int32_t a[kAhead], b[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int32_t e = e0 + 32 * k + lane;
          a[k] = e < same ? mine[e] : 0, b[k] = e < same ? his[e] : 0;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (const uint32_t m = __ballot_sync(~0u, a[k] != b[k])) same = min(same, e0 + 32 * k + __ffs(m) - 1);
      }
    }
    if (lane == 0) {
      const int32_t begin = window && len > window ? len - window : 0;
      atomicMin(&spans[g].x, same);
      atomicMin(&spans[g].y, begin);
      atomicMax(&spans[g].z, begin);
    }
  }
  __threadfence();
  cluster.sync();
  if (least > 0) {  // (tokens of rows that are not read again: by every CTA, so that all decide alike)
    unsigned long long mine = 0;
    for (int32_t g = threadIdx.x; g < n_groups; g += kThreads) {
      const int4 span = __ldcg(spans + g);
      const int32_t members = groups[g + 1] - groups[g], tokens = shared_tokens(c, span, members);
      const int32_t begin = (int32_t)(((int64_t)span.y + span.z) / 2);
      if (tokens > begin) mine += (unsigned long long)((int64_t)(members - kTogether) * (tokens - begin));
    }
    if (mine) atomicAdd(&saved, mine);
    cluster.sync();
    if ((long long)saved < least) {  // not worth two launches' work: every row by itself
      for (int32_t g = me; g < n_groups; g += all) spans[g].x = 0;
      return;
    }
  }
  for (int32_t i0 = me / 32 * 32; i0 < n; i0 += all) {
    int32_t lo = find_item(groups, n_groups, i0), hi = min(n_groups, find_item(groups, n_groups, i0 + 31) + 1);
    const int32_t i = i0 + lane;
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) >> 1;
      if (groups[mid] <= i)
        lo = mid;
      else
        hi = mid;
    }
    const int32_t r0 = groups[lo], r1 = groups[lo + 1];
    if (i < n && i >= r0 && i < r1) skip[i] = shared_tokens(c, __ldcg(spans + lo), r1 - r0);
  }
}

// Groups that are not made use of are looked at all the same.
__global__ void __launch_bounds__(kThreads)
    check_kernel(int32_t* err, int32_t n, int32_t n_groups, const int32_t* groups) {
  begin_kernel();
  for (int32_t g = threadIdx.x; g < n_groups; g += kThreads)
    if (groups[g] < 0 || groups[g + 1] < groups[g] || groups[g + 1] > n) atomicOr(err, KV_BAD_OFFSETS);
}

}  // namespace

cudaError_t launch_kv_share(const KvView& c, int32_t* err, int32_t n, const int32_t* seq, int32_t n_groups,
                            const int32_t* groups, int32_t window, int64_t least, int32_t* skip, int4* spans,
                            cudaStream_t st) {
  return launch_early(share_kernel, dim3(kCluster), kThreads, 0, st, c, err, n, seq, n_groups, groups, window, least,
                      skip, spans);
}

cudaError_t launch_kv_groups(int32_t* err, int32_t n, int32_t n_groups, const int32_t* groups, cudaStream_t st) {
  return launch_early(check_kernel, dim3(1), kThreads, 0, st, err, n, n_groups, groups);
}

}  // namespace p2p
