// kv_pages.cu -- the page tables of the paged key-value cache: extend, trim, fork, compact, write (p2p_kv_*).
//
// A call on the tables is one cluster of eight CTAs.  Each of them checks every item, counts the page entries that it
// concerns and scans the counts in its own shared memory (for long lists the first CTA does, in scratch); the pool's
// reference counts are scanned in eight parts.  The CTAs tell each other what they found through shared memory and
// meet once; then, if every item was good, the entries are worked off as one flat range, so that one long sequence
// and many short ones take the same time.  Nothing is changed before that.  What bounds these calls is the chain of
// loads behind an item (its sequence, the length, the last page, its count), the cluster's meeting and the launch
// itself: 3.6 us for a trim of 33 sequences, 4.3 for an extend (one CTA instead of eight: 33 us for a trim of 20,000
// pages, 88 for an extend by them and 200 for a compaction's plan; eight: 11, 13 and 15).
//
// Pages are copied by a second launch over the whole GPU, from the list of copies that the plan leaves.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv_values.cuh"

// (No load here goes past the coherent path, as __ldg or const __restrict__ would have it: the kernel before may
// still be writing when this one starts, see launch_early.)
namespace p2p {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCluster = 8;
constexpr int kItems = 8192;  // items of a call whose plan fits shared memory

// What a CTA of the cluster tells the others.
struct Found {
  int64_t count, count2;
  int32_t err;
};
struct Plan {
  Found found[kCluster];
  int64_t warp_sum[kWarps];
  int32_t warp_count[kWarps];
  int32_t err, cuts;
};
// The items of a call: their first entry among the call's (start[n]: all), the first page entry they concern, and, for
// extend, the tokens of a shared last page that move to a page of their own (0: none).
struct Items {
  int32_t *start, *first, *cut;
};
extern __shared__ int32_t item_room[];
__device__ __forceinline__ Items items_of(const KvScratch& s, int32_t n) {
  if (n > kItems) return {s.start, s.first, s.cut};
  return {item_room, item_room + n + 1, item_room + 2 * n + 1};
}
size_t item_bytes(int32_t n) { return n > kItems ? 0 : (size_t)(3 * n + 1) * sizeof(int32_t); }

// Exclusive scan of one value a thread over the CTA; total: the sum.
__device__ int64_t block_scan(int64_t v, Plan& p, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // the words of an earlier scan have been read
  if (lane == 31) p.warp_sum[warp] = x;
  __syncthreads();
  int64_t w = p.warp_sum[lane], sum = w;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, sum, d);
    if (lane >= d) sum += y;
  }
  total = __shfl_sync(~0u, sum, 31);
  return __shfl_sync(~0u, sum - w, warp) + x - v;
}
static_assert(kWarps == 32, "a lane a warp");

// The item that entry r belongs to.
__device__ __forceinline__ int32_t item_of(const int32_t* start, int32_t n, int32_t r) {
  int32_t lo = 0, hi = n;  // start[lo] <= r < start[hi]
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (start[mid] <= r)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Fills in the items: item(i, need, first, cut) gives the entries that item i concerns, and its error bits.
template <class F>
__device__ void plan_items(Plan& p, const Items& it, int32_t n, F item) {
  int64_t carry = 0;
  for (int32_t i0 = 0; i0 < n; i0 += kThreads) {
    const int32_t i = i0 + threadIdx.x;
    int32_t need = 0, first = 0, cut = 0;
    if (i < n)
      if (const int32_t bad = item(i, need, first, cut)) atomicOr(&p.err, bad), need = 0;
    int64_t total;
    const int64_t at = carry + block_scan(need, p, total);
    if (i < n) it.start[i] = (int32_t)at, it.first[i] = first, it.cut[i] = cut;
    carry += total;
  }
  if (threadIdx.x == 0) {
    if (carry > INT32_MAX) p.err |= KV_BAD_COUNT;
    it.start[n] = (int32_t)carry;
  }
  __syncthreads();
}

// Tells the cluster what this CTA found and waits for the others; returns all their error bits.
__device__ int32_t meet(Plan& p, int64_t count, int64_t count2) {
  cg::cluster_group cluster = cg::this_cluster();
  __syncthreads();
  if (threadIdx.x < kCluster)
    *cluster.map_shared_rank(&p.found[cluster.block_rank()], threadIdx.x) = Found{count, count2, p.err};
  cluster.sync();
  int32_t err = 0;
#pragma unroll
  for (int k = 0; k < kCluster; ++k) err |= p.found[k].err;
  return err;
}

// This thread block's part of the pool, by warps: pages begin .. end of this warp.
struct Part {
  int32_t begin, end;
};
__device__ __forceinline__ Part part_of(const KvView& c, int rank) {
  const int32_t each = ((c.n_pages + kCluster * kWarps - 1) / (kCluster * kWarps) + 31) / 32 * 32;
  const int64_t begin = (int64_t)(rank * kWarps + (threadIdx.x >> 5)) * each;
  const int64_t n = c.n_pages;
  return {(int32_t)min(begin, n), (int32_t)min(begin + each, n)};
}
// The reference counts of the warp's pages, the first of them read at construction.
struct Counting {
  static constexpr int kFirst = 8;
  Part r;
  int32_t v[kFirst];
  __device__ __forceinline__ Counting(const KvView& c, const Part& part) : r(part) {
#pragma unroll
    for (int k = 0; k < kFirst; ++k) {
      const int32_t page = r.begin + (threadIdx.x & 31) + 32 * k;
      v[k] = page < r.end ? __ldcg(c.refs + page) : -1;
    }
  }
  // How many hold for `what`; every lane gets the sum.
  template <class F>
  __device__ __forceinline__ int32_t count(const KvView& c, F what) const {
    int32_t n = 0;
#pragma unroll
    for (int k = 0; k < kFirst; ++k) {
      const int32_t page = r.begin + (threadIdx.x & 31) + 32 * k;
      n += page < r.end && what(page, v[k]);
    }
#pragma unroll 8
    for (int32_t page = r.begin + (threadIdx.x & 31) + 32 * kFirst; page < r.end; page += 32)
      n += what(page, __ldcg(c.refs + page));
    return __reduce_add_sync(~0u, n);
  }
};
// How many of the warp's pages hold for `what`; every lane gets the sum.
template <class F>
__device__ __forceinline__ int32_t count_pages(const KvView& c, const Part& r, F what) {
  const int lane = threadIdx.x & 31;
  int32_t n = 0;
#pragma unroll 8
  for (int32_t page = r.begin + lane; page < r.end; page += 32) n += what(page, __ldcg(c.refs + page));
  return __reduce_add_sync(~0u, n);
}
// The warps' counts: this warp's place among the CTA's, and the CTA's sum.
__device__ int32_t scan_warps(Plan& p, int32_t mine, int32_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) p.warp_count[warp] = mine;
  __syncthreads();
  const int32_t v = p.warp_count[lane];
  total = __reduce_add_sync(~0u, v);
  return __reduce_add_sync(~0u, lane < warp ? v : 0);
}
// f(page, k) for the warp's pages that hold for `what`, k counting on from `at`; ends when k passes `most`.
template <class F, class G>
__device__ __forceinline__ void each_page(const KvView& c, const Part& r, int64_t at, int64_t most, F what, G f) {
  const int lane = threadIdx.x & 31;
  for (int32_t p0 = r.begin; p0 < r.end && at < most; p0 += 32) {
    const int32_t page = p0 + lane;
    const bool is = page < r.end && what(page, __ldcg(c.refs + page));
    const uint32_t m = __ballot_sync(~0u, is);
    const int64_t k = at + __popc(m & ((1u << lane) - 1));
    if (is && k < most) f(page, k);
    at += __popc(m);
  }
}

// Gives up the claims of a call's sequences; reports its errors and returns whether there are any.  (The first CTA.)
__device__ void settle(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, int32_t err) {
  for (int32_t i = threadIdx.x; i < n; i += kThreads)
    if ((uint32_t)seq[i] < (uint32_t)c.n_seqs) s.claim[seq[i]] = 0;
  if (err && threadIdx.x == 0) {
    atomicOr(s.err, err);
    *s.halt = 1;
  }
}
// (The first CTA alone marks the sequences: what it meets a second time was named twice.  The mark's old value is
// looked at after the item's other loads are on their way.)
__device__ __forceinline__ int32_t claim(const KvScratch& s, int32_t seq, bool first) {
  return first ? atomicExch(&s.claim[seq], 1) : 0;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    extend_kernel(KvView c, KvScratch s, int32_t n, const int32_t* seq, const int32_t* count) {
  __shared__ Plan p;
  begin_kernel();
  const int rank = (int)cg::this_cluster().block_rank();
  const int32_t halt = *s.halt;
  if (threadIdx.x == 0) {
    p.err = p.cuts = 0;
    if (rank == 0) *s.njobs = 0;
  }
  __syncthreads();
  const Part mine = part_of(c, rank);
  const auto is_free = [](int32_t, int32_t refs) { return refs == 0; };
  const Counting counting(c, mine);  // (the first pages' counts, on their way while the items are planned)
  const Items it = items_of(s, n);
  if (rank == 0 || n <= kItems)
    plan_items(p, it, n, [&](int32_t i, int32_t& need, int32_t& first, int32_t& cut) -> int32_t {
      const int32_t q = seq[i], add = count[i];
      if ((uint32_t)q >= (uint32_t)c.n_seqs) return KV_BAD_SEQ;
      const int32_t twice = claim(s, q, rank == 0), len = length_of(c, q);
      if (len < 0 || add < 0 || add > c.max_pages * c.page - len) return KV_BAD_COUNT;
      const int32_t have = (int32_t)c.by_page.ceil(len);
      need = (int32_t)c.by_page.ceil(len + add) - have;
      first = have;
      const int32_t used = len - (int32_t)c.by_page.div(len) * c.page;
      if (add > 0 && used > 0) {
        const int32_t last = row_of(c, q)[have - 1];
        const int32_t refs = (uint32_t)last < (uint32_t)c.n_pages ? __ldcg(c.refs + last) : 0;
        if (refs < 1) return KV_BAD_PAGE;
        if (refs > 1) cut = used, first = have - 1, need += 1, p.cuts = 1;
      }
      return twice ? KV_BAD_SEQ : 0;
    });
  int32_t free_here;
  const int32_t free_before = scan_warps(p, counting.count(c, is_free), free_here);
  int32_t err = meet(p, free_here, p.cuts);
  if (halt) {
    if (rank == 0) settle(c, s, n, seq, 0);
    return;
  }
  const int32_t total = it.start[n];
  int64_t at = free_before, all = 0;
#pragma unroll
  for (int k = 0; k < kCluster; ++k) {
    all += p.found[k].count;
    at += k < rank ? p.found[k].count : 0;
  }
  if (!err && total > all) err = KV_NO_PAGES;
  if (rank == 0) settle(c, s, n, seq, err);
  if (err) return;
  // The free pages, from the lowest on, go to the entries in their order.
  each_page(c, mine, at, total, is_free, [&](int32_t page, int64_t k) {
    const int32_t r = (int32_t)k, i = item_of(it.start, n, r), e = it.first[i] + r - it.start[i];
    int32_t* row = row_of(c, seq[i]);
    if (it.cut[i] && r == it.start[i]) s.jobs[atomicAdd(s.njobs, 1)] = KvJob{row[e], page, it.cut[i], 0};
    row[e] = page;
    c.refs[page] = 1;
  });
  if (p.found[0].count2) {
    cg::this_cluster().sync();  // (a page that all its sharers leave is free from here on, not for this call's entries)
    const int32_t jobs = __ldcg(s.njobs);
    for (int32_t k = rank * kThreads + threadIdx.x; k < jobs; k += kCluster * kThreads)
      atomicSub(&c.refs[__ldcg(&s.jobs[k].from)], 1);
  }
  if (rank == 0)
    for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[seq[i]] += count[i];
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    trim_kernel(KvView c, KvScratch s, int32_t n, const int32_t* seq, const int32_t* to) {
  __shared__ Plan p;
  begin_kernel();
  const int rank = (int)cg::this_cluster().block_rank();
  const int32_t halt = *s.halt;
  if (threadIdx.x == 0) p.err = 0;
  __syncthreads();
  const Items it = items_of(s, n);
  if (rank == 0 || n <= kItems)
    plan_items(p, it, n, [&](int32_t i, int32_t& need, int32_t& first, int32_t&) -> int32_t {
      const int32_t q = seq[i], keep = to[i];
      if ((uint32_t)q >= (uint32_t)c.n_seqs) return KV_BAD_SEQ;
      const int32_t twice = claim(s, q, rank == 0), len = length_of(c, q);
      if (len < 0 || keep < 0 || keep > len) return KV_BAD_COUNT;
      first = (int32_t)c.by_page.ceil(keep);
      need = (int32_t)c.by_page.ceil(len) - first;
      return twice ? KV_BAD_SEQ : 0;
    });
  const int32_t err = meet(p, 0, 0);
  if (halt) {
    if (rank == 0) settle(c, s, n, seq, 0);
    return;
  }
  if (rank == 0) settle(c, s, n, seq, err);
  if (err) return;
  const int32_t total = it.start[n];
  for (int64_t r = rank * kThreads + threadIdx.x; r < total; r += kCluster * kThreads) {
    const int32_t i = item_of(it.start, n, (int32_t)r);
    const int32_t page = row_of(c, seq[i])[it.first[i] + (int32_t)r - it.start[i]];
    if ((uint32_t)page >= (uint32_t)c.n_pages)
      atomicOr(s.err, KV_BAD_PAGE);
    else if (atomicSub(&c.refs[page], 1) < 1)
      atomicAdd(&c.refs[page], 1), atomicOr(s.err, KV_BAD_PAGE);
  }
  if (rank == 0)
    for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[seq[i]] = to[i];
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    fork_kernel(KvView c, KvScratch s, int32_t n, const int32_t* src, const int32_t* dst,
                const int32_t* tokens) {
  __shared__ Plan p;
  begin_kernel();
  const int rank = (int)cg::this_cluster().block_rank();
  const int32_t halt = *s.halt;
  if (threadIdx.x == 0) p.err = 0;
  __syncthreads();
  const Items it = items_of(s, n);
  if (rank == 0 || n <= kItems)
    plan_items(p, it, n, [&](int32_t i, int32_t& need, int32_t&, int32_t&) -> int32_t {
      const int32_t from = src[i], q = dst[i], take = tokens[i];
      if ((uint32_t)q >= (uint32_t)c.n_seqs || (uint32_t)from >= (uint32_t)c.n_seqs) return KV_BAD_SEQ;
      const int32_t twice = claim(s, q, rank == 0), len = length_of(c, from), held = c.length[q];
      if (len < 0 || take < 0 || take > len || held != 0) return KV_BAD_COUNT;
      need = (int32_t)c.by_page.ceil(take);
      return twice ? KV_BAD_SEQ : 0;
    });
  const int32_t err = meet(p, 0, 0);
  if (halt) {
    if (rank == 0) settle(c, s, n, dst, 0);
    return;
  }
  if (rank == 0) settle(c, s, n, dst, err);
  if (err) return;
  const int32_t total = it.start[n];
  for (int64_t r = rank * kThreads + threadIdx.x; r < total; r += kCluster * kThreads) {
    const int32_t i = item_of(it.start, n, (int32_t)r), e = (int32_t)r - it.start[i], page = row_of(c, src[i])[e];
    row_of(c, dst[i])[e] = page;
    if ((uint32_t)page >= (uint32_t)c.n_pages)
      atomicOr(s.err, KV_BAD_PAGE);
    else
      atomicAdd(&c.refs[page], 1);
  }
  if (rank == 0)
    for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[dst[i]] = tokens[i];
}

// Before a compaction: every length is one that the table holds, and every entry within it names a page in use; else
// an error's bits.  `warps` of them, of which this is number `warp`, share the sequences, `each` of them the entries
// of one.
constexpr int kChunk = 256;  // entries that a warp has on their way
__device__ __forceinline__ int32_t check_rows(const KvView& c, int32_t warp, int32_t warps, int32_t each) {
  const int lane = threadIdx.x & 31;
  const int32_t per_turn = warps / each;
  int32_t bad = 0;
  if (warp >= per_turn * each) return 0;
  for (int32_t q = warp / each; q < c.n_seqs; q += per_turn) {
    const int32_t len = length_of(c, q), used = len < 0 ? 0 : (int32_t)c.by_page.ceil(len);
    if (len < 0) bad |= KV_BAD_COUNT;
    const int32_t* row = row_of(c, q);
    for (int64_t e0 = (int64_t)(warp % each) * kChunk; e0 < used; e0 += (int64_t)each * kChunk) {
      int32_t page[kChunk / 32];
#pragma unroll
      for (int k = 0; k < kChunk / 32; ++k) {
        const int64_t e = e0 + 32 * k + lane;
        page[k] = e < used ? __ldcg(row + e) : 0;
      }
#pragma unroll
      for (int k = 0; k < kChunk / 32; ++k)
        if (e0 + 32 * k + lane < used)
          if ((uint32_t)page[k] >= (uint32_t)c.n_pages || __ldcg(c.refs + page[k]) < 1) bad |= KV_BAD_PAGE;
    }
  }
  return bad;
}
// How many warps a sequence, of those there are.
int32_t warps_each(const KvView& c, int32_t warps) {
  return std::max(1, std::min(warps / c.n_seqs, (c.max_pages - 1) / kChunk + 1));
}
constexpr int kCheckThreads = 256, kCheckCtas = 4;
__global__ void __launch_bounds__(kCheckThreads) check_kernel(KvView c, KvScratch s, int32_t each) {
  begin_kernel();
  const int32_t halt = *s.halt, warp = (int32_t)(blockIdx.x * kCheckThreads + threadIdx.x) >> 5;
  const int32_t bad = check_rows(c, warp, (int32_t)(gridDim.x * (kCheckThreads / 32)), each);
  if (bad && !halt) {
    atomicOr(s.err, bad);
    *s.halt = 1;
  }
}

// `live` pages are in use: those numbered live and up go to the free ones below, both in ascending order.  The k-th of
// either kind is job k's; list[page]: where a page goes (the tables follow in copy_pages_kernel).  With `each` the
// cluster checks the tables itself.
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    compact_kernel(KvView c, KvScratch s, int32_t each) {
  __shared__ Plan p;
  begin_kernel();
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank();
  if (threadIdx.x == 0) {
    p.err = 0;
    if (rank == 0) *s.njobs = 0, *s.live = c.n_pages;
  }
  if (*s.halt) return;
  __syncthreads();
  const Part mine = part_of(c, rank);
  if (each)
    if (const int32_t bad = check_rows(c, rank * kWarps + (threadIdx.x >> 5), kCluster * kWarps, each))
      atomicOr(&p.err, bad);
  int32_t used;
  scan_warps(p, count_pages(c, mine, [](int32_t, int32_t refs) { return refs > 0; }), used);
  if (const int32_t err = meet(p, used, 0)) {
    if (rank == 0 && threadIdx.x == 0) atomicOr(s.err, err), *s.halt = 1;
    return;
  }
  int64_t live = 0;
#pragma unroll
  for (int k = 0; k < kCluster; ++k) live += p.found[k].count;
  cluster.sync();  // p.found is written again
  const auto hole = [live](int32_t page, int32_t refs) { return page < live && refs <= 0; };
  const auto mover = [live](int32_t page, int32_t refs) { return page >= live && refs > 0; };
  int32_t holes, movers;
  int64_t h = scan_warps(p, count_pages(c, mine, hole), holes);
  int64_t m = scan_warps(p, count_pages(c, mine, mover), movers);
  meet(p, holes, movers);
  int64_t jobs = 0;
#pragma unroll
  for (int k = 0; k < kCluster; ++k) {
    jobs += p.found[k].count2;
    h += k < rank ? p.found[k].count : 0;
    m += k < rank ? p.found[k].count2 : 0;
  }
  each_page(c, mine, h, jobs, hole, [&](int32_t page, int64_t k) { s.jobs[k].to = page; });
  each_page(c, mine, m, jobs, mover, [&](int32_t page, int64_t k) {
    s.jobs[k].from = page;
    s.jobs[k].tokens = c.page;
  });
  cluster.sync();
  if (rank == 0 && threadIdx.x == 0) *s.njobs = (int32_t)jobs, *s.live = (int32_t)live;
  for (int64_t k = rank * kThreads + threadIdx.x; k < jobs; k += kCluster * kThreads) {
    const int4 j = __ldcg((const int4*)(s.jobs + k));  // from, to
    s.list[j.x] = j.y;
    c.refs[j.y] = c.refs[j.x];
    c.refs[j.x] = 0;
  }
}

// The copies of the plan before it, in 16-byte pieces.  A warp takes 32 pieces of a page, one a lane, in 1 <<
// PLANES_LOG of the 2 * n_layers arrays (keys and values of each layer) and, where those are fewer than kCopies,
// further 32 pieces, so that a lane has kCopies loads in flight whose places differ by strides alone.  Bound by the
// bytes read and written: 3.3 GB of pages moved (6.7 GB in all) in 1.04 ms on one GB300, 94% of the copy bandwidth.
constexpr int kCopies = 8, kCopyThreads = 256, kCopyCtas = 4;
struct PageShape {
  FastDiv by_row, by_token;  // pieces of a head's values of a token, and of a token
};
template <int PLANES_LOG>
__global__ void __launch_bounds__(kCopyThreads, kCopyCtas)
    copy_pages_kernel(KvView c, KvScratch s, PageShape g, int32_t moved) {
  begin_kernel();
  // (Loads past the first cache: this launch may have shared its SM with the plan's.)
  const int32_t njobs = __ldcg(s.njobs);
  if (moved && !__ldcg(s.halt)) {  // the tables of a compaction (which were found to hold together)
    const int32_t live = __ldcg(s.live);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int32_t q = blockIdx.x * (kCopyThreads / 32) + warp; q < c.n_seqs; q += gridDim.x * (kCopyThreads / 32)) {
      const int32_t used = (int32_t)c.by_page.ceil(c.length[q]);
      int32_t* row = row_of(c, q);
      for (int32_t e = lane; e < used; e += 32)
        if (const int32_t page = __ldcg(row + e); page >= live) row[e] = __ldcg(s.list + page);
    }
  }
  if (njobs == 0) return;
  constexpr int kPlanes = 1 << PLANES_LOG, kPieces = kCopies / kPlanes;
  const int lane = threadIdx.x & 31;
  const int32_t chunks = (c.page * (int32_t)g.by_token.d + 32 * kPieces - 1) / (32 * kPieces);
  const int32_t groups = (2 * c.n_layers + kPlanes - 1) / kPlanes;
  const int64_t items = (int64_t)njobs * groups * chunks;
  const int64_t all_warps = (int64_t)gridDim.x * (kCopyThreads / 32);
  for (int64_t x = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); x < items; x += all_warps) {
    const int64_t job = x / ((int64_t)groups * chunks);
    const int32_t rest = (int32_t)(x - job * groups * chunks), group = rest / chunks;
    // (Turned from job to job: where pages are copied in part, no warp has their used beginnings alone.)
    const int32_t chunk = (int32_t)((rest - group * chunks + job) % chunks);
    const int4 j = __ldcg((const int4*)(s.jobs + job));  // from, to, tokens
    const int64_t move = (int64_t)(j.y - j.x) * c.page_stride;
    int64_t at[kPieces];  // of the lane's pieces within their layer; -1: none
#pragma unroll
    for (int y = 0; y < kPieces; ++y) {
      const int32_t z = (chunk * kPieces + y) * 32 + lane;
      const uint32_t t = g.by_token.div(z), in = z - t * g.by_token.d, h = g.by_row.div(in);
      const int64_t in_page = t * c.token_stride + h * c.head_stride + (in - h * g.by_row.d) * 16;
      at[y] = (int32_t)t < j.z ? j.x * c.page_stride + in_page : -1;
    }
    const int32_t layer0 = group * (kPlanes / 2), layers = min(kPlanes / 2, c.n_layers - layer0);
    char *const k0 = c.k + layer0 * c.layer_stride, *const v0 = c.v + layer0 * c.layer_stride;
    uint4 v[kPieces][kPlanes];
#pragma unroll
    for (int y = 0; y < kPieces; ++y)
#pragma unroll
      for (int p = 0; p < kPlanes; ++p)
        if (at[y] >= 0 && p / 2 < layers)
          v[y][p] = __ldcg((const uint4*)((p & 1 ? v0 : k0) + p / 2 * c.layer_stride + at[y]));
#pragma unroll
    for (int y = 0; y < kPieces; ++y)
#pragma unroll
      for (int p = 0; p < kPlanes; ++p)
        if (at[y] >= 0 && p / 2 < layers)
          __stcg((uint4*)((p & 1 ? v0 : k0) + p / 2 * c.layer_stride + at[y] + move), v[y][p]);
  }
}

// ---- write ------------------------------------------------------------------------------------------------

// Where the tokens of a block go is found once, a lane a token, and serves all their heads in the layers and arrays
// that the CTA writes; the first values are read while it is found.  Bound by the bytes read and written: 61 prompts
// of 71,000 tokens, 2.3 GB of bf16 values in and 1.2 GB of 8-bit values out, in 0.53 ms on one GB300 (97% of the copy
// bandwidth).
constexpr int kBlock = 32, kWriteThreads = 256;
constexpr int kFactors = 4096;  // scales of a CTA at most, with 8-bit values: 32 KB of shared memory
static_assert(kBlock == 32, "a warp finds the places, all its lanes together");

// Rounding x / scale to 8 bits, x of at most 11 bits.  What must not happen is that a quotient close to the middle
// between two 8-bit values (a tie: T, odd and below 32, times a power of two) is rounded to it, or across it, first.
// It can for X / T alone that is next to the scale, X of 11 bits: two such ratios are 2^-16 apart, so that it is one
// of them at most, and it says on which side of their ties all quotients lie that are close to one.  So a product with
// a factor 2^-20 above the reciprocal (where the scale is above that ratio: below) rounds as the quotient does.  A
// scale of up to 12 bits can be such a ratio exactly, and is 2^-17 away from all others: there 32 bits of the quotient
// are enough, but for ties they have to be right, and the factor has two parts.  (By division and remainder for each
// value, the 61 prompts above take 597 us, not 534; rounded twice, 574.)
__device__ __forceinline__ bool ordinary(float scale) {
  return fabsf(scale) > 0x1p-60f && fabsf(scale) < 0x1p60f;
}
// The factor for a scale (x: 0 where it is of an extreme size), by the 16 lanes of a half warp, one for each T; every
// lane gets it.  Its second part, if not 0, has the sign of the first.
__device__ __forceinline__ float2 factor_of(float scale) {
  const uint32_t lane = threadIdx.x & 31, x = (__float_as_uint(scale) & 0x7fffff) | 0x800000;
  const uint32_t p = x * (2 * (lane & 15) + 1), n = 31 - __clz(p);  // scale * T, of n + 1 bits
  // beyond its first 11 bits, and 2^-18 of it
  const uint32_t rest = p & ((1u << (n - 10)) - 1), close = 1u << (n - 18);
  const uint32_t above = __ballot_sync(~0u, rest < close) >> (lane & 16) & 0xffff;
  if (!ordinary(scale)) return make_float2(0.f, 0.f);
  if ((x & 0xfff) == 0) {
    const float most = __frcp_rz(scale);
    return make_float2(most, fmaf(-scale, most, 1.f) * most);
  }
  const float inverse = __frcp_rn(scale);
  return make_float2(fmaf(inverse, above ? -0x1p-20f : 0x1p-20f, inverse), 0.f);
}
// 16 values, each by `divide`, to 8 bits.
template <bool BF16, class F>
__device__ __forceinline__ uint4 narrow16(const uint4& a, const uint4& b, F divide) {
  const uint32_t in[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = two_values<BF16>(in[2 * i]), y = two_values<BF16>(in[2 * i + 1]);
    out[i] = narrow(make_float2(divide(x.x), divide(x.y))) | narrow(make_float2(divide(y.x), divide(y.y))) << 16;
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}
// 8 * N values, with WIDE from a 16 * N-byte boundary.  (One load for 16: as two, each
// 32-byte sector is asked for twice, and 61 prompts in 8 bits take 760 us, not 575.)
template <bool WIDE, int N>
__device__ __forceinline__ void read_values(uint4 (&v)[N], const uint16_t* p) {
  if constexpr (WIDE && N == 2) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y), "=r"(v[1].z),
                   "=r"(v[1].w)
                 : "l"(p)
                 : "memory");
  } else if constexpr (WIDE) {
    v[0] = __ldcs((const uint4*)p);
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = p[8 * k + 2 * i] | (uint32_t)p[8 * k + 2 * i + 1] << 16;
      v[k] = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
}

// KIND: the cache's type, BF16: that of the values given.  A CTA takes a block of tokens and `share` of the 2 *
// n_layers arrays (keys and values of each layer).  by_token: 16-byte pieces of a token in one array, by_row: of a
// head.
template <int KIND, bool BF16, bool WIDE>
__global__ void __launch_bounds__(kWriteThreads)
    write_kernel(KvView c, KvScratch s, int32_t layer, int32_t n_layers, int32_t share, int32_t n, const int32_t* seq,
                 const int64_t* offsets, int64_t n_tokens, KvRows in, FastDiv by_token, FastDiv by_row) {
  __shared__ int64_t place[kBlock];  // of a token, within its layer; -1: it is not written
  extern __shared__ float2 factor[];  // 8-bit values: for the scales of the CTA's arrays and heads (see factor_of)
  begin_kernel();
  const int32_t halt = *s.halt;
  const int64_t t0 = (int64_t)blockIdx.x * kBlock;
  const int32_t tokens = (int32_t)min((int64_t)kBlock, n_tokens - t0);
  const int32_t a0 = blockIdx.y * share, a1 = min(a0 + share, 2 * n_layers);
  const uint32_t all = tokens * by_token.d * (uint32_t)(a1 - a0);
  // Values and loads of a piece, and pieces of a thread in flight.
  constexpr int kValues = KIND == P2P_KV_E4M3 ? 16 : 8, kLoads = kValues / 8, kAhead = 4 / kLoads;
  uint4 v[kAhead][kLoads];
  int32_t scaled[kAhead];  // the number of its scale among the CTA's
  char* to[kAhead];      // but for the token's place
  int32_t token[kAhead];  // of the block; -1: no piece
  const auto read = [&](uint32_t y0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t y = y0 + k * kWriteThreads;
      token[k] = -1;
      if (y >= all) continue;
      const uint32_t token_of = by_token.div(y), over = tokens == kBlock ? token_of / kBlock : token_of / tokens;
      const uint32_t t = token_of - over * tokens, array = a0 + over, z = y - token_of * by_token.d;
      const uint32_t h = by_row.div(z), piece = z - h * by_row.d;
      const int32_t l = array >> 1;
      const uint16_t* from = (const uint16_t*)(array & 1 ? in.v : in.k) + l * in.layer_stride +
          (t0 + t) * in.token_stride + h * in.head_stride + piece * kValues;
      read_values<WIDE>(v[k], from);
      scaled[k] = over * c.heads + h;
      to[k] = (array & 1 ? c.v : c.k) + (int64_t)(layer + l) * c.layer_stride + h * c.head_stride + piece * 16;
      token[k] = t;
    }
  };
  const auto scale_at = [&](int32_t i) {
    const int32_t over = i / c.heads, array = a0 + over;
    return (array & 1 ? c.v_scale : c.k_scale)[(layer + (array >> 1)) * c.heads + i - over * c.heads];
  };
  read(threadIdx.x);  // (on their way while it is found where they go)
  if (blockIdx.x == 0 && blockIdx.y == 0) check_offsets(offsets, n, n_tokens, s.err);
  if (threadIdx.x < kBlock) {
    int32_t pos;
    const int64_t at = place_of(c, s, n, seq, offsets, n_tokens, t0, halt, pos);
    place[threadIdx.x] = at;
  } else if (KIND == P2P_KV_E4M3) {  // (the other warps, a scale for each half of one)
    const int32_t scales = (a1 - a0) * c.heads, half = threadIdx.x >> 4 & 1;
    for (int32_t i0 = (threadIdx.x - kBlock) / 32 * 2; i0 < scales; i0 += (kWriteThreads - kBlock) / 16) {
      const float2 f = factor_of(scale_at(min(i0 + half, scales - 1)));
      if ((threadIdx.x & 15) == 0 && i0 + half < scales) factor[i0 + half] = f;
    }
  }
  __syncthreads();
  const auto write = [&]() {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t at = token[k] < 0 ? -1 : place[token[k]];
      if (at < 0) continue;
      if (KIND == P2P_KV_E4M3) {
        uint4 x;
        if (const float2 f = factor[scaled[k]]; f.x == 0.f) {
          const float scale = scale_at(scaled[k]);
          x = narrow16<BF16>(v[k][0], v[k][kLoads - 1], [&](float y) { return divide_extreme(y, scale); });
        } else if (f.y == 0.f) {
          x = narrow16<BF16>(v[k][0], v[k][kLoads - 1], [&](float y) { return y * f.x; });
        } else {
          x = narrow16<BF16>(v[k][0], v[k][kLoads - 1], [&](float y) { return fmaf(y, f.x, y * f.y); });
        }
        __stcs((uint4*)(to[k] + at), x);
      } else {
        __stcs((uint4*)(to[k] + at), v[k][0]);
      }
    }
  };
  write();
  for (uint32_t y0 = threadIdx.x + kAhead * kWriteThreads; y0 < all; y0 += kAhead * kWriteThreads) {
    read(y0);
    write();
  }
}

__global__ void __launch_bounds__(256) stats_kernel(KvView c, unsigned long long* out) {
  unsigned long long used = 0, shared = 0, top = 0, tokens = 0;
  const int32_t step = gridDim.x * blockDim.x;
  for (int32_t p = blockIdx.x * blockDim.x + threadIdx.x; p < c.n_pages; p += step) {
    const int32_t r = c.refs[p];
    used += r > 0;
    shared += r > 1;
    if (r > 0) top = p + 1;
  }
  for (int32_t q = blockIdx.x * blockDim.x + threadIdx.x; q < c.n_seqs; q += step) {
    const int32_t len = length_of(c, q);
    tokens += len > 0 ? len : 0;
  }
  if (used) atomicAdd(&out[0], used);
  if (shared) atomicAdd(&out[1], shared);
  if (top) atomicMax(&out[2], top);
  if (tokens) atomicAdd(&out[3], tokens);
}

cudaError_t launch_copies(const KvView& c, const KvScratch& s, bool moved, int num_sms, cudaStream_t st) {
  PageShape g;
  g.by_row = FastDiv((uint32_t)c.row16);
  g.by_token = FastDiv((uint32_t)(c.heads * c.row16));
  const auto kernel = c.n_layers == 1   ? copy_pages_kernel<1>
                      : c.n_layers == 2 ? copy_pages_kernel<2>
                                        : copy_pages_kernel<3>;
  return launch_early(kernel, dim3(kCopyCtas * num_sms), kCopyThreads, 0, st, c, s, g, (int32_t)moved);
}

template <int KIND, bool BF16, bool WIDE>
cudaError_t write_launch(const KvView& c, const KvScratch& s, int32_t layer, int32_t n_layers, int32_t n,
                         const int32_t* seq, const int64_t* offsets, int64_t n_tokens, const KvRows& rows, int num_sms,
                         cudaStream_t st) {
  const int64_t blocks = (n_tokens + kBlock - 1) / kBlock;
  // All arrays of a block of tokens in one CTA where there are many blocks, else as few as fill the GPU.
  const int64_t want = (8LL * num_sms + blocks - 1) / blocks;
  // (A CTA's pieces are counted in 32 bits.)
  int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / (kBlock * c.heads * c.row16));
  static_assert(kFactors >= 4 * 1024, "with all the heads there may be, those of all layers in a grid of 65,535");
  if (KIND == P2P_KV_E4M3) most = std::min<int64_t>(most, kFactors / c.heads);
  const int64_t arrays = 2 * n_layers;
  const int32_t share = (int32_t)std::min(most, std::max<int64_t>(1, arrays / std::min(want, arrays)));
  const dim3 grid((unsigned)blocks, (unsigned)((2 * n_layers + share - 1) / share));
  const size_t factors = KIND == P2P_KV_E4M3 ? sizeof(float2) * share * c.heads : 0;
  return launch_early(write_kernel<KIND, BF16, WIDE>, grid, kWriteThreads, factors, st, c, s, layer, n_layers, share, n,
                      seq, offsets, n_tokens, rows, FastDiv((uint32_t)(c.heads * c.row16)),
                      FastDiv((uint32_t)c.row16));
}

template <int KIND, bool BF16>
cudaError_t write_wide(bool wide, const KvView& c, const KvScratch& s, int32_t layer, int32_t n_layers, int32_t n,
                       const int32_t* seq, const int64_t* offsets, int64_t n_tokens, const KvRows& rows, int num_sms,
                       cudaStream_t st) {
  return wide ? write_launch<KIND, BF16, true>(c, s, layer, n_layers, n, seq, offsets, n_tokens, rows, num_sms, st)
              : write_launch<KIND, BF16, false>(c, s, layer, n_layers, n, seq, offsets, n_tokens, rows, num_sms, st);
}

}  // namespace

cudaError_t prepare_kv_pages() {
  const int bytes = (int)item_bytes(kItems);
  cudaError_t e = cudaFuncSetAttribute(extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(trim_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e;
}

cudaError_t launch_kv_extend(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* count,
                             int num_sms, cudaStream_t st) {
  const cudaError_t e = launch_early(extend_kernel, dim3(kCluster), kThreads, item_bytes(n), st, c, s, n, seq, count);
  return e == cudaSuccess ? launch_copies(c, s, false, num_sms, st) : e;
}

cudaError_t launch_kv_trim(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* to,
                           cudaStream_t st) {
  return launch_early(trim_kernel, dim3(kCluster), kThreads, item_bytes(n), st, c, s, n, seq, to);
}

cudaError_t launch_kv_fork(const KvView& c, const KvScratch& s, int32_t n, const int32_t* src, const int32_t* dst,
                           const int32_t* tokens, cudaStream_t st) {
  return launch_early(fork_kernel, dim3(kCluster), kThreads, item_bytes(n), st, c, s, n, src, dst, tokens);
}

cudaError_t launch_kv_compact(const KvView& c, const KvScratch& s, int num_sms, cudaStream_t st,
                              int* launches) {
  // Tables of as many chunks as the plan has warps are checked there, larger ones by a launch of their own over the
  // whole GPU: a compaction that finds nothing to move takes, with 40 sequences of 72 pages, 9.5 us (10.3 with the
  // launch, 7.6 without a check), with 600 of 136 14.0 (15.9 by the plan, 10.5), with 200,000 of 3 102 (658, 38).
  int32_t each = warps_each(c, kCluster * kWarps);
  cudaError_t e = cudaSuccess;
  *launches = 2;
  if ((int64_t)c.n_seqs * ((c.max_pages - 1) / kChunk + 1) > kCluster * kWarps) {
    each = warps_each(c, kCheckCtas * num_sms * (kCheckThreads / 32));
    e = launch_early(check_kernel, dim3(kCheckCtas * num_sms), kCheckThreads, 0, st, c, s, each);
    each = 0;
    *launches = 3;
  }
  if (e == cudaSuccess) e = launch_early(compact_kernel, dim3(kCluster), kThreads, 0, st, c, s, each);
  return e == cudaSuccess ? launch_copies(c, s, true, num_sms, st) : e;
}

cudaError_t launch_kv_write(const KvView& c, const KvScratch& s, int32_t layer, int32_t n_layers, int32_t n,
                            const int32_t* seq, const int64_t* offsets, int64_t n_tokens, const KvRows& rows,
                            int num_sms, cudaStream_t st) {
  const int64_t values = c.type == P2P_KV_E4M3 ? 16 : 8;  // that are read together
  const bool wide = (uintptr_t)rows.k % (2 * values) == 0 && (uintptr_t)rows.v % (2 * values) == 0 &&
      rows.layer_stride % values == 0 &&
                    rows.token_stride % values == 0 && rows.head_stride % values == 0;
  if (c.type != P2P_KV_E4M3)  // (16-bit values are stored as they are)
    return write_wide<P2P_KV_BF16, true>(wide, c, s, layer, n_layers, n, seq, offsets, n_tokens, rows, num_sms, st);
  return rows.type == P2P_KV_BF16
             ? write_wide<P2P_KV_E4M3, true>(wide, c, s, layer, n_layers, n, seq, offsets, n_tokens, rows, num_sms, st)
             : write_wide<P2P_KV_E4M3, false>(wide, c, s, layer, n_layers, n, seq, offsets, n_tokens, rows, num_sms,
                 st);
}

cudaError_t launch_kv_stats(const KvView& c, unsigned long long* out, int num_sms, cudaStream_t st) {
  cudaError_t e = cudaMemsetAsync(out, 0, 4 * sizeof(*out), st);
  if (e != cudaSuccess) return e;
  stats_kernel<<<2 * num_sms, 256, 0, st>>>(c, out);
  return cudaGetLastError();
}

}  // namespace p2p
