// kv_pages.cu -- the page tables of the paged key-value cache: extend, trim, fork, compact, write (p2p_kv_*).
//
// A call over a list of sequences is planned by one CTA: every item is checked, the page entries it concerns are
// counted and scanned, and the entries are then worked off as one flat range, so that one long sequence and many short
// ones take the same time.  Nothing is changed before every item has been found good.  Pages are copied by a second
// launch over the whole GPU from the list of copies that the plan leaves.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv.h"

namespace p2p {
namespace {

constexpr int kThreads = 1024;

// Exclusive scan of one value a thread over the CTA; total: the sum.  (warp_sum: one word a warp.)
__device__ int64_t block_scan(int64_t v, int64_t* warp_sum, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t x = v;
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();  // the words of an earlier scan have been read
  if (lane == 31) warp_sum[warp] = x;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += warp_sum[w];
    all += warp_sum[w];
  }
  total = all;
  return before + x - v;
}

struct Plan {  // shared memory of a planning CTA
  int32_t err;
  int64_t warp_sum[kThreads / 32];
};

// The item (index into start[0 .. n], start[n] = total) that entry r belongs to.
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

// Counts of the items (in start[]) -> their exclusive scan in place; returns the total, or -1 (and an error bit) where it
// does not fit the table's entries.
__device__ int64_t scan_items(int32_t* start, int32_t n, Plan& p) {
  int64_t carry = 0;
  for (int32_t i0 = 0; i0 < n; i0 += kThreads) {
    const int32_t i = i0 + threadIdx.x;
    int64_t total;
    const int64_t at = carry + block_scan(i < n ? start[i] : 0, p.warp_sum, total);
    if (i < n) start[i] = (int32_t)at;
    carry += total;
    if (carry > INT32_MAX) return -1;
  }
  if (threadIdx.x == 0) start[n] = (int32_t)carry;
  __syncthreads();
  return carry;
}

// Gives up the claims of a call's sequences and reports its errors; true if there are any.
__device__ bool settle(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, int32_t err) {
  for (int32_t i = threadIdx.x; i < n; i += kThreads)
    if ((uint32_t)seq[i] < (uint32_t)c.n_seqs) s.claim[seq[i]] = 0;
  if (err && threadIdx.x == 0) {
    atomicOr(s.err, err);
    *s.halt = 1;
  }
  return err != 0;
}

__device__ __forceinline__ int32_t claim(const KvView& c, const KvScratch& s, int32_t seq) {
  if ((uint32_t)seq >= (uint32_t)c.n_seqs) return KV_BAD_SEQ;
  return atomicExch(&s.claim[seq], 1) ? KV_BAD_SEQ : 0;
}

// A length as the table can hold it, or -1.
__device__ __forceinline__ int32_t length_of(const KvView& c, int32_t seq) {
  const int32_t n = c.length[seq];
  return n >= 0 && n <= c.max_pages * c.page ? n : -1;
}
__device__ __forceinline__ int32_t* row_of(const KvView& c, int32_t seq) { return c.table + (int64_t)seq * c.max_pages; }

__global__ void __launch_bounds__(kThreads) extend_kernel(KvView c, KvScratch s, int32_t n, const int32_t* __restrict__ seq,
                                                          const int32_t* __restrict__ count) {
  __shared__ Plan p;
  if (threadIdx.x == 0) p.err = 0, *s.njobs = 0;
  __syncthreads();
  if (*s.halt) return;
  for (int32_t i = threadIdx.x; i < n; i += kThreads) {
    int32_t need = 0, first = 0, cut = 0;
    int32_t bad = claim(c, s, seq[i]);
    if (!bad) {
      const int32_t len = length_of(c, seq[i]), add = count[i];
      if (len < 0 || add < 0 || add > c.max_pages * c.page - len) {
        bad = KV_BAD_COUNT;
      } else {
        const int32_t have = (int32_t)c.by_page.ceil(len);
        need = (int32_t)c.by_page.ceil(len + add) - have;
        first = have;
        const int32_t used = len - (int32_t)c.by_page.div(len) * c.page;
        if (add > 0 && used > 0) {
          const int32_t last = row_of(c, seq[i])[have - 1];
          if ((uint32_t)last >= (uint32_t)c.n_pages || c.refs[last] < 1)
            bad = KV_BAD_PAGE;
          else if (c.refs[last] > 1)
            cut = used, first = have - 1, need += 1;
        }
      }
    }
    if (bad) atomicOr(&p.err, bad);
    s.start[i] = need;
    s.first[i] = first;
    s.cut[i] = cut;
  }
  __syncthreads();
  int64_t total = p.err ? 0 : scan_items(s.start, n, p);
  // The lowest free pages, as many as are needed.
  int64_t found = 0;
  if (!p.err && total > c.n_pages) total = -1;
  if (!p.err && total > 0) {
    for (int32_t p0 = 0; p0 < c.n_pages && found < total; p0 += kThreads) {
      const int32_t page = p0 + threadIdx.x;
      const bool free = page < c.n_pages && c.refs[page] == 0;
      int64_t here;
      const int64_t at = found + block_scan(free, p.warp_sum, here);
      if (free && at < total) s.list[at] = page;
      found += here;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && !p.err && (total < 0 || found < total)) p.err = KV_NO_PAGES;
  __syncthreads();
  if (settle(c, s, n, seq, p.err)) return;
  for (int32_t r = threadIdx.x; r < total; r += kThreads) {
    const int32_t i = item_of(s.start, n, r), e = s.first[i] + r - s.start[i], page = s.list[r];
    int32_t* row = row_of(c, seq[i]);
    if (s.cut[i] && r == s.start[i]) {
      const int32_t old = row[e];
      atomicSub(&c.refs[old], 1);
      s.jobs[atomicAdd(s.njobs, 1)] = KvJob{old, page, s.cut[i]};
    }
    row[e] = page;
    c.refs[page] = 1;
  }
  for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[seq[i]] += count[i];
}

__global__ void __launch_bounds__(kThreads) trim_kernel(KvView c, KvScratch s, int32_t n, const int32_t* __restrict__ seq,
                                                        const int32_t* __restrict__ to) {
  __shared__ Plan p;
  if (threadIdx.x == 0) p.err = 0;
  __syncthreads();
  if (*s.halt) return;
  for (int32_t i = threadIdx.x; i < n; i += kThreads) {
    int32_t need = 0, keep = 0;
    int32_t bad = claim(c, s, seq[i]);
    if (!bad) {
      const int32_t len = length_of(c, seq[i]);
      if (len < 0 || to[i] < 0 || to[i] > len) {
        bad = KV_BAD_COUNT;
      } else {
        keep = (int32_t)c.by_page.ceil(to[i]);
        need = (int32_t)c.by_page.ceil(len) - keep;
      }
    }
    if (bad) atomicOr(&p.err, bad);
    s.start[i] = need;
    s.first[i] = keep;
  }
  __syncthreads();
  int64_t total = p.err ? 0 : scan_items(s.start, n, p);
  __syncthreads();
  if (threadIdx.x == 0 && total < 0) p.err = KV_BAD_COUNT;
  __syncthreads();
  if (settle(c, s, n, seq, p.err)) return;
  for (int32_t r = threadIdx.x; r < total; r += kThreads) {
    const int32_t i = item_of(s.start, n, r), page = row_of(c, seq[i])[s.first[i] + r - s.start[i]];
    if ((uint32_t)page >= (uint32_t)c.n_pages)
      atomicOr(s.err, KV_BAD_PAGE);
    else if (atomicSub(&c.refs[page], 1) < 1)
      atomicAdd(&c.refs[page], 1), atomicOr(s.err, KV_BAD_PAGE);
  }
  for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[seq[i]] = to[i];
}

__global__ void __launch_bounds__(kThreads) fork_kernel(KvView c, KvScratch s, int32_t n, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst, const int32_t* __restrict__ tokens) {
  __shared__ Plan p;
  if (threadIdx.x == 0) p.err = 0;
  __syncthreads();
  if (*s.halt) return;
  for (int32_t i = threadIdx.x; i < n; i += kThreads) {
    int32_t need = 0;
    int32_t bad = claim(c, s, dst[i]);
    if (!bad && (uint32_t)src[i] >= (uint32_t)c.n_seqs) bad = KV_BAD_SEQ;
    if (!bad) {
      const int32_t len = length_of(c, src[i]);
      if (len < 0 || tokens[i] < 0 || tokens[i] > len || c.length[dst[i]] != 0)
        bad = KV_BAD_COUNT;
      else
        need = (int32_t)c.by_page.ceil(tokens[i]);
    }
    if (bad) atomicOr(&p.err, bad);
    s.start[i] = need;
  }
  __syncthreads();
  int64_t total = p.err ? 0 : scan_items(s.start, n, p);
  __syncthreads();
  if (threadIdx.x == 0 && total < 0) p.err = KV_BAD_COUNT;
  __syncthreads();
  if (settle(c, s, n, dst, p.err)) return;
  for (int32_t r = threadIdx.x; r < total; r += kThreads) {
    const int32_t i = item_of(s.start, n, r), e = r - s.start[i], page = row_of(c, src[i])[e];
    row_of(c, dst[i])[e] = page;
    if ((uint32_t)page >= (uint32_t)c.n_pages)
      atomicOr(s.err, KV_BAD_PAGE);
    else
      atomicAdd(&c.refs[page], 1);
  }
  for (int32_t i = threadIdx.x; i < n; i += kThreads) c.length[dst[i]] = tokens[i];
}

// n_live pages are in use: those at n_live and beyond go to the free ones below, both in ascending order.  list[page] =
// where a page goes; the copies become jobs.
__global__ void __launch_bounds__(kThreads) compact_kernel(KvView c, KvScratch s) {
  __shared__ Plan p;
  if (threadIdx.x == 0) *s.njobs = 0;
  __syncthreads();
  if (*s.halt) return;
  int64_t live = 0;
  for (int32_t p0 = 0; p0 < c.n_pages; p0 += kThreads) {
    const int32_t page = p0 + threadIdx.x;
    int64_t here;
    block_scan(page < c.n_pages && c.refs[page] > 0, p.warp_sum, here);
    live += here;
  }
  int64_t holes = 0, movers = 0;
  for (int32_t p0 = 0; p0 < c.n_pages; p0 += kThreads) {
    const int32_t page = p0 + threadIdx.x;
    const bool in = page < c.n_pages, used = in && c.refs[page] > 0, hole = in && page < live && !used, mover = used && page >= live;
    int64_t nh, nm;
    const int64_t h = holes + block_scan(hole, p.warp_sum, nh), m = movers + block_scan(mover, p.warp_sum, nm);
    if (hole) s.jobs[h].to = page;
    if (mover) s.jobs[m].from = page, s.jobs[m].tokens = c.page;
    holes += nh;
    movers += nm;
  }
  __syncthreads();
  if (threadIdx.x == 0) *s.njobs = (int32_t)movers;
  for (int32_t m = threadIdx.x; m < movers; m += kThreads) {
    const KvJob j = s.jobs[m];
    s.list[j.from] = j.to;
    c.refs[j.to] = c.refs[j.from];
    c.refs[j.from] = 0;
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int32_t q = warp; q < c.n_seqs; q += kThreads / 32) {
    const int32_t len = length_of(c, q), used = len < 0 ? 0 : (int32_t)c.by_page.ceil(len);
    if (len < 0 && lane == 0) atomicOr(s.err, KV_BAD_COUNT);
    int32_t* row = row_of(c, q);
    for (int32_t e = lane; e < used; e += 32) {
      const int32_t page = row[e];
      if ((uint32_t)page >= (uint32_t)c.n_pages)
        atomicOr(s.err, KV_BAD_PAGE);
      else if (page >= live)
        row[e] = s.list[page];
    }
  }
}

// The copies of the plan before it: one CTA a page, layer and array (keys or values) at a time.
__global__ void __launch_bounds__(256) copy_pages_kernel(KvView c, KvScratch s) {
  const int64_t items = (int64_t)*s.njobs * c.n_layers * 2;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int32_t what = (int32_t)(x % (2 * c.n_layers));
    const KvJob j = s.jobs[x / (2 * c.n_layers)];
    char* base = (what & 1 ? c.v : c.k) + (what >> 1) * c.layer_stride;
    for (int32_t y = threadIdx.x; y < j.tokens * c.heads * c.row16; y += blockDim.x) {
      const int32_t piece = y % c.row16, t = y / c.row16 / c.heads, h = y / c.row16 % c.heads;
      const int64_t at = t * c.token_stride + h * c.head_stride + piece * 16;
      *(uint4*)(base + j.to * c.page_stride + at) = *(const uint4*)(base + j.from * c.page_stride + at);
    }
  }
}

// ---- write ------------------------------------------------------------------------------------------------

__device__ __forceinline__ float load_half(const void* p, int64_t i, int32_t type) {
  return type == P2P_KV_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i]) : __half2float(((const __half*)p)[i]);
}

// One 16-byte piece of a head's values of a token a thread.
__global__ void __launch_bounds__(256) write_kernel(KvView c, KvScratch s, int32_t layer, int32_t n, const int32_t* __restrict__ seq,
                                                    const int64_t* __restrict__ offsets, int64_t n_tokens, KvRows in) {
  if (*s.halt) return;
  const int32_t which = blockIdx.y & 1, l = blockIdx.y >> 1;
  const void* src = which ? in.v : in.k;
  char* dst = (which ? c.v : c.k) + (int64_t)(layer + l) * c.layer_stride;
  const int64_t items = n_tokens * c.heads * c.row16;
  for (int64_t x = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; x < items; x += (int64_t)gridDim.x * blockDim.x) {
    const int32_t piece = (int32_t)(x % c.row16), h = (int32_t)(x / c.row16 % c.heads);
    const int64_t t = x / c.row16 / c.heads;
    // The last item that starts at or before t (items without tokens share a start).
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
      const int32_t mid = (lo + hi) >> 1;
      if (offsets[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    const int64_t o0 = offsets[lo], o1 = offsets[lo + 1];
    if (o0 > t || o1 <= t) {
      // Tokens outside [offsets[0], offsets[n]) belong to no sequence.
      if (o0 < 0 || o1 > n_tokens || o1 < o0) atomicOr(s.err, KV_BAD_OFFSETS);
      continue;
    }
    const int32_t q = seq[lo];
    if ((uint32_t)q >= (uint32_t)c.n_seqs) {
      atomicOr(s.err, KV_BAD_SEQ);
      continue;
    }
    const int32_t len = length_of(c, q);
    if (len < 0 || o0 < 0 || o1 > n_tokens || o1 - o0 > len) {
      atomicOr(s.err, len < 0 || o1 - o0 > len ? KV_BAD_COUNT : KV_BAD_OFFSETS);
      continue;
    }
    const int32_t pos = len - (int32_t)(o1 - t), e = (int32_t)c.by_page.div(pos), page = row_of(c, q)[e];
    if ((uint32_t)page >= (uint32_t)c.n_pages) {
      atomicOr(s.err, KV_BAD_PAGE);
      continue;
    }
    if (c.refs[page] != 1) {
      atomicOr(s.err, c.refs[page] > 1 ? KV_SHARED : KV_BAD_PAGE);
      continue;
    }
    const int32_t per = c.type == P2P_KV_E4M3 ? 16 : 8;
    const int64_t from = l * in.layer_stride + t * in.token_stride + h * in.head_stride + piece * per;
    char* to = dst + page * c.page_stride + (pos - e * c.page) * c.token_stride + h * c.head_stride + piece * 16;
    uint4 w;
    if (c.type == P2P_KV_E4M3) {
      const float scale = (which ? c.v_scale : c.k_scale)[(layer + l) * c.heads + h];
      uint8_t* b = (uint8_t*)&w;
      for (int i = 0; i < 16; ++i)
        b[i] = __nv_cvt_float_to_fp8(__fdiv_rn(load_half(src, from + i, in.type), scale), __NV_SATFINITE, __NV_E4M3);
    } else {
      uint16_t* b = (uint16_t*)&w;
      for (int i = 0; i < 8; ++i) b[i] = ((const uint16_t*)src)[from + i];
    }
    *(uint4*)to = w;
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

cudaError_t launch_copies(const KvView& c, const KvScratch& s, int num_sms, cudaStream_t st) {
  copy_pages_kernel<<<8 * num_sms, 256, 0, st>>>(c, s);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_extend(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* count, int num_sms,
                             cudaStream_t st) {
  extend_kernel<<<1, kThreads, 0, st>>>(c, s, n, seq, count);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? launch_copies(c, s, num_sms, st) : e;
}

cudaError_t launch_kv_trim(const KvView& c, const KvScratch& s, int32_t n, const int32_t* seq, const int32_t* to, cudaStream_t st) {
  trim_kernel<<<1, kThreads, 0, st>>>(c, s, n, seq, to);
  return cudaGetLastError();
}

cudaError_t launch_kv_fork(const KvView& c, const KvScratch& s, int32_t n, const int32_t* src, const int32_t* dst,
                           const int32_t* tokens, cudaStream_t st) {
  fork_kernel<<<1, kThreads, 0, st>>>(c, s, n, src, dst, tokens);
  return cudaGetLastError();
}

cudaError_t launch_kv_compact(const KvView& c, const KvScratch& s, int num_sms, cudaStream_t st) {
  compact_kernel<<<1, kThreads, 0, st>>>(c, s);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? launch_copies(c, s, num_sms, st) : e;
}

cudaError_t launch_kv_write(const KvView& c, const KvScratch& s, int32_t layer, int32_t n_layers, int32_t n, const int32_t* seq,
                            const int64_t* offsets, int64_t n_tokens, const KvRows& rows, int num_sms, cudaStream_t st) {
  const int64_t items = n_tokens * c.heads * c.row16;
  for (int32_t l = 0; l < n_layers; l += 16384) {  // (a grid has at most 65,535 blocks in y)
    const int32_t m = n_layers - l < 16384 ? n_layers - l : 16384;
    const int64_t blocks = (items + 255) / 256, most = (16LL * num_sms + 2 * m - 1) / (2 * m);
    KvRows r = rows;
    r.k = (const char*)rows.k + l * rows.layer_stride * 2;
    r.v = (const char*)rows.v + l * rows.layer_stride * 2;
    write_kernel<<<dim3((unsigned)(blocks < most ? blocks : most), 2 * m), 256, 0, st>>>(c, s, layer + l, n, seq, offsets, n_tokens, r);
    if (const cudaError_t e = cudaGetLastError()) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_kv_stats(const KvView& c, unsigned long long* out, int num_sms, cudaStream_t st) {
  cudaError_t e = cudaMemsetAsync(out, 0, 4 * sizeof(*out), st);
  if (e != cudaSuccess) return e;
  stats_kernel<<<2 * num_sms, 256, 0, st>>>(c, out);
  return cudaGetLastError();
}

}  // namespace p2p
