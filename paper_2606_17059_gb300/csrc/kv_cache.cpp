// kv_cache.cpp -- host side of the paged key-value cache: the p2p_kv_* calls of p2p_router.h.
//
// The pages, the page table, the lengths and the reference counts are the caller's arrays.  The handle holds the
// scratch of the calls, allocated once at its creation, so that no call allocates or waits (but p2p_kv_sync, _stats
// and _set_stream): a decode loop can be captured in a CUDA graph.
#include <algorithm>
#include <atomic>
#include <cstdio>
#include <cstring>
#include <new>
#include <utility>

#include "internal.h"
#include "kv.h"

struct p2p_kv {
  p2p::KvView c = {};
  p2p::KvScratch s = {};
  p2p::KvAttendScratch w = {};
  void* scratch = nullptr;             // one allocation: s's arrays and d_stats
  unsigned long long* d_stats = nullptr;
  int device = 0, num_sms = 0;
  cudaStream_t stream = nullptr;
  int64_t launches = 0;
  char err[256] = {};
};

namespace {

struct DeviceGuard {
  int prev = -1;
  bool changed = false;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) changed = cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() {
    if (changed) cudaSetDevice(prev);
  }
};

// (Messages are kept in the handle's own array: nothing here allocates, so nothing throws through the C calls.)
int fail(p2p_kv* h, int code, const char* msg) {
  if (h) {
    std::snprintf(h->err, sizeof(h->err), "%s", msg);
  } else {
    try {
      p2p::set_global_error(msg);
    } catch (...) {
    }
  }
  return code;
}

int cuda_fail(p2p_kv* h, cudaError_t e, const char* what) {
  (void)cudaGetLastError();  // reported here: the launch of a later call must not find it again
  char m[256];
  std::snprintf(m, sizeof(m), "%s: %s", what, cudaGetErrorString(e));
  return fail(h, P2P_E_CUDA, m);
}

#define CK(call)                                           \
  do {                                                     \
    cudaError_t e_ = (call);                               \
    if (e_ != cudaSuccess) return cuda_fail(h, e_, #call); \
  } while (0)

int esize(int32_t type) { return type == P2P_KV_E4M3 ? 1 : 2; }

// NULL, or what is wrong with the layout.
const char* check_layout(const p2p_kv_layout& a) {
  if (a.type != P2P_KV_BF16 && a.type != P2P_KV_F16 && a.type != P2P_KV_E4M3) return "type is none of P2P_KV_*";
  if (a.n_layers < 1 || a.n_layers > 65536 || a.n_pages < 1 || a.n_pages > (1 << 30) || a.page_tokens < 1 ||
      a.page_tokens > 4096 || a.n_heads < 1 || a.n_heads > 1024 || a.n_seqs < 1 || a.n_seqs > (1 << 20) ||
      a.max_pages < 1)
    return "a size is out of range";
  if (a.head_dim < 1 || a.head_dim > 256 || a.head_dim * esize(a.type) % 16)
    return "head_dim: at most 256, whole 16-byte pieces";
  if ((int64_t)a.max_pages * a.page_tokens > INT32_MAX) return "max_pages * page_tokens exceeds 2^31 - 1";
  if (!a.k || !a.v || !a.table || !a.length || !a.refs) return "NULL device pointer";
  if ((a.type == P2P_KV_E4M3) != (a.k_scale != nullptr) || (a.type == P2P_KV_E4M3) != (a.v_scale != nullptr))
    return "k_scale and v_scale go with P2P_KV_E4M3 alone";
  if ((uintptr_t)a.k % 16 || (uintptr_t)a.v % 16) return "k and v must start on 16-byte boundaries";
  std::pair<int64_t, int64_t> d[4] = {{a.layer_stride, a.n_layers}, {a.page_stride, a.n_pages},
                                      {a.token_stride, a.page_tokens}, {a.head_stride, a.n_heads}};
  std::sort(d, d + 4);
  int64_t extent = a.head_dim;  // values that the dimensions so far reach over
  for (auto& [stride, n] : d) {
    if (n == 1) continue;
    if (stride < extent || stride > (int64_t)1 << 44) return "strides overlap or are out of range";
    if (stride * esize(a.type) % 16) return "strides must be whole 16-byte pieces";
    extent += (n - 1) * stride;
    if (extent > (int64_t)1 << 46) return "the pages reach over more than 2^46 values";
  }
  return nullptr;
}

// Whether the rows of one head are pieces of lines and of pages of memory that other heads share, as a token's heads
// lie together (rows of whole 256 bytes are read as fast alone).  Then the warps of a CTA of the attention take up to
// four neighbouring heads of the same tokens instead of four times the tokens, in calls with enough of them (the kernel
// sees): 191 x 1,000 tokens of 24 heads of 80 16-bit values take 236 us and one head at a time 365; 256 sequences with
// 8 heads of 96 8-bit values 107 and 191, of 128 8-bit values 127 and 143.  (Rows of whole 128 bytes gain least: 192
// 16-bit values 240 us with pages of 16 tokens either way, 304 and 280 with pages of one.)
bool shares_lines(const p2p::KvView& c) { return c.head_stride <= c.token_stride && c.row16 % 16 != 0; }

// Whether two of the rows that a result is written to, `dim` values each at i * row + h * head (i < n, h < heads),
// share a value.
bool rows_overlap(int64_t n, int64_t heads, int64_t dim, int64_t row, int64_t head) {
  using wide = __int128;
  const wide r = row < 0 ? -(wide)row : row, g = head < 0 ? -(wide)head : head;
  if ((n > 1 && r < dim) || (heads > 1 && g < dim)) return true;
  if (n == 1 || heads == 1 || r >= (heads - 1) * g + dim || g >= (n - 1) * r + dim) return false;
  for (int64_t h = 1; h < heads; ++h) {  // (neither dimension lies within the other's steps)
    const wide i = h * g / r;
    if ((i < n && h * g - i * r < dim) || (i + 1 < n && (i + 1) * r - h * g < dim)) return true;
  }
  return false;
}

cudaError_t launch_attend(const p2p::KvView& c, const p2p::KvQuery* q, const p2p::KvAttendScratch& w, int num_sms,
                          cudaStream_t st) {
  using namespace p2p;
  const auto alone = c.type == P2P_KV_BF16  ? launch_kv_attend_bf16
                     : c.type == P2P_KV_F16 ? launch_kv_attend_f16
                                            : launch_kv_attend_e4m3;
  const auto side_by_side = c.type == P2P_KV_BF16  ? launch_kv_attend_bf16_side
                            : c.type == P2P_KV_F16 ? launch_kv_attend_f16_side
                                                   : launch_kv_attend_e4m3_side;
  if (!q) {  // (both are made ready)
    const cudaError_t e = alone(c, q, w, num_sms, st);
    return e != cudaSuccess || c.side == 0 ? e : side_by_side(c, q, w, num_sms, st);
  }
  // Without shared lines it is many short rows that gain (see kSideShort): with fewer the kernel finds too little to
  // take heads together, and is then the slower of the two.
  const int dp = attend_dim(c.type, c.dim), group = q->heads / c.heads;
  const int ctas = attend_ctas(c.type, dp, attend_blocks(c.type, dp, group));
  const bool many = (int64_t)q->n * c.heads >= (int64_t)kSideRows * std::max(2, ctas) * num_sms;
  return (c.side != 0 && (c.lines || many) ? side_by_side : alone)(c, q, w, num_sms, st);
}

// Scratch comes from a memory pool of the library's for each device, which keeps what destroyed handles give back: a
// handle made after them takes 40 us, not 135.  NULL, with *e set, where there is none.
cudaMemPool_t scratch_pool(int device, cudaError_t* e) {
  constexpr int kDevices = 64;
  static std::atomic<cudaMemPool_t> pools[kDevices];
  if (device < 0 || device >= kDevices) {
    *e = cudaErrorInvalidDevice;
    return nullptr;
  }
  cudaMemPool_t have = pools[device].load();
  if (have) return have;
  cudaMemPoolProps props = {};
  props.allocType = cudaMemAllocationTypePinned;
  props.location.type = cudaMemLocationTypeDevice;
  props.location.id = device;
  cudaMemPool_t pool = nullptr;
  *e = cudaMemPoolCreate(&pool, &props);
  if (*e != cudaSuccess) return nullptr;
  uint64_t all = UINT64_MAX;
  *e = cudaMemPoolSetAttribute(pool, cudaMemPoolAttrReleaseThreshold, &all);
  if (*e == cudaSuccess && pools[device].compare_exchange_strong(have, pool)) return pool;
  cudaMemPoolDestroy(pool);  // (another thread was first)
  return *e == cudaSuccess ? have : nullptr;
}

}  // namespace

extern "C" {

int p2p_kv_create(const p2p_kv_layout* layout, p2p_kv** out) {
  p2p_kv* h = nullptr;
  if (!layout || !out) return fail(h, P2P_E_INVAL, "layout or out is NULL");
  *out = nullptr;
  const p2p_kv_layout& a = *layout;
  if (const char* bad = check_layout(a)) return fail(h, P2P_E_INVAL, bad);
  int dev = 0, sms = 0;
  CK(cudaGetDevice(&dev));
  CK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  p2p_kv* n = new (std::nothrow) p2p_kv;
  if (!n) return fail(h, P2P_E_NOMEM, "no memory for the handle");
  n->device = dev;
  n->num_sms = sms;
  p2p::KvView& c = n->c;
  const int64_t es = esize(a.type);
  c.k = (char*)a.k;
  c.v = (char*)a.v;
  c.k_scale = a.k_scale;
  c.v_scale = a.v_scale;
  c.table = a.table;
  c.length = a.length;
  c.refs = a.refs;
  c.n_layers = a.n_layers;
  c.n_pages = a.n_pages;
  c.page = a.page_tokens;
  c.heads = a.n_heads;
  c.dim = a.head_dim;
  c.type = a.type;
  c.n_seqs = a.n_seqs;
  c.max_pages = a.max_pages;
  c.layer_stride = a.layer_stride * es;
  c.page_stride = a.page_stride * es;
  c.token_stride = a.token_stride * es;
  c.head_stride = a.head_stride * es;
  c.by_page = p2p::FastDiv((uint32_t)a.page_tokens);
  c.row16 = (int32_t)(a.head_dim * es / 16);
  c.lines = shares_lines(c);
  c.side = c.heads % 4 == 0 ? 2 : c.heads % 2 == 0 ? 1 : 0;
  // Scratch, each part on a 256-byte boundary.
  size_t at = 0;
  const auto part = [&at](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  const size_t S = (size_t)a.n_seqs, N = (size_t)a.n_pages;
  const size_t words = part(256), claim = part(4 * S),
               arrived = part(sizeof(int32_t) * 4 * p2p::KvAttendScratch::kCtasPerSm * sms), zero = at,
               start = part(4 * (S + 1)), first = part(4 * S), cut = part(4 * S),
               list = part(4 * N), jobs = part(sizeof(p2p::KvJob) * std::max(S, N)),
               parts = part(sizeof(float) * p2p::kv_attend_parts(c, sms));
  cudaError_t e = cudaSuccess;
  if (const cudaMemPool_t pool = scratch_pool(dev, &e)) e = cudaMallocFromPoolAsync(&n->scratch, at, pool, nullptr);
  if (e == cudaSuccess) e = cudaMemsetAsync(n->scratch, 0, zero, nullptr);
  if (e == cudaSuccess) e = p2p::prepare_kv_pages();
  if (e == cudaSuccess) e = launch_attend(c, nullptr, n->w, sms, nullptr);
  // (calls may go to a stream that does not wait for this one)
  if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
  if (e != cudaSuccess) {
    (void)cudaGetLastError();
    if (n->scratch) cudaFreeAsync(n->scratch, nullptr);
    delete n;
    return e == cudaErrorMemoryAllocation ? fail(h, P2P_E_NOMEM, "no device memory for the scratch")
                                          : cuda_fail(h, e, "the scratch");
  }
  char* p = (char*)n->scratch;
  n->s.err = (int32_t*)(p + words);
  n->s.halt = n->s.err + 1;
  n->s.njobs = n->s.err + 2;
  n->s.live = n->s.err + 3;
  n->d_stats = (unsigned long long*)(p + words + 64);
  n->s.claim = (int32_t*)(p + claim);
  n->s.start = (int32_t*)(p + start);
  n->s.first = (int32_t*)(p + first);
  n->s.cut = (int32_t*)(p + cut);
  n->s.list = (int32_t*)(p + list);
  n->s.jobs = (p2p::KvJob*)(p + jobs);
  n->w.parts = (float*)(p + parts);
  n->w.arrived = (int32_t*)(p + arrived);
  n->w.err = n->s.err;
  *out = n;
  return P2P_OK;
}

void p2p_kv_destroy(p2p_kv* h) {
  if (!h) return;
  DeviceGuard g(h->device);
  cudaStreamSynchronize(h->stream);
  cudaFreeAsync(h->scratch, nullptr);
  (void)cudaGetLastError();
  delete h;
}

int p2p_kv_set_stream(p2p_kv* h, void* stream) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  DeviceGuard g(h->device);
  CK(cudaStreamSynchronize(h->stream));
  h->stream = (cudaStream_t)stream;
  return P2P_OK;
}

int p2p_kv_sync(p2p_kv* h) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  DeviceGuard g(h->device);
  int32_t word[2] = {0, 0};
  CK(cudaMemcpyAsync(word, h->s.err, sizeof(word), cudaMemcpyDeviceToHost, h->stream));
  CK(cudaStreamSynchronize(h->stream));
  if (!word[0]) return P2P_OK;
  CK(cudaMemsetAsync(h->s.err, 0, sizeof(word), h->stream));
  CK(cudaStreamSynchronize(h->stream));
  const int b = word[0];
  if (b == p2p::KV_NO_PAGES) return fail(h, P2P_E_NOMEM, "the pool has too few free pages");
  char m[256];
  const auto say = [b](int bit, const char* what) { return b & bit ? what : ""; };
  std::snprintf(m, sizeof(m), "device reported:%s%s%s%s%s%s",
                say(p2p::KV_BAD_SEQ, " a sequence out of range or named twice;"),
                say(p2p::KV_BAD_COUNT, " a count or length out of range;"),
                say(p2p::KV_NO_PAGES, " too few free pages;"),
                say(p2p::KV_BAD_PAGE, " a page table or reference count that does not hold together;"),
                say(p2p::KV_SHARED, " a write to a shared page;"), say(p2p::KV_BAD_OFFSETS, " offsets out of range;"));
  return fail(h, P2P_E_DEVICE, m);
}

const char* p2p_kv_last_error(const p2p_kv* h) { return h ? h->err : p2p::global_error(); }

int64_t p2p_kv_launch_count(const p2p_kv* h) { return h ? h->launches : 0; }

int p2p_kv_stats(p2p_kv* h, int64_t out[4]) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  if (!out) return fail(h, P2P_E_INVAL, "out is NULL");
  DeviceGuard g(h->device);
  unsigned long long v[4];
  CK(p2p::launch_kv_stats(h->c, h->d_stats, h->num_sms, h->stream));
  h->launches += 1;
  CK(cudaMemcpyAsync(v, h->d_stats, sizeof(v), cudaMemcpyDeviceToHost, h->stream));
  CK(cudaStreamSynchronize(h->stream));
  for (int i = 0; i < 4; ++i) out[i] = (int64_t)v[i];
  return P2P_OK;
}

// What the calls over a list of sequences check on the host.
static int check_list(p2p_kv* h, int32_t n, const void* a, const void* b) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  if (n < 0 || n > h->c.n_seqs) return fail(h, P2P_E_INVAL, "n is negative or larger than the number of sequences");
  if (n > 0 && (!a || !b)) return fail(h, P2P_E_INVAL, "NULL device pointer");
  return P2P_OK;
}

int p2p_kv_extend(p2p_kv* h, int32_t n, const int32_t* seq, const int32_t* count) {
  if (int rc = check_list(h, n, seq, count)) return rc;
  if (n == 0) return P2P_OK;
  DeviceGuard g(h->device);
  CK(p2p::launch_kv_extend(h->c, h->s, n, seq, count, h->num_sms, h->stream));
  h->launches += 2;
  return P2P_OK;
}

int p2p_kv_trim(p2p_kv* h, int32_t n, const int32_t* seq, const int32_t* n_tokens) {
  if (int rc = check_list(h, n, seq, n_tokens)) return rc;
  if (n == 0) return P2P_OK;
  DeviceGuard g(h->device);
  CK(p2p::launch_kv_trim(h->c, h->s, n, seq, n_tokens, h->stream));
  h->launches += 1;
  return P2P_OK;
}

int p2p_kv_fork(p2p_kv* h, int32_t n, const int32_t* src, const int32_t* dst, const int32_t* n_tokens) {
  if (int rc = check_list(h, n, src, dst)) return rc;
  if (n == 0) return P2P_OK;
  if (!n_tokens) return fail(h, P2P_E_INVAL, "NULL device pointer");
  DeviceGuard g(h->device);
  CK(p2p::launch_kv_fork(h->c, h->s, n, src, dst, n_tokens, h->stream));
  h->launches += 1;
  return P2P_OK;
}

int p2p_kv_compact(p2p_kv* h) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  DeviceGuard g(h->device);
  int launches = 0;
  CK(p2p::launch_kv_compact(h->c, h->s, h->num_sms, h->stream, &launches));
  h->launches += launches;
  return P2P_OK;
}

int p2p_kv_write(p2p_kv* h, int32_t layer, int32_t n_layers, int32_t n, const int32_t* seq, const int64_t* offsets,
                 int64_t n_tokens, const void* k, const void* v, int64_t layer_stride, int64_t token_stride,
                 int64_t head_stride, int32_t type) {
  if (int rc = check_list(h, n, seq, offsets)) return rc;
  if (layer < 0 || n_layers < 0 || (int64_t)layer + n_layers > h->c.n_layers)
    return fail(h, P2P_E_INVAL, "layers out of range");
  if (n_tokens < 0 || n_tokens > INT32_MAX) return fail(h, P2P_E_INVAL, "n_tokens out of range");
  if (h->c.type == P2P_KV_E4M3 ? type != P2P_KV_BF16 && type != P2P_KV_F16 : type != h->c.type)
    return fail(h, P2P_E_INVAL, "type of k and v: the cache's own (bf16 or f16 for P2P_KV_E4M3)");
  if (n == 0 || n_tokens == 0 || n_layers == 0) return P2P_OK;
  if (!k || !v) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if ((uintptr_t)k % 2 || (uintptr_t)v % 2) return fail(h, P2P_E_INVAL, "k and v must be aligned to their type");
  DeviceGuard g(h->device);
  const p2p::KvRows rows = {k, v, layer_stride, token_stride, head_stride, type};
  CK(p2p::launch_kv_write(h->c, h->s, layer, n_layers, n, seq, offsets, n_tokens, rows, h->num_sms, h->stream));
  h->launches += 1;
  return P2P_OK;
}

int p2p_kv_attend(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, const void* q, int64_t q_row_stride,
                  int64_t q_head_stride, int32_t type, int32_t n_heads, float scale, int32_t window, void* out,
                  int64_t out_row_stride, int64_t out_head_stride, float* lse) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  if (layer < 0 || layer >= h->c.n_layers) return fail(h, P2P_E_INVAL, "layer out of range");
  if (n < 0 || n > (1 << 20) || (!seq && n > h->c.n_seqs)) return fail(h, P2P_E_INVAL, "n out of range");
  if (n_heads < 1 || n_heads > 16384 || n_heads % h->c.heads)
    return fail(h, P2P_E_INVAL, "n_heads must be a multiple of the cache's heads, at most 16,384");
  if (h->c.type == P2P_KV_E4M3 ? type != P2P_KV_BF16 && type != P2P_KV_F16 : type != h->c.type)
    return fail(h, P2P_E_INVAL, "type of q and out: the cache's own (bf16 or f16 for P2P_KV_E4M3)");
  if (window < 0) return fail(h, P2P_E_INVAL, "negative window");
  if (n == 0) return P2P_OK;
  if (!q || !out) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if ((uintptr_t)q % 2 || (uintptr_t)out % 2 || (uintptr_t)lse % 4)
    return fail(h, P2P_E_INVAL, "a pointer is not aligned to its type");
  if (rows_overlap(n, n_heads, h->c.dim, out_row_stride, out_head_stride))
    return fail(h, P2P_E_INVAL, "rows of out overlap");
  DeviceGuard g(h->device);
  const p2p::KvQuery a = {q, out, lse, seq, q_row_stride, q_head_stride, out_row_stride, out_head_stride,
                          n, n_heads, type, window, layer, scale,
                          (uintptr_t)q % 4 == 0 && q_row_stride % 2 == 0 && q_head_stride % 2 == 0,
                          (uintptr_t)out % 8 == 0 && out_row_stride % 4 == 0 && out_head_stride % 4 == 0};
  CK(launch_attend(h->c, &a, h->w, h->num_sms, h->stream));
  h->launches += 1;
  return P2P_OK;
}

}  // extern "C"
