// kv_cache.cpp -- host side of the paged key-value cache: the p2p_kv_* calls of p2p_router.h.
//
// The pages, the page table, the lengths and the reference counts are the caller's arrays.  The handle holds the
// scratch of the calls, allocated once at its creation, so that no call allocates or waits (but p2p_kv_sync, _stats
// and _set_stream): a decode loop can be captured in a CUDA graph.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <utility>

#include "internal.h"
#include "kv.h"
#include "kv_strides.h"

struct p2p_kv {
  p2p::KvView c = {};
  p2p::KvScratch s = {};
  p2p::KvAttendScratch w = {};
  p2p::KvMaps maps = {};
  void* encode = nullptr;              // cuTensorMapEncodeTiled, or NULL
  void* scratch = nullptr;             // one allocation: s's arrays and d_stats
  unsigned long long* d_stats = nullptr;
  int device = 0, num_sms = 0;
  cudaStream_t stream = nullptr;
  int64_t launches = 0;
  int64_t patience = 4000000000;      // (some two seconds)
  bool many_rows = true;              // whether the kernel for many rows can be launched
  char err[320] = {};
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
  using Launch = cudaError_t (*)(const KvView&, const KvQuery*, const KvAttendScratch&, int, cudaStream_t);
  constexpr Launch kBf16[4] = {launch_kv_attend_bf16, launch_kv_attend_bf16_side, launch_kv_attend_bf16_after,
                               launch_kv_attend_bf16_side_after};
  constexpr Launch kF16[4] = {launch_kv_attend_f16, launch_kv_attend_f16_side, launch_kv_attend_f16_after,
                              launch_kv_attend_f16_side_after};
  constexpr Launch kE4m3[4] = {launch_kv_attend_e4m3, launch_kv_attend_e4m3_side, launch_kv_attend_e4m3_after,
                               launch_kv_attend_e4m3_side_after};
  const Launch* const of_type = c.type == P2P_KV_BF16 ? kBf16 : c.type == P2P_KV_F16 ? kF16 : kE4m3;
  if (!q) {  // (all are made ready)
    for (int i = 0; i < 4; ++i) {
      if (i % 2 == 1 && c.side == 0) continue;
      const cudaError_t e = of_type[i](c, q, w, num_sms, st);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
  // Without shared lines it is many short rows that gain (see kSideShort): with fewer the kernel finds too little to
  // take heads together, and is then the slower of the two.
  const int dp = attend_dim(c.type, c.dim), group = q->heads / c.heads;
  const int ctas = attend_ctas(c.type, dp, attend_blocks(c.type, dp, group));
  const bool many = (int64_t)q->n * c.heads >= (int64_t)kSideRows * std::max(2, ctas) * num_sms;
  return of_type[(c.side != 0 && (c.lines || many) ? 1 : 0) + (q->skip ? 2 : 0)](c, q, w, num_sms, st);
}

void* map_encoder() {
  void* entry = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &entry, 12000, cudaEnableDefault, &found) ==
          cudaSuccess &&
      found == cudaDriverEntryPointSuccess)
    return entry;
  (void)cudaGetLastError();
  return nullptr;
}

// The pages as tensors for copies by the tensor memory accelerator, where they are to be had.
void make_maps(const p2p::KvView& c, void* entry, p2p::KvMaps& m) {
  m.rows = 0;
  const bool eight = c.type == P2P_KV_E4M3;
  // Tokens of a copy: a power of two that divides a page (and so lies in one), at most what a warp takes of a step;
  // copies go to whole 128 bytes (1,024 where their pieces are turned).
  uint32_t rows = c.page & -c.page;
  rows = std::min(rows, c.dim > 128 ? 16u : 32u);
  if (!entry || (eight ? rows * c.dim % 128 != 0 : rows < 8)) return;
  const cuuint64_t size[5] = {(cuuint64_t)c.dim, (cuuint64_t)c.page, (cuuint64_t)c.heads, (cuuint64_t)c.n_pages,
                              (cuuint64_t)c.n_layers};
  cuuint64_t stride[4] = {(cuuint64_t)c.token_stride, (cuuint64_t)c.head_stride, (cuuint64_t)c.page_stride,
                          (cuuint64_t)c.layer_stride};
  for (int i = 0; i < 4; ++i) {
    if (size[i + 1] == 1) stride[i] = 16;  // (whatever the caller gave: it is not used)
    if (stride[i] >= (cuuint64_t)1 << 40) return;
  }
  const cuuint32_t box[5] = {eight ? (cuuint32_t)c.dim : 64, rows, 1, 1, 1}, step[5] = {1, 1, 1, 1, 1};
  const auto make = [&](CUtensorMap* map, void* at) {
    return ((decltype(&cuTensorMapEncodeTiled))entry)(
               map, eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, at, size, stride, box,
                   step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, eight ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  };
  if (make(&m.k, c.k) && make(&m.v, c.v)) m.rows = (int32_t)rows;
}

cudaError_t launch_rows(const p2p::KvView& c, const p2p::KvMaps& m, const p2p::KvRowsCall* a,
                        const p2p::KvAttendScratch& w, int num_sms, cudaStream_t st) {
  using namespace p2p;
  return (c.type == P2P_KV_BF16  ? launch_kv_rows_bf16
          : c.type == P2P_KV_F16 ? launch_kv_rows_f16
                                 : launch_kv_rows_e4m3)(c, m, a, w, num_sms, st);
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
               joins = part(sizeof(p2p::KvJoin) * sms),
               parts = part(sizeof(float) * std::max(p2p::kv_attend_parts(c, sms), p2p::kv_rows_parts(c, sms)));
  cudaError_t e = cudaSuccess;
  if (const cudaMemPool_t pool = scratch_pool(dev, &e)) e = cudaMallocFromPoolAsync(&n->scratch, at, pool, nullptr);
  if (e == cudaSuccess) e = cudaMemsetAsync(n->scratch, 0, zero, nullptr);
  if (e == cudaSuccess) e = p2p::prepare_kv_pages();
  if (e == cudaSuccess) e = launch_attend(c, nullptr, n->w, sms, nullptr);
  if (e == cudaSuccess) {
    e = launch_rows(c, n->maps, nullptr, n->w, sms, nullptr);
    // (Compiled to other registers than it shares out: the calls that need it refuse, the cache is there.)
    if (e == cudaErrorInvalidDeviceFunction) n->many_rows = false, e = cudaSuccess, (void)cudaGetLastError();
  }
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
  n->w.joins = (p2p::KvJoin*)(p + joins);
  n->w.err = n->s.err;
  n->encode = map_encoder();
  make_maps(c, n->encode, n->maps);
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
  char m[320];
  const auto say = [b](int bit, const char* what) { return b & bit ? what : ""; };
  std::snprintf(m, sizeof(m), "device reported:%s%s%s%s%s%s%s",
                say(p2p::KV_BAD_SEQ, " a sequence out of range or named twice;"),
                say(p2p::KV_BAD_COUNT, " a count or length out of range;"),
                say(p2p::KV_NO_PAGES, " too few free pages;"),
                say(p2p::KV_BAD_PAGE, " a page table or reference count that does not hold together;"),
                say(p2p::KV_SHARED, " a write to a shared page;"), say(p2p::KV_BAD_OFFSETS, " offsets out of range;"),
                say(p2p::KV_STUCK, " a kernel that gave up waiting for itself;"));
  return fail(h, P2P_E_DEVICE, m);
}

int p2p_kv_set_patience(p2p_kv* h, int64_t cycles) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  if (cycles == 0 || cycles == INT64_MIN) return fail(h, P2P_E_INVAL, "no patience at all");
  h->patience = cycles;
  return P2P_OK;
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

// What the attention's calls check on the host: what is asked for, and where rows of queries and results lie.
static bool bad_type(const p2p_kv* h, int32_t type) {
  return h->c.type == P2P_KV_E4M3 ? type != P2P_KV_BF16 && type != P2P_KV_F16 : type != h->c.type;
}
static int check_attend(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, int32_t type, int32_t n_heads,
                        int32_t window) {
  if (!h) return fail(nullptr, P2P_E_INVAL, "cache is NULL");
  if (layer < 0 || layer >= h->c.n_layers) return fail(h, P2P_E_INVAL, "layer out of range");
  if (n < 0 || n > (1 << 20) || (!seq && n > h->c.n_seqs)) return fail(h, P2P_E_INVAL, "n out of range");
  if (n_heads < 1 || n_heads > 16384 || n_heads % h->c.heads)
    return fail(h, P2P_E_INVAL, "n_heads must be a multiple of the cache's heads, at most 16,384");
  if (bad_type(h, type))
    return fail(h, P2P_E_INVAL, "type of q and out: the cache's own (bf16 or f16 for P2P_KV_E4M3)");
  if (window < 0) return fail(h, P2P_E_INVAL, "negative window");
  return P2P_OK;
}
static int check_kernel(p2p_kv* h) {
  return h->many_rows ? P2P_OK : fail(h, P2P_E_CUDA, "the attention of many rows was not compiled to 128 registers a thread");
}
static int check_rows(p2p_kv* h, int64_t n, const void* q, int32_t n_heads, const void* out, int64_t out_row,
                      int64_t out_head, const float* lse) {
  if (!q || !out) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if ((uintptr_t)q % 2 || (uintptr_t)out % 2 || (uintptr_t)lse % 4)
    return fail(h, P2P_E_INVAL, "a pointer is not aligned to its type");
  if (rows_overlap(n, n_heads, h->c.dim, out_row, out_head)) return fail(h, P2P_E_INVAL, "rows of out overlap");
  return P2P_OK;
}

static p2p::KvQuery query_of(int32_t layer, int32_t n, const int32_t* seq, const void* q, int64_t q_row, int64_t q_head,
                             int32_t type, int32_t n_heads, float scale, int32_t window, void* out, int64_t out_row,
                             int64_t out_head, float* lse) {
  return {q, out, lse, seq, q_row, q_head, out_row, out_head, n, n_heads, type, window, layer, scale,
          (uintptr_t)q % 4 == 0 && q_row % 2 == 0 && q_head % 2 == 0,
          (uintptr_t)out % 8 == 0 && out_row % 4 == 0 && out_head % 4 == 0,
          nullptr, nullptr, nullptr};
}

int p2p_kv_attend(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, const void* q, int64_t q_row_stride,
                  int64_t q_head_stride, int32_t type, int32_t n_heads, float scale, int32_t window, void* out,
                  int64_t out_row_stride, int64_t out_head_stride, float* lse) {
  if (int rc = check_attend(h, layer, n, seq, type, n_heads, window)) return rc;
  if (n == 0) return P2P_OK;
  if (int rc = check_rows(h, n, q, n_heads, out, out_row_stride, out_head_stride, lse)) return rc;
  DeviceGuard g(h->device);
  const p2p::KvQuery a = query_of(layer, n, seq, q, q_row_stride, q_head_stride, type, n_heads, scale, window, out,
                                  out_row_stride, out_head_stride, lse);
  CK(launch_attend(h->c, &a, h->w, h->num_sms, h->stream));
  h->launches += 1;
  return P2P_OK;
}

int p2p_kv_rotation_turns(int32_t n, const double* radians, uint64_t* turns) {
  if (n < 0 || (n > 0 && (!radians || !turns))) return fail(nullptr, P2P_E_INVAL, "n is negative or an array is NULL");
  // 1 / (2 pi) in two parts: the quotient to 2^-64 of a turn or 2^-52 of itself, whichever is more.
  constexpr double kHigh = 0x1.45f306dc9c883p-3, kLow = -0x1.6b01ec5417056p-57;
  for (int32_t j = 0; j < n; ++j)
    if (!(radians[j] >= 0.0) || !(radians[j] < 6.283185307179586))
      return fail(nullptr, P2P_E_INVAL, "radians: 0 <= x < 2 pi");
  for (int32_t j = 0; j < n; ++j) {
    const double high = radians[j] * kHigh, low = std::fma(radians[j], kHigh, -high) + radians[j] * kLow;
    const double scaled = std::ldexp(high, 64), whole = std::floor(scaled);
    turns[j] = (uint64_t)whole + (uint64_t)(int64_t)std::llrint(scaled - whole + std::ldexp(low, 64));
  }
  return P2P_OK;
}

int p2p_kv_write_rotated(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, const int64_t* offsets,
                         int64_t n_tokens, const p2p_kv_rotation* rotation, const void* q, int64_t q_token_stride,
                         int64_t q_head_stride, int32_t n_heads, const void* k, const void* v, int64_t token_stride,
                         int64_t head_stride, int32_t type, void* out, int64_t out_token_stride,
                         int64_t out_head_stride) {
  if (int rc = check_list(h, n, seq, offsets)) return rc;
  if (layer < 0 || layer >= h->c.n_layers) return fail(h, P2P_E_INVAL, "layer out of range");
  if (n_tokens < 0 || n_tokens > INT32_MAX) return fail(h, P2P_E_INVAL, "n_tokens out of range");
  if (n_heads < 1 || n_heads > 16384) return fail(h, P2P_E_INVAL, "n_heads out of range");
  if (bad_type(h, type))
    return fail(h, P2P_E_INVAL, "type of q, k and v: the cache's own (bf16 or f16 for P2P_KV_E4M3)");
  if (!rotation) return fail(h, P2P_E_INVAL, "rotation is NULL");
  const p2p_kv_rotation& r = *rotation;
  if (r.dim < 0 || r.dim > h->c.dim || r.dim % 2) return fail(h, P2P_E_INVAL, "rotated values: even, at most head_dim");
  if (r.dim > 0 && !r.turns) return fail(h, P2P_E_INVAL, "turns is NULL");
  if (n == 0 || n_tokens == 0) return P2P_OK;
  if (!q || !k || !v || !out) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if ((uintptr_t)q % 2 || (uintptr_t)k % 2 || (uintptr_t)v % 2 || (uintptr_t)out % 2 || (uintptr_t)r.turns % 8 ||
      (uintptr_t)r.q_weight % 4 || (uintptr_t)r.k_weight % 4)
    return fail(h, P2P_E_INVAL, "a pointer is not aligned to its type");
  if (rows_overlap(n_tokens, n_heads, h->c.dim, out_token_stride, out_head_stride))
    return fail(h, P2P_E_INVAL, "rows of out overlap");
  // (A row is read whole before it is written, but rows of others are read at any time.)
  using p2p::rows_meet;
  const p2p::RowsAt to = {out, out_token_stride, out_head_stride, n_heads};
  const bool same = q == out && (n_tokens == 1 || q_token_stride == out_token_stride) &&
                    (n_heads == 1 || q_head_stride == out_head_stride);
  if (!same && rows_meet({q, q_token_stride, q_head_stride, n_heads}, to, n_tokens, h->c.dim))
    return fail(h, P2P_E_INVAL, "out overlaps q without being it");
  if (rows_meet({k, token_stride, head_stride, h->c.heads}, to, n_tokens, h->c.dim) ||
      rows_meet({v, token_stride, head_stride, h->c.heads}, to, n_tokens, h->c.dim))
    return fail(h, P2P_E_INVAL, "out overlaps k or v");
  DeviceGuard g(h->device);
  const p2p::KvTurn a = {q, k, v, out, q_token_stride, q_head_stride, out_token_stride, out_head_stride, token_stride,
                         head_stride, r.turns, r.q_weight, r.k_weight, r.amplitude, r.eps, n_heads, type, r.dim,
                         r.interleaved != 0};
  CK(p2p::launch_kv_turn(h->c, h->s, a, layer, n, seq, offsets, n_tokens, h->num_sms, h->stream));
  h->launches += 1;
  return P2P_OK;
}

// Queries as a tensor [row][kv head][query head of it][value], copied a row tile's whole rows at a time; false where
// they do not lie as that takes, or half a tile or more might stay empty.
static bool make_query_map(const p2p_kv* h, const p2p::KvRowsCall& a, int64_t n_rows, CUtensorMap& map) {
  if (!h->encode || a.group > 32 || (uintptr_t)a.q % 16) return false;
  const cuuint64_t size[4] = {(cuuint64_t)h->c.dim, (cuuint64_t)a.group, (cuuint64_t)h->c.heads, (cuuint64_t)n_rows};
  const int64_t given[3] = {a.q_head, a.q_head * a.group, a.q_row};
  cuuint64_t stride[3];
  for (int i = 0; i < 3; ++i) {
    if (size[i + 1] > 1 && (given[i] <= 0 || given[i] % 8 || given[i] >= (int64_t)1 << 39)) return false;
    stride[i] = size[i + 1] > 1 ? given[i] * 2 : 16;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)a.group, 1, (cuuint32_t)(128 / a.group)}, step[4] = {1, 1, 1, 1};
  return ((decltype(&cuTensorMapEncodeTiled))h->encode)(
             &map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, (void*)a.q, size, stride, box, step,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static p2p::KvRowsCall rows_call(const p2p_kv* h, CUtensorMap& q_map, int32_t layer, int32_t n, int64_t n_rows,
                                 const int32_t* seq, const void* q, int64_t q_row, int64_t q_head, int32_t type,
                                 int32_t n_heads, float scale, int32_t window, void* out, int64_t out_row,
                                 int64_t out_head, float* lse) {
  p2p::KvRowsCall a = {};
  a.q = q, a.out = out, a.lse = lse, a.seq = seq;
  a.q_row = q_row, a.q_head = q_head, a.out_row = out_row, a.out_head = out_head;
  a.n = n, a.heads = n_heads, a.group = n_heads / h->c.heads, a.type = type, a.window = window, a.layer = layer,
      a.scale = scale;
  a.by_group = p2p::FastDiv((uint32_t)a.group);
  a.boxes = make_query_map(h, a, n_rows, q_map);
  a.tile_rows = a.boxes ? 128 / a.group * a.group : 128;
  a.q_map = a.boxes ? &q_map : nullptr;
  const int64_t tokens = (int64_t)h->c.max_pages * h->c.page;
  if (window >= tokens) a.window = 0;  // (which is as much as a sequence can have)
  const bool wide = h->c.dim > 128;    // (as RowsShape has it)
  a.patience = h->patience;
  a.count = p2p::rows_scale(n, n_rows, n_heads, h->c.heads, wide ? 1 : 2, a.tile_rows, wide ? 6 : 7, tokens);
  a.out32 = (uintptr_t)out % 32 == 0 && out_row % 16 == 0 && out_head % 16 == 0;
  return a;
}

int p2p_kv_attend_prompt(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, const int64_t* offsets,
                         int64_t n_tokens, const void* q, int64_t q_token_stride, int64_t q_head_stride, int32_t type,
                         int32_t n_heads, float scale, int32_t window, void* out, int64_t out_token_stride,
                         int64_t out_head_stride, float* lse) {
  if (int rc = check_attend(h, layer, n, seq, type, n_heads, window)) return rc;
  if (n_tokens < 0 || n_tokens > INT32_MAX || n_tokens * n_heads > (int64_t)1 << 29)
    return fail(h, P2P_E_INVAL, "n_tokens out of range");
  if (n == 0 || n_tokens == 0) return P2P_OK;
  if (!offsets) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if (int rc = check_rows(h, n_tokens, q, n_heads, out, out_token_stride, out_head_stride, lse)) return rc;
  if (int rc = check_kernel(h)) return rc;
  DeviceGuard g(h->device);
  CUtensorMap q_map;
  p2p::KvRowsCall a = rows_call(h, q_map, layer, n, n_tokens, seq, q, q_token_stride, q_head_stride, type, n_heads,
                                scale, window, out, out_token_stride, out_head_stride, lse);
  a.offsets = offsets;
  a.n_tokens = n_tokens;
  CK(launch_rows(h->c, h->maps, &a, h->w, h->num_sms, h->stream));
  CK(p2p::launch_kv_join(h->c, a, h->w, h->num_sms, h->stream));
  h->launches += 2;
  return P2P_OK;
}

// Where the parts of attend_shared's work lie: each row's result over its group's tokens, its maximum and sum of exp,
// what the groups share, and the tokens of each row that its group works off.
struct SharedWork {
  size_t sum, spans, skip, bytes;
  SharedWork(const p2p::KvView& c, int32_t n, int32_t n_heads) {
    const size_t rows = (size_t)n * n_heads;
    sum = sizeof(float) * rows * c.dim;
    spans = sum + sizeof(float2) * ((rows + 1) / 2 * 2);
    skip = spans + sizeof(int4) * n;
    bytes = skip + sizeof(int32_t) * n + 16;
  }
};

int64_t p2p_kv_attend_shared_work(const p2p_kv* h, int32_t n, int32_t n_heads) {
  if (!h || n < 0 || n > (1 << 20) || n_heads < 1 || n_heads > 16384) return -1;
  return (int64_t)SharedWork(h->c, n, n_heads).bytes;
}

// Bytes of keys and values whose reading has to be saved for groups to be worth three more launches.  Measured on one
// GB300, prefixes read together and row by row, in us: with 256 MB saved 55 and 31 (64 rows, 14 / 2 heads of 64), 43 and
// 36 (200 rows, 40 / 8 of 128), 35 and 29 (32 rows, 32 / 8 of 128), 56 and 43 (8 rows, 64 / 8 of 128); 448 MB 61 and 47,
// 46 and 48, 42 and 42, 73 and 67; 640 MB 63 and 62, 46 and 61, 46 and 56, 82 and 90; 1,024 MB 67 and 94, 49 and 85, 49
// and 83, 104 and 138.  (Few rows gain less, as what they read together is read at a lower rate: kTogether.)  One number
// for all of them: just above it few kv heads lose up to 14 us, and many rows would gain from 384 MB on.
constexpr int64_t kWorthSharing = (int64_t)448 << 20;

int p2p_kv_attend_shared(p2p_kv* h, int32_t layer, int32_t n, const int32_t* seq, int32_t n_groups,
                         const int32_t* groups, int64_t least, const void* q, int64_t q_row_stride,
                         int64_t q_head_stride, int32_t type, int32_t n_heads, float scale, int32_t window, void* out,
                         int64_t out_row_stride, int64_t out_head_stride, float* lse, void* work) {
  if (int rc = check_attend(h, layer, n, seq, type, n_heads, window)) return rc;
  if ((int64_t)n * n_heads > (int64_t)1 << 29) return fail(h, P2P_E_INVAL, "n * n_heads exceeds 2^29");
  if (n_groups < 0 || n_groups > n) return fail(h, P2P_E_INVAL, "n_groups: at most n");
  if (n == 0) return P2P_OK;
  if ((n_groups > 0 && !groups) || !work) return fail(h, P2P_E_INVAL, "NULL device pointer");
  if ((uintptr_t)work % 32) return fail(h, P2P_E_INVAL, "work must start on a 32-byte boundary");
  if (int rc = check_rows(h, n, q, n_heads, out, out_row_stride, out_head_stride, lse)) return rc;
  if (int rc = check_kernel(h)) return rc;
  DeviceGuard g(h->device);
  const SharedWork at(h->c, n, n_heads);
  float* pre = (float*)work;
  float2* pre_sum = (float2*)((char*)work + at.sum);
  int4* spans = (int4*)((char*)work + at.spans);
  int32_t* skip = (int32_t*)((char*)work + at.skip);
  p2p::KvQuery rest = query_of(layer, n, seq, q, q_row_stride, q_head_stride, type, n_heads, scale, window, out,
                               out_row_stride, out_head_stride, lse);
  // In tokens of a row, of which no more can be saved than the tables hold and the windows let see.
  const int64_t token = 2 * (int64_t)h->c.heads * h->c.dim * (h->c.type == P2P_KV_E4M3 ? 1 : 2);
  const int64_t bytes = least < 0 ? kWorthSharing : least, tokens = bytes / token + (bytes % token > 0);
  const int64_t seen = (int64_t)h->c.max_pages * h->c.page;
  if (n_groups > 0 && tokens > 0 && (n - p2p::kTogether) * (window ? std::min<int64_t>(window, seen) : seen) < tokens) {
    CK(p2p::launch_kv_groups(h->s.err, n, n_groups, groups, h->stream));
    h->launches += 1;
  } else if (n_groups > 0) {
    // What the groups share, and the attention over it; then every row's other tokens, put together with that.
    CK(p2p::launch_kv_share(h->c, h->s.err, n, seq, n_groups, groups, window, tokens, skip, spans, h->stream));
    CUtensorMap q_map;
    p2p::KvRowsCall a = rows_call(h, q_map, layer, n_groups, n, seq, q, q_row_stride, q_head_stride, type, n_heads,
                                  scale, window, out, out_row_stride, out_head_stride, lse);
    a.groups = groups;
    a.spans = spans;
    a.pre = pre;
    a.pre_sum = pre_sum;
    a.n_tokens = n;
    CK(launch_rows(h->c, h->maps, &a, h->w, h->num_sms, h->stream));
    CK(p2p::launch_kv_join(h->c, a, h->w, h->num_sms, h->stream));
    h->launches += 3;
    rest.skip = skip;
    rest.pre = pre;
    rest.pre_sum = pre_sum;
  }
  CK(launch_attend(h->c, &rest, h->w, h->num_sms, h->stream));
  h->launches += 1;
  return P2P_OK;
}

}  // extern "C"
