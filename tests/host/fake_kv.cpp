// The cache's host code without a GPU: the CUDA runtime calls it makes, over host memory, and launchers that do nothing
// but count themselves.  The kernel for many rows can be made one that cannot be launched.
#include <cstdlib>
#include <cstring>
#include <string>

#include "kv.h"

namespace {
int rows_fail = 0, launches = 0;
cudaError_t last = cudaSuccess;
std::string message;
}  // namespace

extern "C" {
void fake_rows_fail(int e) { rows_fail = e; }
int fake_launches() { return launches; }

cudaError_t CUDARTAPI cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t CUDARTAPI cudaSetDevice(int) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { return *v = 152, cudaSuccess; }
cudaError_t CUDARTAPI cudaMemPoolCreate(cudaMemPool_t* p, const cudaMemPoolProps*) {
  return *p = (cudaMemPool_t)&launches, cudaSuccess;
}
cudaError_t CUDARTAPI cudaMemPoolDestroy(cudaMemPool_t) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaMemPoolSetAttribute(cudaMemPool_t, cudaMemPoolAttr, void*) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaMallocFromPoolAsync(void** p, size_t n, cudaMemPool_t, cudaStream_t) {
  return *p = std::malloc(n), cudaSuccess;
}
cudaError_t CUDARTAPI cudaFreeAsync(void* p, cudaStream_t) { return std::free(p), cudaSuccess; }
cudaError_t CUDARTAPI cudaMemsetAsync(void* p, int x, size_t n, cudaStream_t) {
  return std::memset(p, x, n), cudaSuccess;
}
cudaError_t CUDARTAPI cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t) {
  return std::memmove(d, s, n), cudaSuccess;
}
cudaError_t CUDARTAPI cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaGetLastError() {
  const cudaError_t e = last;
  last = cudaSuccess;
  return e;
}
const char* CUDARTAPI cudaGetErrorString(cudaError_t) { return "an error"; }
cudaError_t CUDARTAPI cudaGetDriverEntryPointByVersion(const char*, void** f, unsigned, unsigned long long,
                                                       cudaDriverEntryPointQueryResult* found) {
  *f = nullptr, *found = cudaDriverEntryPointSymbolNotFound;
  return cudaSuccess;
}
}

namespace p2p {
void set_global_error(const std::string& m) { message = m; }
const char* global_error() { return message.c_str(); }

namespace {
cudaError_t launched() { return ++launches, cudaSuccess; }
cudaError_t rows(const KvRowsCall* a) {
  if (a) return launched();
  return last = (cudaError_t)rows_fail;
}
}  // namespace

cudaError_t prepare_kv_pages() { return cudaSuccess; }
cudaError_t launch_kv_extend(const KvView&, const KvScratch&, int32_t, const int32_t*, const int32_t*, int,
                             cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_trim(const KvView&, const KvScratch&, int32_t, const int32_t*, const int32_t*, cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_fork(const KvView&, const KvScratch&, int32_t, const int32_t*, const int32_t*, const int32_t*,
                           cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_compact(const KvView&, const KvScratch&, int, cudaStream_t, int* n) { return *n = 1, launched(); }
cudaError_t launch_kv_write(const KvView&, const KvScratch&, int32_t, int32_t, int32_t, const int32_t*, const int64_t*,
                            int64_t, const KvRows&, int, cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_stats(const KvView&, unsigned long long*, int, cudaStream_t) { return launched(); }
cudaError_t launch_kv_turn(const KvView&, const KvScratch&, const KvTurn&, int32_t, int32_t, const int32_t*,
                           const int64_t*, int64_t, int, cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_share(const KvView&, int32_t*, int32_t, const int32_t*, int32_t, const int32_t*, int32_t, int64_t,
                            int32_t*, int4*, cudaStream_t) {
  return launched();
}
cudaError_t launch_kv_groups(int32_t*, int32_t, int32_t, const int32_t*, cudaStream_t) { return launched(); }
cudaError_t launch_kv_join(const KvView&, const KvRowsCall&, const KvAttendScratch&, int, cudaStream_t) {
  return launched();
}
#define ATTEND(name)                                                                                            \
  cudaError_t launch_kv_attend_##name(const KvView&, const KvQuery* q, const KvAttendScratch&, int, cudaStream_t) { \
    return q ? launched() : cudaSuccess;                                                                        \
  }
#define OF_TYPE(type)                                                                                               \
  ATTEND(type)                                                                                                      \
  ATTEND(type##_side)                                                                                               \
  ATTEND(type##_after)                                                                                              \
  ATTEND(type##_side_after)                                                                                         \
  cudaError_t launch_kv_rows_##type(const KvView&, const KvMaps&, const KvRowsCall* a, const KvAttendScratch&, int, \
                                    cudaStream_t) {                                                                 \
    return rows(a);                                                                                                 \
  }
OF_TYPE(bf16)
OF_TYPE(f16)
OF_TYPE(e4m3)
}  // namespace p2p
