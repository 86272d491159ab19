// kv_math.cuh -- what the attention's kernels over the paged key-value cache share: softmax ranges by type, copies into
// shared memory, packed values.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "kv.h"

// (No load here goes past the coherent path, as __ldg or const __restrict__ would have it: the kernel before may
// still be writing when this one starts, see launch_early.)

namespace p2p {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// kUp: exp(x - m) is taken times 2^kUp (m is held less kUp, in log2).  kLag: how far (log2) a logit may pass the
// maximum in use.  P is at most 2^(kUp + kLag), which f16 has to hold.
template <int KIND>
struct Type;
template <>
struct Type<P2P_KV_BF16> {
  static constexpr float kUp = 0.f, kLag = 8.f;
};
template <>
struct Type<P2P_KV_F16> {
  static constexpr float kUp = 12.f, kLag = 3.f;
};
template <>
struct Type<P2P_KV_E4M3> {
  static constexpr float kUp = 12.f, kLag = 3.f;
};

__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ int32_t add_acq_rel(int32_t* p, int32_t x) {
  int32_t y;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(y) : "l"(p), "r"(x) : "memory");
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// ln of a sum of exp that was taken relative to t (in log2): near the largest term, where log2 is small.
template <int KIND>
__device__ __forceinline__ float log_sum(float t, float z) {
  constexpr float kUp = Type<KIND>::kUp, kDown = 1.f / (1 << (int)kUp);
  return (t + kUp + __log2f(z * kDown)) * kLn2;
}
template <int KIND>
__device__ __forceinline__ uint32_t pack(float a, float b) {
  if (KIND == P2P_KV_BF16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *(const uint32_t*)&x;
  }
  const __half2 x = __floats2half2_rn(a, b);
  return *(const uint32_t*)&x;
}
// Two 8-bit values (the low half of x) as two of 16.
__device__ __forceinline__ uint32_t widen(uint32_t x) {
  uint32_t y;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t widen_high(uint32_t x) {
  uint32_t y;
  asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float2 two_halves(uint32_t x, int32_t type) {
  return type == P2P_KV_BF16 ? __bfloat1622float2(*(const __nv_bfloat162*)&x) : __half22float2(*(const __half2*)&x);
}

}  // namespace
}  // namespace p2p
