// kv_attend_bf16.cu -- the attention kernels of kv_attend.cuh for caches of this type, one kv head a CTA at a time (a
// source each, compiled side by side).
#include "kv_attend.cuh"

namespace p2p {
cudaError_t launch_kv_attend_bf16(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                  cudaStream_t st) {
  return launch_dim<P2P_KV_BF16, false, false>(c, q, w, num_sms, st);
}
}  // namespace p2p
