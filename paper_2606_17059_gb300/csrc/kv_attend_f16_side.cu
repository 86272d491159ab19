// kv_attend_f16_side.cu -- the attention kernels of kv_attend.cuh for caches of this type, with kv heads side by side
// (a source each, compiled side by side).
#include "kv_attend.cuh"

namespace p2p {
cudaError_t launch_kv_attend_f16_side(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                      cudaStream_t st) {
  return launch_dim<P2P_KV_F16, true>(c, q, w, num_sms, st);
}
}  // namespace p2p
