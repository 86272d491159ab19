// kv_attend_f16_side_after.cu -- the kernels of kv_attend_f16_side.cu for rows whose
// first tokens are worked off elsewhere (a source each, compiled side by side).
#include "kv_attend.cuh"

namespace p2p {
cudaError_t launch_kv_attend_f16_side_after(const KvView& c, const KvQuery* q, const KvAttendScratch& w, int num_sms,
                                            cudaStream_t st) {
  return launch_dim<P2P_KV_F16, true, true>(c, q, w, num_sms, st);
}
}  // namespace p2p
