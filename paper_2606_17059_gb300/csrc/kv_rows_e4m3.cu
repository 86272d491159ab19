// kv_rows_e4m3.cu -- the kernels of kv_rows.cuh for caches of this type (a source each, compiled side by side).
#include "kv_rows.cuh"

namespace p2p {
cudaError_t launch_kv_rows_e4m3(const KvView& c, const KvMaps& m, const KvRowsCall* a, const KvAttendScratch& w,
    int num_sms,
                                cudaStream_t st) {
  return launch_rows_dim<P2P_KV_E4M3>(c, m, a, w, num_sms, st);
}
}  // namespace p2p
