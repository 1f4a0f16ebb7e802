// The kernels of kv_attend for e4m3 codes (kv_attend.hpp).
#include "kv_attend.hpp"

namespace kmq {

km_status launch_kv_attend_f8(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  return go_attend<KM_KV_F8>(C, S, A, ws, s);
}

}  // namespace kmq
