// The kernels of kv_attend for 4-bit codes (kv_attend.hpp).
#include "kv_attend.hpp"

namespace kmq {

km_status launch_kv_attend_i4(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  return go_attend<KM_KV_I4>(C, S, A, ws, s);
}

}  // namespace kmq
