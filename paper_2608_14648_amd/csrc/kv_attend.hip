// How a call of kv_attend is cut up, its workspace, and the kernels for int8 codes (kv_attend.hpp).
#include "kv_attend.hpp"

namespace kmq {

km_status launch_kv_attend_f8(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s);
km_status launch_kv_attend_i4(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s);

bool kv_attend_fits(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);  // workgroups of eight waves are for few tiles
  return p.prompt || p.tiles / S.n <= kv_piece(64 * kAttendWaves);
}

int64_t kv_attend_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  return std::max(p.tiles * (p.deal ? 1 : p.splits), join_blocks(p));
}

size_t kv_attend_scratch(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  if (p.splits == 1 && !p.deal) return 0;
  return sizeof(float) * (size_t)(p.deal ? 2 : p.tiles) * p.splits * p.rt *
         (p.prompt ? part32_floats(p.nt) : part_floats(p.nt));
}

km_status launch_kv_attend(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  return C.fmt == KM_KV_I8   ? go_attend<KM_KV_I8>(C, S, A, ws, s)
         : C.fmt == KM_KV_F8 ? launch_kv_attend_f8(C, S, A, ws, s)
                             : launch_kv_attend_i4(C, S, A, ws, s);
}

}  // namespace kmq
