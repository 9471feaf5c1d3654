// Calls of the tcgen05 attention kernel in packed_tc.cuh with masks and a cap.
#include "packed_tc.cuh"

namespace samkv {

cudaError_t launch_packed_tc_cap(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  return ptc::launch_scores<ptc::MOD_CAP>(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
}

}  // namespace samkv
