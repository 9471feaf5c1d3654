// Plain calls of the tcgen05 attention kernel in packed_tc.cuh.
#include "packed_tc.cuh"

namespace samkv {

size_t packed_tc_scratch_bytes(int d) {
  return (size_t)kTcSlots * 128 * ((size_t)d * 4 + 12) + (size_t)kMaxPackedCtas * 256 * 4;
}

cudaError_t launch_packed_tc(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                             const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  const ptc::Params p = ptc::make_params(d, seqs, kv, Q, scale, O, lse, h);
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  if (d.head_dim == 128)
    return kv.paged ? ptc::launch<128, true, ptc::MOD_NONE>(p, ctas, stream) : ptc::launch<128, false, ptc::MOD_NONE>(p, ctas, stream);
  return kv.paged ? ptc::launch<64, true, ptc::MOD_NONE>(p, ctas, stream) : ptc::launch<64, false, ptc::MOD_NONE>(p, ctas, stream);
}

}  // namespace samkv
