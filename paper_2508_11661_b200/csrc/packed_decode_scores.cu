// Calls of the decode kernel in packed_decode.cuh with modified scores.
#include "packed_decode.cuh"

namespace samkv {

cudaError_t launch_packed_decode_scores(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                        const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h,
                                        cudaStream_t stream) {
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  pdec::Params p = pdec::make_params(d, seqs, kv, Q, scale, O, lse, h, ctas);
  p.mods = mods;
  p.cap = tc::make_cap(mods.softcap, scale);
  const cudaError_t e = make_score_plan(d, seqs, mods, p.cfg, h, &p.plan, stream);
  if (e != cudaSuccess) return e;
  return d.head_dim == 128 ? pdec::launch<128, true>(p, kv, ctas, stream) : pdec::launch<64, true>(p, kv, ctas, stream);
}

}  // namespace samkv
