// Calls of the tcgen05 attention kernel in packed_tc.cuh with modified scores.
#include "packed_tc.cuh"

namespace samkv {

cudaError_t launch_packed_tc_scores(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                    const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h,
                                    cudaStream_t stream) {
  ptc::Params p = ptc::make_params(d, seqs, kv, Q, scale, O, lse, h);
  p.cfg.wave_slots = 0;
  p.mods = mods;
  if (mods.softcap > 0.f) {
    p.cap_in = scale / mods.softcap;
    p.cap_out = mods.softcap * tc::kLog2e;
  }
  const cudaError_t e = make_score_plan(d, seqs, mods, p.cfg, h, &p.plan, stream);
  if (e != cudaSuccess) return e;
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  if (d.head_dim == 128)
    return kv.paged ? ptc::launch<128, true, true>(p, ctas, stream) : ptc::launch<128, false, true>(p, ctas, stream);
  return kv.paged ? ptc::launch<64, true, true>(p, ctas, stream) : ptc::launch<64, false, true>(p, ctas, stream);
}

}  // namespace samkv
