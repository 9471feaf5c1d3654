// Calls of the fp32 attention kernel in packed_f32.cuh with modified scores.
#include "packed_f32.cuh"

namespace samkv {

cudaError_t launch_packed_f32_scores(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                     const ScoreMods& mods, const Rows& O, float* lse, int rows, const samkv_ctx_impl& h,
                                     cudaStream_t stream) {
  pf32::Params p = pf32::make_params(d, seqs, kv, Q, scale, O, lse, rows, h);
  p.mods = mods;
  p.cap_in = mods.softcap > 0.f ? 1.f / mods.softcap : 0.f;
  p.cfg.tokens = rows / p.cfg.G;
  const cudaError_t e = make_score_plan(d, seqs, mods, p.cfg, h, &p.plan, stream);
  if (e != cudaSuccess) return e;
  return pf32::launch_rows<true>(p, kv.paged, d.head_dim, rows, h, stream);
}

}  // namespace samkv
