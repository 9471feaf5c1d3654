// Attention with modified scores: which kernel a call gets.
#include <math.h>

#include "packed.cuh"

namespace samkv {

#define SAMKV_SCORES_LAUNCHER(name) \
  cudaError_t name(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale, const ScoreMods& mods, \
                   const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream)
SAMKV_SCORES_LAUNCHER(launch_packed_tc_mask);
SAMKV_SCORES_LAUNCHER(launch_packed_tc_cap);
SAMKV_SCORES_LAUNCHER(launch_packed_tc_bias);
SAMKV_SCORES_LAUNCHER(launch_packed_decode_scores);
#undef SAMKV_SCORES_LAUNCHER
cudaError_t launch_packed_f32_scores(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                     const ScoreMods& mods, const Rows& O, float* lse, int rows, const samkv_ctx_impl& h,
                                     cudaStream_t stream);

// The rules of the plain calls, whose borders were measured on plain calls (masks change how much work a row tile has).
cudaError_t launch_scores_attn(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  if (scale <= 0.f) scale = 1.0f / sqrtf((float)d.head_dim);
  if (d.dtype == SAMKV_F32)
    return launch_packed_f32_scores(d, seqs, kv, Q, scale, mods, O, lse, f32_row_tile(d, kv.paged, h.sm_count), h, stream);
  if (kv.paged && few_rows(d)) return launch_packed_decode_scores(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
  if (mods.slopes != nullptr) return launch_packed_tc_bias(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
  if (mods.softcap > 0.f) return launch_packed_tc_cap(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
  return launch_packed_tc_mask(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
}

}  // namespace samkv
