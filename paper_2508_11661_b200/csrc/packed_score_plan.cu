// The plan of calls with modified scores that have too many row tiles for one warp: see packed_scores.cuh.
#include "packed_scores.cuh"

namespace samkv {

__global__ void __launch_bounds__(kPlanThreads, 1)
score_plan_kernel(const __grid_constant__ Seqs q, const __grid_constant__ ScoreMods m, const __grid_constant__ SplitCfg c,
                  const __grid_constant__ ScorePlan plan, int* __restrict__ d_status) {
  __shared__ PlanScratch<kPlanThreads> scratch;
  pdl_launch_dependents();
  pdl_wait();
  make_plan<kPlanThreads>(q, m, c, plan, scratch, true, d_status);
}

// (which kernel a call gets depends on its lengths and the hint, the workspace does not: as many row tiles as any has)
size_t scores_scratch_bytes(const samkv_packed_t& p) {
  const int G = p.n_q_heads / p.n_kv_heads, rows = p.dtype == SAMKV_BF16 ? 16 : 8;
  const size_t shared = plan_bytes(most_row_tiles(p, G < rows ? rows / G : 1)), own = kMaxPackedCtas * plan_bytes(kBlockTiles);
  return packed_scratch_bytes(p) + 256 + (shared > own ? shared : own);
}

cudaError_t make_score_plan(const samkv_packed_t& p, const Seqs& seqs, const ScoreMods& mods, const SplitCfg& cfg,
                            const samkv_ctx_impl& h, ScorePlan* plan, cudaStream_t stream) {
  const long long tiles = most_row_tiles(p, cfg.tokens);
  *plan = {};
  if (tiles <= kWarpTiles && p.n_seq <= 32) return cudaSuccess;
  char* ws = h.workspace + ((kStatusBytes + packed_scratch_bytes(p) + 255) & ~(size_t)255);
  const bool own = tiles <= kBlockTiles && p.n_seq <= kBlockSeqs;
  const long long room = own ? kBlockTiles : tiles;
  plan->own_bytes = own ? plan_bytes(room) : 0;
  plan->tiles = reinterpret_cast<RowTile*>(ws);
  plan->at = reinterpret_cast<long long*>(plan->tiles + room);
  plan->n_tiles = reinterpret_cast<int*>(plan->at + room + 1);
  if (own) return cudaSuccess;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(1);
  lc.blockDim = dim3(kPlanThreads);
  lc.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = &attr;
  lc.numAttrs = 1;
  return cudaLaunchKernelEx(&lc, score_plan_kernel, seqs, mods, cfg, *plan, h.d_status);
}

}  // namespace samkv
