// The plan of calls with modified scores that have too many row tiles for one warp: see packed_scores.cuh.
#include "packed_scores.cuh"

namespace samkv {

// One block: records and lengths of all row tiles of a call.
__global__ void __launch_bounds__(kPlanThreads, 1)
score_plan_kernel(const __grid_constant__ Seqs q, const __grid_constant__ ScoreMods m, const __grid_constant__ SplitCfg c,
                  const __grid_constant__ ScorePlan plan, int* __restrict__ d_status) {
  __shared__ int s_off[kPlanThreads];          // row tiles of the chunk's sequences before each
  __shared__ int s_warp[32];
  __shared__ unsigned s_lo[32], s_hi[32];      // lengths, by halves
  __shared__ int s_end;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_launch_dependents();
  if (tid == 0) s_end = q.n_seq;
  pdl_wait();
  __syncthreads();
  for (int s = tid; s < q.n_seq; s += kPlanThreads) {
    const Seq x = load_seq(q, s);
    if (x.backwards) atomicMin(&s_end, s);
    if (x.clamped) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  }
  __syncthreads();
  const int n_seq = s_end;
  int n_tiles = 0;                             // so far
  long long total = 0;
#pragma unroll 1
  for (int s0 = 0; s0 < n_seq; s0 += kPlanThreads) {
    // row tiles of these sequences
    int R = 0;
    if (s0 + tid < n_seq) R = row_tiles(c, load_seq(q, s0 + tid).n);
    int incl = R;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int w = s_warp[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += v;
    }
    const int chunk = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    s_off[tid] = (warp > 0 ? before : 0) + incl - R;
    __syncthreads();
    const int count = min(kPlanThreads, n_seq - s0);
    // their records, and the lengths
#pragma unroll 1
    for (int i0 = 0; i0 < chunk; i0 += kPlanThreads) {
      const int i = i0 + tid;
      long long len = 0;
      RowTile t = {};
      if (i < chunk) {
        int lo = 0, hi = count - 1;            // last sequence that starts at or before i: the one that owns it
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (s_off[mid] <= i) lo = mid; else hi = mid - 1;
        }
        t = make_row_tile(q, m, c, s0 + lo, load_seq(q, s0 + lo), i - s_off[lo]);
      }
      if (chunk > 256 && c.tokens > 8) finish_row_tiles<true>(q, m, c, i < chunk, t);
      else finish_row_tiles<false>(q, m, c, i < chunk, t);
      if (i < chunk) {
        plan.tiles[n_tiles + i] = t;
        len = (long long)t.nt * c.tile + c.fixed;
      }
      long long li = len;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, li, o);
        if (lane >= o) li += v;
      }
      __syncthreads();
      if (lane == 31) {
        s_lo[warp] = (unsigned)li;
        s_hi[warp] = (unsigned)(li >> 32);
      }
      __syncthreads();
      long long wl = (long long)((unsigned long long)s_hi[lane] << 32 | s_lo[lane]);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, wl, o);
        if (lane >= o) wl += v;
      }
      const long long all = __shfl_sync(0xffffffffu, wl, 31);
      const long long bw = __shfl_sync(0xffffffffu, wl, (warp + 31) & 31);
      if (i < chunk) plan.at[n_tiles + i] = total + (warp > 0 ? bw : 0) + li - len;
      total += all;
    }
    n_tiles += chunk;
  }
  if (tid == 0) {
    plan.at[n_tiles] = total;
    *plan.n_tiles = n_tiles;
  }
}

// (which kernel a call gets depends on its lengths and the hint, the workspace does not: as many row tiles as any has)
size_t scores_scratch_bytes(const samkv_packed_t& p) {
  const int G = p.n_q_heads / p.n_kv_heads, rows = p.dtype == SAMKV_BF16 ? 16 : 8;
  return packed_scratch_bytes(p) + score_plan_bytes(most_row_tiles(p, G < rows ? rows / G : 1));
}

cudaError_t make_score_plan(const samkv_packed_t& p, const Seqs& seqs, const ScoreMods& mods, const SplitCfg& cfg,
                            const samkv_ctx_impl& h, ScorePlan* plan, cudaStream_t stream) {
  const long long tiles = most_row_tiles(p, cfg.tokens);
  *plan = {nullptr, nullptr, nullptr};
  if (tiles <= kWarpTiles && p.n_seq <= 32) return cudaSuccess;
  char* ws = h.workspace + ((kStatusBytes + packed_scratch_bytes(p) + 255) & ~(size_t)255);
  plan->tiles = reinterpret_cast<RowTile*>(ws);
  plan->at = reinterpret_cast<long long*>(plan->tiles + tiles);
  plan->n_tiles = reinterpret_cast<int*>(plan->at + tiles + 1);
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
