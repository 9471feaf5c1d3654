// Attention of packed sequences with modified scores: softcap, distance slopes, windows, prefixes and documents.
//
// One warp per (token, query head) walks the slots that the token sees, one at a time, with a running maximum and sum in
// fp32; a lane owns every 32nd pair of elements.
#include <math.h>

#include "packed.cuh"

namespace samkv {
namespace pscore {

struct Params {
  Seqs seqs;
  ScoreMods mods;
  KvSource kv;
  Rows Q, O;
  float scale;
  float* lse;
  int* d_status;
  int Hq, Hkv;
};

template <typename T>
__device__ __forceinline__ float2 load2(const T* p);
template <>
__device__ __forceinline__ float2 load2<float>(const float* p) { return *reinterpret_cast<const float2*>(p); }
template <>
__device__ __forceinline__ float2 load2<__nv_bfloat16>(const __nv_bfloat16* p) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  return make_float2(bf16_lo(w), bf16_hi(w));
}

template <typename T, int kD>
__global__ void __launch_bounds__(128)
scores_attn_kernel(const __grid_constant__ Params p) {
  constexpr int kPairs = kD / 64;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int tok = (int)(item / p.Hq), hq = (int)(item % p.Hq), h = hq / (p.Hq / p.Hkv);
  if (tok >= p.seqs.n_tokens) return;
  // the sequence that holds the token; one that ends before it starts ends the list
  int s = -1;
  for (int s0 = 0; s0 < p.seqs.n_seq && s < 0; s0 += 32) {
    Seq q = {0, 0, 0, false, false};
    if (s0 + lane < p.seqs.n_seq) q = load_seq(p.seqs, s0 + lane);
    if (q.clamped && item == 0) atomicMax(p.d_status, (int)CHECK_SEQ_RANGE);
    const unsigned back = __ballot_sync(0xffffffffu, q.backwards);
    const unsigned mine = __ballot_sync(0xffffffffu, tok >= q.first && tok < q.first + q.n);
    const unsigned list = back == 0 ? 0xffffffffu : (1u << (__ffs(back) - 1)) - 1u;
    if (mine & list) s = s0 + __ffs(mine & list) - 1;
    if (back != 0) break;
  }
  if (s < 0) return;
  const Seq sq = load_seq(p.seqs, s);
  const int t = tok - sq.first, pos = sq.base + t;
  const int end = visible(p.seqs, sq, t), all = visible(p.seqs, sq, sq.n - 1);
  const int prefix = p.mods.prefix_len != nullptr ? min(max(p.mods.prefix_len[s], 0), all) : 0;
  int low = p.mods.doc_start != nullptr ? max(p.mods.doc_start[tok], 0) : 0;
  if (p.mods.window < INT_MAX) low = max(low, pos - p.mods.window + 1);
  low = max(low, prefix);
  const float slope = p.mods.slopes != nullptr ? p.mods.slopes[hq] : 0.f;
  const T* qp = static_cast<const T*>(p.Q.data) + (size_t)tok * p.Q.ts + (size_t)hq * p.Q.hs;
  float2 q[kPairs], o[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    q[i] = load2<T>(qp + i * 64 + lane * 2);
    o[i] = make_float2(0.f, 0.f);
  }
  float m = -INFINITY, l = 0.f;
  bool bad = false;
  for (int part = 0; part < 2; ++part) {
    for (int j = part == 0 ? 0 : low; j < (part == 0 ? prefix : end); ++j) {
      const T *kp, *vp;
      if (p.kv.paged) {
        const size_t at = page_offset(p.kv.pages, s, j, h, p.Hkv, kD, &bad);
        kp = static_cast<const T*>(p.kv.pages.K) + at;
        vp = static_cast<const T*>(p.kv.pages.V) + at;
      } else {
        kp = static_cast<const T*>(p.kv.K.data) + (size_t)(sq.first + j) * p.kv.K.ts + (size_t)h * p.kv.K.hs;
        vp = static_cast<const T*>(p.kv.V.data) + (size_t)(sq.first + j) * p.kv.V.ts + (size_t)h * p.kv.V.hs;
      }
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 k = load2<T>(kp + i * 64 + lane * 2);
        x = fmaf(q[i].x, k.x, fmaf(q[i].y, k.y, x));
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
      x *= p.scale;
      if (p.mods.softcap > 0.f) x = p.mods.softcap * tanhf(x / p.mods.softcap);
      x -= slope * fabsf((float)(pos - j));
      const float mn = x > m ? x : (x == x ? m : x);       // NaN stays
      const float mu = mn == -INFINITY ? 0.f : mn;
      const float corr = expf(m - mu), w = expf(x - mu);
      m = mn;
      l = l * corr + w;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 v = load2<T>(vp + i * 64 + lane * 2);
        o[i].x = fmaf(w, v.x, o[i].x * corr);
        o[i].y = fmaf(w, v.y, o[i].y * corr);
      }
    }
  }
  if (bad) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T* op = static_cast<T*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    op[i * 64 + lane * 2] = (T)(l == 0.f ? 0.f : o[i].x * inv);
    op[i * 64 + lane * 2 + 1] = (T)(l == 0.f ? 0.f : o[i].y * inv);
  }
  if (lane == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T, int kD>
static cudaError_t launch(const Params& p, cudaStream_t stream) {
  const long long items = (long long)p.seqs.n_tokens * p.Hq;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((items + 3) / 4));
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, scores_attn_kernel<T, kD>, p);
}
}  // namespace pscore

cudaError_t launch_packed_tc_mask(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
cudaError_t launch_packed_tc_cap(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
cudaError_t launch_packed_tc_bias(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);

cudaError_t launch_scores_attn(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const ScoreMods& mods, const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  if (scale <= 0.f) scale = 1.0f / sqrtf((float)d.head_dim);
  if (d.dtype == SAMKV_BF16) {
    auto launch = mods.slopes != nullptr ? launch_packed_tc_bias : mods.softcap > 0.f ? launch_packed_tc_cap : launch_packed_tc_mask;
    return launch(d, seqs, kv, Q, scale, mods, O, lse, h, stream);
  }
  const pscore::Params p = {seqs, mods, kv, Q, O, scale, lse, h.d_status, d.n_q_heads, d.n_kv_heads};
  return d.head_dim == 128 ? pscore::launch<float, 128>(p, stream) : pscore::launch<float, 64>(p, stream);
}

}  // namespace samkv
