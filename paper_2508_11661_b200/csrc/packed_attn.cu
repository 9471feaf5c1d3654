// Attention of packed sequences over packed rows or over a paged cache: the simple form, right for every case.
// One warp per (token, query head); lane e owns d/32 consecutive elements of the head dimension.
#include <math.h>

#include "packed.cuh"

namespace samkv {

template <typename T, int kEpl>
__device__ __forceinline__ void load_part(const T* p, float* f) {
#pragma unroll
  for (int i = 0; i < kEpl; ++i) {
    if constexpr (sizeof(T) == 4) f[i] = p[i]; else f[i] = __bfloat162float(p[i]);
  }
}

template <typename T, int kD>
__global__ void __launch_bounds__(128)
packed_simple_kernel(const Seqs seqs, const KvSource kv, const Rows Q, const Rows O, float* __restrict__ lse, float scale,
                     int Hq, int Hkv, int* __restrict__ d_status) {
  constexpr int kEpl = kD / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long id = (long long)blockIdx.x * 4 + warp;
  const int tok = (int)(id / Hq), hq = (int)(id % Hq), h = hq / (Hq / Hkv);
  if (tok >= seqs.n_tokens) return;
  int lo = 0, hi = seqs.n_seq;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (seqs.off[mid] <= tok) lo = mid; else hi = mid - 1;
  }
  if (lo >= seqs.n_seq) return;
  const Seq sq = load_seq(seqs, lo);
  if (tok < sq.first || tok >= sq.first + sq.n) return;
  bool bad = false;
  if (sq.clamped && lane == 0) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  const int vis = visible(seqs, sq, tok - sq.first);
  float q[kEpl], acc[kEpl], m = -INFINITY, l = 0.f;
  load_part<T, kEpl>(static_cast<const T*>(Q.data) + (size_t)tok * Q.ts + (size_t)hq * Q.hs + lane * kEpl, q);
#pragma unroll
  for (int i = 0; i < kEpl; ++i) acc[i] = 0.f;
  for (int j = 0; j < vis; ++j) {
    const T *kp, *vp;
    if (kv.paged) {
      const size_t off = page_offset(kv.pages, lo, j, h, Hkv, kD, &bad);
      kp = static_cast<const T*>(kv.pages.K) + off;
      vp = static_cast<const T*>(kv.pages.V) + off;
    } else {
      kp = static_cast<const T*>(kv.K.data) + (size_t)(sq.first + j) * kv.K.ts + (size_t)h * kv.K.hs;
      vp = static_cast<const T*>(kv.V.data) + (size_t)(sq.first + j) * kv.V.ts + (size_t)h * kv.V.hs;
    }
    float kf[kEpl], vf[kEpl];
    load_part<T, kEpl>(kp + lane * kEpl, kf);
    load_part<T, kEpl>(vp + lane * kEpl, vf);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < kEpl; ++i) dot = fmaf(q[i], kf[i], dot);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    const float sc = dot * scale;
    const float m_new = fmaxf(m, sc);
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float corr = expf(m - base);
    const float p = expf(sc - base);
    l = l * corr + p;
#pragma unroll
    for (int i = 0; i < kEpl; ++i) acc[i] = fmaf(p, vf[i], acc[i] * corr);
    m = m_new;
  }
  if (bad && lane == 0) atomicMax(d_status, (int)CHECK_PAGE_RANGE);
  T* op = static_cast<T*>(O.data) + (size_t)tok * O.ts + (size_t)hq * O.hs + lane * kEpl;
#pragma unroll
  for (int i = 0; i < kEpl; ++i) {
    const float v = l == 0.f ? 0.f : acc[i] / l;
    if constexpr (sizeof(T) == 4) op[i] = v; else op[i] = __float2bfloat16_rn(v);
  }
  if (lse != nullptr && lane == 0) lse[(size_t)tok * Hq + hq] = l == 0.f ? -INFINITY : m + logf(l);
}

size_t packed_tc_scratch_bytes(int d);
cudaError_t launch_packed_tc(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                             const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);

size_t packed_decode_scratch_bytes(int d);
cudaError_t launch_packed_decode(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                 const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);

// (the decode kernel's pieces are an eighth of the other's)
size_t packed_scratch_bytes(const samkv_packed_t& p) { return p.dtype == SAMKV_BF16 ? packed_tc_scratch_bytes(p.head_dim) : 0; }

cudaError_t launch_packed_attn(const samkv_packed_t& p, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  if (scale <= 0.f) scale = 1.0f / sqrtf((float)p.head_dim);
  if (p.dtype == SAMKV_BF16) {
    // Up to 16 packed rows per KV head: the decode kernel.  Without a hint, one token per sequence is taken for decode.
    const int longest = p.max_seq_tokens > 0 ? p.max_seq_tokens : (p.n_tokens <= p.n_seq ? 1 : p.n_tokens);
    if (kv.paged && (long long)longest * (p.n_q_heads / p.n_kv_heads) <= 16)
      return launch_packed_decode(p, seqs, kv, Q, scale, O, lse, h, stream);
    return launch_packed_tc(p, seqs, kv, Q, scale, O, lse, h, stream);
  }
  const long long blocks = ((long long)p.n_tokens * p.n_q_heads + 3) / 4;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
#define SAMKV_SIMPLE(T, D) \
  packed_simple_kernel<T, D><<<(unsigned)blocks, 128, 0, stream>>>(seqs, kv, Q, O, lse, scale, p.n_q_heads, p.n_kv_heads, h.d_status)
  if (p.head_dim == 128) SAMKV_SIMPLE(float, 128); else SAMKV_SIMPLE(float, 64);
#undef SAMKV_SIMPLE
  return cudaGetLastError();
}

}  // namespace samkv
