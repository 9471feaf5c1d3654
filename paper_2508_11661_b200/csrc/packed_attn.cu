// Attention of packed sequences over packed rows or over a paged cache: which kernel a call gets.
#include <math.h>

#include "packed.cuh"

namespace samkv {

size_t packed_tc_scratch_bytes(int d);
cudaError_t launch_packed_tc(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                             const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
cudaError_t launch_packed_decode(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                 const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
size_t packed_f32_scratch_bytes(int d);
cudaError_t launch_packed_f32(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                              const Rows& O, float* lse, bool few_rows, const samkv_ctx_impl& h, cudaStream_t stream);

// (the decode kernel's partial results are an eighth of the tensor-memory kernel's)
size_t packed_scratch_bytes(const samkv_packed_t& p) {
  return p.dtype == SAMKV_BF16 ? packed_tc_scratch_bytes(p.head_dim) : packed_f32_scratch_bytes(p.head_dim);
}

cudaError_t launch_packed_attn(const samkv_packed_t& p, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  if (scale <= 0.f) scale = 1.0f / sqrtf((float)p.head_dim);
  // Every kernel is right for every length; up to 16 packed rows per KV head the kernels with 16-row tiles are faster
  // (32 requests over 20480 slots each: 403 us against 500 us).  Without a hint, one token per sequence is taken for
  // decode. 
  const int G = p.n_q_heads / p.n_kv_heads;
  const int longest = p.max_seq_tokens > 0 ? p.max_seq_tokens : (p.n_tokens <= p.n_seq ? 1 : p.n_tokens);
  const bool few_rows = (long long)longest * G <= 16;
  if (p.dtype == SAMKV_F32) return launch_packed_f32(p, seqs, kv, Q, scale, O, lse, few_rows, h, stream);
  if (few_rows && kv.paged) return launch_packed_decode(p, seqs, kv, Q, scale, O, lse, h, stream);
  return launch_packed_tc(p, seqs, kv, Q, scale, O, lse, h, stream);
}

}  // namespace samkv
