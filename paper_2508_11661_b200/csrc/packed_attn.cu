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
                              const Rows& O, float* lse, int rows, const samkv_ctx_impl& h, cudaStream_t stream);

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
  if (p.dtype == SAMKV_F32) {
    // 64 rows per tile; 32 where 64 would leave SMs without a tile (4 documents of 256 tokens, 4/2 heads: 27 us with 64),
    // and 16 where a sequence fills less than 64 rows on average (6 sequences of 1 to 64 tokens: 40 us with 64, 26 us).
    const long long rows = (long long)p.n_tokens * p.n_q_heads;
    int tile = few_rows || rows < 64LL * p.n_seq * p.n_kv_heads ? 16 : rows < 64LL * h.sm_count ? 32 : 64;
    if (G > 16 && tile == 16) tile = 32;
    return launch_packed_f32(p, seqs, kv, Q, scale, O, lse, tile, h, stream);
  }
  if (few_rows && kv.paged) return launch_packed_decode(p, seqs, kv, Q, scale, O, lse, h, stream);
  return launch_packed_tc(p, seqs, kv, Q, scale, O, lse, h, stream);
}

}  // namespace samkv
