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
  // Every kernel is right for every length; up to 16 packed rows per KV head the kernels with short row tiles are faster
  // (32 requests over 20480 slots each: 403 us against 500 us).  Without a hint, one token per sequence is taken for
  // decode.
  const int G = p.n_q_heads / p.n_kv_heads;
  const int longest = p.max_seq_tokens > 0 ? p.max_seq_tokens : (p.n_tokens <= p.n_seq ? 1 : p.n_tokens);
  const bool few_rows = (long long)longest * G <= 16;
  if (p.dtype == SAMKV_F32) {
    // Tiles of 64 rows are the quickest per row, but need work for every SM; tiles of 8 rows (their warps on their own) fill
    // it with less, and waste nothing where a sequence has few rows.  Around the borders, 8/2 heads, 8 rows against 64:
    // 4 x 156 tokens of 64 elements 23.6 against 21.3 us, 800 of 128 74.7 against 81.2, 33 tokens over 2049 slots (4/2 heads
    // of 64) 16.8 against 46.1.  Short prompts have one or two key tiles per item, so 8-row items are mostly fixed cost:
    // 12 x 37 tokens of 64 elements take 14.9 us with 8 rows, 9.2 with 32 and 11.7 with 64.
    const long long rows = (long long)p.n_tokens * p.n_q_heads;
    const bool wide = p.head_dim == 128;
    int tile = 8;
    if (!few_rows && rows >= 64LL * p.n_seq * p.n_kv_heads) {
      if (rows >= (wide ? 40LL : 32LL) * h.sm_count) tile = 64;
      else if (!kv.paged && p.n_tokens <= (wide ? 48LL : 256LL) * p.n_seq) tile = 32;
    }
    if (G > 8 && tile == 8) tile = 32;
    return launch_packed_f32(p, seqs, kv, Q, scale, O, lse, tile, h, stream);
  }
  if (few_rows && kv.paged) return launch_packed_decode(p, seqs, kv, Q, scale, O, lse, h, stream);
  return launch_packed_tc(p, seqs, kv, Q, scale, O, lse, h, stream);
}

}  // namespace samkv
