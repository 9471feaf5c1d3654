// Attention of packed sequences over packed rows or over a paged cache: which kernel a call gets.
#include <math.h>

#include "packed.cuh"

namespace samkv {

size_t packed_tc_scratch_bytes(int d);
cudaError_t launch_packed_tc(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                             const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
size_t packed_decode_scratch_bytes(int d);
cudaError_t launch_packed_decode(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                 const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
size_t packed_f32_scratch_bytes(int d);
cudaError_t launch_packed_f32(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                              const Rows& O, float* lse, int rows, const samkv_ctx_impl& h, cudaStream_t stream);

// (which kernel a call gets depends on its lengths, the workspace does not)
size_t packed_scratch_bytes(const samkv_packed_t& p) {
  if (p.dtype != SAMKV_BF16) return packed_f32_scratch_bytes(p.head_dim);
  const size_t tc = packed_tc_scratch_bytes(p.head_dim), decode = packed_decode_scratch_bytes(p.head_dim);
  return tc > decode ? tc : decode;
}

// Every kernel is right for every length; up to 16 packed rows per KV head the kernels with short row tiles are faster
// (32 requests over 20480 slots each 405 us against 425, one over 102400 78 us against 155).  Without a hint, one token
// per sequence is taken for decode.
bool few_rows(const samkv_packed_t& p) {
  const int longest = p.max_seq_tokens > 0 ? p.max_seq_tokens : (p.n_tokens <= p.n_seq ? 1 : p.n_tokens);
  return (long long)longest * (p.n_q_heads / p.n_kv_heads) <= 16;
}

int f32_row_tile(const samkv_packed_t& p, bool paged, int sm_count) {
  // Tiles of 64 rows are the quickest per row but need work for every SM; tiles of 8 rows fill it with an eighth of that
  // and waste nothing where a sequence has few rows; 32 rows lie between.  What decides is the number of 8-row tiles per
  // SM (x below, rows / 8 / SMs).  Measured, us with 8 / 32 / 64 rows:
  //   prompts, d = 64:   x 1.7 (256 tokens, 8/2 heads) 16.8 / 20.3 / 26.0,  x 2.2 (320) 19.0 / 24.1 / 31.4,  x 2.6 (4 x 192, 4/2)
  //                      18.2 / 16.5 / 21.7,  x 4.3 (4 x 320, 4/2) 33.3 / 28.8 / 32.0,  x 5.2 (4 x 192, 8/2) 28.8 / 28.0 / 21.2
  //   prompts, d = 128:  x 2.2 (320, 8/2) 26.9 / 38.2 / 50.1,  x 3.5 (4 x 128) 23.8 / 19.2 / 24.7,  x 5.2 (4 x 192) 40.1 / 45.0 / 33.2
  //   one key tile, d = 64 (where an item is mostly its fixed cost): x 0.9 (4 x 64, 4/2) 6.3 / 8.8 / 11.6,  x 1.7 (4 x 64, 8/2)
  //                      9.3 / 8.7 / 11.1,  x 1.8 (16 x 33, 4/2) 11.2 / 8.1 / 10.7
  //   pages, d = 64:     x 1.8 (16 x 33 over 512) 29.2 / 39.8 / 43.1,  x 3.5 (16 x 64 over 2049) 122 / 130 / 97,  (4 x 256
  //                      over 512) 50.0 / 51.9 / 49.0, over an empty cache, which the host cannot tell, 21.5 / 20.6 / 27.7
  //   pages, d = 128:    x 3.6 (16 x 33 over 512) 62.4 / 85.7 / 83.6,  x 6.9 (16 x 64 over 512) 110 / 129 / 92
  const long long rows = (long long)p.n_tokens * p.n_q_heads, per_x = 8LL * sm_count;
  const bool wide = p.head_dim == 128;
  int tile = 8;
  if (!few_rows(p) && rows >= 64LL * p.n_seq * p.n_kv_heads) {
    if (paged) {
      if (rows >= (wide ? 5 : 3) * per_x) tile = 64;
    } else {
      const bool short_prompts = !wide && p.n_tokens <= 64LL * p.n_seq;
      if (2 * rows >= (wide ? 7 : 9) * per_x) tile = 64;                // x of 3.5 or 4.5
      else if (4 * rows >= (short_prompts ? 5 : 10) * per_x) tile = 32; // x of 1.25 or 2.5
    }
  }
  if (p.n_q_heads / p.n_kv_heads > 8 && tile == 8) tile = 32;
  return tile;
}

cudaError_t launch_packed_attn(const samkv_packed_t& p, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  if (scale <= 0.f) scale = 1.0f / sqrtf((float)p.head_dim);
  if (p.dtype == SAMKV_F32)
    return launch_packed_f32(p, seqs, kv, Q, scale, O, lse, f32_row_tile(p, kv.paged, h.sm_count), h, stream);
  if (few_rows(p) && kv.paged) return launch_packed_decode(p, seqs, kv, Q, scale, O, lse, h, stream);
  return launch_packed_tc(p, seqs, kv, Q, scale, O, lse, h, stream);
}

}  // namespace samkv
