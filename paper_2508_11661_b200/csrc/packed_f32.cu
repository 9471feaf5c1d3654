// Plain calls of the fp32 attention kernel in packed_f32.cuh.
#include "packed_f32.cuh"

namespace samkv {

size_t packed_f32_scratch_bytes(int d) { return (size_t)2 * kMaxPackedCtas * 64 * ((size_t)d * 4 + 8); }

cudaError_t launch_packed_f32(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                              const Rows& O, float* lse, int rows, const samkv_ctx_impl& h, cudaStream_t stream) {
  const pf32::Params p = pf32::make_params(d, seqs, kv, Q, scale, O, lse, rows, h);
  return pf32::launch_rows<false>(p, kv.paged, d.head_dim, rows, h, stream);
}

}  // namespace samkv
