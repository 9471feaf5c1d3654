// Plain calls of the decode kernel in packed_decode.cuh.
#include "packed_decode.cuh"

namespace samkv {

size_t packed_decode_scratch_bytes(int d) { return (size_t)2 * kMaxPackedCtas * pdec::kRows * ((size_t)d * 4 + 8); }

cudaError_t launch_packed_decode(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                 const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  const pdec::Params p = pdec::make_params(d, seqs, kv, Q, scale, O, lse, h, ctas);
  return d.head_dim == 128 ? pdec::launch<128, false>(p, kv, ctas, stream) : pdec::launch<64, false>(p, kv, ctas, stream);
}

}  // namespace samkv
