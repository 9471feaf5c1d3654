// Position rotation and append of new rows to a paged cache (or to packed rows), one pass over the data.
//
// The angle of (token, pair) is position * turn mod 1 turn in 64-bit fixed point: the product wraps exactly, so the
// reduction of far positions costs one integer multiplication and loses nothing.  The top two bits are the quadrant,
// the rest an angle in [-1/8, 1/8] turns whose fp32 sine and cosine are good to an ulp.  Sines and cosines of a token
// are formed once per CTA in shared memory and shared by all its heads.
#include "packed.cuh"

namespace samkv {

constexpr int kAppendThreads = 128;
constexpr int kMaxAppendTokens = 2;            // tokens per CTA

struct AppendArgs {
  Seqs seqs;
  Rows K, V, Q, Q_out, K_out, V_out;
  Pages pages;
  int has_pages, has_rows, has_q;
  const int32_t* positions;
  int Hq, Hkv;
};

__device__ __forceinline__ float2 turn_sincos(unsigned long long phase) {
  // phase / 2^64 turns = quadrant / 4 + r, r in [-1/8, 1/8)
  const unsigned int top = (unsigned int)(phase >> 32);
  const unsigned int shifted = top + 0x20000000u;                 // + 1/8 turn
  const unsigned int quadrant = shifted >> 30;
  const int rest = (int)(shifted & 0x3fffffffu) - 0x20000000;     // 2^-32 turns
  float s, c;
  sincospif((float)rest * 4.656612873077393e-10f, &s, &c);        // 2^-31 half turns each
  float2 r;                                                       // (cos, sin)
  r.x = (quadrant & 1u) ? ((quadrant & 2u) ? s : -s) : ((quadrant & 2u) ? -c : c);
  r.y = (quadrant & 1u) ? ((quadrant & 2u) ? -c : c) : ((quadrant & 2u) ? -s : s);
  return r;
}

template <typename T, int kD>
__global__ void __launch_bounds__(kAppendThreads)
append_rope_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTable rope, int tokens_per_cta,
                   int* __restrict__ d_status) {
  constexpr int kVec = 16 / (int)sizeof(T);      // elements per 16 bytes
  constexpr int kItems = kD / (2 * kVec);        // an item is two 16-byte pieces of a row
  __shared__ float2 cs[kMaxAppendTokens][kD / 2];
  __shared__ long long page_row[kMaxAppendTokens];   // row of (page, head 0) in the pools, -1: do not write
  __shared__ int live[kMaxAppendTokens];             // the token belongs to a sequence
  __shared__ long long pos[kMaxAppendTokens];        // (cache_len + t passes 32 bits)
  const int tid = threadIdx.x;
  const int tok0 = blockIdx.x * tokens_per_cta;
  const int n_tok = min(tokens_per_cta, a.seqs.n_tokens - tok0);
  pdl_launch_dependents();
  pdl_wait();
  if (tid < n_tok) {
    const int tok = tok0 + tid;
    // last sequence whose first row is <= tok; with empty sequences in between that is the one that owns the row
    int lo = 0, hi = a.seqs.n_seq;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.seqs.off[mid] <= tok) lo = mid; else hi = mid - 1;
    }
    int mine = 0;
    long long p = 0, row = -1;
    if (lo < a.seqs.n_seq) {
      const Seq sq = load_seq(a.seqs, lo);
      if (tok >= sq.first && tok < sq.first + sq.n) {
        mine = 1;
        const long long slot = (long long)sq.base + (tok - sq.first);
        if (sq.clamped) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
        p = a.positions != nullptr ? a.positions[tok] : slot;
        if (a.has_pages) {
          const long long col = slot >> a.pages.shift;
          if (col >= a.pages.width) {
            atomicMax(d_status, (int)CHECK_APPEND_CAPACITY);
          } else {
            const int page = a.pages.table[(size_t)lo * a.pages.width + col];
            if ((unsigned)page >= (unsigned)a.pages.n_pages)
              atomicMax(d_status, (int)CHECK_PAGE_RANGE);
            else
              row = (((long long)page * a.Hkv) << a.pages.shift) + (slot & ((1 << a.pages.shift) - 1));
          }
        }
      }
    }
    live[tid] = mine;
    pos[tid] = p;
    page_row[tid] = row;
  }
  __syncthreads();
  const int half = rope.rot_dim >> 1;
  for (int i = tid; i < n_tok * half; i += kAppendThreads) {
    const int t = i / half, e = i - t * half;
    cs[t][e] = turn_sincos((unsigned long long)pos[t] * rope.turn[e]);
  }
  __syncthreads();

  // items: [token][Q heads, K heads, V heads][kItems]
  const int n_q = a.has_q ? a.Hq : 0;
  const int heads = n_q + 2 * a.Hkv;
  const int per_tok = heads * kItems;
  const int rot_items = half / kVec;             // items of a row that hold rotated pairs (both layouts)
  for (int i = tid; i < n_tok * per_tok; i += kAppendThreads) {
    const int t = i / per_tok, r = i - t * per_tok;
    const int head = r / kItems, it = r - head * kItems;
    if (!live[t]) continue;
    const int tok = tok0 + t;
    const bool is_q = head < n_q, is_v = head >= n_q + a.Hkv;
    const int h = is_q ? head : head - n_q - (is_v ? a.Hkv : 0);
    const bool rotated = !is_v && it < rot_items;
    // element offsets of the two pieces: halves of the rotated part when pairs are (i, i + half), else neighbours
    int e0, e1;
    if (rotated && !rope.interleaved) {
      e0 = it * kVec;
      e1 = half + it * kVec;
    } else {
      e0 = it * 2 * kVec;
      e1 = e0 + kVec;
    }
    const Rows& src = is_q ? a.Q : is_v ? a.V : a.K;
    const T* sp = static_cast<const T*>(src.data) + (size_t)tok * src.ts + (size_t)h * src.hs;
    uint4 x0 = *reinterpret_cast<const uint4*>(sp + e0), x1 = *reinterpret_cast<const uint4*>(sp + e1);
    if (rotated) {
      float u[kVec], w[kVec];
      ElemTraits<T>::unpack(x0, u);
      ElemTraits<T>::unpack(x1, w);
      if (rope.interleaved) {
#pragma unroll
        for (int k = 0; k < kVec; k += 2) {
          const float2 c0 = cs[t][(e0 + k) >> 1], c1 = cs[t][(e1 + k) >> 1];
          const float a0 = u[k], b0 = u[k + 1], a1 = w[k], b1 = w[k + 1];
          u[k] = a0 * c0.x - b0 * c0.y;
          u[k + 1] = b0 * c0.x + a0 * c0.y;
          w[k] = a1 * c1.x - b1 * c1.y;
          w[k + 1] = b1 * c1.x + a1 * c1.y;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          const float2 c = cs[t][e0 + k];
          const float a0 = u[k], b0 = w[k];
          u[k] = a0 * c.x - b0 * c.y;
          w[k] = b0 * c.x + a0 * c.y;
        }
      }
      x0 = ElemTraits<T>::pack(u);
      x1 = ElemTraits<T>::pack(w);
    }
    auto put = [&](T* dst) {
      *reinterpret_cast<uint4*>(dst + e0) = x0;
      *reinterpret_cast<uint4*>(dst + e1) = x1;
    };
    if (is_q) {
      put(static_cast<T*>(a.Q_out.data) + (size_t)tok * a.Q_out.ts + (size_t)h * a.Q_out.hs);
    } else {
      if (a.has_rows) {
        const Rows& dst = is_v ? a.V_out : a.K_out;
        put(static_cast<T*>(dst.data) + (size_t)tok * dst.ts + (size_t)h * dst.hs);
      }
      if (page_row[t] >= 0)
        put(static_cast<T*>(is_v ? a.pages.V : a.pages.K) + ((size_t)page_row[t] + ((size_t)h << a.pages.shift)) * kD);
    }
  }
}

cudaError_t launch_append(const samkv_packed_t& p, const Seqs& seqs, const Rows& K, const Rows& V, const Pages* pages,
                          const RopeTable& rope, const int32_t* positions, const Rows* Q, const Rows* Q_out,
                          const Rows* K_out, const Rows* V_out, int sm_count, int* d_status, cudaStream_t stream) {
  AppendArgs a = {};
  a.seqs = seqs;
  a.K = K;
  a.V = V;
  if (pages != nullptr) { a.pages = *pages; a.has_pages = 1; }
  if (Q != nullptr) { a.Q = *Q; a.Q_out = *Q_out; a.has_q = 1; }
  if (K_out != nullptr) { a.K_out = *K_out; a.V_out = *V_out; a.has_rows = 1; }
  a.positions = positions;
  a.Hq = p.n_q_heads;
  a.Hkv = p.n_kv_heads;
  int per_cta = p.n_tokens / (sm_count * 4);
  if (per_cta > kMaxAppendTokens) per_cta = kMaxAppendTokens;
  if (per_cta < 1) per_cta = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.n_tokens + per_cta - 1) / per_cta));
  cfg.blockDim = dim3(kAppendThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (p.dtype == SAMKV_BF16)
    return p.head_dim == 128
               ? cudaLaunchKernelEx(&cfg, append_rope_kernel<__nv_bfloat16, 128>, a, rope, per_cta, d_status)
               : cudaLaunchKernelEx(&cfg, append_rope_kernel<__nv_bfloat16, 64>, a, rope, per_cta, d_status);
  return p.head_dim == 128 ? cudaLaunchKernelEx(&cfg, append_rope_kernel<float, 128>, a, rope, per_cta, d_status)
                           : cudaLaunchKernelEx(&cfg, append_rope_kernel<float, 64>, a, rope, per_cta, d_status);
}

}  // namespace samkv
