// Position rotation and append of new rows to a paged cache (or to packed rows), one pass over the data.
//
// The angle of (token, pair) is position * turn mod 1 turn in 64-bit fixed point: the product wraps exactly, so the
// reduction of far positions costs one integer multiplication and loses nothing.  The top two bits are the quadrant,
// the rest an angle in [-1/8, 1/8] turns whose fp32 sine and cosine are good to an ulp.  Sines and cosines of a token
// are formed once per CTA in shared memory and shared by all its heads.
// Bound by HBM: 20480 tokens, 32/8 heads of 128: 85 us (a copy of the same bytes 83), with three axes and a slot map 88 us.  A
// thread's first two items are fetched before the positions are looked up (92 and 99 us without; 3 items 93, 4 97, 6 110).
#include "packed.cuh"

namespace samkv {

constexpr int kAppendThreads = 128;
constexpr int kMaxAppendTokens = 2;            // tokens per CTA
constexpr int kBatch = 2;                       // items of a thread under way at a time

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

// kAxes: positions of several axes, and rows found by a slot map where one is given.
template <typename T, int kD, bool kAxes>
__global__ void __launch_bounds__(kAppendThreads)
append_rope_kernel(const __grid_constant__ AppendArgs a, const __grid_constant__ RopeTable rope,
                   const __grid_constant__ AppendAxes axes, int tokens_per_cta, int* __restrict__ d_status) {
  constexpr int kVec = 16 / (int)sizeof(T);      // elements per 16 bytes
  constexpr int kItems = kD / (2 * kVec);        // an item is two 16-byte pieces of a row
  __shared__ float2 cs[kMaxAppendTokens][kD / 2];
  __shared__ long long page_row[kMaxAppendTokens];   // row of (page, head 0) in the pools, -1: do not write
  __shared__ int live[kMaxAppendTokens];             // the token belongs to a sequence
  __shared__ long long pos[kMaxAppendTokens * (kAxes ? SAMKV_MAX_AXES : 1)];   // (cache_len + t passes 32 bits)
  const int tid = threadIdx.x;
  const int tok0 = blockIdx.x * tokens_per_cta;
  const int n_tok = min(tokens_per_cta, a.seqs.n_tokens - tok0);
  pdl_launch_dependents();
  pdl_wait();
  // items: [token][Q heads, K heads, V heads][kItems]; a thread's first kBatch are fetched before the positions are known
  const int half = rope.rot_dim >> 1;
  const int n_q = a.has_q ? a.Hq : 0;
  const int per_tok = (n_q + 2 * a.Hkv) * kItems, n_items = n_tok * per_tok;
  const int rot_items = half / kVec;             // items of a row that hold rotated pairs (both layouts)
  struct Item {
    int t, h, e0, e1;                            // token, head, element offsets of the two pieces
    bool is_q, is_v, rotated;
  };
  auto item = [&](int i) {
    Item x;
    x.t = i >= per_tok ? 1 : 0;
    static_assert(kMaxAppendTokens == 2, "tokens of a CTA");
    const int r = i - x.t * per_tok, head = r / kItems, it = r % kItems;
    x.is_q = head < n_q;
    x.is_v = head >= n_q + a.Hkv;
    x.h = x.is_q ? head : head - n_q - (x.is_v ? a.Hkv : 0);
    x.rotated = !x.is_v && it < rot_items;
    // halves of the rotated part when pairs are (i, i + half), else neighbours
    const bool halves = x.rotated && !rope.interleaved;
    x.e0 = halves ? it * kVec : it * 2 * kVec;
    x.e1 = halves ? half + it * kVec : x.e0 + kVec;
    return x;
  };
  uint4 x0[kBatch], x1[kBatch];
  auto fetch = [&](int first) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = first + k * kAppendThreads;
      if (i >= n_items) break;
      const Item x = item(i);
      const Rows& src = x.is_q ? a.Q : x.is_v ? a.V : a.K;
      const T* sp = static_cast<const T*>(src.data) + (size_t)(tok0 + x.t) * src.ts + (size_t)x.h * src.hs;
      x0[k] = *reinterpret_cast<const uint4*>(sp + x.e0);
      x1[k] = *reinterpret_cast<const uint4*>(sp + x.e1);
    }
  };
  fetch(tid);
  const bool mapped = kAxes && axes.slots != nullptr;
  if (mapped && tid < n_tok) {
    const int slot = axes.slots[tok0 + tid];
    const bool in_pool = slot < a.pages.n_pages << a.pages.shift;
    if (!in_pool) atomicMax(d_status, (int)CHECK_PAGE_RANGE);
    const int page = slot >> a.pages.shift;
    live[tid] = slot >= 0 && in_pool;
    page_row[tid] = (((long long)page * a.Hkv) << a.pages.shift) + (slot & ((1 << a.pages.shift) - 1));
  }
  if (!mapped && tid < n_tok) {
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
        p = !kAxes && a.positions != nullptr ? a.positions[tok] : slot;
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
    page_row[tid] = row;
    if constexpr (kAxes) {
#pragma unroll
      for (int i = 0; i < SAMKV_MAX_AXES; ++i) pos[tid * SAMKV_MAX_AXES + i] = p;
    } else {
      pos[tid] = p;
    }
  }
  if constexpr (kAxes) {
    if (a.positions != nullptr) {
      __syncthreads();
      if (tid < n_tok * axes.n_axes) {
        const int t = tid / axes.n_axes, i = tid - t * axes.n_axes;
        pos[t * SAMKV_MAX_AXES + i] = a.positions[i * axes.axis_stride + tok0 + t];
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < n_tok * half; i += kAppendThreads) {
    const int t = i / half, e = i - t * half;
    const long long at = kAxes ? pos[t * SAMKV_MAX_AXES + axes.axis[e]] : pos[t];
    cs[t][e] = turn_sincos((unsigned long long)at * rope.turn[e]);
  }
  __syncthreads();

#pragma unroll 1
  for (int first = tid; first < n_items; first += kBatch * kAppendThreads) {
    if (first != tid) fetch(first);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = first + k * kAppendThreads;
      if (i >= n_items) break;
      const Item x = item(i);
      if (!live[x.t]) continue;
      if (x.rotated) {
        float u[kVec], w[kVec];
        ElemTraits<T>::unpack(x0[k], u);
        ElemTraits<T>::unpack(x1[k], w);
        if (rope.interleaved) {
#pragma unroll
          for (int e = 0; e < kVec; e += 2) {
            const float2 c0 = cs[x.t][(x.e0 + e) >> 1], c1 = cs[x.t][(x.e1 + e) >> 1];
            const float a0 = u[e], b0 = u[e + 1], a1 = w[e], b1 = w[e + 1];
            u[e] = a0 * c0.x - b0 * c0.y;
            u[e + 1] = b0 * c0.x + a0 * c0.y;
            w[e] = a1 * c1.x - b1 * c1.y;
            w[e + 1] = b1 * c1.x + a1 * c1.y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float2 c = cs[x.t][x.e0 + e];
            const float a0 = u[e], b0 = w[e];
            u[e] = a0 * c.x - b0 * c.y;
            w[e] = b0 * c.x + a0 * c.y;
          }
        }
        x0[k] = ElemTraits<T>::pack(u);
        x1[k] = ElemTraits<T>::pack(w);
      }
      const int tok = tok0 + x.t;
      auto put = [&](T* dst) {
        *reinterpret_cast<uint4*>(dst + x.e0) = x0[k];
        *reinterpret_cast<uint4*>(dst + x.e1) = x1[k];
      };
      if (x.is_q) {
        put(static_cast<T*>(a.Q_out.data) + (size_t)tok * a.Q_out.ts + (size_t)x.h * a.Q_out.hs);
      } else {
        if (a.has_rows) {
          const Rows& dst = x.is_v ? a.V_out : a.K_out;
          put(static_cast<T*>(dst.data) + (size_t)tok * dst.ts + (size_t)x.h * dst.hs);
        }
        if (page_row[x.t] >= 0)
          put(static_cast<T*>(x.is_v ? a.pages.V : a.pages.K) + ((size_t)page_row[x.t] + ((size_t)x.h << a.pages.shift)) * kD);
      }
    }
  }
}

cudaError_t launch_append(const samkv_packed_t& p, const Seqs& seqs, const Rows& K, const Rows& V, const Pages* pages,
                          const RopeTable& rope, const int32_t* positions, const Rows* Q, const Rows* Q_out,
                          const Rows* K_out, const Rows* V_out, const AppendAxes* axes, int sm_count, int* d_status,
                          cudaStream_t stream) {
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
  const AppendAxes none = {};
#define SAMKV_APPEND(T, D) \
  (axes != nullptr ? cudaLaunchKernelEx(&cfg, append_rope_kernel<T, D, true>, a, rope, *axes, per_cta, d_status) \
                   : cudaLaunchKernelEx(&cfg, append_rope_kernel<T, D, false>, a, rope, none, per_cta, d_status))
  if (p.dtype == SAMKV_BF16) return p.head_dim == 128 ? SAMKV_APPEND(__nv_bfloat16, 128) : SAMKV_APPEND(__nv_bfloat16, 64);
  return p.head_dim == 128 ? SAMKV_APPEND(float, 128) : SAMKV_APPEND(float, 64);
#undef SAMKV_APPEND
}

}  // namespace samkv
