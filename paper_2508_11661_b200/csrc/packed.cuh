// Packed sequences and the paged cache: what the kernels behind samkv_prefill, samkv_append and samkv_paged_attn share
// (internal; the public surface is include/samkv.h).
#pragma once

#include "common.cuh"

namespace samkv {

// A packed tensor as kernels see it: element (token t, head h, e) at data[t * ts + h * hs + e].
struct Rows {
  void* data;
  long long ts, hs;
};

struct Pages {
  void *K, *V;                 // [n_pages][Hkv][page_size][d]
  const int32_t* table;        // [n_seq][width]
  int width, n_pages, shift;   // page_size == 1 << shift
};

// The sequences of a call and what their tokens see.
struct Seqs {
  const int32_t* off;          // [n_seq + 1]
  const int32_t* cache_len;    // [n_seq], null: 0
  int n_seq, n_tokens;
  int limit;                   // most slots of a sequence (pages * page size; INT_MAX without pages)
  int causal;                  // token t sees slots < base + t + 1; otherwise slots < base
};

struct Seq {
  int first, n;                // first packed row, new tokens
  int base;                    // slots seen by every new token
  bool clamped;
  bool backwards;              // ends before it starts
};

__device__ __forceinline__ Seq load_seq(const Seqs& q, int s) {
  Seq r;
  const int a = q.off[s], b = q.off[s + 1], c = q.cache_len != nullptr ? q.cache_len[s] : 0;
  r.first = min(max(a, 0), q.n_tokens);
  r.n = min(max(b, r.first), q.n_tokens) - r.first;
  r.backwards = b < a;
  r.base = min(max(c, 0), q.limit);
  r.clamped = r.first != a || r.first + r.n != b || (r.n > 0 && (r.base != c || (q.causal && r.n > q.limit - r.base)));
  return r;
}

// Slots that token t of the sequence sees: a table that ends sooner cuts them off there (base <= limit, so that nothing
// here passes 32 bits).
__device__ __forceinline__ int visible(const Seqs& q, const Seq& r, int t) {
  return q.causal ? (int)min((unsigned)r.base + (unsigned)t + 1u, (unsigned)q.limit) : r.base;
}

// Where the keys and values of an attention call live: pages, or packed rows (slot j of a sequence = row first + j).
struct KvSource {
  Rows K, V;                   // packed rows (paged == 0)
  Pages pages;
  int paged;
};

// Offset, in elements, of slot j of KV head h in a page pool of one tensor; a bad table entry reads page 0.
__device__ __forceinline__ size_t page_offset(const Pages& p, int s, int j, int h, int Hkv, int d, bool* bad) {
  int page = p.table[(size_t)s * p.width + (j >> p.shift)];
  if ((unsigned)page >= (unsigned)p.n_pages) {
    *bad = true;
    page = 0;
  }
  return ((((size_t)page * Hkv + h) << p.shift) + (j & ((1 << p.shift) - 1))) * d;
}

// Two fp32 values in one 64-bit register, for the two-wide instructions: half the issue slots, the same arithmetic.
typedef unsigned long long f2;
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 join2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ f2 both(float a) { return join2(a, a); }
__device__ __forceinline__ float2 split2(f2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}

struct RopeTable {
  unsigned long long turn[64]; // fraction of a turn per position, 64-bit fixed point
  int rot_dim, interleaved;    // rot_dim == 0: no rotation
};

// ----- launchers (all enqueue on `stream`) ----------------------------------------------------------------
cudaError_t launch_append(const samkv_packed_t& p, const Seqs& seqs, const Rows& K, const Rows& V, const Pages* pages,
                          const RopeTable& rope, const int32_t* positions, const Rows* Q, const Rows* Q_out,
                          const Rows* K_out, const Rows* V_out, int sm_count, int* d_status, cudaStream_t stream);
cudaError_t launch_packed_attn(const samkv_packed_t& p, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                               const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream);
size_t packed_scratch_bytes(const samkv_packed_t& p);

}  // namespace samkv
