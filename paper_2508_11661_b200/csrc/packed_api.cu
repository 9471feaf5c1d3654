// Entry points for packed sequences and the paged cache: argument validation and dispatch.  Arguments are checked before
// the handle's device is, so that a refusal does not depend on the machine it is asked on.
#include <limits.h>
#include <math.h>

#include "packed.cuh"

using namespace samkv;

namespace {

samkv_status_t check_packed(const samkv_packed_t* p) {
  if (p == nullptr) return SAMKV_ERR_INVALID_ARG;
  if (p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) return SAMKV_ERR_INVALID_ARG;
  if (p->n_q_heads / p->n_kv_heads > 32 || p->n_q_heads > 65535) return SAMKV_ERR_UNSUPPORTED;
  if (p->head_dim != 64 && p->head_dim != 128) return SAMKV_ERR_UNSUPPORTED;
  if (p->dtype != SAMKV_F32 && p->dtype != SAMKV_BF16) return SAMKV_ERR_UNSUPPORTED;
  if (p->n_seq < 1 || p->n_tokens < 0 || p->max_seq_tokens < 0) return SAMKV_ERR_INVALID_ARG;
  if (p->n_seq > SAMKV_MAX_SEQ) return SAMKV_ERR_UNSUPPORTED;
  if (p->seq_offsets == nullptr || (reinterpret_cast<uintptr_t>(p->seq_offsets) & 3u) != 0) return SAMKV_ERR_INVALID_ARG;
  return SAMKV_OK;
}

// Validates a packed tensor of n_tokens x heads rows; strides along an axis of extent 1 are replaced by a dense one.
samkv_status_t check_rows(const samkv_packed_t& p, const samkv_rows_t* r, int heads, bool output, Rows* out) {
  if (r == nullptr || r->data == nullptr || !aligned16(r->data)) return SAMKV_ERR_INVALID_ARG;
  const int d = p.head_dim, vec = p.dtype == SAMKV_BF16 ? 8 : 4;
  long long ts = r->token_stride, hs = r->head_stride;
  if (heads == 1) hs = d;
  if (p.n_tokens == 1) ts = (long long)heads * (hs > d ? hs : d);
  if (ts < d || hs < d || ts % vec != 0 || hs % vec != 0) return SAMKV_ERR_INVALID_ARG;
  if (ts > (1LL << 36) || hs > (1LL << 36) || ts > (1LL << 46) / p.n_tokens) return SAMKV_ERR_UNSUPPORTED;
  if (output && ts < (long long)(heads - 1) * hs + d && hs < (long long)(p.n_tokens - 1) * ts + d)
    return SAMKV_ERR_INVALID_ARG;                                  // rows overlap
  out->data = r->data;
  out->ts = ts;
  out->hs = hs;
  return SAMKV_OK;
}

samkv_status_t check_pages(const samkv_packed_t& p, const samkv_pages_t* g, Pages* out) {
  if (g == nullptr || g->K == nullptr || g->V == nullptr || g->block_table == nullptr) return SAMKV_ERR_INVALID_ARG;
  if (!aligned16(g->K) || !aligned16(g->V) || (reinterpret_cast<uintptr_t>(g->block_table) & 3u) != 0)
    return SAMKV_ERR_INVALID_ARG;
  if (g->n_pages < 1 || g->table_width < 1) return SAMKV_ERR_INVALID_ARG;
  int shift = 4;
  while (shift <= 8 && (1 << shift) != g->page_size) ++shift;
  if (shift > 8) return SAMKV_ERR_UNSUPPORTED;
  if ((long long)g->table_width * g->page_size > (1LL << 30)) return SAMKV_ERR_UNSUPPORTED;
  if ((long long)g->n_pages * p.n_kv_heads * g->page_size > INT_MAX) return SAMKV_ERR_UNSUPPORTED;
  out->K = g->K;
  out->V = g->V;
  out->table = g->block_table;
  out->width = g->table_width;
  out->n_pages = g->n_pages;
  out->shift = shift;
  return SAMKV_OK;
}

samkv_status_t make_rope(const samkv_packed_t& p, const samkv_rope_t* r, RopeTable* out) {
  out->rot_dim = 0;
  out->interleaved = 0;
  if (r == nullptr) return SAMKV_OK;
  if (r->rot_dim < 16 || r->rot_dim > p.head_dim || r->rot_dim % 16 != 0) return SAMKV_ERR_INVALID_ARG;
  if (r->inv_freq == nullptr && !(r->base > 0.0 && isfinite(r->base))) return SAMKV_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559005768L;
  if (r->inv_freq == nullptr) {
    // base^(-2i/rot_dim) as powers of one ratio: a call pays for one power, and 63 products in 64-bit mantissas lose 2^-58.
    // A base below 1 turns faster than once in 2 pi; its turns are reduced like given ones.
    const long double ratio = powl((long double)r->base, -2.0L / r->rot_dim), unit = 18446744073709551616.0L / two_pi;
    long double power = unit;
    for (int i = 0; i < r->rot_dim / 2; ++i, power *= ratio) {
      const long double x = (power < 18446744073709551616.0L ? power : fmodl(power, 18446744073709551616.0L)) + 0.5L;
      out->turn[i] = x >= 18446744073709551616.0L ? 0ull : (unsigned long long)x;
    }
  } else {
    for (int i = 0; i < r->rot_dim / 2; ++i) {
      if (!isfinite(r->inv_freq[i])) return SAMKV_ERR_INVALID_ARG;
      long double turn = (long double)r->inv_freq[i] / two_pi;
      turn -= floorl(turn);                                        // whole turns of a position change nothing
      const long double scaled = roundl(ldexpl(turn, 64));
      out->turn[i] = scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
    }
  }
  out->rot_dim = r->rot_dim;
  out->interleaved = r->interleaved != 0;
  return SAMKV_OK;
}

bool same_rows(const Rows& a, const Rows& b) { return a.data == b.data && a.ts == b.ts && a.hs == b.hs; }

// May two packed tensors share memory?  (No only where their strides show it.)
bool rows_overlap(const samkv_packed_t& p, const Rows& a, int heads_a, const Rows& b, int heads_b) {
  const long long e = p.dtype == SAMKV_BF16 ? 2 : 4;
  auto bytes = [&](const Rows& r, int heads) {
    return e * ((p.n_tokens - 1) * r.ts + (heads - 1) * r.hs + p.head_dim);
  };
  const char *a0 = (const char*)a.data, *b0 = (const char*)b.data;
  if (a0 + bytes(a, heads_a) <= b0 || b0 + bytes(b, heads_b) <= a0) return false;
  // Slices of one matrix or slab share an address range without sharing rows: with one stride along an axis, two tensors
  // that lie in disjoint ranges of it at every step do not overlap.  (Columns of one fused matrix: the token axis; heads of
  // K and V that alternate in one slab: the head axis.)
  auto apart = [&](long long stride, long long width_a, long long width_b) {
    long long gap = (b0 - a0) % stride;
    if (gap < 0) gap += stride;
    return gap >= width_a && gap + width_b <= stride;
  };
  const long long row = e * p.head_dim;
  if (a.ts == b.ts && apart(a.ts * e, e * (heads_a - 1) * a.hs + row, e * (heads_b - 1) * b.hs + row)) return false;
  if (a.hs == b.hs && apart(a.hs * e, e * (p.n_tokens - 1) * a.ts + row, e * (p.n_tokens - 1) * b.ts + row)) return false;
  return true;
}

// Does a packed tensor's address range meet one of the pools, or (r == nullptr) one pool the other?
bool meets_pools(const samkv_packed_t& p, const Pages& g, const Rows* r, int heads) {
  const long long e = p.dtype == SAMKV_BF16 ? 2 : 4, pool = (((long long)g.n_pages * p.n_kv_heads) << g.shift) * p.head_dim * e;
  const char *k = (const char*)g.K, *v = (const char*)g.V;
  if (r == nullptr) return k < v + pool && v < k + pool;
  const char* a = (const char*)r->data;
  const char* b = a + e * ((p.n_tokens - 1) * r->ts + (heads - 1) * r->hs + p.head_dim);
  return (a < k + pool && k < b) || (a < v + pool && v < b);
}

samkv_status_t check_workspace(const samkv_ctx_impl* h, const samkv_packed_t& p) {
  return h->workspace_bytes < kStatusBytes + packed_scratch_bytes(p) ? SAMKV_ERR_WORKSPACE : SAMKV_OK;
}

}  // namespace

extern "C" {

size_t samkv_packed_workspace_bytes(const samkv_packed_t* packed) {
  // (the offsets need not exist yet when the workspace is sized)
  if (packed == nullptr) return 0;
  samkv_packed_t p = *packed;
  static const int32_t kSomeOffsets = 0;
  if (p.seq_offsets == nullptr) p.seq_offsets = &kSomeOffsets;
  if (check_packed(&p) != SAMKV_OK) return 0;
  return kStatusBytes + packed_scratch_bytes(p);
}

samkv_status_t samkv_prefill(samkv_handle_t handle, const samkv_packed_t* packed, const samkv_rows_t* Q,
                             const samkv_rows_t* K, const samkv_rows_t* V, float scale, const samkv_rows_t* O,
                             float* lse, void* stream) {
  samkv_ctx_impl* h = reinterpret_cast<samkv_ctx_impl*>(handle);
  samkv_status_t st = check_packed(packed);
  if (st != SAMKV_OK || h == nullptr) return SAMKV_OK == st ? SAMKV_ERR_INVALID_ARG : st;
  if (packed->n_tokens == 0) return check_handle(h);
  Rows q, o;
  KvSource kv = {};
  if ((st = check_rows(*packed, Q, packed->n_q_heads, false, &q)) != SAMKV_OK) return st;
  if ((st = check_rows(*packed, K, packed->n_kv_heads, false, &kv.K)) != SAMKV_OK) return st;
  if ((st = check_rows(*packed, V, packed->n_kv_heads, false, &kv.V)) != SAMKV_OK) return st;
  if ((st = check_rows(*packed, O, packed->n_q_heads, true, &o)) != SAMKV_OK) return st;
  if (scale != scale || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return SAMKV_ERR_INVALID_ARG;
  const int Hq = packed->n_q_heads, Hkv = packed->n_kv_heads;
  if (rows_overlap(*packed, o, Hq, q, Hq) || rows_overlap(*packed, o, Hq, kv.K, Hkv) ||
      rows_overlap(*packed, o, Hq, kv.V, Hkv))
    return SAMKV_ERR_INVALID_ARG;
  if ((st = check_handle(h)) != SAMKV_OK) return st;
  if ((st = check_workspace(h, *packed)) != SAMKV_OK) return st;
  const Seqs seqs = {packed->seq_offsets, nullptr, packed->n_seq, packed->n_tokens, INT_MAX, 1};
  return from_cuda(launch_packed_attn(*packed, seqs, kv, q, scale, o, lse, *h, static_cast<cudaStream_t>(stream)));
}

samkv_status_t samkv_append(samkv_handle_t handle, const samkv_packed_t* packed, const samkv_rows_t* K,
                            const samkv_rows_t* V, const samkv_pages_t* pages, const int32_t* cache_len,
                            const samkv_rope_t* rope, const int32_t* positions, const samkv_rows_t* Q,
                            const samkv_rows_t* Q_out, const samkv_rows_t* K_out, const samkv_rows_t* V_out,
                            void* stream) {
  samkv_ctx_impl* h = reinterpret_cast<samkv_ctx_impl*>(handle);
  samkv_status_t st = check_packed(packed);
  if (st != SAMKV_OK || h == nullptr) return SAMKV_OK == st ? SAMKV_ERR_INVALID_ARG : st;
  if ((Q == nullptr) != (Q_out == nullptr) || (K_out == nullptr) != (V_out == nullptr)) return SAMKV_ERR_INVALID_ARG;
  if (pages == nullptr && K_out == nullptr) return SAMKV_ERR_INVALID_ARG;       // no destination
  if (((reinterpret_cast<uintptr_t>(cache_len) | reinterpret_cast<uintptr_t>(positions)) & 3u) != 0)
    return SAMKV_ERR_INVALID_ARG;
  RopeTable table;
  if ((st = make_rope(*packed, rope, &table)) != SAMKV_OK) return st;
  if (packed->n_tokens == 0) return check_handle(h);
  const int Hq = packed->n_q_heads, Hkv = packed->n_kv_heads;
  Rows k, v, q, qo, ko, vo;
  Pages pg = {};
  if ((st = check_rows(*packed, K, Hkv, false, &k)) != SAMKV_OK) return st;
  if ((st = check_rows(*packed, V, Hkv, false, &v)) != SAMKV_OK) return st;
  if (pages != nullptr && (st = check_pages(*packed, pages, &pg)) != SAMKV_OK) return st;
  if (Q != nullptr) {
    if ((st = check_rows(*packed, Q, Hq, false, &q)) != SAMKV_OK) return st;
    if ((st = check_rows(*packed, Q_out, Hq, true, &qo)) != SAMKV_OK) return st;
  }
  if (K_out != nullptr) {
    if ((st = check_rows(*packed, K_out, Hkv, true, &ko)) != SAMKV_OK) return st;
    if ((st = check_rows(*packed, V_out, Hkv, true, &vo)) != SAMKV_OK) return st;
  }
  // an output may be the very rows of its own input, and must not touch anything else
  struct Out { const Rows* r; int heads; const Rows* own; };
  const Out outs[3] = {{Q != nullptr ? &qo : nullptr, Hq, &q},
                       {K_out != nullptr ? &ko : nullptr, Hkv, &k},
                       {K_out != nullptr ? &vo : nullptr, Hkv, &v}};
  for (int i = 0; i < 3; ++i) {
    if (outs[i].r == nullptr) continue;
    const Rows& o = *outs[i].r;
    if (!same_rows(o, *outs[i].own) && rows_overlap(*packed, o, outs[i].heads, *outs[i].own, outs[i].heads))
      return SAMKV_ERR_INVALID_ARG;
    if (&k != outs[i].own && rows_overlap(*packed, o, outs[i].heads, k, Hkv)) return SAMKV_ERR_INVALID_ARG;
    if (&v != outs[i].own && rows_overlap(*packed, o, outs[i].heads, v, Hkv)) return SAMKV_ERR_INVALID_ARG;
    if (Q != nullptr && &q != outs[i].own && rows_overlap(*packed, o, outs[i].heads, q, Hq)) return SAMKV_ERR_INVALID_ARG;
    for (int j = i + 1; j < 3; ++j)
      if (outs[j].r != nullptr && rows_overlap(*packed, o, outs[i].heads, *outs[j].r, outs[j].heads))
        return SAMKV_ERR_INVALID_ARG;
  }
  if (pages != nullptr) {
    if (meets_pools(*packed, pg, nullptr, 0) || meets_pools(*packed, pg, &k, Hkv) || meets_pools(*packed, pg, &v, Hkv))
      return SAMKV_ERR_INVALID_ARG;
    if (Q != nullptr && (meets_pools(*packed, pg, &q, Hq) || meets_pools(*packed, pg, &qo, Hq))) return SAMKV_ERR_INVALID_ARG;
    if (K_out != nullptr && (meets_pools(*packed, pg, &ko, Hkv) || meets_pools(*packed, pg, &vo, Hkv)))
      return SAMKV_ERR_INVALID_ARG;
  }
  if ((st = check_handle(h)) != SAMKV_OK) return st;
  const Seqs seqs = {packed->seq_offsets, cache_len, packed->n_seq, packed->n_tokens, INT_MAX, 0};
  return from_cuda(launch_append(*packed, seqs, k, v, pages != nullptr ? &pg : nullptr, table, positions,
                                 Q != nullptr ? &q : nullptr, Q != nullptr ? &qo : nullptr,
                                 K_out != nullptr ? &ko : nullptr, K_out != nullptr ? &vo : nullptr, h->sm_count,
                                 h->d_status, static_cast<cudaStream_t>(stream)));
}

samkv_status_t samkv_paged_attn(samkv_handle_t handle, const samkv_packed_t* packed, const samkv_pages_t* pages,
                                const int32_t* cache_len, const samkv_rows_t* Q, float scale, int32_t causal,
                                const samkv_rows_t* O, float* lse, void* stream) {
  samkv_ctx_impl* h = reinterpret_cast<samkv_ctx_impl*>(handle);
  samkv_status_t st = check_packed(packed);
  if (st != SAMKV_OK || h == nullptr) return SAMKV_OK == st ? SAMKV_ERR_INVALID_ARG : st;
  if (packed->n_tokens == 0) return check_handle(h);
  if (cache_len == nullptr || ((reinterpret_cast<uintptr_t>(cache_len) | reinterpret_cast<uintptr_t>(lse)) & 3u) != 0)
    return SAMKV_ERR_INVALID_ARG;
  if (scale != scale) return SAMKV_ERR_INVALID_ARG;
  Rows q, o;
  KvSource kv = {};
  kv.paged = 1;
  if ((st = check_rows(*packed, Q, packed->n_q_heads, false, &q)) != SAMKV_OK) return st;
  if ((st = check_rows(*packed, O, packed->n_q_heads, true, &o)) != SAMKV_OK) return st;
  if ((st = check_pages(*packed, pages, &kv.pages)) != SAMKV_OK) return st;
  if (rows_overlap(*packed, o, packed->n_q_heads, q, packed->n_q_heads)) return SAMKV_ERR_INVALID_ARG;
  if (meets_pools(*packed, kv.pages, &o, packed->n_q_heads)) return SAMKV_ERR_INVALID_ARG;
  if ((st = check_handle(h)) != SAMKV_OK) return st;
  if ((st = check_workspace(h, *packed)) != SAMKV_OK) return st;
  const Seqs seqs = {packed->seq_offsets, cache_len, packed->n_seq, packed->n_tokens,
                     pages->table_width * pages->page_size, causal != 0};
  return from_cuda(launch_packed_attn(*packed, seqs, kv, q, scale, o, lse, *h, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
