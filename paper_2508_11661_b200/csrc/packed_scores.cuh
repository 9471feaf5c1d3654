// Attention with modified scores: which key tiles a row tile needs, how the work is divided, and the modifications themselves.
//
// With masks the tiles of a row tile have no closed form any more.  A plan is made first: a record per row tile of a sequence
// (all its heads share it) with the slots that its tokens see, and the lengths of all row tiles before it.  CTA c then takes
// the stretch [c, c + 1) * chunk of the axis as in packed_plan.cuh, finds its place by a search over those lengths, and walks
// the records; pieces, borders, workspace slots and tickets are those of packed_plan.cuh.
// The plan is a kernel of one block in front of the attention kernel.  Where a call has at most 32 row tiles by the sizes
// the host knows, the warp that walks the plan makes it in its registers, a record per lane, and there is no such kernel.
//
// Token i of a row tile sees the slots below the sequence's prefix and those of [low_i, end_i): low_i is the largest of 0,
// its document's start and the window's edge, end_i rises with i.  A row tile's key tiles are those of the prefix and those
// of [any0, any1), any0 the lowest low_i and any1 the last end_i: a list with at most one gap, counted from 0 ("virtual").
// With slopes a piece's tiles are taken from the last to the first: the scores rise towards the diagonal, so that the running
// maximum is found at once.  Without, from the first to the last, since the last one often shows a row few of its slots.
#pragma once

#include "packed_plan.cuh"

namespace samkv {

constexpr int kPlanThreads = 1024;
constexpr int kWarpTiles = 32;                 // row tiles that one warp plans by itself

struct alignas(16) RowTile {
  int s, r, R;                 // sequence, row tile of it, its row tiles
  int first;                   // first packed row of the sequence
  int tok0, n_tok;             // first packed row and tokens of the row tile
  int pos0, end0;              // position of the first token, slots behind which it sees nothing
  int pre;                     // slots of the prefix
  int any0, all0;              // lowest and highest low_i
  int nt;                      // key tiles, 1 at least
};
constexpr int kRowTileInts = sizeof(RowTile) / 4;

// What the plan kernel leaves in the workspace.
struct ScorePlan {
  long long* at;               // [n_tiles + 1] lengths before each row tile (of one head)
  int* n_tiles;
  RowTile* tiles;
};

__device__ __forceinline__ int end_of(const Seqs& q, int end0, int i) {
  return q.causal ? (int)min((unsigned)end0 + (unsigned)i, (unsigned)q.limit) : end0;
}

// The list of key tiles: actual tile of virtual tile v is v for v < np, v + gap behind.
struct TileList {
  int np, gap, nt;
};
__device__ __forceinline__ TileList tile_list(int pre, int any0, int any1, int tile) {
  const int shift = 31 - __clz(tile);
  const int np = (pre + tile - 1) >> shift;
  TileList t = {np, 0, np};
  if (any0 < any1) {
    const int m0 = any0 >> shift, m1 = (any1 + tile - 1) >> shift;
    t.gap = max(m0 - np, 0);
    t.nt = max(np, m1 - t.gap);
  }
  t.nt = max(t.nt, 1);
  return t;
}

__device__ __forceinline__ int low_of(const ScoreMods& m, int tok, int pos) {
  int low = m.doc_start != nullptr ? max(m.doc_start[tok], 0) : 0;
  if (m.window < 0x7fffffff) low = max(low, pos - m.window + 1);
  return low;
}

// Record of row tile r of sequence s.
__device__ __forceinline__ RowTile make_row_tile(const Seqs& q, const ScoreMods& m, const SplitCfg& c, int s, const Seq& sq, int r) {
  RowTile t;
  t.s = s;
  t.r = r;
  t.R = row_tiles(c, sq.n);
  t.first = sq.first;
  const int t0 = r * c.tokens;
  t.tok0 = sq.first + t0;
  t.n_tok = min(c.tokens, sq.n - t0);
  t.pos0 = sq.base + t0;
  t.end0 = visible(q, sq, t0);
  t.pre = m.prefix_len != nullptr ? min(max(m.prefix_len[s], 0), visible(q, sq, sq.n - 1)) : 0;
  const int any1 = end_of(q, t.end0, t.n_tok - 1);
  t.any0 = any1;
  t.all0 = 0;
  if (m.doc_start == nullptr) {
    // (lows rise with the position: the first token has the lowest one)
    const int low = low_of(m, 0, t.pos0);
    t.any0 = min(low, any1);
    t.all0 = low_of(m, 0, t.pos0 + t.n_tok - 1);
  } else {
#pragma unroll 4
    for (int i = 0; i < t.n_tok; ++i) {
      const int low = low_of(m, t.tok0 + i, t.pos0 + i);
      if (low < end_of(q, t.end0, i)) t.any0 = min(t.any0, low);
      t.all0 = max(t.all0, low);
    }
  }
  t.nt = tile_list(t.pre, t.any0, any1, c.tile).nt;
  return t;
}

// A piece of a masked item, as the kernels hand it around (14 words: shared memory is full).
struct MaskedPiece {
  int kv;                      // packed keys: first row of the sequence; pages: the sequence
  int tok0, pos0, end0;        // as in RowTile
  int pre, any0, all0;
  int gap;                     // TileList
  int tile0, tile1;            // virtual tiles; tile0 < 0: no more pieces
  int seen;                    // slots behind which no token sees anything
  short h_, n_tok;
  short slot, slot0;           // workspace slot of the partial result (-1: the piece is the whole item), and of the first one
  short ticket, n_pieces;
  __device__ __forceinline__ int h() const { return (unsigned short)h_; }
  // tile that is taken i-th, of so many slots
  template <bool kDown>
  __device__ __forceinline__ int tile(int i, int slots) const {
    const int v = kDown ? tile1 - 1 - i : tile0 + i;
    return v * slots < pre ? v : v + gap;
  }
};
static_assert(sizeof(MaskedPiece) == 56, "descriptors");
__device__ __forceinline__ int piece_slot(const MaskedPiece& p, int k) { return p.slot0 + 2 * k - (k > 0 ? 1 : 0); }
__device__ __forceinline__ int any1_of(const Seqs& q, const MaskedPiece& p) { return end_of(q, p.end0, p.n_tok - 1); }
// Some token sees some slot of [j0, j1).
__device__ __forceinline__ bool any_sees(const MaskedPiece& p, int any1, int j0, int j1) {
  return j0 < p.pre || (j0 < any1 && j1 > p.any0);
}
// Of the slots [*j0, *j1) the stretch that holds those that not every token sees: empty (*j0 >= *j1) if all do.
__device__ __forceinline__ void hidden_from_some(const MaskedPiece& p, int* j0, int* j1) {
  if (*j0 < p.pre) *j0 = p.pre;
  if (p.all0 <= *j0 && *j0 < p.end0) *j0 = p.end0;
  if (p.all0 < *j1 && *j1 <= p.end0) *j1 = p.all0;
}

// What one row (a token of a head) sees.
struct RowView {
  int pre, low, end, pos;
  __device__ __forceinline__ bool sees(int j) const { return j < pre || (j >= low && j < end); }
  __device__ __forceinline__ bool sees_all(int j0, int j1) const { return j1 <= pre || (low <= j0 && j1 <= end); }
  // bit i: sees slot j + i
  __device__ __forceinline__ unsigned bits(int j) const { return below(pre - j) | (below(end - j) & ~below(low - j)); }
  static __device__ __forceinline__ unsigned below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
};
// Token i of the piece's row tile (one behind the last: as the last).
__device__ __forceinline__ RowView row_view(const Seqs& q, const ScoreMods& m, const MaskedPiece& p, int i) {
  i = min(i, p.n_tok - 1);
  RowView v;
  v.pre = p.pre;
  v.pos = p.pos0 + i;
  v.end = end_of(q, p.end0, i);
  v.low = low_of(m, p.tok0 + i, v.pos);
  return v;
}

// Walks the pieces of this CTA; run by one whole warp.
struct TileWalker {
  long long chunk, p1, item_start, total_len;
  int n_tiles, w0, h, i;                       // row tiles of the call, first one in the lanes, head, current row tile
  RowTile mine, cur;                           // lane k: row tile w0 + k
  int first_piece_tile;
  bool more;

  __device__ __forceinline__ RowTile from_lane(int k) const {
    RowTile t;
    const int* a = reinterpret_cast<const int*>(&mine);
    int* b = reinterpret_cast<int*>(&t);
#pragma unroll
    for (int x = 0; x < kRowTileInts; ++x) b[x] = __shfl_sync(0xffffffffu, a[x], k);
    return t;
  }
  __device__ __forceinline__ void fetch(const ScorePlan& plan, int at) {
    if (at < w0 || at >= w0 + 32) {
      w0 = at;
      const int k = min(at + (int)(threadIdx.x & 31), n_tiles - 1);
      const int4* src = reinterpret_cast<const int4*>(plan.tiles + k);
      static_assert(sizeof(RowTile) == 48, "three vectors");
      int4* dst = reinterpret_cast<int4*>(&mine);
#pragma unroll
      for (int x = 0; x < 3; ++x) dst[x] = src[x];
    }
    cur = from_lane(at - w0);
    i = at;
  }
  __device__ __forceinline__ int border(const SplitCfg& c, long long p, int nt) const {
    const long long y = p - item_start - c.fixed;
    if (y <= 0) return 0;
    const long long t = (y + c.tile / 2) >> (31 - __clz(c.tile));
    if (t < 2) return 0;
    if (t > nt - 2) return nt;
    return (int)t;
  }
  // Lays a call of at most 32 row tiles out; the lanes keep the records.
  __device__ __forceinline__ long long plan_in_warp(const Seqs& q, const ScoreMods& m, const SplitCfg& c, int* d_status) {
    const int lane = threadIdx.x & 31;
    Seq x = {0, 0, 0, false, false};
    if (lane < q.n_seq) x = load_seq(q, lane);
    const unsigned back = __ballot_sync(0xffffffffu, x.backwards);
    if (x.clamped && blockIdx.x == 0) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
    if (back != 0 && lane >= __ffs(back) - 1) x.n = 0;
    const int R = row_tiles(c, x.n);
    int incl = R;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    n_tiles = __shfl_sync(0xffffffffu, incl, 31);
    // the sequence of row tile `lane`: as many as end at or before it
    int s = 0;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += __shfl_sync(0xffffffffu, incl, k) <= lane;
    const int from = min(s, 31);
    Seq sq;
    sq.first = __shfl_sync(0xffffffffu, x.first, from);
    sq.n = __shfl_sync(0xffffffffu, x.n, from);
    sq.base = __shfl_sync(0xffffffffu, x.base, from);
    const int r = lane - __shfl_sync(0xffffffffu, incl - R, from);
    long long len = 0;
    w0 = 0;
    if (lane < n_tiles) {
      mine = make_row_tile(q, m, c, s, sq, r);
      len = (long long)mine.nt * c.tile + c.fixed;
    }
    return len;
  }
  __device__ __forceinline__ void begin(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan, int* d_status) {
    const int lane = threadIdx.x & 31;
    long long in_lane = 0, before = 0;         // lengths of the row tiles in the lanes, of those before them
    const bool small = plan.at == nullptr;
    if (small) {
      long long incl = plan_in_warp(q, m, c, d_status);
      in_lane = incl;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      before = incl - in_lane;
      total_len = c.Hkv * __shfl_sync(0xffffffffu, incl, 31);
    } else {
      n_tiles = *plan.n_tiles;
      total_len = c.Hkv * plan.at[n_tiles];
      w0 = -64;
    }
    chunk = stretch(c, total_len, c.Hkv * n_tiles);
    const long long p0 = chunk * blockIdx.x;
    more = p0 < total_len;
    if (!more) return;
    p1 = min(p0 + chunk, total_len);
    auto at = [&](int k) { return small ? __shfl_sync(0xffffffffu, before, k) : plan.at[k]; };
    // last row tile of [lo, lo + n) that starts at or before x (of one head): 32 candidates at a time
    auto search = [&](int lo, int n, long long scale, long long x) {
      if (small) {
        const unsigned fits = __ballot_sync(0xffffffffu, lane >= lo && lane < lo + n && scale * before <= x);
        return 31 - __clz(fits);
      }
#pragma unroll 1
      while (n > 1) {
        const int step = (n + 31) >> 5, k = lane * step;
        const unsigned fits = __ballot_sync(0xffffffffu, k < n && scale * plan.at[lo + min(k, n - 1)] <= x);
        const int skip = (__popc(fits) - 1) * step;
        lo += skip;
        n = min(step, n - skip);
      }
      return lo;
    };
    fetch(plan, search(0, n_tiles, c.Hkv, p0));          // some row tile of the sequence that holds p0
    const int r0 = i - cur.r, R = cur.R;
    const long long start = at(r0);
    const long long end = !small ? plan.at[r0 + R]
                                 : __shfl_sync(0xffffffffu, before, r0 + R - 1) + __shfl_sync(0xffffffffu, in_lane, r0 + R - 1);
    const long long per_head = end - start;
    long long rem = p0 - c.Hkv * start;
    h = (int)quotient(rem, per_head);
    rem -= h * per_head;
    const int k = search(r0, R, 1, start + rem);
    item_start = c.Hkv * start + h * per_head + (at(k) - start);
    fetch(plan, k);
    first_piece_tile = border(c, p0, cur.nt);
  }
  __device__ __forceinline__ bool next(const Seqs& q, const SplitCfg& c, const ScorePlan& plan, bool paged, MaskedPiece* out) {
#pragma unroll 1
    while (more) {
      const int nt = cur.nt;
      const long long end = item_start + (long long)nt * c.tile + c.fixed;
      const int t0 = first_piece_tile >= 0 ? first_piece_tile : 0;
      const bool starts_inside = first_piece_tile > 0;
      first_piece_tile = -1;
      const int t1 = p1 >= end ? nt : border(c, p1, nt);
      const bool ends_inside = t1 < nt;
      const bool emit = t0 < t1;
      if (emit) {
        out->kv = paged ? cur.s : cur.first;
        out->tok0 = cur.tok0;
        out->pos0 = cur.pos0;
        out->end0 = cur.end0;
        out->pre = cur.pre;
        out->any0 = cur.any0;
        out->all0 = cur.all0;
        const int any1 = end_of(q, cur.end0, cur.n_tok - 1);
        const TileList l = tile_list(cur.pre, cur.any0, any1, c.tile);
        out->gap = l.gap;
        out->seen = max(cur.pre, cur.any0 < any1 ? any1 : 0);
        out->tile0 = t0;
        out->tile1 = t1;
        out->h_ = (short)h;
        out->n_tok = (short)cur.n_tok;
        out->slot = -1;
        out->slot0 = 0;
        out->ticket = 0;
        out->n_pieces = 1;
        if (starts_inside || ends_inside) {
          // borders inside the item, after they have been moved to tile borders
          long long ca = quotient(item_start, chunk) + 1, cb = quotient(end - 1, chunk);
#pragma unroll 1
          while (ca <= cb && border(c, ca * chunk, nt) == 0) ++ca;
#pragma unroll 1
          while (cb >= ca && border(c, cb * chunk, nt) >= nt) --cb;
          out->slot = (short)(2 * (int)blockIdx.x + (starts_inside ? 0 : 1));
          out->ticket = (short)ca;
          out->n_pieces = (short)((int)(cb - ca) + 2);
          out->slot0 = (short)(2 * ((int)ca - 1) + 1);
        }
      }
      if (p1 <= end) {
        more = false;
      } else {
        item_start = end;
        int next_tile = i + 1;
        if (cur.r + 1 == cur.R) {
          if (++h == c.Hkv) h = 0;
          else next_tile = i + 1 - cur.R;
        }
        if (next_tile < n_tiles) fetch(plan, next_tile);
        else more = false;
      }
      if (emit) return true;
    }
    return false;
  }
};

// ----- host side -----
// Most row tiles of a call, by what the host knows.
inline long long most_row_tiles(const samkv_packed_t& p, int tokens) {
  const long long a = p.n_tokens, b = ((long long)p.n_tokens + (long long)p.n_seq * (tokens - 1)) / tokens;
  return a < b ? a : b;
}
inline size_t score_plan_bytes(long long tiles) { return 256 + (size_t)tiles * (sizeof(RowTile) + 8) + 16; }
// Lays a call out: its plan's place in the workspace (null where the warps make it themselves); enqueues the plan's kernel.
cudaError_t make_score_plan(const samkv_packed_t& p, const Seqs& seqs, const ScoreMods& mods, const SplitCfg& cfg,
                            const samkv_ctx_impl& h, ScorePlan* plan, cudaStream_t stream);

}  // namespace samkv
