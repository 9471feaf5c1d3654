// Attention with modified scores: which key tiles a row tile needs, how the work is divided, and the modifications themselves.
//
// With masks the tiles of a row tile have no closed form any more.  A plan is made first: a record per row tile of a sequence
// (all its heads share it) with the slots that its tokens see, and the lengths of all row tiles before it.  CTA c then takes
// the stretch [c, c + 1) * chunk of the axis as in packed_plan.cuh, finds its place by a search over those lengths, and one of
// its warps works its pieces out 32 at a time, a piece per lane; borders, workspace slots and tickets are those of packed_plan.cuh.
// (Walking from piece to piece as there, with the records in registers, made a call on 20 documents 4 % slower: the warp that
// does it also has the key tiles to load.)
// Who makes the plan goes by the sizes that the host knows.  Up to 32 row tiles: that warp, in its registers, a record per lane;
// such calls run in waves by the rules of packed_plan.cuh.  Up to 256: every CTA for itself, all of its threads, in a part of
// the workspace of its own, which takes 3 us less than a kernel in front (5 us and the step to the next kernel) although all CTAs
// do the same.  More: a kernel of one block in front of the attention kernel.
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
constexpr int kBlockTiles = 256, kBlockSeqs = 1024;      // most of a call whose CTAs make their plans themselves

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

// A plan in the workspace.
struct ScorePlan {
  long long* at;               // [n_tiles + 1] lengths before each row tile (of one head); null: a warp makes the plan
  int* n_tiles;
  RowTile* tiles;
  long long own_bytes;         // every CTA makes a plan of its own, so far apart; 0: there is one, made before
};
__device__ __forceinline__ ScorePlan own_plan(ScorePlan p) {
  const long long by = p.own_bytes * blockIdx.x;
  p.at = reinterpret_cast<long long*>(reinterpret_cast<char*>(p.at) + by);
  p.n_tiles = reinterpret_cast<int*>(reinterpret_cast<char*>(p.n_tiles) + by);
  p.tiles = reinterpret_cast<RowTile*>(reinterpret_cast<char*>(p.tiles) + by);
  return p;
}

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

// Record of row tile r of sequence s, up to its lows and its tiles.
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
  return t;
}
// The rest of the lanes' records (of those with `valid`); all lanes of the warp.  kTogether: eight lanes go through a row tile's
// tokens, four row tiles at a time.  A lane for itself fetches a line per token and is the quicker for few row tiles (66 of 16
// tokens 4.6 us for the plan kernel against 7.8, 966 of 32 tokens 22 us against 12).
template <bool kTogether>
__device__ __forceinline__ void finish_row_tiles(const Seqs& q, const ScoreMods& m, const SplitCfg& c, bool valid, RowTile& t) {
  constexpr unsigned kAll = 0xffffffffu;
  constexpr int kNone = 0x7fffffff;            // no token sees anything of its document
  int lowest = kNone, highest = 0;
  if (m.doc_start == nullptr) {
    // (lows rise with the position: the first token has the lowest one)
    if (valid) {
      lowest = low_of(m, 0, t.pos0);
      highest = low_of(m, 0, t.pos0 + t.n_tok - 1);
    }
  } else if constexpr (!kTogether) {
    if (valid)
#pragma unroll 8
      for (int i = 0; i < t.n_tok; ++i) {
        const int low = low_of(m, t.tok0 + i, t.pos0 + i);
        if (low < end_of(q, t.end0, i)) lowest = min(lowest, low);
        highest = max(highest, low);
      }
  } else {
    const int lane = threadIdx.x & 31, sub = lane >> 3;
    const unsigned some = __ballot_sync(kAll, valid);
#pragma unroll 4
    for (int l0 = 0; l0 < 32; l0 += 4) {
      if (some >> l0 == 0) break;
      const int n = __shfl_sync(kAll, valid ? t.n_tok : 0, l0 + sub), tok0 = __shfl_sync(kAll, t.tok0, l0 + sub);
      const int pos0 = __shfl_sync(kAll, t.pos0, l0 + sub), end0 = __shfl_sync(kAll, t.end0, l0 + sub);
      int low = kNone, high = 0;
#pragma unroll 4
      for (int i = lane & 7; i < n; i += 8) {
        const int x = low_of(m, tok0 + i, pos0 + i);
        if (x < end_of(q, end0, i)) low = min(low, x);
        high = max(high, x);
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        low = min(low, __shfl_xor_sync(kAll, low, o));
        high = max(high, __shfl_xor_sync(kAll, high, o));
      }
      const int from = (lane - l0 & 3) * 8;
      low = __shfl_sync(kAll, low, from);
      high = __shfl_sync(kAll, high, from);
      if (lane >> 2 == l0 >> 2) {
        lowest = low;
        highest = high;
      }
    }
  }
  if (valid) {
    const int any1 = end_of(q, t.end0, t.n_tok - 1);
    t.any0 = min(lowest, any1);
    t.all0 = highest;
    t.nt = tile_list(t.pre, t.any0, any1, c.tile).nt;
  }
}

template <int kThreads>
struct PlanScratch {
  int off[kThreads];           // row tiles of the chunk's sequences before each
  int warp[32];
  unsigned lo[32], hi[32];     // lengths, by halves
  int end;
};
// Records and lengths of all row tiles of a call, by kThreads threads of a block; report: this block records clamped values.
template <int kThreads>
__device__ __forceinline__ void make_plan(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan,
                                          PlanScratch<kThreads>& sh, bool report, int* d_status) {
  constexpr int kWarps = kThreads / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) sh.end = q.n_seq;
  __syncthreads();
  for (int s = tid; s < q.n_seq; s += kThreads) {
    const Seq x = load_seq(q, s);
    if (x.backwards) atomicMin(&sh.end, s);
    if (x.clamped && report) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  }
  __syncthreads();
  const int n_seq = sh.end;
  int n_tiles = 0;                             // so far
  long long total = 0;
#pragma unroll 1
  for (int s0 = 0; s0 < n_seq; s0 += kThreads) {
    // row tiles of these sequences
    int R = 0;
    if (s0 + tid < n_seq) R = row_tiles(c, load_seq(q, s0 + tid).n);
    int incl = R;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) sh.warp[warp] = incl;
    __syncthreads();
    int w = (lane < kWarps ? sh.warp[lane] : 0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += v;
    }
    const int chunk = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    sh.off[tid] = (warp > 0 ? before : 0) + incl - R;
    __syncthreads();
    const int count = min(kThreads, n_seq - s0);
    // their records, and the lengths
#pragma unroll 1
    for (int i0 = 0; i0 < chunk; i0 += kThreads) {
      const int i = i0 + tid;
      long long len = 0;
      RowTile t = {};
      if (i < chunk) {
        int lo = 0, hi = count - 1;            // last sequence that starts at or before i: the one that owns it
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (sh.off[mid] <= i) lo = mid; else hi = mid - 1;
        }
        t = make_row_tile(q, m, c, s0 + lo, load_seq(q, s0 + lo), i - sh.off[lo]);
      }
      if (chunk > 256 && c.tokens > 8) finish_row_tiles<true>(q, m, c, i < chunk, t);
      else finish_row_tiles<false>(q, m, c, i < chunk, t);
      if (i < chunk) {
        plan.tiles[n_tiles + i] = t;
        len = (long long)t.nt * c.tile + c.fixed;
      }
      long long li = len;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, li, o);
        if (lane >= o) li += v;
      }
      __syncthreads();
      if (lane == 31) {
        sh.lo[warp] = (unsigned)li;
        sh.hi[warp] = (unsigned)(li >> 32);
      }
      __syncthreads();
      long long wl = lane < kWarps ? (long long)((unsigned long long)sh.hi[lane] << 32 | sh.lo[lane]) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, wl, o);
        if (lane >= o) wl += v;
      }
      const long long all = __shfl_sync(0xffffffffu, wl, 31);
      const long long bw = __shfl_sync(0xffffffffu, wl, (warp + 31) & 31);
      if (i < chunk) plan.at[n_tiles + i] = total + (warp > 0 ? bw : 0) + li - len;
      total += all;
    }
    n_tiles += chunk;
  }
  if (tid == 0) {
    plan.at[n_tiles] = total;
    *plan.n_tiles = n_tiles;
  }
}
// In front of the roles of an attention kernel, by all of its threads: the plan of a call whose CTAs make their own.
template <int kThreads>
__device__ __forceinline__ ScorePlan plan_of_block(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan,
                                                   void* scratch, int* d_status) {
  if (plan.own_bytes == 0) return plan;
  const ScorePlan own = own_plan(plan);
  make_plan<kThreads>(q, m, c, own, *static_cast<PlanScratch<kThreads>*>(scratch), blockIdx.x == 0, d_status);
  __syncthreads();
  return own;
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
  unsigned char ticket, n_pieces, slot_step, unused;   // slot_step 0: slots as in piece_slot, else so far apart
  __device__ __forceinline__ int h() const { return (unsigned short)h_; }
  // tile that is taken i-th, of so many slots
  template <bool kDown>
  __device__ __forceinline__ int tile(int i, int slots) const {
    const int v = kDown ? tile1 - 1 - i : tile0 + i;
    return v * slots < pre ? v : v + gap;
  }
};
static_assert(sizeof(MaskedPiece) == 56, "descriptors");
__device__ __forceinline__ int piece_slot(const MaskedPiece& p, int k) {
  return p.slot_step > 0 ? p.slot0 + k * p.slot_step : p.slot0 + 2 * k - (k > 0 ? 1 : 0);
}
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

// Some token sees some slot of [j0, j1), by each token's own range: any_sees goes by the range from the lowest slot to the last
// end, within which slots may be nobody's where tokens see nothing of their own.  Such a page is asked for like the others (what
// it names is hidden from every row), but where its table entry is no page, that is nobody's concern: asked only then.
__device__ __forceinline__ bool token_sees(const Seqs& q, const ScoreMods& m, const MaskedPiece& p, int j0, int j1) {
  if (j0 < p.pre) return true;
#pragma unroll 1
  for (int i = 0; i < p.n_tok; ++i) {
    const RowView v = row_view(q, m, p, i);
    if (max(v.low, j0) < min(v.end, j1)) return true;
  }
  return false;
}

// The pieces of this CTA, 32 items (or units of a call in waves) at a time; run by one whole warp.
struct PieceWindow {
  MaskedPiece mine;                            // of item (unit) next - 32 + lane
  unsigned left;                               // lanes whose pieces are still to be taken
  int next;                                    // first item (unit of this CTA) behind the window
  int n_tiles;                                 // row tiles of the call
  int wave_tiles, wave_blocks;                 // a call in waves: tiles of a block, blocks; 0: contiguous stretches
  long long chunk, p0, p1;                     // this CTA's stretch of the axis
  bool more;                                   // there may be items behind the window

  // A call of at most 32 row tiles: lane i gets the record of row tile i, its length and those before it.
  __device__ __forceinline__ void plan_in_warp(const Seqs& q, const ScoreMods& m, const SplitCfg& c, RowTile& t, long long& before,
                                               long long& len, int* d_status) {
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
    if (lane < n_tiles) t = make_row_tile(q, m, c, s, sq, r);
    finish_row_tiles<false>(q, m, c, lane < n_tiles, t);
    len = lane < n_tiles ? (long long)t.nt * c.tile + c.fixed : 0;
    before = len;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += v;
    }
    before -= len;
  }
  // Whether such a call runs in waves: the rules of packed_plan.cuh, by the tiles that the masks leave.
  __device__ __forceinline__ void choose_waves(const SplitCfg& c, const RowTile& t, long long total) {
    const int lane = threadIdx.x & 31;
    wave_tiles = wave_blocks = 0;
    if (c.wave_slots == 0 || c.Hkv * n_tiles > kMaxTickets || total <= 2 * c.wave_slots) return;
    const int nt = lane < n_tiles ? t.nt : 0, most = __reduce_max_sync(0xffffffffu, nt);
    // (of a sequence's row tiles the last one sees most)
    const long long distinct = (long long)c.Hkv * c.tile * __reduce_add_sync(0xffffffffu, lane < n_tiles && t.r + 1 == t.R ? nt : 0);
    if (distinct <= c.wave_slots || total <= 2 * distinct) return;
    long long best = -1;
#pragma unroll 1
    for (int k = 1; k <= kWaveTries; ++k) {
      const int bt = (most + k - 1) / k;
      const int units = c.Hkv * __reduce_add_sync(0xffffffffu, (nt + bt - 1) / bt);
      if (c.Hkv * k * n_tiles > kMaxUnits || bt < 8) continue;
      const long long cost = (long long)((units + gridDim.x - 1) / gridDim.x) * (bt * c.tile + c.fixed);
      if (best < 0 || cost < best) {
        best = cost;
        wave_tiles = bt;
        wave_blocks = (most + bt - 1) / bt;
      }
    }
    // (an uneven mix of lengths leaves holes in the waves; the keys are fetched again instead)
    if (best > total / (long long)gridDim.x * 3 / 2) wave_tiles = 0;
  }
  // Tile border of an item nearest to position p of the axis; pieces shorter than two tiles are not worth their merge.
  static __device__ __forceinline__ int border(const SplitCfg& c, long long p, long long item_start, int nt) {
    const long long y = p - item_start - c.fixed;
    if (y <= 0) return 0;
    const long long t = (y + c.tile / 2) >> (31 - __clz(c.tile));
    if (t < 2) return 0;
    if (t > nt - 2) return nt;
    return (int)t;
  }
  // The lane's piece of row tile t and head h, tiles [tile0, tile1).
  __device__ __forceinline__ void describe(const Seqs& q, const SplitCfg& c, const RowTile& t, int h, bool paged, int tile0, int tile1) {
    mine.kv = paged ? t.s : t.first;
    mine.tok0 = t.tok0;
    mine.pos0 = t.pos0;
    mine.end0 = t.end0;
    mine.pre = t.pre;
    mine.any0 = t.any0;
    mine.all0 = t.all0;
    const int any1 = end_of(q, t.end0, t.n_tok - 1);
    mine.gap = tile_list(t.pre, t.any0, any1, c.tile).gap;
    mine.seen = max(t.pre, t.any0 < any1 ? any1 : 0);
    mine.tile0 = tile0;
    mine.tile1 = tile1;
    mine.h_ = (short)h;
    mine.n_tok = (short)t.n_tok;
    mine.slot = -1;
    mine.slot0 = 0;
    mine.ticket = mine.slot_step = mine.unused = 0;
    mine.n_pieces = 1;
  }
  // tile_at(k): record of row tile k (each lane its own k); before(k): lengths before it, k = n_tiles: all.
  template <typename TileAt, typename Before>
  __device__ __forceinline__ void fill(const Seqs& q, const SplitCfg& c, bool paged, TileAt tile_at, Before before) {
    const int lane = threadIdx.x & 31, g = next + lane;
    next += 32;
    bool emit;
    if (wave_tiles > 0) {
      // unit ((h * blocks) + b) * n_tiles + i is block b of row tile i and head h
      const int u = g * (int)gridDim.x + (int)blockIdx.x, units = c.Hkv * wave_blocks * n_tiles;
      const int x = min(u, units - 1), rest = x / n_tiles, i = x - rest * n_tiles, h = rest / wave_blocks, b = rest - h * wave_blocks;
      const RowTile t = tile_at(i);
      emit = u < units && b * wave_tiles < t.nt;
      describe(q, c, t, h, paged, b * wave_tiles, min((b + 1) * wave_tiles, t.nt));
      mine.n_pieces = (unsigned char)((t.nt + wave_tiles - 1) / wave_tiles);
      mine.ticket = (unsigned char)(h * n_tiles + i);
      mine.slot0 = (short)(u - b * n_tiles);
      mine.slot_step = (unsigned char)n_tiles;
      if (mine.n_pieces > 1) mine.slot = (short)u;
      more = __all_sync(0xffffffffu, u < units);
    } else {
      // items run sequence by sequence, head by head, row tile by row tile: item g is among those of row tile g / Hkv's sequence
      const int last = c.Hkv * n_tiles - 1, x = min(g, last);
      const RowTile some = tile_at(x / c.Hkv);
      const int r0 = x / c.Hkv - some.r, rest = x - c.Hkv * r0, h = rest / some.R, k = r0 + rest - h * some.R;
      const RowTile t = tile_at(k);
      const long long at0 = before(r0);
      const long long start = c.Hkv * at0 + h * (before(r0 + some.R) - at0) + (before(k) - at0);
      const long long end = start + (long long)t.nt * c.tile + c.fixed;
      const bool in = g <= last && start < p1;
      const int t0 = border(c, p0, start, t.nt), t1 = p1 >= end ? t.nt : border(c, p1, start, t.nt);
      emit = in && t0 < t1;
      describe(q, c, t, h, paged, t0, t1);
      if (emit && (t0 > 0 || t1 < t.nt)) {
        // borders inside the item, after they have been moved to tile borders
        long long ca = quotient(start, chunk) + 1, cb = quotient(end - 1, chunk);
#pragma unroll 1
        while (ca <= cb && border(c, ca * chunk, start, t.nt) == 0) ++ca;
#pragma unroll 1
        while (cb >= ca && border(c, cb * chunk, start, t.nt) >= t.nt) --cb;
        mine.slot = (short)(2 * (int)blockIdx.x + (t0 > 0 ? 0 : 1));
        mine.ticket = (unsigned char)ca;
        mine.n_pieces = (unsigned char)((int)(cb - ca) + 2);
        mine.slot0 = (short)(2 * ((int)ca - 1) + 1);
      }
      more = __all_sync(0xffffffffu, in);
    }
    left = __ballot_sync(0xffffffffu, emit);
  }
  // The next window; the first one if `begin`.
  __device__ __forceinline__ void refill(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan, bool paged, bool begin,
                                         int* d_status) {
    const int lane = threadIdx.x & 31;
    if (plan.at == nullptr) {
      RowTile t = {};
      long long at, len;
      plan_in_warp(q, m, c, t, at, len, d_status);         // (again for every window: few calls have a second one)
      const long long total = __shfl_sync(0xffffffffu, at + len, 31);
      auto tile_at = [&](int k) {
        RowTile x;
        const int* from = reinterpret_cast<const int*>(&t);
        int* to = reinterpret_cast<int*>(&x);
#pragma unroll
        for (int i = 0; i < kRowTileInts; ++i) to[i] = __shfl_sync(0xffffffffu, from[i], k);
        return x;
      };
      if (begin) {
        choose_waves(c, t, c.Hkv * total);
        next = 0;
        more = n_tiles > 0;
        left = 0;
        if (wave_tiles == 0 && more) {
          place(c, c.Hkv * total);
          if (more) {
            // the last row tile that starts at or before p0, were there one head; then that of p0's head
            const int some = 31 - __clz(__ballot_sync(0xffffffffu, lane < n_tiles && c.Hkv * at <= p0));
            const int r0 = some - __shfl_sync(0xffffffffu, t.r, some), R = __shfl_sync(0xffffffffu, t.R, some);
            const long long start = __shfl_sync(0xffffffffu, at, r0), per_head = __shfl_sync(0xffffffffu, at + len, r0 + R - 1) - start;
            const int h = (int)quotient(p0 - c.Hkv * start, per_head);
            const long long rest = p0 - c.Hkv * start - h * per_head;
            const int k = 31 - __clz(__ballot_sync(0xffffffffu, lane >= r0 && lane < r0 + R && at - start <= rest));
            next = c.Hkv * r0 + h * R + (k - r0);
          }
        }
        if (!more) return;
      }
      // (a shuffle is for all lanes: the sum of all lengths stands behind the last row tile)
      auto before_any = [&](int k) {
        const long long v = __shfl_sync(0xffffffffu, at, min(k, 31));
        return k < n_tiles ? v : total;
      };
      fill(q, c, paged, tile_at, before_any);
    } else {
      if (begin) {
        n_tiles = *plan.n_tiles;
        wave_tiles = wave_blocks = 0;
        left = 0;
        more = n_tiles > 0;
        if (more) place(c, c.Hkv * plan.at[n_tiles]);
        if (!more) return;
        // last row tile of [lo, lo + n) that starts at or before x (of one head): 32 candidates at a time
        auto search = [&](int lo, int n, long long scale, long long x) {
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
        const int some = search(0, n_tiles, c.Hkv, p0);
        const int r0 = some - plan.tiles[some].r, R = plan.tiles[some].R;
        const long long start = plan.at[r0], per_head = plan.at[r0 + R] - start;
        const int h = (int)quotient(p0 - c.Hkv * start, per_head);
        next = c.Hkv * r0 + h * R + (search(r0, R, 1, p0 - (c.Hkv - 1) * start - h * per_head) - r0);
      }
      auto tile_at = [&](int k) {
        RowTile t;
        const int4* src = reinterpret_cast<const int4*>(plan.tiles + k);
        static_assert(sizeof(RowTile) == 48, "three vectors");
        int4* dst = reinterpret_cast<int4*>(&t);
#pragma unroll
        for (int i = 0; i < 3; ++i) dst[i] = src[i];
        return t;
      };
      fill(q, c, paged, tile_at, [&](int k) { return plan.at[k]; });
    }
  }
  // This CTA's stretch.
  __device__ __forceinline__ void place(const SplitCfg& c, long long total) {
    chunk = stretch(c, total, c.Hkv * n_tiles);
    p0 = chunk * blockIdx.x;
    p1 = min(p0 + chunk, total);
    more = p0 < total;
  }
  __device__ __forceinline__ void begin(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan, bool paged,
                                        int* d_status) {
    refill(q, m, c, plan, paged, true, d_status);
  }
  // The lane that holds the next piece, -1: there is none.
  __device__ __forceinline__ int take(const Seqs& q, const ScoreMods& m, const SplitCfg& c, const ScorePlan& plan, bool paged,
                                      int* d_status) {
#pragma unroll 1
    while (left == 0) {
      if (!more) return -1;
      refill(q, m, c, plan, paged, false, d_status);
    }
    const int k = __ffs(left) - 1;
    left &= left - 1;
    return k;
  }
};

// ----- host side -----
// Most row tiles of a call, by what the host knows.
inline long long most_row_tiles(const samkv_packed_t& p, int tokens) {
  const long long a = p.n_tokens, b = ((long long)p.n_tokens + (long long)p.n_seq * (tokens - 1)) / tokens;
  return a < b ? a : b;
}
inline size_t plan_bytes(long long tiles) { return ((size_t)tiles * (sizeof(RowTile) + 8) + 16 + 255) & ~(size_t)255; }
// Where the plan of a call lies, and who makes it; enqueues the plan's kernel where there is one.
cudaError_t make_score_plan(const samkv_packed_t& p, const Seqs& seqs, const ScoreMods& mods, const SplitCfg& cfg,
                            const samkv_ctx_impl& h, ScorePlan* plan, cudaStream_t stream);

}  // namespace samkv
