// How the attention kernels over packed sequences divide their work among persistent CTAs.
//
// An item is a row tile (up to `rows` packed query rows: tokens x group members) of one sequence and KV head; its keys
// come in tiles of `tile` slots.  All items of a call are laid out on one axis, sequence by sequence, head by head, row
// tile by row tile, each as long as the slots its last token sees plus a fixed share for prologue and epilogue.  CTA c
// takes the stretch [c, c + 1) * chunk of that axis; a border inside an item is moved to the nearest tile border.  The
// CTAs' shares are alike whatever the mix of lengths, an item is cut into more than one piece only where a border falls,
// and the host needs to know none of the lengths.  Lengths along the axis are linear in the row tile's index, so positions
// are found by closed forms and a binary search.
// How alike: a border moves by up to the fixed share and two tiles, the last row tile of a sequence is charged for tokens
// that it does not have, and tiles are not charged whole.  Key tiles per CTA of 20 x 1536 tokens, 32/8 heads: 327 to 342,
// 337 on average; of 10 ragged prompts of 1 to 5000 tokens 124 to 237, 219 on average (with each piece's fixed share as two
// tiles 246 to 278, 253 on average).
//
// A cut item's pieces leave (m, l, O) in the workspace, at most two pieces per CTA: the one a CTA starts with (slot 2c)
// and the one it ends with (slot 2c + 1).  The CTA that finishes an item's last piece merges them in order of the axis,
// so results do not depend on timing.  Tickets are bytes of the workspace's status block, one per first border of an
// item, and return to zero.
//
// That order walks each row tile of a sequence through all of its keys before the next one.  Where several row tiles
// share keys that the L2 cache cannot hold, every one of them would fetch them from HBM again; such calls are laid out in
// waves instead: keys are cut into blocks of one length, a unit is a row tile times a block, units run block by block
// with the row tiles next to one another, and CTA c takes units c, c + grid, ...: the row tiles of a block run at the same
// time and share its keys through L2 (128 tokens over 102400, 8 row tiles per KV head: see packed_tc.cu).  Calls of more
// than 240 items (kMaxTickets; 8 KV heads with 8 query heads each: 480 tokens) keep the contiguous layout.
//
// A sequence that ends before it starts also ends the list of sequences: those behind it could own the same rows again,
// which two CTAs would write at the same time and which no bound on the call's work would cover.
#pragma once

#include "packed.cuh"

namespace samkv {

constexpr int kMaxPackedCtas = 160;
constexpr int kMaxTickets = 240;               // bytes of status words 1..31 and 33..61 (0 and 32 have other uses)
constexpr int kMaxUnits = 896;                 // workspace slots of a call in waves

struct SplitCfg {
  int G, Hkv;
  int tokens;                  // tokens per row tile (rows / G)
  int tile;                    // slots per key tile
  int fixed;                   // slots that an item's fixed cost amounts to (>= 2 * tile)
  int min_chunk;               // least slots (fixed cost included) worth a CTA of its own (>= 2 * tile)
  long long wave_slots;        // lay out in waves where the distinct key slots of a call exceed this; 0: never
};

struct Piece {
  int s, h, r;                 // sequence, KV head, row tile
  int first, n, base;          // of the sequence, as in Seq
  int seen0, seen;             // slots that the row tile's first and last token see
  int tile0, tile1;            // key tiles of this piece
  int slot;                    // workspace slot of the partial result, -1: the piece is the whole item
  int slot0, slot_step;        // slots of the item's pieces, see piece_slot()
  int ticket;
  int n_pieces;
};
// Workspace slot of an item's piece k.  In waves the pieces are slot_step apart; else (slot_step 0) the first is the last
// piece of the CTA before the first border, the others are the first ones of the CTAs that start at the borders.
__device__ __forceinline__ int piece_slot(const Piece& p, int k) {
  return p.slot_step > 0 ? p.slot0 + k * p.slot_step : p.slot0 + 2 * k - (k > 0 ? 1 : 0);
}

__device__ __forceinline__ int row_tiles(const SplitCfg& c, int n) { return (n + c.tokens - 1) / c.tokens; }
// length of the first x items of one (sequence, head)
__device__ __forceinline__ long long items_length(const SplitCfg& c, int causal, int base, int x) {
  long long len = (long long)x * (base + c.fixed);
  if (causal) len += (long long)c.tokens * x * (x + 1) / 2;
  return len;
}

constexpr int kWaveTries = 12;
struct PlanShared {
  long long warp_len[32];
  int warp_items[32];
  int warp_end[32];
  int n_seq;                   // sequences before one that ends before it starts
  long long start;             // position of the sequence found
  int s;
  long long total;             // length of the axis
  int items;
  unsigned long long distinct; // key slots of the call, each counted once
  int longest;                 // most tiles of an item
  int wave_tiles;              // tiles per block of a call in waves, 0: contiguous stretches
  unsigned units[kWaveTries];  // units for each length tried
};

// Sequences that the warp which walks the plan can also lay out by itself, next to whatever the other warps do; more of
// them take the whole block.
constexpr int kWarpPlanSeqs = 512;

// Most quotients here fit 32 bits, whose division is a fifth of the 64-bit one.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  return ((unsigned long long)(a | b) >> 32) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// Length of a CTA's stretch of the axis.
__device__ __forceinline__ long long stretch(const SplitCfg& c, long long total, int items) {
  long long ctas = quotient(total, c.min_chunk);
  if (ctas < items) ctas = items;
  if (ctas > (long long)gridDim.x) ctas = gridDim.x;
  if (ctas < 1) ctas = 1;
  return quotient(total + ctas - 1, ctas);
}
// Calls of this size may be laid out in waves.
__device__ __forceinline__ bool maybe_waves(const SplitCfg& c, long long total, int items) {
  return c.wave_slots > 0 && total > 2 * c.wave_slots && items <= kMaxTickets;
}

// Finds the sequence that holds this CTA's first position.  Called by kThreads threads, a whole block or (32) one warp,
// with their index among them; afterwards *chunk is the length of a CTA's stretch (0: nothing to do) and sh->s,
// sh->start are set for CTAs that have one.  No thread looks at *sh behind the last barrier in here, so that the warp which
// walks the plan may give the memory away once it has begun.
template <int kThreads>
__device__ __forceinline__ void plan_block(const Seqs& q, const SplitCfg& c, PlanShared* sh, long long* chunk, int* d_status,
                                           int tid) {
  const int warp = tid >> 5, lane = tid & 31;
  constexpr int kWarps = kThreads / 32;
  auto sync = []() {
    if constexpr (kThreads == 32) __syncwarp(); else __syncthreads();
  };
  const int per = (q.n_seq + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, q.n_seq);
  int s1 = min(s0 + per, q.n_seq);
  if (tid == 0) {
    sh->distinct = 0;
    sh->longest = 0;
    sh->wave_tiles = 0;
  }
  if (tid < kWaveTries) sh->units[tid] = 0;
  long long len = 0;
  int items = 0;
  bool clamped = false;
  int n_seq = q.n_seq;
#pragma unroll 1
  for (int s = s0; s < s1; ++s) {
    const Seq sq = load_seq(q, s);
    const int R = row_tiles(c, sq.n);
    clamped |= sq.clamped;
    if (sq.backwards) {
      n_seq = s;
      break;
    }
    len += c.Hkv * items_length(c, q.causal, sq.base, R);
    items += c.Hkv * R;
  }
  if (clamped && blockIdx.x == 0) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
  n_seq = __reduce_min_sync(0xffffffffu, n_seq);
  if constexpr (kThreads > 32) {
    if (lane == 0) sh->warp_end[warp] = n_seq;
    sync();
    n_seq = __reduce_min_sync(0xffffffffu, sh->warp_end[lane < kWarps ? lane : 0]);
  }
  if (tid == 0) sh->n_seq = n_seq;
  s1 = min(s1, n_seq);
  if (s0 >= n_seq) {
    len = 0;
    items = 0;
  }
  long long incl = len;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) items += __shfl_xor_sync(0xffffffffu, items, o);
  if (lane == 31) sh->warp_len[warp] = incl;
  if (lane == 0) sh->warp_items[warp] = items;
  sync();
  if (warp == 0) {
    const long long w = lane < kWarps ? sh->warp_len[lane] : 0;
    int it = lane < kWarps ? sh->warp_items[lane] : 0;
    long long wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, wi, o);
      if (lane >= o) wi += v;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) it += __shfl_xor_sync(0xffffffffu, it, o);
    if (lane < kWarps) sh->warp_len[lane] = wi - w;          // exclusive prefix
    if (lane == 31) sh->total = wi;
    if (lane == 0) sh->items = it;
  }
  sync();
  const long long total = sh->total;
  if (maybe_waves(c, total, sh->items)) {
    // candidates for waves: a second look at the lengths
    unsigned long long distinct = 0;
    int longest = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s) {
      const Seq sq = load_seq(q, s);
      if (sq.n == 0) continue;
      const int seen = visible(q, sq, sq.n - 1);
      distinct += (unsigned long long)c.Hkv * seen;
      longest = max(longest, (seen + c.tile - 1) / c.tile);
    }
    if (distinct > 0) {
      atomicAdd(&sh->distinct, distinct);
      atomicMax(&sh->longest, longest);
    }
    sync();
    if ((long long)sh->distinct > c.wave_slots && total > 2 * (long long)sh->distinct) {
      const int most = sh->longest;
#pragma unroll 1
      for (int s = s0; s < s1; ++s) {
        const Seq sq = load_seq(q, s);
        if (sq.n == 0) continue;
        const int nt = max(1, (visible(q, sq, sq.n - 1) + c.tile - 1) / c.tile);
#pragma unroll 1
        for (int k = 0; k < kWaveTries; ++k) {
          const int bt = (most + k) / (k + 1);
          atomicAdd(&sh->units[k], (unsigned)(c.Hkv * row_tiles(c, sq.n) * ((nt + bt - 1) / bt)));
        }
      }
      sync();
      if (tid == 0) {
        long long best = -1;
        for (int k = 0; k < kWaveTries; ++k) {
          const int bt = (most + k) / (k + 1);
          if (sh->units[k] > kMaxUnits || bt < 8) continue;
          const long long cost = (long long)((sh->units[k] + gridDim.x - 1) / gridDim.x) * (bt * c.tile + c.fixed);
          if (best < 0 || cost < best) {
            best = cost;
            sh->wave_tiles = bt;
          }
        }
        // (an uneven mix of lengths leaves holes in the waves; the keys are fetched again instead)
        if (best > total / (long long)gridDim.x * 3 / 2) sh->wave_tiles = 0;
      }
      sync();
      const bool waves = sh->wave_tiles > 0;
      sync();                  // (the memory may be the destination of copies as soon as one warp goes on)
      if (waves) return;
    }
  }
  const long long ch = stretch(c, total, sh->items);
  *chunk = ch;
  const long long p0 = ch * blockIdx.x;
  const long long excl = sh->warp_len[warp] + incl - len;
  if (p0 < total && p0 >= excl && p0 < excl + len) {          // one thread holds the sequence
    long long at = excl;
    for (int s = s0; s < s1; ++s) {
      const Seq sq = load_seq(q, s);
      const long long w = c.Hkv * items_length(c, q.causal, sq.base, row_tiles(c, sq.n));
      if (p0 < at + w) {
        sh->s = s;
        sh->start = at;
        break;
      }
      at += w;
    }
  }
  sync();
}

// Walks the pieces of this CTA; run by one whole warp (all lanes hold the same state but for the sequence window).
struct Walker {
  long long chunk, p1, item_start;
  long long total_len;
  int s, h, r, R, n_seq;
  int w_first, w_n, w_base, w_s0;          // lane i: sequence w_s0 + i
  Seq cur;
  int wave_tiles, unit, unit0, item0, nb;  // calls in waves: next unit, units and items before the current sequence
  int first_piece_tile;                    // tile the first piece starts with, -1 once taken
  bool more;

  __device__ __forceinline__ void fetch(const Seqs& q, int s_) {
    const int lane = threadIdx.x & 31;
    if (s_ < w_s0 || s_ >= w_s0 + 32) {
      w_s0 = s_;
      Seq x = {0, 0, 0, false, false};
      if (s_ + lane < n_seq) x = load_seq(q, s_ + lane);
      w_first = x.first;
      w_n = x.n;
      w_base = x.base;
    }
    const int from = s_ - w_s0;
    cur.first = __shfl_sync(0xffffffffu, w_first, from);
    cur.n = __shfl_sync(0xffffffffu, w_n, from);
    cur.base = __shfl_sync(0xffffffffu, w_base, from);
  }
  __device__ __forceinline__ long long item_length(const Seqs& q, const SplitCfg& c) const {
    return (long long)cur.base + c.fixed + (q.causal ? (long long)(r + 1) * c.tokens : 0);
  }
  __device__ __forceinline__ int tiles(const Seqs& q, const SplitCfg& c) const {
    const int t = min((r + 1) * c.tokens, cur.n) - 1;
    return max(1, (visible(q, cur, t) + c.tile - 1) >> (31 - __clz(c.tile)));
  }
  // tile border nearest to position p of the current item; pieces shorter than two tiles are not worth their merge
  __device__ __forceinline__ int border(const SplitCfg& c, long long p, int nt) const {
    const long long y = p - item_start - c.fixed;
    if (y <= 0) return 0;
    long long t = (y + c.tile / 2) >> (31 - __clz(c.tile));
    if (t < 2) return 0;
    if (t > nt - 2) return nt;
    return (int)t;
  }
  // Lays the call out, unless the block has (ch is its result then), and finds this CTA's place.
  __device__ __forceinline__ void begin(const Seqs& q, const SplitCfg& c, PlanShared* sh, long long ch, int* d_status) {
    const int lane = threadIdx.x & 31;
    wave_tiles = 0;
    w_s0 = -64;
    if (q.n_seq <= 32) {
      // A sequence per lane, nothing through shared memory: 1.6 us of every call's latency, 2.6 us with the general form
      // below (chains of loads and 64-bit arithmetic that only many sequences need).
      Seq x = {0, 0, 0, false, false};
      if (lane < q.n_seq) x = load_seq(q, lane);
      const unsigned back = __ballot_sync(0xffffffffu, x.backwards);
      n_seq = back != 0 ? __ffs(back) - 1 : q.n_seq;
      if (lane >= n_seq) x.n = 0;
      const int tiles_x = row_tiles(c, x.n);
      const long long len = c.Hkv * items_length(c, q.causal, x.base, tiles_x);
      const int items = __reduce_add_sync(0xffffffffu, c.Hkv * tiles_x);
      long long incl = len;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      total_len = __shfl_sync(0xffffffffu, incl, 31);
      if (!maybe_waves(c, total_len, items)) {
        if (x.clamped && blockIdx.x == 0) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
        chunk = stretch(c, total_len, items);
        const long long p0 = chunk * blockIdx.x;
        more = p0 < total_len;
        if (!more) return;
        s = __ffs(__ballot_sync(0xffffffffu, p0 < incl)) - 1;
        w_s0 = 0;
        w_first = x.first;
        w_n = x.n;
        w_base = x.base;
        place(q, c, p0, __shfl_sync(0xffffffffu, incl - len, s));
        return;
      }
    }
    if (q.n_seq <= kWarpPlanSeqs) plan_block<32>(q, c, sh, &ch, d_status, lane);
    n_seq = sh->n_seq;
    total_len = sh->total;
    chunk = ch;
    wave_tiles = sh->wave_tiles;
    if (wave_tiles > 0) {
      unit = blockIdx.x;
      unit0 = item0 = 0;
      s = -1;
      R = nb = 0;
      more = true;
      return;
    }
    more = ch * blockIdx.x < total_len;
    if (!more) return;
    s = sh->s;
    place(q, c, ch * blockIdx.x, sh->start);
  }
  // The item at position p0 of the axis, in sequence s, which starts at position `start`.
  __device__ __forceinline__ void place(const Seqs& q, const SplitCfg& c, long long p0, long long start) {
    p1 = min(p0 + chunk, total_len);
    fetch(q, s);
    R = row_tiles(c, cur.n);
    const long long per_head = items_length(c, q.causal, cur.base, R);
    long long rem = p0 - start;
    h = (int)quotient(rem, per_head);
    rem -= h * per_head;
    // largest r whose items before it are no longer than rem: 32 candidates at a time
    const int lane = threadIdx.x & 31;
    int lo = 0, n = R;                       // it is one of lo .. lo + n - 1
#pragma unroll 1
    while (n > 1) {
      const int step = (n + 31) >> 5, at = lane * step;
      const unsigned fits = __ballot_sync(0xffffffffu, at < n && items_length(c, q.causal, cur.base, lo + at) <= rem);
      const int skip = (__popc(fits) - 1) * step;          // (lengths rise with r, and lane 0's fits)
      lo += skip;
      n = min(step, n - skip);
    }
    r = lo;
    item_start = start + h * per_head + items_length(c, q.causal, cur.base, r);
    first_piece_tile = border(c, p0, tiles(q, c));
  }
  // Next unit of a call in waves.
  __device__ __forceinline__ bool next_unit(const Seqs& q, const SplitCfg& c, Piece* out) {
#pragma unroll 1
    while (true) {
      while (s < 0 || unit >= unit0 + c.Hkv * R * nb) {     // the sequence that holds it
        if (s >= 0) {
          unit0 += c.Hkv * R * nb;
          item0 += c.Hkv * R;
        }
        if (++s >= n_seq) return false;
        fetch(q, s);
        R = row_tiles(c, cur.n);
        // (a sequence whose rows see nothing still gets its rows written)
        nb = R == 0 ? 0 : max(1, (visible(q, cur, cur.n - 1) + c.tile * wave_tiles - 1) / (c.tile * wave_tiles));
      }
      int rest = unit - unit0;
      r = rest % R;
      rest /= R;
      const int b = rest % nb;
      h = rest / nb;
      const int nt = tiles(q, c);
      const int u = unit;
      unit += gridDim.x;
      if (b * wave_tiles >= nt) continue;
      out->tile0 = b * wave_tiles;
      out->tile1 = min(out->tile0 + wave_tiles, nt);
      describe(q, c, out);
      out->n_pieces = (nt + wave_tiles - 1) / wave_tiles;
      out->ticket = item0 + h * R + r;
      out->slot0 = u - b * R;
      out->slot_step = R;
      out->slot = out->n_pieces > 1 ? u : -1;
      return true;
    }
  }
  __device__ __forceinline__ void describe(const Seqs& q, const SplitCfg& c, Piece* out) const {
    out->s = s;
    out->h = h;
    out->r = r;
    out->first = cur.first;
    out->n = cur.n;
    out->base = cur.base;
    out->seen0 = visible(q, cur, r * c.tokens);
    out->seen = visible(q, cur, min((r + 1) * c.tokens, cur.n) - 1);
  }
  // Next piece; false when the CTA's stretch is done.
  __device__ __forceinline__ bool next(const Seqs& q, const SplitCfg& c, Piece* out) {
    if (wave_tiles > 0) return next_unit(q, c, out);
#pragma unroll 1
    while (more) {
      const int nt = tiles(q, c);
      const long long end = item_start + item_length(q, c);
      const int t0 = first_piece_tile >= 0 ? first_piece_tile : 0;
      const bool starts_inside = first_piece_tile > 0;
      first_piece_tile = -1;
      const int t1 = p1 >= end ? nt : border(c, p1, nt);
      const bool ends_inside = t1 < nt;
      const bool emit = t0 < t1;
      if (emit) {
        describe(q, c, out);
        out->tile0 = t0;
        out->tile1 = t1;
        out->slot = -1;
        out->ticket = 0;
        out->n_pieces = 1;
        if (starts_inside || ends_inside) {
          // borders inside the item, after they have been moved to tile borders
          long long ca = quotient(item_start, chunk) + 1, cb = quotient(end - 1, chunk);
#pragma unroll 1
          while (ca <= cb && border(c, ca * chunk, nt) == 0) ++ca;
#pragma unroll 1
          while (cb >= ca && border(c, cb * chunk, nt) >= nt) --cb;
          out->slot = 2 * (int)blockIdx.x + (starts_inside ? 0 : 1);
          out->ticket = (int)ca;
          out->n_pieces = (int)(cb - ca) + 2;
          out->slot0 = 2 * ((int)ca - 1) + 1;
          out->slot_step = 0;
        }
      }
      // move on
      if (p1 <= end) {
        more = false;
      } else {
        item_start = end;
        if (++r == R) {
          r = 0;
          if (++h == c.Hkv) {
            h = 0;
#pragma unroll 1
            do {
              ++s;
              if (s >= n_seq) { more = false; break; }
              fetch(q, s);
            } while (cur.n == 0);
            if (more) R = row_tiles(c, cur.n);
          }
        }
      }
      if (emit) return true;
    }
    return false;
  }
};

// Takes a ticket of a cut item; true for the CTA that comes last, which also clears the ticket.  One thread per piece,
// after its CTA's partial results are written and fenced.
__device__ __forceinline__ bool last_piece(int* d_status, int ticket, int n_pieces) {
  const int word = ticket / 4 < 31 ? 1 + ticket / 4 : 2 + ticket / 4;
  const int shift = 8 * (ticket & 3);
  const unsigned old = atomicAdd(reinterpret_cast<unsigned*>(d_status) + word, 1u << shift);
  if (((old >> shift) & 255u) != (unsigned)(n_pieces - 1)) return false;
  atomicSub(reinterpret_cast<unsigned*>(d_status) + word, (unsigned)n_pieces << shift);
  return true;
}

}  // namespace samkv
