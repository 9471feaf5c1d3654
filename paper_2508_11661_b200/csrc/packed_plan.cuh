// How the attention kernels over packed sequences divide their work among persistent CTAs.
//
// An item is a row tile (up to `rows` packed query rows: tokens x group members) of one sequence and KV head; its keys
// come in tiles of `tile` slots.  All items of a call are laid out on one axis, sequence by sequence, head by head, row
// tile by row tile, each as long as the slots its last token sees plus a fixed share for prologue and epilogue.  CTA c
// takes the stretch [c, c + 1) * chunk of that axis; a border inside an item is moved to the nearest tile border.  Every
// CTA therefore gets the same work whatever the mix of lengths, an item is cut into more than one piece only where a
// border falls, and the host needs to know none of the lengths.  Lengths along the axis are linear in the row tile's
// index, so positions are found by closed forms and a binary search.
//
// A cut item's pieces leave (m, l, O) in the workspace, at most two pieces per CTA: the one a CTA starts with (slot 2c)
// and the one it ends with (slot 2c + 1).  The CTA that finishes an item's last piece merges them in order of the axis,
// so results do not depend on timing.  Tickets are bytes of the workspace's status block, one per first border of an
// item, and return to zero.
#pragma once

#include "packed.cuh"

namespace samkv {

constexpr int kMaxPackedCtas = 160;            // tickets: bytes of status words 1..31 and 33..41 (0 and 32 have other uses)

struct SplitCfg {
  int G, Hkv;
  int tokens;                  // tokens per row tile (rows / G)
  int tile;                    // slots per key tile
  int fixed;                   // slots that an item's fixed cost amounts to (>= 2 * tile)
  int min_chunk;               // least slots (fixed cost included) worth a CTA of its own (>= 2 * tile)
};

struct Piece {
  int s, h, r;                 // sequence, KV head, row tile
  int first, n, base;          // of the sequence, as in Seq
  int seen0, seen;             // slots that the row tile's first and last token see
  int tile0, tile1;            // key tiles of this piece
  int slot;                    // workspace slot of the partial result, -1: the piece is the whole item
  int ticket;                  // first border inside the item
  int n_pieces;
};

__device__ __forceinline__ int row_tiles(const SplitCfg& c, int n) { return (n + c.tokens - 1) / c.tokens; }
// length of the first x items of one (sequence, head)
__device__ __forceinline__ long long items_length(const SplitCfg& c, int causal, int base, int x) {
  long long len = (long long)x * (base + c.fixed);
  if (causal) len += (long long)c.tokens * x * (x + 1) / 2;
  return len;
}

struct PlanShared {
  long long warp_len[32];
  int warp_items[32];
  long long start;             // position of the sequence found
  int s;
  long long total;             // length of the axis
  int items;
};

// Block-wide: finds the sequence that holds this CTA's first position.  All kThreads threads call it; afterwards
// *chunk is the length of a CTA's stretch (0: nothing to do) and sh->s, sh->start are set for CTAs that have one.
template <int kThreads>
__device__ __forceinline__ void plan_block(const Seqs& q, const SplitCfg& c, PlanShared* sh, long long* chunk, int* d_status) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kWarps = kThreads / 32;
  const int per = (q.n_seq + kThreads - 1) / kThreads;
  const int s0 = min(tid * per, q.n_seq), s1 = min(s0 + per, q.n_seq);
  long long len = 0;
  int items = 0;
  bool clamped = false;
#pragma unroll 1
  for (int s = s0; s < s1; ++s) {
    const Seq sq = load_seq(q, s);
    const int R = row_tiles(c, sq.n);
    len += c.Hkv * items_length(c, q.causal, sq.base, R);
    items += c.Hkv * R;
    clamped |= sq.clamped;
  }
  if (clamped && blockIdx.x == 0) atomicMax(d_status, (int)CHECK_SEQ_RANGE);
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
  __syncthreads();
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
  __syncthreads();
  const long long total = sh->total;
  long long ctas = total / c.min_chunk;
  if (ctas < sh->items) ctas = sh->items;
  if (ctas > (long long)gridDim.x) ctas = gridDim.x;
  if (ctas < 1) ctas = 1;
  const long long ch = (total + ctas - 1) / ctas;
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
  __syncthreads();
}

// Walks the pieces of this CTA; run by one whole warp (all lanes hold the same state but for the sequence window).
struct Walker {
  long long chunk, p1, item_start;
  long long total_len;
  int s, h, r, R;
  int w_first, w_n, w_base, w_s0;          // lane i: sequence w_s0 + i
  Seq cur;
  int first_piece_tile;                    // tile the first piece starts with, -1 once taken
  bool more;

  __device__ __forceinline__ void fetch(const Seqs& q, int s_) {
    const int lane = threadIdx.x & 31;
    if (s_ < w_s0 || s_ >= w_s0 + 32) {
      w_s0 = s_;
      Seq x = {0, 0, 0, false};
      if (s_ + lane < q.n_seq) x = load_seq(q, s_ + lane);
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
    return max(1, (visible(q, cur, t) + c.tile - 1) / c.tile);
  }
  // tile border nearest to position p of the current item; pieces shorter than two tiles are not worth their merge
  __device__ __forceinline__ int border(const SplitCfg& c, long long p, int nt) const {
    const long long y = p - item_start - c.fixed;
    if (y <= 0) return 0;
    long long t = (y + c.tile / 2) / c.tile;
    if (t < 2) return 0;
    if (t > nt - 2) return nt;
    return (int)t;
  }
  __device__ __forceinline__ void init(const Seqs& q, const SplitCfg& c, const PlanShared* sh, long long ch) {
    const long long p0 = ch * blockIdx.x;
    total_len = sh->total;
    chunk = ch;
    more = p0 < total_len;
    if (!more) return;
    p1 = min(p0 + ch, total_len);
    s = sh->s;
    w_s0 = -64;
    fetch(q, s);
    R = row_tiles(c, cur.n);
    const long long per_head = items_length(c, q.causal, cur.base, R);
    long long rem = p0 - sh->start;
    h = (int)(rem / per_head);
    rem -= h * per_head;
    int lo = 0, hi = R - 1;                  // largest r whose items before it are no longer than rem
#pragma unroll 1
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (items_length(c, q.causal, cur.base, mid) <= rem) lo = mid; else hi = mid - 1;
    }
    r = lo;
    item_start = sh->start + h * per_head + items_length(c, q.causal, cur.base, r);
    first_piece_tile = border(c, p0, tiles(q, c));
  }
  // Next piece; false when the CTA's stretch is done.
  __device__ __forceinline__ bool next(const Seqs& q, const SplitCfg& c, Piece* out) {
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
        out->s = s;
        out->h = h;
        out->r = r;
        out->first = cur.first;
        out->n = cur.n;
        out->base = cur.base;
        out->seen0 = visible(q, cur, r * c.tokens);
        out->seen = visible(q, cur, min((r + 1) * c.tokens, cur.n) - 1);
        out->tile0 = t0;
        out->tile1 = t1;
        out->slot = -1;
        out->ticket = 0;
        out->n_pieces = 1;
        if (starts_inside || ends_inside) {
          // borders inside the item, after they have been moved to tile borders
          long long ca = item_start / chunk + 1, cb = (end - 1) / chunk;
#pragma unroll 1
          while (ca <= cb && border(c, ca * chunk, nt) == 0) ++ca;
#pragma unroll 1
          while (cb >= ca && border(c, cb * chunk, nt) >= nt) --cb;
          out->slot = 2 * (int)blockIdx.x + (starts_inside ? 0 : 1);
          out->ticket = (int)ca;
          out->n_pieces = (int)(cb - ca) + 2;
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
              if (s >= q.n_seq) { more = false; break; }
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

// Workspace slot of an item's piece k (0 = the one at the item's start): the first is the last piece of the CTA before
// the first border, the others are the first pieces of the CTAs that start at the borders.
__device__ __forceinline__ int piece_slot(int ticket, int k) { return k == 0 ? 2 * (ticket - 1) + 1 : 2 * (ticket + k - 1); }

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
