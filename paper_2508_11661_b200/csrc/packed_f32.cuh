// Attention of packed sequences over packed rows or over a paged cache, fp32 throughout (tensor cores would round the
// operands to tf32).
//
// Persistent, one CTA of 256 threads per SM, work divided by packed_plan.cuh, key tiles of 64 slots, two to four of them in
// shared memory with cp.async.  Multiply-adds are issued two at a time (fma.rn.f32x2: the same roundings, half the issue
// slots).  Row tiles of 64, 32 or 8 packed rows; launch_packed_attn chooses.
//   64 and 32 rows: a thread owns kRows/16 rows x 4 slots of the scores and the same rows x d/16 columns of the result.
//     The 16 threads of a row agree on maxima and sums by shuffles.
//   8 rows: each warp takes 8 slots of every tile, loads them itself and runs its own online softmax, so that nothing in
//     the loop waits for another warp; the eight results are joined when a piece ends.  A thread keeps 8 rows x 8 elements
//     of Q in registers, reads a slot's key once, and the d / 8 threads of a slot are added up by shuffles that leave each
//     with a row of its own; for the result it owns 8 rows x 4 columns.
// Measured: prompts of 1024 and 700 tokens, 32/8 heads of 128, 64 rows: 538 us, 30 TFLOP/s of the FMA pipe's nominal 74
// (shared memory is busy 62 % of the cycles, and two warps per scheduler cover little of their chains).  Decode, 32 requests x 1000
// slots, 32/8 heads of 128, 8 rows: 55 us, 4.9 TB/s (138 us when the CTA shared tiles of 16 rows).  Little work is latency:
// an item costs about 2 us besides its tiles (a third until its first tile is there, 0.5 us to join the warps' results);
// 6 sequences of 1 to 64 tokens, 4/2 heads of 64: 16 us (22 us with 16 rows).  Starting the next item's loads before the
// results leave made every shape 4 to 8 % slower (the code grew), so it is not done.
// Modified scores (kMod; see packed_scores.cuh): 4 documents of 256 tokens and a question of 32 in one sequence, slopes, 4/2 heads of 64:
// 33 us; 4 prompts of 256 with a window 25 us (21 us plain: the plan, and partly seen tiles slot by slot).
#pragma once

#include <math.h>

#include <type_traits>

#include "packed_scores.cuh"

namespace samkv {
namespace pf32 {

constexpr int kBN = 64, kThreads = 256;

template <int kD, int kRows>
struct Smem {
  static constexpr bool kFew = kRows == 8;
  static constexpr int kLd = kFew ? kD : kD + 4;         // row stride in floats: 16 bytes on in the banks, or rows read whole
  static constexpr int kPLd = kFew ? 12 : kBN + 4;
  static constexpr int kTile = kBN * kLd * 4;
  static constexpr int kQ = 0;                           // (8 rows: Q is in registers)
  // [kStages][K, V]; P takes K's place once the scores are done (8 rows: has its own); a piece's results leave by the first
  static constexpr int kKv = kFew ? 0 : kRows * kLd * 4;
  // tiles in shared memory: as many as fit, since a short tile is done before the next one has come
  static constexpr int kStages = kD == 64 ? 4 : kRows == 64 ? 2 : 3;
  static constexpr int kP = kKv + kStages * 2 * kTile;             // 8 rows: [warp][slot][row] weights
  static constexpr int kCorr = kP + (kFew ? 8 * 8 * kPLd * 4 : 0);  // 8 rows: [warp][row] rescaling factors
  static constexpr int kMl = kCorr + (kFew ? 8 * 8 * 4 : 0);       // [warp, or one][row] maximum and sum
  static constexpr int kPiece = kMl + (kFew ? 8 : 1) * kRows * 8;  // [2]
  static constexpr int kBytes = kPiece + 256;
  static_assert(sizeof(Piece) <= 96 && sizeof(MaskedPiece) <= 96 && kBytes <= 227 * 1024, "shared memory of a CTA");
};

struct Params {
  Seqs seqs;
  SplitCfg cfg;
  Pages pages;
  Rows Q, K, V, O;                                       // K, V: packed rows, or the pools
  float scale;
  float* lse;
  float* part_o;                                         // [slot][kRows][kD]
  float2* part_ml;                                       // [slot][kRows]
  int* d_status;
  int Hq;
  // calls with modified scores
  ScoreMods mods;
  ScorePlan plan;
  float cap_in;                                          // 1 / softcap
};

// A score that a row sees, modified.
__device__ __forceinline__ float modify(const Params& p, float x, float slope, int distance) {
  if (p.mods.softcap > 0.f) x = p.mods.softcap * tanhf(x * p.cap_in);
  return fmaf(-slope, fabsf((float)distance), x);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  const int sz = valid ? 16 : 0;                         // 0: the 16 bytes are zero-filled
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(sz) : "memory");
}
__device__ __forceinline__ float4 lds4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ ulonglong2 lds4x2(const float* p) { return *reinterpret_cast<const ulonglong2*>(p); }
}  // namespace pf32

// kMod: with modified scores.
template <int kD, int kRows, bool kPaged, bool kMod>
__global__ void __launch_bounds__(pf32::kThreads, 1)
packed_f32_kernel(const __grid_constant__ pf32::Params p) {
  using namespace pf32;
  using L = Smem<kD, kRows>;
  using P = std::conditional_t<kMod, MaskedPiece, Piece>;
  constexpr bool kFew = L::kFew;
  constexpr int kLd = L::kLd, kPLd = L::kPLd;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float* sQ = reinterpret_cast<float*>(smem_raw + L::kQ);
  auto sK = [&](int st) { return reinterpret_cast<float*>(smem_raw + L::kKv + st * 2 * L::kTile); };
  auto sV = [&](int st) { return reinterpret_cast<float*>(smem_raw + L::kKv + st * 2 * L::kTile + L::kTile); };
  float2* sMl = reinterpret_cast<float2*>(smem_raw + L::kMl);
  P* s_piece = reinterpret_cast<P*>(smem_raw + L::kPiece);
  volatile int* s_flag = reinterpret_cast<volatile int*>(smem_raw + L::kPiece + 200);
  PlanShared& plan = *reinterpret_cast<PlanShared*>(smem_raw + L::kKv);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.cfg.G;
  pdl_wait();
  long long chunk = 0;
  std::conditional_t<kMod, PieceWindow, Walker> w;
  w.more = false;
  ScorePlan tiles = {};
  if constexpr (kMod) {
    tiles = plan_of_block<kThreads>(p.seqs, p.mods, p.cfg, p.plan, smem_raw + L::kKv, p.d_status);
    if (warp == 0) w.begin(p.seqs, p.mods, p.cfg, tiles, kPaged, p.d_status);
  } else {
    if (p.seqs.n_seq > kWarpPlanSeqs) plan_block<kThreads>(p.seqs, p.cfg, &plan, &chunk, p.d_status, tid);
    if (warp == 0) w.begin(p.seqs, p.cfg, &plan, chunk, p.d_status);
  }
  bool bad = false, lost = false;                        // a table entry that is no page; one that some token sees
  auto next_piece = [&](int at) {
    if constexpr (kMod) {
      const int from = w.take(p.seqs, p.mods, p.cfg, tiles, kPaged, p.d_status);
      if (lane == from) s_piece[at] = w.mine;
      if (from < 0 && lane == 0) s_piece[at].tile0 = -1;
    } else {
      P next;
      if (!w.next(p.seqs, p.cfg, &next)) next.tile0 = -1;
      if (lane == 0) s_piece[at] = next;
    }
  };
  // slot that a tile begins with, by its number in the piece's list of tiles (from the first to the last: results are rescaled
  // at every tile anyway)
  auto slot0_of = [&](const P& pc, int t) {
    if constexpr (kMod) return pc.template tile<false>(t - pc.tile0, kBN) * kBN; else return t * kBN;
  };
  // whether some row sees the slot
  auto is_used = [&](const P& pc, int j) {
    if constexpr (kMod) return j < pc.seen && any_sees(pc, any1_of(p.seqs, pc), j, j + 1); else return j < pc.seen;
  };
  if (warp == 0) next_piece(0);

#pragma unroll 1
  for (int k = 0;; ++k) {
    __syncthreads();                                     // everybody is done with the previous piece (and the plan)
    const P pc = s_piece[k & 1];
    if (pc.tile0 < 0) break;
    int n_rows, tok0, head, seq, key0, last_tok = 0;
    Seq sq;
    if constexpr (kMod) {
      n_rows = pc.n_tok * G;
      tok0 = pc.tok0;
      head = pc.h();
      seq = key0 = pc.kv;
    } else {
      n_rows = min(p.cfg.tokens, pc.n - pc.r * p.cfg.tokens) * G;
      tok0 = pc.first + pc.r * p.cfg.tokens;
      head = pc.h;
      seq = pc.s;
      key0 = pc.first;
      sq.first = pc.first; sq.n = pc.n; sq.base = pc.base;
      last_tok = min((pc.r + 1) * p.cfg.tokens, pc.n) - 1;
    }
    const uint32_t smem = (uint32_t)__cvta_generic_to_shared(smem_raw);
    float* part = sK(0);                                 // [warp, or one][row][column]: results on their way out
    if constexpr (kFew) {
      // ================= 8 rows: the warps on their own =================
      constexpr int kDs = kD / 8, kKeys = 32 / kDs, kIter = 8 / kKeys;     // lanes of a slot, slots at a time
      const int ds = lane % kDs, sub = lane / kDs;
      const int row = kDs == 16 ? ds >> 1 : ds;                            // whose score the lane is left with
      const bool b0 = ds & (kDs / 2), b1 = ds & (kDs / 4), b2 = ds & (kDs / 8);
      constexpr int kLanes = kD / 4, kStep = 32 / kLanes;                  // lanes of a row of K or V
      const int c4 = lane % kLanes * 4, half = lane / kLanes;              // (d = 64: even and odd slots of the result)
      float* sP = reinterpret_cast<float*>(smem_raw + L::kP) + warp * 8 * kPLd;
      float* sCorr = reinterpret_cast<float*>(smem_raw + L::kCorr) + warp * 8;
      // The lanes hold the page numbers of four tiles, lane 8 i + j that of slot j of this warp's share of tile t4 + i.  The
      // next four are asked for when the last of them is used, and first looked at a tile later.
      int t4 = pc.tile0, page = 0;
      auto slot_of_lane = [&]() { return slot0_of(pc, t4 + (lane >> 3)) + warp * 8 + (lane & 7); };
      auto wanted = [&]() { return t4 + (lane >> 3) < pc.tile1 && is_used(pc, slot_of_lane()); };
      auto look_up = [&]() {
        if (kPaged && wanted()) page = p.pages.table[(size_t)seq * p.pages.width + (slot_of_lane() >> p.pages.shift)];
      };
      look_up();
      auto load_kv = [&](int t, int st) {
        const int four = (t - t4) * 8;
        long long where = -1;                            // row of K and V for the lane's slot
        if (wanted()) {
          where = key0 + slot_of_lane();
          if constexpr (kPaged) {
            if ((unsigned)page >= (unsigned)p.pages.n_pages) {
              bad = true;
              page = 0;
            }
            const int shift = p.pages.shift;
            where = (((long long)page * p.cfg.Hkv + head) << shift) + (slot_of_lane() & ((1 << shift) - 1));
          }
        }
        const uint32_t dk = smem + L::kKv + st * 2 * L::kTile + (warp * 8 + half) * kD * 4 + c4 * 4, dv = dk + L::kTile;
#pragma unroll
        for (int r = 0; r < 8; r += kStep) {
          const long long x = __shfl_sync(0xffffffffu, where, four + r + half);
          const bool ok = x >= 0;                        // slots that no row sees read as zero
          size_t ko = ok ? (size_t)x * kD + c4 : 0, vo = ko;
          if constexpr (!kPaged) {
            ko = ok ? (size_t)x * p.K.ts + (size_t)head * p.K.hs + c4 : 0;
            vo = ok ? (size_t)x * p.V.ts + (size_t)head * p.V.hs + c4 : 0;
          }
          cp_async16(dk + r * kD * 4, static_cast<const float*>(p.K.data) + ko, ok);
          cp_async16(dv + r * kD * 4, static_cast<const float*>(p.V.data) + vo, ok);
        }
        if (four == 24) {
          t4 += 4;
          look_up();
        }
      };
#pragma unroll 1
      for (int i = 0; i < L::kStages - 1; ++i) {
        if (pc.tile0 + i < pc.tile1) load_kv(pc.tile0 + i, i);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      f2 q[8][4];                                        // (after the copies of K and V are on their way: 1 to 5 % faster)
      const float* qp = static_cast<const float*>(p.Q.data) + (size_t)tok0 * p.Q.ts + (size_t)head * G * p.Q.hs + ds * 4;
      int member = 0;                                    // row i: token i / G, group member i % G
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const ulonglong2 x = i < n_rows ? *reinterpret_cast<const ulonglong2*>(qp + e * (kD / 2)) : make_ulonglong2(0ull, 0ull);
          q[i][e * 2] = x.x;
          q[i][e * 2 + 1] = x.y;
        }
        qp += p.Q.hs;
        if (++member == G) {
          member = 0;
          qp += (ptrdiff_t)p.Q.ts - (ptrdiff_t)G * p.Q.hs;
        }
      }
      if (warp == 0) next_piece((k + 1) & 1);
      int vis = 0;
      RowView view = {};
      float slope = 0.f;
      if constexpr (kMod) {
        view = row_view(p.seqs, p.mods, pc, row / G);
        if (p.mods.slopes != nullptr) slope = p.mods.slopes[head * G + row % G];
      } else {
        vis = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + row / G, last_tok));
      }
      float m = -INFINITY, l = 0.f;
      f2 acc[4][4];                                      // [pair of rows][column]
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0ull;
#pragma unroll 1
      for (int t = pc.tile0; t < pc.tile1; ++t) {
        const int st = (t - pc.tile0) % L::kStages, j0 = slot0_of(pc, t) + warp * 8;
        asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
        __syncwarp();                                    // the warp's share of tile t is there, that of tile t - 1 used up
        if (t + L::kStages - 1 < pc.tile1) load_kv(t + L::kStages - 1, (t - pc.tile0 + L::kStages - 1) % L::kStages);
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (!kMod && j0 >= pc.seen) break;               // (only in the last tile)
        // ---- scores ----
        float x[kIter], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const float* kp = sK(st) + (warp * 8 + i * kKeys + sub) * kD + ds * 4;
          const ulonglong2 a = lds4x2(kp), b = lds4x2(kp + kD / 2);
          float v[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float2 z = split2(fma2(q[r][3], b.y, fma2(q[r][2], b.x, fma2(q[r][1], a.y, mul2(q[r][0], a.x)))));
            v[r] = z.x + z.y;
          }
          // every exchange halves the rows that a lane still adds up
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = (b0 ? v[r + 4] : v[r]) + __shfl_xor_sync(0xffffffffu, b0 ? v[r] : v[r + 4], kDs / 2);
#pragma unroll
          for (int r = 0; r < 2; ++r) v[r] = (b1 ? v[r + 2] : v[r]) + __shfl_xor_sync(0xffffffffu, b1 ? v[r] : v[r + 2], kDs / 4);
          v[0] = (b2 ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, b2 ? v[0] : v[1], kDs / 8);
          if constexpr (kDs == 16) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
          const int j = j0 + i * kKeys + sub;
          if constexpr (kMod) x[i] = view.sees(j) ? modify(p, v[0] * p.scale, slope, view.pos - j) : -INFINITY;
          else x[i] = j < vis ? v[0] * p.scale : -INFINITY;
          mx = fmaxf(mx, x[i]);
        }
        // ---- online softmax ----
#pragma unroll
        for (int o = kDs; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float mn = fmaxf(m, mx), mu = mn == -INFINITY ? 0.f : mn;
        const float corr = m == mn ? 1.f : expf(m - mu);
        m = mn;
        l *= corr;
        const bool mine = kDs == 8 || (ds & 1) == 0;
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          x[i] = expf(x[i] - mu);
          l += x[i];                                     // (this lane's slots; joined at the end)
          if (mine) sP[(i * kKeys + sub) * kPLd + row] = x[i];
        }
        if (mine && sub == 0) sCorr[row] = corr;
        __syncwarp();
        // ---- result ----
        const float* v = sV(st) + warp * 8 * kD + c4;
        const ulonglong2 corr01 = lds4x2(sCorr), corr23 = lds4x2(sCorr + 4);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          acc[0][c] = mul2(acc[0][c], corr01.x);
          acc[1][c] = mul2(acc[1][c], corr01.y);
          acc[2][c] = mul2(acc[2][c], corr23.x);
          acc[3][c] = mul2(acc[3][c], corr23.y);
        }
        bool all_see;
        if constexpr (kMod) {
          int z0 = j0, z1 = j0 + 8;
          hidden_from_some(pc, &z0, &z1);
          all_see = z0 >= z1;
        } else {
          all_see = j0 + 8 <= pc.seen0;
        }
        if (all_see) {
#pragma unroll
          for (int j = 0; j < 8; j += kStep) {
            const float4 b = lds4(v + (j + half) * kD);
            const ulonglong2 w01 = lds4x2(sP + (j + half) * kPLd), w23 = lds4x2(sP + (j + half) * kPLd + 4);
            const f2 bb[4] = {both(b.x), both(b.y), both(b.z), both(b.w)};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              acc[0][c] = fma2(w01.x, bb[c], acc[0][c]);
              acc[1][c] = fma2(w01.y, bb[c], acc[1][c]);
              acc[2][c] = fma2(w23.x, bb[c], acc[2][c]);
              acc[3][c] = fma2(w23.y, bb[c], acc[3][c]);
            }
          }
        } else {
          // some row does not see some slot: a weight of zero would still carry over infinities and NaN
          const int n_any = min(8, pc.seen - j0);
          unsigned sees[8];                              // bit j: the row sees slot j0 + j
          unsigned bits = RowView::below(vis - j0);
          if constexpr (kMod) bits = view.bits(j0);
#pragma unroll
          for (int i = 0; i < 8; ++i) sees[i] = __shfl_sync(0xffffffffu, bits, kDs == 16 ? i * 2 : i);
#pragma unroll 1
          for (int j = half; j < n_any; j += kStep) {
            const float4 b = lds4(v + j * kD);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f2 w2 = *reinterpret_cast<const f2*>(sP + j * kPLd + i * 2);
              const bool s0 = sees[i * 2] >> j & 1u, s1 = sees[i * 2 + 1] >> j & 1u;
              acc[i][0] = fma2(w2, join2(s0 ? b.x : 0.f, s1 ? b.x : 0.f), acc[i][0]);
              acc[i][1] = fma2(w2, join2(s0 ? b.y : 0.f, s1 ? b.y : 0.f), acc[i][1]);
              acc[i][2] = fma2(w2, join2(s0 ? b.z : 0.f, s1 ? b.z : 0.f), acc[i][2]);
              acc[i][3] = fma2(w2, join2(s0 ? b.w : 0.f, s1 ? b.w : 0.f), acc[i][3]);
            }
          }
        }
      }
#pragma unroll
      for (int o = kDs; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
      if (sub == 0 && (kDs == 8 || (ds & 1) == 0)) sMl[warp * 8 + row] = make_float2(m, l);
      if constexpr (kStep == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float2 y = split2(acc[i][c]);
            acc[i][c] = join2(y.x + __shfl_xor_sync(0xffffffffu, y.x, 16), y.y + __shfl_xor_sync(0xffffffffu, y.y, 16));
          }
      }
      __syncthreads();                                   // the tiles are used up
      static_assert(8 * 8 * kD * 4 <= 2 * L::kTile, "the warps' results take the first stage");
      if (half == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = split2(acc[i][0]), b = split2(acc[i][1]), c = split2(acc[i][2]), d = split2(acc[i][3]);
          float* at = part + (warp * 8 + i * 2) * kD + c4;
          *reinterpret_cast<float4*>(at) = make_float4(a.x, b.x, c.x, d.x);
          *reinterpret_cast<float4*>(at + kD) = make_float4(a.y, b.y, c.y, d.y);
        }
      }
    } else {
      // ================= 64 and 32 rows: the CTA together =================
      constexpr int kR = kRows / 16;                     // rows per thread
      constexpr int kC = kD / 64;                        // result columns per thread: kC vectors of 4
      const int ty = tid >> 4, tx = tid & 15;            // rows ty * kR + i, slots tx + 16 j, columns tx * 4 + 64 c
      auto load_kv = [&](int t, int st) {
        const int j0 = slot0_of(pc, t);
        const uint32_t dk = smem + L::kKv + st * 2 * L::kTile, dv = dk + L::kTile;
        // a thread keeps its 16-byte column and steps through the rows
        constexpr int kLanes = kD / 4, kStep = kThreads / kLanes;
        const int c = tid % kLanes, r0 = tid / kLanes;
#pragma unroll 4
        for (int r = r0; r < kBN; r += kStep) {
          const bool ok = is_used(pc, j0 + r);             // slots that no row sees read as zero
          size_t ko = 0, vo = 0;
          if (ok) {
            if constexpr (kPaged) {
              ko = vo = page_offset(p.pages, seq, j0 + r, head, p.cfg.Hkv, kD, &bad) + c * 4;
            } else {
              ko = (size_t)(key0 + j0 + r) * p.K.ts + (size_t)head * p.K.hs + c * 4;
              vo = (size_t)(key0 + j0 + r) * p.V.ts + (size_t)head * p.V.hs + c * 4;
            }
          }
          cp_async16(dk + (r * kLd + c * 4) * 4, static_cast<const float*>(p.K.data) + ko, ok);
          cp_async16(dv + (r * kLd + c * 4) * 4, static_cast<const float*>(p.V.data) + vo, ok);
        }
      };
#pragma unroll 2
      for (int i = tid; i < kRows * (kD / 4); i += kThreads) {
        const int r = i / (kD / 4), c = i % (kD / 4);
        const bool ok = r < n_rows;
        const size_t off = ok ? (size_t)(tok0 + r / G) * p.Q.ts + (size_t)(head * G + r % G) * p.Q.hs + c * 4 : 0;
        cp_async16(smem + L::kQ + (r * kLd + c * 4) * 4, static_cast<const float*>(p.Q.data) + off, ok);
      }
      // (the last stage is filled from the loop on)
#pragma unroll 1
      for (int i = 0; i < L::kStages - 1; ++i) {
        if (pc.tile0 + i < pc.tile1) load_kv(pc.tile0 + i, i);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      if (warp == 0) next_piece((k + 1) & 1);
      int vis[kR];
      RowView view[kR];
      float slope[kR];
      float m[kR], l[kR];
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        const int row = ty * kR + i;
        if constexpr (kMod) {
          view[i] = row_view(p.seqs, p.mods, pc, row / G);
          slope[i] = p.mods.slopes != nullptr ? p.mods.slopes[head * G + row % G] : 0.f;
        } else {
          vis[i] = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + row / G, last_tok));
        }
        m[i] = -INFINITY;
        l[i] = 0.f;
      }
      f2 o2[kR][kC * 2];
#pragma unroll
      for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int c = 0; c < kC * 2; ++c) o2[i][c] = 0ull;
#pragma unroll 1
      for (int t = pc.tile0; t < pc.tile1; ++t) {
        const int st = (t - pc.tile0) % L::kStages, j0 = slot0_of(pc, t);
        asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
        __syncthreads();                                   // tile t is there, and tile t - 1 is used up
        if (t + L::kStages - 1 < pc.tile1) load_kv(t + L::kStages - 1, (t - pc.tile0 + L::kStages - 1) % L::kStages);
        asm volatile("cp.async.commit_group;" ::: "memory");
        // ---- scores ----
        f2 sum[kR][4];                                     // even and odd elements of the head dimension apart
#pragma unroll
        for (int i = 0; i < kR; ++i) sum[i][0] = sum[i][1] = sum[i][2] = sum[i][3] = 0ull;
        const float *k = sK(st) + tx * kLd, *q = sQ + ty * kR * kLd;
#pragma unroll 4
        for (int e = 0; e < kD; e += 4) {
          ulonglong2 kv[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) kv[j] = lds4x2(k + j * 16 * kLd + e);
#pragma unroll
          for (int i = 0; i < kR; ++i) {
            const ulonglong2 a = lds4x2(q + i * kLd + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[i][j] = fma2(a.y, kv[j].y, fma2(a.x, kv[j].x, sum[i][j]));
          }
        }
        float s[kR][4];
#pragma unroll
        for (int i = 0; i < kR; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 x = split2(sum[i][j]);
            s[i][j] = x.x + x.y;
          }
        // ---- online softmax ----
#pragma unroll
        for (int i = 0; i < kR; ++i) {
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int slot = j0 + tx + 16 * j;
            if constexpr (kMod) s[i][j] = view[i].sees(slot) ? modify(p, s[i][j] * p.scale, slope[i], view[i].pos - slot) : -INFINITY;
            else s[i][j] = slot < vis[i] ? s[i][j] * p.scale : -INFINITY;
            mx = fmaxf(mx, s[i][j]);
          }
#pragma unroll
          for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
          const float mn = fmaxf(m[i], mx), mu = mn == -INFINITY ? 0.f : mn;
          const float corr = m[i] == mn ? 1.f : expf(m[i] - mu);
          m[i] = mn;
          l[i] *= corr;
          const f2 corr2 = both(corr);
#pragma unroll
          for (int c = 0; c < kC * 2; ++c) o2[i][c] = mul2(o2[i][c], corr2);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = expf(s[i][j] - mu);
            l[i] += s[i][j];                               // (this thread's slots; joined at the end)
          }
        }
        __syncthreads();                                   // K is used up
        float* sP = sK(st);
#pragma unroll
        for (int i = 0; i < kR; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) sP[(ty * kR + i) * kPLd + tx + 16 * j] = s[i][j];
        __syncthreads();
        // ---- result ----
        const float *v = sV(st) + tx * 4, *pr = sP + ty * kR * kPLd;
        // slots that every row sees come four at a time; [n_all, n_any) holds those that some row does not see
        int n_all, n_any;
        if constexpr (kMod) {
          int z0 = j0, z1 = min(j0 + kBN, pc.seen);
          hidden_from_some(pc, &z0, &z1);
          n_all = z0 < z1 ? (z0 - j0) & ~3 : kBN;
          n_any = z0 < z1 ? z1 - j0 : kBN;
        } else {
          n_all = min(max(pc.seen0 - j0, 0), kBN) & ~3;
          n_any = min(pc.seen - j0, kBN);
        }
        auto four_at_a_time = [&](int from, int to) {
#pragma unroll 2
        for (int j = from; j < to; j += 4) {
          float4 a[kR];
#pragma unroll
          for (int i = 0; i < kR; ++i) a[i] = lds4(pr + i * kPLd + j);
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            ulonglong2 b[kC];
#pragma unroll
            for (int c = 0; c < kC; ++c) b[c] = lds4x2(v + (j + u) * kLd + c * 64);
#pragma unroll
            for (int i = 0; i < kR; ++i) {
              const f2 w2 = both(u == 0 ? a[i].x : u == 1 ? a[i].y : u == 2 ? a[i].z : a[i].w);
#pragma unroll
              for (int c = 0; c < kC; ++c) {
                o2[i][c * 2] = fma2(w2, b[c].x, o2[i][c * 2]);
                o2[i][c * 2 + 1] = fma2(w2, b[c].y, o2[i][c * 2 + 1]);
              }
            }
          }
        }
        };
        four_at_a_time(0, n_all);
        // slots that some row does not see: a weight of zero would still carry over infinities and NaN
        if constexpr (kMod) n_any = min((n_any + 3) & ~3, kBN);
#pragma unroll 1
        for (int j = n_all; j < n_any; ++j) {
          ulonglong2 b[kC];
#pragma unroll
          for (int c = 0; c < kC; ++c) b[c] = lds4x2(v + j * kLd + c * 64);
#pragma unroll
          for (int i = 0; i < kR; ++i) {
            const f2 w2 = both(pr[i * kPLd + j]);
            bool sees;
            if constexpr (kMod) sees = view[i].sees(j0 + j); else sees = j0 + j < vis[i];
            if (sees) {
#pragma unroll
              for (int c = 0; c < kC; ++c) {
                o2[i][c * 2] = fma2(w2, b[c].x, o2[i][c * 2]);
                o2[i][c * 2 + 1] = fma2(w2, b[c].y, o2[i][c * 2 + 1]);
              }
            }
          }
        }
        if constexpr (kMod) four_at_a_time(n_any, kBN);
      }
#pragma unroll
      for (int i = 0; i < kR; ++i) {
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
        if (tx == 0) sMl[ty * kR + i] = make_float2(m[i], l[i]);
      }
      __syncthreads();                                   // the tiles are used up
#pragma unroll
      for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int c = 0; c < kC; ++c)
          *reinterpret_cast<ulonglong2*>(part + (ty * kR + i) * kD + c * 64 + tx * 4) = make_ulonglong2(o2[i][c * 2], o2[i][c * 2 + 1]);
    }
    if constexpr (kMod && kPaged) {
      if (__builtin_expect(bad, 0)) {                    // was it the entry of a page that some token sees?
        bad = false;
#pragma unroll 1
        for (int i = pc.tile0 * kBN; i < pc.tile1 * kBN && !lost; ++i) {
          const int j = slot0_of(pc, i / kBN) + i % kBN;
          if (is_used(pc, j)) page_offset(p.pages, seq, j, head, p.cfg.Hkv, kD, &bad);
          lost = bad && token_sees(p.seqs, p.mods, pc, j, j + 1);
          bad = false;
        }
      }
    }
    __syncthreads();
    // rows leave the CTA (or their parts do) as whole lines
    auto write_row = [&](int r, int c, float4 x, float M, float Ls) {
      const int tok = tok0 + r / G, hq = head * G + r % G;
      const float inv = 1.0f / Ls;
      *reinterpret_cast<float4*>(static_cast<float*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs + c) =
          Ls == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
      if (c == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = Ls == 0.f ? -INFINITY : M + logf(Ls);
    };
    const int n_vec = n_rows * (kD / 4);
#pragma unroll 1
    for (int i = tid; i < n_vec; i += kThreads) {
      const int r = i / (kD / 4), c = i % (kD / 4) * 4;
      float2 ml = sMl[r];
      float4 x = lds4(part + r * kD + c);
      if constexpr (kFew) {
        float M = -INFINITY;
#pragma unroll
        for (int y = 0; y < 8; ++y)
          M = fmaxf(M, sMl[y * 8 + r].y != 0.f ? sMl[y * 8 + r].x : -INFINITY);
        ml = make_float2(M, 0.f);
        x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const float2 a = sMl[y * 8 + r];
          const bool any = a.y != 0.f;                   // (no branch: the eight go on side by side)
          const float wgt = any ? expf(a.x - M) : 0.f;
          const float4 z = lds4(part + (y * 8 + r) * kD + c);
          x.x = any ? fmaf(z.x, wgt, x.x) : x.x;
          x.y = any ? fmaf(z.y, wgt, x.y) : x.y;
          x.z = any ? fmaf(z.z, wgt, x.z) : x.z;
          x.w = any ? fmaf(z.w, wgt, x.w) : x.w;
          ml.y += a.y * wgt;
        }
      }
      if (pc.slot < 0) {
        write_row(r, c, x, ml.x, ml.y);
      } else {
        *reinterpret_cast<float4*>(p.part_o + ((size_t)pc.slot * kRows + r) * kD + c) = x;
        if (c == 0) p.part_ml[(size_t)pc.slot * kRows + r] = ml;
      }
    }
    if (pc.slot < 0) continue;
    // a piece of a cut item left (m, l, O); whoever takes the last ticket merges them in order of the pieces
    __threadfence();
    __syncthreads();
    if (tid == 0) *s_flag = last_piece(p.d_status, pc.ticket, pc.n_pieces);
    __syncthreads();
    if (*s_flag) {
      __threadfence();
#pragma unroll 1
      for (int i = tid; i < n_vec; i += kThreads) {
        const int r = i / (kD / 4), c = i % (kD / 4) * 4;
        float M = -INFINITY, Ls = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int n = 0; n < pc.n_pieces; ++n) {
          const float2 ml = __ldcg(p.part_ml + piece_slot(pc, n) * kRows + r);
          M = fmaxf(M, ml.y != 0.f ? ml.x : -INFINITY);
        }
#pragma unroll 4
        for (int n = 0; n < pc.n_pieces; ++n) {
          const size_t at = (size_t)piece_slot(pc, n) * kRows + r;
          const float2 ml = __ldcg(p.part_ml + at);
          const float4 z = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kD + c));
          const bool any = ml.y != 0.f;                  // (no branch: four loads under way at a time)
          const float wgt = any ? expf(ml.x - M) : 0.f;
          x.x = any ? fmaf(z.x, wgt, x.x) : x.x;
          x.y = any ? fmaf(z.y, wgt, x.y) : x.y;
          x.z = any ? fmaf(z.z, wgt, x.z) : x.z;
          x.w = any ? fmaf(z.w, wgt, x.w) : x.w;
          Ls += ml.y * wgt;
        }
        write_row(r, c, x, M, Ls);
      }
    }
  }
  if (bad || lost) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
  pdl_launch_dependents();
}

namespace pf32 {
template <int kD, int kRows, bool kPaged, bool kMod>
static cudaError_t launch(Params p, int ctas, char* ws, cudaStream_t stream) {
  p.cfg.tokens = kRows / p.cfg.G;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)2 * ctas * kRows * kD * 4);
  auto kern = packed_f32_kernel<kD, kRows, kPaged, kMod>;
  cudaError_t e = ensure_dynamic_smem<5000 + kD * 8 + kRows * 4 + kPaged * 2 + kMod>(kern, Smem<kD, kRows>::kBytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Smem<kD, kRows>::kBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

template <bool kMod>
static cudaError_t launch_rows(const Params& p, bool paged, int d, int rows, const samkv_ctx_impl& h, cudaStream_t stream) {
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  char* ws = h.workspace + kStatusBytes;
#define SAMKV_F32_CASE(D, R) (paged ? launch<D, R, true, kMod>(p, ctas, ws, stream) : launch<D, R, false, kMod>(p, ctas, ws, stream))
  if (d == 128) return rows == 8 ? SAMKV_F32_CASE(128, 8) : rows == 32 ? SAMKV_F32_CASE(128, 32) : SAMKV_F32_CASE(128, 64);
  return rows == 8 ? SAMKV_F32_CASE(64, 8) : rows == 32 ? SAMKV_F32_CASE(64, 32) : SAMKV_F32_CASE(64, 64);
#undef SAMKV_F32_CASE
}

inline Params make_params(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale, const Rows& O,
                          float* lse, int rows, const samkv_ctx_impl& h) {
  Params p = {};
  p.seqs = seqs;
  p.cfg.G = d.n_q_heads / d.n_kv_heads;
  p.cfg.Hkv = d.n_kv_heads;
  p.cfg.tile = kBN;
  p.cfg.fixed = (rows == 8 ? 3 : 2) * kBN;
  p.cfg.min_chunk = 4 * kBN;
  p.pages = kv.pages;
  p.Q = Q;
  p.O = O;
  p.K = kv.K;
  p.V = kv.V;
  if (kv.paged) {
    p.K.data = kv.pages.K;
    p.V.data = kv.pages.V;
  }
  p.scale = scale;
  p.lse = lse;
  p.d_status = h.d_status;
  p.Hq = d.n_q_heads;
  return p;
}
}  // namespace pf32

}  // namespace samkv
