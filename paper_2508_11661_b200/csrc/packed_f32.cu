// Attention of packed sequences over packed rows or over a paged cache, fp32 throughout (tensor cores would round the
// operands to tf32).
//
// Persistent, one CTA of 256 threads per SM, work divided by packed_plan.cuh.  Row tiles of 64, 32 or 16 packed rows
// (launch_packed_attn chooses), key tiles of 64 slots, two to four of them in shared memory with cp.async.  With 64 and 32
// rows a thread owns kRows/16 rows x 4 slots of the scores and the same rows x d/16 columns of the result: per 64
// multiply-adds of the score product it reads 4 + 4 vectors of 16 bytes, so the FMA pipe and shared memory are about level.
// With 16 rows it keeps that ratio by splitting the head dimension, and the slots, between threads.  The 16 threads of a
// row agree on maxima and sums by shuffles.
// Bound by instruction issue at 64 rows (61 % of the slots; 4 sequences of 1024 tokens, 8/2 heads of 128: 27 TFLOP/s of the
// FMA pipe's nominal 74), by latency where there is little work: 4 documents of 256 tokens, 4/2 heads of 64, 21 us.
#include <math.h>

#include "packed_plan.cuh"

namespace samkv {
namespace pf32 {

constexpr int kBN = 64, kThreads = 256;

template <int kD, int kRows>
struct Smem {
  static constexpr int kLd = kD + 4;                     // row stride in floats: rows 16 bytes apart in their banks
  static constexpr int kPLd = kBN + 4;
  static constexpr int kTile = kBN * kLd * 4;
  static constexpr int kQ = 0;
  static constexpr int kKv = kRows * kLd * 4;            // [kStages][K, V]; P takes K's place once the scores are done
  // tiles in shared memory: as many as fit, since a short tile is done before the next one has come
  static constexpr int kStages = kD == 64 ? 4 : kRows == 64 ? 2 : 3;
  static constexpr int kP = kKv + kStages * 2 * kTile;             // 16-row tiles: scores and weights, rescaling factors
  static constexpr int kPiece = kP + (kRows == 16 ? 16 * kPLd * 4 + 64 : 0);
  static constexpr int kBytes = kPiece + 128;
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
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  const int sz = valid ? 16 : 0;                         // 0: the 16 bytes are zero-filled
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(sz) : "memory");
}
__device__ __forceinline__ float4 lds4(const float* p) { return *reinterpret_cast<const float4*>(p); }
}  // namespace pf32

template <int kD, int kRows, bool kPaged>
__global__ void __launch_bounds__(pf32::kThreads, 1)
packed_f32_kernel(const __grid_constant__ pf32::Params p) {
  using namespace pf32;
  using L = Smem<kD, kRows>;
  constexpr int kR = kRows / 16;                         // rows per thread
  constexpr int kC = kD / 64;                            // result columns per thread: kC vectors of 4
  constexpr int kLd = L::kLd, kPLd = L::kPLd;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float* sQ = reinterpret_cast<float*>(smem_raw + L::kQ);
  auto sK = [&](int st) { return reinterpret_cast<float*>(smem_raw + L::kKv + st * 2 * L::kTile); };
  auto sV = [&](int st) { return reinterpret_cast<float*>(smem_raw + L::kKv + st * 2 * L::kTile + L::kTile); };
  Piece* s_piece = reinterpret_cast<Piece*>(smem_raw + L::kPiece);
  volatile int* s_flag = reinterpret_cast<volatile int*>(smem_raw + L::kPiece + 96);
  PlanShared& plan = *reinterpret_cast<PlanShared*>(smem_raw + L::kKv);
  const int tid = threadIdx.x, warp = tid >> 5;
  const int ty = tid >> 4, tx = tid & 15;                // rows ty * kR + i, slots tx + 16 j, columns tx * 4 + 64 c
  const int G = p.cfg.G;
  pdl_wait();
  long long chunk = 0;
  const bool warp_plans = p.seqs.n_seq <= kWarpPlanSeqs;
  if (!warp_plans) plan_block<kThreads>(p.seqs, p.cfg, &plan, &chunk, p.d_status, tid);
  Walker w;
  w.more = false;
  if (warp == 0) {
    if (warp_plans) plan_block<32>(p.seqs, p.cfg, &plan, &chunk, p.d_status, tid);
    w.init(p.seqs, p.cfg, &plan, chunk);
  }
  bool bad = false;

  while (true) {
    __syncthreads();                                     // everybody is done with the previous piece (and the plan)
    if (warp == 0) {
      Piece next;
      const bool have = w.next(p.seqs, p.cfg, &next);
      if (!have) next.tile0 = -1;
      if (tid == 0) *s_piece = next;
    }
    __syncthreads();
    const Piece pc = *s_piece;
    if (pc.tile0 < 0) break;
    const int n_rows = min(p.cfg.tokens, pc.n - pc.r * p.cfg.tokens) * G;
    const int tok0 = pc.first + pc.r * p.cfg.tokens;
    const uint32_t smem = (uint32_t)__cvta_generic_to_shared(smem_raw);
    auto load_kv = [&](int t, int st) {
      const int j0 = t * kBN;
      const uint32_t dk = smem + L::kKv + st * 2 * L::kTile, dv = dk + L::kTile;
      // a thread keeps its 16-byte column and steps through the rows
      constexpr int kLanes = kD / 4, kStep = kThreads / kLanes;
      const int c = tid % kLanes, r0 = tid / kLanes;
#pragma unroll 4
      for (int r = r0; r < kBN; r += kStep) {
        const bool ok = j0 + r < pc.seen;                // slots that no row sees read as zero
        size_t ko = 0, vo = 0;
        if (ok) {
          if constexpr (kPaged) {
            ko = vo = page_offset(p.pages, pc.s, j0 + r, pc.h, p.cfg.Hkv, kD, &bad) + c * 4;
          } else {
            ko = (size_t)(pc.first + j0 + r) * p.K.ts + (size_t)pc.h * p.K.hs + c * 4;
            vo = (size_t)(pc.first + j0 + r) * p.V.ts + (size_t)pc.h * p.V.hs + c * 4;
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
      const size_t off = ok ? (size_t)(tok0 + r / G) * p.Q.ts + (size_t)(pc.h * G + r % G) * p.Q.hs + c * 4 : 0;
      cp_async16(smem + L::kQ + (r * kLd + c * 4) * 4, static_cast<const float*>(p.Q.data) + off, ok);
    }
    // (the last stage is filled from the loop on)
#pragma unroll 1
    for (int i = 0; i < L::kStages - 1; ++i) {
      if (pc.tile0 + i < pc.tile1) load_kv(pc.tile0 + i, i);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    Seq sq;
    sq.first = pc.first; sq.n = pc.n; sq.base = pc.base;
    const int last_tok = min((pc.r + 1) * p.cfg.tokens, pc.n) - 1;
    int vis[kR];
    float m[kR], l[kR], o[kR][kC * 4];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      vis[i] = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + (ty * kR + i) / G, last_tok));
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < kC * 4; ++c) o[i][c] = 0.f;
    }
    if constexpr (kRows == 16) {
      // Few rows: a thread owns 4 rows x 4 slots over a quarter of the head dimension, then 4 rows x 4 columns over half
      // (d = 128) or a quarter (d = 64) of the slots, so that it still has 64 multiply-adds for 8 vectors read; the scores
      // pass through shared memory in between.
      const int lane = tid & 31, rg = (warp & 3) * 4;
      const int ds = lane & 3, kg = (warp >> 2) * 8 + (lane >> 2);
      constexpr int kColLanes = kD / 4, kSplits = 256 / (4 * kColLanes);
      const int c4 = (lane & (kColLanes - 1)) * 4, split = (warp >> 2) * (32 / kColLanes) + lane / kColLanes;
      float* sP = reinterpret_cast<float*>(smem_raw + L::kP);
      float* sCorr = sP + 16 * kPLd;
      const int my_vis = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + (rg + ds) / G, last_tok));
      int row_vis[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) row_vis[i] = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + (rg + i) / G, last_tok));
      float acc[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll 1
      for (int t = pc.tile0; t < pc.tile1; ++t) {
        const int st = (t - pc.tile0) % L::kStages, j0 = t * kBN;
        asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
        __syncthreads();                                 // tile t is there, and tile t - 1 is used up
        if (t + L::kStages - 1 < pc.tile1) load_kv(t + L::kStages - 1, (t - pc.tile0 + L::kStages - 1) % L::kStages);
        asm volatile("cp.async.commit_group;" ::: "memory");
        // ---- scores ----
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
        const float *k = sK(st) + kg * kLd + ds * 4, *q = sQ + rg * kLd + ds * 4;
#pragma unroll 2
        for (int e = 0; e < kD; e += 16) {
          float4 kv[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) kv[j] = lds4(k + j * 16 * kLd + e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 a = lds4(q + i * kLd + e);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              s[i][j] = fmaf(a.x, kv[j].x, s[i][j]);
              s[i][j] = fmaf(a.y, kv[j].y, s[i][j]);
              s[i][j] = fmaf(a.z, kv[j].z, s[i][j]);
              s[i][j] = fmaf(a.w, kv[j].w, s[i][j]);
            }
          }
        }
        // the quarters are added up; lane ds keeps row rg + ds
        const bool hi = ds & 2, lo = ds & 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float a = (hi ? s[2][j] : s[0][j]) + __shfl_xor_sync(0xffffffffu, hi ? s[0][j] : s[2][j], 2);
          const float b = (hi ? s[3][j] : s[1][j]) + __shfl_xor_sync(0xffffffffu, hi ? s[1][j] : s[3][j], 2);
          const float x = (lo ? b : a) + __shfl_xor_sync(0xffffffffu, lo ? a : b, 1);
          sP[(rg + ds) * kPLd + kg + 16 * j] = j0 + kg + 16 * j < my_vis ? x * p.scale : -INFINITY;
        }
        __syncthreads();
        // ---- online softmax: 16 threads per row ----
        {
          float x[4], mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = sP[ty * kPLd + tx + 16 * j];
            mx = fmaxf(mx, x[j]);
          }
#pragma unroll
          for (int o2 = 8; o2 > 0; o2 >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o2));
          const float mn = fmaxf(m[0], mx), mu = mn == -INFINITY ? 0.f : mn;
          const float corr = m[0] == mn ? 1.f : expf(m[0] - mu);
          m[0] = mn;
          l[0] *= corr;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = expf(x[j] - mu);
            l[0] += x[j];                                // (this thread's slots; joined at the end)
            sP[ty * kPLd + tx + 16 * j] = x[j];
          }
          if (tx == 0) sCorr[ty] = corr;
        }
        __syncthreads();
        // ---- result ----
        const bool edge = j0 + kBN > pc.seen0;           // some row does not see some slot: zero weights times what it holds
        constexpr int kSlots = kBN / kSplits;
        const float *v = sV(st) + split * kSlots * kLd + c4, *pr = sP + rg * kPLd + split * kSlots;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float corr = sCorr[rg + i];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[i][c] *= corr;
        }
        if (!edge) {
#pragma unroll 2
          for (int j = 0; j < kSlots; j += 4) {
            float4 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = lds4(pr + i * kPLd + j);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const float4 b = lds4(v + (j + u) * kLd);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float w2 = u == 0 ? a[i].x : u == 1 ? a[i].y : u == 2 ? a[i].z : a[i].w;
                acc[i][0] = fmaf(w2, b.x, acc[i][0]);
                acc[i][1] = fmaf(w2, b.y, acc[i][1]);
                acc[i][2] = fmaf(w2, b.z, acc[i][2]);
                acc[i][3] = fmaf(w2, b.w, acc[i][3]);
              }
            }
          }
        } else {
#pragma unroll 1
          for (int j = 0; j < kSlots; ++j) {
            const float4 b = lds4(v + j * kLd);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float w2 = pr[i * kPLd + j];
              if (j0 + split * kSlots + j < row_vis[i]) {
                acc[i][0] = fmaf(w2, b.x, acc[i][0]);
                acc[i][1] = fmaf(w2, b.y, acc[i][1]);
                acc[i][2] = fmaf(w2, b.z, acc[i][2]);
                acc[i][3] = fmaf(w2, b.w, acc[i][3]);
              }
            }
          }
        }
      }
      // the splits' parts through shared memory into the layout below
      __syncthreads();
      float* part = sK(0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(part + (split * 16 + rg + i) * kD + c4) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
      __syncthreads();
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int x = 0; x < kSplits; ++x) {
          const float4 y = lds4(part + (x * 16 + ty) * kD + c * 64 + tx * 4);
          o[0][c * 4] += y.x;
          o[0][c * 4 + 1] += y.y;
          o[0][c * 4 + 2] += y.z;
          o[0][c * 4 + 3] += y.w;
        }
    } else {
#pragma unroll 1
    for (int t = pc.tile0; t < pc.tile1; ++t) {
      const int st = (t - pc.tile0) % L::kStages, j0 = t * kBN;
      asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
      __syncthreads();                                   // tile t is there, and tile t - 1 is used up
      if (t + L::kStages - 1 < pc.tile1) load_kv(t + L::kStages - 1, (t - pc.tile0 + L::kStages - 1) % L::kStages);
      asm volatile("cp.async.commit_group;" ::: "memory");
      // ---- scores ----
      float s[kR][4];
#pragma unroll
      for (int i = 0; i < kR; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
      const float *k = sK(st) + tx * kLd, *q = sQ + ty * kR * kLd;
#pragma unroll 4
      for (int e = 0; e < kD; e += 4) {
        float4 kv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = lds4(k + j * 16 * kLd + e);
#pragma unroll
        for (int i = 0; i < kR; ++i) {
          const float4 a = lds4(q + i * kLd + e);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(a.x, kv[j].x, s[i][j]);
            s[i][j] = fmaf(a.y, kv[j].y, s[i][j]);
            s[i][j] = fmaf(a.z, kv[j].z, s[i][j]);
            s[i][j] = fmaf(a.w, kv[j].w, s[i][j]);
          }
        }
      }
      // ---- online softmax ----
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] = j0 + tx + 16 * j < vis[i] ? s[i][j] * p.scale : -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int x = 8; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
        const float mn = fmaxf(m[i], mx), mu = mn == -INFINITY ? 0.f : mn;
        const float corr = m[i] == mn ? 1.f : expf(m[i] - mu);
        m[i] = mn;
        l[i] *= corr;
#pragma unroll
        for (int c = 0; c < kC * 4; ++c) o[i][c] *= corr;
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
      const bool edge = j0 + kBN > pc.seen0;             // some row does not see some slot: zero weights times what it holds
#pragma unroll 2
      for (int j = 0; j < kBN; j += 4) {
        float4 a[kR];
#pragma unroll
        for (int i = 0; i < kR; ++i) a[i] = lds4(pr + i * kPLd + j);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float4 b[kC];
#pragma unroll
          for (int c = 0; c < kC; ++c) b[c] = lds4(v + (j + u) * kLd + c * 64);
#pragma unroll
          for (int i = 0; i < kR; ++i) {
            const float w = u == 0 ? a[i].x : u == 1 ? a[i].y : u == 2 ? a[i].z : a[i].w;
            if (!edge || j0 + j + u < vis[i]) {
#pragma unroll
              for (int c = 0; c < kC; ++c) {
                o[i][c * 4] = fmaf(w, b[c].x, o[i][c * 4]);
                o[i][c * 4 + 1] = fmaf(w, b[c].y, o[i][c * 4 + 1]);
                o[i][c * 4 + 2] = fmaf(w, b[c].z, o[i][c * 4 + 2]);
                o[i][c * 4 + 3] = fmaf(w, b[c].w, o[i][c * 4 + 3]);
              }
            }
          }
        }
      }
    }
    }
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    auto write_row = [&](int i, const float* acc, float M, float Ls) {
      const int row = ty * kR + i;
      if (row >= n_rows) return;
      const int tok = tok0 + row / G, hq = pc.h * G + row % G;
      const float inv = 1.0f / Ls;
      float* op = static_cast<float*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs + tx * 4;
#pragma unroll
      for (int c = 0; c < kC; ++c)
        *reinterpret_cast<float4*>(op + c * 64) =
            Ls == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                      : make_float4(acc[c * 4] * inv, acc[c * 4 + 1] * inv, acc[c * 4 + 2] * inv, acc[c * 4 + 3] * inv);
      if (tx == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = Ls == 0.f ? -INFINITY : M + logf(Ls);
    };
    if (pc.slot < 0) {
#pragma unroll
      for (int i = 0; i < kR; ++i) write_row(i, o[i], m[i], l[i]);
      continue;
    }
    // a piece of a cut item leaves (m, l, O); whoever takes the last ticket merges them in order of the pieces
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const size_t row = (size_t)pc.slot * kRows + ty * kR + i;
#pragma unroll
      for (int c = 0; c < kC; ++c)
        *reinterpret_cast<float4*>(p.part_o + row * kD + c * 64 + tx * 4) =
            make_float4(o[i][c * 4], o[i][c * 4 + 1], o[i][c * 4 + 2], o[i][c * 4 + 3]);
      if (tx == 0) p.part_ml[row] = make_float2(m[i], l[i]);
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) *s_flag = last_piece(p.d_status, pc.ticket, pc.n_pieces);
    __syncthreads();
    if (*s_flag) {
      __threadfence();
#pragma unroll 1
      for (int i = 0; i < kR; ++i) {
        const int row = ty * kR + i;
        if (row >= n_rows) continue;
        float M = -INFINITY, Ls = 0.f, acc[kC * 4];
#pragma unroll
        for (int c = 0; c < kC * 4; ++c) acc[c] = 0.f;
#pragma unroll 4
        for (int n = 0; n < pc.n_pieces; ++n) {
          const float2 x = __ldcg(p.part_ml + piece_slot(pc, n) * kRows + row);
          if (x.y != 0.f) M = fmaxf(M, x.x);
        }
#pragma unroll 4
        for (int n = 0; n < pc.n_pieces; ++n) {
          const size_t at = (size_t)piece_slot(pc, n) * kRows + row;
          const float2 x = __ldcg(p.part_ml + at);
          const float wgt = x.y == 0.f ? 0.f : expf(x.x - M);
#pragma unroll
          for (int c = 0; c < kC; ++c) {
            const float4 v4 = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kD + c * 64 + tx * 4));
            if (x.y != 0.f) {
              acc[c * 4] = fmaf(v4.x, wgt, acc[c * 4]);
              acc[c * 4 + 1] = fmaf(v4.y, wgt, acc[c * 4 + 1]);
              acc[c * 4 + 2] = fmaf(v4.z, wgt, acc[c * 4 + 2]);
              acc[c * 4 + 3] = fmaf(v4.w, wgt, acc[c * 4 + 3]);
            }
          }
          if (x.y != 0.f) Ls += x.y * wgt;
        }
        write_row(i, acc, M, Ls);
      }
    }
  }
  if (bad) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
  pdl_launch_dependents();
}

size_t packed_f32_scratch_bytes(int d) { return (size_t)2 * kMaxPackedCtas * 64 * ((size_t)d * 4 + 8); }

namespace pf32 {
template <int kD, int kRows, bool kPaged>
static cudaError_t launch(Params p, int ctas, char* ws, cudaStream_t stream) {
  p.cfg.tokens = kRows / p.cfg.G;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)2 * ctas * kRows * kD * 4);
  auto kern = packed_f32_kernel<kD, kRows, kPaged>;
  cudaError_t e = ensure_dynamic_smem<5000 + kD * 4 + kRows * 2 + kPaged>(kern, Smem<kD, kRows>::kBytes);
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
}  // namespace pf32

cudaError_t launch_packed_f32(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                              const Rows& O, float* lse, int rows, const samkv_ctx_impl& h, cudaStream_t stream) {
  pf32::Params p = {};
  p.seqs = seqs;
  p.cfg.G = d.n_q_heads / d.n_kv_heads;
  p.cfg.Hkv = d.n_kv_heads;
  p.cfg.tile = pf32::kBN;
  p.cfg.fixed = 2 * pf32::kBN;
  p.cfg.min_chunk = 4 * pf32::kBN;
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
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  char* ws = h.workspace + kStatusBytes;
#define SAMKV_F32_CASE(D, R) (kv.paged ? pf32::launch<D, R, true>(p, ctas, ws, stream) : pf32::launch<D, R, false>(p, ctas, ws, stream))
  if (d.head_dim == 128)
    return rows == 16 ? SAMKV_F32_CASE(128, 16) : rows == 32 ? SAMKV_F32_CASE(128, 32) : SAMKV_F32_CASE(128, 64);
  return rows == 16 ? SAMKV_F32_CASE(64, 16) : rows == 32 ? SAMKV_F32_CASE(64, 32) : SAMKV_F32_CASE(64, 64);
#undef SAMKV_F32_CASE
}

}  // namespace samkv
