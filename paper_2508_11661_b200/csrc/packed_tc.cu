// tcgen05 attention of packed sequences over packed rows or over a paged cache; bf16, head dimension 64 or 128.
//
// Persistent, one CTA per SM.  An item is a tile of up to 128 query rows (row = token x group member, so the G query
// heads that share a KV head share its keys) against key tiles of 128 slots; packed_plan.cuh divides the call's items
// evenly among the CTAs.  Roles of the 12 warps:
//   warps 0-3   softmax of the even key tiles of the CTA's running count, thread = row
//   warps 4-7   softmax of the odd ones
//   warp 8      issues S(T) = Q K(T)^T into the score buffer T & 1
//   warp 9      issues O += P(T) V(T)
//   warp 10     walks the plan, loads Q (two buffers) and K (three stages) by TMA
//   warp 11     loads V (two stages), clears value rows behind a sequence's last slot
// Both groups add into ONE accumulator: they use a common reference maximum per row, kept in shared memory and handed
// from tile to tile in order (tile T + 1 reads it after tile T has decided).  The reference only has to be within a factor
// of 2^64 of the row's maximum (P is bf16 and O, l are fp32: all have the exponent range for it), so after a row's first
// tile it practically never moves; when it does, the group waits for the products in flight and rescales O in tensor
// memory.  That frees tensor memory for P buffers of their own (S0 S1 128 columns each, O 128, P0 P1 64 each: all 512),
// so S(T+2) is issued as soon as S(T) sits in registers and never waits for the exponentials of T: score product,
// exponentials and value product of different tiles overlap without a chain between them.
// Probabilities are rounded to bf16 on the integer pipe (round half away, one byte permute per pair); the denominator
// sums them before that rounding, so lse is good to fp32.
// Every wait is bounded; a wait that runs out sets a flag that ends all others, the CTA drains its copies and frees its
// tensor memory, and the failure is recorded as a device check.  TMA reads this GPU's memory only, without multicast.
#include "packed_plan.cuh"
#include "tc_common.cuh"

namespace samkv {
namespace ptc {
using namespace tc;

constexpr int kBM = 128, kBN = 128;
constexpr int kKStages = 3, kVStages = 2, kQStages = 2, kRing = 4;
constexpr int kThreads = 384;
constexpr int kRegsSoftmax = 216, kRegsOther = 72;     // 256 x 216 + 128 x 72 = 384 x 168, the launch's registers
constexpr float kGrow = 64.0f;                         // log2
constexpr uint32_t kTmemCols = 512, kColO = 256, kColP = 384;

template <int kD>
struct Smem {
  static constexpr int kTile = 128 * kD * 2;           // a Q, K or V tile
  static constexpr int kQ = 0;
  static constexpr int kK = kQ + kQStages * kTile;
  static constexpr int kV = kK + kKStages * kTile;
  static constexpr int kRef = kV + kVStages * kTile;   // reference maxima, 128 fp32
  static constexpr int kSum = kRef + 512;              // denominators of both groups, [2][128] fp32
  static constexpr int kPieces = kSum + 1024;          // kRing descriptors
  static constexpr int kCur = kPieces + kRing * 64;    // the softmax warps' copy
  static constexpr int kBar = kCur + 64;
  static constexpr int kMisc = kBar + 256;             // tensor memory address, failure flag, "merge" flag
  static constexpr int kBytes = kMisc + 64;
};
static_assert(sizeof(Piece) <= 64, "descriptor size");
static_assert(Smem<128>::kBytes <= 232448, "shared memory of one CTA");

enum Bar {
  FR_FULL = 0, FR_FREE = FR_FULL + kRing, Q_FULL = FR_FREE + kRing, Q_FREE = Q_FULL + kQStages, K_FULL = Q_FREE + kQStages,
  K_FREE = K_FULL + kKStages, V_FULL = K_FREE + kKStages, V_TMA = V_FULL + kVStages, S_FULL = V_TMA + 1, S_FREE = S_FULL + 2,
  P_READY = S_FREE + 2, PV_DONE = P_READY + 2, O_FREE = PV_DONE + 2, kBars = O_FREE + 1
};
static_assert(kBars * 8 <= 256, "barrier area");

__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// maximum that keeps NaN
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// two probabilities -> packed bf16, rounded to nearest (ties away); inputs are non-negative and finite or NaN (a row
// with a NaN is recognised by its maximum)
__device__ __forceinline__ uint32_t round_pair(float lo, float hi) {
  uint32_t r;
  asm("prmt.b32 %0, %1, %2, 0x7632;" : "=r"(r) : "r"(__float_as_uint(lo) + 0x8000u), "r"(__float_as_uint(hi) + 0x8000u));
  return r;
}

__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// Bounded; gives up as soon as another role has failed.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile uint32_t* fail) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (try_wait(bar, parity)) return true;
    if (*fail) return false;
  }
  *fail = 1;
  return false;
}
// For copies in flight at the end: bounded, whatever has failed.
__device__ __forceinline__ void drain_bar(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kSpinLimit; ++i)
    if (try_wait(bar, parity)) return;
}

struct Params {
  Seqs seqs;
  SplitCfg cfg;
  Pages pages;                 // table, width, n_pages, shift; paged calls
  Rows Q, K, V, O;             // K, V: packed rows, or the pools' data pointers
  int paged, box;              // slots per TMA box
  float scale;
  float* lse;
  float4* part_o;              // [slot][d/4][128]
  float2* part_ml;             // [slot][128]
  int* d_status;
  int Hq;
};

__device__ __forceinline__ const __nv_bfloat16* kv_row(const Params& p, const Rows& rows, const Piece& pc, int j, int kD) {
  const __nv_bfloat16* base = static_cast<const __nv_bfloat16*>(rows.data);
  if (p.paged) {
    bool bad = false;
    return base + page_offset(p.pages, pc.s, j, pc.h, p.cfg.Hkv, kD, &bad);
  }
  return base + (size_t)(pc.first + j) * rows.ts + (size_t)pc.h * rows.hs;
}

// Loads the boxes of one key or value tile; `pages` holds this tile's page numbers in the lanes.
template <int kD, bool kPaged>
__device__ __forceinline__ void load_tile(const Params& p, const CUtensorMap* map, const Piece& pc, int tile, uint32_t dst,
                                          uint32_t bar, int page) {
  const int lane = threadIdx.x & 31;
  const int j0 = tile * kBN;
  if constexpr (!kPaged) {
    if (lane == 0) {
      mbar_expect_tx(bar, Smem<kD>::kTile);
#pragma unroll
      for (int x = 0; x < kD; x += 64) tma_load_3d(dst + (x >> 6) * (kBN * 128), map, x, pc.first + j0, pc.h, bar);
    }
  } else {
    const int n_box = min(kBN / p.box, (pc.seen - j0 + p.box - 1) / p.box);     // boxes that no row sees stay unloaded
    if (lane == 0) mbar_expect_tx(bar, max(n_box, 0) * p.box * kD * 2);
    __syncwarp();
    if (lane < n_box) {
      const int row = (((page * p.cfg.Hkv) + pc.h) << p.pages.shift) + ((j0 + lane * p.box) & ((1 << p.pages.shift) - 1));
#pragma unroll
      for (int x = 0; x < kD; x += 64)
        tma_load_3d(dst + (x >> 6) * (kBN * 128) + lane * p.box * 128, map, x, row, 0, bar);
    }
  }
  __syncwarp();
}
// Page numbers of a tile, lane i: box i.  Entries of slots that no row sees are not read.
__device__ __forceinline__ int tile_page(const Params& p, const Piece& pc, int tile, bool* bad) {
  const int lane = threadIdx.x & 31;
  const int j = tile * kBN + lane * p.box;
  int page = 0;
  if (lane < kBN / p.box && j < pc.seen) {
    page = p.pages.table[(size_t)pc.s * p.pages.width + (j >> p.pages.shift)];
    if ((unsigned)page >= (unsigned)p.pages.n_pages) {
      page = 0;
      *bad = true;
    }
  }
  return page;
}
// Whether a value row of slots [j0, j1) holds an infinity or NaN (one warp, global memory).
template <int kD>
__device__ __forceinline__ bool any_nonfinite(const Params& p, const Piece& pc, int j0, int j1) {
  const int lane = threadIdx.x & 31;
  constexpr int kChunks = kD / 8;
  uint32_t hit = 0;
#pragma unroll 4
  for (int i = lane; i < (j1 - j0) * kChunks; i += 32) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(kv_row(p, p.V, pc, j0 + i / kChunks, kD)) + i % kChunks);
    // an exponent of all ones carries into the sign's place
    hit |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) |
           ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
  }
  return __any_sync(0xffffffffu, (hit & 0x80008000u) != 0);
}
}  // namespace ptc

template <int kD, bool kPaged>
__global__ void __launch_bounds__(ptc::kThreads, 1)
packed_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ ptc::Params p) {
  using namespace ptc;
  using L = Smem<kD>;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const uint32_t sBar = base + L::kBar;
  auto bar = [&](int i) { return sBar + 8u * i; };
  PlanShared& plan = *reinterpret_cast<PlanShared*>(smem_raw + L::kK);   // read by the K loader before its first copy
  float* ref_max = reinterpret_cast<float*>(smem_raw + L::kRef);
  volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem_raw + L::kMisc);
  volatile uint32_t* s_fail = s_tmem + 1;
  volatile uint32_t* s_merge = s_tmem + 2;
  volatile uint32_t* s_scrub = s_tmem + 4;   // per ring entry
  float* sums = reinterpret_cast<float*>(smem_raw + L::kSum);
  Piece* ring = reinterpret_cast<Piece*>(smem_raw + L::kPieces);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.cfg.G;

  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) { mbar_init(bar(FR_FULL + i), 1); mbar_init(bar(FR_FREE + i), 4); }
    for (int i = 0; i < kQStages; ++i) { mbar_init(bar(Q_FULL + i), 1); mbar_init(bar(Q_FREE + i), 1); }
    for (int i = 0; i < kKStages; ++i) { mbar_init(bar(K_FULL + i), 1); mbar_init(bar(K_FREE + i), 1); }
    for (int i = 0; i < kVStages; ++i) mbar_init(bar(V_FULL + i), 1);
    mbar_init(bar(V_TMA), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(S_FULL + i), 1);
      mbar_init(bar(S_FREE + i), 4);
      mbar_init(bar(P_READY + i), 4);
      mbar_init(bar(PV_DONE + i), 1);
    }
    mbar_init(bar(O_FREE), 8);
    *s_fail = (base & 1023u) != 0;          // (never seen: the declaration asks for 1024 bytes)
    if (*s_fail) atomicMax(p.d_status, (int)CHECK_SMEM_ALIGNMENT);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(base + L::kMisc), "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  pdl_wait();                               // everything below reads what earlier kernels may have written
  long long chunk = 0;
  plan_block<kThreads>(p.seqs, p.cfg, &plan, &chunk, p.d_status);

  auto wait = [&](int i, uint32_t phase) { return wait_bar(bar(i), phase & 1u, s_fail); };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 10) {
      // ================= plan, Q and K =================
      Walker w;
      w.init(p.seqs, p.cfg, &plan, chunk);
      Piece pc;
      uint32_t f = 0, T = 0;                // pieces, key tiles so far
      bool bad = false;
      while (true) {
        const bool have = *s_fail == 0 && w.next(p.seqs, p.cfg, &pc);
        if (f >= kRing) wait(FR_FREE + f % kRing, f / kRing - 1);
        if (lane == 0) {
          if (!have) pc.tile0 = -1;
          ring[f % kRing] = pc;
          mbar_arrive(bar(FR_FULL + f % kRing));
        }
        __syncwarp();
        if (!have) break;
        int page = 0;
        if constexpr (kPaged) page = tile_page(p, pc, pc.tile0, &bad);
        if (f >= kQStages) wait(Q_FREE + f % kQStages, f / kQStages - 1);
        if (lane == 0) {
          const uint32_t q = bar(Q_FULL + f % kQStages), dst = base + L::kQ + (f % kQStages) * L::kTile;
          mbar_expect_tx(q, p.cfg.tokens * G * kD * 2);
#pragma unroll
          for (int x = 0; x < kD; x += 64)
            tma_load_3d(dst + (x >> 6) * (kBM * 128), &tmQ, x, pc.h * G, pc.first + pc.r * p.cfg.tokens, q);
        }
        __syncwarp();
        for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
          int next = 0;
          if constexpr (kPaged) { if (t + 1 < pc.tile1) next = tile_page(p, pc, t + 1, &bad); }
          const uint32_t st = T % kKStages;
          if (T >= kKStages) wait(K_FREE + st, T / kKStages - 1);
          load_tile<kD, kPaged>(p, &tmK, pc, t, base + L::kK + st * L::kTile, bar(K_FULL + st), page);
          page = next;
        }
        ++f;
      }
      if (__any_sync(0xffffffffu, bad) && lane == 0) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
      for (uint32_t i = 0; i < kKStages; ++i)                     // no copy of this CTA outlives it
        if (T > i) drain_bar(bar(K_FULL + (T - 1 - i) % kKStages), ((T - 1 - i) / kKStages) & 1u);
      for (uint32_t i = 0; i < kQStages; ++i)
        if (f > i) drain_bar(bar(Q_FULL + (f - 1 - i) % kQStages), ((f - 1 - i) / kQStages) & 1u);
    } else {
      // warps 8, 9, 11 follow the ring of pieces
      uint32_t f = 0, T = 0, partial_tiles = 0;
      while (true) {
        if (!wait(FR_FULL + f % kRing, f / kRing)) break;
        const Piece pc = ring[f % kRing];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
        if (pc.tile0 < 0) break;
        if (warp == 8) {
          // ================= S = Q K^T =================
          constexpr uint32_t kIdesc = instr_desc(kBM, kBN, false);
          const uint64_t dQ = smem_desc(base + L::kQ + (f % kQStages) * L::kTile, 16, 1024);
          wait(Q_FULL + f % kQStages, f / kQStages);
          for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
            const uint32_t st = T % kKStages, g = T & 1u;
            wait(K_FULL + st, T / kKStages);
            if (T >= 2) wait(S_FREE + g, (T >> 1) - 1);
            tc_fence_after();
            if (lane == 0) {
              const uint64_t dK = smem_desc(base + L::kK, 16, 1024) + (uint64_t)(st * (L::kTile >> 4));
#pragma unroll
              for (int ks = 0; ks < kD / 16; ++ks) {
                const uint32_t aoff = ((ks >> 2) * (kBM * 128) + (ks & 3) * 32) >> 4;
                const uint32_t boff = ((ks >> 2) * (kBN * 128) + (ks & 3) * 32) >> 4;
                mma_ss(tmem + g * kBN, dQ + aoff, dK + boff, kIdesc, ks > 0);
              }
              mma_commit(bar(S_FULL + g));
              mma_commit(bar(K_FREE + st));
              if (t + 1 == pc.tile1) mma_commit(bar(Q_FREE + f % kQStages));
            }
            __syncwarp();
          }
        } else if (warp == 9) {
          // ================= O += P V =================
          constexpr uint32_t kIdesc = instr_desc(kBM, kD, true);
          for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
            const uint32_t g = T & 1u;
            wait(V_FULL + g, T >> 1);
            if (t == pc.tile0 && f > 0) wait(O_FREE, f - 1);
            wait(P_READY + g, T >> 1);
            tc_fence_after();
            if (lane == 0) {
              const uint64_t dV = smem_desc(base + L::kV, kBN * 128, 1024) + (uint64_t)(g * (L::kTile >> 4));
              const int slots = pc.seen - t * kBN;                 // steps of 16 slots that some row sees
#pragma unroll
              for (int ks = 0; ks < kBN / 16; ++ks)
                if (ks == 0 || ks * 16 < slots) mma_ts(tmem + kColO, tmem + kColP + g * 64 + ks * 8, dV + ((ks * 16 * 128) >> 4), kIdesc,
                       (t > pc.tile0) | (ks > 0));
              mma_commit(bar(PV_DONE + g));
            }
            __syncwarp();
          }
        } else {
          // ================= V =================
          // Of the slots that only some rows of the tile see, infinities and NaN must not meet the zero weights of the
          // others: they are looked for ahead of time (L2 reads of at most 127 rows), and in the rare case that there are
          // any they are cleared in shared memory and added back, row by row, when the result is written.
          int page = 0;
          bool bad = false;                                        // (reported by the K loader)
          if constexpr (kPaged) page = tile_page(p, pc, pc.tile0, &bad);
          bool scrub = false;
          const int zone0 = max(pc.seen0, pc.tile0 * kBN), zone1 = min(pc.seen, pc.tile1 * kBN);
          const int scan_at = max(pc.tile0, zone0 / kBN - 1);
          if (lane == 0) s_scrub[f % kRing] = 0;
          __syncwarp();
          for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
            int next = 0;
            if constexpr (kPaged) { if (t + 1 < pc.tile1) next = tile_page(p, pc, t + 1, &bad); }
            if (t == scan_at && zone0 < zone1) {
              scrub = any_nonfinite<kD>(p, pc, zone0, zone1);
              if (scrub && lane == 0) s_scrub[f % kRing] = 1;
              __syncwarp();
            }
            const uint32_t g = T & 1u, dst = base + L::kV + g * L::kTile;
            if (T >= 2) wait(PV_DONE + g, (T >> 1) - 1);
            const int slots = pc.seen - t * kBN;                   // slots behind `seen` that a step of 16 still covers
            const bool clear = slots < kBN && (slots & 15) != 0 || slots <= 0;
            const bool wash = scrub && t * kBN + kBN > zone0;
            if (!clear && !wash) {
              load_tile<kD, kPaged>(p, &tmV, pc, t, dst, bar(V_FULL + g), page);
            } else {
              load_tile<kD, kPaged>(p, &tmV, pc, t, dst, bar(V_TMA), page);
              wait(V_TMA, partial_tiles++);
              if (clear) {
                const int first = max(slots, 0), end = max((first + 15) & ~15, 16);
                for (int i = lane; i < (end - first) * (kD / 8); i += 32) {
                  const int r = first + i / (kD / 8), c = i % (kD / 8);
                  asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(dst + (c >> 3) * (kBN * 128) + blk_off(r, c & 7)),
                               "r"(0) : "memory");
                }
              }
              if (wash) {
                const int r0 = max(zone0 - t * kBN, 0), r1 = min(zone1 - t * kBN, kBN);
                for (int i = lane; i < (r1 - r0) * (kD / 2); i += 32) {
                  const int r = r0 + i / (kD / 2), w = i % (kD / 2);
                  const uint32_t at = dst + (w >> 5) * (kBN * 128) + blk_off(r, (w >> 2) & 7) + (w & 3) * 4;
                  uint32_t v;
                  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
                  if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
                  if ((v & 0x7f800000u) == 0x7f800000u) v &= 0x0000ffffu;
                  asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
                }
              }
              fence_proxy_async();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(V_FULL + g));
              __syncwarp();
            }
            page = next;
          }
        }
        ++f;
      }
      if (warp == 11)
        for (uint32_t i = 0; i < kVStages; ++i)
          if (T > i) drain_bar(bar(V_FULL + (T - 1 - i) % kVStages), ((T - 1 - i) / kVStages) & 1u);
    }
  } else {
    // ================= softmax =================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int g = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t tS = lane_addr + g * kBN, tO = lane_addr + kColO, tP = lane_addr + kColP + g * 64;
    const float sl2 = p.scale * kLog2e;
    const uint64_t sl2_2 = pack2(sl2, sl2);
    const int t_local = row / G, member = row - t_local * G;
    auto bar_sync = [&](int id) { asm volatile("bar.sync %0, 256;" ::"r"(id) : "memory"); };
    uint32_t f = 0, T = 0;
    Piece* cur = reinterpret_cast<Piece*>(smem_raw + L::kCur);
    while (true) {
      if (tid == 0) {                                    // one decision for all eight warps
        const bool ok = wait(FR_FULL + f % kRing, f / kRing);
        *cur = ring[f % kRing];
        if (!ok) cur->tile0 = -1;
        mbar_arrive(bar(FR_FREE + f % kRing));
      }
      bar_sync(1);
      const Piece pc = *cur;
      if (pc.tile0 < 0) break;
      const int t_seq = pc.r * p.cfg.tokens + t_local;
      const bool valid = t_local < p.cfg.tokens && t_seq < pc.n;
      Seq sq;
      sq.first = pc.first; sq.n = pc.n; sq.base = pc.base;
      // rows without a token follow the last one: their results are dropped
      const int vis = visible(p.seqs, sq, min(t_seq, min((pc.r + 1) * p.cfg.tokens, pc.n) - 1));
      float m = -INFINITY, l = 0.f;
      bool poison = false;
      for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
        if ((T & 1u) != (uint32_t)g) continue;
        wait(S_FULL + g, T >> 1);
        tc_fence_after();
        float sv[kBN];
#pragma unroll
        for (int c0 = 0; c0 < kBN; c0 += 32) tmem_ld32_nowait(tS + c0, sv + c0);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(S_FREE + g));     // the next score product may overwrite the buffer
        const int limit = vis - t * kBN;
        if (__any_sync(0xffffffffu, limit < kBN)) {
#pragma unroll
          for (int i = 0; i < kBN; ++i)
            if (i >= limit) sv[i] = -INFINITY;
        }
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
        for (int i = 0; i < kBN; i += 8) {
          mx0 = max3_nan(mx0, sv[i], sv[i + 1]);
          mx1 = max3_nan(mx1, sv[i + 2], sv[i + 3]);
          mx2 = max3_nan(mx2, sv[i + 4], sv[i + 5]);
          mx3 = max3_nan(mx3, sv[i + 6], sv[i + 7]);
        }
        const float cand = max3_nan(max3_nan(mx0, mx1, mx2), mx3, mx3) * sl2;
        poison |= !(cand < INFINITY);                    // NaN or +infinity among the row's scores
        // the reference maximum, handed on from tile to tile
        float ref = -INFINITY;
        if (t > pc.tile0) {
          bar_sync(2 + g);
          ref = ref_max[row];
        }
        const bool grow = cand - ref > kGrow || (ref == -INFINITY && cand > -INFINITY);
        const float ref_new = grow ? cand : ref;
        if (grow || t == pc.tile0) ref_max[row] = ref_new;
        if (t + 1 < pc.tile1) asm volatile("bar.arrive %0, 256;" ::"r"(2 + (g ^ 1)) : "memory");
        if (m != ref_new) {                              // (also when the other group moved it)
          l = l > 0.f ? l * fast_exp2(m - ref_new) : l;
          m = ref_new;
        }
        if (T >= 2) wait(PV_DONE + g, (T >> 1) - 1);     // this group's P buffer is free
        if (t > pc.tile0 && __any_sync(0xffffffffu, grow)) {
          wait(PV_DONE + (g ^ 1), (T - 1) >> 1);         // O holds everything before this tile, at the old reference
          tc_fence_after();
          const float corr = grow ? fast_exp2(ref - ref_new) : 1.0f;
#pragma unroll 1
          for (int c0 = 0; c0 < kD; c0 += 32) {
            float o[32];
            tmem_ld32(tO + c0, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= corr;
            tmem_st32(tO + c0, o);
          }
        }
        const float mu = m == -INFINITY ? 0.f : m;
        const uint64_t negmu2 = pack2(-mu, -mu);
        uint64_t suma = pack2(0.f, 0.f), sumb = suma;
#pragma unroll
        for (int c0 = 0; c0 < kBN; c0 += 32) {
          if (c0 > 0 && c0 >= pc.seen - t * kBN) break;  // no row sees these slots: the value product skips them
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x0, x1;
            unpack2(fma2(pack2(sv[c0 + 2 * i], sv[c0 + 2 * i + 1]), sl2_2, negmu2), x0, x1);
            const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
            if (i & 1) sumb = add2(sumb, pack2(p0, p1)); else suma = add2(suma, pack2(p0, p1));
            pk[i] = round_pair(p0, p1);
          }
          tmem_st16(tP + (c0 >> 1), pk);
        }
        float a, b;
        unpack2(add2(suma, sumb), a, b);
        l += a + b;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(P_READY + g));
      }
      if (poison) l = __int_as_float(0x7fffffff);
      // ---- the piece's result: denominators of both groups, this group's half of the columns ----
      bar_sync(1);                                       // every tile has decided on the reference
      const float m_fin = ref_max[row];
      const float mu_fin = m_fin == -INFINITY ? 0.f : m_fin;
      if (l != 0.f) l *= fast_exp2(m - mu_fin);
      sums[g * 128 + row] = l;
      bar_sync(1);
      l += sums[(g ^ 1) * 128 + row];
      const uint32_t last = T - 1;
      wait(PV_DONE + (last & 1u), last >> 1);
      tc_fence_after();
      float o[kD / 2];
#pragma unroll
      for (int c0 = 0; c0 < kD / 2; c0 += 32) tmem_ld32_nowait(tO + g * (kD / 2) + c0, o + c0);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(O_FREE));
      const bool store = valid && *s_fail == 0;
      if (s_scrub[f % kRing] != 0 && store) {
        // infinities and NaN that were cleared from the value tile: back into the rows that see them
        for (int j = max(pc.seen0, pc.tile0 * kBN); j < min(vis, pc.tile1 * kBN); ++j) {
          const __nv_bfloat16* v = kv_row(p, p.V, pc, j, kD) + g * (kD / 2);
#pragma unroll
          for (int i = 0; i < kD / 2; ++i) {
            const float x = __bfloat162float(v[i]);
            if (!(fabsf(x) < INFINITY)) o[i] += x;
          }
        }
      }
      const int tok = pc.first + t_seq, hq = pc.h * G + member;
      if (pc.slot < 0) {
        if (store) {
          const float inv = l == 0.f ? 0.f : 1.0f / l;
          __nv_bfloat16* op = static_cast<__nv_bfloat16*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs + g * (kD / 2);
#pragma unroll
          for (int i = 0; i < kD / 2; i += 8) {
            uint4 v;
            v.x = pack_bf16(o[i] * inv, o[i + 1] * inv);
            v.y = pack_bf16(o[i + 2] * inv, o[i + 3] * inv);
            v.z = pack_bf16(o[i + 4] * inv, o[i + 5] * inv);
            v.w = pack_bf16(o[i + 6] * inv, o[i + 7] * inv);
            if (l == 0.f) v = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4*>(op + i) = v;
          }
          if (g == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = l == 0.f ? -INFINITY : m_fin * kLn2 + logf(l);
        }
      } else {
        // ---- a piece of a cut item: leave (m, l, O); whoever takes the last ticket merges in order of the pieces ----
        float4* po = p.part_o + ((size_t)pc.slot * (kD / 4) + g * (kD / 8)) * 128 + row;
#pragma unroll
        for (int i = 0; i < kD / 2; i += 4) po[(i >> 2) * 128] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        if (g == 0) p.part_ml[pc.slot * 128 + row] = make_float2(m_fin, l);
        __threadfence();
        bar_sync(1);
        if (tid == 0) *s_merge = last_piece(p.d_status, pc.ticket, pc.n_pieces);
        bar_sync(1);
        if (*s_merge) {
          __threadfence();
          float M = -INFINITY;
          for (int k = 0; k < pc.n_pieces; ++k) {
            const float2 x = __ldcg(p.part_ml + piece_slot(pc.ticket, k) * 128 + row);
            M = x.y == 0.f ? M : fmaxf(M, x.x);
          }
          const float Mu = M == -INFINITY ? 0.f : M;
          float Ls = 0.f;
#pragma unroll
          for (int i = 0; i < kD / 2; ++i) o[i] = 0.f;
          for (int k = 0; k < pc.n_pieces; ++k) {
            const int slot = piece_slot(pc.ticket, k);
            const float2 x = __ldcg(p.part_ml + slot * 128 + row);
            if (x.y == 0.f) continue;                    // a piece that saw nothing of this row
            const float w = fast_exp2(x.x - Mu);
            Ls += x.y * w;
            const float4* src = p.part_o + ((size_t)slot * (kD / 4) + g * (kD / 8)) * 128 + row;
#pragma unroll
            for (int i = 0; i < kD / 2; i += 4) {
              const float4 v = __ldcg(src + (i >> 2) * 128);
              o[i] = fmaf(v.x, w, o[i]);
              o[i + 1] = fmaf(v.y, w, o[i + 1]);
              o[i + 2] = fmaf(v.z, w, o[i + 2]);
              o[i + 3] = fmaf(v.w, w, o[i + 3]);
            }
          }
          if (store) {
            const float inv = Ls == 0.f ? 0.f : 1.0f / Ls;
            __nv_bfloat16* op = static_cast<__nv_bfloat16*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs + g * (kD / 2);
#pragma unroll
            for (int i = 0; i < kD / 2; i += 8) {
              uint4 v;
              v.x = pack_bf16(o[i] * inv, o[i + 1] * inv);
              v.y = pack_bf16(o[i + 2] * inv, o[i + 3] * inv);
              v.z = pack_bf16(o[i + 4] * inv, o[i + 5] * inv);
              v.w = pack_bf16(o[i + 6] * inv, o[i + 7] * inv);
              *reinterpret_cast<uint4*>(op + i) = v;
            }
            if (g == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = Ls == 0.f ? -INFINITY : M * kLn2 + logf(Ls);
          }
        }
      }
      ++f;
    }
  }
  tc_fence_before();
  __syncthreads();
  pdl_launch_dependents();
  if (tid == 0 && *s_fail) atomicMax(p.d_status, (int)CHECK_WAIT_TIMEOUT);
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

namespace ptc {
inline bool make_map(CUtensorMap* map, const void* data, int d, long long n1, long long n2, long long stride1,
                     long long stride2, int box1, int box2) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)n1, (cuuint64_t)n2};
  const cuuint64_t strides[2] = {(cuuint64_t)stride1 * 2, (cuuint64_t)stride2 * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box1, (cuuint32_t)box2};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(data), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kD, bool kPaged>
static cudaError_t launch(const Params& p, int ctas, cudaStream_t stream) {
  CUtensorMap q, k, v;
  const int G = p.cfg.G, Hkv = p.cfg.Hkv;
  if (!make_map(&q, p.Q.data, kD, p.Hq, p.seqs.n_tokens, p.Q.hs, p.Q.ts, G, p.cfg.tokens)) return cudaErrorInvalidValue;
  if (kPaged) {
    const long long rows = ((long long)p.pages.n_pages * Hkv) << p.pages.shift;
    if (!make_map(&k, p.K.data, kD, rows, 1, kD, rows * kD, p.box, 1) ||
        !make_map(&v, p.V.data, kD, rows, 1, kD, rows * kD, p.box, 1))
      return cudaErrorInvalidValue;
  } else {
    if (!make_map(&k, p.K.data, kD, p.seqs.n_tokens, Hkv, p.K.ts, p.K.hs, kBN, 1) ||
        !make_map(&v, p.V.data, kD, p.seqs.n_tokens, Hkv, p.V.ts, p.V.hs, kBN, 1))
      return cudaErrorInvalidValue;
  }
  auto kern = packed_tc_kernel<kD, kPaged>;
  cudaError_t e = ensure_dynamic_smem<3000 + kD * 2 + kPaged>(kern, Smem<kD>::kBytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Smem<kD>::kBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, q, k, v, p);
}
}  // namespace ptc

size_t packed_tc_scratch_bytes(int d) { return (size_t)2 * kMaxPackedCtas * 128 * ((size_t)d * 4 + 8); }

cudaError_t launch_packed_tc(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                             const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  ptc::Params p = {};
  p.seqs = seqs;
  const int G = d.n_q_heads / d.n_kv_heads;
  p.cfg.G = G;
  p.cfg.Hkv = d.n_kv_heads;
  p.cfg.tokens = ptc::kBM / G;
  p.cfg.tile = ptc::kBN;
  p.cfg.fixed = 2 * ptc::kBN;
  p.cfg.min_chunk = 6 * ptc::kBN;
  p.pages = kv.pages;
  p.paged = kv.paged;
  p.Q = Q;
  p.O = O;
  p.K = kv.K;
  p.V = kv.V;
  if (kv.paged) {
    p.K.data = kv.pages.K;
    p.V.data = kv.pages.V;
    p.box = (1 << kv.pages.shift) < ptc::kBN ? 1 << kv.pages.shift : ptc::kBN;
  }
  p.scale = scale;
  p.lse = lse;
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  char* ws = h.workspace + kStatusBytes;
  p.part_o = reinterpret_cast<float4*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)2 * ctas * 128 * d.head_dim * 4);
  p.d_status = h.d_status;
  p.Hq = d.n_q_heads;
  if (d.head_dim == 128)
    return kv.paged ? ptc::launch<128, true>(p, ctas, stream) : ptc::launch<128, false>(p, ctas, stream);
  return kv.paged ? ptc::launch<64, true>(p, ctas, stream) : ptc::launch<64, false>(p, ctas, stream);
}

}  // namespace samkv
