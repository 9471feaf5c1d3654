// tcgen05 attention of packed sequences over packed rows or over a paged cache; bf16, head dimension 64 or 128.
//
// Persistent, one CTA per SM.  An item is a tile of up to 128 query rows (row = token x group member, so the G query
// heads that share a KV head share its keys) against key tiles of 128 slots; packed_plan.cuh divides the call's items
// among the CTAs.  Roles of the 16 warps:
//   warps 0-11  softmax, three groups of four; tile T (the CTA's running count) belongs to group T mod 3, thread = row
//   warp 12     issues S(T) = Q K(T)^T into score buffer T mod 3
//   warp 13     issues O += P(T) V(T)
//   warp 14     walks the plan, loads Q (two buffers) and K (two stages) by TMA
//   warp 15     loads V (three stages), sees to value rows that not every query row sees
// All groups add into ONE accumulator.  They share a reference maximum per row: a piece's first tile sets it, the others
// use it as it stands, since it only has to be within a factor of 2^16 of the row's maximum (P is bf16 and O, l are fp32:
// all have the exponent range for it, and values of 2^90 over 10^5 slots still add up below 2^128).  A tile that needs a
// larger one waits for everything before it and rescales O in tensor memory; tiles behind it that used the old one rescale
// their probabilities before they hand them over.  A reference moves by whole steps of log2, so that rescaled
// probabilities are not rounded again.  Which reference a row's tile starts from is fixed (the first tile's, or the one
// its group ended the tile three before with), and each row decides for itself, so that results repeat bit for bit and
// depend on no other row.
// P(T) overlays the first half of S(T), so tensor memory holds three score buffers and O: 512 columns.
// The group with a piece's last tile writes the result while the others are at the next piece's tiles.
//
// What bounds it.  A tile costs 1024 cycles on the tensor pipe (16 products of 64 cycles), 1024 on the special-function
// unit, and 1280 of shared-memory bandwidth (operands 768, TMA writes 512), but the three groups run a tile each through
// a chain of about 6000 cycles (poll, maximum, exponentials, hand-over, two products, polls), about 2000 per tile: tensor
// pipe 36-45 % busy.  Measured steps: two groups taking turns 4000 cycles per tile; the loops rolled so that a tile's code
// fits the schedulers' instruction caches (straight-line code ran at 5 cycles an instruction) 2550; three groups 2100.
// One thread issuing both kinds of products, packed two-wide arithmetic, 64 scores at a time, every fourth exponential as
// a polynomial, and not loading K and V at all (as an experiment) change nothing or cost up to 15 %.
// 20 documents of 1536 tokens, 32/8 heads: 0.52 ms (740 TFLOP/s) with pauses between the calls; back to back the board's
// 1000 W cap lowers the clock: 0.59 ms (650 TFLOP/s).  128 tokens over 102400 slots, 64/8 heads: 0.53 ms (810 TFLOP/s; a
// fifth more without the layout in waves, which keeps the eight row tiles of a KV head on the same keys at the same time).
//
// Probabilities are rounded to bf16 for the second product.  O is divided by the sum of the rounded ones, so that the
// rounding of a probability moves the result only by how far its value is from the others' (with the other sum, a row that
// one key dominates was off by half a step of bf16 besides the output's own); lse takes the sum before rounding.
// Every wait is bounded; a wait that runs out sets a flag that ends all others, the CTA drains its copies and frees its
// tensor memory, and the failure is recorded as a device check.  TMA reads and writes this GPU's memory only, without
// multicast.
#include "packed_plan.cuh"
#include "tc_common.cuh"

namespace samkv {
namespace ptc {
using namespace tc;

constexpr int kBM = 128, kBN = 128;
constexpr int kKStages = 2, kVStages = 3, kQStages = 2, kRing = 3;
constexpr int kGroups = 3;                             // softmax groups, and score buffers
constexpr int kThreads = (4 * kGroups + 4) * 32;
constexpr int kWarpS = 4 * kGroups, kWarpPV = kWarpS + 1, kWarpK = kWarpS + 2, kWarpV = kWarpS + 3;
constexpr int kRegsSoftmax = 144, kRegsOther = 80;     // 384 x 144 + 128 x 80 = 512 x 128, the launch's registers
constexpr float kGrow = 16.0f;                         // log2
constexpr uint32_t kTmemCols = 512, kColO = 384;       // three score buffers of 128 columns, then O

template <int kD>
struct Smem {
  static constexpr int kTile = 128 * kD * 2;           // a Q, K or V tile
  static constexpr int kQ = 0;
  static constexpr int kK = kQ + kQStages * kTile;
  static constexpr int kV = kK + kKStages * kTile;
  static constexpr int kRef = kV + kVStages * kTile;   // reference maxima, [kGroups (piece mod)][128] fp32
  static constexpr int kSum = kRef + kGroups * 512;    // sums handed to the finishing group, [2][128] fp32
  static constexpr int kBar = kSum + 1024;
  static constexpr int kPieces = kBar + 296;           // kRing descriptors
  static constexpr int kMisc = kPieces + 180;          // tensor memory address, failure flag, "merge" and "scrub" flags
  static constexpr int kBytes = kMisc + 36;
};
static_assert(kRing * sizeof(Piece) <= 180, "descriptors");

static_assert(Smem<128>::kBytes <= 232448, "shared memory of one CTA");

enum Bar {
  FR_FULL = 0, FR_FREE = FR_FULL + kRing,
  Q_FULL = FR_FREE + kRing, Q_FREE = Q_FULL + kQStages,
  S_GO = Q_FREE + kQStages,             // K(T) has landed, the buffer for S(T) is used up
  GO = S_GO + kGroups,                  // P(T) complete, V(T) landed
  V_TMA = GO + kGroups,                 // a value tile that needs touching up has landed
  S_FULL = V_TMA + 1, PV_DONE = S_FULL + kGroups,
  TURN = PV_DONE + kGroups,             // tile T's probabilities are final
  REF = TURN + kGroups,                 // a piece's first tile has set the reference
  O_FREE = REF + kGroups, PARTS = O_FREE + 1, MERGE = PARTS + kGroups,
  SEEN = MERGE + kGroups,               // a piece's third tile has read the reference that the first one set
  kBars = SEEN + 1
};
static_assert(kBars * 8 <= 296, "barrier area");
static_assert(kVStages == kGroups, "a V stage is free when the value product of its group has completed");

// maximum that keeps NaN
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 16 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr) : "memory");
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 16; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                 "+f"(v[i + 6]), "+f"(v[i + 7]));
}

// Scores at and behind `limit` become -infinity.
template <int kN>
__device__ __forceinline__ void mask_row(float* v, int limit) {
#pragma unroll
  for (int i = 0; i < kN; ++i)
    if (i >= limit) v[i] = -INFINITY;
}

// lo += the lower, hi += the upper of two packed bf16 values (widened by the addition itself).
__device__ __forceinline__ void add_bf16_pair(float& lo, float& hi, uint32_t packed) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}"
      : "+f"(lo), "+f"(hi) : "r"(packed));
}

// Pins registers that tcgen05.ld filled behind the wait for it.
template <int kN>
__device__ __forceinline__ void settle(float* v) {
#pragma unroll
  for (int i = 0; i < kN; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                 "+f"(v[i + 6]), "+f"(v[i + 7]));
}

struct Params {
  Seqs seqs;
  SplitCfg cfg;
  Pages pages;                 // table, width, n_pages, shift; paged calls
  Rows Q, K, V, O;             // K, V: packed rows, or the pools' data pointers
  int paged, box;              // slots per TMA box
  int store_tokens;            // tokens of a warp's 32 rows, 0: rows are not whole tokens
  float scale;
  float* lse;
  float4* part_o;              // [slot][d/4][128]
  float2* part_ml;             // [slot][128] reference, sum of the rounded probabilities
  float* part_l;               // [slot][128] sum of the probabilities
  float* hand_l;               // [CTA][2][128] such sums on their way to the finishing group
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

// 2 kN packed columns of a row into a 128-byte-swizzled tile, from 16-byte piece `piece` on.
template <int kN>
__device__ __forceinline__ void stage_row(const uint32_t* v, uint32_t tile, int row, int piece) {
#pragma unroll
  for (int i = 0; i < kN; i += 4)
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(tile + blk_off(row, piece + (i >> 2))), "r"(v[i]), "r"(v[i + 1]),
                 "r"(v[i + 2]), "r"(v[i + 3]) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y),
               "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void bulk_commit_and_wait_read() {
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
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
// Whether rows [r0, r1) of a landed value tile hold an infinity or NaN (one warp).
template <int kD>
__device__ __forceinline__ bool any_nonfinite(uint32_t tile, int r0, int r1) {
  const int lane = threadIdx.x & 31;
  constexpr int kChunks = kD / 8;
  uint32_t hit = 0;
#pragma unroll 4
  for (int i = lane; i < (r1 - r0) * kChunks; i += 32) {
    const int r = r0 + i / kChunks, c = i % kChunks;
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(tile + (c >> 3) * (kBN * 128) + blk_off(r, c & 7)) : "memory");
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
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                 const __grid_constant__ ptc::Params p) {
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
  volatile uint32_t* s_scrub = s_merge + kGroups;            // [4]: number of the piece + 1 whose value tile was touched
  float* x_l = reinterpret_cast<float*>(smem_raw + L::kSum);
  Piece* ring = reinterpret_cast<Piece*>(smem_raw + L::kPieces);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.cfg.G;

  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) { mbar_init(bar(FR_FULL + i), 1); mbar_init(bar(FR_FREE + i), 3 + 4 * kGroups); }
    for (int i = 0; i < kQStages; ++i) { mbar_init(bar(Q_FULL + i), 1); mbar_init(bar(Q_FREE + i), 4); }
    mbar_init(bar(V_TMA), 1);
    for (int i = 0; i < kGroups; ++i) {
      mbar_init(bar(S_GO + i), 1 + 1);
      mbar_init(bar(GO + i), 4 + 1);
      mbar_init(bar(S_FULL + i), 1);
      mbar_init(bar(PV_DONE + i), 1);
      mbar_init(bar(TURN + i), 4);
      mbar_init(bar(REF + i), 4);
      mbar_init(bar(PARTS + i), 4);
      mbar_init(bar(MERGE + i), 1);
    }
    mbar_init(bar(O_FREE), 4);
    mbar_init(bar(SEEN), 4);
    for (int i = 0; i < 4; ++i) s_scrub[i] = 0;
    *s_fail = (base & 1023u) != 0;          // (never seen: the declaration asks for 1024 bytes)
    if (*s_fail) atomicMax(p.d_status, (int)CHECK_SMEM_ALIGNMENT);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    for (int i = 0; i < kGroups; ++i) mbar_arrive(bar(S_GO + i));      // (every score buffer starts out free)
  }
  if (warp == kWarpS) {
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
  if (p.seqs.n_seq > kWarpPlanSeqs) plan_block<kThreads>(p.seqs, p.cfg, &plan, &chunk, p.d_status, tid);

  auto wait = [&](int i, uint32_t phase) { return wait_bar(bar(i), phase & 1u, s_fail); };

  if (warp >= kWarpS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == kWarpK) {
      // ================= plan and K =================
      Walker w;
      w.begin(p.seqs, p.cfg, &plan, chunk, p.d_status);
      __syncwarp();
      fence_proxy_async();                  // the plan's memory becomes the destination of copies
      __syncwarp();
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
#pragma unroll 1
        for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
          int next = 0;
          if constexpr (kPaged) { if (t + 1 < pc.tile1) next = tile_page(p, pc, t + 1, &bad); }
          if (T >= kKStages) wait(S_FULL + (T - kKStages) % kGroups, (T - kKStages) / kGroups);     // its score product is done
          load_tile<kD, kPaged>(p, &tmK, pc, t, base + L::kK + (T % kKStages) * L::kTile, bar(S_GO + T % kGroups), page);
          page = next;
        }
        ++f;
      }
      if (__any_sync(0xffffffffu, bad) && lane == 0) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
      // no copy of this CTA outlives it: the products have waited for them, unless something failed
#pragma unroll 1
      for (uint32_t i = 0; i < kGroups; ++i)
        if (T > i) drain_bar(bar(S_GO + (T - 1 - i) % kGroups), ((T - 1 - i) / kGroups) & 1u);
#pragma unroll 1
      for (uint32_t i = 0; i < kQStages; ++i)
        if (f > i) drain_bar(bar(Q_FULL + (f - 1 - i) % kQStages), ((f - 1 - i) / kQStages) & 1u);
    } else if (warp == kWarpS) {
      // ================= S = Q K^T =================
      // Two warps issue, one the score products and one the value products: a poll next to running products costs 150-300
      // cycles, which the other warp's products cover.  One barrier collects everything a product needs.
      constexpr uint32_t kIdesc = instr_desc(kBM, kBN, false);
      const uint64_t dQ0 = smem_desc(base + L::kQ, 16, 1024), dK0 = smem_desc(base + L::kK, 16, 1024);
      uint32_t f = 0, T = 0;
      while (true) {
        if (!wait(FR_FULL + f % kRing, f / kRing)) break;
        const int t0 = ring[f % kRing].tile0, t1 = ring[f % kRing].tile1;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
        if (t0 < 0) break;
        wait(Q_FULL + f % kQStages, f / kQStages);
        const uint64_t dQ = dQ0 + (uint64_t)((f % kQStages) * (L::kTile >> 4));
#pragma unroll 1
        for (int t = t0; t < t1; ++t, ++T) {
          wait(S_GO + T % kGroups, T / kGroups);
          tc_fence_after();
          __syncwarp();
          if (lane == 0) {
            const uint64_t dK = dK0 + (uint64_t)((T % kKStages) * (L::kTile >> 4));
#pragma unroll
            for (int ks = 0; ks < kD / 16; ++ks) {
              const uint32_t aoff = ((ks >> 2) * (kBM * 128) + (ks & 3) * 32) >> 4;
              const uint32_t boff = ((ks >> 2) * (kBN * 128) + (ks & 3) * 32) >> 4;
              mma_ss(tmem + (T % kGroups) * kBN, dQ + aoff, dK + boff, kIdesc, ks > 0);
            }
            mma_commit(bar(S_FULL + T % kGroups));
          }
          __syncwarp();
        }
        ++f;
      }
    } else if (warp == kWarpPV) {
      // ================= O += P V =================
      constexpr uint32_t kIdesc = instr_desc(kBM, kD, true);
      const uint64_t dV0 = smem_desc(base + L::kV, kBN * 128, 1024);
      uint32_t f = 0, T = 0;
      while (true) {
        if (!wait(FR_FULL + f % kRing, f / kRing)) break;
        const int t0 = ring[f % kRing].tile0, t1 = ring[f % kRing].tile1, seen = ring[f % kRing].seen;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
        if (t0 < 0) break;
        if (f > 0) wait(O_FREE, f - 1);
#pragma unroll 1
        for (int t = t0; t < t1; ++t, ++T) {
          const uint32_t g = T % kGroups;
          wait(GO + g, T / kGroups);
          tc_fence_after();
          __syncwarp();
          if (lane == 0) {
            const uint64_t dV = dV0 + (uint64_t)(g * (L::kTile >> 4));
            const int slots = seen - t * kBN;              // steps of 16 slots that some row sees
#pragma unroll
            for (int ks = 0; ks < kBN / 16; ++ks)
              if (ks == 0 || ks * 16 < slots)
                mma_ts(tmem + kColO, tmem + g * kBN + ks * 8, dV + ((ks * 16 * 128) >> 4), kIdesc, (t > t0) | (ks > 0));
            mma_commit(bar(S_GO + g));
            mma_commit(bar(PV_DONE + g));
          }
          __syncwarp();
        }
        ++f;
      }
    } else if (warp == kWarpV) {
      uint32_t f = 0, T = 0, partial_tiles = 0;
      while (true) {
        if (!wait(FR_FULL + f % kRing, f / kRing)) break;
        const Piece pc = ring[f % kRing];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
        if (pc.tile0 < 0) break;
        {
          // ================= V =================
          // Of the slots that only some rows of the tile see, infinities and NaN must not meet the zero weights of the
          // others: they are looked for in the landed tile (at most 127 rows of it), and in the rare case that there are
          // any they are cleared there and added back, row by row, when the result is written.
          int page = 0;
          bool bad = false;                                        // (reported by the K loader)
          if constexpr (kPaged) page = tile_page(p, pc, pc.tile0, &bad);
          const int zone0 = max(pc.seen0, pc.tile0 * kBN), zone1 = min(pc.seen, pc.tile1 * kBN);
#pragma unroll 1
          for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
            int next = 0;
            if constexpr (kPaged) { if (t + 1 < pc.tile1) next = tile_page(p, pc, t + 1, &bad); }
            const uint32_t st = T % kVStages, dst = base + L::kV + st * L::kTile;
            if (T >= kVStages) wait(PV_DONE + st, T / kVStages - 1);
            const int slots = pc.seen - t * kBN;                   // slots behind `seen` that a step of 16 still covers
            const bool clear = slots < kBN && (slots & 15) != 0 || slots <= 0;
            const int r0 = max(zone0 - t * kBN, 0), r1 = min(zone1 - t * kBN, kBN);
            const bool look = r0 < r1;
            if (!clear && !look) {
              load_tile<kD, kPaged>(p, &tmV, pc, t, dst, bar(GO + st), page);
            } else {
              load_tile<kD, kPaged>(p, &tmV, pc, t, dst, bar(V_TMA), page);
              wait(V_TMA, partial_tiles++);
              if (clear) {
                const int first = max(slots, 0), end = max((first + 15) & ~15, 16);
#pragma unroll 1
                for (int i = lane; i < (end - first) * (kD / 8); i += 32) {
                  const int r = first + i / (kD / 8), c = i % (kD / 8);
                  asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(dst + (c >> 3) * (kBN * 128) + blk_off(r, c & 7)),
                               "r"(0) : "memory");
                }
              }
              if (look && any_nonfinite<kD>(dst, r0, r1)) {
                if (lane == 0) s_scrub[f % 4] = f + 1;   // (this warp is at most three pieces ahead of the epilogues)
#pragma unroll 1
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
              if (lane == 0) mbar_arrive(bar(GO + st));
              __syncwarp();
            }
            page = next;
          }
        }
        ++f;
      }
#pragma unroll 1
      for (uint32_t i = 0; i < kVStages; ++i)
        if (T > i) drain_bar(bar(GO + (T - 1 - i) % kVStages), ((T - 1 - i) / kVStages) & 1u);
    }
  } else {
    // ================= softmax =================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int g = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t tS = lane_addr + g * kBN, tO = lane_addr + kColO;      // P overlays the first half of the scores
    const float sl2 = p.scale * kLog2e;
    const int t_local = row / G, member = row - t_local * G;
    uint32_t f = 0, T = 0, n_merged = 0, n_seen = 0;     // n_seen: pieces of three or more tiles
    while (true) {
      if (!wait(FR_FULL + f % kRing, f / kRing)) break;
      const Piece pc = ring[f % kRing];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
      if (pc.tile0 < 0) break;
      const uint32_t Tend = T + (uint32_t)(pc.tile1 - pc.tile0);
      // The group with the piece's last tile finishes it; the others go on to the next piece at once.
      const bool finishes = (Tend - 1) % kGroups == (uint32_t)g;
      const int t_seq = pc.r * p.cfg.tokens + t_local;
      const bool valid = t_local < p.cfg.tokens && t_seq < pc.n;
      Seq sq;
      sq.first = pc.first; sq.n = pc.n; sq.base = pc.base;
      // rows without a token follow the last one: their results are dropped
      const int vis = visible(p.seqs, sq, min(t_seq, min((pc.r + 1) * p.cfg.tokens, pc.n) - 1));
      float* ref_row = ref_max + (f % kGroups) * 128 + row;
      // sums of the groups with the tile before the last ([0]) and the one before that ([128]): of the rounded probabilities
      // through shared memory, the exact ones, which only lse needs, through global memory (shared memory is full)
      float* r_row = x_l + row;
      volatile float* l_row = p.hand_l + (size_t)blockIdx.x * 256 + row;
      float m = -INFINITY, l = 0.f, rl = 0.f;             // rl: sum of the rounded probabilities
      bool poison = false, ref_known = false;
#pragma unroll 1
      for (int t = pc.tile0 + (int)((kGroups + g - T % kGroups) % kGroups); t < pc.tile1; t += kGroups) {
        const uint32_t Tt = T + (uint32_t)(t - pc.tile0);
        wait(S_FULL + g, Tt / kGroups);
        tc_fence_after();
        // first pass over the scores: their maximum.  (The loops stay rolled: the code of a tile has to fit the schedulers'
        // instruction caches, straight-line code that does not runs at 3-5 cycles an instruction.)
        const int limit = vis - t * kBN;
        const int width = min(pc.seen - t * kBN, kBN);   // slots that some row sees
        const bool masked = __any_sync(0xffffffffu, limit < kBN);
        float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll 1
        for (int c0 = 0; c0 < kBN; c0 += 32) {
          float sv[32];
          tmem_ld32_nowait(tS + c0, sv);
          tmem_wait_ld();
          settle<32>(sv);
          if (masked) mask_row<32>(sv, limit - c0);
#pragma unroll
          for (int i = 0; i < 32; i += 8) {
            mx0 = max3_nan(mx0, sv[i], sv[i + 1]);
            mx1 = max3_nan(mx1, sv[i + 2], sv[i + 3]);
            mx2 = max3_nan(mx2, sv[i + 4], sv[i + 5]);
            mx3 = max3_nan(mx3, sv[i + 6], sv[i + 7]);
          }
        }
        const float cand = max3_nan(max3_nan(mx0, mx1, mx2), mx3, mx3) * sl2;
        poison |= !(cand < INFINITY);                    // NaN or +infinity among the row's scores
        // The piece's first tile sets the row's reference; the others use the one they know.  Whether a tile before this one
        // has moved it meanwhile is looked at when the probabilities are done.
        const bool first = t == pc.tile0;
        if (!first && !ref_known) wait(REF + f % kGroups, f / kGroups);
        float ref = first ? cand : ref_known ? m : *ref_row;
        ref_known = true;
        if (first) {
          *ref_row = ref;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(REF + f % kGroups));
        } else {
          if (t == pc.tile0 + 2) {                       // (the second tile may move it from here on)
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(SEEN));
          }
          auto too_small = [&](float r) { return cand - r > kGrow || (r == -INFINITY && cand > -INFINITY); };
          const bool far = valid && too_small(ref);      // (rows without a token have no say)
          if (__any_sync(0xffffffffu, far)) {
            // some row needs a larger reference: O has to follow, so everything before this tile is finished first
            wait(TURN + (Tt - 1) % kGroups, (Tt - 1) / kGroups);
            wait(PV_DONE + (Tt - 1) % kGroups, (Tt - 1) / kGroups);
            if (t == pc.tile0 + 1 && pc.tile1 - pc.tile0 > 2) wait(SEEN, n_seen);
            tc_fence_after();
            const float old = *ref_row;
            const bool grow = far && too_small(old);
            const float step = rintf(cand - old), up = step < 1e7f ? old + step : cand;
            const float corr = grow ? fast_exp2(old - up) : 1.0f;
            if (grow) *ref_row = up;
            if (far) ref = grow ? up : old;
#pragma unroll 1
            for (int c0 = 0; c0 < kD; c0 += 32) {
              float o[32];
              tmem_ld32(tO + c0, o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] *= corr;
              tmem_st32(tO + c0, o);
            }
            // denominators that other groups have handed over already follow too
            if (grow && t + 2 >= pc.tile1 && pc.tile1 - pc.tile0 > 2 && r_row[128] > 0.f) {
              r_row[128] *= corr;
              l_row[128] = l_row[128] * corr;
            }
            if (grow && t + 1 == pc.tile1 && r_row[0] > 0.f) {
              r_row[0] *= corr;
              l_row[0] = l_row[0] * corr;
            }
          }
        }
        if (m != ref) {
          const float corr = fast_exp2(m - ref);
          l = l > 0.f ? l * corr : l;
          rl = rl > 0.f ? rl * corr : rl;
          m = ref;
        }
        const float mu = m == -INFINITY ? 0.f : m;
        // second pass: probabilities, 32 columns at a time.  (No row sees slots behind `width`: the value product skips them.)
        // The second sum and its hand-over cost 3 % (128 tokens over 102400) to 5 % (20 x 1536) of the time; with the rounded
        // values widened by shifts and masks instead of the mixed-precision addition they cost 6 and 7 %.
        f2 exact0 = 0ull, exact1 = 0ull;
        float r0 = 0.f, r1 = 0.f, r2 = 0.f, r3 = 0.f;
        const f2 sl22 = both(sl2), mu2 = both(-mu);
#pragma unroll 1
        for (int c0 = 0; c0 < max(width, 1); c0 += 32) {
          float x[32];
          tmem_ld32_nowait(tS + c0, x);
          tmem_wait_ld();
          settle<32>(x);
          if (masked) mask_row<32>(x, limit - c0);
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float2 a = split2(fma2(join2(x[i], x[i + 1]), sl22, mu2)), b = split2(fma2(join2(x[i + 2], x[i + 3]), sl22, mu2));
            x[i] = fast_exp2(a.x);
            x[i + 1] = fast_exp2(a.y);
            x[i + 2] = fast_exp2(b.x);
            x[i + 3] = fast_exp2(b.y);
            exact0 = add2(exact0, join2(x[i], x[i + 1]));
            exact1 = add2(exact1, join2(x[i + 2], x[i + 3]));
            pk[i / 2] = pack_bf16(x[i], x[i + 1]);
            pk[i / 2 + 1] = pack_bf16(x[i + 2], x[i + 3]);
            add_bf16_pair(r0, r1, pk[i / 2]);
            add_bf16_pair(r2, r3, pk[i / 2 + 1]);
          }
          tmem_st16(tS + (c0 >> 1), pk);
        }
        const float2 sums = split2(add2(exact0, exact1));
        l += sums.x + sums.y;
        float tile_r = (r0 + r1) + (r2 + r3);
        if (Tt > 0) wait(TURN + (Tt - 1) % kGroups, (Tt - 1) / kGroups);
        if (!first) {
          const float now = *ref_row;
          const bool moved = valid && now != m && now == now;
          if (__any_sync(0xffffffffu, moved)) {          // by a tile before this one: follow
            tmem_wait_st();
            const float corr = moved ? fast_exp2(m - now) : 1.0f;
            float again = 0.f;
#pragma unroll 1
            for (int c0 = 0; c0 < kBN; c0 += 32) {
              float q[16];
              tmem_ld16(tS + (c0 >> 1), q);
              uint32_t pk[16];
#pragma unroll
              for (int i = 0; i < 16; ++i)
                pk[i] = pack_bf16(bf16_lo(__float_as_uint(q[i])) * corr, bf16_hi(__float_as_uint(q[i])) * corr);
              tmem_st16(tS + (c0 >> 1), pk);
              if (c0 < width) {
#pragma unroll
                for (int i = 0; i < 16; ++i) again += bf16_lo(pk[i]) + bf16_hi(pk[i]);
              }
            }
            if (moved) {                                 // (the others keep their sum, added up in its own order)
              tile_r = again;
              l = l > 0.f ? l * corr : l;
              rl = rl > 0.f ? rl * corr : rl;
              m = now;
            }
          }
        }
        rl += tile_r;
        if (t + 2 == pc.tile1 || t + 3 == pc.tile1) {    // this group's last tile of the piece, but not the piece's last
          if (f > 0) wait(O_FREE, f - 1);                // (the piece before has read its own)
          const int at = t + 2 == pc.tile1 ? 0 : 128;
          r_row[at] = poison ? __int_as_float(0x7fffffff) : rl;
          if (p.lse != nullptr) l_row[at] = l;
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(TURN + g));
          mbar_arrive(bar(GO + g));
        }
      }
      T = Tend;
      if (pc.tile1 - pc.tile0 > 2) ++n_seen;
      if (finishes) {
        // ---- the piece's result ----
        if (poison) l = rl = __int_as_float(0x7fffffff);
        if (p.lse != nullptr) {                          // (ordered by the turns that the last tile has waited for)
          if (pc.tile1 - pc.tile0 > 1) l += l_row[0];
          if (pc.tile1 - pc.tile0 > 2) l += l_row[128];
        }
        wait(PV_DONE + g, (T - 1) / kGroups);
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kGroups - 1; ++k) {          // (their products come before this tile's)
          const float r_other = pc.tile1 - pc.tile0 > k + 1 ? r_row[k * 128] : 0.f;
          if (r_other != 0.f) rl += r_other;             // (at the last tile's reference)
        }
        const bool store = valid && *s_fail == 0;
        const bool scrubbed = s_scrub[f % 4] == f + 1;
        const int tok = pc.first + t_seq, hq = pc.h * G + member;
        const uint32_t sO = base + L::kQ + (f % kQStages) * L::kTile;       // over the piece's Q tile: no product reads it now
        // a whole item is normalised into shared memory, a piece of a cut item goes to the workspace as it is
        const float inv = rl == 0.f ? 0.f : 1.0f / rl;
#pragma unroll 1
        for (int c0 = 0; c0 < kD; c0 += 16) {
          float o[16];
          tmem_ld16(tO + c0, o);
          if (scrubbed && store) {
            // infinities and NaN that were cleared from the value tile: back into the rows that see them
#pragma unroll 1
            for (int j = max(pc.seen0, pc.tile0 * kBN); j < min(vis, pc.tile1 * kBN); ++j) {
              const __nv_bfloat16* v = kv_row(p, p.V, pc, j, kD) + c0;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float y = __bfloat162float(v[i]);
                if (!(fabsf(y) < INFINITY)) o[i] += y;
              }
            }
          }
          if (pc.slot < 0) {
            uint32_t pk[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) pk[i / 2] = rl == 0.f ? 0u : pack_bf16(o[i] * inv, o[i + 1] * inv);
            stage_row<8>(pk, sO + (c0 >> 6) * (kBM * 128), row, (c0 & 63) >> 3);
          } else {
            float4* po = p.part_o + ((size_t)pc.slot * (kD / 4) + c0 / 4) * 128 + row;
#pragma unroll
            for (int i = 0; i < 16; i += 4) po[(i >> 2) * 128] = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(O_FREE));
        bool write = true;
        float m_out = m;
        if (pc.slot >= 0) {
          // whoever takes the last ticket merges the item's pieces in their order
          p.part_ml[pc.slot * 128 + row] = make_float2(m, rl);
          p.part_l[pc.slot * 128 + row] = l;
          __threadfence();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(PARTS + g));
          wait(PARTS + g, n_merged);
          if (warp == 4 * g && lane == 0) {
            s_merge[g] = last_piece(p.d_status, pc.ticket, pc.n_pieces);
            mbar_arrive(bar(MERGE + g));
          }
          wait(MERGE + g, n_merged++);
          write = s_merge[g] != 0;
          if (write) {
            __threadfence();
            m_out = -INFINITY;
#pragma unroll 1
            for (int k = 0; k < pc.n_pieces; ++k) {
              const float2 x = __ldcg(p.part_ml + piece_slot(pc, k) * 128 + row);
              m_out = x.y == 0.f ? m_out : fmaxf(m_out, x.x);
            }
            const float Mu = m_out == -INFINITY ? 0.f : m_out;
            l = rl = 0.f;
#pragma unroll 1
            for (int k = 0; k < pc.n_pieces; ++k) {
              const float2 x = __ldcg(p.part_ml + piece_slot(pc, k) * 128 + row);
              if (x.y != 0.f) {
                const float w = fast_exp2(x.x - Mu);
                rl += x.y * w;
                l += __ldcg(p.part_l + piece_slot(pc, k) * 128 + row) * w;
              }
            }
            const float inv_all = rl == 0.f ? 0.f : 1.0f / rl;
#pragma unroll 1
            for (int c0 = 0; c0 < kD; c0 += 32) {
              float o[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = 0.f;
#pragma unroll 2
              for (int k = 0; k < pc.n_pieces; ++k) {
                const int slot = piece_slot(pc, k);
                const float2 x = __ldcg(p.part_ml + slot * 128 + row);
                const float w = x.y == 0.f ? 0.f : fast_exp2(x.x - Mu);
                const float4* src = p.part_o + ((size_t)slot * (kD / 4) + c0 / 4) * 128 + row;
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                  const float4 v = __ldcg(src + (i >> 2) * 128);
                  if (x.y != 0.f) {                      // (a piece that saw nothing of this row adds nothing)
                    o[i] = fmaf(v.x, w, o[i]);
                    o[i + 1] = fmaf(v.y, w, o[i + 1]);
                    o[i + 2] = fmaf(v.z, w, o[i + 2]);
                    o[i + 3] = fmaf(v.w, w, o[i + 3]);
                  }
                }
              }
              uint32_t pk[16];
#pragma unroll
              for (int i = 0; i < 32; i += 2) pk[i / 2] = rl == 0.f ? 0u : pack_bf16(o[i] * inv_all, o[i + 1] * inv_all);
              stage_row<16>(pk, sO + (c0 >> 6) * (kBM * 128), row, (c0 & 63) >> 3);
            }
          }
        }
        if (write) {
          if (store && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = rl == 0.f ? -INFINITY : m_out * kLn2 + logf(l);
          fence_proxy_async();
          __syncwarp();
          const unsigned rows_ok = __ballot_sync(0xffffffffu, store);
          const int row0 = (warp & 3) * 32;
          if (p.store_tokens > 0 && rows_ok == 0xffffffffu) {
            // the warp's 32 rows are whole tokens: out by TMA, straight from the staged tile
            if (lane == 0) {
#pragma unroll
              for (int x = 0; x < kD; x += 64)
                tma_store_3d(&tmO, x, pc.h * G, tok, sO + (x >> 6) * (kBM * 128) + row0 * 128);
              bulk_commit_and_wait_read();
            }
          } else {
            constexpr int kLanes = kD / 8;               // lanes per row
            const long long row_off = (long long)tok * p.O.ts + (long long)hq * p.O.hs;
#pragma unroll 1
            for (int i = 0; i < 32; i += 32 / kLanes) {
              const int r = i + lane / kLanes, c = lane % kLanes;
              const long long off = __shfl_sync(0xffffffffu, row_off, r);
              uint4 v;
              asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                           : "r"(sO + (c >> 3) * (kBM * 128) + blk_off(row0 + r, c & 7)) : "memory");
              if (rows_ok >> r & 1u) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.O.data) + off + c * 8) = v;
            }
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(Q_FREE + f % kQStages));
      }
      ++f;
    }
  }
  tc_fence_before();
  __syncthreads();
  pdl_launch_dependents();
  if (tid == 0 && *s_fail) atomicMax(p.d_status, (int)CHECK_WAIT_TIMEOUT);
  if (warp == kWarpS) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

namespace ptc {
template <int kD, bool kPaged>
static cudaError_t launch(const Params& p, int ctas, cudaStream_t stream) {
  CUtensorMap q, k, v, o;
  const int G = p.cfg.G, Hkv = p.cfg.Hkv;
  if (!make_rows_map(&q, p.Q.data, kD, p.Hq, p.seqs.n_tokens, p.Q.hs, p.Q.ts, G, p.cfg.tokens)) return cudaErrorInvalidValue;
  if (!make_rows_map(&o, p.O.data, kD, p.Hq, p.seqs.n_tokens, p.O.hs, p.O.ts, G, p.store_tokens > 0 ? p.store_tokens : 1))
    return cudaErrorInvalidValue;
  if (kPaged) {
    const long long rows = ((long long)p.pages.n_pages * Hkv) << p.pages.shift;
    if (!make_rows_map(&k, p.K.data, kD, rows, 1, kD, rows * kD, p.box, 1) ||
        !make_rows_map(&v, p.V.data, kD, rows, 1, kD, rows * kD, p.box, 1))
      return cudaErrorInvalidValue;
  } else {
    if (!make_rows_map(&k, p.K.data, kD, p.seqs.n_tokens, Hkv, p.K.ts, p.K.hs, kBN, 1) ||
        !make_rows_map(&v, p.V.data, kD, p.seqs.n_tokens, Hkv, p.V.ts, p.V.hs, kBN, 1))
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
  return cudaLaunchKernelEx(&cfg, kern, q, k, v, o, p);
}
}  // namespace ptc

constexpr int kTcSlots = kMaxUnits > 2 * kMaxPackedCtas ? kMaxUnits : 2 * kMaxPackedCtas;
size_t packed_tc_scratch_bytes(int d) {
  return (size_t)kTcSlots * 128 * ((size_t)d * 4 + 12) + (size_t)kMaxPackedCtas * 256 * 4;
}

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
  p.cfg.wave_slots = (64LL << 20) / (d.head_dim * 4);        // K and V of half the L2 cache
  p.store_tokens = 32 % G == 0 ? 32 / G : 0;
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
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)kTcSlots * 128 * d.head_dim * 4);
  p.part_l = reinterpret_cast<float*>(p.part_ml + (size_t)kTcSlots * 128);
  p.hand_l = p.part_l + (size_t)kTcSlots * 128;
  p.d_status = h.d_status;
  p.Hq = d.n_q_heads;
  if (d.head_dim == 128)
    return kv.paged ? ptc::launch<128, true>(p, ctas, stream) : ptc::launch<128, false>(p, ctas, stream);
  return kv.paged ? ptc::launch<64, true>(p, ctas, stream) : ptc::launch<64, false>(p, ctas, stream);
}

}  // namespace samkv
