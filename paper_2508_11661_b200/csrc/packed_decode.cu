// Attention of a few new tokens per sequence (decode) over a paged cache: at most 16 packed query rows (token x group
// member) per KV head, bf16, head dimension 64 or 128.  Bound by reading the cache once.
//
// Persistent, one CTA per SM; packed_plan.cuh gives every CTA the same number of slots.  One producer warp walks the
// plan and keeps a ring of four 64-slot tiles (K and V, 32 KB at d = 128) in flight by TMA, so 128 KB per SM cover the
// latency of HBM.  Eight consumer warps: tile T belongs to the four warps of parity T & 1, 16 slots each.  A warp runs
// its own online softmax over its slots on mma.sync m16n8k16 (16 rows fill one instruction; tcgen05's 128 rows would
// not), so warps exchange nothing until a piece ends; then the eight (m, l, O) are merged through shared memory.
// The second product takes each weight as the sum of two bf16 values, good to 2^-15: next to the reads of the cache the
// second set of products costs 1 %, and the result is as good as one from fp32 weights (relative error of 32 x 20480
// slots 1.66e-3, all of it the output's rounding; 2.24e-3 with weights of 8 bits).
// 32 requests over 20480 slots, 32/8 heads of 128: 0.405 ms, 6.63 TB/s, the rate of a plain copy (1.03 of the measured
// one); one request over 102400 slots, 64/8 heads: 78 us, 5.4 TB/s (start-up, the ring's first fill and the merge of 19
// pieces per KV head are about 12 us of it).  The tensor-memory kernel takes 0.42-0.43 ms and 155 us for the same calls.
// Every wait is bounded; a wait that runs out ends the others and is recorded as a device check.
#include "packed_plan.cuh"
#include "tc_common.cuh"

namespace samkv {
namespace pdec {
using namespace tc;

constexpr int kRows = 16, kBN = 64, kStages = 4, kRing = 4;
constexpr int kConsumers = 8, kThreads = (kConsumers + 1) * 32;

template <int kD>
struct Smem {
  static constexpr int kTile = kBN * kD * 2;                       // K or V of a tile
  static constexpr int kQTile = kRows * kD * 2;
  static constexpr int kKv = 0;                                    // [kStages][K, V]
  static constexpr int kQ = kKv + kStages * 2 * kTile;             // [kRing]
  static constexpr int kO = kQ + kRing * kQTile;                   // [kConsumers][kRows][kD] fp32
  static constexpr int kMl = kO + kConsumers * kRows * kD * 4;     // [kConsumers][kRows] float2
  static constexpr int kPieces = kMl + kConsumers * kRows * 8;
  static constexpr int kBar = kPieces + kRing * 64;
  static constexpr int kMisc = kBar + 192;
  static constexpr int kBytes = kMisc + 64;
};
static_assert(Smem<128>::kBytes <= 232448, "shared memory of one CTA");

enum Bar {
  FR_FULL = 0, FR_FREE = FR_FULL + kRing, KV_FULL = FR_FREE + kRing, KV_FREE = KV_FULL + kStages, JOIN = KV_FREE + kStages,
  kBars = JOIN + 1
};
static_assert(kBars * 8 <= 192, "barrier area");

struct Params {
  Seqs seqs;
  SplitCfg cfg;
  Pages pages;
  Rows Q, O;
  int box;
  float scale;
  float* lse;
  float* part_o;               // [slot][kRows][kD]
  float2* part_ml;             // [slot][kRows]
  int* d_status;
  int Hq;
};

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A weight's two parts: its bits cut off to bf16, and the rest.  The rest of a weight that is not zero is not zero either
// (2^-126 at least), so that an infinite value times both parts is that infinity and no NaN.
__device__ __forceinline__ uint32_t upper_parts(float lo, float hi) {
  return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);
}
__device__ __forceinline__ float lower_part(float p) {
  const float rest = fmaxf(p - __uint_as_float(__float_as_uint(p) & 0xffff0000u), 1.17549435e-38f);
  return p > 0.f ? rest : 0.f;
}
}  // namespace pdec

template <int kD>
__global__ void __launch_bounds__(pdec::kThreads, 1)
packed_decode_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const __grid_constant__ pdec::Params p) {
  using namespace pdec;
  using L = Smem<kD>;
  constexpr int kHalves = kD / 64;                       // 128-byte column blocks of a row
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  const uint32_t sBar = base + L::kBar;
  auto bar = [&](int i) { return sBar + 8u * i; };
  PlanShared& plan = *reinterpret_cast<PlanShared*>(smem_raw + L::kO);     // read by the producer before any piece ends
  Piece* ring = reinterpret_cast<Piece*>(smem_raw + L::kPieces);
  volatile uint32_t* s_fail = reinterpret_cast<volatile uint32_t*>(smem_raw + L::kMisc);
  volatile uint32_t* s_merge = s_fail + 1;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = p.cfg.G;
  if (tid == 0) {
    for (int i = 0; i < kRing; ++i) { mbar_init(bar(FR_FULL + i), 1); mbar_init(bar(FR_FREE + i), kConsumers); }
    for (int i = 0; i < kStages; ++i) { mbar_init(bar(KV_FULL + i), 1); mbar_init(bar(KV_FREE + i), 4); }
    mbar_init(bar(JOIN), kConsumers);
    *s_fail = (base & 1023u) != 0;
    if (*s_fail) atomicMax(p.d_status, (int)CHECK_SMEM_ALIGNMENT);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  long long chunk = 0;
  if (p.seqs.n_seq > kWarpPlanSeqs) plan_block<kThreads>(p.seqs, p.cfg, &plan, &chunk, p.d_status, tid);
  auto wait = [&](int i, uint32_t phase) { return wait_bar(bar(i), phase & 1u, s_fail); };

  if (warp == kConsumers) {
    // ================= producer: plan, Q, K and V =================
    Walker w;
    w.begin(p.seqs, p.cfg, &plan, chunk, p.d_status);
    __syncwarp();
    Piece pc;
    uint32_t f = 0, T = 0;
    bool bad = false;
    while (true) {
      const bool have = *s_fail == 0 && w.next(p.seqs, p.cfg, &pc);
      if (f >= kRing) wait(FR_FREE + f % kRing, f / kRing - 1);
      if (lane == 0) {
        if (!have) pc.tile0 = -1;
        ring[f % kRing] = pc;
        if (have) {                                       // descriptor and queries complete one barrier
          const uint32_t dst = base + L::kQ + (f % kRing) * L::kQTile;
          mbar_expect_tx(bar(FR_FULL + f % kRing), p.cfg.tokens * G * kD * 2);
#pragma unroll
          for (int x = 0; x < kHalves; ++x)
            tma_load_3d(dst + x * (kRows * 128), &tmQ, x * 64, pc.h * G, pc.first + pc.r * p.cfg.tokens, bar(FR_FULL + f % kRing));
        } else {
          mbar_arrive(bar(FR_FULL + f % kRing));
        }
      }
      __syncwarp();
      ++f;
      if (!have) break;
      const int per_tile = kBN / p.box;
      // page numbers of up to 32 boxes ahead sit in the lanes
      int first_box = 0, page = 0;
      auto fetch = [&](int box) {
        first_box = box;
        const int j = (box + lane) * p.box;
        page = 0;
        if (j < pc.seen && j < pc.tile1 * kBN) {
          page = p.pages.table[(size_t)pc.s * p.pages.width + (j >> p.pages.shift)];
          if ((unsigned)page >= (unsigned)p.pages.n_pages) {
            page = 0;
            bad = true;
          }
        }
      };
      fetch(pc.tile0 * per_tile);
#pragma unroll 1
      for (int t = pc.tile0; t < pc.tile1; ++t, ++T) {
        const uint32_t st = T % kStages;
        if ((t + 1) * per_tile - first_box > 32) fetch(t * per_tile);
        if (T >= kStages) wait(KV_FREE + st, T / kStages - 1);
        const int j0 = t * kBN;
        const int n_box = min(per_tile, (pc.seen - j0 + p.box - 1) / p.box);          // boxes that no row sees stay unloaded
        const uint32_t dst = base + L::kKv + st * 2 * L::kTile;
        if (lane == 0) mbar_expect_tx(bar(KV_FULL + st), max(n_box, 0) * p.box * kD * 4);
        __syncwarp();
        const int b = lane;
        const int pg = __shfl_sync(0xffffffffu, page, (t * per_tile - first_box + b) & 31);
        if (b < n_box) {
          const int row = (((pg * p.cfg.Hkv) + pc.h) << p.pages.shift) + ((j0 + b * p.box) & ((1 << p.pages.shift) - 1));
#pragma unroll
          for (int x = 0; x < kHalves; ++x) {
            tma_load_3d(dst + x * (kBN * 128) + b * p.box * 128, &tmK, x * 64, row, 0, bar(KV_FULL + st));
            tma_load_3d(dst + L::kTile + x * (kBN * 128) + b * p.box * 128, &tmV, x * 64, row, 0, bar(KV_FULL + st));
          }
        }
        __syncwarp();
      }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) atomicMax(p.d_status, (int)CHECK_PAGE_RANGE);
#pragma unroll 1
    for (uint32_t i = 0; i < kStages; ++i)                // no copy of this CTA outlives it
      if (T > i) drain_bar(bar(KV_FULL + (T - 1 - i) % kStages), ((T - 1 - i) / kStages) & 1u);
#pragma unroll 1
    for (uint32_t i = 0; i < kRing; ++i)
      if (f > i) drain_bar(bar(FR_FULL + (f - 1 - i) % kRing), ((f - 1 - i) / kRing) & 1u);
  } else {
    // ================= consumers =================
    const int parity = warp >> 2, q16 = (warp & 3) * 16;  // tiles of this parity, slots q16 .. q16 + 15 of each
    const int grp = lane >> 2, qd = lane & 3;             // accumulator rows grp, grp + 8; columns 2 qd, 2 qd + 1 of 8
    const float sl2 = p.scale * kLog2e;
    uint32_t f = 0, T = 0, joins = 0;
    auto join = [&]() {                                   // all consumers
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(JOIN));
      wait(JOIN, joins++);
    };
    float* sO = reinterpret_cast<float*>(smem_raw + L::kO);
    float2* sMl = reinterpret_cast<float2*>(smem_raw + L::kMl);
    while (true) {
      if (!wait(FR_FULL + f % kRing, f / kRing)) break;
      const Piece pc = ring[f % kRing];
      if (pc.tile0 < 0) break;
      // queries: row = token x group member, swizzled 16-byte pieces
      uint32_t qf[kD / 16][4];
      {
        const uint32_t sq = base + L::kQ + (f % kRing) * L::kQTile;
#pragma unroll
        for (int ks = 0; ks < kD / 16; ++ks) {
          const int c = ks * 2 + (lane >> 4);
          ldsm_x4(sq + (c >> 3) * (kRows * 128) + blk_off(lane & 15, c & 7), qf[ks]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(FR_FREE + f % kRing));
      Seq sq;
      sq.first = pc.first; sq.n = pc.n; sq.base = pc.base;
      const int last_tok = min((pc.r + 1) * p.cfg.tokens, pc.n) - 1;
      const int vis0 = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + grp / G, last_tok));
      const int vis1 = visible(p.seqs, sq, min(pc.r * p.cfg.tokens + (grp + 8) / G, last_tok));
      float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
      float o[kD / 8][4];
#pragma unroll
      for (int i = 0; i < kD / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

      const uint32_t Tend = T + (uint32_t)(pc.tile1 - pc.tile0);
#pragma unroll 1
      for (int t = pc.tile0 + (int)((T ^ (uint32_t)parity) & 1u); t < pc.tile1; t += 2) {
        const uint32_t Tt = T + (uint32_t)(t - pc.tile0), st = Tt % kStages;
        const uint32_t sK = base + L::kKv + st * 2 * L::kTile, sV = sK + L::kTile;
        wait(KV_FULL + st, Tt / kStages);
        const int j0 = t * kBN + q16;                     // this warp's first slot
        // slots that not every row sees: value rows that no row sees are cleared, and so are infinities and NaN among
        // those that only some rows see (they are added to the rows that do); a zero weight times them is not zero
        const bool edge = j0 + 16 > pc.seen0;
        bool cleared = false;
        if (__builtin_expect(edge, 0)) {
#pragma unroll 1
          for (int i = lane; i < 16 * (kD / 8); i += 32) {
            const int r = i / (kD / 8), c = i % (kD / 8), j = j0 + r;
            const uint32_t at = sV + (c >> 3) * (kBN * 128) + blk_off(q16 + r, c & 7);
            if (j >= pc.seen) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
          }
          __syncwarp();
          const int z0 = max(j0, pc.seen0), z1 = min(j0 + 16, pc.seen);
          uint32_t hit = 0;
#pragma unroll 1
          for (int i = lane; i < (z1 - z0) * (kD / 2); i += 32) {
            const int r = q16 + z0 - j0 + i / (kD / 2), c = i % (kD / 2);
            const uint32_t at = sV + (c >> 5) * (kBN * 128) + blk_off(r, (c >> 2) & 7) + (c & 3) * 4;
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
            const uint32_t old = v;
            if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
            if ((v & 0x7f800000u) == 0x7f800000u) v &= 0x0000ffffu;
            if (v != old) {
              hit = 1;
              asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
            }
          }
          cleared = __any_sync(0xffffffffu, hit != 0);
          fence_proxy_async();                            // the stage is refilled by TMA
          __syncwarp();
        }
        // ---- S = Q K^T, 16 slots ----
        float s[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
        const int mi = lane >> 3;
#pragma unroll
        for (int ks = 0; ks < kD / 16; ++ks) {
          const int r = q16 + (lane & 7) + (mi >> 1) * 8, c = ks * 2 + (mi & 1);
          uint32_t b[4];
          ldsm_x4(sK + (c >> 3) * (kBN * 128) + blk_off(r, c & 7), b);
          mma_bf16(s[0], qf[ks], b[0], b[1]);
          mma_bf16(s[1], qf[ks], b[2], b[3]);
        }
        if (__builtin_expect(edge, 0)) {
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const int j = j0 + nt * 8 + qd * 2;
            if (j >= vis0) s[nt][0] = -INFINITY;
            if (j + 1 >= vis0) s[nt][1] = -INFINITY;
            if (j >= vis1) s[nt][2] = -INFINITY;
            if (j + 1 >= vis1) s[nt][3] = -INFINITY;
          }
        }
        // ---- online softmax (exp2 domain) ----
        float mx0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
        float mx1 = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
        mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
        mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
        const float mn0 = fmaxf(m0, mx0 * sl2), mn1 = fmaxf(m1, mx1 * sl2);
        const float mu0 = mn0 == -INFINITY ? 0.f : mn0, mu1 = mn1 == -INFINITY ? 0.f : mn1;
        if (__any_sync(0xffffffffu, mn0 != m0 || mn1 != m1)) {
          const float c0 = fast_exp2(m0 - mu0), c1 = fast_exp2(m1 - mu1);
          l0 *= c0;
          l1 *= c1;
#pragma unroll
          for (int dt = 0; dt < kD / 8; ++dt) {
            o[dt][0] *= c0; o[dt][1] *= c0; o[dt][2] *= c1; o[dt][3] *= c1;
          }
          m0 = mn0;
          m1 = mn1;
        }
        uint32_t pf[4], pl[4];                            // upper and lower parts of the weights
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          const float p0 = fast_exp2(fmaf(s[nt][0], sl2, -mu0)), p1 = fast_exp2(fmaf(s[nt][1], sl2, -mu0));
          const float p2 = fast_exp2(fmaf(s[nt][2], sl2, -mu1)), p3 = fast_exp2(fmaf(s[nt][3], sl2, -mu1));
          l0 += p0 + p1;
          l1 += p2 + p3;
          pf[nt * 2] = upper_parts(p0, p1);
          pf[nt * 2 + 1] = upper_parts(p2, p3);
          pl[nt * 2] = pack_bf16(lower_part(p0), lower_part(p1));
          pl[nt * 2 + 1] = pack_bf16(lower_part(p2), lower_part(p3));
        }
        // ---- O += P V ----
#pragma unroll
        for (int dp = 0; dp < kD / 16; ++dp) {
          const int r = q16 + (lane & 7) + (mi & 1) * 8, c = dp * 2 + (mi >> 1);
          uint32_t b[4];
          ldsm_x4_t(sV + (c >> 3) * (kBN * 128) + blk_off(r, c & 7), b);
          mma_bf16(o[dp * 2], pl, b[0], b[1]);
          mma_bf16(o[dp * 2 + 1], pl, b[2], b[3]);
          mma_bf16(o[dp * 2], pf, b[0], b[1]);
          mma_bf16(o[dp * 2 + 1], pf, b[2], b[3]);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(KV_FREE + st));
        if (__builtin_expect(cleared, 0)) {               // back into the rows that see them
#pragma unroll 1
          for (int j = max(j0, pc.seen0); j < min(j0 + 16, pc.seen); ++j) {
            bool bad = false;
            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.pages.V) + page_offset(p.pages, pc.s, j, pc.h, p.cfg.Hkv, kD, &bad);
#pragma unroll
            for (int dt = 0; dt < kD / 8; ++dt) {
              const float a = __bfloat162float(v[dt * 8 + qd * 2]), b = __bfloat162float(v[dt * 8 + qd * 2 + 1]);
              if (!(fabsf(a) < INFINITY)) {
                if (j < vis0) o[dt][0] += a;
                if (j < vis1) o[dt][2] += a;
              }
              if (!(fabsf(b) < INFINITY)) {
                if (j < vis0) o[dt][1] += b;
                if (j < vis1) o[dt][3] += b;
              }
            }
          }
        }
      }
      T = Tend;
      // ---- the piece's result: eight partial ones ----
#pragma unroll
      for (int x = 1; x <= 2; x <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, x);
        l1 += __shfl_xor_sync(0xffffffffu, l1, x);
      }
      if (qd == 0) {
        sMl[warp * kRows + grp] = make_float2(m0, l0);
        sMl[warp * kRows + grp + 8] = make_float2(m1, l1);
      }
      float* mine = sO + warp * kRows * kD;
#pragma unroll
      for (int dt = 0; dt < kD / 8; ++dt) {
        *reinterpret_cast<float2*>(mine + grp * kD + dt * 8 + qd * 2) = make_float2(o[dt][0], o[dt][1]);
        *reinterpret_cast<float2*>(mine + (grp + 8) * kD + dt * 8 + qd * 2) = make_float2(o[dt][2], o[dt][3]);
      }
      join();
      const bool store = *s_fail == 0;
      const int n_rows = min(p.cfg.tokens, pc.n - pc.r * p.cfg.tokens) * G;
      constexpr int kVecs = kD / 4;
      auto write_row = [&](int row, int c4, const float* acc, float M, float Ls) {
        const float inv = Ls == 0.f ? 0.f : 1.0f / Ls;
        const int tok = pc.first + pc.r * p.cfg.tokens + row / G, hq = pc.h * G + row % G;
        uint2 v;
        v.x = pack_bf16(acc[0] * inv, acc[1] * inv);
        v.y = pack_bf16(acc[2] * inv, acc[3] * inv);
        if (Ls == 0.f) v = make_uint2(0, 0);
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.O.data) + (size_t)tok * p.O.ts + (size_t)hq * p.O.hs + c4 * 4) = v;
        if (c4 == 0 && p.lse != nullptr) p.lse[(size_t)tok * p.Hq + hq] = Ls == 0.f ? -INFINITY : M * kLn2 + logf(Ls);
      };
#pragma unroll 1
      for (int i = tid; i < n_rows * kVecs; i += kConsumers * 32) {
        const int row = i / kVecs, c4 = i % kVecs;
        float M = -INFINITY, Ls = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kConsumers; ++k) {
          const float2 x = sMl[k * kRows + row];
          if (x.y != 0.f) M = fmaxf(M, x.x);
        }
#pragma unroll
        for (int k = 0; k < kConsumers; ++k) {
          const float2 x = sMl[k * kRows + row];
          if (x.y == 0.f) continue;                       // a warp that saw nothing of this row
          const float w = fast_exp2(x.x - M);
          const float4 v = *reinterpret_cast<const float4*>(sO + (k * kRows + row) * kD + c4 * 4);
          Ls += x.y * w;
          acc[0] = fmaf(v.x, w, acc[0]);
          acc[1] = fmaf(v.y, w, acc[1]);
          acc[2] = fmaf(v.z, w, acc[2]);
          acc[3] = fmaf(v.w, w, acc[3]);
        }
        if (pc.slot < 0) {
          if (store) write_row(row, c4, acc, M, Ls);
        } else {
          *reinterpret_cast<float4*>(p.part_o + ((size_t)pc.slot * kRows + row) * kD + c4 * 4) =
              make_float4(acc[0], acc[1], acc[2], acc[3]);
          if (c4 == 0) p.part_ml[pc.slot * kRows + row] = make_float2(M, Ls);
        }
      }
      if (pc.slot >= 0) {
        // whoever takes the last ticket of a cut item merges its pieces in their order
        __threadfence();
        join();
        if (tid == 0) *s_merge = last_piece(p.d_status, pc.ticket, pc.n_pieces);
        join();
        if (*s_merge) {
          __threadfence();
#pragma unroll 1
          for (int i = tid; i < n_rows * kVecs; i += kConsumers * 32) {
            const int row = i / kVecs, c4 = i % kVecs;
            float M = -INFINITY, Ls = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (int k = 0; k < pc.n_pieces; ++k) {
              const float2 x = __ldcg(p.part_ml + piece_slot(pc, k) * kRows + row);
              if (x.y != 0.f) M = fmaxf(M, x.x);
            }
#pragma unroll 4
            for (int k = 0; k < pc.n_pieces; ++k) {
              const int slot = piece_slot(pc, k);
              const float2 x = __ldcg(p.part_ml + slot * kRows + row);
              const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part_o + ((size_t)slot * kRows + row) * kD + c4 * 4));
              if (x.y == 0.f) continue;
              const float w = fast_exp2(x.x - M);
              Ls += x.y * w;
              acc[0] = fmaf(v.x, w, acc[0]);
              acc[1] = fmaf(v.y, w, acc[1]);
              acc[2] = fmaf(v.z, w, acc[2]);
              acc[3] = fmaf(v.w, w, acc[3]);
            }
            if (store) write_row(row, c4, acc, M, Ls);
          }
        }
      }
      join();                                             // the merge area may be written again
      ++f;
    }
  }
  __syncthreads();
  pdl_launch_dependents();
  if (tid == 0 && *s_fail) atomicMax(p.d_status, (int)CHECK_WAIT_TIMEOUT);
}

namespace pdec {
template <int kD>
static cudaError_t launch(const Params& p, const KvSource& kv, int ctas, cudaStream_t stream) {
  CUtensorMap q, k, v;
  const long long rows = ((long long)p.pages.n_pages * p.cfg.Hkv) << p.pages.shift;
  if (!make_rows_map(&q, p.Q.data, kD, p.Hq, p.seqs.n_tokens, p.Q.hs, p.Q.ts, p.cfg.G, p.cfg.tokens) ||
      !make_rows_map(&k, kv.pages.K, kD, rows, 1, kD, rows * kD, p.box, 1) ||
      !make_rows_map(&v, kv.pages.V, kD, rows, 1, kD, rows * kD, p.box, 1))
    return cudaErrorInvalidValue;
  auto kern = packed_decode_kernel<kD>;
  cudaError_t e = ensure_dynamic_smem<4000 + kD>(kern, Smem<kD>::kBytes);
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
}  // namespace pdec

size_t packed_decode_scratch_bytes(int d) { return (size_t)2 * kMaxPackedCtas * pdec::kRows * ((size_t)d * 4 + 8); }

cudaError_t launch_packed_decode(const samkv_packed_t& d, const Seqs& seqs, const KvSource& kv, const Rows& Q, float scale,
                                 const Rows& O, float* lse, const samkv_ctx_impl& h, cudaStream_t stream) {
  pdec::Params p = {};
  p.seqs = seqs;
  p.cfg.G = d.n_q_heads / d.n_kv_heads;
  p.cfg.Hkv = d.n_kv_heads;
  p.cfg.tokens = pdec::kRows / p.cfg.G;
  p.cfg.tile = pdec::kBN;
  p.cfg.fixed = 2 * pdec::kBN;
  p.cfg.min_chunk = 6 * pdec::kBN;
  p.pages = kv.pages;
  p.box = (1 << kv.pages.shift) < pdec::kBN ? 1 << kv.pages.shift : pdec::kBN;
  p.Q = Q;
  p.O = O;
  p.scale = scale;
  p.lse = lse;
  const int ctas = h.sm_count < kMaxPackedCtas ? h.sm_count : kMaxPackedCtas;
  char* ws = h.workspace + kStatusBytes;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)2 * ctas * pdec::kRows * d.head_dim * 4);
  p.d_status = h.d_status;
  p.Hq = d.n_q_heads;
  return d.head_dim == 128 ? pdec::launch<128>(p, kv, ctas, stream) : pdec::launch<64>(p, kv, ctas, stream);
}

}  // namespace samkv
