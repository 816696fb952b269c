// Attention of ragged chunks of new tokens over the paged cache, on Blackwell tensor cores (tcgen05 + TMEM + TMA).  Query i
// of the n of a sequence whose cache holds L tokens (the chunk's own among them) sees slots 0 .. L - n + i.
//
// A query tile is 128 rows: tpt = 128 / G consecutive tokens, the G query heads of one KV head beside each other, so K and V
// are read for all of them at once, whatever the chunk's length.  A unit of work is two neighbouring tiles of a sequence and
// KV head that walk the keys from the diagonal down, 128 (two pages) a step, sharing the K / V tiles; the last tile of an
// odd number is a unit by itself, whose key tiles are taken in turn by the streams of both and added up at the end.
//
// One block per SM.  The walks of all units, laid end to end (their keys, and some more for a unit's fixed parts), are
// dealt out in equal shares, so that one request's few drafted tokens, a ragged batch and a long prompt's chunk keep every SM
// equally busy.  A unit inside one share is finished there; one that a share boundary cuts leaves a partial result per
// share (fp32 sums, row maxima and sums) that a second kernel adds up in order: the same bits every run.
//
// Roles: softmax warpgroups (a stream each, a query row per thread), then the TMA warp, the MMA issuer, and a warp that blanks
// what lies behind the sequence's end in its last V page (whatever is there, an infinity or NaN too, would reach O through a
// weight of zero).  Heads of 128: a query tile is a stream, with 128 columns of scores and of O in tensor memory.  Heads of 64: it
// is two streams, one for either half (page) of its key tiles, each with 64 columns of scores, a maximum, a sum and 64 columns of O
// of its own, which meet at the unit's end: four times the independent chains scores -> softmax -> P V of a step, and twice the
// warps for the exponentials.  The two streams of 128 columns that these heads had first fell into step, so that no exponentials
// were taken while both waited for their products (a step of 3050 clocks, 2500 now; one chunk of 4096 over 30000 slots, 12 / 4
// heads: 604 against 519 us, a mixed batch of 17: 117 against 111).
// Bound: few rows read K and V once (HBM); many are bound by the chain scores -> softmax -> P V of a step.
#include "chunk_walk.cuh"
#include "softmax_row.cuh"

namespace ug {
namespace {

constexpr int PG = UNIGIST_PAGE_TOKENS;
constexpr int BM = 128, BN = 128;
static_assert(kCols == BN && BN == 2 * PG, "a key tile is two pages, and a thread's row of scores");
constexpr uint32_t kTmemCols = 512;
// kHalves: streams of a query tile.
template <int D>
struct ChunkShape {
  static constexpr int kHalves = D == 64 ? 2 : 1;
  static constexpr int kStreams = 2 * kHalves, kSmWarps = 4 * kStreams;
  static constexpr int kStages = D == 64 ? 6 : 4;  // ring slots; K and V tiles alternate through them
  static_assert(kStages % 2 == 0, "V tiles take every other slot");
  static constexpr int kStageBytes = kHalves * 32 * 1024;  // rows on their way out; sums that meet
  static constexpr int kTmaWarp = kSmWarps, kMmaWarp = kSmWarps + 1, kBlankWarp = kSmWarps + 2;
  static constexpr int kThreads = (kSmWarps + 4) * 32;
  static constexpr int kRegsLaunch = D == 64 ? 96 : 168, kRegsSoftmax = D == 64 ? 104 : 216, kRegsOther = D == 64 ? 64 : 72;
  static_assert(kThreads * kRegsLaunch <= 65536 && kSmWarps / 4 * kRegsSoftmax + kRegsOther <= kThreads / 128 * kRegsLaunch,
                "register split exceeds the block's allocation");
};
constexpr int kEmuHalf = 2;  // of kEmuDen column pairs, exponentials of heads of 64 on the FMA pipe
constexpr float kRescaleThreshold = 8.0f;  // log2 units: O is rescaled only when the max grows by > 2^8
constexpr float LOG2E = 1.4426950408889634f;
// What a unit costs beside its steps, in keys (about 4 us and three steps, heads of 128 4 and two: the mixed batch takes 116, 108,
// 105, 105 us with 256, 330, 400, 480, one of heads of 128 340 with 256 and 348 with 220), and a step of a single query tile in
// sixteenths of one of two (heads of 64: 0.75 us against 1.3; of 128: 1.45 against 2.4).  No share is worth less than kMinShare.
constexpr int kUnitCost64 = 400, kUnitCost128 = 256, kSingleCost64 = 9, kSingleCost128 = 10, kMinShare = 280;

__device__ unsigned int g_chunk_timeout = 0;

template <int D>
struct ChunkSmem {
  static constexpr int kSlab = BM * 128;
  static constexpr int kTile = kSlab * (D / 64);
  static constexpr int kOffRing = 2 * kTile;
  static constexpr int kOffStage = kOffRing + ChunkShape<D>::kStages * kTile;
  static constexpr int kOffMl = kOffStage + ChunkShape<D>::kStageBytes;  // heads of 64: [stream][128] float2 (maximum, sum)
  static constexpr int kOffBars = kOffMl + (ChunkShape<D>::kHalves - 1) * 4096;
  static constexpr int kBytes = kOffBars + 512 + 1024 /*align*/;
};
static_assert(ChunkSmem<128>::kBytes <= 232448 && ChunkSmem<64>::kBytes <= 232448, "shared memory of a block");

// Of half a row of scores in registers (heads of 64): hidden columns (behind `hi`) become -inf; the maximum; and the pass of row_exp.
constexpr int kHalf = BN / 2;
__device__ __forceinline__ void half_mask(uint32_t (&sc)[kHalf], int hi) {
#pragma unroll
  for (int c = 0; c < kHalf / 32; ++c) {
    const uint32_t bits = chunk_mask(0, hi, c);
#pragma unroll
    for (int e = 0; e < 32; ++e) sc[c * 32 + e] = (bits >> e) & 1u ? sc[c * 32 + e] : 0xff800000u;
  }
}
__device__ __forceinline__ float half_max(const uint32_t (&sc)[kHalf]) {
  float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
  for (int e = 0; e < kHalf; e += 4) {
    m0 = max3<true>(m0, __uint_as_float(sc[e]), __uint_as_float(sc[e + 1]));
    m1 = max3<true>(m1, __uint_as_float(sc[e + 2]), __uint_as_float(sc[e + 3]));
  }
  return max2<true>(m0, m1);
}
__device__ __forceinline__ float half_exp(const uint32_t (&sc)[kHalf], uint32_t t_p, float scale_log2, float m) {
  uint64_t l01 = f32x2(0.f, 0.f), l23 = l01;
  const uint64_t scale2 = f32x2(scale_log2, scale_log2), negm2 = f32x2(-m, -m);
#pragma unroll
  for (int c = 0; c < kHalf / 32; ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int e = 0; e < 32; e += 4) {
      const int i0 = c * 32 + e;
      float x[4];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        f32x2_split(fma2(f32x2(__uint_as_float(sc[i0 + 2 * q]), __uint_as_float(sc[i0 + 2 * q + 1])), scale2, negm2),
                    x[2 * q], x[2 * q + 1]);
        if (((i0 / 2 + q) * kEmuHalf) % kEmuDen < kEmuHalf) {
          ex2_fma2(x[2 * q], x[2 * q + 1]);
        } else {
          x[2 * q] = ex2(x[2 * q]);
          x[2 * q + 1] = ex2(x[2 * q + 1]);
        }
      }
      l01 = add2(l01, f32x2(x[0], x[1]));
      l23 = add2(l23, f32x2(x[2], x[3]));
      pk[e / 2] = pack_bf16(x[0], x[1]);
      pk[e / 2 + 1] = pack_bf16(x[2], x[3]);
    }
    tmem_st(t_p + c * 16, pk);
  }
  float l0, l1, l2, l3;
  f32x2_split(l01, l0, l1);
  f32x2_split(l23, l2, l3);
  return (l0 + l1) + (l2 + l3);
}

// kWaves: one sequence of at least as many units as there are blocks (a kernel of its own: what the others carry along for it in
// their registers made a mixed batch 3 - 8 % longer).
// All of them spill (ptxas, bytes stored / loaded: heads of 64 168 / 240, with kWaves 324 / 444; heads of 128 284 / 344 and 460 / 616):
// it goes by the registers that a thread has at the launch, 96 and 168, whatever its role has later.
template <int D, bool kWaves>
__global__ void __launch_bounds__(ChunkShape<D>::kThreads, 1)
chunk_attn_sm100_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ChunkParams P) {
  using SM = ChunkSmem<D>;
  using SH = ChunkShape<D>;
  constexpr int kStages = SH::kStages, kHalves = SH::kHalves, kStreams = SH::kStreams, kThreads = SH::kThreads, kSmWarps = SH::kSmWarps;
  constexpr int kTmaWarp = SH::kTmaWarp, kMmaWarp = SH::kMmaWarp, kBlankWarp = SH::kBlankWarp;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* gen = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t sQ[2] = {base, base + SM::kTile};
  const uint32_t ring = base + SM::kOffRing;
  const uint32_t bars = base + SM::kOffBars;
  const uint32_t bar_q = bars, bar_qfree = bars + 8;
  const uint32_t bar_s = bars + 16, bar_p = bars + 48, bar_p2 = bars + 80, bar_o = bars + 96;  // + 8 * stream
  // A V tile that is to be blanked has arrived, + 8 * (ring slot / 2): V tiles take every other slot, and two short walks' last
  // pages can be on their way at once.
  const uint32_t bar_raw = bars + 128;
  const uint32_t bar_full = bar_raw + 4 * kStages, bar_empty = bar_full + 8 * kStages, tmem_slot = bar_empty + 8 * kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(bar_q, 1);
    mbar_init(bar_qfree, 1);
    for (int i = 0; i < kStages / 2; ++i) mbar_init(bar_raw + 8 * i, 1);
    for (int i = 0; i < kStreams; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, 4);
      if (kHalves == 1) mbar_init(bar_p2 + 8 * i, 4);
      mbar_init(bar_o + 8 * i, 1);
    }
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 1);
    }
    mbar_fence_init();
  }
  if (warp == kMmaWarp) tmem_alloc(tmem_slot, kTmemCols);
  // Rows of a Q tile that no token fills (G does not divide 128) are zeros.
  for (int i = P.tpt * P.G * 8 + threadIdx.x; i < BM * 8; i += kThreads)
    for (int sl = 0; sl < 2 * (D / 64); ++sl) st_shared_v4(base + sl * SM::kSlab + i * 16, make_uint4(0u, 0u, 0u, 0u));
  fence_proxy_async_smem();
  pdl_wait();  // nothing above touches global memory
  long long* first = reinterpret_cast<long long*>(gen + SM::kOffStage);
  const int per = (P.seqs.S + kThreads - 1) / kThreads;
  cost_prefix<kThreads>(P.seqs.S, per, first, first + kThreads + 1, [&](int b) {
    int row0;
    const int n = P.seqs.rows(b, row0);
    return ug::Share<BN>::head_cost(P, n, P.seqs.len(b)) * P.Hkv;
  });
  using Share = ug::Share<BN, kWaves>;
  Share share;
  bool dealt = false;
  if constexpr (kWaves) dealt = share.template deal_waves<kThreads>(P, first);
  if (!dealt) share.deal(P, first, per, first[kThreads]);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(gen + SM::kOffBars + (tmem_slot - bars));
  bool ok = true;
  Unit x;
  // One query tile, taken by the streams of both; key tiles that tile i sees: [0, tiles_of(i)).
  auto is_single = [&](const Unit& it) { return it.ntok <= P.tpt; };
  auto tiles_of = [&](const Unit& it, int i) { return max(it.base + (i == 0 ? min(P.tpt, it.ntok) : it.ntok) - 1, 0) / BN + 1; };
  // A step whose V tile reaches into a page that the sequence fills only in part (a page it does not reach reads as zero).
  auto blanked = [&](const Unit& it, int j) { return j == 0 && it.L % PG != 0 && it.nt * BN > it.L; };

  if (warp >= kSmWarps) {
    reg_dealloc<SH::kRegsOther>();
    if (warp == kTmaWarp) {
      // ------------------------------------------------------------ TMA producer
      int t = 0, nq = 0;  // ring items, units
      while (ok && share.next(P, x)) {
        const int pages = (x.L + PG - 1) / PG;
        int batch = -1, mine = 0;
        // first row of a page of the cache; a page that the sequence does not have reads as zero
        auto row_of = [&](int page) {
          if (page >> 5 != batch) {  // 32 entries of the table at a time, one per lane
            batch = page >> 5;
            const int i = batch * 32 + lane;
            mine = i < pages ? P.seqs.page(x.seq, i) : P.seqs.num_blocks;
          }
          const int p = __shfl_sync(0xffffffffu, mine, page & 31);
          return p < P.seqs.num_blocks ? (p * P.Hkv + x.hk) * PG : P.seqs.num_blocks * P.Hkv * PG;
        };
        for (int j = x.j0; j < x.j1 && ok; ++j) {
          const int kt = x.nt - 1 - j, r1 = row_of(2 * kt + 1), r0 = row_of(2 * kt);
#pragma unroll
          for (int v = 0; v < 2; ++v, ++t) {
            const int slot = t % kStages, use = t / kStages;
            if (use > 0) ok = mbar_wait_warp(bar_empty + 8 * slot, (use - 1) & 1);
            if (!ok) break;
            if (lane == 0) {
              const uint32_t full = v && blanked(x, j) ? bar_raw + 8 * (slot / 2) : bar_full + 8 * slot, dst = ring + slot * SM::kTile;
              const CUtensorMap* m = v ? &tm_v : &tm_k;
              mbar_arrive_expect_tx(full, SM::kTile);
#pragma unroll
              for (int sl = 0; sl < D / 64; ++sl) {
                tma_load_2d(dst + sl * SM::kSlab, m, full, sl * 64, r0);
                tma_load_2d(dst + sl * SM::kSlab + PG * 128, m, full, sl * 64, r1);
              }
            }
            __syncwarp();
          }
          if (j == x.j0 && ok) {  // the unit's Q, behind its first keys: those need not wait for the unit before
            if (nq > 0) ok = mbar_wait_warp(bar_qfree, (nq - 1) & 1);
            if (!ok) break;
            ++nq;
            if (lane == 0) {
              const int tiles = is_single(x) ? 1 : 2;
              mbar_arrive_expect_tx(bar_q, tiles * P.tpt * P.G * D * 2);
              for (int i = 0; i < tiles; ++i) {
#pragma unroll
                for (int sl = 0; sl < D / 64; ++sl)
                  tma_load_3d(sQ[i] + sl * SM::kSlab, &tm_q, bar_q, sl * 64, x.hk * P.G, x.row0 + i * P.tpt);
              }
            }
            __syncwarp();
          }
        }
      }
    } else if (warp == kMmaWarp) {
      // ------------------------------------------------------------ MMA issuer
      // Streams in turn: P V of a stream, then its next scores, so that the softmax of the others runs under them.  (The loops over
      // the streams are unrolled: rolled, they took 588 us for 498.)
      if (elect_one()) {
        constexpr uint32_t leader = 1;
        constexpr uint32_t idesc_qk = make_idesc_bf16(BM, BN / kHalves, false, false);
        constexpr uint32_t idesc_pv = make_idesc_bf16(BM, D, false, true);
        constexpr uint32_t kHi = smem_desc_hi(1024);
        int n_pv[2] = {0, 0};  // products of a query tile's streams so far
        int t0 = 0, nu = 0;    // ring items and units before this one
        auto wait_full = [&](int t) { return mbar_wait(bar_full + 8 * (t % kStages), (t / kStages) & 1); };
        auto tile_of = [&](int t) { return ring + (t % kStages) * SM::kTile; };
        auto issue_s = [&](int i, int half, uint32_t q, uint32_t sK) {
          const uint32_t q_lo = smem_desc_lo(q, 16), k_lo = smem_desc_lo(sK + half * PG * 128, 16);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = ((kk / 4) * SM::kSlab + (kk % 4) * 32) >> 4;
            umma_ss(leader, tmem + i * 128 + half * 64, smem_desc_join(q_lo + off, kHi), smem_desc_join(k_lo + off, kHi), idesc_qk, kk > 0);
          }
          umma_commit(leader, bar_s + 8 * (i * kHalves + half));
        };
        // P V over half of the V tile: P's first column in tensor memory, the accumulator's
        auto issue_pv = [&](uint32_t t_p, uint32_t t_o, uint32_t sV, int half, bool fresh) {
          const uint32_t v_lo = smem_desc_lo(sV + half * PG * 128, SM::kSlab);
#pragma unroll
          for (int kk = 0; kk < PG / 16; ++kk)
            umma_ts(leader, t_o, t_p + kk * 8, smem_desc_join(v_lo + kk * (2048 >> 4), kHi), idesc_pv, !fresh || kk > 0 ? 1u : 0u);
        };
        auto step_pv = [&](int i, int half, uint32_t sV, bool fresh) {
          const uint32_t parity = n_pv[i] & 1, t = tmem + i * 128 + half * 64;
          ok = mbar_wait(bar_p + 8 * (i * kHalves + half), parity);
          if (!ok) return;
          tc_fence_after();
          issue_pv(t, t + 256, sV, half, fresh);
          if (kHalves == 1) {  // the first half of P is handed over while the softmax still works on the second
            ok = mbar_wait(bar_p2 + 8 * i, parity);
            if (!ok) return;
            tc_fence_after();
            issue_pv(t + 32, t + 256, sV, 1, false);
          }
          if (half == kHalves - 1) ++n_pv[i];
        };
        while (ok && share.next(P, x)) {
          const int cnt = x.j1 - x.j0;
          const bool single = is_single(x);
          ok = mbar_wait(bar_q, nu & 1);
          if (!ok) break;
          if (!single) {
            // step j of tile 0 only from its own diagonal tile on
            const int skip0 = max(x.nt - tiles_of(x, 0) - x.j0, 0);  // first steps that tile 0 does not see
            ok = wait_full(t0);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int st = 0; st < kStreams; ++st)
              if (st >= kHalves || skip0 == 0) issue_s(st / kHalves, st % kHalves, sQ[st / kHalves], tile_of(t0));
            umma_commit(leader, bar_empty + 8 * (t0 % kStages));
            if (cnt == 1) umma_commit(leader, bar_qfree);
            for (int j = 0; j < cnt && ok; ++j) {
              const int tv = t0 + 2 * j + 1, tk = tv + 1;
              ok = wait_full(tv);
#pragma unroll
              for (int st = 0; st < kStreams; ++st) {
                const int i = st / kHalves, half = st % kHalves;
                if (!ok) break;
                if (i || j >= skip0) step_pv(i, half, tile_of(tv), j == (i ? 0 : skip0));
                if (!ok) break;
                if (st == kStreams - 1) umma_commit(leader, bar_empty + 8 * (tv % kStages));
                if (j + 1 < cnt) {
                  if (st == 0) ok = wait_full(tk);
                  if (!ok) break;
                  tc_fence_after();
                  if (i || j + 1 >= skip0) issue_s(i, half, sQ[i], tile_of(tk));
                  if (st == kStreams - 1) {
                    umma_commit(leader, bar_empty + 8 * (tk % kStages));
                    if (j + 2 == cnt) umma_commit(leader, bar_qfree);
                  }
                } else if (i || skip0 < cnt) {
                  umma_commit(leader, bar_o + 8 * st);
                }
              }
            }
          } else {
            // the streams of both tiles take the one there is, those of tile j % 2 step j
            for (int j = 0; j < 2 && j < cnt && ok; ++j) {
              ok = wait_full(t0 + 2 * j);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int half = 0; half < kHalves; ++half) issue_s(j, half, sQ[0], tile_of(t0 + 2 * j));
              umma_commit(leader, bar_empty + 8 * ((t0 + 2 * j) % kStages));
              if (j + 1 == cnt) umma_commit(leader, bar_qfree);
            }
            for (int j = 0; j < cnt && ok; ++j) {
              const int i = j & 1, tv = t0 + 2 * j + 1, tk = tv + 3;
              ok = wait_full(tv);
#pragma unroll
              for (int half = 0; half < kHalves; ++half)
                if (ok) step_pv(i, half, tile_of(tv), j < 2);
              if (!ok) break;
              umma_commit(leader, bar_empty + 8 * (tv % kStages));
              if (j + 2 < cnt) {
                ok = wait_full(tk);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int half = 0; half < kHalves; ++half) issue_s(i, half, sQ[0], tile_of(tk));
                umma_commit(leader, bar_empty + 8 * (tk % kStages));
                if (j + 3 == cnt) umma_commit(leader, bar_qfree);
              } else {
                for (int half = 0; half < kHalves; ++half) umma_commit(leader, bar_o + 8 * (i * kHalves + half));
              }
            }
          }
          t0 += 2 * cnt;
          ++nu;
        }
      }
    } else if (warp == kBlankWarp) {
      // ------------------------------------------------------------ rows of the last V page behind the sequence's end
      int t0 = 0;            // ring items before the unit
      uint32_t parities = 0;  // of bar_raw
      while (ok && share.next(P, x)) {
        if (x.j0 == 0 && blanked(x, 0)) {
          const int tv = t0 + 1, s = tv % kStages / 2;
          ok = mbar_wait_warp(bar_raw + 8 * s, parities >> s & 1);
          if (!ok) break;
          parities ^= 1u << s;
          const int r0 = x.L - (x.nt - 1) * BN, r1 = (r0 + PG - 1) / PG * PG;  // rows [r0, r1) of the tile
          for (int e = r0 * 8 + lane; e < r1 * 8; e += 32) {
#pragma unroll
            for (int sl = 0; sl < D / 64; ++sl)
              st_shared_v4(ring + (tv % kStages) * SM::kTile + sl * SM::kSlab + e * 16, make_uint4(0u, 0u, 0u, 0u));
          }
          fence_proxy_async_smem();
          mbar_arrive_warp(bar_full + 8 * (tv % kStages));
        }
        t0 += 2 * (x.j1 - x.j0);
      }
    }
  } else {
    reg_alloc<SH::kRegsSoftmax>();
    // ------------------------------------------------------------ softmax + epilogue (one row per thread)
    const int st = warp / 4, i = st / kHalves, half = st % kHalves;  // stream: query tile, half of the key tiles
    const int r = (warp & 3) * 32 + lane;
    const int tok_r = fdiv(P.g_div, r);
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + i * 128 + half * 64 + lane_base, tO = tS + 256;
    // Room for 8 columns (the p-th of 32) of row rr of a warp's 32 rows on their way out: the warp's own, or what the thread has read
    // of the other half's sums (see below).
    auto stage_at = [&](int rr, int p) -> uint32_t {
      return SM::kOffStage + (kHalves == 2 ? st * 16384 + p * 4096 + ((warp & 3) * 32 + rr) * 16 : warp * 4096 + rr * 64 + ((p ^ (rr >> 1 & 3)) << 4));
    };
    if (threadIdx.x == 0) P.parts[2 * blockIdx.x].valid = P.parts[2 * blockIdx.x + 1].valid = 0;
    int n_s = 0, n_o = 0;  // tiles and units of the stream so far
    while (share.next(P, x)) {  // to the end even when a wait gave up: the streams meet at barriers
      const bool single = is_single(x);
      const int tile_tok0 = single ? 0 : i * P.tpt;                         // the tile's first token in the unit
      const int tile_tok = min(x.ntok - tile_tok0, P.tpt);                  // tokens
      const bool busy = (warp & 3) * 32 < tile_tok * P.G;                   // the warp has rows
      const bool real = r < tile_tok * P.G;
      const int hi_row = x.base + tile_tok0 + min(tok_r, tile_tok - 1);     // last slot that the row sees
      const int hi_all = x.base + tile_tok0;                                // ... that every row sees
      const int first_j = single ? x.j0 + i : max(x.j0, x.nt - tiles_of(x, i)), step = single ? 2 : 1;
      float m_run = -INFINITY, l_run = 0.f;
      int cnt = 0;
      for (int j = first_j; j < x.j1 && ok; j += step) {
        const int col0 = (x.nt - 1 - j) * BN;
        ok = mbar_wait_warp(bar_s + 8 * st, n_s & 1);
        if (!ok) break;
        tc_fence_after();
        ++n_s;
        if (!busy) {  // (what lies in its rows of P reaches its rows of O only)
          mbar_arrive_warp(bar_p + 8 * st);
          if (kHalves == 1) mbar_arrive_warp(bar_p2 + 8 * st);
          ++cnt;
          continue;
        }
        // A score that is NaN or without end leaves the row none: with a NaN for its maximum all of its weights are NaN.  (The weights
        // alone would not show it: those on the FMA pipe are numbers whatever comes in.)
        auto maximum = [&](float mx) {
          const float mx_s = mx * P.scale_log2;
          return mx_s < INFINITY ? mx_s : __int_as_float(0x7fffffff);
        };
        // Some row of this warp outgrew its running maximum: O is rescaled, and the exponentials are to be taken again.
        auto outgrown = [&](float mx) {
          const float mx_s = maximum(mx);
          const bool need = !(mx_s <= m_run + kRescaleThreshold);
          if (!__any_sync(0xffffffffu, need)) return false;
          const float m_new = need ? mx_s : m_run;
          const float f = need ? ex2(m_run - m_new) : 1.f;  // m_run = -inf gives 0
          l_run *= f;
          m_run = m_new;
          tmem_wait_st();
          constexpr int kAtOnce = kHalves == 2 ? 8 : 32;  // (the scores are in registers)
          if (cnt > 0) {
#pragma unroll 1
            for (int c = 0; c < D; c += kAtOnce) {
              uint32_t v[kAtOnce];
              tmem_ld(tO + c, v);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < kAtOnce; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
              tmem_st(tO + c, v);
            }
          }
          return true;
        };
        float mx, tile_sum;
        if constexpr (kHalves == 2) {
          uint32_t sc[kHalf];
#pragma unroll
          for (int c = 0; c < kHalf / 32; ++c) tmem_ld32(tS + c * 32, sc + c * 32);
          tmem_wait_ld();
          const int c0 = col0 + half * kHalf;
          if (c0 + kHalf - 1 > hi_all) half_mask(sc, hi_row - c0);
          // (the maximum first: kept for another pass, the scores would not fit the registers)
          mx = half_max(sc);
          if (cnt == 0) m_run = maximum(mx);
          else outgrown(mx);
          tile_sum = half_exp(sc, tS, P.scale_log2, m_run == -INFINITY ? 0.f : m_run);
        } else {
          uint32_t sc[kCols];
#pragma unroll
          for (int c = 0; c < kCols / 32; ++c) tmem_ld32(tS + c * 32, sc + c * 32);
          tmem_wait_ld();
          if (col0 + BN - 1 > hi_all) mask_row(sc, 0, hi_row - col0);
          if (cnt == 0) m_run = maximum(row_max<true>(sc));
          for (int pass = 0; pass < 2; ++pass) {
            tile_sum = row_exp<0, true>(sc, tS, P.scale_log2, m_run == -INFINITY ? 0.f : m_run, mx);
            if (!outgrown(mx)) break;
          }
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive_warp(bar_p + 8 * st);
          tile_sum += row_exp<1>(sc, tS, P.scale_log2, m_run == -INFINITY ? 0.f : m_run, mx);
        }
        l_run += tile_sum;
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_warp((kHalves == 2 ? bar_p : bar_p2) + 8 * st);
        ++cnt;
      }
      if (cnt > 0 && ok) {
        ok = mbar_wait_warp(bar_o + 8 * st, n_o & 1);
        tc_fence_after();
        ++n_o;
      }
      if (m_run == -INFINITY) l_run = 0.f;  // the row has seen nothing (what the exponentials gave for it is no weight)
      const bool whole = x.j0 == 0 && x.j1 == x.nt;
      const long long slot = 2ll * blockIdx.x + (x.j0 == 0 ? 1 : 0);
      if (threadIdx.x == 0 && !whole) {
        const Part part = {x.row0, x.ntok, x.hk, x.nt, x.j0, x.j1, 1, 0};
        P.parts[slot] = part;
      }
      // Out it goes, 32 columns of the sums at a time, in loops that stay rolled: unrolled they outgrow the instruction cache, and a
      // unit of few steps takes longer to leave than to walk.
      auto out_row = [&](int row) {  // of a row of the tile
        const int tok = fdiv(P.g_div, row);
        return (long long)(x.row0 + tile_tok0 + tok) * P.Hq + x.hk * P.G + (row - tok * P.G);
      };
      auto leave_stats = [&](float m, float l) {  // of row r
        if (!real || !ok) return;
        if (!whole)
          P.part_ml[slot * P.slot_rows + (single ? 0 : i * BM) + r] = make_float2(m, l);
        else if (P.lse)
          P.lse[out_row(r)] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
      };
      // Streams that hold sums of this tile's rows (of a single tile's one step those of tile 1 had none).
      const int joined = single && x.j1 - x.j0 > 1 ? 2 * kHalves : kHalves;
      if (single && joined == kHalves && i == 1) {
      } else if (joined == kHalves) {
        const bool mine = busy && ok;
        float m = m_run, l = l_run, f = 1.f, f_other = 0.f;
        if (kHalves == 2) {
          // A warpgroup finishes 32 columns of the rows and leaves its sums of the others to the other half's: [chunk of 4][row] of
          // the room that is the other's, its maximum and sum behind them.
          const uint32_t other = base + SM::kOffStage + (st ^ 1) * 16384 + r * 16;
#pragma unroll 1
          for (int p = 0; p < 4 && mine && cnt > 0; ++p) {
            uint32_t v[8];
            tmem_ld(tO + (1 - half) * 32 + p * 8, v);
            tmem_wait_ld();
            st_shared_v4(other + p * 4096, make_uint4(v[0], v[1], v[2], v[3]));
            st_shared_v4(other + p * 4096 + 2048, make_uint4(v[4], v[5], v[6], v[7]));
          }
          float2* ml = reinterpret_cast<float2*>(gen + SM::kOffMl);
          ml[st * BM + r] = make_float2(m_run, l_run);
          named_barrier_sync(4 + i, 256);
          const float2 y = ml[(st ^ 1) * BM + r];
          m = fmaxf(m_run, y.x);
          f = m_run == -INFINITY ? 0.f : ex2(m_run - m), f_other = y.x == -INFINITY ? 0.f : ex2(y.x - m);
          l = l_run * f + y.y * f_other;
        }
        const float inv_l = l != 0.f ? 1.f / l : 0.f;  // (a NaN stays one)
        if (whole) f *= inv_l, f_other *= inv_l;
#pragma unroll 1
        for (int c = half; c < (kHalves == 2 ? half + 1 : D / 32) && mine; ++c) {
          // (few columns at a time where many warps come here at once: it is the instructions that are waited for, 111 against 115 us of
          // a mixed batch; heads of 128 as many as there are, 358 against 375)
          constexpr int kPiece = kHalves == 2 ? 8 : 32;
#pragma unroll 1
          for (int p = 0; p < 32; p += kPiece) {
            uint32_t v[kPiece] = {};
            if (cnt > 0) {
              tmem_ld(tO + c * 32 + p, v);
              tmem_wait_ld();
            }
            // (the sums of a stream that has seen nothing of the row are not worth reading)
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[e] = f != 0.f ? __float_as_uint(__uint_as_float(v[e]) * f) : 0u;
            if (kHalves == 2 && f_other != 0.f) {
              const float4* y = reinterpret_cast<const float4*>(gen + SM::kOffStage + st * 16384 + p * 512 + r * 16);
#pragma unroll
              for (int e = 0; e < kPiece; e += 4) {
                const float4 z = y[e * 32];
                auto add = [&](uint32_t& x, float w) { x = __float_as_uint(fmaf(w, f_other, __uint_as_float(x))); };
                add(v[e], z.x), add(v[e + 1], z.y), add(v[e + 2], z.z), add(v[e + 3], z.w);
              }
            }
            if (whole) {
              auto two = [&](int k) { return pack_bf16(__uint_as_float(v[k]), __uint_as_float(v[k + 1])); };
#pragma unroll
              for (int e = 0; e < kPiece; e += 8)
                st_shared_v4(base + stage_at(lane, (p + e) / 8), make_uint4(two(e), two(e + 2), two(e + 4), two(e + 6)));
            } else if (real) {
              float4* to = reinterpret_cast<float4*>(P.part_o) + (slot * (D / 4) + c * 8 + p / 4) * P.slot_rows + (single ? 0 : i * BM) + r;
#pragma unroll
              for (int e = 0; e < kPiece; e += 4)
                to[(e >> 2) * P.slot_rows] = make_float4(__uint_as_float(v[e]), __uint_as_float(v[e + 1]), __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
            }
          }
          if (whole) {
            // rows leave through the warp's own room: straight from the registers an instruction would touch 32 rows
            __syncwarp();
#pragma unroll (kHalves == 2 ? 1 : 4)
            for (int q = 0; q < 4; ++q) {
              const int rr = q * 8 + (lane >> 2), row = (warp & 3) * 32 + rr;
              if (row < tile_tok * P.G)
                *reinterpret_cast<uint4*>(P.o + out_row(row) * D + c * 32 + (lane & 3) * 8) =
                    *reinterpret_cast<const uint4*>(gen + stage_at(rr, lane & 3));
            }
            __syncwarp();
          }
        }
        if (half == 0) leave_stats(m, l);
        if (kHalves == 2) named_barrier_sync(4 + i, 256);  // the room is free again
      } else {
        // The sums of the same rows meet in shared memory, weighed, as many columns at a time as there is room for, and all threads
        // that hold some add them up.
        constexpr int kBar = 3, kSumThreads = kSmWarps * 32;
        const int n_rows = tile_tok * P.G, room_rows = (n_rows + 31) & ~31;
        const int cols = min(D, room_rows <= 32 ? 128 : room_rows <= 64 ? 64 : 32);
        const int chunks = cols / 4, chunk_bits = 31 - __clz(chunks);  // chunks: 16 bytes of a row
        const int row_bits = 32 - __clz(n_rows - 1);
        const float4* room = reinterpret_cast<const float4*>(gen + SM::kOffStage);  // [stream][row][chunk], the chunk's place turned by the row
        float2* ml = reinterpret_cast<float2*>(gen + SM::kOffStage);                // [stream][row], before the sums
        ml[st * BM + r] = make_float2(m_run, l_run);
        named_barrier_sync(kBar, kSumThreads);
        float M = -INFINITY, l = 0.f;
        for (int g = 0; g < kStreams; ++g) M = fmaxf(M, ml[g * BM + r].x);
        for (int g = 0; g < kStreams; ++g) {
          const float2 y = ml[g * BM + r];
          if (y.x != -INFINITY) l += y.y * ex2(y.x - M);
        }
        named_barrier_sync(kBar, kSumThreads);
        float f = m_run == -INFINITY ? 0.f : ex2(m_run - M);
        if (whole) f *= l != 0.f ? 1.f / l : 0.f;
        if (st == 0) leave_stats(M, l);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += cols) {
#pragma unroll 1
          for (int c = 0; c < cols && busy; c += 32) {
            uint32_t v[32];
            tmem_ld32(tO + c0 + c, v);
            tmem_wait_ld();
            // (the sums of a stream that has seen nothing of the row are not worth reading)
            auto weighed = [&](int e) { return f != 0.f ? __float_as_uint(__uint_as_float(v[e]) * f) : 0u; };
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              st_shared_v4(base + SM::kOffStage + (((st * room_rows + r) * chunks + (((c + e) >> 2) ^ (r & 7))) << 4),
                           make_uint4(weighed(e), weighed(e + 1), weighed(e + 2), weighed(e + 3)));
          }
          named_barrier_sync(kBar, kSumThreads);
          // neighbouring threads write neighbouring pieces of a row, or of the partial sums' transposed rows
#pragma unroll 1
          for (int e = threadIdx.x; e < (whole ? n_rows << chunk_bits : chunks << row_bits); e += kSumThreads) {
            const int row = whole ? e >> chunk_bits : e & ((1 << row_bits) - 1), chunk = whole ? e & (chunks - 1) : e >> row_bits;
            if (row >= n_rows || !ok) continue;
            const float4* from = room + row * chunks + (chunk ^ (row & 7));
            const int apart = room_rows * chunks;
            float4 s = from[0];
            auto add = [&](const float4 y) { s.x += y.x, s.y += y.y, s.z += y.z, s.w += y.w; };
            add(from[apart]);
            if (kHalves == 2) add(from[2 * apart]), add(from[3 * apart]);
            if (whole)
              *reinterpret_cast<uint2*>(P.o + out_row(row) * D + c0 + chunk * 4) = make_uint2(pack_bf16(s.x, s.y), pack_bf16(s.z, s.w));
            else
              reinterpret_cast<float4*>(P.part_o)[(slot * (D / 4) + c0 / 4 + chunk) * P.slot_rows + row] = s;
          }
          named_barrier_sync(kBar, kSumThreads);  // the room is free again
        }
      }
      tc_fence_before();  // this stream's reads of O come before the next unit's products
    }
  }
  if (!ok) atomicExch(&g_chunk_timeout, 1u);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    __syncwarp();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Adds up the parts of the units that share boundaries cut.  A block takes 32 rows of the unit that begins in share blockIdx.x
// and ends in a later one, a lane a row, a warp D / 8 of its dims (partial sums lie transposed: a warp reads 512 contiguous bytes).
constexpr int kCombineThreads = 256;
constexpr int kMaxParts = 512;  // no more than there are shares, two an SM at most
template <int D>
__global__ void __launch_bounds__(kCombineThreads)
chunk_combine_kernel(const __grid_constant__ ChunkParams P) {
  constexpr int kVecs = D / 4 / (kCombineThreads / 32);
  pdl_wait();
  const Part head = P.parts[2 * blockIdx.x + 1];
  if (!head.valid) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.y * 32 + lane, tile = row / BM, r = row % BM, tok = tile * P.tpt + fdiv(P.g_div, r);
  const bool real = r < P.tpt * P.G && tok < head.ntok;
  if (!__syncthreads_or(real)) return;
  // the slots of the unit's parts, in order: the shares behind this one that hold the same unit
  __shared__ int slots[kMaxParts];
  __shared__ int n_slots;
  if (warp == 0) {
    int n = 1, done = head.j1;  // parts so far, steps of the unit's walk in them
    if (lane == 0) slots[0] = 2 * blockIdx.x + 1;
    for (int c0 = blockIdx.x + 1; done < head.nt && c0 < (int)gridDim.x; c0 += 32) {
      const int c = c0 + lane;
      const Part p = P.parts[2 * min(c, (int)gridDim.x - 1)];
      const bool mine = c < (int)gridDim.x && p.valid && p.row0 == head.row0 && p.hk == head.hk;
      const unsigned same = __ballot_sync(0xffffffffu, mine);
      if (mine) slots[n + __popc(same & ((1u << lane) - 1))] = 2 * c;
      n += __popc(same);
      done = max(done, __reduce_max_sync(0xffffffffu, mine ? p.j1 : 0));
    }
    if (lane == 0) n_slots = n;
  }
  __syncthreads();
  if (!real) return;
  float M = -INFINITY, sum = 0.f;
  bool none = false;  // some part holds a score that is no number
  float4 acc[kVecs];
#pragma unroll
  for (int q = 0; q < kVecs; ++q) acc[q] = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kLoads = 4;  // parts in flight
  const int n = n_slots;
  for (int s0 = 0; s0 < n; s0 += kLoads) {
    float2 ml[kLoads];
    float4 y[kLoads][kVecs];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const long long slot = slots[min(s0 + u, n - 1)];
      ml[u] = P.part_ml[slot * P.slot_rows + row];
      if (s0 + u >= n) ml[u].x = -INFINITY;
#pragma unroll
      for (int q = 0; q < kVecs; ++q)
        y[u][q] = reinterpret_cast<const float4*>(P.part_o)[(slot * (D / 4) + warp * kVecs + q) * P.slot_rows + row];
    }
    float m = M;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) m = fmaxf(m, ml[u].x), none |= ml[u].y != ml[u].y;
    if (m == -INFINITY) continue;  // nothing seen so far
    const float f = ex2(M - m);
    M = m;
    sum *= f;
#pragma unroll
    for (int q = 0; q < kVecs; ++q) acc[q].x *= f, acc[q].y *= f, acc[q].z *= f, acc[q].w *= f;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (ml[u].x == -INFINITY) continue;  // nothing seen there (its sums are not worth reading)
      const float g = ex2(ml[u].x - m);
      sum += ml[u].y * g;
#pragma unroll
      for (int q = 0; q < kVecs; ++q)
        acc[q].x += y[u][q].x * g, acc[q].y += y[u][q].y * g, acc[q].z += y[u][q].z * g, acc[q].w += y[u][q].w * g;
    }
  }
  const long long out = (long long)(head.row0 + tok) * P.Hq + head.hk * P.G + (r - (tok - tile * P.tpt) * P.G);
  if (none) sum = __int_as_float(0x7fffffff);
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  uint2 pk[kVecs];
#pragma unroll
  for (int q = 0; q < kVecs; ++q)
    pk[q] = sum != 0.f ? make_uint2(pack_bf16(acc[q].x * inv, acc[q].y * inv), pack_bf16(acc[q].z * inv, acc[q].w * inv)) : make_uint2(0u, 0u);
#pragma unroll
  for (int q = 0; q < kVecs; q += 2)
    *reinterpret_cast<uint4*>(P.o + out * D + (warp * kVecs + q) * 4) = make_uint4(pk[q].x, pk[q].y, pk[q + 1].x, pk[q + 1].y);
  if (P.lse && warp == 0) P.lse[out] = sum != 0.f ? (M + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

// Blocks of a call: no more than there can be steps.
int chunk_grid(int S, int num_rows, int G, int Hkv, int max_blocks) {
  const long long per = 2 * (BM / G), units = num_rows / per + (S < num_rows ? S : num_rows);
  const long long steps = units * Hkv * ((max_blocks + 1) / 2);
  const long long most = sm_count() < kMaxParts / 2 ? sm_count() : kMaxParts / 2;
  return (int)(steps < most ? (steps > 0 ? steps : 1) : most);
}
int chunk_slot_rows(int num_rows, int G) {
  return num_rows <= BM / G ? (num_rows * G + 31) / 32 * 32 : 2 * BM;
}

template <int D>
int32_t go(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const ChunkParams& P, int grid, cudaStream_t st) {
  const bool waves = P.seqs.S == 1 && (long long)(P.seqs.num_rows / P.unit_tokens) * P.Hkv >= grid;
  const auto kern = waves ? chunk_attn_sm100_kernel<D, true> : chunk_attn_sm100_kernel<D, false>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, ChunkSmem<D>::kBytes);
  if (e != cudaSuccess) return fail(UNIGIST_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  {
    KernelScope ks("chunk_attn_sm100_kernel", st);
    launch_chained(kern, dim3(grid), ChunkShape<D>::kThreads, ChunkSmem<D>::kBytes, st, 1, mq, mk, mv, P);
  }
  if (int32_t rc = check_launch("chunk attention kernel")) return rc;
  return launch_chunk_combine(P, D, grid, st);
}

}  // namespace

int32_t launch_chunk_combine(const ChunkParams& P, int D, int grid, cudaStream_t st) {
  if (grid == 1) return UNIGIST_OK;  // nothing is cut
  {
    KernelScope ks("chunk_combine_kernel", st);
    launch_chained(D == 128 ? chunk_combine_kernel<128> : chunk_combine_kernel<64>, dim3(grid, P.slot_rows / 32), kCombineThreads, 0, st, 1, P);
  }
  return check_launch("chunk combine kernel");
}

size_t chunk_attn_scratch_bytes(int S, int num_rows, int Hq, int Hkv, int D, int max_blocks) {
  if (num_rows < 1) return 0;
  const int G = Hq / Hkv;
  const int route = chunk_route(S, num_rows, G, Hkv, D, max_blocks);
  if (route == kChunkFew) return chunk_few_scratch_bytes(S, num_rows, Hq, Hkv, D, max_blocks);
  if (route == kChunkThin) return chunk_thin_scratch_bytes();
  return chunk_parts_bytes(chunk_grid(S, num_rows, G, Hkv, max_blocks), chunk_slot_rows(num_rows, G), D);
}

int32_t launch_chunk_attn(const ChunkBatch& b, int Hq, int Hkv, int D, float scale, const void* q, int64_t q_stride,
                          const void* kc, const void* vc, void* o, float* lse, void* ws, cudaStream_t st) {
  ChunkParams P = {};
  P.seqs = b;
  P.q = (const __nv_bfloat16*)q, P.q_stride = q_stride;
  P.o = (__nv_bfloat16*)o, P.lse = lse;
  P.Hq = Hq, P.Hkv = Hkv, P.G = Hq / Hkv;
  P.g_div = make_fastdiv(P.G);
  P.scale_log2 = scale * LOG2E;
  CUtensorMap mq, mk, mv;
  const long long rows = (long long)b.num_blocks * Hkv * PG;
  if (int32_t rc = encode_map_2d_bf16(&mk, kc, rows, D, PG, 64)) return rc;
  if (int32_t rc = encode_map_2d_bf16(&mv, vc, rows, D, PG, 64)) return rc;
  const int route = chunk_route(b.S, b.num_rows, P.G, Hkv, D, b.max_blocks);
  if (route == kChunkFew) return launch_chunk_few(P, D, mk, mv, ws, st);
  if (route == kChunkThin) return launch_chunk_thin(P, q, q_stride, mk, mv, ws, st);
  P.tpt = BM / P.G, P.unit_tokens = 2 * P.tpt;
  P.unit_cost = D == 128 ? kUnitCost128 : kUnitCost64, P.single_cost = D == 128 ? kSingleCost128 : kSingleCost64, P.min_share = kMinShare;
  P.unit_div = make_fastdiv(P.unit_tokens);
  const int grid = chunk_grid(b.S, b.num_rows, P.G, Hkv, b.max_blocks);
  set_chunk_parts(&P, ws, grid, chunk_slot_rows(b.num_rows, P.G), D);
  if (int32_t rc = encode_row_map(&mq, q, D, Hq, b.num_rows, q_stride, P.G, P.tpt)) return rc;
  return D == 128 ? go<128>(mq, mk, mv, P, grid, st) : go<64>(mq, mk, mv, P, grid, st);
}

int32_t chunk_attn_timeout_flag(unsigned int** at) { return flag_address(at, g_chunk_timeout); }

}  // namespace ug
