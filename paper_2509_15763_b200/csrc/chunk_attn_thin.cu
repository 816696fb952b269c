// Attention of ragged chunks of few rows over long caches (heads of 128): up to 32 rows of a KV head's queries against all its
// keys, on Blackwell tensor cores with the operands the other way round.  The 128 keys of a tile are the rows of the products and
// the queries their columns, so that a product costs what the queries fill and not 128 of them:
//   tcgen05:  S^T = K Q^T (128 keys x 32 queries),  O^T += V^T P (128 dims x 32 queries), both in TMEM
//   softmax:  four warps, a key per thread; a query's maximum lies across the threads, but it is needed only where the running one is
//             outgrown by more than 2^8 (the threads vote); sums of weights stay per thread until the unit's end.  P goes to shared
//             memory, [query][key].
// Bound by reading K and V once.  (As rows of 128 the queries of drafted tokens cost four times the products, under the power limit;
// as warp-level products twice the time of the memory.  64 sequences of 9216 slots, 1 to 8 tokens each: 432, 411 and 368 us.)
// Work is dealt out as in the kernel for many rows: shares of all walks, parts of cut units added up by a second kernel.
// Spills (ptxas): 8 bytes stored, 16 loaded.
#include "chunk_walk.cuh"

namespace ug {
namespace {

using namespace sm100;

constexpr int PG = UNIGIST_PAGE_TOKENS;
constexpr int D = 128, BN = 128, NQ = 32;  // head size, keys per tile, queries
constexpr int kStages = 6;                 // ring slots; K and V tiles alternate through them
constexpr int kSmWarps = 4, kTmaWarp = 4, kMmaWarp = 5, kBlankWarp = 6;
constexpr int kThreads = 256;
constexpr int kSBufs = 2, kPBufs = 2;
constexpr uint32_t kTmemCols = 128;  // S0 | S1 | O
constexpr float kThreshold = 8.0f;   // log2 units by which the running maximum may be outgrown

__device__ unsigned int g_thin_timeout = 0;

struct Thin {
  static constexpr int kSlab = BN * 128, kTile = 2 * kSlab;           // a K or V tile
  static constexpr int kOffQ = kStages * kTile, kQSlab = NQ * 128;    // the unit's rows; the share counts first
  static constexpr int kOffP = kOffQ + 2 * kQSlab;                    // [kPBufs] [query][key], 64 keys a slab
  static constexpr int kOffMax = kOffP + kPBufs * 2 * kQSlab;         // [4 warps][NQ] fp32
  static constexpr int kOffBars = kOffMax + kSmWarps * NQ * 4;
  static constexpr int kBytes = kOffBars + 256 + 1024 /*align*/;
  static_assert(kBytes <= 232448 && (kThreads + 1 + kThreads / 32 + 1) * 8 <= 2 * kQSlab, "");
};

using Tiles = Share<BN>;

// Column c of 32 lanes' 32 columns to lane c, by the given operation: 31 exchanges.
template <typename Op>
__device__ __forceinline__ float across_lanes(float (&v)[NQ], int lane, Op op) {
#pragma unroll
  for (int w = 16; w >= 1; w >>= 1) {
    const bool up = lane & w;
#pragma unroll
    for (int e = 0; e < w; ++e) {
      const float keep = up ? v[e + w] : v[e], give = up ? v[e] : v[e + w];
      v[e] = op(keep, __shfl_xor_sync(0xffffffffu, give, w));
    }
  }
  return v[0];
}
// Barrier among the softmax warps that tells whether any thread said yes.
__device__ __forceinline__ bool vote(bool yes) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "barrier.cta.red.or.pred q, 1, 128, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n" : "=r"(r) : "r"((uint32_t)yes) : "memory");
  return r != 0;
}

__global__ void __launch_bounds__(kThreads, 1)
chunk_thin_sm100_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ChunkParams P) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* gen = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bars = base + Thin::kOffBars;
  const uint32_t bar_q = bars, bar_qfree = bars + 8, bar_o = bars + 16;
  const uint32_t bar_s = bars + 24, bar_sfree = bar_s + 8 * kSBufs, bar_p = bar_sfree + 8 * kSBufs, bar_pfree = bar_p + 8 * kPBufs;
  // bar_raw: a V tile that is to be blanked has arrived, + 8 * (ring slot / 2)
  const uint32_t bar_raw = bar_pfree + 8 * kPBufs, bar_full = bar_raw + 4 * kStages, bar_empty = bar_full + 8 * kStages,
                 tmem_slot = bar_empty + 8 * kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(bar_q, 1);
    mbar_init(bar_qfree, 1);
    mbar_init(bar_o, 1);
    for (int i = 0; i < kSBufs; ++i) mbar_init(bar_s + 8 * i, 1), mbar_init(bar_sfree + 8 * i, kSmWarps);
    for (int i = 0; i < kPBufs; ++i) mbar_init(bar_p + 8 * i, kSmWarps), mbar_init(bar_pfree + 8 * i, 1);
    for (int i = 0; i < kStages / 2; ++i) mbar_init(bar_raw + 8 * i, 1);
    for (int i = 0; i < kStages; ++i) mbar_init(bar_full + 8 * i, 1), mbar_init(bar_empty + 8 * i, 1);
    mbar_fence_init();
  }
  if (warp == kMmaWarp) tmem_alloc(tmem_slot, kTmemCols);
  pdl_wait();  // nothing above touches global memory
  Tiles share;
  {
    long long* first = reinterpret_cast<long long*>(gen + Thin::kOffQ);
    const int per = (P.seqs.S + kThreads - 1) / kThreads;
    cost_prefix<kThreads>(P.seqs.S, per, first, first + kThreads + 1, [&](int b) {
      int row0;
      const int n = P.seqs.rows(b, row0);
      return Tiles::head_cost(P, n, P.seqs.len(b)) * P.Hkv;
    });
    share.deal(P, first, per, first[kThreads]);
    __syncthreads();  // the counts have been read
    // rows of the Q tile that no token fills (G does not divide 32) are zeros
    for (int i = P.tpt * P.G * 8 + threadIdx.x; i < NQ * 8; i += kThreads)
      for (int sl = 0; sl < 2; ++sl) st_shared_v4(base + Thin::kOffQ + sl * Thin::kQSlab + i * 16, make_uint4(0u, 0u, 0u, 0u));
    fence_proxy_async_smem();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(gen + Thin::kOffBars + (tmem_slot - bars));
  const uint32_t tO = tmem + kSBufs * NQ;
  Unit x;
  bool ok = true;
  // A step whose V tile reaches into a page that the sequence fills only in part (a page it does not reach reads as zero).
  auto blanked = [&](const Unit& it, int j) { return j == 0 && it.L % PG != 0 && it.nt * BN > it.L; };

  if (warp == kTmaWarp) {
    // ------------------------------------------------------------ TMA producer
    int t = 0, nq = 0;  // ring items, units
    while (ok && share.next(P, x)) {
      const int pages = (x.L + PG - 1) / PG;
      int batch = -1, mine = 0;
      auto row_of = [&](int page) {  // first row of a page of the cache; a page that the sequence does not have reads as zero
        if (page >> 5 != batch) {    // 32 entries of the table at a time, one per lane
          batch = page >> 5;
          mine = batch * 32 + lane < pages ? P.seqs.page(x.seq, batch * 32 + lane) : P.seqs.num_blocks;
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
            const uint32_t full = v && blanked(x, j) ? bar_raw + 8 * (slot / 2) : bar_full + 8 * slot, dst = base + slot * Thin::kTile;
            const CUtensorMap* m = v ? &tm_v : &tm_k;
            mbar_arrive_expect_tx(full, Thin::kTile);
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
              tma_load_2d(dst + sl * Thin::kSlab, m, full, sl * 64, r0);
              tma_load_2d(dst + sl * Thin::kSlab + PG * 128, m, full, sl * 64, r1);
            }
          }
          __syncwarp();
        }
        if (j == x.j0 && ok) {  // the unit's rows, behind its first keys: those need not wait for the unit before
          if (nq > 0) ok = mbar_wait_warp(bar_qfree, (nq - 1) & 1);
          if (!ok) break;
          ++nq;
          if (lane == 0) {
            mbar_arrive_expect_tx(bar_q, P.tpt * P.G * D * 2);
#pragma unroll
            for (int sl = 0; sl < 2; ++sl)
              tma_load_3d(base + Thin::kOffQ + sl * Thin::kQSlab, &tm_q, bar_q, sl * 64, x.hk * P.G, x.row0);
          }
          __syncwarp();
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ MMA issuer: the whole warp runs the loop, one lane issues
    const uint32_t leader = elect_one();
    constexpr uint32_t kHi = smem_desc_hi(1024);
    constexpr uint32_t idesc_s = make_idesc_bf16(BN, NQ, false, false), idesc_o = make_idesc_bf16(D, NQ, true, false);
    int t0 = 0, nu = 0, ns = 0, np = 0;  // ring items, units, scores and P V products before the next
    auto wait_full = [&](int t) { return mbar_wait_warp(bar_full + 8 * (t % kStages), (t / kStages) & 1); };
    auto issue_s = [&](int t) {
      const int buf = ns % kSBufs, use = ns / kSBufs;
      ok = wait_full(t);
      if (ok && use > 0) ok = mbar_wait_warp(bar_sfree + 8 * buf, (use - 1) & 1);
      if (!ok) return;
      ++ns;
      tc_fence_after();
      const uint32_t k_lo = smem_desc_lo(base + (t % kStages) * Thin::kTile, 16), q_lo = smem_desc_lo(base + Thin::kOffQ, 16);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        umma_ss(leader, tmem + buf * NQ, smem_desc_join(k_lo + (((kk / 4) * Thin::kSlab + (kk % 4) * 32) >> 4), kHi),
                smem_desc_join(q_lo + (((kk / 4) * Thin::kQSlab + (kk % 4) * 32) >> 4), kHi), idesc_s, kk > 0);
      umma_commit(leader, bar_s + 8 * buf);
      umma_commit(leader, bar_empty + 8 * (t % kStages));
    };
    while (ok && share.next(P, x)) {
      const int cnt = x.j1 - x.j0;
      ok = mbar_wait_warp(bar_q, nu & 1);
      if (!ok) break;
      issue_s(t0);
      if (ok && cnt == 1) umma_commit(leader, bar_qfree);
      for (int j = 0; j < cnt && ok; ++j) {
        if (j + 1 < cnt) {
          issue_s(t0 + 2 * j + 2);
          if (ok && j + 2 == cnt) umma_commit(leader, bar_qfree);
        }
        const int tv = t0 + 2 * j + 1, buf = np % kPBufs;
        if (ok) ok = wait_full(tv);
        if (ok) ok = mbar_wait_warp(bar_p + 8 * buf, (np / kPBufs) & 1);
        if (!ok) break;
        ++np;
        tc_fence_after();
        const uint32_t v_lo = smem_desc_lo(base + (tv % kStages) * Thin::kTile, Thin::kSlab), p_lo = smem_desc_lo(base + Thin::kOffP + buf * 2 * Thin::kQSlab, 16);
#pragma unroll
        for (int kk = 0; kk < BN / 16; ++kk)
          umma_ss(leader, tO, smem_desc_join(v_lo + kk * (2048 >> 4), kHi),
                  smem_desc_join(p_lo + (((kk / 4) * Thin::kQSlab + (kk % 4) * 32) >> 4), kHi), idesc_o, j > 0 || kk > 0);
        umma_commit(leader, bar_pfree + 8 * buf);
        umma_commit(leader, bar_empty + 8 * (tv % kStages));
      }
      if (ok) umma_commit(leader, bar_o);
      t0 += 2 * cnt;
      ++nu;
    }
  } else if (warp == kBlankWarp) {
    // ------------------------------------------------------------ rows of the last V page behind the sequence's end
    int t0 = 0, n_raw[kStages / 2] = {};
    while (ok && share.next(P, x)) {
      if (x.j0 == 0 && blanked(x, 0)) {
        const int tv = t0 + 1, s = tv % kStages / 2;
        int uses = 0;
#pragma unroll
        for (int i = 0; i < kStages / 2; ++i)
          if (i == s) uses = n_raw[i]++;
        ok = mbar_wait_warp(bar_raw + 8 * s, uses & 1);
        if (!ok) break;
        const int r0 = x.L - (x.nt - 1) * BN, r1 = (r0 + PG - 1) / PG * PG;  // rows [r0, r1) of the tile
        for (int e = r0 * 8 + lane; e < r1 * 8; e += 32) {
#pragma unroll
          for (int sl = 0; sl < 2; ++sl) st_shared_v4(base + (tv % kStages) * Thin::kTile + sl * Thin::kSlab + e * 16, make_uint4(0u, 0u, 0u, 0u));
        }
        fence_proxy_async_smem();
        mbar_arrive_warp(bar_full + 8 * (tv % kStages));
      }
      t0 += 2 * (x.j1 - x.j0);
    }
  } else if (warp < kSmWarps) {
    // ------------------------------------------------------------ softmax: a key per thread; at the end a dim per thread
    const int key = threadIdx.x;
    const uint32_t lane_base = static_cast<uint32_t>(warp * 32) << 16;
    float* wmax = reinterpret_cast<float*>(gen + Thin::kOffMax);
    // this key's place in a row of P
    const uint32_t p_at = base + Thin::kOffP + (key >> 6) * Thin::kQSlab + (key & 7) * 2;
    const uint32_t p_chunk = (key & 63) >> 3;
    if (threadIdx.x == 0) P.parts[2 * blockIdx.x].valid = P.parts[2 * blockIdx.x + 1].valid = 0;
    int n = 0, nu = 0;  // tiles, units so far
    // All four warps take the same way through here whatever their waits return: they meet at barriers.
    while (share.next(P, x)) {
      const int rows = x.ntok * P.G;
      const uint32_t row_bits = rows >= 32 ? 0xffffffffu : (1u << rows) - 1;
      float m[NQ], l[NQ];  // running maxima (log2 units, the same in all threads), this thread's sums of weights
#pragma unroll
      for (int q = 0; q < NQ; ++q) m[q] = -INFINITY, l[q] = 0.f;
      for (int j = x.j0; j < x.j1; ++j, ++n) {
        const int sb = n % kSBufs, pb = n % kPBufs, kpos = (x.nt - 1 - j) * BN + key;
        if (ok) ok = mbar_wait_warp(bar_s + 8 * sb, (n / kSBufs) & 1);
        tc_fence_after();
        uint32_t sc[NQ];
        tmem_ld32(tmem + sb * NQ + lane_base, sc);
        tmem_wait_ld();
        tc_fence_before();
        if (ok) mbar_arrive_warp(bar_sfree + 8 * sb);
        // the key is seen by rows of token kpos - base on
        const int q_lo = max(kpos - x.base, 0) < 32 ? max(kpos - x.base, 0) * P.G : 32;
        const uint32_t seen = q_lo < 32 ? row_bits & (0xffffffffu << q_lo) : 0u;
        float s[NQ];
        bool outgrown = false;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          s[q] = (seen >> q) & 1u ? __uint_as_float(sc[q]) * P.scale_log2 : -INFINITY;
          outgrown |= s[q] > m[q] + kThreshold;
        }
        if (vote(outgrown)) {
          // new maxima where the old ones were outgrown; what there is goes by them
          float v[NQ];
#pragma unroll
          for (int q = 0; q < NQ; ++q) v[q] = s[q];
          wmax[warp * NQ + lane] = across_lanes(v, lane, [](float a, float b) { return fmaxf(a, b); });
          named_barrier_sync(2, 128);
          float f[NQ];
#pragma unroll
          for (int q = 0; q < NQ; q += 4) {
            float4 t = *reinterpret_cast<const float4*>(wmax + q);
#pragma unroll
            for (int w = 1; w < kSmWarps; ++w) {
              const float4 y = *reinterpret_cast<const float4*>(wmax + w * NQ + q);
              t = make_float4(fmaxf(t.x, y.x), fmaxf(t.y, y.y), fmaxf(t.z, y.z), fmaxf(t.w, y.w));
            }
            const float top[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool need = top[e] > m[q + e] + kThreshold;
              f[q + e] = need ? ex2(m[q + e] - top[e]) : 1.f;  // (-inf: 0)
              m[q + e] = need ? top[e] : m[q + e];
              l[q + e] *= f[q + e];
            }
          }
          if (j > x.j0) {
            // O is stable once the P V of the step before has completed
            if (ok) ok = mbar_wait_warp(bar_pfree + 8 * ((n - 1) % kPBufs), ((n - 1) / kPBufs) & 1);
            tc_fence_after();
            uint32_t o[NQ];
            tmem_ld32(tO + lane_base, o);
            tmem_wait_ld();
#pragma unroll
            for (int q = 0; q < NQ; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * f[q]);
            tmem_st(tO + lane_base, o);
            tmem_wait_st();
          }
          named_barrier_sync(2, 128);  // the maxima have been read
        }
        if (ok && n >= kPBufs) ok = mbar_wait_warp(bar_pfree + 8 * pb, (n / kPBufs - 1) & 1);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const float p = (seen >> q) & 1u ? ex2(s[q] - (m[q] == -INFINITY ? 0.f : m[q])) : 0.f;
          l[q] += p;
          const uint32_t h = pack_bf16(p, 0.f);
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(p_at + pb * 2 * Thin::kQSlab + q * 128 + ((p_chunk ^ (q & 7)) << 4)), "h"((uint16_t)h) : "memory");
        }
        fence_proxy_async_smem();
        tc_fence_before();
        if (ok) mbar_arrive_warp(bar_p + 8 * pb);
      }
      if (ok) ok = mbar_wait_warp(bar_o, nu & 1);
      ++nu;
      tc_fence_after();
      uint32_t o[NQ];
      tmem_ld32(tO + lane_base, o);
      tmem_wait_ld();
      tc_fence_before();  // before the next unit's products
      // the rows' sums of weights meet
      const float mine = across_lanes(l, lane, [](float a, float b) { return a + b; });
      wmax[warp * NQ + lane] = mine;
      named_barrier_sync(2, 128);
      const bool whole = x.j0 == 0 && x.j1 == x.nt;
      const long long slot = 2ll * blockIdx.x + (x.j0 == 0 ? 1 : 0);
      if (threadIdx.x == 0 && !whole) {
        const Part part = {x.row0, x.ntok, x.hk, x.nt, x.j0, x.j1, 1, 0};
        P.parts[slot] = part;
      }
      // of row `lane`: the sum of its weights, and what its outputs are multiplied by
      const float my_sum = (wmax[lane] + wmax[NQ + lane]) + (wmax[2 * NQ + lane] + wmax[3 * NQ + lane]);
      const float my_inv = my_sum != 0.f ? 1.f / my_sum : 0.f;  // (a NaN stays one)
      float my_m = -INFINITY;
#pragma unroll
      for (int q = 0; q < NQ; ++q) my_m = q == lane ? m[q] : my_m;
      if (ok && lane < rows && warp == 0) {
        const int tok = fdiv(P.g_div, lane);
        if (!whole)
          P.part_ml[slot * P.slot_rows + lane] = make_float2(my_sum != 0.f ? my_m : -INFINITY, my_sum);
        else if (P.lse)
          P.lse[(long long)(x.row0 + tok) * P.Hq + x.hk * P.G + (lane - tok * P.G)] = my_sum != 0.f ? (my_m + log2f(my_sum)) * 0.6931471805599453f : -INFINITY;
      }
      if (ok && whole) {
        __nv_bfloat16* to = P.o + ((long long)x.row0 * P.Hq + x.hk * P.G) * D + key;
        int g = 0;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          if (q >= rows) break;
          const float inv = __shfl_sync(0xffffffffu, my_inv, q);
          *to = __float2bfloat16_rn(inv != 0.f ? __uint_as_float(o[q]) * inv : 0.f);
          const bool last = ++g == P.G;  // of the token
          to += last ? (long long)(P.Hq - P.G + 1) * D : D;
          g = last ? 0 : g;
        }
      } else if (ok) {
        float* to = P.part_o + (slot * (D / 4) + (key >> 2)) * P.slot_rows * 4 + (key & 3);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          if (q >= rows) break;
          to[4 * q] = __shfl_sync(0xffffffffu, my_inv, q) != 0.f ? __uint_as_float(o[q]) : 0.f;
        }
      }
      named_barrier_sync(2, 128);  // the sums have been read
    }
  }
  if (!ok) atomicExch(&g_thin_timeout, 1u);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    __syncwarp();
    tmem_dealloc(tmem, kTmemCols);
  }
}

}  // namespace

size_t chunk_thin_scratch_bytes() { return chunk_parts_bytes(chunk_thin_grid(), NQ, D); }

int32_t launch_chunk_thin(ChunkParams P, const void* q, int64_t q_stride, const CUtensorMap& mk, const CUtensorMap& mv, void* ws, cudaStream_t st) {
  const int grid = chunk_thin_grid();
  P.tpt = P.unit_tokens = NQ / P.G;
  P.unit_div = make_fastdiv(P.unit_tokens);
  P.unit_cost = 2 * BN, P.single_cost = 16, P.min_share = 3 * BN;
  set_chunk_parts(&P, ws, grid, NQ, D);
  CUtensorMap mq;
  if (int32_t rc = encode_row_map(&mq, q, D, P.Hq, P.seqs.num_rows, q_stride, P.G, P.tpt)) return rc;
  cudaError_t e = cudaFuncSetAttribute(chunk_thin_sm100_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Thin::kBytes);
  if (e != cudaSuccess) return fail(UNIGIST_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  {
    KernelScope ks("chunk_thin_sm100_kernel", st);
    launch_chained(chunk_thin_sm100_kernel, dim3(grid), kThreads, Thin::kBytes, st, 1, mq, mk, mv, P);
  }
  if (int32_t rc = check_launch("chunk attention kernel for few rows")) return rc;
  return launch_chunk_combine(P, D, grid, st);
}

int32_t chunk_thin_timeout_flag(unsigned int** at) { return flag_address(at, g_thin_timeout); }

}  // namespace ug
