// Attention of ragged chunks of few rows over the paged cache, short walks: one token or a handful of drafted ones per sequence.
// Up to 16 or 32 rows (32 / G tokens, the G query heads of a KV head beside each other) are a unit of work; the products are
// warp-level (mma m16n8k16): a few short walks are bound by latency, and the set-up of the tcgen05 kernels alone takes as long as
// all of this one (five tokens over 1337 slots, 8 KV heads: 16.7 us there, 8.8 here).  Long walks of more than 16 rows would be
// bound by the warp-level products, about 24 clocks each.
//   producer warp:   per page one K and one V tile by TMA, 128-byte swizzle, into a ring of three stages; two blocks per SM
//   consumer warps:  one per stage and 16 rows, each takes every third page and keeps its rows' running maxima, sums and outputs;
//                    those of the same rows merge at the unit's end
// Two ways to cut a call, as in the one-token decode, by sizes alone: a cluster of blocks for each (sequence, KV head) shares its
// pages evenly and merges through distributed shared memory (one launch); or all pages, laid end to end, are dealt out in equal
// shares and the units that a boundary cuts are added up by a second kernel.
#include "chunk_walk.cuh"

namespace ug {
namespace {

using namespace sm100;

constexpr int PG = UNIGIST_PAGE_TOKENS;
constexpr int kStages = 3;
constexpr float kLn2 = 0.6931471805599453f;

__device__ unsigned int g_few_timeout = 0;

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_trans(uint32_t addr, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(addr) : "memory");
}
// D (16x8 fp32) += A (16x16 bf16, row) * B (16x8 bf16, col)
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

using Pages = Share<PG>;

// MT: tiles of 16 rows.  A consumer warp takes one of them with every third page, so that a page costs a warp the same whatever MT.
template <int D, int MT>
struct Few {
  static constexpr int kRows = 16 * MT, kConsumers = kStages * MT, kThreads = (kConsumers + 1) * 32;
  static constexpr int kSlab = PG * 128, kPage = kSlab * (D / 64), kStage = 2 * kPage;  // a K or V page; both
  static constexpr int kOffQ = kStages * kStage;  // the unit's rows; after its walk what the warps hand over; first of all the page counts
  static constexpr int kQBytes = 8192;
  static constexpr int kOffMl = kOffQ + kQBytes;  // [kStages][kRows] float2: the warps' maxima and sums
  static constexpr int kOffMerged = kOffMl + kStages * kRows * 8;  // [kRows] float2: the block's, for the cluster
  static constexpr int kOffBars = kOffMerged + kRows * 8;
  static constexpr int kBytes = kOffBars + 64 + 1024 /*align*/;
  static constexpr int kHandOver = kQBytes / (MT * 2 * 512);  // 8-dim tiles that two warps of each row tile hand over at a time
  static_assert((kThreads + 1 + kThreads / 32 + 1) * 8 <= kQBytes && kRows * D * 2 <= kQBytes && kRows * D * 4 <= kStage && D / 8 % kHandOver == 0, "");
};
static_assert(2 * (Few<128, 2>::kBytes + 1024) <= 233472, "two blocks per SM");
// Spills (ptxas): heads of 128 with two row tiles 56 bytes stored, 80 loaded; the others none.

// kFlat = false: grid (c, Hkv, S), clusters of c along x.  kFlat = true: a one-dimensional grid of shares.
template <int D, int MT, bool kFlat>
__global__ void __launch_bounds__((Few<D, MT>::kThreads), 2)
chunk_few_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ChunkParams P) {
  using F = Few<D, MT>;
  constexpr int kConsumers = F::kConsumers, kThreads = F::kThreads;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* gen = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar_full = base + F::kOffBars, bar_free = bar_full + 8 * kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_free + 8 * i, MT);
    }
    mbar_fence_init();
  }
  pdl_wait();  // nothing above touches global memory
  Pages walk;
  if constexpr (kFlat) {
    long long* first = reinterpret_cast<long long*>(gen + F::kOffQ);
    const int per = (P.seqs.S + kThreads - 1) / kThreads;
    cost_prefix<kThreads>(P.seqs.S, per, first, first + kThreads + 1, [&](int b) {
      int row0;
      const int n = P.seqs.rows(b, row0);
      return Pages::head_cost(P, n, P.seqs.len(b)) * P.Hkv;
    });
    walk.deal(P, first, per, first[kThreads]);
    __syncthreads();  // the counts have been read
    if (threadIdx.x == 0) P.parts[2 * blockIdx.x].valid = P.parts[2 * blockIdx.x + 1].valid = 0;
  } else {
    walk.seq = blockIdx.z, walk.hk = blockIdx.y, walk.u = 0;
    walk.load(P);
    __syncthreads();
  }
  // The next unit of the block: of its share; or of its sequence and head, with the rank's part of its pages.
  Unit x;
  auto next = [&]() {
    if constexpr (kFlat) {
      return walk.next(P, x);
    } else {
      if (walk.u >= walk.units) return false;
      walk.unit(P, x);
      x.j0 = (int)((long long)x.nt * blockIdx.x / gridDim.x), x.j1 = (int)((long long)x.nt * (blockIdx.x + 1) / gridDim.x);
      ++walk.u;
      return true;
    }
  };
  bool ok = true;
  int i0 = 0;  // ring position of the unit's first page

  if (warp == kConsumers) {
    // ------------------------------------------------------------ producer
    while (next()) {
      const int pages = (x.L + PG - 1) / PG;
      int batch = -1, mine = 0;
      for (int j = x.j0; j < x.j1 && ok; ++j) {
        const int page = x.nt - 1 - j, i = i0 + j - x.j0, st = i % kStages, use = i / kStages;
        if (page >> 5 != batch) {  // 32 entries of the table at a time, one per lane; a page that the sequence does not have reads as zero
          batch = page >> 5;
          mine = batch * 32 + lane < pages ? P.seqs.page(x.seq, batch * 32 + lane) : P.seqs.num_blocks;
        }
        const int p = __shfl_sync(0xffffffffu, mine, page & 31);
        const int row = p < P.seqs.num_blocks ? (p * P.Hkv + x.hk) * PG : P.seqs.num_blocks * P.Hkv * PG;
        if (use > 0) ok = mbar_wait_warp(bar_free + 8 * st, (use - 1) & 1);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t full = bar_full + 8 * st, dst = base + st * F::kStage;
          mbar_arrive_expect_tx(full, F::kStage);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl) tma_load_2d(dst + sl * F::kSlab, &tm_k, full, sl * 64, row);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl) tma_load_2d(dst + F::kPage + sl * F::kSlab, &tm_v, full, sl * 64, row);
        }
        __syncwarp();
      }
      i0 += x.j1 - x.j0;
      if (!kFlat) {  // the ring holds the results now; not the next unit's pages before they have been read
        cluster_sync();
        cluster_sync();
      }
    }
  } else {
    // ------------------------------------------------------------ consumers
    const int g = lane >> 2, qc = lane & 3;   // row of an 8-row group, column pair
    const int lr = lane & 7, lj = lane >> 3;  // ldmatrix: this lane supplies row lr of matrix lj
    const int stage = warp % kStages, mt = warp / kStages;
    const uint32_t sK = base + stage * F::kStage, sV = sK + F::kPage;
    float2* ml = reinterpret_cast<float2*>(gen + F::kOffMl);
    auto out_row = [&](int row) {  // of a row of the unit
      const int tok = fdiv(P.g_div, row);
      return (long long)(x.row0 + tok) * P.Hq + x.hk * P.G + (row - tok * P.G);
    };
    while (next()) {  // to the end even when a wait gave up: the warps meet at barriers
      const int rows = x.ntok * P.G, cnt = x.j1 - x.j0;
      // the unit's rows: 16 bytes a thread, swizzled like the tiles; rows that are none are zeros
      for (int e = threadIdx.x; e < F::kRows * (D / 8); e += kConsumers * 32) {
        const int r = e / (D / 8), c = e % (D / 8), tok = fdiv(P.g_div, r);
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) v = *reinterpret_cast<const uint4*>(P.q + (x.row0 + tok) * P.q_stride + (x.hk * P.G + (r - tok * P.G)) * D + c * 8);
        st_shared_v4(base + F::kOffQ + (c >> 3) * (F::kRows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), v);
      }
      named_barrier_sync(1, kConsumers * 32);
      float o[D / 8][4], m_run[2], l_run[2];
      int hi[2];  // last slot that the row sees
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        m_run[r] = -INFINITY, l_run[r] = 0.f;
        hi[r] = x.base + min(fdiv(P.g_div, mt * 16 + r * 8 + g), x.ntok - 1);
      }
      const bool busy = mt * 16 < rows;
      int j = x.j0 + (stage + kStages - i0 % kStages) % kStages;
      const bool any = j < x.j1 && busy;  // this warp has something to hand over
      for (; j < x.j1 && ok; j += kStages) {
        ok = mbar_wait_warp(bar_full + 8 * stage, (i0 + j - x.j0) / kStages & 1);
        if (!ok) break;
        // With two row tiles half a page at a time: the scores and weights of all 64 tokens beside the outputs would not fit the
        // 128 registers that two blocks of seven warps leave each thread.
        constexpr int kTok = MT == 1 ? PG : PG / 2, kTiles = kTok / 8;
        const int live = x.L - (x.nt - 1 - j) * PG;  // tokens of the page that are the sequence's
#pragma unroll 1
        for (int row0 = 0; row0 < PG && busy; row0 += kTok) {
          const int tok0 = (x.nt - 1 - j) * PG + row0;
          // S = Q K^T, fp32, in token tiles of 8
          float s[kTiles][4];
#pragma unroll
          for (int nt = 0; nt < kTiles; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
          for (int kq = 0; kq < D / 32; ++kq) {  // 32 dims: two k-steps
            uint32_t qa[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = mt * 16 + (lj & 1) * 8 + lr, chunk = (kq & 1) * 4 + 2 * h + (lj >> 1);
              ldsm_x4(base + F::kOffQ + (kq >> 1) * (F::kRows * 128) + r * 128 + ((chunk ^ (r & 7)) << 4), qa[h][0], qa[h][1], qa[h][2], qa[h][3]);
            }
#pragma unroll
            for (int nt = 0; nt < kTiles; ++nt) {
              const int t = row0 + 8 * nt + lr, chunk = (kq & 1) * 4 + lj;  // token and 16 bytes whose address this lane supplies
              uint32_t k0, k1, k2, k3;
              ldsm_x4(sK + (kq >> 1) * F::kSlab + t * 128 + ((chunk ^ lr) << 4), k0, k1, k2, k3);
              mma_bf16(s[nt], qa[0][0], qa[0][1], qa[0][2], qa[0][3], k0, k1);
              mma_bf16(s[nt], qa[1][0], qa[1][1], qa[1][2], qa[1][3], k2, k3);
            }
          }
          // running softmax: of row r * 8 + g this lane holds tokens 8 nt + 2 qc + {0, 1}
          uint32_t p[2][kTiles];
          const bool partly = tok0 + kTok - 1 > x.base;  // some row does not see all of them
          float f[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float mx = -INFINITY;
#pragma unroll
            for (int nt = 0; nt < kTiles; ++nt) {
              float s0 = s[nt][2 * r] * P.scale_log2, s1 = s[nt][2 * r + 1] * P.scale_log2;
              if (partly) {
                const int left = hi[r] - tok0 - (8 * nt + 2 * qc);
                s0 = left >= 0 ? s0 : -INFINITY;
                s1 = left >= 1 ? s1 : -INFINITY;
              }
              s[nt][2 * r] = s0, s[nt][2 * r + 1] = s1;
              mx = fmaxf(mx, fmaxf(s0, s1));
            }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            const float m_new = fmaxf(m_run[r], mx), m_use = m_new == -INFINITY ? 0.f : m_new;  // (nothing seen yet: weights of 0)
            f[r] = ex2(m_run[r] - m_use);
            m_run[r] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int nt = 0; nt < kTiles; ++nt) {
              const float p0 = ex2(s[nt][2 * r] - m_use), p1 = ex2(s[nt][2 * r + 1] - m_use);
              sum += p0 + p1;
              p[r][nt] = pack_bf16(p0, p1);
            }
            l_run[r] = l_run[r] * f[r] + sum;  // (this lane's tokens; the row's four lanes meet at the end)
          }
          if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f)) {
#pragma unroll
            for (int d = 0; d < D / 8; ++d) o[d][0] *= f[0], o[d][1] *= f[0], o[d][2] *= f[1], o[d][3] *= f[1];
          }
          // O += P V, k-steps of 16 tokens, pairs of 8-dim tiles.  What lies behind the sequence's end in its last page would
          // reach O through a weight of zero, an infinity or NaN too: it is taken out of the fragments.
#pragma unroll
          for (int np = 0; np < D / 16; ++np) {
            const int chunk = 2 * np + (lj >> 1);  // 16-byte chunk of the V row
#pragma unroll
            for (int ks = 0; ks < kTiles / 2; ++ks) {
              const int t = row0 + 16 * ks + (lj & 1) * 8 + lr;
              uint32_t v0, v1, v2, v3;
              ldsm_x4_trans(sV + (chunk >> 3) * F::kSlab + t * 128 + (((chunk & 7) ^ lr) << 4), v0, v1, v2, v3);
              if (live < PG) {  // a fragment holds tokens 16 ks + 2 qc + {0, 1}, and 8 further on
                const int at = row0 + 16 * ks + 2 * qc;
                auto mask = [&](int first) { return first + 1 < live ? 0xffffffffu : first < live ? 0x0000ffffu : 0u; };
                v0 &= mask(at), v2 &= mask(at), v1 &= mask(at + 8), v3 &= mask(at + 8);
              }
              mma_bf16(o[2 * np], p[0][2 * ks], p[1][2 * ks], p[0][2 * ks + 1], p[1][2 * ks + 1], v0, v1);
              mma_bf16(o[2 * np + 1], p[0][2 * ks], p[1][2 * ks], p[0][2 * ks + 1], p[1][2 * ks + 1], v2, v3);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_free + 8 * stage);
      }
      i0 += cnt;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 1);
        l_run[r] += __shfl_xor_sync(0xffffffffu, l_run[r], 2);
      }
      if (qc == 0) {
#pragma unroll
        for (int r = 0; r < 2; ++r)  // (scores that are NaN pass the maximum by; what the warps add up goes by it, so it becomes one too)
          ml[stage * F::kRows + mt * 16 + r * 8 + g] = make_float2(l_run[r] == l_run[r] ? m_run[r] : l_run[r], l_run[r]);
      }
      if constexpr (!kFlat) {
        // The warps' results lie in the ring, each in its own stage, [row][D] fp32 in 16-byte pieces whose place turns with the row;
        // all threads add them up, then the blocks of the cluster their shares of the rows over all the blocks' sums.
        auto piece = [&](int row, int d4) { return row * (D / 4) + (d4 ^ ((row & 7) << 1 & (D / 4 - 1))); };
        // Row tiles of one stage's warps lie one behind the other; a warp that has finished may write while the other still reads
        // the stage's page, so all wait for each other first.
        named_barrier_sync(1, kConsumers * 32);
        if (any) {
          float4* mine = reinterpret_cast<float4*>(gen + stage * F::kStage);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int d = 0; d < D / 8; ++d) {
              const int row = mt * 16 + r * 8 + g;
              float* to = reinterpret_cast<float*>(mine + piece(row, 2 * d + (qc >> 1))) + 2 * (qc & 1);
              *reinterpret_cast<float2*>(to) = make_float2(o[d][2 * r], o[d][2 * r + 1]);
            }
        }
        named_barrier_sync(1, kConsumers * 32);
        float2* merged = reinterpret_cast<float2*>(gen + F::kOffMerged);
        const int c = gridDim.x;
        for (int e = threadIdx.x; e < rows * (D / 4); e += kConsumers * 32) {
          const int row = e / (D / 4), d4 = e % (D / 4);
          float2 a[kStages];
          float M = -INFINITY, L = 0.f;
#pragma unroll
          for (int k = 0; k < kStages; ++k) a[k] = ml[k * F::kRows + row], M = fmaxf(M, a[k].x);
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < kStages; ++k) {
            if (a[k].x == -INFINITY) continue;  // (it may not have written any sums)
            const float w = ex2(a[k].x - M);
            const float4 y = reinterpret_cast<const float4*>(gen + k * F::kStage)[piece(row, d4)];
            acc.x += w * y.x, acc.y += w * y.y, acc.z += w * y.z, acc.w += w * y.w;
            L += w * a[k].y;
          }
          if (c > 1) {
            reinterpret_cast<float4*>(gen)[piece(row, d4)] = acc;
            if (d4 == 0) merged[row] = make_float2(M, L);
          } else if (ok) {
            const float inv = L != 0.f ? 1.f / L : 0.f;
            const long long out = out_row(row);
            *reinterpret_cast<uint2*>(P.o + out * D + 4 * d4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (P.lse && d4 == 0) P.lse[out] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
          }
        }
        cluster_sync();
        if (c > 1) {
          const int per = (rows * (D / 4) + c - 1) / c, e_end = min(((int)blockIdx.x + 1) * per, rows * (D / 4));
          for (int e = blockIdx.x * per + threadIdx.x; e < e_end; e += kConsumers * 32) {
            const int row = e / (D / 4), d4 = e % (D / 4);
            const uint32_t ml_at = base + F::kOffMerged + row * 8, o_at = base + piece(row, d4) * 16;
            float M = -INFINITY, L = 0.f;
#pragma unroll 8
            for (int k = 0; k < c; ++k) M = fmaxf(M, ld_cluster_f32(ml_at, k));
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
            for (int k = 0; k < c; ++k) {
              const float m = ld_cluster_f32(ml_at, k), w = m == -INFINITY ? 0.f : ex2(m - M);
              const float4 y = ld_cluster_v4(o_at, k);
              acc.x += w * y.x, acc.y += w * y.y, acc.z += w * y.z, acc.w += w * y.w;
              L += w * ld_cluster_f32(ml_at + 4, k);
            }
            const float inv = L != 0.f ? 1.f / L : 0.f;
            const long long out = out_row(row);
            *reinterpret_cast<uint2*>(P.o + out * D + 4 * d4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
            if (P.lse && d4 == 0) P.lse[out] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
          }
        }
        fence_proxy_async_smem();  // (what follows in the ring is written by the other proxy)
        cluster_sync();            // the peers have read this block's results
      } else {
        // The ring holds the next unit's pages already.  The first stage's warps take over what the others have found of their rows,
        // kHandOver 8-dim tiles at a time.
        named_barrier_sync(1, kConsumers * 32);  // every warp has finished its walk: the rows' place is free
        float fac[2][kStages];
        if (stage == 0) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float2 a[kStages];
            float M = -INFINITY;
#pragma unroll
            for (int k = 0; k < kStages; ++k) a[k] = ml[k * F::kRows + mt * 16 + r * 8 + g], M = fmaxf(M, a[k].x);
            const float use = M == -INFINITY ? 0.f : M;
            m_run[r] = M, l_run[r] = 0.f;
#pragma unroll
            for (int k = 0; k < kStages; ++k) fac[r][k] = ex2(a[k].x - use), l_run[r] += fac[r][k] * a[k].y;
          }
        }
        float4* room = reinterpret_cast<float4*>(gen + F::kOffQ) + mt * 2 * F::kHandOver * 32;
#pragma unroll
        for (int d0 = 0; d0 < D / 8; d0 += F::kHandOver) {
          if (stage > 0) {
#pragma unroll
            for (int d = 0; d < F::kHandOver; ++d)
              room[((stage - 1) * F::kHandOver + d) * 32 + lane] = make_float4(o[d0 + d][0], o[d0 + d][1], o[d0 + d][2], o[d0 + d][3]);
          }
          named_barrier_sync(1, kConsumers * 32);
          if (stage == 0) {
#pragma unroll
            for (int d = 0; d < F::kHandOver; ++d) {
              const float4 a = room[d * 32 + lane], b = room[(F::kHandOver + d) * 32 + lane];
              float(&v)[4] = o[d0 + d];
              v[0] = v[0] * fac[0][0] + a.x * fac[0][1] + b.x * fac[0][2];
              v[1] = v[1] * fac[0][0] + a.y * fac[0][1] + b.y * fac[0][2];
              v[2] = v[2] * fac[1][0] + a.z * fac[1][1] + b.z * fac[1][2];
              v[3] = v[3] * fac[1][0] + a.w * fac[1][1] + b.w * fac[1][2];
            }
          }
          named_barrier_sync(1, kConsumers * 32);
        }
        const bool whole = x.j0 == 0 && x.j1 == x.nt;
        if (stage == 0 && ok) {
          const long long slot = 2ll * blockIdx.x + (x.j0 == 0 ? 1 : 0);
          if (!whole && threadIdx.x == 0) {
            const Part part = {x.row0, x.ntok, x.hk, x.nt, x.j0, x.j1, 1, 0};
            P.parts[slot] = part;
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int row = mt * 16 + r * 8 + g;
            const float l = l_run[r], m = m_run[r];
            if (row >= rows) continue;
            if (whole) {
              const long long out = out_row(row);
              const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
              for (int d = 0; d < D / 8; ++d)
                *reinterpret_cast<uint32_t*>(P.o + out * D + 8 * d + 2 * qc) = pack_bf16(o[d][2 * r] * inv, o[d][2 * r + 1] * inv);
              if (P.lse && qc == 0) P.lse[out] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
            } else {
#pragma unroll
              for (int d = 0; d < D / 8; ++d)
                *reinterpret_cast<float2*>(P.part_o + ((slot * (D / 4) + 2 * d + (qc >> 1)) * P.slot_rows + row) * 4 + 2 * (qc & 1)) =
                    make_float2(o[d][2 * r], o[d][2 * r + 1]);
              if (qc == 0) P.part_ml[slot * P.slot_rows + row] = make_float2(m, l);
            }
          }
        }
      }
    }
  }
  if (!ok) atomicExch(&g_few_timeout, 1u);
}

// How a call is cut: `c` blocks for each (sequence, KV head), a cluster; or (c = 0) `shares` shares of all pages.  mt = 0: not here.
struct FewPlan {
  int mt, c, shares;
};
FewPlan few_plan(int S, int num_rows, int G, int Hkv, int max_blocks) {
  const long long pairs = (long long)S * Hkv, slots = sm_count() < 256 ? 2ll * sm_count() : 512, rows = (long long)num_rows * G;
  if (G > 32 || rows > 32ll * S) return {0, 0, 0};
  const int mt = num_rows <= S && G <= 16 ? 1 : 2;
  auto rounds = [&](long long pages) { return (pages + kStages - 1) / kStages; };
  // As many blocks as shorten the longest possible walk and as the chip holds at once (clusters do not leave their group of
  // SMs: of 2, 4, 8, 16 blocks it holds 148, 71, 33, 14).
  constexpr int kHeld[4] = {148, 71, 33, 14};
  int best = 1;
  for (int c = 2, i = 0; c <= 16 && pairs <= kHeld[i]; c *= 2, ++i)
    if (rounds((max_blocks + c - 1) / c) < rounds((max_blocks + best - 1) / best)) best = c;
  // Short walks stay with the clusters, longer ones are dealt out.
  const long long longest = rounds((max_blocks + best - 1) / best);
  if (longest <= (pairs * best <= slots ? 6 : 4)) return {mt, best, 0};
  // (Heads of 64, which alone come here: 64 sequences of 9000 slots, 4 heads a group, 4 tokens each 214 us; 8 tokens 248 us against 272
  // of the kernel for many rows.  But the lengths are on the device: of twelve sequences with 1 to 60 rows, 30 on average, some are
  // more than one unit here, 163 us against 114.)
  if (rows > 16ll * S) return {0, 0, 0};
  return {mt, 0, (int)slots};
}

template <int D, int MT>
int32_t go(const ChunkParams& P, const FewPlan& plan, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t st) {
  using F = Few<D, MT>;
  auto kern = chunk_few_kernel<D, MT, false>;
  if constexpr (D == 64) {  // (the calls of heads of 128 that are dealt out go to the kernel with the operands turned round)
    if (!plan.c) kern = chunk_few_kernel<D, MT, true>;
  } else if (!plan.c) {
    return fail(UNIGIST_ERR_UNSUPPORTED, "no kernel for this cut");
  }
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kBytes);
  if (e == cudaSuccess && plan.c > 8) e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return fail(UNIGIST_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  {
    KernelScope ks("chunk_few_kernel", st);
    launch_chained(kern, plan.c ? dim3(plan.c, P.Hkv, P.seqs.S) : dim3(plan.shares), F::kThreads, F::kBytes, st, plan.c ? plan.c : 1, mk, mv, P);
  }
  if (int32_t rc = check_launch("chunk attention kernel for few rows")) return rc;
  return plan.c ? UNIGIST_OK : launch_chunk_combine(P, D, plan.shares, st);
}

}  // namespace

int chunk_route(int S, int num_rows, int G, int Hkv, int D, int max_blocks) {
  const FewPlan plan = few_plan(S, num_rows, G, Hkv, max_blocks);
  if (plan.mt > 0 && plan.c > 0) return kChunkFew;
  if (D == 128 && G <= 32 && (long long)num_rows * G <= 32ll * S) return kChunkThin;
  return plan.mt > 0 ? kChunkFew : kChunkRows;
}

size_t chunk_few_scratch_bytes(int S, int num_rows, int Hq, int Hkv, int D, int max_blocks) {
  const FewPlan plan = few_plan(S, num_rows, Hq / Hkv, Hkv, max_blocks);
  return plan.c ? 256 : chunk_parts_bytes(plan.shares, 32, D);
}

int32_t launch_chunk_few(ChunkParams P, int D, const CUtensorMap& mk, const CUtensorMap& mv, void* ws, cudaStream_t st) {
  const FewPlan plan = few_plan(P.seqs.S, P.seqs.num_rows, P.G, P.Hkv, P.seqs.max_blocks);
  P.tpt = P.unit_tokens = 16 * plan.mt / P.G;
  P.unit_div = make_fastdiv(P.unit_tokens);
  P.unit_cost = 2 * PG, P.single_cost = 16, P.min_share = 5 * PG;
  if (!plan.c) set_chunk_parts(&P, ws, plan.shares, 32, D);
  if (plan.mt == 1) return D == 128 ? go<128, 1>(P, plan, mk, mv, st) : go<64, 1>(P, plan, mk, mv, st);
  return D == 128 ? go<128, 2>(P, plan, mk, mv, st) : go<64, 2>(P, plan, mk, mv, st);
}

int32_t chunk_few_timeout_flag(unsigned int** at) { return flag_address(at, g_few_timeout); }

}  // namespace ug
