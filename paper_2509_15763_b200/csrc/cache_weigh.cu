// Accumulated attention weights of a paged cache's slots, on Blackwell tensor cores (tcgen05 + TMEM + TMA):
//   weights_out[slot] = decay * weights_in[slot] + sum over the chunk's queries i that see the slot, and the query heads h
//                       of its KV head, of exp(scale * q_ih . k_slot - lse_ih).
// The log-sum-exp is given (the attention over the same cache left it), so there is no running maximum and a slot's sum needs
// nothing but its own key: a block owns keys and walks the queries, each key's sum stays in registers, nothing is added
// atomically and the result is the same bit for bit from run to run.
//
// A work item is one or two neighbouring tiles of 128 keys (two pages) of one KV head.  Per step it takes a tile of kBQ query
// rows (kBQ / G tokens, the G heads of a token beside each other) against them:
//   TMA:      the item's K tiles, the step's Q tile, each through a ring; 128-byte swizzle
//   tcgen05:  S^T = K Q^T - 1 lse^T / scale into TMEM, a tile per key tile and step, two buffers each.  The log-sum-exps are 16
//             more columns of the contraction: ones on the keys' side, on the queries' the number in three bf16 parts (24
//             bits).  (Read from shared memory by every thread they took as much of its bandwidth as the products' operands.)
//   weights:  a key per thread and kCols columns: 2^(s * scale_log2) summed over the columns
// The key tiles of all sequences and heads, laid end to end and weighed by the queries that see them, are dealt out in
// equal shares, one per SM.  A single token per sequence is bound by reading K once; there kBQ = 32 leaves the shared memory to
// K tiles on their way.  A chunk is bound by its exponentials (16 a clock and SM; the products take half as long).
#include "chunk_tma.cuh"

namespace ug {
namespace {

using namespace sm100;

constexpr int PG = UNIGIST_PAGE_TOKENS;
constexpr int BK = 128;  // keys per tile, two tiles per item
constexpr int kSBufs = 2;
constexpr float LOG2E = 1.4426950408889634f;

__device__ unsigned int g_weigh_timeout = 0;

template <int D, int BQ>
struct Weigh {
  // Warps that sum: 2 key tiles x kParts parts of the columns x 4 lane quarters.  Two parts of 64 columns where there are 128: one
  // warpgroup a tile leaves a scheduler two warps, which wait for each other's latencies (2048 tokens over 32768 slots, heads of
  // 128 and 64: 558 and 535 us; with two parts 544 and 499).
  static constexpr int kParts = BQ == 128 ? 2 : 1, kCols = BQ / kParts;
  static constexpr int kSumWarps = 8 * kParts, kTmaWarp = kSumWarps, kMmaWarp = kSumWarps + 1, kLseWarp = kSumWarps + 2;
  static constexpr int kThreads = (kSumWarps + 4) * 32;
  static constexpr int kKSlots = BQ == 128 ? 3 : 6, kQSlots = BQ == 128 ? 3 : 2;
  // shared memory
  static constexpr int kKSlab = BK * 128, kQSlab = BQ * 128;  // [rows x 64 bf16]
  static constexpr int kKTile = kKSlab * (D / 64), kQTile = kQSlab * (D / 64);
  static constexpr int kOffQ = kKSlots * kKTile;
  // [rows x 16 bf16], no swizzle: groups of 8 rows, in each two 8 x 8 matrices (128 bytes) beside each other
  static constexpr int kOffOnes = kOffQ + kQSlots * kQTile, kThinK = BK * 32, kThinQ = BQ * 32;
  static constexpr int kOffLse = kOffOnes + kThinK;  // [kQSlots]
  static constexpr int kOffFirst = kOffLse + kQSlots * kThinQ;                         // [kThreads + 1] 64-bit, and a number per warp
  static constexpr int kOffMeet = kOffFirst + (kThreads + 1 + kThreads / 32 + 1) * 8;  // [2][2 * BK] fp32
  static constexpr int kOffBars = kOffMeet + 2 * 2 * BK * 4;
  static constexpr int kBytes = kOffBars + 256 + 1024 /*align*/;
  static constexpr uint32_t kTmemCols = 2 * kSBufs * BQ;
};
static_assert(Weigh<128, 128>::kBytes <= 232448 && Weigh<128, 32>::kBytes <= 232448, "shared memory of a block");

struct WeighParams {
  ChunkBatch seqs;
  const float* lse;
  const float* w_in;
  float* w_out;
  int Hq, Hkv, G, tpt, tile_cost;  // tpt: tokens per step
  FastDiv g_div, tpt_div;
  float scale_log2, inv_scale, decay;
};

// One item: `tiles` tiles of 128 keys from key0 on of KV head hk of a sequence with n new rows (the first is row0) and length L;
// steps [t0, t1).
struct Item {
  int seq, hk, key0, tiles, n, row0, L, t0, t1;
};

// The items of a share.  Positions are in tokens: a key tile costs the tokens that see its first key, in whole steps, and
// P.tile_cost more for what it costs by itself; a tile belongs to the share in which it begins.
struct Share {
  int seq, hk, u, n, row0, L, units;  // u: the next tile of `units`
  long long at, end;                  // its position; the share's end

  static __device__ __forceinline__ int units_of(int L) { return (L + BK - 1) / BK; }
  static __device__ __forceinline__ long long steps_tokens(const WeighParams& P, int n) { return fdiv(P.tpt_div, n + P.tpt - 1) * (long long)P.tpt; }
  static __device__ __forceinline__ long long cost(const WeighParams& P, int n, int L, int u) {
    return P.tile_cost + steps_tokens(P, min(n, L)) - max(u * BK - max(L - n, 0), 0);
  }
  static __device__ __forceinline__ long long cost_before(const WeighParams& P, int n, int L, int u) {  // of the first u tiles
    const int base = max(L - n, 0), v0 = base / BK + 1;  // from tile v0 on the chunk's own keys come first
    const long long m = max(u - v0, 0);
    return u * (P.tile_cost + steps_tokens(P, min(n, L))) - (BK * (m * v0 + m * (m - 1) / 2) - m * base);
  }
  __device__ __forceinline__ void load(const WeighParams& P) {
    n = P.seqs.rows(seq, row0);
    L = P.seqs.len(seq);
    units = units_of(L);
  }
  __device__ __forceinline__ void start(const WeighParams& P, const long long* first, int per, long long begin) {
    at = begin;
    if (begin >= end) return;
    const int group = cost_group(first, (P.seqs.S - 1) / per, begin);
    long long left = begin - first[group], one;
    for (seq = group * per;; ++seq) {
      load(P);
      one = cost_before(P, n, L, units);
      if (left < one * P.Hkv) break;
      left -= one * P.Hkv;
    }
    hk = min((int)__fdividef((float)left, (float)one), P.Hkv - 1);  // (a 64-bit division takes longer than the two corrections)
    left -= hk * one;
    while (left < 0) --hk, left += one;
    while (left >= one) ++hk, left -= one;
    int lo = 0, hi = units;  // the first tile that begins at or behind `left`; `units`: none of this head
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (cost_before(P, n, L, mid) >= left) hi = mid; else lo = mid + 1;
    }
    u = lo;
    at += cost_before(P, n, L, u) - left;
  }
  __device__ __forceinline__ bool next(const WeighParams& P, Item& x) {
    if (at >= end) return false;
    if (u >= units) {
      u = 0;
      if (++hk >= P.Hkv) {
        hk = 0;
        do {
          if (++seq >= P.seqs.S) return false;
          load(P);
        } while (units == 0);
      }
    }
    x.seq = seq, x.hk = hk, x.n = n, x.row0 = row0, x.L = L;
    x.key0 = u * BK;
    at += cost(P, n, L, u++);
    x.tiles = 1;
    if (u < units && at < end) {
      at += cost(P, n, L, u++);
      x.tiles = 2;
    }
    // a key is seen by query i of the chunk from i = key - (L - n) on
    x.t0 = fdiv(P.tpt_div, max(x.key0 - (L - n), 0));
    x.t1 = fdiv(P.tpt_div, n + P.tpt - 1);
    return true;
  }
};

// 2^x for two values on the FMA pipe: x = n + f with n = round(x) (taken from the low mantissa bits of x + 1.5 * 2^23), 2^f on
// [-0.5, 0.5] by the polynomial of degree 5 of least relative error (Remez' exchange; 2.1e-7 as evaluated, what ex2.approx
// leaves too), times 2^n.  Below -126 about 2^-126 instead of 0, above 127.49 2^127.49 instead of infinity; a NaN stays one (which it
// would not with n added to the exponent field of a NaN).
__device__ __forceinline__ float clamp_nan(float x, float lo, float hi) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(x), "f"(lo));
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(d), "f"(hi));
  return d;
}
__device__ __forceinline__ void ex2_fma2_deg5(float& x0, float& x1) {
  const uint64_t magic = f32x2(12582912.f, 12582912.f);
  const uint64_t x = f32x2(clamp_nan(x0, -126.f, 127.49f), clamp_nan(x1, -126.f, 127.49f));
  const uint64_t t = add2(x, magic);
  const uint64_t f = sub2(x, sub2(t, magic));
  uint64_t p = fma2(f, f32x2(0.00132764725f, 0.00132764725f), f32x2(0.00967554096f, 0.00967554096f));
  p = fma2(p, f, f32x2(0.0555071309f, 0.0555071309f));
  p = fma2(p, f, f32x2(0.240221202f, 0.240221202f));
  p = fma2(p, f, f32x2(0.693146944f, 0.693146944f));
  p = fma2(p, f, f32x2(1.00000012f, 1.00000012f));
  float t0, t1;
  f32x2_split(t, t0, t1);
  auto pow2 = [](float t) { return __uint_as_float((__float_as_uint(t) << 23) + 0x3f800000u); };
  f32x2_split(mul2(p, f32x2(pow2(t0), pow2(t1))), x0, x1);
}

// The special-function unit (16 exponentials a clock and SM) bounds a chunk's sums, so kEmuNum of every 8 column pairs that
// everyone sees go to the FMA pipe.
constexpr int kEmuNum = 2;

// Adds 2^(s * scale) of 32 columns of a key's row to acc; hidden columns (bit clear) add nothing.
template <bool kMasked>
__device__ __forceinline__ void sum_columns(const uint32_t* s, float scale_log2, uint32_t bits, uint64_t (&acc)[2]) {
  const uint64_t scale2 = f32x2(scale_log2, scale_log2);
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    float x[4];
    f32x2_split(mul2(f32x2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale2), x[0], x[1]);
    f32x2_split(mul2(f32x2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), scale2), x[2], x[3]);
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      const int pair = (e + q) / 2;
      if (!kMasked && (pair * kEmuNum) % 8 < kEmuNum) {
        ex2_fma2_deg5(x[q], x[q + 1]);
      } else {
        x[q] = ex2(!kMasked || (bits >> (e + q)) & 1u ? x[q] : -INFINITY);
        x[q + 1] = ex2(!kMasked || (bits >> (e + q + 1)) & 1u ? x[q + 1] : -INFINITY);
      }
    }
    acc[0] = add2(acc[0], f32x2(x[0], x[1]));
    acc[1] = add2(acc[1], f32x2(x[2], x[3]));
  }
}


template <int D, int BQ>
__global__ void __launch_bounds__(Weigh<D, BQ>::kThreads, 1)
cache_weigh_sm100_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                         const __grid_constant__ WeighParams P) {
  using W = Weigh<D, BQ>;
  constexpr int kThreads = W::kThreads, kKSlots = W::kKSlots, kQSlots = W::kQSlots, kCols = W::kCols;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* gen = smem_dyn + (base - smem_u32(smem_dyn));
  long long* first = reinterpret_cast<long long*>(gen + W::kOffFirst);
  const uint32_t bars = base + W::kOffBars;
  const uint32_t k_full = bars, k_empty = k_full + 8 * kKSlots, q_full = k_empty + 8 * kKSlots, q_empty = q_full + 8 * kQSlots,
                 s_full = q_empty + 8 * kQSlots /* [tile][buffer] */, s_empty = s_full + 16 * kSBufs,
                 tmem_slot = s_empty + 16 * kSBufs;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kKSlots; ++i) {
      mbar_init(k_full + 8 * i, 1);
      mbar_init(k_empty + 8 * i, 1);
    }
    for (int i = 0; i < kQSlots; ++i) {
      mbar_init(q_full + 8 * i, 2);  // the tile, and its log-sum-exps
      mbar_init(q_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2 * kSBufs; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(s_empty + 8 * i, W::kSumWarps / 2);
    }
    mbar_fence_init();
  }
  if (warp == W::kMmaWarp) tmem_alloc(tmem_slot, W::kTmemCols);
  // Rows of a Q tile that no token fills (G does not divide BQ) are zeros: with a log-sum-exp without end they add nothing.
  for (int i = P.tpt * P.G * 8 + threadIdx.x; i < BQ * 8; i += kThreads)
    for (int sl = 0; sl < kQSlots * (D / 64); ++sl) st_shared_v4(base + W::kOffQ + sl * W::kQSlab + i * 16, make_uint4(0u, 0u, 0u, 0u));
  for (int i = threadIdx.x; i < W::kThinK / 16; i += kThreads)  // 1 1 1 0 ...: 16 bytes of the left and of the right matrix in turn
    st_shared_v4(base + W::kOffOnes + i * 16, (i & 8) == 0 ? make_uint4(0x3f803f80u, 0x00003f80u, 0u, 0u) : make_uint4(0u, 0u, 0u, 0u));
  for (int i = threadIdx.x; i < kQSlots * W::kThinQ / 16; i += kThreads)  // (three columns are written later, the others stay)
    st_shared_v4(base + W::kOffLse + i * 16, make_uint4(0u, 0u, 0u, 0u));
  fence_proxy_async_smem();
  pdl_wait();  // nothing above touches global memory
  const int per = (P.seqs.S + kThreads - 1) / kThreads;
  cost_prefix<kThreads>(P.seqs.S, per, first, first + kThreads + 1, [&](int b) {
    int row0;
    const int n = P.seqs.rows(b, row0), L = P.seqs.len(b);
    return Share::cost_before(P, n, L, Share::units_of(L)) * P.Hkv;
  });
  Share share;
  share.end = share_begin(first[kThreads], gridDim.x, blockIdx.x + 1);
  share.start(P, first, per, share_begin(first[kThreads], gridDim.x, blockIdx.x));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(gen + W::kOffBars + (tmem_slot - bars));
  Item x;
  bool ok = true;
  auto step_rows = [&](const Item& it, int t) { return min(P.tpt, it.n - t * P.tpt) * P.G; };

  if (warp == W::kTmaWarp) {
    // ------------------------------------------------------------ producer: K tiles of the item, then its Q tiles
    int nk = 0, nq = 0;
    while (ok && share.next(P, x)) {
      if (x.t0 >= x.t1) continue;  // nobody looks at these keys
      const int pages = (x.L + PG - 1) / PG, p0 = x.key0 / PG;
      // the item's four pages, a lane each; one past the end reads as zero
      const int row_mine = lane < 4 && p0 + lane < pages ? (P.seqs.page(x.seq, p0 + lane) * P.Hkv + x.hk) * PG : P.seqs.num_blocks * P.Hkv * PG;
      for (int h = 0; h < x.tiles && ok; ++h, ++nk) {
        const int slot = nk % kKSlots, use = nk / kKSlots;
        if (use > 0) ok = mbar_wait_warp(k_empty + 8 * slot, (use - 1) & 1);
        if (!ok) break;
        const int r0 = __shfl_sync(0xffffffffu, row_mine, 2 * h), r1 = __shfl_sync(0xffffffffu, row_mine, 2 * h + 1);
        if (lane == 0) {
          const uint32_t full = k_full + 8 * slot, dst = base + slot * W::kKTile;
          mbar_arrive_expect_tx(full, W::kKTile);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl) {
            tma_load_2d(dst + sl * W::kKSlab, &tm_k, full, sl * 64, r0);
            tma_load_2d(dst + sl * W::kKSlab + PG * 128, &tm_k, full, sl * 64, r1);
          }
        }
        __syncwarp();
      }
      for (int t = x.t0; t < x.t1 && ok; ++t, ++nq) {
        const int slot = nq % kQSlots, use = nq / kQSlots;
        if (use > 0) ok = mbar_wait_warp(q_empty + 8 * slot, (use - 1) & 1);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t full = q_full + 8 * slot, dst = base + W::kOffQ + slot * W::kQTile;
          mbar_arrive_expect_tx(full, P.tpt * P.G * D * 2);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl)
            tma_load_3d(dst + sl * W::kQSlab, &tm_q, full, sl * 64, x.hk * P.G, x.row0 + t * P.tpt);
        }
        __syncwarp();
      }
    }
  } else if (warp == W::kLseWarp) {
    // ------------------------------------------------------------ log-sum-exps of each Q tile's rows, negated, in units of the scores
    int nq = 0;
    while (ok && share.next(P, x)) {
      for (int t = x.t0; t < x.t1 && ok; ++t, ++nq) {
        const int slot = nq % kQSlots, use = nq / kQSlots, rows = step_rows(x, t);
        float l[BQ / 32];
#pragma unroll
        for (int u = 0; u < BQ / 32; ++u) {
          const int c = u * 32 + lane, tok = fdiv(P.g_div, c);
          l[u] = c < rows ? P.lse[(long long)(x.row0 + t * P.tpt + tok) * P.Hq + x.hk * P.G + (c - tok * P.G)] : INFINITY;
        }
        if (use > 0) ok = mbar_wait_warp(q_empty + 8 * slot, (use - 1) & 1);
        if (!ok) break;
#pragma unroll
        for (int u = 0; u < BQ / 32; ++u) {
          const int c = u * 32 + lane;
          // three parts of 8 bits each; a row of no token, or with nothing to see, as if its weights were e^-256
          const float y = -(fabsf(l[u]) == INFINITY ? 256.f : l[u]) * P.inv_scale;
          const float hi = __bfloat162float(__float2bfloat16_rn(y)), mid = __bfloat162float(__float2bfloat16_rn(y - hi)), lo = y - hi - mid;
          st_shared_v4(base + W::kOffLse + slot * W::kThinQ + (c >> 3) * 256 + (c & 7) * 16, make_uint4(pack_bf16(hi, mid), pack_bf16(lo, 0.f), 0u, 0u));
        }
        fence_proxy_async_smem();
        mbar_arrive_warp(q_full + 8 * slot);
      }
    }
  } else if (warp == W::kMmaWarp) {
    // ------------------------------------------------------------ MMA issuer: the whole warp runs the loop, one lane issues
    const uint32_t leader = elect_one();
    constexpr uint32_t kHi = smem_desc_hi(1024);
    constexpr uint32_t kThinHi = (256 >> 4) | (1u << 14);  // no swizzle: groups of eight rows 256 bytes apart, the two matrices 128
    int nk = 0, nq = 0, ns[2] = {0, 0};  // K tiles, Q tiles, products of either key tile so far
    while (ok && share.next(P, x)) {
      if (x.t0 >= x.t1) continue;
      for (int t = x.t0; t < x.t1 && ok; ++t, ++nq) {
        const int slot = nq % kQSlots;
        ok = mbar_wait_warp(q_full + 8 * slot, (nq / kQSlots) & 1);
        if (!ok) break;
        const int cols = (step_rows(x, t) + 31) & ~31;  // as the sums take them
        const uint32_t idesc = make_idesc_bf16(BK, cols, false, false);
        const uint32_t q_lo = smem_desc_lo(base + W::kOffQ + slot * W::kQTile, 16);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (h >= x.tiles) break;
          const int kslot = (nk + h) % kKSlots, buf = h * kSBufs + ns[h] % kSBufs, use = ns[h] / kSBufs;
          if (t == x.t0) ok = mbar_wait_warp(k_full + 8 * kslot, ((nk + h) / kKSlots) & 1);
          if (ok && use > 0) ok = mbar_wait_warp(s_empty + 8 * buf, (use - 1) & 1);
          if (!ok) break;
          ++ns[h];
          tc_fence_after();
          const uint32_t k_lo = smem_desc_lo(base + kslot * W::kKTile, 16);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            umma_ss(leader, tmem + buf * BQ, smem_desc_join(k_lo + (((kk / 4) * W::kKSlab + (kk % 4) * 32) >> 4), kHi),
                    smem_desc_join(q_lo + (((kk / 4) * W::kQSlab + (kk % 4) * 32) >> 4), kHi), idesc, kk > 0);
          umma_ss(leader, tmem + buf * BQ, smem_desc_join(smem_desc_lo(base + W::kOffOnes, 128), kThinHi),
                  smem_desc_join(smem_desc_lo(base + W::kOffLse + slot * W::kThinQ, 128), kThinHi), idesc, 1);
          umma_commit(leader, s_full + 8 * buf);
          if (t == x.t1 - 1) umma_commit(leader, k_empty + 8 * kslot);
        }
        if (ok) umma_commit(leader, q_empty + 8 * slot);
      }
      nk += x.tiles;
    }
  } else if (warp < W::kSumWarps) {
    // ------------------------------------------------------------ sums: a key and kCols columns per thread
    const int h = warp / (4 * W::kParts), part = warp / 4 % W::kParts, key_of_item = h * BK + (warp & 3) * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    float* meet = reinterpret_cast<float*>(gen + W::kOffMeet);
    int ns = 0, n_items = 0;
    while (share.next(P, x)) {  // to the end even when a wait gave up: the warpgroups meet at barriers
      if (h >= x.tiles) continue;
      const int key = x.key0 + key_of_item;
      // where the sum goes; what was there comes under the walk
      long long at = -1;
      if (key < x.L && part == 0) {
        const int page = P.seqs.table[(long long)x.seq * P.seqs.max_blocks + key / PG];
        if (page >= 0 && page < P.seqs.num_blocks) at = ((long long)page * P.Hkv + x.hk) * PG + key % PG;  // never outside the cache
      }
      const float before = at >= 0 && P.decay != 0.f ? P.w_in[at] : 0.f;
      uint64_t acc[2] = {0, 0};  // four partial sums
      for (int t = x.t0; t < x.t1 && ok; ++t, ++ns) {
        const int buf = h * kSBufs + ns % kSBufs, rows = step_rows(x, t) - part * kCols;  // from this part on
        ok = mbar_wait_warp(s_full + 8 * buf, (ns / kSBufs) & 1);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tS = tmem + buf * BQ + part * kCols + lane_base, empty = s_empty + 8 * buf;
        // every key of the tile sees every row
        const bool full = rows >= min(P.tpt * P.G - part * kCols, kCols) && x.key0 + h * BK + BK - 1 - (x.L - x.n) - t * P.tpt <= 0;
        uint32_t s[kCols];
        if (full && rows > kCols - 32) {
#pragma unroll
          for (int c = 0; c < kCols / 32; ++c) tmem_ld32(tS + c * 32, s + c * 32);
          tmem_wait_ld();
          tc_fence_before();
          mbar_arrive_warp(empty);  // the buffer is free while its scores are worked on
#pragma unroll
          for (int c = 0; c < kCols / 32; ++c) sum_columns<false>(s + c * 32, P.scale_log2, 0u, acc);
        } else {
          // visible columns of this key: the rows of tokens from key - (L - n) on
          const int c_lo = min(max(key - (x.L - x.n) - t * P.tpt, 0), BQ) * P.G - part * kCols;
#pragma unroll
          for (int c = 0; c < kCols / 32; ++c) {
            if (c * 32 >= rows) break;
            tmem_ld32(tS + c * 32, s + c * 32);
            tmem_wait_ld();
            const int a = max(c_lo - c * 32, 0), b = min(rows - 1 - c * 32, 31);
            sum_columns<true>(s + c * 32, P.scale_log2, a > b ? 0u : (0xffffffffu >> (31 - b)) & (0xffffffffu << a), acc);
          }
          tc_fence_before();
          mbar_arrive_warp(empty);
        }
      }
      float sum[4];
      f32x2_split(acc[0], sum[0], sum[1]);
      f32x2_split(acc[1], sum[2], sum[3]);
      float mine = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if (W::kParts == 2) {
        // the two parts of a key meet (two buffers: the next item's sums may come while these are read)
        float* other = meet + (n_items++ & 1) * 2 * BK + key_of_item;
        if (part == 1) *other = mine;
        named_barrier_sync(1 + h, 256);
        mine += *other;
      }
      if (ok && at >= 0) P.w_out[at] = fmaf(P.decay, before, mine);
    }
  }
  if (!ok) atomicExch(&g_weigh_timeout, 1u);
  tc_fence_before();
  __syncthreads();
  if (warp == W::kMmaWarp) {
    __syncwarp();
    tmem_dealloc(tmem, W::kTmemCols);
  }
}

template <int D, int BQ>
int32_t go(const CUtensorMap& mq, const CUtensorMap& mk, const WeighParams& P, int grid, cudaStream_t st) {
  const auto kern = cache_weigh_sm100_kernel<D, BQ>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Weigh<D, BQ>::kBytes);
  if (e != cudaSuccess) return fail(UNIGIST_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  {
    KernelScope ks("cache_weigh_sm100_kernel", st);
    launch_chained(kern, dim3(grid), Weigh<D, BQ>::kThreads, Weigh<D, BQ>::kBytes, st, 1, mq, mk, P);
  }
  return check_launch("cache weights kernel");
}

}  // namespace

int32_t launch_cache_weigh(const ChunkBatch& b, int Hq, int Hkv, int D, float scale, const void* q, int64_t q_stride,
                           const float* lse, const void* kc, const float* weights_in, float decay, float* weights_out,
                           cudaStream_t st) {
  WeighParams P;
  P.seqs = b;
  P.lse = lse, P.w_in = weights_in, P.w_out = weights_out;
  P.Hq = Hq, P.Hkv = Hkv, P.G = Hq / Hkv;
  // Tiles of 32 rows where the sequences bring no more than that on average.
  const bool few = P.G <= 32 && (long long)b.num_rows * P.G <= 32ll * b.S;
  P.tpt = (few ? 32 : 128) / P.G;
  P.tile_cost = (few ? 4 : 1) * P.tpt;  // (reading 32 KB takes as long as the products with 128 rows, four with 32)
  P.g_div = make_fastdiv(P.G), P.tpt_div = make_fastdiv(P.tpt);
  P.scale_log2 = scale * LOG2E, P.inv_scale = 1.0f / scale, P.decay = decay;
  CUtensorMap mq, mk;
  // (a map cannot be empty; without rows it is never used)
  if (int32_t rc = b.num_rows > 0 ? encode_row_map(&mq, q, D, Hq, b.num_rows, q_stride, P.G, P.tpt)
                                  : encode_row_map(&mq, kc, D, Hkv, 1, (int64_t)Hkv * D, 1, 1))
    return rc;
  if (int32_t rc = encode_map_2d_bf16(&mk, kc, (long long)b.num_blocks * Hkv * PG, D, PG, 64)) return rc;
  const long long most = (long long)b.S * Hkv * ((b.max_blocks + 1) / 2);
  const int grid = (int)(most < sm_count() ? most : sm_count());
  if (few) return D == 128 ? go<128, 32>(mq, mk, P, grid, st) : go<64, 32>(mq, mk, P, grid, st);
  return D == 128 ? go<128, 128>(mq, mk, P, grid, st) : go<64, 128>(mq, mk, P, grid, st);
}

int32_t cache_weigh_timeout_flag(unsigned int** at) { return flag_address(at, g_weigh_timeout); }

}  // namespace ug
