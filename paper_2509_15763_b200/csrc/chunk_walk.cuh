// What the kernels of the attention of ragged chunks share: units of work, the shares into which all of it is dealt out, and the
// partial results of units that a share boundary cuts.
#pragma once
#include "chunk_tma.cuh"

namespace ug {

// A cut unit's part: where it lies in the unit's walk, and whose rows it holds.
struct alignas(16) Part {
  int row0, ntok, hk, nt, j0, j1, valid, pad;
};

struct ChunkParams {
  ChunkBatch seqs;
  const __nv_bfloat16* q;
  int64_t q_stride;
  __nv_bfloat16* o;
  float* lse;
  Part* parts;      // [grid][2]: the share's part of a unit begun earlier; its part of a unit that ends later
  float* part_o;    // [grid][2][D / 4][slot_rows] float4
  float2* part_ml;  // [grid][2][slot_rows] (maximum in log2 units, sum)
  // tpt: tokens of a query tile; a unit of work has unit_tokens, a share of all work is worth at least min_share keys
  int Hq, Hkv, G, tpt, slot_rows, unit_tokens, unit_cost, single_cost, min_share;
  FastDiv g_div, unit_div;
  float scale_log2;
};

// Steps [j0, j1) of the walk of one unit over its keys, kStep a step from the diagonal down: step j takes tile nt - 1 - j.
struct Unit {
  int hk, row0, ntok;  // first row of the row tensors, tokens
  int base;            // token i of the unit sees slots 0 .. base + i
  int L, seq, nt, j0, j1;
};

// The units of a share, in order.  All positions are in keys: a unit costs the slots that its last token sees and P.unit_cost more
// (its loads, first scores and epilogue), which has a closed form over the units of a sequence.  The last unit of a sequence may
// be a single query tile, whose steps cost P.single_cost sixteenths of others'.
// kWaves: with whole units dealt out in turn before the shares (deal_waves).
template <int kStep, bool kWaves = false>
struct Share {
  int seq, hk, u;
  int n, row0, L, units;
  long long at, begin, end;      // position of the next unit; the share
  int waves = 0, wave_unit = 0;  // whole units to come before it, of the whole grid's order, and the next of them

  static __device__ __forceinline__ long long cost_before(const ChunkParams& P, int n, int L, int u) {  // of a sequence's first u units, u < units
    const long long per = P.unit_tokens;
    return u * (long long)(max(L - n, 0) + P.unit_cost) + per * u * (u + 1) / 2;
  }
  static __device__ __forceinline__ long long unit_cost(const ChunkParams& P, int n, int L, int u) {
    const long long keys = max(L - n, 0) + min((long long)n, (long long)(u + 1) * P.unit_tokens);
    return (n - u * (long long)P.unit_tokens <= P.tpt ? keys * P.single_cost >> 4 : keys) + P.unit_cost;
  }
  static __device__ __forceinline__ int units_of(const ChunkParams& P, int n) { return fdiv(P.unit_div, n + P.unit_tokens - 1); }
  static __device__ __forceinline__ long long head_cost(const ChunkParams& P, int n, int L) {
    const int units = units_of(P, n);
    return units > 0 ? cost_before(P, n, L, units - 1) + unit_cost(P, n, L, units - 1) : 0;
  }
  // A boundary inside a unit is one of its steps, the same for the shares on either side of it (no contraction, no approximation).
  static __device__ __forceinline__ int step_of(long long offset, int nt, long long cost) {
    return min((int)__fmul_rn((float)offset, __fdiv_rn((float)nt, (float)cost)), nt);
  }
  __device__ __forceinline__ void load(const ChunkParams& P) {
    n = P.seqs.rows(seq, row0);
    L = P.seqs.len(seq);
    units = units_of(P, n);
  }
  // The share [begin, end) of all the work; `first` and `per` from cost_prefix.
  __device__ __forceinline__ void start(const ChunkParams& P, const long long* first, int per) {
    at = begin;
    if (begin >= end) return;
    const int group = cost_group(first, (P.seqs.S - 1) / per, begin);
    long long left = begin - first[group], one;
    for (seq = group * per;; ++seq) {
      load(P);
      one = head_cost(P, n, L);
      if (left < one * P.Hkv) break;
      left -= one * P.Hkv;
    }
    hk = min((int)__fdividef((float)left, (float)one), P.Hkv - 1);  // (a 64-bit division takes longer than the two corrections)
    left -= hk * one;
    while (left < 0) --hk, left += one;
    while (left >= one) ++hk, left -= one;
    seek(P, left);
  }
  // The unit of the current sequence and head in which position `left` of the head lies; `at` is that position's.
  __device__ __forceinline__ void seek(const ChunkParams& P, long long left) {
    int lo = 0, hi = units - 1;  // the last unit that begins at or before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (cost_before(P, n, L, mid) <= left) lo = mid; else hi = mid - 1;
    }
    u = lo;
    at -= left - cost_before(P, n, L, u);
  }
  // Unit u of the current sequence and head, with its whole walk; returns its cost.
  __device__ __forceinline__ long long unit(const ChunkParams& P, Unit& x) const {
    const int tok0 = u * P.unit_tokens;
    x.seq = seq, x.hk = hk, x.L = L;
    x.row0 = row0 + tok0;
    x.ntok = min(P.unit_tokens, n - tok0);
    x.base = L - n + tok0;
    x.nt = max(x.base + x.ntok - 1, 0) / kStep + 1;
    x.j0 = 0, x.j1 = x.nt;
    return unit_cost(P, n, L, u);
  }
  __device__ __forceinline__ bool next(const ChunkParams& P, Unit& x) {
    if (kWaves && waves > 0) {  // (one sequence)
      const int part_hk = hk, part_u = u;
      hk = wave_unit / units, u = wave_unit - hk * units;
      unit(P, x);
      hk = part_hk, u = part_u;
      wave_unit += gridDim.x;
      --waves;
      return true;
    }
    while (at < end) {
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
      const long long cost = unit(P, x);
      if (begin > at) x.j0 = step_of(begin - at, x.nt, cost);
      if (at + cost > end) x.j1 = step_of(end - at, x.nt, cost);
      at += cost;
      ++u;
      if (x.j1 > x.j0) return true;
    }
    return false;
  }
  // The share of this block of a one-dimensional grid: `first`, `per` as cost_prefix leaves them.
  __device__ __forceinline__ void deal(const ChunkParams& P, const long long* first, int per, long long total) {
    const int shares = (int)max(1ll, min((long long)gridDim.x, total / P.min_share)), c = blockIdx.x;
    begin = c < shares ? share_begin(total, shares, c) : 0;
    end = c < shares ? share_begin(total, shares, c + 1) : 0;
    start(P, first, per);
  }
  // The same for one sequence of at least as many units as there are blocks, by all threads of the block.  Equal shares of the
  // walks laid end to end start all over the keys, and with a long cache the blocks at work read more K and V than the L2 holds
  // (4096 tokens over 65536 slots, 8 KV heads: 11.3 GB for 0.3, and 4.4 ms where 3.7 do).  So the blocks take whole units first, neighbouring ones side by
  // side, which walk the same keys in step; what is left is cut, and a block gets of it what its whole units leave it short of
  // an equal share of everything.  `first`: room for kThreads + 1 numbers.
  template <int kThreads>
  __device__ __forceinline__ bool deal_waves(const ChunkParams& P, long long* first) {
    seq = 0;
    load(P);
    const int grid = gridDim.x;
    const long long all = (long long)units * P.Hkv, one = head_cost(P, n, L), total = one * P.Hkv;
    int w = (int)min(all / grid, 1ll << 20);
    if (w == 0 || all > 0x7fffffff) return false;
    auto before = [&](long long unit) {  // cost of the units before it
      const int h = (int)(unit / units), k = (int)(unit - (long long)h * units);
      return h * one + cost_before(P, n, L, k);
    };
    if (total - before((long long)w * grid) < (long long)grid * P.min_share) --w;  // too little left to be cut
    const long long rest_at = before((long long)w * grid), rest = total - rest_at;
    auto short_of = [&](int c) {  // cost that block c's whole units leave it short of an equal share
      long long mine = 0;
      for (int i = 0; i < w; ++i) mine += unit_cost(P, n, L, (int)((c + (long long)i * grid) % units));
      return max(total / grid - mine, 0ll);
    };
    __syncthreads();  // `first` may be in use
    cost_prefix<kThreads>(grid, (grid + kThreads - 1) / kThreads, first, first + kThreads + 1, short_of);
    // (at most one block a thread: the grid is no larger than the block)
    const int c = blockIdx.x;
    const float scale = __fdiv_rn((float)rest, (float)max(first[grid], 1ll));
    auto edge = [&](int k) { return rest_at + (k >= grid ? rest : min((long long)__fmul_rn((float)first[k], scale), rest)); };
    begin = edge(c), end = edge(c + 1);
    waves = w, wave_unit = c;
    at = begin;
    if (begin < end) {
      long long left = begin;
      hk = min((int)(left / one), P.Hkv - 1);
      left -= hk * one;
      seek(P, left);
    }
    return true;
  }
};

// Adds up the parts of the units that the shares of a grid cut (their order is that of the shares: the same bits every run).
int32_t launch_chunk_combine(const ChunkParams& P, int D, int grid, cudaStream_t st);
// Which kernel takes a call of these sizes: the one for many rows (chunk_attn.cu), or for chunks of few the warp-level one
// (chunk_attn_few.cu: short walks, and heads of 64) or the one with the operands turned round (chunk_attn_thin.cu: long walks).
enum { kChunkRows, kChunkFew, kChunkThin };
int chunk_route(int S, int num_rows, int G, int Hkv, int D, int max_blocks);
size_t chunk_few_scratch_bytes(int S, int num_rows, int Hq, int Hkv, int D, int max_blocks);
int32_t launch_chunk_few(ChunkParams P, int D, const CUtensorMap& mk, const CUtensorMap& mv, void* ws, cudaStream_t st);
inline int chunk_thin_grid() { return sm_count() < 256 ? sm_count() : 256; }
size_t chunk_thin_scratch_bytes();
int32_t launch_chunk_thin(ChunkParams P, const void* q, int64_t q_stride, const CUtensorMap& mk, const CUtensorMap& mv, void* ws, cudaStream_t st);

// Bytes of `grid` shares' parts, and the pointers to them.
inline size_t chunk_parts_bytes(int grid, int rows, int D) {
  return ((size_t)2 * grid * (sizeof(Part) + rows * (sizeof(float2) + (size_t)D * 4)) + 255) / 256 * 256;
}
inline void set_chunk_parts(ChunkParams* P, void* ws, int grid, int rows, int D) {
  P->slot_rows = rows;
  P->parts = (Part*)ws;
  P->part_o = reinterpret_cast<float*>(P->parts + 2 * grid);
  P->part_ml = reinterpret_cast<float2*>(P->part_o + (size_t)2 * grid * rows * D);
}

}  // namespace ug
