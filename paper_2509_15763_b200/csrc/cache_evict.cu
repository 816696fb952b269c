// Eviction from a paged cache by accumulated attention weight.  Per sequence of length L and KV head, of L > keep slots the
// first `keep_first`, the last `keep_last` and, of those between, the keep - keep_first - keep_last of largest weight stay (of
// equal weights the lowest slots); they move together into slots 0 .. keep - 1 in their order.  Every KV head keeps
// slots of its own: attention does not care about the order of a head's slots, and keys carry their position in them.
//
// The threshold weight is found by radix (the weights are not negative, so their bits order them: 11, 11 and 10 bits a pass),
// then the kept slots are listed in order and their rows moved.  Up to 16K slots or so one kernel does both, several blocks a
// (sequence, KV head), each of which finds the slots for itself and moves its share of the rows.  Longer caches: the blocks of a
// cluster share the search, adding up their counts through distributed shared memory, and a second kernel moves the rows.
// Bound: the weights once, the kept rows read and written once (32 sequences of 5000 - 9216 slots cut to 4096: 193 us into other
// pages, 209 in place, at the memory's rate 166; one of 65000 cut to 8192 38 and 71 us for 11: a search in a cluster, and in place
// rounds of one cluster's blocks).
#include "chunk.cuh"
#include "sm100_ptx.cuh"

namespace ug {
namespace {

constexpr int PG = UNIGIST_PAGE_TOKENS;
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMany = 4;  // rows in flight per thread, 16 bytes of K and of V each

struct Evict {
  int Hkv, keep, first, last;
};

// The weight's bits as a number that orders weights; what is no weight (below zero, NaN) counts as zero.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

constexpr int kBins = 2048;  // of a pass; the last has half as many
struct Select {              // shared memory of a search
  uint32_t hist[3][kBins];   // all zero at the start
  uint32_t warp_sum[kWarps], warp_ties[kWarps], bin, left, held, ties;
};

// Sum over the lanes up to this one.
__device__ __forceinline__ uint32_t warp_prefix(uint32_t x, int lane) {
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, off);
    if (lane >= off) x += y;
  }
  return x;
}
// Sum of the warps' numbers before this warp's.
__device__ __forceinline__ uint32_t before_warp(const uint32_t* of_warp, int warp, int lane) {
  return __reduce_add_sync(0xffffffffu, lane < warp ? of_warp[lane] : 0u);
}

// Lists the slots of [s_begin, s_end) (s_begin a multiple of 128) that stay: emit(number among all kept slots, slot).  Whole
// blocks; L > E.keep.  page_of(i): page of the cache that holds the sequence's i-th 64 slots.  keys: room for the slots' keys, or
// null where they do not fit (they are then read again each time).  kSplit: the slots are the block's share, the rest is with
// the other blocks of the cluster, whose shared memory must not go away before they have all returned from here.
//
// The first and last slots, which stay in any case, take part as keys above any weight's; what a load of four slots reads behind
// the last one as zeros, which come after every slot of weight zero.
template <bool kSplit, typename PageOf, typename Emit>
__device__ __forceinline__ void select_kept(const Evict& E, int hk, int L, int s_begin, int s_end, const float* __restrict__ weights,
                                            uint32_t* keys, Select& sh, PageOf page_of, Emit emit) {
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int ranks = kSplit ? gridDim.x : 1;
  const int lo = E.first, hi = L - E.last;
  auto weights_of = [&](int i) {  // (i a multiple of four: the four lie in one page)
    return *reinterpret_cast<const float4*>(weights + ((long long)page_of(i / PG) * E.Hkv + hk) * PG + i % PG);
  };
  auto keys_of = [&](float4 w, int i) {
    auto one = [&](float x, int slot) { return slot >= L ? 0u : slot < lo || slot >= hi ? 0xffffffffu : weight_key(x); };
    return make_uint4(one(w.x, i), one(w.y, i + 1), one(w.z, i + 2), one(w.w, i + 3));
  };
  auto key4 = [&](int i) { return keys ? *reinterpret_cast<const uint4*>(keys + (i - s_begin)) : keys_of(weights_of(i), i); };
  uint32_t left = E.keep, prefix = 0;  // the left-th largest key of those that begin with `prefix` is the threshold
  // digit of a pass: 11, 11, 10 bits
  auto count4 = [&](uint4 k, int pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
    const uint32_t mask = pass < 2 ? kBins - 1 : kBins / 2 - 1;
    const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (pass == 0 || key[e] >> (pass == 1 ? 21 : 10) == prefix) atomicAdd(&sh.hist[pass][(key[e] >> shift) & mask], 1u);
  };
  constexpr int kLoads = 4;  // in flight
  for (int i0 = s_begin + 4 * t; i0 < s_end; i0 += kLoads * 4 * kThreads) {
    float4 w[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      if (i0 + u * 4 * kThreads < s_end) w[u] = weights_of(i0 + u * 4 * kThreads);
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = i0 + u * 4 * kThreads;
      if (i >= s_end) continue;
      const uint4 k = keys_of(w[u], i);
      if (keys) *reinterpret_cast<uint4*>(keys + (i - s_begin)) = k;
      count4(k, 0);
    }
  }
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    if (pass > 0)
      for (int i = s_begin + 4 * t; i < s_end; i += 4 * kThreads) count4(key4(i), pass);
    if (kSplit) sm100::cluster_sync(); else __syncthreads();
    // from the largest digit down, a thread takes four neighbouring bins: n.w is the largest
    const int bins = pass < 2 ? kBins : kBins / 2, at = bins - 4 - 4 * t;
    uint4 n = make_uint4(0u, 0u, 0u, 0u);
    if (at >= 0) {
      if (kSplit) {
        const uint32_t addr = sm100::smem_u32(&sh.hist[pass][at]);
#pragma unroll 8
        for (int r = 0; r < ranks; ++r) {
          const float4 f = sm100::ld_cluster_v4(addr, r);
          n.x += __float_as_uint(f.x), n.y += __float_as_uint(f.y), n.z += __float_as_uint(f.z), n.w += __float_as_uint(f.w);
        }
      } else {
        n = *reinterpret_cast<const uint4*>(&sh.hist[pass][at]);
      }
    }
    const uint32_t mine = n.x + n.y + n.z + n.w, incl = warp_prefix(mine, lane);
    if (lane == 31) sh.warp_sum[warp] = incl;
    __syncthreads();
    uint32_t above = incl - mine + before_warp(sh.warp_sum, warp, lane);
    if (above < left && above + mine >= left) {  // the threshold lies in one of these bins
      int e = 3;
      if (above + n.w < left) above += n.w, e = 2;
      if (e == 2 && above + n.z < left) above += n.z, e = 1;
      if (e == 1 && above + n.y < left) above += n.y, e = 0;
      sh.bin = at + e;
      sh.left = left - above;
    }
    __syncthreads();
    prefix = (prefix << (pass < 2 ? 11 : 10)) | sh.bin;
    left = sh.left;
  }
  // All slots above the threshold stay, and of those that are equal to it the lowest `left`.  A warp lists a run of neighbouring
  // slots, of which it has counted both kinds.
  const int run = ((s_end - s_begin + kWarps - 1) / kWarps + 127) / 128 * 128, r0 = min(s_begin + warp * run, s_end), r1 = min(r0 + run, s_end);
  uint32_t helds = 0, ties = 0;
  for (int i = r0 + 4 * lane; i < r1; i += 128) {
    const uint4 k = key4(i);
    helds += (k.x > prefix) + (k.y > prefix) + (k.z > prefix) + (k.w > prefix);
    ties += (k.x == prefix) + (k.y == prefix) + (k.z == prefix) + (k.w == prefix);
  }
  helds = __reduce_add_sync(0xffffffffu, helds), ties = __reduce_add_sync(0xffffffffu, ties);
  if (lane == 0) sh.warp_sum[warp] = helds, sh.warp_ties[warp] = ties;
  __syncthreads();
  const uint32_t my_helds = helds, my_ties = ties;
  helds = before_warp(sh.warp_sum, warp, lane), ties = before_warp(sh.warp_ties, warp, lane);
  if (kSplit) {
    if (t == kThreads - 1) sh.held = helds + my_helds, sh.ties = ties + my_ties;  // of the last warp: with its own run, the block's
    sm100::cluster_sync();
    for (int r = 0; r < (int)blockIdx.x; ++r) {
      helds += __float_as_uint(sm100::ld_cluster_f32(sm100::smem_u32(&sh.held), r));
      ties += __float_as_uint(sm100::ld_cluster_f32(sm100::smem_u32(&sh.ties), r));
    }
  }
  for (int i = r0; i < r1; i += 128) {
    const int slot = i + 4 * lane;
    const uint4 k = slot < r1 ? key4(slot) : make_uint4(0u, 0u, 0u, 0u);
    const bool in = slot < r1;
    const uint32_t key[4] = {k.x, k.y, k.z, k.w};
    uint32_t both = 0;  // low half: above, high half: equal (at most 128 a step)
#pragma unroll
    for (int e = 0; e < 4; ++e) both += in ? (uint32_t)(key[e] > prefix) + ((uint32_t)(key[e] == prefix) << 16) : 0u;
    const uint32_t incl = warp_prefix(both, lane), all = __shfl_sync(0xffffffffu, incl, 31);
    uint32_t h = helds + ((incl - both) & 0xffffu), s = ties + ((incl - both) >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool held = in && key[e] > prefix, tie = in && key[e] == prefix;
      if (held || (tie && s < left)) emit(h + min(s, left), slot + e);
      h += held, s += tie;
    }
    helds += all & 0xffffu, ties += all >> 16;
  }
}

// Moves rows [0, n): row j from slot kept(j).  The blocks of a (sequence, KV head) take `step` rows of a round in turn.
// In place a row moves to its own slot or a lower one, where another row may still lie that is to move too: the blocks are a
// cluster, and once all rows of the rounds up to this one have been read, its slots can be written, since a row that is read
// later lies at or above its own number, and so above them.
template <int D, bool kInPlace, typename Kept, typename From, typename To>
__device__ __forceinline__ void move_rows(const ChunkBatch& B, int Hkv, int hk, int n, uint4* kc, uint4* vc, float* weights, Kept kept,
                                          From from_page, To to_page) {
  constexpr int kVecs = D / 8, kRows = kThreads / kVecs;
  const int vec = threadIdx.x % kVecs, sub = threadIdx.x / kVecs, c = gridDim.x;
  for (long long base = 0; base < n; base += (long long)c * kRows * kMany) {
    long long to[kMany];
    uint4 k[kMany], v[kMany];
    float w[kMany];
#pragma unroll
    for (int u = 0; u < kMany; ++u) {
      const long long j = base + (u * c + (int)blockIdx.x) * kRows + sub;
      to[u] = -1;
      if (j >= n) continue;
      const int src = kept((int)j);
      if (kInPlace && src == j) continue;  // stays where it is
      const int page = to_page((int)j / PG);
      if (page < 0 || page >= B.num_blocks) continue;  // never write outside the cache
      to[u] = ((long long)page * Hkv + hk) * PG + j % PG;
      const long long from = ((long long)from_page(src / PG) * Hkv + hk) * PG + src % PG;
      k[u] = kc[from * kVecs + vec];
      v[u] = vc[from * kVecs + vec];
      if (vec == 0) w[u] = weights[from];
    }
    if (kInPlace) sm100::cluster_sync();
#pragma unroll
    for (int u = 0; u < kMany; ++u) {
      if (to[u] < 0) continue;
      kc[to[u] * kVecs + vec] = k[u];
      vc[to[u] * kVecs + vec] = v[u];
      if (vec == 0) weights[to[u]] = w[u];
    }
  }
}

__device__ __forceinline__ void clear(Select& sh) {
  for (int i = threadIdx.x; i < 3 * kBins / 4; i += kThreads) reinterpret_cast<uint4*>(&sh.hist[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
}
__device__ __forceinline__ void set_new_len(const ChunkBatch& B, const Evict& E, int b, int32_t* new_lens) {
  new_lens[b] = B.lens[b] < 0 ? B.lens[b] : min(B.len(b), E.keep);
}

// ------------------------------------------------------------------------------------------------ one kernel
struct FusedSmem {  // dynamic: the keys, the two rows of pages, the kept slots (below 65536)
  size_t old_pages, new_pages, kept, bytes;
  __host__ __device__ FusedSmem(int max_blocks, int keep) {
    const size_t slots = (size_t)max_blocks * PG, most = (size_t)keep < slots ? keep : slots;
    old_pages = slots * 4;
    new_pages = old_pages + (size_t)max_blocks * 4;
    kept = new_pages + (most + PG - 1) / PG * 4;
    bytes = kept + (most * 2 + 15) / 16 * 16;
  }
};
constexpr size_t kFusedMost = 84 * 1024;  // two blocks an SM, with the histograms

// grid (c, Hkv, S), in place clusters of c
template <int D, bool kInPlace>
__global__ void __launch_bounds__(kThreads)
evict_fused_kernel(const __grid_constant__ ChunkBatch B, const __grid_constant__ Evict E, uint4* kc, uint4* vc, float* weights,
                   const int32_t* __restrict__ new_table, int new_max_blocks, int32_t* __restrict__ new_lens,
                   int32_t* __restrict__ kept_idx) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Select sh;
  const FusedSmem at(B.max_blocks, E.keep);
  uint32_t* keys = reinterpret_cast<uint32_t*>(smem);
  int32_t* old_pages = reinterpret_cast<int32_t*>(smem + at.old_pages);
  int32_t* new_pages = reinterpret_cast<int32_t*>(smem + at.new_pages);
  uint16_t* kept = reinterpret_cast<uint16_t*>(smem + at.kept);
  const int t = threadIdx.x;
  clear(sh);
  pdl_wait();
  const int b = blockIdx.z, hk = blockIdx.y, rank = blockIdx.x, c = gridDim.x;
  for (int i = t; i < B.max_blocks; i += kThreads) old_pages[i] = B.page(b, i);  // (beside the length: not all of them may be needed)
  const int L = B.len(b), n = min(L, E.keep);  // n rows stay
  if (rank == 0 && hk == 0 && t == 0) set_new_len(B, E, b, new_lens);
  int32_t* kept_out = kept_idx + ((long long)b * E.Hkv + hk) * E.keep;
  if (L <= E.keep) {
    for (int j = rank * kThreads + t; j < E.keep; j += c * kThreads) kept_out[j] = j < L ? j : -1;
    if (kInPlace) return;  // (the whole cluster)
  }
  if (!kInPlace)
    for (int i = t; i < (n + PG - 1) / PG; i += kThreads) new_pages[i] = new_table[(long long)b * new_max_blocks + i];
  __syncthreads();
  auto old_page = [&](int i) { return old_pages[i]; };
  if (L > E.keep) {
    select_kept<false>(E, hk, L, 0, L, weights, keys, sh, old_page, [&](uint32_t j, int slot) {
      kept[j] = (uint16_t)slot;
      if (rank == 0) kept_out[j] = slot;
    });
  } else {
    for (int j = t; j < n; j += kThreads) kept[j] = (uint16_t)j;
  }
  __syncthreads();
  const int32_t* row = B.table + (long long)b * B.max_blocks;
  move_rows<D, kInPlace>(B, E.Hkv, hk, n, kc, vc, weights, [&](int j) { return (int)kept[j]; }, old_page,
                         [&](int i) { return kInPlace ? row[i] : new_pages[i]; });
}

// ------------------------------------------------------------------------------------------------ two kernels
constexpr int kSplitKeys = 22 * 1024;      // keys a block holds (88 KB, two blocks an SM); a longer share is read again each time

// grid (c, Hkv, S), clusters of c that share a search
__global__ void __launch_bounds__(kThreads)
evict_select_kernel(const __grid_constant__ ChunkBatch B, const __grid_constant__ Evict E, const float* __restrict__ weights,
                    int32_t* __restrict__ new_lens, int32_t* __restrict__ kept_idx) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ Select sh;
  clear(sh);
  pdl_wait();
  const int b = blockIdx.z, hk = blockIdx.y, t = threadIdx.x;
  const int L = B.len(b);
  if (blockIdx.x == 0 && hk == 0 && t == 0) set_new_len(B, E, b, new_lens);
  int32_t* kept = kept_idx + ((long long)b * E.Hkv + hk) * E.keep;
  if (L <= E.keep) {  // (the whole cluster)
    for (int j = blockIdx.x * kThreads + t; j < E.keep; j += gridDim.x * kThreads) kept[j] = j < L ? j : -1;
    return;
  }
  const int share = ((L + gridDim.x - 1) / gridDim.x + 127) / 128 * 128, s0 = (int)min((long long)blockIdx.x * share, (long long)L), s1 = min(s0 + share, L);
  __syncthreads();
  select_kept<true>(E, hk, L, s0, s1, weights, share <= kSplitKeys ? reinterpret_cast<uint32_t*>(smem) : nullptr, sh,
                    [&](int i) { return B.page(b, i); }, [&](uint32_t j, int slot) { kept[j] = slot; });
  sm100::cluster_sync();  // the others have read this block's counts
}

// grid (c, Hkv, S), in place clusters of c
template <int D, bool kInPlace>
__global__ void __launch_bounds__(kThreads)
evict_move_kernel(const __grid_constant__ ChunkBatch B, const __grid_constant__ Evict E, uint4* kc, uint4* vc, float* weights,
                  const int32_t* __restrict__ new_table, int new_max_blocks, const int32_t* __restrict__ kept_idx) {
  pdl_wait();
  const int b = blockIdx.z, hk = blockIdx.y, L = B.len(b);
  if (kInPlace && L <= E.keep) return;  // (the whole cluster)
  const int32_t* kept = kept_idx + ((long long)b * E.Hkv + hk) * E.keep;
  const int32_t* row = new_table + (long long)b * new_max_blocks;
  move_rows<D, kInPlace>(B, E.Hkv, hk, min(L, E.keep), kc, vc, weights, [&](int j) { return kept[j]; }, [&](int i) { return B.page(b, i); },
                         [&](int i) { return row[i]; });
}

}  // namespace

int32_t launch_cache_evict(const ChunkBatch& b, int Hkv, int D, int keep, int keep_first, int keep_last, void* kc, void* vc,
                           float* weights, const int32_t* new_table, int new_max_blocks, int32_t* new_lens, int32_t* kept_idx,
                           cudaStream_t st) {
  const Evict E = {Hkv, keep, keep_first, keep_last};
  const bool in_place = new_table == b.table;
  // Blocks for each (sequence, KV head): two an SM at a time, where that is none two all the same (32 x 8 pairs: 209 us with one,
  // 192 with two, 195 with three), and no more than have rows to move.
  const long long pairs = (long long)b.S * Hkv, at_once = 2ll * sm_count();
  const long long slots = (long long)b.max_blocks * PG, kept = slots < keep ? slots : keep;
  const int rows = kThreads / (D / 8) * kMany;
  const long long fit = at_once / pairs, want = fit > 1 ? fit : pairs < 2 * at_once ? 2 : 1, useful = (kept + rows - 1) / rows;
  auto cluster_of = [](long long n) { return n >= 8 ? 8 : n >= 4 ? 4 : n >= 2 ? 2 : 1; };
  int c = (int)(want < useful ? want : useful);
  if (in_place) c = cluster_of(c);
  auto set_smem = [&](auto kern, size_t bytes) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    return e == cudaSuccess ? UNIGIST_OK : fail(UNIGIST_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
  };
  const FusedSmem fused(b.max_blocks, keep);
  if (fused.bytes <= kFusedMost) {
    const auto kern = D == 128 ? (in_place ? evict_fused_kernel<128, true> : evict_fused_kernel<128, false>)
                               : (in_place ? evict_fused_kernel<64, true> : evict_fused_kernel<64, false>);
    if (int32_t rc = set_smem(kern, kFusedMost)) return rc;
    {
      KernelScope ks("evict_fused_kernel", st);
      launch_chained(kern, dim3(c, Hkv, b.S), kThreads, fused.bytes, st, in_place ? c : 1, b, E, (uint4*)kc, (uint4*)vc, weights,
                     new_table, new_max_blocks, new_lens, kept_idx);
    }
    return check_launch("eviction kernel");
  }
  // a search is shared by as many blocks as run at once, and where that is too few by as many as hold its keys
  int split = cluster_of(fit);
  while (split < 8 && slots > (long long)split * kSplitKeys) split *= 2;
  const size_t share = ((size_t)slots / split + 256) / 128 * 128;  // keys, at most
  if (int32_t rc = set_smem(evict_select_kernel, kSplitKeys * 4)) return rc;
  {
    KernelScope ks("evict_select_kernel", st);
    launch_chained(evict_select_kernel, dim3(split, Hkv, b.S), kThreads, (share < kSplitKeys ? share : kSplitKeys) * 4, st, split, b, E,
                   (const float*)weights, new_lens, kept_idx);
  }
  if (int32_t rc = check_launch("eviction select kernel")) return rc;
  {
    KernelScope ks("evict_move_kernel", st);
    launch_chained(D == 128 ? (in_place ? evict_move_kernel<128, true> : evict_move_kernel<128, false>)
                            : (in_place ? evict_move_kernel<64, true> : evict_move_kernel<64, false>),
                   dim3(c, Hkv, b.S), kThreads, 0, st, in_place ? c : 1, b, E, (uint4*)kc, (uint4*)vc, weights, new_table, new_max_blocks,
                   (const int32_t*)kept_idx);
  }
  return check_launch("eviction move kernel");
}

}  // namespace ug
