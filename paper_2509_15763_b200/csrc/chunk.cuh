// What the calls on ragged chunks over a paged cache share: the batch as the kernels see it, and their launchers.
#pragma once
#include <cuda.h>

#include "ug_common.cuh"

namespace ug {

// S sequences; rows [cu[b], cu[b + 1]) of the row tensors are the chunk of sequence b, whose cache holds lens[b] tokens in the
// pages that its row of the table names.  All of it lies on the device, so nothing that is read here is trusted: rows are
// held inside [0, num_rows], lengths inside the table, pages inside the cache.
struct ChunkBatch {
  const int32_t *cu, *lens, *table;
  int S, num_rows, max_blocks, num_blocks;
  __host__ __device__ __forceinline__ int rows(int b, int& row0) const {
    row0 = min(max(cu[b], 0), num_rows);
    return max(min(cu[b + 1], num_rows), row0) - row0;  // (in this order: an end near the least int has no difference to row0)
  }
  __host__ __device__ __forceinline__ int len(int b) const { return min(max(lens[b], 0), max_blocks * UNIGIST_PAGE_TOKENS); }
  __device__ __forceinline__ int page(int b, int i) const {  // i < max_blocks
    return min(max(table[(long long)b * max_blocks + i], 0), num_blocks - 1);
  }
};

// Running totals of a 64-bit cost over the sequences, which are taken in groups of `per` neighbours, one group a thread:
// first[t] = cost of the groups before t, first[kThreads] = all.  `tmp`: one number per warp.  Whole blocks of kThreads
// threads; ends with a barrier.
template <int kThreads, typename Cost>
__device__ __forceinline__ void cost_prefix(int S, int per, long long* first, long long* tmp, Cost cost) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int s0 = (int)min((long long)threadIdx.x * per, (long long)S), s1 = min(s0 + per, S);
  long long sum = 0;
  for (int i = s0; i < s1; ++i) sum += cost(i);
  long long incl = sum;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, incl, off);
    if (lane >= off) incl += x;
  }
  if (lane == 31) tmp[warp] = incl;
  __syncthreads();
  long long at = incl - sum;
  for (int w = 0; w < warp; ++w) at += tmp[w];
  first[threadIdx.x] = at;
  if (threadIdx.x == kThreads - 1) first[kThreads] = at + sum;
  __syncthreads();
}
// The last of the groups 0 .. last that begins at or before `at`.
__device__ __forceinline__ int cost_group(const long long* first, int last, long long at) {
  int lo = 0, hi = last;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= at) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Where share c of n begins when `total` is dealt out evenly: rounded, but in one way everywhere (no contraction, no
// approximation), rising with c, and exact at both ends.
__device__ __forceinline__ long long share_begin(long long total, int n, int c) {
  return c >= n ? total : (long long)__fmul_rn((float)c, __fdiv_rn((float)total, (float)n));
}

// Rotary embedding by given positions: pair j of a head turns by pos[axis[j]][token] * inv_freq[j].
struct RopeAxes {
  double inv_freq[64];
  uint8_t axis[64];
};
// (const uint8_t freq_axis[head_dim / 2], theta_base) -> the kernel's parameters
void make_rope_axes(RopeAxes* r, int head_dim, const uint8_t* freq_axis, float theta_base);

int32_t launch_rope_axes(const RopeAxes& r, int tokens, int heads, int D, bool inverse, const void* src, int64_t src_stride,
                         void* dst, int64_t dst_stride, const int32_t* pos, cudaStream_t st);
// r null: the keys are copied as they are.
int32_t launch_chunk_append(const ChunkBatch& b, int Hkv, int D, const void* k_new, int64_t k_stride, const void* v_new,
                            int64_t v_stride, const RopeAxes* r, const int32_t* pos, void* kc, void* vc, float* weights,
                            int32_t* new_lens, cudaStream_t st);
size_t chunk_attn_scratch_bytes(int S, int num_rows, int Hq, int Hkv, int D, int max_blocks);
int32_t launch_chunk_attn(const ChunkBatch& b, int Hq, int Hkv, int D, float scale, const void* q, int64_t q_stride,
                          const void* kc, const void* vc, void* o, float* lse, void* ws, cudaStream_t st);
int32_t chunk_attn_timeout_flag(unsigned int** at);
int32_t chunk_few_timeout_flag(unsigned int** at);
int32_t chunk_thin_timeout_flag(unsigned int** at);
int32_t launch_cache_weigh(const ChunkBatch& b, int Hq, int Hkv, int D, float scale, const void* q, int64_t q_stride,
                           const float* lse, const void* kc, const float* weights_in, float decay, float* weights_out,
                           cudaStream_t st);
int32_t cache_weigh_timeout_flag(unsigned int** at);
int32_t launch_cache_evict(const ChunkBatch& b, int Hkv, int D, int keep, int keep_first, int keep_last, void* kc, void* vc,
                           float* weights, const int32_t* new_table, int new_max_blocks, int32_t* new_lens, int32_t* kept_idx,
                           cudaStream_t st);

}  // namespace ug
