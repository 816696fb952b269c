// C-ABI entry points of the calls on ragged chunks over a paged cache: argument validation, dispatch to the launchers.
#include <cmath>

#include "chunk.cuh"

using namespace ug;

namespace {

constexpr int kMaxGridYZ = 65535;
constexpr int kMaxBlocksPerSeq = 1 << 24;
constexpr int kMaxRows = 1 << 30;

int32_t check_num_rows(int32_t n) {
  if (n < 0) return fail(UNIGIST_ERR_INVALID_ARG, "the number of rows is below zero");
  if (n > kMaxRows) return fail(UNIGIST_ERR_SHAPE, "%d rows exceed %d", n, kMaxRows);
  return UNIGIST_OK;
}

int32_t check_heads(int32_t heads, int32_t D) {
  if (heads < 1) return fail(UNIGIST_ERR_INVALID_ARG, "the number of heads is not positive");
  if (heads > kMaxGridYZ) return fail(UNIGIST_ERR_SHAPE, "%d heads exceed %d", heads, kMaxGridYZ);
  if (D != 64 && D != 128) return fail(UNIGIST_ERR_SHAPE, "head_dim %d is not 64 or 128", D);
  return UNIGIST_OK;
}

int32_t check_group(int32_t Hq, int32_t Hkv) {
  if (Hq < 1) return fail(UNIGIST_ERR_INVALID_ARG, "the number of heads is not positive");
  if (Hq > kMaxGridYZ) return fail(UNIGIST_ERR_SHAPE, "%d heads exceed %d", Hq, kMaxGridYZ);
  if (Hq % Hkv) return fail(UNIGIST_ERR_SHAPE, "num_q_heads %d is not a multiple of num_kv_heads %d", Hq, Hkv);
  if (Hq / Hkv > 128) return fail(UNIGIST_ERR_UNSUPPORTED, "at most 128 query heads per KV head, got %d", Hq / Hkv);
  return UNIGIST_OK;
}

// Sizes of a batch over the cache.
int32_t check_cache(int32_t S, int32_t Hkv, int32_t D, int32_t num_blocks, int32_t max_blocks) {
  if (S < 1 || num_blocks < 1 || max_blocks < 1) return fail(UNIGIST_ERR_INVALID_ARG, "the batch or the cache has a non-positive size");
  if (int32_t rc = check_heads(Hkv, D)) return rc;
  if (S > kMaxGridYZ) return fail(UNIGIST_ERR_SHAPE, "num_seqs %d exceeds %d", S, kMaxGridYZ);
  if (max_blocks > kMaxBlocksPerSeq) return fail(UNIGIST_ERR_SHAPE, "%d pages per sequence exceed %d", max_blocks, kMaxBlocksPerSeq);
  if ((int64_t)num_blocks * Hkv * UNIGIST_PAGE_TOKENS > 0x7fffffffLL - 128) return fail(UNIGIST_ERR_SHAPE, "the cache has too many rows");
  return UNIGIST_OK;
}

// A [rows, heads, D] tensor with `stride` elements from row to row.
int32_t check_rows(const void* x, int64_t stride, int32_t rows, int32_t heads, int32_t D) {
  if (!x) return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned16(x) || stride % 8) return fail(UNIGIST_ERR_ALIGNMENT, "tensor pointers and rows must be 16-byte aligned");
  if (stride < (int64_t)heads * D) return fail(UNIGIST_ERR_SHAPE, "rows of %lld elements do not hold %d heads of %d", (long long)stride, heads, D);
  if (stride > 1ll << 36) return fail(UNIGIST_ERR_SHAPE, "rows too far apart");
  (void)rows;
  return UNIGIST_OK;
}
size_t rows_bytes(int64_t stride, int32_t rows, int32_t heads, int32_t D) {
  return rows > 0 ? ((size_t)(rows - 1) * (size_t)stride + (size_t)heads * D) * 2 : 0;
}

// Whether all of some 32-bit numbers' addresses (which may be null) are aligned.
template <typename... P>
bool aligned4(P... p) {
  return (((reinterpret_cast<uintptr_t>(p) & 3) == 0) && ...);
}
int32_t misaligned4() { return fail(UNIGIST_ERR_ALIGNMENT, "32-bit numbers must be 4-byte aligned"); }

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const char *x = (const char*)a, *y = (const char*)b;
  return a && b && a_bytes && b_bytes && x < y + b_bytes && y < x + a_bytes;
}

int32_t check_scale(float softmax_scale, int32_t D, float* scale) {
  if (!(softmax_scale >= 0.f) || std::isinf(softmax_scale)) return fail(UNIGIST_ERR_INVALID_ARG, "softmax_scale must be finite and >= 0");
  // (its reciprocal and products with scores and log-sum-exps have to be numbers)
  if (softmax_scale > 0.f && (softmax_scale < 1e-30f || softmax_scale > 1e30f))
    return fail(UNIGIST_ERR_UNSUPPORTED, "softmax_scale %g is not in 1e-30 .. 1e30", softmax_scale);
  *scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D);
  return UNIGIST_OK;
}

int32_t check_rope(int32_t D, const int32_t* pos_ids, int32_t num_axes, const uint8_t* freq_axis, float theta_base) {
  if (!pos_ids || !freq_axis) return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned4(pos_ids)) return misaligned4();
  if (num_axes < 1 || num_axes > 255) return fail(UNIGIST_ERR_INVALID_ARG, "num_axes %d is not in 1 .. 255", num_axes);
  if (!(theta_base > 1.f) || std::isinf(theta_base)) return fail(UNIGIST_ERR_INVALID_ARG, "theta_base must be finite and above 1");
  for (int j = 0; j < D / 2; ++j)
    if (freq_axis[j] >= num_axes) return fail(UNIGIST_ERR_INVALID_ARG, "freq_axis[%d] = %d names none of %d axes", j, freq_axis[j], num_axes);
  return UNIGIST_OK;
}

}  // namespace

extern "C" {

int32_t unigist_rope_axes(int32_t num_tokens, int32_t heads, int32_t head_dim, const void* src, int64_t src_stride, void* dst,
                          int64_t dst_stride, const int32_t* pos_ids, int32_t num_axes, const uint8_t* freq_axis,
                          float theta_base, uint32_t flags, void* stream) {
  if (int32_t rc = check_num_rows(num_tokens)) return rc;
  if (int32_t rc = check_heads(heads, head_dim)) return rc;
  if (flags & ~UNIGIST_ROPE_INVERSE) return fail(UNIGIST_ERR_INVALID_ARG, "unknown flags 0x%x", flags);
  static const int32_t no_positions = 0;
  if (int32_t rc = check_rope(head_dim, num_tokens ? pos_ids : &no_positions, num_axes, freq_axis, theta_base)) return rc;
  if (num_tokens == 0) return UNIGIST_OK;
  if (int32_t rc = check_rows(src, src_stride, num_tokens, heads, head_dim)) return rc;
  if (int32_t rc = check_rows(dst, dst_stride, num_tokens, heads, head_dim)) return rc;
  if (!(src == dst && src_stride == dst_stride) &&
      overlap(src, rows_bytes(src_stride, num_tokens, heads, head_dim), dst, rows_bytes(dst_stride, num_tokens, heads, head_dim)))
    return fail(UNIGIST_ERR_INVALID_ARG, "src and dst overlap and are not the same tensor");
  RopeAxes r;
  make_rope_axes(&r, head_dim, freq_axis, theta_base);
  return launch_rope_axes(r, num_tokens, heads, head_dim, (flags & UNIGIST_ROPE_INVERSE) != 0, src, src_stride, dst, dst_stride,
                          pos_ids, (cudaStream_t)stream);
}

int32_t unigist_chunk_append(int32_t S, int32_t Hkv, int32_t D, int32_t num_rows, const void* k_new, int64_t k_stride,
                             const void* v_new, int64_t v_stride, const int32_t* cu_rows, const int32_t* pos_ids,
                             int32_t num_axes, const uint8_t* freq_axis, float theta_base, void* kc, void* vc, float* weights,
                             int32_t num_blocks, const int32_t* table, int32_t max_blocks, const int32_t* seq_lens,
                             int32_t* new_lens, void* stream) {
  if (int32_t rc = check_cache(S, Hkv, D, num_blocks, max_blocks)) return rc;
  if (int32_t rc = check_num_rows(num_rows)) return rc;
  if (!cu_rows || !kc || !vc || !table || !seq_lens || !new_lens) return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned16(kc) || !aligned16(vc)) return fail(UNIGIST_ERR_ALIGNMENT, "tensor pointers must be 16-byte aligned");
  if (!aligned4(cu_rows, table, seq_lens, new_lens, weights)) return misaligned4();
  if (overlap(seq_lens, (size_t)S * 4, new_lens, (size_t)S * 4)) return fail(UNIGIST_ERR_INVALID_ARG, "new_lens overlaps seq_lens");
  if (num_rows > 0) {
    if (int32_t rc = check_rows(k_new, k_stride, num_rows, Hkv, D)) return rc;
    if (int32_t rc = check_rows(v_new, v_stride, num_rows, Hkv, D)) return rc;
  }
  RopeAxes r;
  if (pos_ids) {
    if (int32_t rc = check_rope(D, pos_ids, num_axes, freq_axis, theta_base)) return rc;
    make_rope_axes(&r, D, freq_axis, theta_base);
  }
  const ChunkBatch b = {cu_rows, seq_lens, table, S, num_rows, max_blocks, num_blocks};
  return launch_chunk_append(b, Hkv, D, k_new, k_stride, v_new, v_stride, pos_ids ? &r : nullptr, pos_ids, kc, vc, weights,
                             new_lens, (cudaStream_t)stream);
}

size_t unigist_chunk_attn_workspace_bytes(int32_t S, int32_t num_rows, int32_t Hq, int32_t Hkv, int32_t D, int32_t max_blocks) {
  if (check_num_rows(num_rows) != UNIGIST_OK || check_cache(S, Hkv, D, 1, max_blocks) != UNIGIST_OK || check_group(Hq, Hkv) != UNIGIST_OK) return 0;
  return chunk_attn_scratch_bytes(S, num_rows, Hq, Hkv, D, max_blocks);
}

int32_t unigist_chunk_attn(int32_t S, int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t num_rows, const void* q,
                           int64_t q_stride, const int32_t* cu_rows, const void* kc, const void* vc, int32_t num_blocks,
                           const int32_t* table, int32_t max_blocks, const int32_t* seq_lens, void* o, float* lse,
                           void* workspace, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_cache(S, Hkv, D, num_blocks, max_blocks)) return rc;
  if (int32_t rc = check_group(Hq, Hkv)) return rc;
  if (int32_t rc = check_num_rows(num_rows)) return rc;
  float scale;
  if (int32_t rc = check_scale(softmax_scale, D, &scale)) return rc;
  if (num_rows == 0) return UNIGIST_OK;
  if (!cu_rows || !kc || !vc || !table || !seq_lens || !o) return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (int32_t rc = check_rows(q, q_stride, num_rows, Hq, D)) return rc;
  if (!aligned16(kc) || !aligned16(vc) || !aligned16(o) || !aligned16(workspace))
    return fail(UNIGIST_ERR_ALIGNMENT, "tensor pointers must be 16-byte aligned");
  if (!aligned4(cu_rows, table, seq_lens, lse)) return misaligned4();
  if (overlap(q, rows_bytes(q_stride, num_rows, Hq, D), o, rows_bytes((int64_t)Hq * D, num_rows, Hq, D)))
    return fail(UNIGIST_ERR_INVALID_ARG, "o overlaps q");
  const size_t need = chunk_attn_scratch_bytes(S, num_rows, Hq, Hkv, D, max_blocks);
  if (!workspace || ws_bytes < need)
    return fail(UNIGIST_ERR_WORKSPACE, "chunk attention needs %zu bytes of workspace, got %zu", need, ws_bytes);
  const size_t o_bytes = rows_bytes((int64_t)Hq * D, num_rows, Hq, D), lse_bytes = lse ? (size_t)num_rows * Hq * 4 : 0;
  const size_t cache_bytes = (size_t)num_blocks * Hkv * UNIGIST_PAGE_TOKENS * D * 2;
  const struct {
    const void* p;
    size_t bytes;
  } others[] = {{kc, cache_bytes}, {vc, cache_bytes}, {cu_rows, ((size_t)S + 1) * 4}, {table, (size_t)S * max_blocks * 4}, {seq_lens, (size_t)S * 4}, {workspace, need}};
  for (const auto& x : others)
    if (overlap(o, o_bytes, x.p, x.bytes) || overlap(lse, lse_bytes, x.p, x.bytes))
      return fail(UNIGIST_ERR_INVALID_ARG, "o or lse overlaps an input or the workspace");
  if (overlap(o, o_bytes, lse, lse_bytes) || overlap(lse, lse_bytes, q, rows_bytes(q_stride, num_rows, Hq, D)))
    return fail(UNIGIST_ERR_INVALID_ARG, "lse overlaps o or q");
  const ChunkBatch b = {cu_rows, seq_lens, table, S, num_rows, max_blocks, num_blocks};
  return launch_chunk_attn(b, Hq, Hkv, D, scale, q, q_stride, kc, vc, o, lse, workspace, (cudaStream_t)stream);
}

int32_t unigist_cache_weigh(int32_t S, int32_t Hq, int32_t Hkv, int32_t D, float softmax_scale, int32_t num_rows, const void* q,
                            int64_t q_stride, const int32_t* cu_rows, const float* lse, const void* kc, int32_t num_blocks,
                            const int32_t* table, int32_t max_blocks, const int32_t* seq_lens, const float* weights_in,
                            float decay, float* weights_out, void* stream) {
  if (int32_t rc = check_cache(S, Hkv, D, num_blocks, max_blocks)) return rc;
  if (int32_t rc = check_group(Hq, Hkv)) return rc;
  if (int32_t rc = check_num_rows(num_rows)) return rc;
  float scale;
  if (int32_t rc = check_scale(softmax_scale, D, &scale)) return rc;
  if (!(decay >= 0.f && decay <= 1.f)) return fail(UNIGIST_ERR_INVALID_ARG, "decay is not in 0 .. 1");
  if (!cu_rows || !kc || !table || !seq_lens || !weights_out || (decay > 0.f && !weights_in))
    return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned16(kc)) return fail(UNIGIST_ERR_ALIGNMENT, "tensor pointers must be 16-byte aligned");
  if (!aligned4(cu_rows, lse, table, seq_lens, weights_in, weights_out)) return misaligned4();
  if (num_rows > 0) {
    if (!lse) return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
    if (int32_t rc = check_rows(q, q_stride, num_rows, Hq, D)) return rc;
  }
  const size_t bytes = (size_t)num_blocks * Hkv * UNIGIST_PAGE_TOKENS * 4;
  if (decay > 0.f && weights_in != weights_out && overlap(weights_in, bytes, weights_out, bytes))
    return fail(UNIGIST_ERR_INVALID_ARG, "weights_in and weights_out overlap and are not the same tensor");
  const ChunkBatch b = {cu_rows, seq_lens, table, S, num_rows, max_blocks, num_blocks};
  return launch_cache_weigh(b, Hq, Hkv, D, scale, q, q_stride, lse, kc, weights_in, decay, weights_out, (cudaStream_t)stream);
}

int32_t unigist_cache_evict(int32_t S, int32_t Hkv, int32_t D, int32_t keep, int32_t keep_first, int32_t keep_last, void* kc,
                            void* vc, float* weights, int32_t num_blocks, const int32_t* table, int32_t max_blocks,
                            const int32_t* seq_lens, const int32_t* new_table, int32_t new_max_blocks, int32_t* new_lens,
                            int32_t* kept_idx, void* stream) {
  if (int32_t rc = check_cache(S, Hkv, D, num_blocks, max_blocks)) return rc;
  if (keep < 1 || keep_first < 0 || keep_last < 0) return fail(UNIGIST_ERR_INVALID_ARG, "keep is not positive, or a part of it below zero");
  if (keep > kMaxRows) return fail(UNIGIST_ERR_SHAPE, "keep %d exceeds %d", keep, kMaxRows);
  if ((int64_t)keep_first + keep_last > keep)
    return fail(UNIGIST_ERR_INVALID_ARG, "keep_first %d and keep_last %d exceed keep %d", keep_first, keep_last, keep);
  if (!kc || !vc || !weights || !table || !seq_lens || !new_table || !new_lens || !kept_idx)
    return fail(UNIGIST_ERR_INVALID_ARG, "a pointer is NULL");
  if (!aligned16(kc) || !aligned16(vc) || !aligned16(weights)) return fail(UNIGIST_ERR_ALIGNMENT, "tensor pointers must be 16-byte aligned");
  if (!aligned4(table, seq_lens, new_table, new_lens, kept_idx)) return misaligned4();
  if (overlap(seq_lens, (size_t)S * 4, new_lens, (size_t)S * 4)) return fail(UNIGIST_ERR_INVALID_ARG, "new_lens overlaps seq_lens");
  const int64_t most = (int64_t)max_blocks * UNIGIST_PAGE_TOKENS < keep ? (int64_t)max_blocks * UNIGIST_PAGE_TOKENS : keep;
  if (new_max_blocks < 1 || (int64_t)new_max_blocks * UNIGIST_PAGE_TOKENS < most)
    return fail(UNIGIST_ERR_SHAPE, "the new table has %d entries per sequence, %lld slots are kept", new_max_blocks, (long long)most);
  if (new_table == table ? new_max_blocks != max_blocks
                         : overlap(table, (size_t)S * max_blocks * 4, new_table, (size_t)S * new_max_blocks * 4))
    return fail(UNIGIST_ERR_INVALID_ARG, "the new table overlaps the old one and is not the same");
  const ChunkBatch b = {nullptr, seq_lens, table, S, 0, max_blocks, num_blocks};
  return launch_cache_evict(b, Hkv, D, keep, keep_first, keep_last, kc, vc, weights, new_table, new_max_blocks, new_lens, kept_idx,
                            (cudaStream_t)stream);
}

}  // extern "C"
