// Entry points of the 8-bit cache's operators: the checks of their arguments, on the host alone (lengths and block ids live in
// device memory and are checked by the kernels).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/flowprefill.h"
#include "kernels.h"
#include "kv8_plan.h"

namespace {

fp_status refuse(const char* message) {
  fp::set_last_error(message);
  return FP_ERR_INVALID;
}
fp_status launched() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return FP_OK;
  fp::set_last_error(hipGetErrorString(e));
  return FP_ERR_DEVICE;
}
bool aligned16(const void* p) { return p && !(reinterpret_cast<uintptr_t>(p) & 15); }
bool aligned4(const void* p) { return p && !(reinterpret_cast<uintptr_t>(p) & 3); }

const char* bad_cache(const fp_kv8_cache* c) {
  if (!c) return "kv8: null cache";
  if (!aligned16(c->k_pool) || !aligned16(c->v_pool) || !aligned4(c->k_scale) || !aligned4(c->v_scale))
    return "kv8: null or misaligned pool or scales";
  if (c->num_blocks <= 0 || c->num_blocks > INT32_MAX) return "kv8: num_blocks must be in 1..2^31-1";
  if (c->n_kv_heads <= 0 || c->n_kv_heads > 65536) return "kv8: n_kv_heads must be in 1..65536";
  if (c->head_dim != 64 && c->head_dim != 128) return "kv8: head_dim must be 64 or 128";
  return nullptr;
}
const char* bad_batch(const fp_kv8_batch* b) {
  if (!b) return "kv8: null batch";
  if (b->n_seqs < 0 || (b->n_seqs > 0 && b->max_blocks <= 0)) return "kv8: negative n_seqs or max_blocks not positive";
  if (b->n_seqs > 0 && (!aligned4(b->cu_seqlens) || !aligned4(b->cached_lens) || !aligned4(b->block_tables)))
    return "kv8: null or misaligned cu_seqlens, cached_lens or block_tables";
  static_assert(fp::kKv8MaxBlocks == 1 << 26, "the message below");
  if (b->max_blocks > fp::kKv8MaxBlocks) return "kv8: max_blocks must be at most 2^26 (positions below 2^30)";
  return nullptr;
}
bool bad_heads(int32_t n_q_heads, int32_t n_kv_heads) { return n_q_heads <= 0 || n_q_heads > 65536 || n_q_heads % n_kv_heads; }
}  // namespace

extern "C" {

fp_status fp_op_kv8_append(const fp_kv8_cache* cache, const fp_kv8_batch* batch, const void* qkv, int64_t qkv_stride, int64_t n_tokens,
                           int32_t n_q_heads, const float* rope_cos, const float* rope_sin, int32_t max_position, void* q_out,
                           int64_t q_stride, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (const char* bad = bad_batch(batch)) return refuse(bad);
  const int64_t hkv = cache->n_kv_heads, dim = cache->head_dim;
  if (bad_heads(n_q_heads, cache->n_kv_heads)) return refuse("fp_op_kv8_append: n_q_heads must be a multiple of n_kv_heads");
  if (n_tokens < 0 || fp::kv8_too_large(n_tokens, batch->n_seqs, n_q_heads, cache->n_kv_heads)) return refuse("fp_op_kv8_append: bad number of tokens");
  if (max_position <= 0) return refuse("fp_op_kv8_append: max_position must be positive");
  if (n_tokens == 0 || batch->n_seqs == 0) return FP_OK;
  if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(rope_cos) || !aligned16(rope_sin))
    return refuse("fp_op_kv8_append: null or misaligned (16 bytes) qkv, q_out or rotation table");
  if (qkv_stride % 8 || q_stride % 8 || qkv_stride < (n_q_heads + 2 * hkv) * dim || q_stride < n_q_heads * dim)
    return refuse("fp_op_kv8_append: strides must be multiples of 8 and at least a row");
  if (q_out == qkv && q_stride != qkv_stride) return refuse("fp_op_kv8_append: in place needs q_stride == qkv_stride");
  fp::launch_kv8_append(*cache, *batch, qkv, qkv_stride, n_tokens, n_q_heads, rope_cos, rope_sin, max_position, q_out, q_stride,
                        reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

int64_t fp_op_kv8_attention_workspace_bytes(int64_t n_tokens, int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                            int32_t max_new, int32_t max_len) {
  if (n_tokens <= 0 || n_seqs <= 0 || n_kv_heads <= 0 || bad_heads(n_q_heads, n_kv_heads) || fp::kv8_too_large(n_tokens, n_seqs, n_q_heads, n_kv_heads) ||
      (head_dim != 64 && head_dim != 128) || max_new <= 0 || max_len <= 0)
    return 0;
  return (int64_t)fp::kv8_plan(n_tokens, n_seqs, n_q_heads, n_kv_heads, head_dim, max_new, max_len, SIZE_MAX).workspace;
}

fp_status fp_op_kv8_attention(const fp_kv8_cache* cache, const fp_kv8_batch* batch, const void* q, int64_t q_stride, void* o,
                              int64_t o_stride, int64_t n_tokens, int32_t n_q_heads, float scale, int32_t max_new, int32_t max_len,
                              void* workspace, int64_t workspace_bytes, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (const char* bad = bad_batch(batch)) return refuse(bad);
  const int64_t dim = cache->head_dim;
  if (bad_heads(n_q_heads, cache->n_kv_heads)) return refuse("fp_op_kv8_attention: n_q_heads must be a multiple of n_kv_heads");
  if (n_tokens < 0 || fp::kv8_too_large(n_tokens, batch->n_seqs, n_q_heads, cache->n_kv_heads)) return refuse("fp_op_kv8_attention: bad number of tokens");
  // (the kernels multiply the scores by scale * log2(e))
  if (!(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f))
    return refuse("fp_op_kv8_attention: scale must be positive, and finite also as scale * log2(e)");
  if (max_new <= 0 || max_len <= 0) return refuse("fp_op_kv8_attention: max_new and max_len must be positive");
  if (workspace_bytes < 0 || (workspace_bytes > 0 && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255))))
    return refuse("fp_op_kv8_attention: workspace null, misaligned (256 bytes) or negative size");
  if (n_tokens == 0 || batch->n_seqs == 0) return FP_OK;
  if (!aligned16(q) || !aligned16(o)) return refuse("fp_op_kv8_attention: null or misaligned (16 bytes) q or o");
  if (q_stride % 8 || o_stride % 8 || q_stride < n_q_heads * dim || o_stride < n_q_heads * dim)
    return refuse("fp_op_kv8_attention: strides must be multiples of 8 and at least a row");
  fp::launch_kv8_attention(*cache, *batch, q, q_stride, o, o_stride, n_tokens, n_q_heads, scale, max_new, max_len, workspace,
                           (size_t)workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

fp_status fp_op_kv8_gather(const fp_kv8_cache* cache, const int32_t* block_table, int64_t len, void* k_out, void* v_out, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (len < 0 || len > INT32_MAX || (len + 16) * cache->n_kv_heads >= 1 << 29) return refuse("fp_op_kv8_gather: bad length");
  if (len == 0) return FP_OK;
  if (!aligned4(block_table) || !aligned16(k_out) || !aligned16(v_out)) return refuse("fp_op_kv8_gather: null or misaligned block table or output");
  fp::launch_kv8_gather(*cache, block_table, len, k_out, v_out, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

}  // extern "C"
