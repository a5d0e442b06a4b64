// Entry points of latent attention: the checks of their arguments, on the host alone (lengths and block ids live in device memory and are
// checked by the kernels).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/flowprefill.h"
#include "kernels.h"
#include "latent_plan.h"

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
bool aligned(const void* p, unsigned to) { return p && !(reinterpret_cast<uintptr_t>(p) & (to - 1)); }
constexpr int64_t kMaxStride = 1 << 23;               // elements: 64 rows of a tile stay within 2^30 bytes
bool stride_ok(int64_t stride, int64_t row) { return stride % 8 == 0 && stride >= row && stride <= INT64_MAX / 4; }

const char* bad_cache(const fp_latent_cache* c) {
  if (!c) return "latent: null cache";
  if (!aligned(c->pool, 16)) return "latent: null or misaligned pool";
  if (c->num_blocks <= 0 || c->num_blocks > INT32_MAX) return "latent: num_blocks must be in 1..2^31-1";
  if (!fp::latent_dims(c->latent_dim, c->rope_dim)) return "latent: latent_dim must be 128, 256 or 512 and rope_dim 32 or 64";
  return nullptr;
}
const char* bad_batch(const fp_latent_batch* b) {
  if (!b) return "latent: null batch";
  if (b->n_seqs < 0 || (b->n_seqs > 0 && b->max_blocks <= 0)) return "latent: negative n_seqs or max_blocks not positive";
  if (b->n_seqs > 0 && !aligned(b->block_tables, 4)) return "latent: null or misaligned block_tables";
  static_assert(fp::kLatentMaxBlocks == 1 << 26, "the message below");
  if (b->max_blocks > fp::kLatentMaxBlocks) return "latent: max_blocks must be at most 2^26 (positions below 2^30)";
  return nullptr;
}
const char* bad_lengths(const fp_latent_batch* b) {
  if (b->n_seqs > 0 && (!aligned(b->cu_seqlens, 4) || !aligned(b->cached_lens, 4))) return "latent: null or misaligned cu_seqlens or cached_lens";
  return nullptr;
}
// (the kernels multiply the scores by scale * log2(e))
bool bad_scale(float scale) { return !(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f); }
bool bad_workspace(const void* p, int64_t bytes) { return bytes < 0 || (bytes > 0 && !aligned(p, 256)); }
bool bad_heads(int32_t n) { return n <= 0 || n > 65536; }

}  // namespace

extern "C" {

fp_status fp_op_latent_append(const fp_latent_cache* cache, const fp_latent_batch* batch, const void* latent, int64_t latent_stride,
                              const void* gain, float eps, int64_t n_tokens, const float* rope_cos, const float* rope_sin,
                              int32_t max_position, int32_t pairing, int32_t n_q_heads, const void* q_rope, int64_t q_stride,
                              int64_t q_head_stride, void* q_out, int64_t q_out_stride, int64_t q_out_head_stride, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (const char* bad = bad_batch(batch)) return refuse(bad);
  if (const char* bad = bad_lengths(batch)) return refuse(bad);
  if (n_q_heads < 0 || n_q_heads > 65536) return refuse("fp_op_latent_append: n_q_heads must be in 0..65536");
  if (n_tokens < 0 || fp::latent_too_large(n_tokens, batch->n_seqs, n_q_heads > 0 ? n_q_heads : 1))
    return refuse("fp_op_latent_append: bad number of tokens");
  if (max_position <= 0) return refuse("fp_op_latent_append: max_position must be positive");
  if (pairing != FP_ROPE_HALF && pairing != FP_ROPE_INTERLEAVED) return refuse("fp_op_latent_append: unknown pairing");
  if (gain && !(eps >= 0.f && std::isfinite(eps))) return refuse("fp_op_latent_append: eps must be finite and not negative");
  if (n_tokens == 0 || batch->n_seqs == 0) return FP_OK;
  if (!aligned(latent, 16) || !aligned(rope_cos, 16) || !aligned(rope_sin, 16) || (gain && !aligned(gain, 16)))
    return refuse("fp_op_latent_append: null or misaligned (16 bytes) latent, gain or rotation table");
  if (!stride_ok(latent_stride, cache->latent_dim + cache->rope_dim))
    return refuse("fp_op_latent_append: strides must be multiples of 8 and at least a row");
  if (n_q_heads > 0) {
    const int64_t rope = cache->rope_dim, more = n_q_heads - 1;
    if (!aligned(q_rope, 16) || !aligned(q_out, 16)) return refuse("fp_op_latent_append: null or misaligned (16 bytes) q_rope or q_out");
    if (!stride_ok(q_head_stride, rope) || !stride_ok(q_out_head_stride, rope) || q_head_stride > kMaxStride || q_out_head_stride > kMaxStride ||
        !stride_ok(q_stride, more * q_head_stride + rope) || !stride_ok(q_out_stride, more * q_out_head_stride + rope))
      return refuse("fp_op_latent_append: strides must be multiples of 8 and at least a row");
    if (q_out == q_rope && (q_stride != q_out_stride || q_head_stride != q_out_head_stride))
      return refuse("fp_op_latent_append: in place needs equal strides");
  }
  fp::launch_latent_append(*cache, *batch, latent, latent_stride, gain, eps, n_tokens, rope_cos, rope_sin, max_position, pairing, n_q_heads,
                           q_rope, q_stride, q_head_stride, q_out, q_out_stride, q_out_head_stride, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

fp_status fp_op_latent_gather(const fp_latent_cache* cache, const fp_latent_batch* batch, const int32_t* cu_out, int64_t n_rows,
                              void* latent_out, void* rope_out, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (const char* bad = bad_batch(batch)) return refuse(bad);
  // (a launch has fewer than 2^32 threads: 128 for a slot, two slots to a workgroup)
  if (n_rows < 0 || n_rows > INT32_MAX || n_rows / 16 + (int64_t)batch->n_seqs >= (1 << 25) - 1) return refuse("fp_op_latent_gather: bad number of rows");
  if (n_rows == 0 || batch->n_seqs == 0) return FP_OK;
  if (!aligned(cu_out, 4) || !aligned(latent_out, 16) || !aligned(rope_out, 16))
    return refuse("fp_op_latent_gather: null or misaligned cu_out or output");
  fp::launch_latent_gather(*cache, *batch, cu_out, n_rows, latent_out, rope_out, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

int64_t fp_op_latent_attention_workspace_bytes(int64_t n_tokens, int32_t n_seqs, int32_t n_q_heads, int32_t latent_dim, int32_t rope_dim,
                                               int32_t max_new, int32_t max_len) {
  if (n_tokens <= 0 || n_seqs <= 0 || bad_heads(n_q_heads) || fp::latent_too_large(n_tokens, n_seqs, n_q_heads) ||
      !fp::latent_dims(latent_dim, rope_dim) || max_new <= 0 || max_len <= 0)
    return 0;
  return (int64_t)fp::latent_plan(n_tokens, n_seqs, n_q_heads, latent_dim, 1, max_new, max_len, SIZE_MAX).workspace;
}

fp_status fp_op_latent_attention(const fp_latent_cache* cache, const fp_latent_batch* batch, const void* q, int64_t q_stride, void* o,
                                 int64_t o_stride, int64_t n_tokens, int32_t n_q_heads, float scale, int32_t max_new, int32_t max_len,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
  if (const char* bad = bad_cache(cache)) return refuse(bad);
  if (const char* bad = bad_batch(batch)) return refuse(bad);
  if (const char* bad = bad_lengths(batch)) return refuse(bad);
  if (bad_heads(n_q_heads)) return refuse("fp_op_latent_attention: n_q_heads must be in 1..65536");
  if (n_tokens < 0 || fp::latent_too_large(n_tokens, batch->n_seqs, n_q_heads)) return refuse("fp_op_latent_attention: bad number of tokens");
  if (bad_scale(scale)) return refuse("fp_op_latent_attention: scale must be positive, and finite also as scale * log2(e)");
  if (max_new <= 0 || max_len <= 0) return refuse("fp_op_latent_attention: max_new and max_len must be positive");
  if (bad_workspace(workspace, workspace_bytes)) return refuse("fp_op_latent_attention: workspace null, misaligned (256 bytes) or negative size");
  if (n_tokens == 0 || batch->n_seqs == 0) return FP_OK;
  if (!aligned(q, 16) || !aligned(o, 16)) return refuse("fp_op_latent_attention: null or misaligned (16 bytes) q or o");
  if (!stride_ok(q_stride, (int64_t)n_q_heads * (cache->latent_dim + cache->rope_dim)) || !stride_ok(o_stride, (int64_t)n_q_heads * cache->latent_dim))
    return refuse("fp_op_latent_attention: strides must be multiples of 8 and at least a row");
  fp::launch_latent_attention(*cache, *batch, q, q_stride, o, o_stride, n_tokens, n_q_heads, scale, max_new, max_len, workspace,
                              (size_t)workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

int64_t fp_op_latent_expanded_attention_workspace_bytes(int64_t n_tokens, int32_t n_seqs, int32_t n_heads, int32_t v_dim, int32_t max_new,
                                                        int32_t max_len) {
  if (n_tokens <= 0 || n_seqs <= 0 || bad_heads(n_heads) || fp::latent_too_large(n_tokens, n_seqs, n_heads) || (v_dim != 64 && v_dim != 128) ||
      max_new <= 0 || max_len <= 0)
    return 0;
  return (int64_t)fp::expanded_plan(n_tokens, n_seqs, n_heads, v_dim, max_new, max_len, SIZE_MAX).workspace;
}

fp_status fp_op_latent_expanded_attention(const int32_t* cu_seqlens, const int32_t* cu_kv, int32_t n_seqs, const void* q, int64_t q_stride,
                                          const void* kv, int64_t kv_stride, const void* k_rope, int64_t k_rope_stride, void* o,
                                          int64_t o_stride, int64_t n_tokens, int64_t n_rows, int32_t n_heads, int32_t nope_dim,
                                          int32_t rope_dim, int32_t v_dim, float scale, int32_t max_new, int32_t max_len, void* workspace,
                                          int64_t workspace_bytes, void* hip_stream) {
  if (!fp::expanded_dims(nope_dim, rope_dim, v_dim))
    return refuse("fp_op_latent_expanded_attention: nope_dim and v_dim must be 64 or 128 and rope_dim 32 or 64");
  if (bad_heads(n_heads)) return refuse("fp_op_latent_expanded_attention: n_heads must be in 1..65536");
  if (n_seqs < 0 || n_tokens < 0 || fp::latent_too_large(n_tokens, n_seqs, n_heads) || n_rows < 0 || n_rows > 1 << 30)
    return refuse("fp_op_latent_expanded_attention: bad number of sequences, tokens or rows");
  if (bad_scale(scale)) return refuse("fp_op_latent_expanded_attention: scale must be positive, and finite also as scale * log2(e)");
  if (max_new <= 0 || max_len <= 0) return refuse("fp_op_latent_expanded_attention: max_new and max_len must be positive");
  if (bad_workspace(workspace, workspace_bytes))
    return refuse("fp_op_latent_expanded_attention: workspace null, misaligned (256 bytes) or negative size");
  if (n_tokens == 0 || n_seqs == 0) return FP_OK;
  if (!aligned(cu_seqlens, 4) || !aligned(cu_kv, 4)) return refuse("fp_op_latent_expanded_attention: null or misaligned cu_seqlens or cu_kv");
  if (!aligned(q, 16) || !aligned(o, 16) || !aligned(kv, 16) || !aligned(k_rope, 16))
    return refuse("fp_op_latent_expanded_attention: null or misaligned (16 bytes) q, kv, k_rope or o");
  if (!stride_ok(q_stride, (int64_t)n_heads * (nope_dim + rope_dim)) || !stride_ok(o_stride, (int64_t)n_heads * v_dim) ||
      !stride_ok(kv_stride, (int64_t)n_heads * (nope_dim + v_dim)) || !stride_ok(k_rope_stride, rope_dim) || kv_stride > kMaxStride ||
      k_rope_stride > kMaxStride)
    return refuse("fp_op_latent_expanded_attention: strides must be multiples of 8 and at least a row, those of kv and k_rope at most 2^23");
  const fp::ExpandedArgs args{cu_seqlens, cu_kv, n_seqs, q, q_stride, kv, kv_stride, k_rope, k_rope_stride, o, o_stride, n_tokens, n_rows,
                              n_heads, nope_dim, rope_dim, v_dim, scale};
  fp::launch_latent_expanded(args, max_new, max_len, workspace, (size_t)workspace_bytes, reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

fp_status fp_op_gemm_heads(const void* a, int64_t a_stride, int64_t a_head_stride, const void* w, int64_t w_head_stride, void* c,
                           int64_t c_stride, int64_t c_head_stride, int64_t m, int32_t n_heads, int64_t n, int64_t k, void* hip_stream) {
  if (m < 0 || bad_heads(n_heads) || n <= 0 || k <= 0 || n % 8 || k % 8 || n > 1 << 20 || k > 1 << 20)
    return refuse("fp_op_gemm_heads: n and k must be positive multiples of 8, at most 2^20, and n_heads in 1..65536");
  // (a launch has fewer than 2^32 threads: 256 for 16 tokens and 128 outputs of a head)
  if (m > INT32_MAX || (m + 127) / 128 * 8 * n_heads * ((n + 127) / 128) >= 1 << 24) return refuse("fp_op_gemm_heads: too large");
  if (m == 0) return FP_OK;
  if (!aligned(a, 16) || !aligned(w, 16) || !aligned(c, 16)) return refuse("fp_op_gemm_heads: null or misaligned (16 bytes) operand");
  if (!stride_ok(a_head_stride, k) || !stride_ok(c_head_stride, n) || !stride_ok(w_head_stride, n * k) || a_head_stride > 1ll << 40 ||
      c_head_stride > 1ll << 40 || !stride_ok(a_stride, (n_heads - 1) * a_head_stride + k) || !stride_ok(c_stride, (n_heads - 1) * c_head_stride + n))
    return refuse("fp_op_gemm_heads: strides must be multiples of 8 and at least what they step over");
  fp::launch_gemm_heads(a, a_stride, a_head_stride, w, w_head_stride, c, c_stride, c_head_stride, m, n_heads, n, k,
                        reinterpret_cast<hipStream_t>(hip_stream));
  return launched();
}

}  // extern "C"
