// The paged cache of latent attention: normalising and rotating new tokens into it, and reading sequences back out of it (operator
// `rope_kvwrite` of Section 5.1's list, and what the expanded form's keys and values are projected from).  Both are bound by HBM.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "kv8.h"
#include "latent_plan.h"
#include "launch.h"

namespace fp {

namespace {

// Eight pairs of a head's rotated part, turned by the angles of their position.  Half layout: pair (j, j + P/2); interleaved: (2j, 2j + 1).
template <int P, bool INTERLEAVED>
__device__ __forceinline__ void rotate_pairs(const bf16* src, bf16* dst, int piece, f32x8 c, f32x8 sn) {
  const int lo = piece * (INTERLEAVED ? 16 : 8), hi = INTERLEAVED ? lo + 8 : lo + P / 2;
  const f32x8 x = Vec8<bf16>::load(src + lo), y = Vec8<bf16>::load(src + hi);
  f32x8 a, b;
  if (INTERLEAVED) {
    a = __builtin_shufflevector(x, y, 0, 2, 4, 6, 8, 10, 12, 14);
    b = __builtin_shufflevector(x, y, 1, 3, 5, 7, 9, 11, 13, 15);
  } else {
    a = x;
    b = y;
  }
  f32x8 ra, rb;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    ra[e] = a[e] * c[e] - b[e] * sn[e];
    rb[e] = b[e] * c[e] + a[e] * sn[e];
  }
  if (INTERLEAVED) {
    Vec8<bf16>::store(dst + lo, __builtin_shufflevector(ra, rb, 0, 8, 1, 9, 2, 10, 3, 11));
    Vec8<bf16>::store(dst + hi, __builtin_shufflevector(ra, rb, 4, 12, 5, 13, 6, 14, 7, 15));
  } else {
    Vec8<bf16>::store(dst + lo, ra);
    Vec8<bf16>::store(dst + hi, rb);
  }
}

constexpr int kHeadsPerTask = 32;                     // query heads that a wave rotates

}  // namespace

// ------------------------------------------------------------------------------------------
// Append.  One wave per task: the cache row of a token -- its latent, eight numbers a lane, normalised in fp32 over the wave, and the
// key's rotated part -- or the rotated parts of up to 32 of its query heads, eight pairs a lane.
// What bounds it: HBM.  8192 tokens of 20 heads move 63 MB in 13.9 us (4.5 TB/s; a copy of 1 GiB reaches 5.2 on the same card); 32 tokens of 128 heads
// take 4.0: a launch and the chain cached length -> block table or angles -> store.
// ------------------------------------------------------------------------------------------
template <int R, int P, bool INTERLEAVED>
__global__ __launch_bounds__(256) void latent_append_kernel(
    const bf16* __restrict__ latent, int64_t latent_stride, const bf16* __restrict__ gain, float eps, int64_t n_tokens,
    const float* __restrict__ rope_cos, const float* __restrict__ rope_sin, int max_position, int n_heads, int head_tasks, const bf16* q,
    int64_t q_stride, int64_t q_head_stride, bf16* q_out, int64_t q_out_stride, int64_t q_out_head_stride, bf16* __restrict__ pool,
    int64_t num_blocks, int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cached_lens,
    const int32_t* __restrict__ block_tables) {
  constexpr int PIECES = P / 16, ROW = R + P;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = task / (1 + head_tasks);
  const int part = (int)(task - t * (1 + head_tasks));
  if (t >= n_tokens) return;
  const int s = kv8_find_seq(cu_seqlens, n_seqs, t, n_tokens, 1, 1, 0);
  if (s < 0 || t >= cu_seqlens[s + 1] || t < cu_seqlens[s]) return;
  const int cached = cached_lens[s];
  const int64_t pos = (int64_t)cached + (t - cu_seqlens[s]);
  if (cached < 0 || pos >= max_position) return;
  const int piece = lane % PIECES;
  const f32x8 c = Vec8<float>::load(rope_cos + pos * (P / 2) + piece * 8), sn = Vec8<float>::load(rope_sin + pos * (P / 2) + piece * 8);
  if (part > 0) {
    const int first = (part - 1) * kHeadsPerTask, last = min(first + kHeadsPerTask, n_heads);
    const bf16* src = q + t * q_stride;
    bf16* dst = q_out + t * q_out_stride;
#pragma unroll
    for (int i = 0; i < kHeadsPerTask * PIECES / 64; ++i) {
      const int h = first + i * (64 / PIECES) + lane / PIECES;
      if (h < last) rotate_pairs<P, INTERLEAVED>(src + h * q_head_stride, dst + h * q_out_head_stride, piece, c, sn);
    }
    return;
  }
  const int64_t lb = pos / kLatentBlock;
  if (lb >= max_blocks) return;
  const int64_t blk = block_tables[(int64_t)s * max_blocks + lb];
  if (blk < 0 || blk >= num_blocks) return;
  const bf16* src = latent + t * latent_stride;
  bf16* dst = pool + (blk * kLatentBlock + pos % kLatentBlock) * ROW;
  f32x8 x = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, g = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
  if (lane < R / 8) {
    x = Vec8<bf16>::load(src + lane * 8);
    if (gain) g = Vec8<bf16>::load(gain + lane * 8);
  }
  if (lane < PIECES) rotate_pairs<P, INTERLEAVED>(src + R, dst + R, piece, c, sn);
  if (gain) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
    const float inv = rsqrtf(wave_sum(sum) * (1.0f / R) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * g[e];
  }
  if (lane < R / 8) Vec8<bf16>::store(dst + lane * 8, x);
}

// ------------------------------------------------------------------------------------------
// Gather.  One wave to half a block: eight rows, contiguous in the pool and, apart from the rotated parts, in the output.
// What bounds it: HBM.  70278 rows of 576 in scattered blocks, 162 MB read and written, take 39 us (4.1 TB/s) and 25 where the rows come out of the
// caches; 777 rows 4.6.
// ------------------------------------------------------------------------------------------
template <int R, int P>
__global__ __launch_bounds__(256) void latent_gather_kernel(const bf16* __restrict__ pool, int64_t num_blocks, int n_seqs, int max_blocks,
                                                            const int32_t* __restrict__ block_tables, const int32_t* __restrict__ cu_out,
                                                            int64_t n_rows, int64_t n_slots, bf16* __restrict__ latent_out,
                                                            bf16* __restrict__ rope_out) {
  constexpr int CH = (R + P) / 8, PER = (8 * CH + 63) / 64;
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t slot = task >> 1;
  if (slot >= n_slots) return;
  const int s = kv8_find_seq(cu_out, n_seqs, slot, n_slots, 1, kLatentBlock, 1);
  if (s < 0) return;
  const int64_t lo = cu_out[s], n = min((int64_t)cu_out[s + 1], n_rows) - lo;
  const int64_t lb = slot - kv8_slot(lo, s, kLatentBlock, 1);
  const int64_t pos0 = lb * kLatentBlock + (task & 1) * 8;
  if (lo < 0 || pos0 >= n) return;
  const int64_t blk = lb < max_blocks ? block_tables[(int64_t)s * max_blocks + lb] : -1;
  const bool have = blk >= 0 && blk < num_blocks;
  const int rows = (int)min(n - pos0, (int64_t)8);
  const bf16* src = pool + ((have ? blk : 0) * kLatentBlock + (task & 1) * 8) * (R + P);
  u32x4 v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = i * 64 + lane;
    v[i] = u32x4{0, 0, 0, 0};
    if (have && at < rows * CH) v[i] = *reinterpret_cast<const u32x4*>(src + at * 8);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int at = i * 64 + lane, row = at / CH, c = at - row * CH;
    if (at >= rows * CH) continue;
    const int64_t r = lo + pos0 + row;
    bf16* dst = c < R / 8 ? latent_out + r * R + c * 8 : rope_out + r * P + (c - R / 8) * 8;
    *reinterpret_cast<u32x4*>(dst) = v[i];
  }
}

namespace {

template <int R, int P>
void append_for(const fp_latent_cache& c, const fp_latent_batch& b, const bf16* latent, int64_t latent_stride, const bf16* gain, float eps,
                int64_t n_tokens, const float* rope_cos, const float* rope_sin, int max_position, int pairing, int n_heads, const bf16* q,
                int64_t q_stride, int64_t q_head_stride, bf16* q_out, int64_t q_out_stride, int64_t q_out_head_stride, hipStream_t s) {
  const int head_tasks = (n_heads + kHeadsPerTask - 1) / kHeadsPerTask;
  const int64_t tasks = n_tokens * (1 + head_tasks);
  launch_kernel(pairing == FP_ROPE_INTERLEAVED ? latent_append_kernel<R, P, true> : latent_append_kernel<R, P, false>,
                dim3((unsigned)((tasks + 3) / 4)), 256, 0, s, latent, latent_stride, gain, eps, n_tokens, rope_cos, rope_sin, max_position,
                n_heads, head_tasks, q, q_stride, q_head_stride, q_out, q_out_stride, q_out_head_stride, (bf16*)c.pool, c.num_blocks, b.n_seqs,
                b.max_blocks, b.cu_seqlens, b.cached_lens, b.block_tables);
}

template <int R, int P>
void gather_for(const fp_latent_cache& c, const fp_latent_batch& b, const int32_t* cu_out, int64_t n_rows, bf16* latent_out, bf16* rope_out,
                hipStream_t s) {
  const int64_t slots = kv8_slot(n_rows, b.n_seqs, kLatentBlock, 1);
  launch_kernel(latent_gather_kernel<R, P>, dim3((unsigned)((slots * 2 + 3) / 4)), 256, 0, s, (const bf16*)c.pool, c.num_blocks, b.n_seqs,
                b.max_blocks, b.block_tables, cu_out, n_rows, slots, latent_out, rope_out);
}

// `go` for the cache's widths.
template <typename F> void for_dims(const fp_latent_cache& c, F&& go) {
  auto rope = [&](auto r) {
    if (c.rope_dim == 64) go(r, std::integral_constant<int, 64>{});
    else go(r, std::integral_constant<int, 32>{});
  };
  if (c.latent_dim == 512) rope(std::integral_constant<int, 512>{});
  else if (c.latent_dim == 256) rope(std::integral_constant<int, 256>{});
  else rope(std::integral_constant<int, 128>{});
}

}  // namespace

void launch_latent_append(const fp_latent_cache& c, const fp_latent_batch& b, const void* latent, int64_t latent_stride, const void* gain,
                          float eps, int64_t n_tokens, const float* rope_cos, const float* rope_sin, int max_position, int pairing,
                          int n_heads, const void* q_rope, int64_t q_stride, int64_t q_head_stride, void* q_out, int64_t q_out_stride,
                          int64_t q_out_head_stride, hipStream_t s) {
  if (n_tokens == 0 || b.n_seqs == 0) return;
  for_dims(c, [&](auto r, auto p) {
    append_for<r(), p()>(c, b, (const bf16*)latent, latent_stride, (const bf16*)gain, eps, n_tokens, rope_cos, rope_sin, max_position, pairing,
                         n_heads, (const bf16*)q_rope, q_stride, q_head_stride, (bf16*)q_out, q_out_stride, q_out_head_stride, s);
  });
}

void launch_latent_gather(const fp_latent_cache& c, const fp_latent_batch& b, const int32_t* cu_out, int64_t n_rows, void* latent_out,
                          void* rope_out, hipStream_t s) {
  if (n_rows == 0 || b.n_seqs == 0) return;
  for_dims(c, [&](auto r, auto p) { gather_for<r(), p()>(c, b, cu_out, n_rows, (bf16*)latent_out, (bf16*)rope_out, s); });
}

}  // namespace fp
