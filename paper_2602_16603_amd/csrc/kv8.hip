// The 8-bit paged KV cache: rotating and quantising new tokens into it, and reading a sequence back out of it (operator
// `rope_kvwrite` of Section 5.1's list, and the hand-over to a decode instance, on a cache of half the bytes).  Both are bound by HBM.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "kv8.h"
#include "launch.h"

namespace fp {

namespace {

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // e in [-126, 127]
__device__ __forceinline__ int exponent_of(float scale) { return (int)((__float_as_uint(scale) >> 23) & 255) - 127; }

// Exponent of the smallest power of two that brings `amax` down to 448 = 1.75 * 2^8.
__device__ __forceinline__ int scale_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
  return min(max(e, kKv8MinExp), kKv8MaxExp);
}

// fp64 -> fp32 rounded to odd (a value that fp32 does not hold gets an odd last bit, towards zero), so that rounding the result to
// e4m3 rounds the fp64 value once; rounding to nearest twice moves values that lie next to a midpoint of two codes.  Beyond fp32:
// the largest finite value, which quantises alike.
__device__ __forceinline__ float round_to_odd(double d) {
  uint64_t u = __builtin_bit_cast(uint64_t, d);
  u = (u & ~0x1fffffffull) | ((u & 0x1fffffffull) ? 0x20000000ull : 0ull);
  const float f = (float)__builtin_bit_cast(double, u);
  const bool over = __builtin_isinf(f) && !__builtin_isinf(d);
  return over ? __builtin_copysignf(3.402823466e38f, f) : f;
}

__device__ __forceinline__ float finite_abs(float v) {
  const float a = __builtin_fabsf(v);
  return a < __builtin_inff() ? a : 0.f;
}

// x / scale within the codes' range; NaN stays.
__device__ __forceinline__ float to_range(float x, float inv) {
  const float y = x * inv;
  return y != y ? y : __builtin_fminf(__builtin_fmaxf(y, -448.f), 448.f);
}
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
// Four codes rounded to a scale 2^-by times as fine (by <= 0).
__device__ __forceinline__ uint32_t requantise4(uint32_t codes, int by) {
  float v[4];
  v[0] = __builtin_amdgcn_cvt_f32_fp8(codes, 0); v[1] = __builtin_amdgcn_cvt_f32_fp8(codes, 1);
  v[2] = __builtin_amdgcn_cvt_f32_fp8(codes, 2); v[3] = __builtin_amdgcn_cvt_f32_fp8(codes, 3);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], by);
  return pack4(v[0], v[1], v[2], v[3]);
}

template <typename V> __device__ __forceinline__ V load_as(const void* p) { return *reinterpret_cast<const V*>(p); }

}  // namespace

// ------------------------------------------------------------------------------------------
// Append.  One wave per task:
//   keys   (block that gets tokens, kv head): four lanes to a token, each with D/8 channels of both halves of the rotation, so
//          a pair is in one lane and a token's codes leave as 16-byte (D = 64: 8-byte) pieces
//   values (block, kv head): a lane holds two channels of 16 tokens (D = 64: of 8) and writes them as the transposed block
//          wants them
//   queries (token): eight channels of both halves per lane, several heads one after the other with the same angles.
// The largest value of a block is known to its wave alone, so the scale costs one reduction over the wave and no second
// pass; the order of the tokens in memory needs no list from the host (kv8_plan.h).  Keys are rotated in fp64: an fp32 rotation puts
// keys that lie next to a border between two codes on its other side now and then, and a long prompt is bound by its bytes all the same.
//
// What bounds it: HBM.  8192 tokens of 40/8 heads of 128 move 222 MB in 50 us, 4096 tokens of 32/8 in five sequences 94 MB in 22.5
// (4.4 and 4.2 TB/s; a copy of 2 GiB reaches 4.9 on the same card).  One token of a sequence takes 5.2 us, 64 of them 6.8: a launch
// and the chain cached length -> block table -> old scale -> old codes, each an access to memory.
// ------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void kv8_append_kernel(
    const bf16* qkv, int64_t qkv_stride, bf16* q_out, int64_t q_stride, int64_t n_tokens, int n_q_heads,
    const float* __restrict__ rope_cos, const float* __restrict__ rope_sin, int max_position, uint8_t* __restrict__ k_pool,
    uint8_t* __restrict__ v_pool, float* __restrict__ k_scale, float* __restrict__ v_scale, int64_t num_blocks, int n_kv_heads,
    int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cached_lens,
    const int32_t* __restrict__ block_tables, int n_slots) {
  constexpr int HALF = D / 2;
  const int lane = threadIdx.x & 63;
  const int task = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (task >= n_slots * 2 * n_kv_heads) {
    // ---- queries of one token ----
    const int t = task - n_slots * 2 * n_kv_heads;
    if (t >= n_tokens) return;
    const int s = kv8_find_seq(cu_seqlens, n_seqs, t, n_tokens, 1, 1, 0);
    if (s < 0 || t >= cu_seqlens[s + 1]) return;
    const int cached = cached_lens[s];
    const int64_t pos = (int64_t)cached + (t - cu_seqlens[s]);
    if (cached < 0 || pos >= max_position) return;
    constexpr int PER = HALF / 8;                     // lanes to a head
    const int j = (lane % PER) * 8;
    const f32x8 c = Vec8<float>::load(rope_cos + pos * HALF + j), sn = Vec8<float>::load(rope_sin + pos * HALF + j);
    const bf16* src = qkv + (int64_t)t * qkv_stride + j;
    bf16* dst = q_out + (int64_t)t * q_stride + j;
#pragma unroll 4
    for (int h = lane / PER; h < n_q_heads; h += 64 / PER) {
      const f32x8 a = Vec8<bf16>::load(src + h * D), b = Vec8<bf16>::load(src + h * D + HALF);
      f32x8 ra, rb;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ra[e] = a[e] * c[e] - b[e] * sn[e];
        rb[e] = b[e] * c[e] + a[e] * sn[e];
      }
      Vec8<bf16>::store(dst + h * D, ra);
      Vec8<bf16>::store(dst + h * D + HALF, rb);
    }
    return;
  }
  // ---- keys or values of one (block, kv head) ----
  const int slot = task / (2 * n_kv_heads), rest = task - slot * (2 * n_kv_heads);
  const int kvh = rest >> 1;
  const int s = kv8_find_seq(cu_seqlens, n_seqs, slot, n_slots, 1, kKv8Block, 2);
  if (s < 0) return;
  const int64_t seq_lo = cu_seqlens[s];
  const int cached = cached_lens[s];
  if (cached < 0 || seq_lo < 0) return;
  // New tokens of the sequence: those that the launch has rows for, and that have a row of the tables.
  const int64_t n = min(min((int64_t)cu_seqlens[s + 1], n_tokens) - seq_lo, (int64_t)max_position - cached);
  if (n <= 0) return;
  const int64_t lb = (int64_t)cached / kKv8Block + (slot - kv8_slot(seq_lo, s, kKv8Block, 2));
  if (lb >= max_blocks || lb * kKv8Block >= cached + n) return;
  const int64_t blk = block_tables[(int64_t)s * max_blocks + lb];
  if (blk < 0 || blk >= num_blocks) return;
  const int lo = (int)max((int64_t)cached - lb * kKv8Block, (int64_t)0);             // slots [lo, hi) are new
  const int hi = (int)min(cached + n - lb * kKv8Block, (int64_t)kKv8Block);
  const int64_t row0 = seq_lo + lb * kKv8Block - cached;                             // row of slot 0
  const int64_t at = blk * n_kv_heads + kvh;
  float* const scale_at = (rest & 1 ? v_scale : k_scale) + at;
  const int e_old = lo > 0 ? min(max(exponent_of(*scale_at), kKv8MinExp), kKv8MaxExp) : kKv8MinExp;

  if ((rest & 1) == 0) {
    constexpr int E = D / 8;                          // channels of each half per lane
    constexpr int W = E / 4;                          // dwords of codes of each half
    const int tok = lane >> 2, c0 = (lane & 3) * E;
    const bool is_new = tok >= lo && tok < hi;
    float lower[E], upper[E];
    float amax = 0.f;
    if (is_new) {
      const bf16* src = qkv + (row0 + tok) * qkv_stride + (int64_t)(n_q_heads + kvh) * D + c0;
      const int64_t pos = lb * kKv8Block + tok;
#pragma unroll
      for (int g = 0; g < E; g += 8) {
        const f32x8 a = Vec8<bf16>::load(src + g), b = Vec8<bf16>::load(src + HALF + g);
        const f32x8 c = Vec8<float>::load(rope_cos + pos * HALF + c0 + g), sn = Vec8<float>::load(rope_sin + pos * HALF + c0 + g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lower[g + e] = round_to_odd((double)a[e] * c[e] - (double)b[e] * sn[e]);
          upper[g + e] = round_to_odd((double)b[e] * c[e] + (double)a[e] * sn[e]);
          amax = __builtin_fmaxf(amax, __builtin_fmaxf(finite_abs(lower[g + e]), finite_abs(upper[g + e])));
        }
      }
    }
    amax = wave_max(amax);
    const int e_new = max(scale_exponent(amax), e_old);
    const float inv = exp2_int(-e_new);
    if (lane == 0) *scale_at = exp2_int(e_new);
    uint32_t out[2][W];
    uint8_t* dst = k_pool + (at * kKv8Block + tok) * D + c0;
    if (is_new) {
#pragma unroll
      for (int w = 0; w < W; ++w) {
        out[0][w] = pack4(to_range(lower[4 * w], inv), to_range(lower[4 * w + 1], inv), to_range(lower[4 * w + 2], inv), to_range(lower[4 * w + 3], inv));
        out[1][w] = pack4(to_range(upper[4 * w], inv), to_range(upper[4 * w + 1], inv), to_range(upper[4 * w + 2], inv), to_range(upper[4 * w + 3], inv));
      }
    } else if (tok < lo) {
      if (e_new == e_old) return;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        out[0][w] = requantise4(load_as<uint32_t>(dst + 4 * w), e_old - e_new);
        out[1][w] = requantise4(load_as<uint32_t>(dst + HALF + 4 * w), e_old - e_new);
      }
    } else {
#pragma unroll
      for (int w = 0; w < W; ++w) out[0][w] = out[1][w] = 0;
    }
    using piece = uint32_t __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      piece v;
#pragma unroll
      for (int w = 0; w < W; ++w) v[w] = out[p][w];
      *reinterpret_cast<piece*>(dst + p * HALF) = v;
    }
    return;
  }

  constexpr int TOK = D == 128 ? 16 : 8;              // tokens per lane
  constexpr int W = TOK / 4;
  const int c0 = D == 128 ? lane * 2 : (lane & 31) * 2;
  const int t0 = D == 128 ? 0 : (lane >> 5) * 8;
  const bf16* src = qkv + (int64_t)(n_q_heads + n_kv_heads + kvh) * D + c0;
  bf16x2 v[TOK];
#pragma unroll
  for (int i = 0; i < TOK; ++i)                       // (slots that are not new: a row again that is)
    v[i] = load_as<bf16x2>(src + (row0 + min(max(t0 + i, lo), hi - 1)) * qkv_stride);
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < TOK; ++i) amax = __builtin_fmaxf(amax, __builtin_fmaxf(finite_abs((float)v[i][0]), finite_abs((float)v[i][1])));
  amax = wave_max(amax);
  const int e_new = max(scale_exponent(amax), e_old);
  const float inv = exp2_int(-e_new);
  if (lane == 0) *scale_at = exp2_int(e_new);
  using piece = uint32_t __attribute__((ext_vector_type(W)));
#pragma unroll
  for (int ch = 0; ch < 2; ++ch) {
    uint8_t* dst = v_pool + at * (kKv8Block * D) + (c0 + ch) * kKv8Block + t0;
    piece old{};
    if (lo > 0) old = load_as<piece>(dst);
    piece out;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint32_t fresh = pack4(to_range((float)v[4 * w][ch], inv), to_range((float)v[4 * w + 1][ch], inv),
                                   to_range((float)v[4 * w + 2][ch], inv), to_range((float)v[4 * w + 3][ch], inv));
      const uint32_t kept = e_new == e_old ? old[w] : requantise4(old[w], e_old - e_new);
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int tok = t0 + 4 * w + i;
        const uint32_t byte = 0xffu << (8 * i);
        word |= tok < lo ? kept & byte : tok < hi ? fresh & byte : 0u;
      }
      out[w] = word;
    }
    *reinterpret_cast<piece*>(dst) = out;
  }
}

void launch_kv8_append(const fp_kv8_cache& c, const fp_kv8_batch& b, const void* qkv, int64_t qkv_stride, int64_t n_tokens,
                       int n_q_heads, const float* rope_cos, const float* rope_sin, int max_position, void* q_out, int64_t q_stride,
                       hipStream_t s) {
  if (n_tokens == 0 || b.n_seqs == 0) return;
  const int64_t n_slots = kv8_slot(n_tokens, b.n_seqs, kKv8Block, 2);
  const dim3 grid((unsigned)((n_slots * 2 * c.n_kv_heads + n_tokens + 3) / 4));
  launch_kernel(c.head_dim == 128 ? kv8_append_kernel<128> : kv8_append_kernel<64>, grid, 256, 0, s, (const bf16*)qkv, qkv_stride,
                (bf16*)q_out, q_stride, n_tokens, n_q_heads, rope_cos, rope_sin, max_position, (uint8_t*)c.k_pool, (uint8_t*)c.v_pool,
                c.k_scale, c.v_scale, c.num_blocks, c.n_kv_heads, b.n_seqs, b.max_blocks, b.cu_seqlens, b.cached_lens, b.block_tables,
                (int)n_slots);
}

// ------------------------------------------------------------------------------------------
// Gather.  One wave per (block, kv head, keys or values).  Keys: 16 codes per lane become 32 bytes of a row.  Values: a lane takes four
// tokens of eight channels and turns them over in registers, so that a token's row leaves in 16-byte pieces; a wave's 4-byte reads
// of it cover whole lines between them.  Bound by HBM: 32768 positions of 8 heads of 128 move 201 MB in 45 us (4.5 TB/s), 777 take 3.9.
// ------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void kv8_gather_kernel(const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool,
                                                         const float* __restrict__ k_scale, const float* __restrict__ v_scale,
                                                         int64_t num_blocks, int n_kv_heads, const int32_t* __restrict__ table,
                                                         int64_t len, bf16* __restrict__ k_out, bf16* __restrict__ v_out) {
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t lb = task / n_kv_heads;
  const int kvh = (int)(task - lb * n_kv_heads);
  const int64_t p0 = lb * kKv8Block;
  if (p0 >= len) return;
  const int64_t blk = table[lb];
  const bool there = blk >= 0 && blk < num_blocks;
  const int64_t at = (there ? blk : 0) * n_kv_heads + kvh;
  const int64_t row = (int64_t)n_kv_heads * D;
  const int left = (int)min(len - p0, (int64_t)kKv8Block);
  if (blockIdx.y == 0) {
    const float scale = there ? k_scale[at] : 1.f;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const int piece = i * 64 + lane, tok = piece / (D / 16), ch = piece % (D / 16) * 16;
      u32x4 w = *reinterpret_cast<const u32x4*>(k_pool + at * (kKv8Block * D) + piece * 16);
      if (!there) w = u32x4{0, 0, 0, 0};
      if (tok < left) {
        bf16* dst = k_out + (p0 + tok) * row + kvh * D + ch;
        *reinterpret_cast<bf16x8*>(dst) = kv8_widen8(w[0], w[1], scale);
        *reinterpret_cast<bf16x8*>(dst + 8) = kv8_widen8(w[2], w[3], scale);
      }
    }
    return;
  }
  constexpr int GROUPS = D / 8;                       // groups of eight channels
  if (lane >= GROUPS * 4) return;
  const int ch = (lane % GROUPS) * 8, t0 = lane / GROUPS * 4;
  const float scale = there ? v_scale[at] : 1.f;
  bf16x4 v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(v_pool + at * (kKv8Block * D) + (ch + e) * kKv8Block + t0);
    v[e] = kv8_widen4(there ? w : 0, scale);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = v[e][t];
    if (t0 + t < left) *reinterpret_cast<bf16x8*>(v_out + (p0 + t0 + t) * row + kvh * D + ch) = o;
  }
}

void launch_kv8_gather(const fp_kv8_cache& c, const int32_t* table, int64_t len, void* k_out, void* v_out, hipStream_t s) {
  if (len == 0) return;
  const int64_t tasks = (len + kKv8Block - 1) / kKv8Block * c.n_kv_heads;
  const dim3 grid((unsigned)((tasks + 3) / 4), 2);
  launch_kernel(c.head_dim == 128 ? kv8_gather_kernel<128> : kv8_gather_kernel<64>, grid, 256, 0, s, (const uint8_t*)c.k_pool,
                (const uint8_t*)c.v_pool, c.k_scale, c.v_scale, c.num_blocks, c.n_kv_heads, table, len, (bf16*)k_out, (bf16*)v_out);
}

}  // namespace fp
