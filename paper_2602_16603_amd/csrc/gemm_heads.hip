// A product per head, C[t, h, :] = W[h] A[t, h, :]: what takes the queries of latent attention to the latents, and its outputs back to the
// heads.  Plain strides, so a head's numbers may be part of a longer row on either side.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "latent_plan.h"
#include "launch.h"

namespace fp {

namespace {

// Both kernels: C^T = W A^T on 16x16x32 tiles, tokens in lane % 16.  Of a pair of output blocks, row 4 q + r of the first is output 8 q + r
// and of the second 8 q + 4 + r, so that a quarter of the wave holds eight neighbouring outputs of a token: 16 bytes a store.
__device__ __forceinline__ int output_of(int block, int row) { return (block >> 1) * 32 + (row >> 2) * 8 + (block & 1) * 4 + (row & 3); }

__device__ __forceinline__ bf16x8 both(f32x4 a, f32x4 b) {
  return __builtin_convertvector((f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}), bf16x8);
}

}  // namespace

// ------------------------------------------------------------------------------------------
// Few tokens, and every k.  One workgroup = 4 waves side by side over the outputs of one head; a wave has TB blocks of 16 tokens and 32
// outputs, fragments straight from memory, 128 k at a time and the next 128 on their way (ONCE: there are no more, and none are held).
// What bounds it: W's bytes, and with few of them two accesses to memory in a row; A is read by every wave of a head.  64 tokens of 128 heads of
// 512 x 128 move 27 MB in 9.8 us (2.8 TB/s; W alone is 17 MB).
// ------------------------------------------------------------------------------------------
template <int TB, bool ONCE>
__global__ __launch_bounds__(256) void gemm_heads_kernel(const bf16* __restrict__ a, int64_t a_stride, int64_t a_head_stride,
                                                         const bf16* __restrict__ w, int64_t w_head_stride, bf16* __restrict__ c,
                                                         int64_t c_stride, int64_t c_head_stride, int64_t m, int n_heads, int n, int k,
                                                         int n_tiles) {
  constexpr int KC = 4;                                // k-steps of a round
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_tile = blockIdx.x % n_tiles;
  const int64_t rest = blockIdx.x / n_tiles;
  const int head = (int)(rest % n_heads);
  const int64_t t0 = (rest / n_heads) * (TB * 16);
  const int n0 = (n_tile * 4 + wave) * 32;
  if (n0 >= n) return;
  const bf16* a_row[TB];
  const bf16* w_row[2];
#pragma unroll
  for (int i = 0; i < TB; ++i) a_row[i] = a + min(t0 + i * 16 + col, m - 1) * a_stride + head * a_head_stride + quarter * 8;
#pragma unroll
  for (int i = 0; i < 2; ++i) w_row[i] = w + head * w_head_stride + (int64_t)min(n0 + output_of(i, col), n - 1) * k + quarter * 8;
  f32x4 acc[2][TB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 af[ONCE ? 1 : 2][KC][TB], wf[ONCE ? 1 : 2][KC][2];
  // (k-steps beyond k are zeros on both sides)
  auto load = [&](int kk, bf16x8 (&x)[KC][TB], bf16x8 (&y)[KC][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < KC; ++s) {
      const int at = kk + s * 32;
      const bool in = at + quarter * 8 < k;
      const bf16x8 zero = {};
#pragma unroll
      for (int i = 0; i < 2; ++i) y[s][i] = in ? *reinterpret_cast<const bf16x8*>(w_row[i] + at) : zero;
#pragma unroll
      for (int j = 0; j < TB; ++j) x[s][j] = in ? *reinterpret_cast<const bf16x8*>(a_row[j] + at) : zero;
    }
  };
  auto multiply = [&](const bf16x8 (&x)[KC][TB], const bf16x8 (&y)[KC][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int s = 0; s < KC; ++s)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[s][i], x[s][j], acc[i][j], 0, 0, 0);
  };
  load(0, af[0], wf[0]);
  if constexpr (ONCE) {
    multiply(af[0], wf[0]);
  } else {
    for (int kk = 0; kk < k; kk += 2 * KC * 32) {
      load(kk + KC * 32, af[1], wf[1]);
      multiply(af[0], wf[0]);
      if (kk + KC * 32 >= k) break;
      load(kk + 2 * KC * 32, af[0], wf[0]);
      multiply(af[1], wf[1]);
    }
  }
  const int at = n0 + quarter * 8;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int64_t t = t0 + j * 16 + col;
    if (t < m && at < n) *reinterpret_cast<bf16x8*>(c + t * c_stride + head * c_head_stride + at) = both(acc[0][j], acc[1][j]);
  }
}

// ------------------------------------------------------------------------------------------
// Many tokens, k = 32 KS.  One workgroup = 8 waves = a head's outputs, as many as fit 128 KB of LDS, and a run of tokens; W's rows stay
// in LDS, and a wave holds all k of 16 tokens in registers while it goes through the outputs, and has the next 16 on their way.
// What bounds it: HBM.  4096 tokens of 32 heads of 128 x 512 move 172 MB in 42 us (4.1 TB/s; a copy of 1 GiB reaches 5.2), and in 35 where they
// come out of the caches.  32 tokens at a time and none ahead took 49, all straight from memory 75.
// ------------------------------------------------------------------------------------------
template <int KS>
__global__ __launch_bounds__(512, 2) void gemm_heads_many_kernel(const bf16* __restrict__ a, int64_t a_stride, int64_t a_head_stride,
                                                                 const bf16* __restrict__ w, int64_t w_head_stride, bf16* __restrict__ c,
                                                                 int64_t c_stride, int64_t c_head_stride, int64_t m, int n_heads, int n,
                                                                 int n_tiles, int64_t run) {
  constexpr int K = 32 * KS, CH = K / 8, NT = heads_outputs(K);
  __shared__ __attribute__((aligned(1024))) bf16 s_w[NT * K];
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_tile = blockIdx.x % n_tiles;
  const int64_t rest = blockIdx.x / n_tiles;
  const int head = (int)(rest % n_heads);
  const int64_t from = (rest / n_heads) * run, to = min(from + run, m);
  const int n0 = n_tile * NT, rows = min(n - n0, NT);
  // 16-byte chunks XORed with the row, so that a fragment's reads meet on no bank.
  auto swizzle = [](int row) { return CH == 8 ? (row >> 1) & 7 : row & 15; };
  const bf16* const a_head = a + head * a_head_stride + quarter * 8;
  bf16* const c_head = c + head * c_head_stride + n0 + quarter * 8;
  bf16x8 af[2][KS];
  auto load = [&](bf16x8 (&x)[KS], int64_t t0) __attribute__((always_inline)) {
    const bf16* src = a_head + min(t0 + col, m - 1) * a_stride;
#pragma unroll
    for (int s = 0; s < KS; ++s) x[s] = *reinterpret_cast<const bf16x8*>(src + s * 32);
  };
  auto multiply = [&](const bf16x8 (&x)[KS], int64_t t0) __attribute__((always_inline)) {
#pragma unroll 1
    for (int b0 = 0; b0 < rows; b0 += 32) {
      f32x4 acc[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = min(b0 + output_of(i, col), rows - 1);
          const bf16x8 wf = *reinterpret_cast<const bf16x8*>(s_w + row * K + (((s * 4 + quarter) ^ swizzle(row)) << 3));
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, x[s], acc[i], 0, 0, 0);
        }
      const int64_t t = t0 + col;
      if (t < to && b0 + quarter * 8 < rows) *reinterpret_cast<bf16x8*>(c_head + t * c_stride + b0) = both(acc[0], acc[1]);
    }
  };
  int64_t t0 = from + wave * 16;
  load(af[0], t0);                                     // (on its way while W is laid out)
#pragma unroll 4
  for (int at = threadIdx.x; at < rows * CH; at += 512) {
    const int row = at / CH, ch = at % CH;
    *reinterpret_cast<bf16x8*>(s_w + row * K + ((ch ^ swizzle(row)) << 3)) =
        *reinterpret_cast<const bf16x8*>(w + head * w_head_stride + (int64_t)(n0 + row) * K + ch * 8);
  }
  __syncthreads();
  while (t0 < to) {
    if (t0 + 128 < to) load(af[1], t0 + 128);
    multiply(af[0], t0);
    if (t0 + 128 >= to) break;
    if (t0 + 256 < to) load(af[0], t0 + 256);
    multiply(af[1], t0 + 128);
    t0 += 256;
  }
}

void launch_gemm_heads(const void* a, int64_t a_stride, int64_t a_head_stride, const void* w, int64_t w_head_stride, void* c, int64_t c_stride,
                       int64_t c_head_stride, int64_t m, int n_heads, int64_t n, int64_t k, hipStream_t s) {
  if (m == 0) return;
  // (32 tokens to a workgroup rather than 64 where that leaves the chip half empty)
  auto few = [&](auto kernel, int tile_t) {
    const int n_tiles = (int)((n + 127) / 128);
    launch_kernel(kernel, dim3((unsigned)((m + tile_t - 1) / tile_t * n_heads * n_tiles)), 256, 0, s, (const bf16*)a, a_stride, a_head_stride,
                  (const bf16*)w, w_head_stride, (bf16*)c, c_stride, c_head_stride, m, n_heads, (int)n, (int)k, n_tiles);
  };
  auto many = [&](auto kernel) {
    const int n_tiles = (int)((n + heads_outputs((int)k) - 1) / heads_outputs((int)k));
    const int64_t run = heads_run(m, n_heads, n_tiles);
    launch_kernel(kernel, dim3((unsigned)((m + run - 1) / run * n_heads * n_tiles)), 512, 0, s, (const bf16*)a, a_stride, a_head_stride,
                  (const bf16*)w, w_head_stride, (bf16*)c, c_stride, c_head_stride, m, n_heads, (int)n, n_tiles, run);
  };
  const bool wide = heads_in_lds(m, n_heads, k);
  if (wide && k == 64) many(gemm_heads_many_kernel<2>);
  else if (wide && k == 128) many(gemm_heads_many_kernel<4>);
  else if (wide && k == 256) many(gemm_heads_many_kernel<8>);
  else if (wide) many(gemm_heads_many_kernel<16>);
  else if (m <= 16) few(k <= 128 ? gemm_heads_kernel<1, true> : gemm_heads_kernel<1, false>, 16);
  else if (m <= 32 || (m + 63) / 64 * n_heads * ((n + 127) / 128) < 512) few(k <= 128 ? gemm_heads_kernel<2, true> : gemm_heads_kernel<2, false>, 32);
  else few(k <= 128 ? gemm_heads_kernel<4, true> : gemm_heads_kernel<4, false>, 64);
}

}  // namespace fp
