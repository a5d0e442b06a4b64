// A product per head, C[t, h, :] = W[h] A[t, h, :]: what takes the queries of latent attention to the latents, and its outputs back to the
// heads.  Plain strides, so a head's numbers may be part of a longer row on either side.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace fp {

namespace {

// A fragment's eight neighbours along k, zeros from k on.
__device__ __forceinline__ bf16x8 piece_of(const bf16* row, int at, int k) {
  const bf16x8 zero = {};
  return at < k ? *reinterpret_cast<const bf16x8*>(row + at) : zero;
}

}  // namespace

// ------------------------------------------------------------------------------------------
// One workgroup = 4 waves = WT x WN; a wave has TB blocks of 16 tokens and NB of 16 outputs of one head, with fragments straight from
// memory.  C^T = W A^T: a lane holds four neighbouring outputs of a token.
// ------------------------------------------------------------------------------------------
template <int WT, int TB, int NB>
__global__ __launch_bounds__(256) void gemm_heads_kernel(const bf16* __restrict__ a, int64_t a_stride, int64_t a_head_stride,
                                                         const bf16* __restrict__ w, int64_t w_head_stride, bf16* __restrict__ c,
                                                         int64_t c_stride, int64_t c_head_stride, int64_t m, int n_heads, int n, int k,
                                                         int n_tiles) {
  constexpr int WN = 4 / WT;
  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_tile = blockIdx.x % n_tiles;
  const int64_t rest = blockIdx.x / n_tiles;
  const int head = (int)(rest % n_heads);
  const int64_t t0 = (rest / n_heads) * (WT * TB * 16) + (wave / WN) * (TB * 16);
  const int n0 = (n_tile * WN + wave % WN) * (NB * 16);
  if (t0 >= m || n0 >= n) return;
  const bf16* a_row[TB];
  const bf16* w_row[NB];
#pragma unroll
  for (int i = 0; i < TB; ++i) a_row[i] = a + min(t0 + i * 16 + col, m - 1) * a_stride + head * a_head_stride;
#pragma unroll
  for (int i = 0; i < NB; ++i) w_row[i] = w + head * w_head_stride + (int64_t)min(n0 + i * 16 + col, n - 1) * k;
  f32x4 acc[NB][TB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < TB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kk = 0; kk < k; kk += 32) {
    const int at = kk + quarter * 8;
    bf16x8 af[TB], wf[NB];
#pragma unroll
    for (int j = 0; j < TB; ++j) af[j] = piece_of(a_row[j], at, k);
#pragma unroll
    for (int i = 0; i < NB; ++i) wf[i] = piece_of(w_row[i], at, k);
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[i], af[j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int64_t t = t0 + j * 16 + col;
    if (t >= m) continue;
    bf16* dst = c + t * c_stride + head * c_head_stride;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int at = n0 + i * 16 + quarter * 4;
      if (at < n) *reinterpret_cast<bf16x4*>(dst + at) = __builtin_convertvector(acc[i][j], bf16x4);
    }
  }
}

void launch_gemm_heads(const void* a, int64_t a_stride, int64_t a_head_stride, const void* w, int64_t w_head_stride, void* c, int64_t c_stride,
                       int64_t c_head_stride, int64_t m, int n_heads, int64_t n, int64_t k, hipStream_t s) {
  if (m == 0) return;
  auto go = [&](auto kernel, int tile_t, int tile_n) {
    const int n_tiles = (int)((n + tile_n - 1) / tile_n);
    const int64_t grid = (m + tile_t - 1) / tile_t * n_heads * n_tiles;
    launch_kernel(kernel, dim3((unsigned)grid), 256, 0, s, (const bf16*)a, a_stride, a_head_stride, (const bf16*)w, w_head_stride, (bf16*)c,
                  c_stride, c_head_stride, m, n_heads, (int)n, (int)k, n_tiles);
  };
  if (m <= 16) go(gemm_heads_kernel<1, 1, 2>, 16, 128);
  else if (m <= 256) go(gemm_heads_kernel<1, 4, 2>, 64, 128);
  else go(gemm_heads_kernel<2, 4, 4>, 128, 128);
}

}  // namespace fp
