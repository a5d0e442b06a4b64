// Device-side helpers of the 8-bit cache's kernels.
#pragma once
#include "common.h"
#include "kv8_plan.h"

namespace fp {

// The sequence that owns `slot` of the launch's `slots` (kv8_plan.h): the last one whose first slot is at or before it; `mult` rows of
// the launch per token.  `slot` is the same in all lanes.  The sequence that it would be if all were of one length -- as in a decode step -- is
// looked at by scalar loads, which do not queue behind the vector loads that other waves of the CU have on their way; if it is
// another, the wave looks at 64 sequences at a time.
__device__ __forceinline__ int kv8_find_seq(const int32_t* cu_seqlens, int n_seqs, int64_t slot, int64_t slots, int mult, int per, int extra) {
  const int guess = (int)min((int64_t)(((float)slot + 0.5f) * (float)n_seqs / (float)slots), (int64_t)n_seqs - 1);
  if (kv8_slot((int64_t)cu_seqlens[guess] * mult, guess, per, extra) <= slot &&
      slot < kv8_slot((int64_t)cu_seqlens[guess + 1] * mult, guess + 1, per, extra))
    return guess;
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int base = 0; base < n_seqs; base += 64) {
    const int s = base + lane;
    const bool before = s < n_seqs && kv8_slot((int64_t)cu_seqlens[s < n_seqs ? s : 0] * mult, s, per, extra) <= slot;
    count += __popcll(__ballot(before));
  }
  return __builtin_amdgcn_readfirstlane(count - 1);
}

// Four codes in a dword -> four bf16, times the power of two `scale` (exact).
__device__ __forceinline__ bf16x4 kv8_widen4(uint32_t codes, float scale) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
  return bf16x4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ bf16x8 kv8_widen8(uint32_t a, uint32_t b, float scale) {
  const bf16x4 x = kv8_widen4(a, scale), y = kv8_widen4(b, scale);
  return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

}  // namespace fp
