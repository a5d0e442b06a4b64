// Device-side helpers of the latent attention's kernels.
#pragma once
#include "common.h"
#include "kv8.h"
#include "latent_plan.h"

#include <type_traits>
#include <utility>

namespace fp {

// vmcnt(n), the other counters left alone.
constexpr int latent_wait_loads(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }

// f(0) .. f(N - 1), the numbers as constants.
template <typename F, int... I> __device__ __forceinline__ void latent_each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void latent_each(F&& f) { latent_each_of(f, std::make_integer_sequence<int, N>{}); }


// Workgroup barrier for what lies in LDS; the fence of __syncthreads would also wait for the loads of a later tile.
__device__ __forceinline__ void latent_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// a * b rounded, also where a sum follows that the compiler could fuse it with.
__device__ __forceinline__ float latent_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Weight of a partial result with reference m and sum l among those whose largest reference is `top`.  One that has seen no key, or
// only scores of NaN, has no reference.
__device__ __forceinline__ float latent_weight(float m, float l, float top) {
  return m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);
}

// Running sum over the lanes.
__device__ __forceinline__ int latent_scan(int v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int w = __shfl_up(v, off, 64);
    if ((int)(threadIdx.x & 63) >= off) v += w;
  }
  return v;
}

// Tiles of `per` rows, `mult` rows a token, without the gaps of kv8_slot: sequence and tile number of the tile that `rank` tiles follow
// (so that a prompt's last tile, the longest, comes first), or s < 0.
__device__ __forceinline__ void latent_tile_from_end(int rank, int mult, int per, int64_t n_tokens, int n_seqs, const int32_t* cu_seqlens,
                                                     int& s, int& j) {
  const int lane = threadIdx.x & 63;
  s = -1;
  for (int top = n_seqs; top > 0; top -= 64) {        // lane 0 has the last sequence
    const int mine = top - 1 - lane;
    int tiles = 0;
    if (mine >= 0) {
      const int64_t lo = cu_seqlens[mine], n = min((int64_t)cu_seqlens[mine + 1], n_tokens) - lo;
      tiles = lo >= 0 && n > 0 ? (int)((n * mult + per - 1) / per) : 0;
    }
    const int ends = latent_scan(tiles);
    const uint64_t past = __ballot(ends > rank);
    if (past) {
      const int first = (int)__builtin_ctzll(past);
      s = top - 1 - first;
      j = __builtin_amdgcn_readlane(ends, first) - 1 - rank;
      return;
    }
    rank -= __builtin_amdgcn_readlane(ends, 63);
  }
}

// One 8-byte piece a lane of 16-bit elements in LDS, turned within each 16 lanes: lane i of them gives the address of four neighbours of
// row i/4, from column 4 (i%4) on, and gets column i of the four rows.
__device__ __forceinline__ bf16x4 latent_turned(const bf16* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  return __builtin_bit_cast(bf16x4, v);
}
__device__ __forceinline__ bf16x8 latent_join(bf16x4 a, bf16x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// c += v w on 16x16x32 tiles.  In assembly, to accumulate in place: the compiler leaves the destination of this instruction free to differ
// from its accumulator input, and copies all of a kernel's accumulators back in every step.  What the compiler does not see it does not
// wait for, so: the next product may add to the same accumulator at once, as its destination and its accumulator input are just the registers that the
// one before wrote (the compiler places such products next to each other, too), and nothing else touches them before the last has
// settled; LDS results reach the operands through the waits that the compiler places for the block's inputs; operands that vector
// instructions have just written (FRESH) are two instructions old first; and vector instructions read accumulators behind latent_settle()
// only.
template <bool FRESH = false> __device__ __forceinline__ void latent_add_product(f32x4& c, bf16x8 v, bf16x8 w) {
  if (FRESH) asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(v), "v"(w));
  else asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(v), "v"(w));
}
__device__ __forceinline__ void latent_settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// What a load into LDS reads: `bytes` bytes at `base`, offsets beyond them give zeros.  The same in all lanes.
__device__ __forceinline__ u32x4 latent_source(const bf16* base, int bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32) & 0xffffu),
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)bytes), 0x00020000u};
}
__device__ __forceinline__ uint32_t latent_lds_address(const bf16* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const bf16*)p);
}
// 16 bytes a lane into LDS, lane i's to address lds + add + 16 i.  In assembly, since the compiler has every LDS read that it cannot tell
// apart from such a load's target wait for all loads on their way, and the turning reads are among those: a tile would be waited for
// as soon as it is asked for.  The kernels wait by themselves, and a load that the compiler counts is not mistaken: these come on top of
// what it counts and return in order.  (m0 is a register that the compiler sets in front of the instructions that take it and keeps nothing
// in, and takes in no list of what a block changes; the pause is what a vector instruction that has just written one of the source's scalar registers asks for.)
template <int ADD> __device__ __forceinline__ void latent_load_lds(u32x4 source, uint32_t lds, uint32_t offset) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(source), "n"(ADD)
               : "memory", "scc");
}

// The elements with infinities and NaN replaced by zero.
__device__ __forceinline__ bf16x8 latent_finite(bf16x8 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] &= ((w[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((w[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
  return __builtin_bit_cast(bf16x8, w);
}

// Joins partial results.  Part i of a row lies at base + (i ? second + (i - 1) * stride : 0), D unnormalised sums at r * D and {reference,
// sum} at rows * D + 2 r; with M the largest reference the output is sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.  Four columns a thread,
// D/4 threads to a row and SIDE such groups that take its parts side by side: what a row waits for is a chain of loads, and with many
// parts each link of it asks for all there is.  A thread's parts are added in order, the groups' sums in order of the groups.  SIDE > 1: a
// workgroup to a row.
template <int D, int SIDE>
__device__ __forceinline__ void latent_join_row(const float* base, int64_t second, int64_t stride, int used, int rows, int r, bf16* out) {
  constexpr int LANES = D / 4, WAVES = SIDE * LANES / 64;
  __shared__ __attribute__((aligned(16))) f32x4 s_sum[SIDE > 1 ? SIDE * LANES : 1];
  __shared__ float s_top[SIDE > 1 ? WAVES : 1], s_l[SIDE];
  const int lane = threadIdx.x % LANES, side = SIDE > 1 ? threadIdx.x / LANES : 0;
  auto of = [&](int i) { return base + (i > 0 ? second + (i - 1) * stride : 0); };
  const int ml = rows * D + 2 * r;
  float top = -INFINITY;
  if (SIDE > 1) {
    for (int i = threadIdx.x; i < used; i += SIDE * LANES) top = fmaxf(top, of(i)[ml]);
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_top[i]);
  } else {
    for (int i0 = 0; i0 < used; i0 += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, of(min(i0 + i, used - 1))[ml]);
    }
  }
  float l = 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = side; i0 < used; i0 += 8 * SIDE) {
    f32x4 v[8];
    f32x2 m[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* p = of(min(i0 + i * SIDE, used - 1));
      v[i] = *reinterpret_cast<const f32x4*>(p + r * D + lane * 4);
      m[i] = *reinterpret_cast<const f32x2*>(p + ml);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + i * SIDE >= used) break;
      const float w = latent_weight(m[i][0], m[i][1], top);
      l += w * m[i][1];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += w * v[i][e];
    }
  }
  if (SIDE > 1) {
    s_sum[threadIdx.x] = sum;
    if (lane == 0) s_l[side] = l;
    __syncthreads();
    if (side > 0) return;
#pragma unroll
    for (int i = 1; i < SIDE; ++i) {
      const f32x4 v = s_sum[i * LANES + lane];
      l += s_l[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
  }
  const float inv = 1.0f / l;
  bf16x4 o4;
#pragma unroll
  for (int e = 0; e < 4; ++e) o4[e] = static_cast<bf16>(l == 0.f ? 0.f : sum[e] * inv);
  *reinterpret_cast<bf16x4*>(out + lane * 4) = o4;
}

}  // namespace fp
