// Latent attention in its expanded form: causal attention over keys and values that were projected from the latents for every head, the
// keys' rotated part apart and shared by the heads (Eq. (2) with the causal mask of Section 3.1), packed sequences.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "latent.h"
#include "launch.h"

namespace fp {

namespace {

constexpr int kRows = kExpandedRows, kKeys = kExpandedStep;

// References (in units of exp2) up to which fma(score, scale, -reference) may be the exponent: it is off by half a step of the reference,
// 2^-5 here, for all keys of a row alike.  Beyond, the scores are multiplied and rounded first, and the largest one's exponent is zero.
__device__ __forceinline__ bool far_reference(float m) {
  const float a = __builtin_fabsf(m);
  return a > 0x1p20f && a < INFINITY;
}

// XORs of the 16-byte chunks of a row of C, so that no read meets another on a bank.  LDS serves a 16-byte read in four turns of lanes 0-3,
// 12-15, 20-23, 24-27; 4-11, 16-19, 28-31; and the same of the upper half; an 8-byte read in two turns of 32 lanes.  A score fragment
// reads rows 16 h + 4 j + r for r, h = 0..3, one chunk in lanes 0-15 and its neighbour in lanes 16-31; a value fragment four neighbouring
// rows of two quarters, two neighbouring chunks of each.
template <int C> __device__ __forceinline__ int key_swizzle(int row) {
  const int h = (0 - (row >> 4)) & 3;
  return C == 16 ? (row & 3) << 2 | h : C == 8 ? (row & 2) << 1 | h : h;
}
template <int C> __device__ __forceinline__ int value_swizzle(int row) {
  return C == 16 ? ((row & 3) | ((row >> 4) & 1) << 2) << 1 : (((row >> 1) & 1) | ((row >> 4) & 1) << 1) << 1;
}

// What a tile of 256 rows of sequence s sees.
struct Tile {
  int64_t q_lo, kv_lo;
  int row0, n_rows, cached, n_keys, steps;
};
__device__ __forceinline__ bool tile_at(Tile& x, int s, int j, const int32_t* cu_seqlens, const int32_t* cu_kv, int64_t n_tokens, int64_t n_kv) {
  x.q_lo = cu_seqlens[s];
  x.kv_lo = cu_kv[s];
  const int64_t all = cu_seqlens[s + 1] - x.q_lo, rows = min((int64_t)cu_seqlens[s + 1], n_tokens) - x.q_lo;
  const int64_t len = cu_kv[s + 1] - x.kv_lo, have = x.kv_lo < 0 ? 0 : max(min((int64_t)cu_kv[s + 1], n_kv) - x.kv_lo, (int64_t)0);
  const int64_t row0 = (int64_t)j * kRows;
  if (x.q_lo < 0 || row0 >= rows) return false;
  x.row0 = (int)row0;
  x.n_rows = (int)min(rows - row0, (int64_t)kRows);
  x.cached = (int)max(min(len - all, n_kv), -(int64_t)(1 << 30));      // (from the last key on all of them are visible)
  x.n_keys = (int)max(min(have, (len - all) + row0 + x.n_rows), (int64_t)0);
  x.steps = (x.n_keys + kKeys - 1) / kKeys;
  return true;
}

// Tiles of a sequence that have c steps or more: its last ones, a row's keys never being fewer than those of the row before.
__device__ __forceinline__ int tiles_with(int c, int tiles, int rows, int cached, int have) {
  const int keys = (c - 1) * kKeys + 1;
  if (c <= 0) return tiles;
  if (min(have, cached + rows) < keys) return 0;
  return tiles - min(max(keys - cached - 1, 0) / kRows, tiles - 1);
}

// Batches whose tiles start longest first, so that none of the long ones is left to the end: of 2 to 8 sequences, with more workgroups than
// CUs (fewer all start at once).  us, in the batch's order | by steps: 32 heads, 227, 2002, 590, 64 and 1213 tokens behind 1600, 515, 0, 37 and 0
// 148 | 117, the same the other way round 118 | 114; 40 heads, 300, 1200, 40 and 900 behind 4000, 0, 900 and 100 128 | 99; 20 heads, 8 x 1024
// 102 | 92, 8 x 512 48 | 42, 2 x 2000 78 | 79.  Looking for a place costs 0.8 us, of 16 sequences 1.6: 12 x 200 22.3 | 23.8, 16 x 512 75.9 | 76.5, and
// ragged batches of 10 to 16 sequences gain and lose: 20 heads 116 | 107, 105 | 100, 125 | 124, 127 | 136, 62 | 65, 32 heads 77 | 78, 119 | 123, 40 heads
// 114 | 121, 128 heads 97 | 107.
constexpr int kOrdered = 8;

// Sequence and tile number of the tile that `rank` tiles with more steps, or as many, come before, or s < 0; at most kOrdered sequences,
// one to a lane.  The smallest number of steps that `rank` tiles or fewer reach is searched by 64 guesses at a time.
__device__ __forceinline__ void tile_by_steps(int rank, int64_t n_tokens, int64_t n_kv, int n_seqs, const int32_t* cu_seqlens,
                                              const int32_t* cu_kv, int& s, int& j) {
  const int lane = threadIdx.x & 63;
  int tiles = 0, rows = 0, cached = 0, have = 0;
  Tile first;
  if (lane < n_seqs && tile_at(first, lane, 0, cu_seqlens, cu_kv, n_tokens, n_kv)) {
    rows = (int)(min((int64_t)cu_seqlens[lane + 1], n_tokens) - first.q_lo);
    tiles = (rows + kRows - 1) / kRows;
    cached = first.cached;
    have = (int)(first.kv_lo < 0 ? 0 : max(min((int64_t)cu_kv[lane + 1], n_kv) - first.kv_lo, (int64_t)0));
  }
  const int most = tiles > 0 ? (max(min(have, cached + rows), 0) + kKeys - 1) / kKeys : 0;
  int lo = 0, hi = 1, all = 0;
#pragma unroll
  for (int i = 0; i < kOrdered; ++i) {                 // (lanes without a sequence have no tiles)
    all += __builtin_amdgcn_readlane(tiles, i);
    hi = max(hi, __builtin_amdgcn_readlane(most, i) + 1);
  }
  s = -1;
  if (rank >= all) return;
  while (hi - lo > 1) {                                // lo: more than `rank` tiles have as many; hi: no more than that
    const int width = (hi - lo + 63) / 64;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kOrdered; ++i)
      n += tiles_with(lo + lane * width, __builtin_amdgcn_readlane(tiles, i), __builtin_amdgcn_readlane(rows, i),
                      __builtin_amdgcn_readlane(cached, i), __builtin_amdgcn_readlane(have, i));
    const int k = __popcll(__ballot(n > rank));
    hi = min(hi, lo + k * width);
    lo += (k - 1) * width;
  }
  const int more = tiles_with(hi, tiles, rows, cached, have), equal = tiles_with(lo, tiles, rows, cached, have) - more;
#pragma unroll
  for (int i = 0; i < kOrdered; ++i) rank -= __builtin_amdgcn_readlane(more, i);
  // (the tiles with `lo` steps in the order of the sequences)
#pragma unroll
  for (int i = 0; i < kOrdered; ++i) {
    const int n = __builtin_amdgcn_readlane(equal, i);
    if (s < 0 && rank < n) {
      s = i;
      j = __builtin_amdgcn_readlane(tiles - more, i) - (n - rank);
    }
    rank -= n;
  }
}

}  // namespace

// ------------------------------------------------------------------------------------------
// One workgroup = 8 waves = 256 rows of one head, 32 to a wave, over all or a part of their keys, 64 at a time, out of three LDS stages
// that DMA fills two steps ahead.  S^T = K Q^T puts a row into lane % 16; row 4h + r of score tile j is key 16h + 4j + r, so a quarter
// of the wave holds 16 neighbouring keys and their probabilities already lie as the second product O^T += V^T P^T wants them.  Its
// other operand comes out of LDS by reads that turn 4 x 16 elements.
//
// A row's reference moves when a score lies more than 2^8 above it.  Probabilities are rounded to bf16 for the second product (the matrix
// cores' type), and the sum that divides is taken over the rounded ones.  Where a step hides keys from some of a wave's rows, a product
// with zeros says whether their values are finite; those that are not stay out of the second product, and come in at the end for the rows that
// see them.
//
// What bounds it: the chain of a step, in which no unit is full.  8192 tokens of 20 heads (128 + 64 and 128), 430 GFLOP, take 408 to 437 us from
// card to card (0.98 to 1.05 PFLOP/s; a large library product reaches 1.4), and the matrix cores are busy for 44 % of the clocks.  On a card where it
// took 418 it would take 363 without the keys' LDS reads, 356 without DMA, 294 without both and the values' reads, 393 without exp2, 234 with
// products alone.  No gain: the two waves of a SIMD in turns (scores of one beside the softmax of the other), priorities, deeper prefetch,
// score products in place.
// ------------------------------------------------------------------------------------------
template <int N, int P, int V>
__global__ __launch_bounds__(512, 2) void latent_expanded_kernel(
    const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cu_kv, int n_seqs, const bf16* __restrict__ q, int64_t q_stride,
    const bf16* __restrict__ kv, int64_t kv_stride, const bf16* __restrict__ k_rope, int64_t k_rope_stride, bf16* __restrict__ o,
    int64_t o_stride, float* __restrict__ part_out, int parts, int part_steps, int64_t n_tokens, int64_t n_kv, int n_heads, float scale_log2) {
  constexpr int KN = N / 32, KP = P / 32, VB = V / 16;
  constexpr int CN = N / 8, CP = P / 8, CV = V / 8;   // 16-byte chunks of a row
  constexpr int IN = N / 64, IV = V / 64;             // DMA instructions of a wave per tile (the rotated part: one)
  constexpr int LOADS = IN + IV + 1;
  __shared__ __attribute__((aligned(1024))) bf16 s_n[3][kKeys * N];
  __shared__ __attribute__((aligned(1024))) bf16 s_r[3][kKeys * P];
  __shared__ __attribute__((aligned(1024))) bf16 s_v[3][kKeys * V];

  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = blockIdx.x % n_heads;
  const int rest = blockIdx.x / n_heads;
  const int part = rest % parts;
  int s, j = 0;
  if (n_seqs > 1 && n_seqs <= kOrdered && gridDim.x > kLatentWorkgroups) tile_by_steps(rest / parts, n_tokens, n_kv, n_seqs, cu_seqlens, cu_kv, s, j);
  else latent_tile_from_end(rest / parts, 1, kRows, n_tokens, n_seqs, cu_seqlens, s, j);
  if (s < 0) return;
  s = __builtin_amdgcn_readfirstlane(s);
  j = __builtin_amdgcn_readfirstlane(j);
  Tile x;
  if (!tile_at(x, s, j, cu_seqlens, cu_kv, n_tokens, n_kv)) return;
  int begin = 0, end = x.steps;
  if (parts > 1) {
    const int each = kv8_part_steps(x.steps, part_steps, parts);
    begin = part * each;
    end = min(x.steps, begin + each);
    if (begin >= end && part > 0) return;             // (the first part stands for a tile without keys)
  }

  const int wr0 = wave * 32;
  uint32_t n_off[IN], v_off[IV], r_off;
#pragma unroll
  for (int i = 0; i < IN; ++i) {
    const int at = (wave * IN + i) * 64 + lane, row = at / CN, c = at % CN;
    n_off[i] = (uint32_t)(row * kv_stride * 2 + ((c ^ key_swizzle<CN>(row)) * 16));
  }
#pragma unroll
  for (int i = 0; i < IV; ++i) {
    const int at = (wave * IV + i) * 64 + lane, row = at / CV, c = at % CV;
    v_off[i] = (uint32_t)(row * kv_stride * 2 + N * 2 + ((c ^ value_swizzle<CV>(row)) * 16));
  }
  const int r_inst = wave % (P / 8);                  // (P = 32: waves 4-7 fetch what 0-3 do)
  {
    const int at = r_inst * 64 + lane, row = at / CP, c = at % CP;
    r_off = (uint32_t)(row * k_rope_stride * 2 + ((c ^ key_swizzle<CP>(row)) * 16));
  }
  const uint32_t to_n = latent_lds_address(s_n[0]) + wave * IN * 1024, to_r = latent_lds_address(s_r[0]) + r_inst * 1024,
                 to_v = latent_lds_address(s_v[0]) + wave * IV * 1024;
  const int kv_step = __builtin_amdgcn_readfirstlane((int)kv_stride * 2), r_step = __builtin_amdgcn_readfirstlane((int)k_rope_stride * 2);
  const bf16* const kv_head = kv + x.kv_lo * kv_stride + (int64_t)head * (N + V);
  const bf16* const r_head = k_rope + x.kv_lo * k_rope_stride;
  const int n_keys = __builtin_amdgcn_readfirstlane(x.n_keys);
  u32x4 kv_src, r_src;
  // Rows behind the last key arrive as zeros.
  auto aim = [&](int t) __attribute__((always_inline)) {
    const int rows = min(max(n_keys - t * kKeys, 0), kKeys);
    const int64_t first = rows > 0 ? t * kKeys : 0;
    kv_src = latent_source(kv_head + first * kv_stride, rows > 0 ? (rows - 1) * kv_step + (N + V) * 2 : 0);
    r_src = latent_source(r_head + first * k_rope_stride, rows > 0 ? (rows - 1) * r_step + P * 2 : 0);
  };
  auto fetch = [&](auto i, int stage) __attribute__((always_inline)) {
    if constexpr (i() < IN) latent_load_lds<i() * 1024>(kv_src, to_n + stage * (kKeys * N * 2), n_off[i()]);
    else if constexpr (i() < IN + IV) latent_load_lds<(i() - IN) * 1024>(kv_src, to_v + stage * (kKeys * V * 2), v_off[i() - IN]);
    else latent_load_lds<0>(r_src, to_r + stage * (kKeys * P * 2), r_off);
  };
  auto fetch_all = [&](int t, int stage) __attribute__((always_inline)) {
    aim(t);
    latent_each<LOADS>([&](auto i) __attribute__((always_inline)) { fetch(i, stage); });
  };

  // ---- queries (B operand) ----
  bf16x8 qf[2][KN + KP];
  int q_pos[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int r = wr0 + g * 16 + col;
    q_pos[g] = r < x.n_rows ? min(x.cached + x.row0 + r, x.n_keys - 1) : -1;
    const bf16* src = q + (x.q_lo + x.row0 + min(r, x.n_rows - 1)) * q_stride + (int64_t)head * (N + P) + quarter * 8;
#pragma unroll
    for (int kk = 0; kk < KN + KP; ++kk) qf[g][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 32);
  }
  const int wave_min = min(x.cached + x.row0 + wr0, x.n_keys - 1), wave_max = x.cached + x.row0 + wr0 + 31;   // positions of the wave's rows
  const bool busy = wr0 < x.n_rows;

  const int k_row = 16 * (col >> 2) + (col & 3);
  int kn_off[KN], kr_off[KP], vv_off[VB];
#pragma unroll
  for (int kk = 0; kk < KN; ++kk) kn_off[kk] = k_row * N + (((kk * 4 + quarter) ^ key_swizzle<CN>(k_row)) << 3);
#pragma unroll
  for (int kk = 0; kk < KP; ++kk) kr_off[kk] = k_row * P + (((kk * 4 + quarter) ^ key_swizzle<CP>(k_row)) << 3);
  const int v_row = 16 * quarter + (col >> 2);
#pragma unroll
  for (int i = 0; i < VB; ++i) vv_off[i] = v_row * V + (((i * 2 + ((col & 3) >> 1)) ^ value_swizzle<CV>(v_row)) << 3) + (col & 1) * 4;

  f32x4 acc[2][VB];
  float m_ref[2], l_run[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    m_ref[g] = -INFINITY;
    l_run[g] = 0.f;
#pragma unroll
    for (int i = 0; i < VB; ++i) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool far = false, dirty = false;
  // The accumulators stay in vector registers (held in those that matrix instructions alone address, they would leave half as many for everything
  // else and be copied there and back around the blocks that are rarely entered); no read of them moves up.
  auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < VB; ++i) asm volatile("" : "+v"(acc[g][i]));
  };

  // Multiplies tile t of stage `stage`; the DMA of tile t + 2 into stage `next` lies behind the sums' products (behind the scores',
  // 8192 tokens of 20 heads take 418 us instead of 404: the keys' reads leave LDS less room).  Fragments are asked for AHEAD of their
  // products, a read behind each pair.
  constexpr int KT = KN + KP, AHEAD = 4, AHEAD_V = 4, APART = 2 * VB / LOADS;
  static_assert(AHEAD_V == AHEAD && APART > 0, "the first values are read behind the last keys, and all DMA instructions have a place");
  auto multiply = [&](int t, int stage, int next) __attribute__((always_inline)) {
    const int key0 = t * kKeys;
    const bf16 *tn = s_n[stage], *tr = s_r[stage], *tv = s_v[stage];
    f32x4 sc[2][4];
    bf16x8 kf[4 * KT], vf[2 * VB];
    auto key = [&](int at) __attribute__((always_inline)) {
      const int jj = at / KT, kk = at % KT;
      kf[at] = *reinterpret_cast<const bf16x8*>(kk < KN ? tn + jj * 4 * N + kn_off[kk < KN ? kk : 0] : tr + jj * 4 * P + kr_off[kk < KN ? 0 : kk - KN]);
    };
    auto value = [&](int at) __attribute__((always_inline)) {
      const bf16* p = tv + (at & 1) * 8 * V + vv_off[at >> 1];
      vf[at] = latent_join(latent_turned(p), latent_turned(p + 4 * V));
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) key(i);
    aim(t + 2);
    __builtin_amdgcn_sched_barrier(0);
    latent_each<4 * KT>([&](auto at) __attribute__((always_inline)) {
      constexpr int jj = at() / KT, kk = at() % KT;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        if constexpr (kk == 0) sc[g][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
        sc[g][jj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[at()], qf[g][kk], sc[g][jj], 0, 0, 0);
      }
      if constexpr (at() + AHEAD < 4 * KT) key(at() + AHEAD);
      else value(at() + AHEAD - 4 * KT);
      __builtin_amdgcn_sched_barrier(0);
    });
    const bool masked = key0 + kKeys - 1 > wave_min;
    if (__builtin_expect(masked, 0)) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[g][jj][r] = key0 + 16 * quarter + 4 * jj + r <= q_pos[g] ? sc[g][jj][r] : -INFINITY;
    }
    float mx[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      mx[g] = -INFINITY;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) mx[g] = max3(max3(mx[g], sc[g][jj][0], sc[g][jj][1]), sc[g][jj][2], sc[g][jj][3]);
      mx[g] *= scale_log2;
    }
    if (__builtin_expect(__any(mx[0] > m_ref[0] + 8.f || mx[1] > m_ref[1] + 8.f) != 0, 0)) {
      latent_settle();
      pin();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float top = fmaxf(m_ref[g], xhalf_max(xquarter_max(mx[g])));
        // (equal ones may be infinite)
        const float alpha = top == m_ref[g] ? 1.f : m_ref[g] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref[g] - top);
        m_ref[g] = top;
        l_run[g] *= alpha;
#pragma unroll
        for (int i = 0; i < VB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[g][i][r] *= alpha;
        far |= __any(far_reference(top)) != 0;
      }
      pin();
    }
    if (__builtin_expect(far, 0)) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj)
#pragma unroll
          for (int r = 0; r < 4; ++r) sc[g][jj][r] = latent_product(sc[g][jj][r], scale_log2);
    }
    const float factor = far ? 1.f : scale_log2;
    bf16x8 p[2][2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float m = m_ref[g] == -INFINITY ? 0.f : m_ref[g];          // (a row that has seen nothing yet)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[g][2 * u + (i >> 2)][i & 3], factor, -m));
        p[g][u] = __builtin_convertvector(e, bf16x8);
#pragma unroll
        for (int i = 0; i < 8; i += 2) l_run[g] = pair_sum(p[g][u][i], p[g][u][i + 1], l_run[g]);
      }
    }
    if (__builtin_expect(masked, 0)) {
      const bf16x8 zero = {};
      f32x4 any = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int at = 0; at < 2 * VB; ++at) {
        if (at >= AHEAD_V) value(at);
        any = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[at], zero, any, 0, 0, 0);
      }
      if (__any(!(any[0] == 0.f && any[1] == 0.f && any[2] == 0.f && any[3] == 0.f))) {
        dirty = true;
#pragma unroll
        for (int at = 0; at < 2 * VB; ++at) {
          value(at);
          const bf16x8 v = latent_finite(vf[at]);
#pragma unroll
          for (int g = 0; g < 2; ++g) latent_add_product<true>(acc[g][at >> 1], v, p[g][at & 1]);
          __builtin_amdgcn_sched_barrier(0);
        }
        latent_each<LOADS>([&](auto i) __attribute__((always_inline)) { fetch(i, next); });
        return;
      }
#pragma unroll
      for (int at = 0; at < AHEAD_V; ++at) value(at);
    }
    __builtin_amdgcn_sched_barrier(0);
    latent_each<2 * VB>([&](auto at) __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 2; ++g) latent_add_product<(at() < 2)>(acc[g][at() >> 1], vf[at()], p[g][at() & 1]);
      if constexpr (at() + AHEAD_V < 2 * VB) value(at() + AHEAD_V);
      if constexpr (at() % APART == 0 && at() / APART < LOADS) fetch(std::integral_constant<int, at() / APART>{}, next);
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  // ---- tile t is multiplied while t + 1 and t + 2 are on their way ----
  if (begin < end) {
    fetch_all(begin, 0);
    fetch_all(begin + 1, 1);
    __builtin_amdgcn_s_waitcnt(latent_wait_loads(LOADS));
    latent_barrier();
    int stage = 0;
    pin();
#pragma unroll 1
    for (int t = begin; t < end; ++t) {
      const int next = stage == 0 ? 2 : stage - 1;    // (that of tile t + 2, which t - 1 has left)
      if (__builtin_expect(busy && t * kKeys <= wave_max, 1)) multiply(t, stage, next);
      else fetch_all(t + 2, next);
      __builtin_amdgcn_s_waitcnt(latent_wait_loads(LOADS));        // tile t + 1 is there
      latent_barrier();
      stage = stage == 2 ? 0 : stage + 1;
    }
    latent_settle();
    pin();
    __builtin_amdgcn_s_waitcnt(latent_wait_loads(0)); // (tiles that were asked for beyond the last step)
  }

  if (dirty) {
    // What the steps that hide keys left out: values that are not finite, times the weights of the rows that see them.  The scores once
    // more, a quarter of the channels to a lane.
#pragma unroll 1
    for (int at = max(begin, wave_min / kKeys) * kKeys; at < min(end * kKeys, n_keys); ++at) {
      const bf16* const k_row = kv_head + at * kv_stride;
      bf16x4 v[VB];
      bool all = true;
#pragma unroll
      for (int i = 0; i < VB; ++i) {
        v[i] = *reinterpret_cast<const bf16x4*>(k_row + N + i * 16 + quarter * 4);
#pragma unroll
        for (int b = 0; b < 4; ++b) all &= (float)v[i][b] - (float)v[i][b] == 0.f;
      }
      if (__all(all)) continue;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int r = wr0 + g * 16 + col;
        const bf16* const q_row = q + (x.q_lo + x.row0 + min(r, x.n_rows - 1)) * q_stride + (int64_t)head * (N + P);
        float dot = 0.f;
#pragma unroll 1
        for (int c = quarter; c < N + P; c += 4)
          dot += (float)q_row[c] * (float)(c < N ? k_row[c] : r_head[at * k_rope_stride + c - N]);
        const float w = __builtin_amdgcn_exp2f(latent_product(xhalf_sum(xquarter_sum(dot)), scale_log2) - m_ref[g]);
#pragma unroll
        for (int i = 0; i < VB; ++i)
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const bool lost = (float)v[i][b] - (float)v[i][b] != 0.f && at <= q_pos[g];
            acc[g][i][b] += lost ? w * (float)v[i][b] : 0.f;
          }
      }
    }
  }

#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int r = wr0 + g * 16 + col;
    const float l = xhalf_sum(xquarter_sum(l_run[g]));
    if (r >= x.n_rows) continue;
    if (parts > 1) {
      const int64_t slot = kv8_slot(x.q_lo, s, kRows, 1) + j;
      float* dst = part_out + ((slot * n_heads + head) * parts + part) * (int64_t)(kRows * (V + 2));
#pragma unroll
      for (int i = 0; i < VB; ++i) *reinterpret_cast<f32x4*>(dst + r * V + i * 16 + quarter * 4) = acc[g][i];
      if (quarter == 0) *reinterpret_cast<f32x2*>(dst + kRows * V + 2 * r) = f32x2{m_ref[g], l};
      continue;
    }
    const float inv = 1.0f / l;
    bf16* dst = o + (x.q_lo + x.row0 + r) * o_stride + (int64_t)head * V + quarter * 4;
#pragma unroll
    for (int i = 0; i < VB; ++i) {
      bf16x4 v;
#pragma unroll
      for (int b = 0; b < 4; ++b) v[b] = static_cast<bf16>(l == 0.f ? 0.f : acc[g][i][b] * inv);
      *reinterpret_cast<bf16x4*>(dst + i * 16) = v;
    }
  }
}

template <int V>
__global__ __launch_bounds__(256) void latent_expanded_merge_kernel(const float* __restrict__ part_in, bf16* __restrict__ o, int64_t o_stride,
                                                                    int parts, int part_steps, int64_t n_tokens, int64_t n_kv, int n_heads,
                                                                    int n_seqs, const int32_t* __restrict__ cu_seqlens,
                                                                    const int32_t* __restrict__ cu_kv) {
  constexpr int LANES = V / 4, PER = 256 / LANES;
  const int64_t row_all = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
  const int64_t t = row_all / n_heads;
  const int head = (int)(row_all - t * n_heads);
  const int64_t t0 = __builtin_amdgcn_readfirstlane((int)min(t, n_tokens - 1));
  int s = kv8_find_seq(cu_seqlens, n_seqs, t0, n_tokens, 1, 1, 0);
  if (s < 0 || t >= n_tokens) return;
  while (s + 1 < n_seqs && cu_seqlens[s + 1] <= t) ++s;
  const int64_t lo = cu_seqlens[s];
  if (lo < 0 || t >= cu_seqlens[s + 1]) return;
  Tile x;
  const int j = (int)((t - lo) / kRows);
  if (!tile_at(x, s, j, cu_seqlens, cu_kv, n_tokens, n_kv)) return;
  const int each = kv8_part_steps(x.steps, part_steps, parts);
  const int used = each > 0 ? max(1, (x.steps + each - 1) / each) : 1;
  const int64_t size = kRows * (V + 2);
  const int64_t slot = kv8_slot(lo, s, kRows, 1) + j;
  latent_join_row<V, 1>(part_in + (slot * n_heads + head) * parts * size, size, size, used, kRows, (int)((t - lo) % kRows),
                     o + t * o_stride + (int64_t)head * V);
}

namespace {

template <int N, int P, int V> void launch_for(const ExpandedArgs& a, const ExpandedPlan& p, float* part, hipStream_t s) {
  const float scale_log2 = a.scale * 1.4426950408889634f;
  launch_kernel(latent_expanded_kernel<N, P, V>, dim3((unsigned)(p.tiles * p.parts * a.n_heads)), 512, 0, s, a.cu_seqlens, a.cu_kv, a.n_seqs,
                (const bf16*)a.q, a.q_stride, (const bf16*)a.kv, a.kv_stride, (const bf16*)a.k_rope, a.k_rope_stride, (bf16*)a.o, a.o_stride, part,
                p.parts, p.part_steps, a.n_tokens, a.n_rows, a.n_heads, scale_log2);
  if (p.parts > 1) {
    constexpr int PER = 256 / (V / 4);
    launch_kernel(latent_expanded_merge_kernel<V>, dim3((unsigned)((a.n_tokens * a.n_heads + PER - 1) / PER)), 256, 0, s, part, (bf16*)a.o,
                  a.o_stride, p.parts, p.part_steps, a.n_tokens, a.n_rows, a.n_heads, a.n_seqs, a.cu_seqlens, a.cu_kv);
  }
}

}  // namespace

void launch_latent_expanded(const ExpandedArgs& a, int max_new, int max_len, void* workspace, size_t workspace_bytes, hipStream_t s) {
  if (a.n_tokens == 0 || a.n_seqs == 0) return;
  const ExpandedPlan p = expanded_plan(a.n_tokens, a.n_seqs, a.n_heads, a.v_dim, max_new, max_len, workspace ? workspace_bytes : 0);
  float* part = static_cast<float*>(workspace);
  auto rope = [&](auto n, auto v) {
    if (a.rope_dim == 64) launch_for<n(), 64, v()>(a, p, part, s);
    else launch_for<n(), 32, v()>(a, p, part, s);
  };
  using Wide = std::integral_constant<int, 128>;
  using Narrow = std::integral_constant<int, 64>;
  if (a.nope_dim == 128) a.v_dim == 128 ? rope(Wide{}, Wide{}) : rope(Wide{}, Narrow{});
  else a.v_dim == 128 ? rope(Narrow{}, Wide{}) : rope(Narrow{}, Narrow{});
}

}  // namespace fp
