// Causal grouped-query attention over the 8-bit paged KV cache (operator `attn` of Section 5.1, Eq. (2) with the causal mask): a
// form for few query rows per sequence, bound by the bytes of the cache, and one for prompts and chunks, bound by the matrix cores.
//
// Both widen codes to bf16 times their block's scale, which is exact (four significant bits, a power of two), and take the queries as
// they are; the softmax factor multiplies the fp32 score.  Rounding to fewer bits happens once, to the probabilities: they enter
// the second product in bf16, and the sum they are divided by is taken over the rounded ones.
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "kv8.h"
#include "launch.h"

namespace fp {

namespace {

__device__ __forceinline__ float max3f(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// acc + a + b on a packed bf16 pair.
__device__ __forceinline__ float pair_sum(bf16 a, bf16 b, float acc) {
  const bf16x2 p = {a, b};
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
  return __builtin_amdgcn_fdot2_f32_bf16(p, one, acc, false);
}
__device__ __forceinline__ float other32_max(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other32_sum(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float other16_max(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other16_sum(float v) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Nonzero where one of the four codes is NaN (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// The codes with NaN replaced by zero, and bf16 ones where they were.
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
  const uint32_t n = nan_codes(w) >> 7;              // 0x01 in every NaN byte
  return w & ~(n * 0xffu);
}

// Workgroup barrier for what lies in LDS; the fence of __syncthreads would also wait for the loads of a later tile.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a workgroup of either form works on.
struct Kv8Rows {
  int s;             // sequence
  int64_t seq_lo;    // its first row
  int n_rows;        // rows of this slot: (token, head of the group), heads fastest
  int row0;          // first of them within the sequence
  int cached;
  int n_keys;        // positions that some row of the slot sees; 0: idle
  int steps;
};

template <int ROWS>
__device__ __forceinline__ bool kv8_rows(Kv8Rows& r, int64_t slot, int group, int64_t n_tokens, int n_seqs, int max_blocks,
                                         const int32_t* cu_seqlens, const int32_t* cached_lens) {
  r.s = kv8_find_seq(cu_seqlens, n_seqs, slot, group, ROWS, 1);
  if (r.s < 0) return false;
  r.seq_lo = cu_seqlens[r.s];
  if (r.seq_lo < 0) return false;
  const int64_t rows = (min((int64_t)cu_seqlens[r.s + 1], n_tokens) - r.seq_lo) * group;
  const int64_t row0 = (slot - kv8_slot(r.seq_lo * group, r.s, ROWS, 1)) * ROWS;
  if (row0 >= rows) return false;
  r.row0 = (int)row0;
  r.n_rows = (int)min(rows - row0, (int64_t)ROWS);
  r.cached = cached_lens[r.s];
  const int64_t last = (row0 + r.n_rows - 1) / group;
  r.n_keys = r.cached < 0 ? 0 : (int)min((int64_t)r.cached + last + 1, (int64_t)max_blocks * kKv8Block);
  r.steps = (r.n_keys + kKv8Step - 1) / kKv8Step;
  return true;
}

}  // namespace

// ------------------------------------------------------------------------------------------
// Few rows (one token, or a few drafted ones, of every sequence).  One workgroup = 4 waves = (16 R rows, kv head, part of the
// keys); a wave takes every fourth step of 64 keys = four blocks and reads each code once, straight into registers: no LDS, since
// nobody else wants it.  The matrix cores do both products on 16x16x32 tiles; with one token and four heads of a group four of
// their 16 columns are in use, and they are far from what bounds the kernel.
//
// S^T = K Q^T puts a query row into lane % 16 and four keys into the registers of each quarter of the wave.  Which key a row of K
// is may be chosen: row 4h + r of score tile j is token 4j + r of block h.  Then a quarter holds all 16 tokens of its own
// block, the probabilities of tokens 8u .. 8u+7 lie in the lane that the second product O^T += V^T P^T wants them in, and the matching
// operand is 8 of the 16 bytes that the cache keeps together for a channel: no exchange between lanes in either product.
// Along the channels any order does as long as K and Q agree: quarter q takes channels 16q .. 16q+15 of each 64, one
// 16-byte load.
//
// The exponent reference of a row moves when a score lies more than 2^8 above it (checked lane by lane, no reduction over the
// wave until then), so nearly all steps skip the rescaling.
// ------------------------------------------------------------------------------------------
constexpr int kFewWaves = 4;

template <int D, int R>
__global__ __launch_bounds__(kFewWaves * 64) void kv8_attn_few_kernel(
    const bf16* __restrict__ q, int64_t q_stride, bf16* __restrict__ o, int64_t o_stride, float* __restrict__ part_out, int parts,
    int part_steps, int64_t n_tokens, int n_q_heads, int n_kv_heads, float scale_log2, const uint8_t* __restrict__ k_pool,
    const uint8_t* __restrict__ v_pool, const float* __restrict__ k_scale, const float* __restrict__ v_scale, int64_t num_blocks,
    int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cached_lens,
    const int32_t* __restrict__ block_tables) {
  constexpr int ROWS = 16 * R, DC = D / 16, KH = D / 64, KK = D / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int group = n_q_heads / n_kv_heads;
  const int kvh = blockIdx.x % n_kv_heads;
  const int part = blockIdx.x / n_kv_heads % parts;
  const int64_t slot = blockIdx.x / n_kv_heads / parts;
  Kv8Rows rw;
  if (!kv8_rows<ROWS>(rw, slot, group, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens)) return;
  const int size = kv8_part_steps(rw.steps, part_steps, parts);
  const int begin = part * size, end = min(rw.steps, begin + size);
  if (part > 0 && begin >= end) return;                // (part 0 of an idle sequence writes the zeros)

  // ---- queries (B operand), zero behind the last row ----
  bf16x8 qf[R][KK];
  int q_pos[R];
#pragma unroll
  for (int g = 0; g < R; ++g) {
    const int r = g * 16 + col, row = rw.row0 + min(r, rw.n_rows - 1), tok = row / group;
    q_pos[g] = r < rw.n_rows ? rw.cached + tok : -1;
    const bf16* src = q + (rw.seq_lo + tok) * q_stride + (kvh * group + row % group) * D + quarter * 16;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[g][kk] = *reinterpret_cast<const bf16x8*>(src + (kk >> 1) * 64 + (kk & 1) * 8);
      if (r >= rw.n_rows) qf[g][kk] = bf16x8{};
    }
  }
  const int first_pos = rw.cached + rw.row0 / group;   // the position that the fewest keys are visible to

  f32x4 acc[R][DC];
  float m_ref[R], l_run[R];
#pragma unroll
  for (int g = 0; g < R; ++g) {
    m_ref[g] = -INFINITY;
    l_run[g] = 0.f;
#pragma unroll
    for (int i = 0; i < DC; ++i) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const int32_t* table = block_tables + (int64_t)rw.s * max_blocks;
  const int n_blocks = (rw.n_keys + kKv8Block - 1) / kKv8Block;
  auto block_of = [&](int lb) { return lb < n_blocks ? table[lb] : -1; };
  struct Step { u32x4 k[4][KH], v[DC]; float ks, vs; bool there; };
  // Codes and scales of one step; blocks that are not there are read from block 0 and masked.
  auto fetch = [&](Step& st, int k_id, int v_id) __attribute__((always_inline)) {
    st.there = v_id >= 0 && v_id < num_blocks;
    const int64_t kb = (k_id >= 0 && k_id < num_blocks ? (int64_t)k_id : 0) * n_kv_heads + kvh;
    const int64_t vb = (st.there ? (int64_t)v_id : 0) * n_kv_heads + kvh;
    const uint8_t* kp = k_pool + kb * (kKv8Block * D) + (col & 3) * D + quarter * 16;
    const uint8_t* vp = v_pool + vb * (kKv8Block * D) + col * kKv8Block;
    st.ks = k_scale[kb];
    st.vs = v_scale[vb];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < KH; ++h) st.k[j][h] = *reinterpret_cast<const u32x4*>(kp + j * 4 * D + h * 64);
#pragma unroll
    for (int i = 0; i < DC; ++i) st.v[i] = *reinterpret_cast<const u32x4*>(vp + i * 16 * kKv8Block);
  };

  Step st;
  int step = begin + wave;
  int k_id = 0, v_id = 0;
  if (step < end) {
    fetch(st, block_of(step * 4 + (col >> 2)), block_of(step * 4 + quarter));
    if (step + kFewWaves < end) {
      k_id = block_of((step + kFewWaves) * 4 + (col >> 2));
      v_id = block_of((step + kFewWaves) * 4 + quarter);
    }
  }
  for (; step < end; step += kFewWaves) {
    const int key0 = step * kKv8Step + quarter * kKv8Block;       // first key of this quarter's block
    const bool masked = __any(!st.there) || step * kKv8Step + kKv8Step - 1 > first_pos;

    f32x4 s[R][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int g = 0; g < R; ++g) s[g][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const u32x4 w = st.k[j][kk >> 1];
        const bf16x8 kf = kv8_widen8(w[2 * (kk & 1)], w[2 * (kk & 1) + 1], st.ks);
#pragma unroll
        for (int g = 0; g < R; ++g) s[g][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g][kk], s[g][j], 0, 0, 0);
      }
    }
    const bool there = st.there;
    const float vs = st.vs;
    u32x4 v[DC];
#pragma unroll
    for (int i = 0; i < DC; ++i) v[i] = st.v[i];
    if (step + kFewWaves < end) {
      fetch(st, k_id, v_id);
      if (step + 2 * kFewWaves < end) {
        k_id = block_of((step + 2 * kFewWaves) * 4 + (col >> 2));
        v_id = block_of((step + 2 * kFewWaves) * 4 + quarter);
      }
    }

    if (masked) {
#pragma unroll
      for (int g = 0; g < R; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[g][j][r] = there && key0 + 4 * j + r <= q_pos[g] ? s[g][j][r] : -INFINITY;
    }
    bf16x8 p[R][2];
#pragma unroll
    for (int g = 0; g < R; ++g) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = max3f(max3f(mx, s[g][j][0], s[g][j][1]), s[g][j][2], s[g][j][3]);
      mx *= scale_log2;
      if (__any(mx > m_ref[g] + 8.f)) {
        const float top = fmaxf(m_ref[g], other32_max(other16_max(mx)));
        const float alpha = m_ref[g] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref[g] - top);
        m_ref[g] = top;
        l_run[g] *= alpha;
#pragma unroll
        for (int i = 0; i < DC; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[g][i][r] *= alpha;
      }
      const float m = m_ref[g] == -INFINITY ? 0.f : m_ref[g];      // (a row that has seen nothing yet)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][2 * u + (i >> 2)][i & 3], scale_log2, -m));
        p[g][u] = __builtin_convertvector(e, bf16x8);
#pragma unroll
        for (int i = 0; i < 8; i += 2) l_run[g] = pair_sum(p[g][u][i], p[g][u][i + 1], l_run[g]);
      }
    }
    uint32_t nan = 0;
    if (masked) {
#pragma unroll
      for (int i = 0; i < DC; ++i) nan |= nan_codes(v[i][0]) | nan_codes(v[i][1]) | nan_codes(v[i][2]) | nan_codes(v[i][3]);
    }
    if (!__any(nan)) {
#pragma unroll
      for (int i = 0; i < DC; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 vf = kv8_widen8(v[i][2 * u], v[i][2 * u + 1], vs);
#pragma unroll
          for (int g = 0; g < R; ++g) acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[g][u], acc[g][i], 0, 0, 0);
        }
    } else {
      // A NaN value next to keys that some rows do not see: their zero weight would still make NaN of it.  The values go in
      // without the NaN, and a second product counts, for every (channel, row), the NaN that the row does see.
      bf16x8 sees[R][2];
#pragma unroll
      for (int g = 0; g < R; ++g)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 8; ++i) sees[g][u][i] = there && key0 + 8 * u + i <= q_pos[g] ? (bf16)1.0f : (bf16)0.0f;
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        f32x4 seen[R];
#pragma unroll
        for (int g = 0; g < R; ++g) seen[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t a = v[i][2 * u], b = v[i][2 * u + 1];
          const bf16x8 vf = kv8_widen8(without_nan(a), without_nan(b), vs);
          const bf16x8 is = kv8_widen8((nan_codes(a) >> 7) * 0x38u, (nan_codes(b) >> 7) * 0x38u, 1.f);   // 0x38 = 1.0
#pragma unroll
          for (int g = 0; g < R; ++g) {
            acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[g][u], acc[g][i], 0, 0, 0);
            seen[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, sees[g][u], seen[g], 0, 0, 0);
          }
        }
#pragma unroll
        for (int g = 0; g < R; ++g)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[g][i][r] = seen[g][r] > 0.f ? __builtin_nanf("") : acc[g][i][r];
      }
    }
  }

  // ---- the four waves' results joined through LDS, rows in order of the waves ----
  __shared__ __attribute__((aligned(16))) float s_acc[kFewWaves][ROWS][D];
  __shared__ float s_m[kFewWaves][ROWS], s_l[kFewWaves][ROWS];
#pragma unroll
  for (int g = 0; g < R; ++g) {
    const float l = other32_sum(other16_sum(l_run[g]));
    if (quarter == 0) { s_m[wave][g * 16 + col] = m_ref[g]; s_l[wave][g * 16 + col] = l; }
#pragma unroll
    for (int i = 0; i < DC; ++i) {
      const int piece = i * 4 + quarter;               // 16-byte piece of the row; swizzled over the banks by the row
      *reinterpret_cast<f32x4*>(&s_acc[wave][g * 16 + col][(piece ^ (col & 7)) * 4]) = acc[g][i];
    }
  }
  __syncthreads();
  const int64_t slab = ((slot * n_kv_heads + kvh) * parts + part) * (ROWS * (D + 2));
  for (int idx = threadIdx.x; idx < rw.n_rows * (D / 4); idx += kFewWaves * 64) {
    const int r = idx / (D / 4), piece = idx % (D / 4);
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) m = fmaxf(m, s_m[w][r]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = s_m[w][r] == -INFINITY ? (s_l[w][r] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(s_m[w][r] - m);
      l += f * s_l[w][r];
      const f32x4 a = *reinterpret_cast<const f32x4*>(&s_acc[w][r][(piece ^ (r & 7)) * 4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += f * a[e];
    }
    if (parts > 1) {
      *reinterpret_cast<f32x4*>(part_out + slab + r * D + piece * 4) = sum;
      if (piece == 0) {
        part_out[slab + ROWS * D + 2 * r] = m;
        part_out[slab + ROWS * D + 2 * r + 1] = l;
      }
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const int row = rw.row0 + r;
      bf16x4 out;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[e] = static_cast<bf16>(l == 0.f ? 0.f : sum[e] * inv);
      *reinterpret_cast<bf16x4*>(o + (rw.seq_lo + row / group) * o_stride + (kvh * group + row % group) * D + piece * 4) = out;
    }
  }
}

// ------------------------------------------------------------------------------------------
// Joins the parts of the keys: with reference m_i, sum l_i and unnormalised output O_i of part i and M = max m_i, the output is
// sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i, parts in index order.  A wave per (slot, kv head, row).
// ------------------------------------------------------------------------------------------
template <int D, int ROWS>
__global__ __launch_bounds__(256) void kv8_attn_merge_kernel(const float* __restrict__ part_in, bf16* __restrict__ o, int64_t o_stride,
                                                             int parts, int part_steps, int64_t n_tokens, int n_q_heads, int n_kv_heads,
                                                             int64_t n_slots, int n_seqs, int max_blocks,
                                                             const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cached_lens) {
  const int lane = threadIdx.x & 63;
  const int64_t task = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t slot = task / ((int64_t)n_kv_heads * ROWS);
  if (slot >= n_slots) return;
  const int rest = (int)(task - slot * ((int64_t)n_kv_heads * ROWS));
  const int kvh = rest / ROWS, r = rest % ROWS;
  const int group = n_q_heads / n_kv_heads;
  Kv8Rows rw;
  if (!kv8_rows<ROWS>(rw, slot, group, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens)) return;
  if (r >= rw.n_rows) return;
  const int size = kv8_part_steps(rw.steps, part_steps, parts);
  const int used = max(1, (rw.steps + size - 1) / size);
  const int64_t stride = ROWS * (D + 2);
  const float* base = part_in + (slot * n_kv_heads + kvh) * parts * stride;
  const float* ml = base + ROWS * D + 2 * r;
  constexpr int V = D / 64;
  float m = -INFINITY;
  for (int p = lane; p < used; p += 64) m = fmaxf(m, ml[p * stride]);
  m = wave_max(m);
  float l = 0.f, sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.f;
#pragma unroll 4
  for (int p = 0; p < used; ++p) {
    const float mp = ml[p * stride], lp = ml[p * stride + 1];
    const float f = mp == -INFINITY ? (lp == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(mp - m);
    l += f * lp;
    const float* src = base + p * stride + r * D + lane * V;
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] += f * src[e];
  }
  const float inv = 1.0f / l;
  const int row = rw.row0 + r;
  bf16* dst = o + (rw.seq_lo + row / group) * o_stride + (kvh * group + row % group) * D + lane * V;
#pragma unroll
  for (int e = 0; e < V; ++e) dst[e] = static_cast<bf16>(l == 0.f ? 0.f : sum[e] * inv);
}

// ------------------------------------------------------------------------------------------
// Many rows (prompts and chunks of them).  One workgroup = 8 waves = (256 rows, kv head, part of the keys); rows are (token, head of the
// group) pairs, so four heads share a tile's keys and a workgroup's rows span 64 tokens, which leaves little of a tile
// behind the diagonal and fills the tile with a chunk of a few dozen tokens.  Each wave owns 32 rows; 64 keys at a time.
//
// The products are those of the bf16 kernel (attention.hip): S^T = K Q^T on 32x32x16 tiles with key pi(i) in row i, pi = swap of
// bits 2 and 3, so that exp2 of the scores lies in the lanes as the operand of O^T += V^T P^T; LDS chunks swizzled alike.  What
// differs is how a tile comes in: every thread loads 16 codes of K and 16 of V (a channel's 16 tokens) into registers while the
// tile before is multiplied, widens them once for all eight waves, and stores bf16 into the other LDS stage.  Widening
// at the reads instead would halve the LDS bytes and repeat 128 conversions in every wave.
// Scores start from -m in the accumulator, in units of the unscaled product; the softmax factor is one multiplication ahead of
// exp2, which keeps the queries unrounded.
// ------------------------------------------------------------------------------------------
namespace {

template <int D> __device__ __forceinline__ int tile_key_of(int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); }
__device__ __forceinline__ int swap23(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }

}  // namespace

template <int D>
__global__ __launch_bounds__(512) void kv8_attn_tile_kernel(
    const bf16* __restrict__ q, int64_t q_stride, bf16* __restrict__ o, int64_t o_stride, float* __restrict__ part_out, int parts,
    int part_steps, int64_t n_slots, int64_t n_tokens, int n_q_heads, int n_kv_heads, float scale_log2,
    const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool, const float* __restrict__ k_scale,
    const float* __restrict__ v_scale, int64_t num_blocks, int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ block_tables) {
  constexpr int ROWS = kKv8TileRows;
  constexpr int CPR = D / 8;                 // 16-byte chunks of a bf16 row
  constexpr int DB = D / 32, KK = D / 16;
  constexpr int TILE = kKv8Step * D;
  constexpr int LOADS = D == 128 ? 2 : 1;    // D = 64: half of the threads bring K, half V
  __shared__ __attribute__((aligned(1024))) bf16 s_k[2][TILE];
  __shared__ __attribute__((aligned(1024))) bf16 s_v[2][TILE];
  __shared__ uint32_t s_nan[2][8];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, lh = lane >> 5;
  const int group = n_q_heads / n_kv_heads;
  const int kvh = blockIdx.x % n_kv_heads;
  const int part = blockIdx.x / n_kv_heads % parts;
  const int64_t slot = n_slots - 1 - blockIdx.x / n_kv_heads / parts;   // most keys first
  Kv8Rows rw;
  if (!kv8_rows<ROWS>(rw, slot, group, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens)) return;
  const int size = kv8_part_steps(rw.steps, part_steps, parts);
  const int begin = part * size, end = min(rw.steps, begin + size);
  if (part > 0 && begin >= end) return;

  const int32_t* table = block_tables + (int64_t)rw.s * max_blocks;
  const int n_blocks = (rw.n_keys + kKv8Block - 1) / kKv8Block;

  // ---- this thread's piece of a tile ----
  const int half_tid = tid & 255;
  const bool brings_v = D == 64 && wave >= 4;
  const int k_row = D == 128 ? tid >> 3 : half_tid >> 2;                // key of the tile
  const int k_c16 = D == 128 ? tid & 7 : half_tid & 3;                  // which 16 channels
  const int v_ch = D == 128 ? tid & 127 : half_tid & 63;
  const int my_block = D == 128 ? wave >> 1 : wave & 3;                 // block of the tile, K and V alike
  const int k_key = tile_key_of<D>(swap23(k_row & 31));
  const int v_flip = (v_ch >> 3) & 1;
  const uint32_t k_off = (uint32_t)((k_row & 15) * D + k_c16 * 16);
  const uint32_t v_off = (uint32_t)(v_ch * kKv8Block);
  u32x4 raw[LOADS];
  float raw_scale[LOADS];
  auto id_of = [&](int step) {               // wave-uniform
    const int lb = step * 4 + my_block;
    return __builtin_amdgcn_readfirstlane(step < end && lb < n_blocks ? table[lb] : -1);
  };
  auto fetch = [&](int id) __attribute__((always_inline)) {
    const int64_t at = (id >= 0 && id < num_blocks ? (int64_t)id : 0) * n_kv_heads + kvh;
    if (D == 128) {
      raw[0] = *reinterpret_cast<const u32x4*>(k_pool + at * (kKv8Block * D) + k_off);
      raw[LOADS - 1] = *reinterpret_cast<const u32x4*>(v_pool + at * (kKv8Block * D) + v_off);
      raw_scale[0] = k_scale[at];
      raw_scale[LOADS - 1] = v_scale[at];
    } else {
      raw[0] = *reinterpret_cast<const u32x4*>((brings_v ? v_pool + v_off : k_pool + k_off) + at * (kKv8Block * D));
      raw_scale[0] = (brings_v ? v_scale : k_scale)[at];
    }
  };
  auto put_k = [&](u32x4 w, float scale, int stage) __attribute__((always_inline)) {
    bf16* row = s_k[stage] + k_row * D;
    *reinterpret_cast<bf16x8*>(row + (((2 * k_c16) ^ k_key) << 3)) = kv8_widen8(w[0], w[1], scale);
    *reinterpret_cast<bf16x8*>(row + (((2 * k_c16 + 1) ^ k_key) << 3)) = kv8_widen8(w[2], w[3], scale);
  };
  auto put_v = [&](u32x4 w, float scale, int stage) __attribute__((always_inline)) {
    bf16* row = s_v[stage] + my_block * (D * kKv8Block) + v_ch * kKv8Block;
    *reinterpret_cast<bf16x8*>(row + v_flip * 8) = kv8_widen8(w[0], w[1], scale);
    *reinterpret_cast<bf16x8*>(row + (v_flip ^ 1) * 8) = kv8_widen8(w[2], w[3], scale);
  };
  // Widens the fetched piece into `stage`.  `careful`: the tile has keys that some row does not see; says whether V holds NaN.
  auto put = [&](int stage, bool careful) __attribute__((always_inline)) {
    const u32x4 wv = raw[LOADS - 1];
    if (D == 128) {
      put_k(raw[0], raw_scale[0], stage);
      put_v(wv, raw_scale[LOADS - 1], stage);
    } else if (brings_v) {
      put_v(wv, raw_scale[0], stage);
    } else {
      put_k(wv, raw_scale[0], stage);
    }
    if (careful) {
      const bool nan = (D == 128 || brings_v) && (nan_codes(wv[0]) | nan_codes(wv[1]) | nan_codes(wv[2]) | nan_codes(wv[3]));
      const uint64_t any = __ballot(nan);
      if (lane == 0) s_nan[stage][wave] = any != 0;
    }
  };
  // Which of the step's four blocks are there (wave-uniform).
  auto there_of = [&](int step) {
    uint32_t bits = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int lb = step * 4 + b;
      const int id = lb < n_blocks ? table[lb] : -1;
      bits |= (id >= 0 && id < num_blocks ? 1u : 0u) << b;
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane(bits);
  };
  const int first_pos = rw.cached + rw.row0 / group;
  auto straddles = [&](int step) { return step * kKv8Step + kKv8Step - 1 > first_pos; };

  // ---- queries ----
  const int wr0 = wave * 32;                  // first row of the wave within the slot
  const int r_mine = min(wr0 + lq, rw.n_rows - 1);
  const int row_mine = rw.row0 + r_mine;
  const int q_tok = row_mine / group;
  const int q_pos = rw.cached + q_tok;
  bf16x8 qf[KK];
  {
    const bf16* src = q + (rw.seq_lo + q_tok) * q_stride + (kvh * group + row_mine % group) * D + lh * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 16);
  }
  const bool wave_valid = wr0 < rw.n_rows;
  const int wave_first = rw.cached + (rw.row0 + min(wr0, rw.n_rows - 1)) / group;
  const int wave_last = rw.cached + (rw.row0 + min(wr0 + 31, rw.n_rows - 1)) / group;

  f32x16 oacc[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[i][r] = 0.f;
  float m_use = -INFINITY, l_run = 0.f, l_run2 = 0.f;
  f32x16 neg_m;
#pragma unroll
  for (int r = 0; r < 16; ++r) neg_m[r] = 0.f;
  const int pi_row = swap23(lq);
  const int k_swz = tile_key_of<D>(lq);
  const float gap = 8.0f / scale_log2;        // 2^8 of head-room, in score units

  auto multiply = [&](int step, int stage, uint32_t there) __attribute__((always_inline)) {
    const int key0 = step * kKv8Step;
    if (!wave_valid || key0 > wave_last) return;
    const bf16* ck = s_k[stage];
    const bf16* cv = s_v[stage];
    f32x16 sacc[2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      const bf16* krow = ck + (rb * 32 + pi_row) * D;
      bf16x8 kf[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[kk] = *reinterpret_cast<const bf16x8*>(krow + (((kk * 2 + lh) ^ k_swz) << 3));
      __builtin_amdgcn_sched_barrier(0);
      sacc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[0], qf[0], neg_m, 0, 0, 0);
#pragma unroll
      for (int kk = 1; kk < KK; ++kk) sacc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[kk], qf[kk], sacc[rb], 0, 0, 0);
    }
    // Register r of block rb: key 32 rb + 16 (r >> 3) + 8 lh + (r & 7), which is in the step's block 2 rb + (r >> 3).
    const bool masked = there != 15u || key0 + kKv8Step - 1 > wave_first;
    if (masked) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = key0 + rb * 32 + 16 * (r >> 3) + 8 * lh + (r & 7);
          sacc[rb][r] = key <= q_pos && (there >> (2 * rb + (r >> 3)) & 1) ? sacc[rb][r] : -INFINITY;
        }
    }
    float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      mx0 = max3f(mx0, sacc[0][r], sacc[0][r + 1]);
      mx1 = max3f(mx1, sacc[1][r], sacc[1][r + 1]);
    }
    const float mx = other32_max(fmaxf(mx0, mx1));
    // (a row without a reference yet has neg_m = 0: its scores are plain, and its first finite maximum becomes the reference)
    if (__any((m_use == -INFINITY && mx > -INFINITY) || mx > gap)) {
      const bool first = m_use == -INFINITY;
      const float shift = first ? (mx > -INFINITY ? mx : 0.f) : fmaxf(mx, 0.f);
      const float alpha = first ? 0.f : __builtin_amdgcn_exp2f(-shift * scale_log2);
      if (!first || mx > -INFINITY) m_use = (first ? 0.f : m_use) + shift;
      l_run *= alpha;
      l_run2 *= alpha;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[i][r] *= alpha;
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[rb][r] -= shift;
      const float nm = m_use == -INFINITY ? 0.f : -m_use;
#pragma unroll
      for (int r = 0; r < 16; ++r) neg_m[r] = nm;
    }
    bf16x8 pf[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      f32x8 pv;
#pragma unroll
      for (int e = 0; e < 8; ++e) pv[e] = __builtin_amdgcn_exp2f(sacc[c >> 1][8 * (c & 1) + e] * scale_log2);
      pf[c] = __builtin_convertvector(pv, bf16x8);
      l_run = pair_sum(pf[c][0], pf[c][1], l_run);
      l_run2 = pair_sum(pf[c][2], pf[c][3], l_run2);
      l_run = pair_sum(pf[c][4], pf[c][5], l_run);
      l_run2 = pair_sum(pf[c][6], pf[c][7], l_run2);
    }
    uint32_t nan = 0;
    if (masked) {
#pragma unroll
      for (int w = 0; w < 8; ++w) nan |= s_nan[stage][w];
      nan = __builtin_amdgcn_readfirstlane(nan);
    }
    if (nan == 0) {
#pragma unroll
      for (int i = 0; i < DB; ++i) {
        const int d = i * 32 + lq;
        const int phys = d * 2 + (lh ^ ((d >> 3) & 1));
        bf16x8 vf[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) vf[c] = *reinterpret_cast<const bf16x8*>(cv + c * (D * kKv8Block) + (phys << 3));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < 4; ++c) oacc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c], pf[c], oacc[i], 0, 0, 0);
      }
    } else {
      // As in the few-rows form: the values without NaN, and a count of the NaN that each row does see.
#pragma unroll 1
      for (int i = 0; i < DB; ++i) {
        const int d = i * 32 + lq;
        const int phys = d * 2 + (lh ^ ((d >> 3) & 1));
        f32x16 seen, add;
#pragma unroll
        for (int r = 0; r < 16; ++r) seen[r] = add[r] = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          bf16x8 vf = *reinterpret_cast<const bf16x8*>(cv + c * (D * kKv8Block) + (phys << 3)), is, sees;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool bad = vf[e] != vf[e];
            is[e] = bad ? (bf16)1.0f : (bf16)0.0f;
            vf[e] = bad ? (bf16)0.0f : vf[e];
            sees[e] = key0 + 16 * c + 8 * lh + e <= q_pos && (there >> c & 1) ? (bf16)1.0f : (bf16)0.0f;
          }
          add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[c], add, 0, 0, 0);
          seen = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is, sees, seen, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < DB; ++k)
          if (k == i) {
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[k][r] = seen[r] > 0.f ? __builtin_nanf("") : oacc[k][r] + add[r];
          }
      }
    }
  };

  // ---- tile t is multiplied from one stage while t + 1 waits in registers; it goes to the other stage behind the products ----
  int id = id_of(begin);
  uint32_t there = there_of(begin);
  if (begin < end) {
    fetch(id);
    put(0, straddles(begin) || there != 15u);
    id = id_of(begin + 1);
    if (begin + 1 < end) fetch(id);
    id = id_of(begin + 2);
  }
  lds_barrier();
  for (int t = begin; t < end; ++t) {
    const int stage = (t - begin) & 1;
    const uint32_t there_next = t + 1 < end ? there_of(t + 1) : 15u;
    multiply(t, stage, there);
    there = there_next;
    if (t + 1 < end) {
      put(stage ^ 1, straddles(t + 1) || there != 15u);
      if (t + 2 < end) {
        fetch(id);
        id = id_of(t + 3);
      }
    }
    lds_barrier();
  }

  if (parts > 1) {
    // One part of the keys, rows by channels as the merge reads them.
    const int64_t slab = ((slot * n_kv_heads + kvh) * parts + part) * (ROWS * (D + 2));
    const float l_tot = other32_sum(l_run + l_run2);
    if (wr0 + lq < rw.n_rows) {
      float* dst = part_out + slab + (wr0 + lq) * D;
#pragma unroll
      for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int a = 0; a < 4; ++a)
          *reinterpret_cast<f32x4*>(dst + i * 32 + 8 * a + 4 * lh) = f32x4{oacc[i][4 * a], oacc[i][4 * a + 1], oacc[i][4 * a + 2], oacc[i][4 * a + 3]};
      float* ml = part_out + slab + ROWS * D + (wr0 + lq) * 2;
      ml[lh] = lh ? l_tot : m_use == -INFINITY ? m_use : m_use * scale_log2;
    }
    return;
  }

  // ---- normalise, stage through LDS (all waves are past their last tile), store rows with 16-byte accesses ----
  bf16* stage = (wave < 4 ? s_k[0] : s_v[0]) + (wave & 3) * (32 * D);
  static_assert(4 * 32 * D <= 2 * TILE, "the waves' rows fit the stages");
  {
    const float l_tot = other32_sum(l_run + l_run2);
    const float inv = 1.0f / l_tot;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const int d = i * 32 + 8 * a + 4 * lh;
        bf16x4 v4;
#pragma unroll
        for (int b = 0; b < 4; ++b) v4[b] = static_cast<bf16>(l_tot == 0.f ? 0.f : oacc[i][4 * a + b] * inv);
        *reinterpret_cast<bf16x4*>(stage + lq * D + (((d >> 3) ^ (lq & 7)) << 3) + (d & 7)) = v4;
      }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32 * CPR / 64; ++i) {
    const int idx = lane + i * 64;
    const int r = idx / CPR, dch = idx % CPR;
    if (wr0 + r < rw.n_rows) {
      const int row = rw.row0 + wr0 + r;
      const u32x4 v = *reinterpret_cast<const u32x4*>(stage + r * D + ((dch ^ (r & 7)) << 3));
      *reinterpret_cast<u32x4*>(o + (rw.seq_lo + row / group) * o_stride + (kvh * group + row % group) * D + dch * 8) = v;
    }
  }
}

template <int D>
static void launch_kv8_attn(const fp_kv8_cache& c, const fp_kv8_batch& b, const bf16* q, int64_t q_stride, bf16* o, int64_t o_stride,
                            int64_t n_tokens, int n_q_heads, float scale_log2, const Kv8Plan& p, float* part, hipStream_t s) {
  const int hkv = c.n_kv_heads;
  const uint8_t *kp = (const uint8_t*)c.k_pool, *vp = (const uint8_t*)c.v_pool;
  const dim3 grid((unsigned)(p.slots * p.parts * hkv));
  if (p.rows < kKv8TileRows)
    launch_kernel(p.rows == 16 ? kv8_attn_few_kernel<D, 1> : kv8_attn_few_kernel<D, 2>, grid, kFewWaves * 64, 0, s, q, q_stride, o, o_stride,
                  part, p.parts, p.part_steps, n_tokens, n_q_heads, hkv, scale_log2, kp, vp, c.k_scale, c.v_scale, c.num_blocks,
                  b.n_seqs, b.max_blocks, b.cu_seqlens, b.cached_lens, b.block_tables);
  else
    launch_kernel(kv8_attn_tile_kernel<D>, grid, 512, 0, s, q, q_stride, o, o_stride, part, p.parts, p.part_steps, p.slots, n_tokens,
                  n_q_heads, hkv, scale_log2, kp, vp, c.k_scale, c.v_scale, c.num_blocks, b.n_seqs, b.max_blocks, b.cu_seqlens,
                  b.cached_lens, b.block_tables);
  if (p.parts > 1) {
    auto* merge = p.rows == 16 ? kv8_attn_merge_kernel<D, 16> : p.rows == 32 ? kv8_attn_merge_kernel<D, 32> : kv8_attn_merge_kernel<D, kKv8TileRows>;
    launch_kernel(merge, dim3((unsigned)((p.slots * hkv * p.rows + 3) / 4)), 256, 0, s, part, o, o_stride, p.parts, p.part_steps, n_tokens,
                  n_q_heads, hkv, p.slots, b.n_seqs, b.max_blocks, b.cu_seqlens, b.cached_lens);
  }
}

void launch_kv8_attention(const fp_kv8_cache& c, const fp_kv8_batch& b, const void* q, int64_t q_stride, void* o, int64_t o_stride,
                          int64_t n_tokens, int n_q_heads, float scale, int max_new, int max_len, void* workspace,
                          size_t workspace_bytes, hipStream_t s) {
  if (n_tokens == 0 || b.n_seqs == 0) return;
  const Kv8Plan p = kv8_plan(n_tokens, b.n_seqs, n_q_heads, c.n_kv_heads, c.head_dim, max_new, max_len, workspace ? workspace_bytes : 0);
  const float scale_log2 = scale * 1.4426950408889634f;
  if (c.head_dim == 128)
    launch_kv8_attn<128>(c, b, (const bf16*)q, q_stride, (bf16*)o, o_stride, n_tokens, n_q_heads, scale_log2, p, (float*)workspace, s);
  else
    launch_kv8_attn<64>(c, b, (const bf16*)q, q_stride, (bf16*)o, o_stride, n_tokens, n_q_heads, scale_log2, p, (float*)workspace, s);
}

}  // namespace fp
