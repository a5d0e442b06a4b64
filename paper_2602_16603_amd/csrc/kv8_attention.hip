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

#include <type_traits>

namespace fp {

namespace {

// Scores (in units of exp2) up to which fma(score, scale, -reference) may be the exponent: it is off by half a step of the reference, 2^-5 here,
// for all keys of a row alike, since the reference is the rounded product.  Beyond, half a step becomes a number that overflows or that
// leaves a row nothing: the scores are multiplied and rounded first, and the largest one's exponent is exactly zero.
constexpr float kFarScore = 0x1p20f;
__device__ __forceinline__ bool far_score(float reference) {
  const float a = __builtin_fabsf(reference);
  return a > kFarScore && a < INFINITY;
}
// a * b rounded, also where a sum follows that the compiler could fuse it with.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// Nonzero where one of the four codes is NaN (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// The codes with NaN replaced by zero.
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

// The rows from `row0` of sequence s, at most `most` of them; false: none.
__device__ __forceinline__ bool kv8_rows_at(Kv8Rows& r, int s, int64_t row0, int most, int group, int64_t n_tokens, int max_blocks,
                                            const int32_t* cu_seqlens, const int32_t* cached_lens) {
  r.s = s;
  const int64_t rows = (min((int64_t)cu_seqlens[s + 1], n_tokens) - r.seq_lo) * group;
  if (row0 >= rows) return false;
  r.row0 = (int)row0;
  r.n_rows = (int)min(rows - row0, (int64_t)most);
  r.cached = min(cached_lens[s], max_blocks * kKv8Block);       // (from the table's end on all of it is visible; positions stay within 32 bits)
  const int64_t last = (row0 + r.n_rows - 1) / group;
  r.n_keys = r.cached < 0 ? 0 : (int)min((int64_t)r.cached + last + 1, (int64_t)max_blocks * kKv8Block);
  r.steps = (r.n_keys + kKv8Step - 1) / kKv8Step;
  return true;
}

// Weight of a partial result with reference m and sum l among those whose largest reference is `top`.  One that has seen no key, or
// only scores of NaN, has no reference.
__device__ __forceinline__ float part_weight(float m, float l, float top) {
  return m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(m - top);
}

// Slots of sequence s and the steps that are counted for each: those of its last row, and one for a sequence that sees
// nothing, whose rows are to be zero.
template <int ROWS>
__device__ __forceinline__ void few_steps(int s, int group, int64_t n_tokens, int max_blocks, const int32_t* cu_seqlens,
                                          const int32_t* cached_lens, int& slots, int& steps) {
  const int64_t lo = cu_seqlens[s], n = min((int64_t)cu_seqlens[s + 1], n_tokens) - lo, cached = cached_lens[s];
  slots = lo >= 0 && n > 0 ? (int)((n * group + ROWS - 1) / ROWS) : 0;
  const int64_t keys = cached < 0 ? 0 : min(cached + n, (int64_t)max_blocks * kKv8Block);
  steps = (int)max((keys + kKv8Step - 1) / kKv8Step, (int64_t)1);
}

// Running sum over the lanes.
__device__ __forceinline__ int wave_scan(int v) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int w = __shfl_up(v, off, 64);
    if ((int)(threadIdx.x & 63) >= off) v += w;
  }
  return v;
}

// Where the steps of sequence s (one per lane, 64 neighbours) end, counted from the first lane's.
template <int ROWS>
__device__ __forceinline__ int few_ends(int s, int group, int64_t n_tokens, int n_seqs, int max_blocks, const int32_t* cu_seqlens,
                                        const int32_t* cached_lens) {
  int slots = 0, steps = 0;
  if (s < n_seqs) few_steps<ROWS>(s, group, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
  return wave_scan(slots * steps);
}

// The tile form's slots without the gaps of kv8_slot, which would leave whole XCDs without work (slots in use are often every second
// one, and workgroups go to the XCDs in turn): sequence and slot number of the tile that `rank` tiles follow, or s < 0.
template <int ROWS>
__device__ __forceinline__ void tile_from_end(int rank, int group, int64_t n_tokens, int n_seqs, const int32_t* cu_seqlens, int& s, int& j) {
  const int lane = threadIdx.x & 63;
  s = -1;
  if (n_seqs == 1) {                                  // (scalar loads, no sums)
    const int64_t lo = cu_seqlens[0], n = min((int64_t)cu_seqlens[1], n_tokens) - lo;
    j = (int)((n * group + ROWS - 1) / ROWS) - 1 - rank;
    if (lo >= 0 && n > 0 && j >= 0) s = 0;
    return;
  }
  for (int top = n_seqs; top > 0; top -= 64) {        // lane 0 has the last sequence
    const int mine = top - 1 - lane;
    int tiles = 0;
    if (mine >= 0) {
      const int64_t lo = cu_seqlens[mine], n = min((int64_t)cu_seqlens[mine + 1], n_tokens) - lo;
      tiles = lo >= 0 && n > 0 ? (int)((n * group + ROWS - 1) / ROWS) : 0;
    }
    const int ends = wave_scan(tiles);
    const uint64_t past = __ballot(ends > rank);
    if (past) {
      const int first = (int)__builtin_ctzll(past);
      s = top - 1 - first;
      j = __builtin_amdgcn_readlane(ends, first) - 1 - rank;       // (the sequence's last tile first)
      return;
    }
    rank -= __builtin_amdgcn_readlane(ends, 63);
  }
}

}  // namespace

// ------------------------------------------------------------------------------------------
// Few rows (one token, or a few drafted ones, of every sequence).  One workgroup = 4 waves = a share of one kv head's work: the steps
// of 64 keys = four blocks of all slots of 16 R rows, one slot after the other, are dealt out in equal runs.  A wave takes every
// fourth step of a slot and reads each code once, straight into registers: no LDS, since nobody else wants it.  The matrix cores do
// both products on 16x16x32 tiles; with one token and four heads of a group four of their 16 columns are in use, and they are far from
// what bounds the kernel.
//
// S^T = K Q^T puts a query row into lane % 16 and four keys into the registers of each quarter of the wave.  Which key a row of K is
// may be chosen: row 4h + r of score tile j is token 4j + r of block h.  Then a quarter holds all 16 tokens of its own block, the
// probabilities of tokens 8u .. 8u+7 lie in the lane that the second product O^T += V^T P^T wants them in, and the matching operand is
// 8 of the 16 bytes that the cache keeps together for a channel: no exchange between lanes in either product. Along the channels any
// order does as long as K and Q agree: quarter q takes channels 16q .. 16q+15 of each 64, one 16-byte load.
//
// The exponent reference of a row moves when a score lies more than 2^8 above it (checked lane by lane, no reduction over the
// wave until then), so nearly all steps skip the rescaling.
//
// What bounds it: the codes' bytes.  64 tokens behind 512 .. 16384 positions of 8 heads of 128 read 702 MB in 130 us (5.4 TB/s; reads
// of 2 KB each, scattered like the blocks, reach 6.0 when nothing else is done).  With a part of the keys of one slot to a workgroup
// instead of equal shares the same call took 175: the longest sequences' parts ran on alone.  One token behind 32767 takes 16 (4.2
// TB/s): two steps to a wave do not hide their start.  16 sequences with 3 .. 5 drafted tokens, 8 heads to a group, 70 MB, take 29:
// four or five steps to a wave, and most sequences' codes are read for two slots, the second time out of the caches.  No gain:
// non-temporal loads, three or four waves to a SIMD (at fewer registers), steps of 32 keys, 64 rows to a slot.  With D = 128 and R =
// 2, eleven vector registers are spilled; all four kernels hold 33 to 40 scalars in lanes of a vector register.
// ------------------------------------------------------------------------------------------
constexpr int kFewWaves = 4;

template <int D, int R>
__global__ __launch_bounds__(kFewWaves * 64, 2) void kv8_attn_few_kernel(
    const bf16* __restrict__ q, int64_t q_stride, bf16* __restrict__ o, int64_t o_stride, i32x4* __restrict__ list_out,
    float* __restrict__ part_out, int shares, int n_slots, int64_t n_tokens, int n_q_heads, int n_kv_heads, float scale_log2,
    const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool, const float* __restrict__ k_scale,
    const float* __restrict__ v_scale, int64_t num_blocks, int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ block_tables) {
  constexpr int ROWS = 16 * R, DC = D / 16, KH = D / 64, KK = D / 32;
  __shared__ __attribute__((aligned(16))) bf16x8 s_q[R][KK][64];
  __shared__ __attribute__((aligned(16))) float s_acc[kFewWaves][16][D];
  __shared__ float s_m[kFewWaves][16], s_l[kFewWaves][16];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = n_q_heads / n_kv_heads;
  const int kvh = blockIdx.x % n_kv_heads;
  const int share = blockIdx.x / n_kv_heads;

  // ---- this workgroup's share of the steps: from step `begin` of slot j of sequence s on, as positions pos .. stop among all ----
  int s = 0, j = 0, begin = 0, slots = 0, steps = 0;
  int total = 1, n_shares = 1, pos = 0, stop = 1;
  if (shares == 0) {
    s = kv8_find_seq(cu_seqlens, n_seqs, share, n_slots, group, ROWS, 1);
    if (s < 0) return;
    few_steps<ROWS>(s, group, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
    j = (int)(share - kv8_slot((int64_t)cu_seqlens[s] * group, s, ROWS, 1));
    if (j >= slots) return;
    stop = steps;
  } else {
    int ends = 0;
    total = 0;
    for (int base = 0; base < n_seqs; base += 64) {
      ends = few_ends<ROWS>(base + (int)(threadIdx.x & 63), group, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens);
      total += __builtin_amdgcn_readlane(ends, 63);
    }
    n_shares = (int)kv8_shares(shares, total);
    if (share >= n_shares || total == 0) return;
    pos = (int)kv8_share(share, n_shares, total);
    stop = (int)kv8_share(share + 1, n_shares, total);
    int before = 0;
    for (int base = 0;; base += 64) {
      if (n_seqs > 64) ends = few_ends<ROWS>(base + (int)(threadIdx.x & 63), group, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens);
      const uint64_t past = __ballot(before + ends > pos);
      if (past) {
        const int first = (int)__builtin_ctzll(past);
        s = base + first;
        if (first > 0) before += __builtin_amdgcn_readlane(ends, first - 1);
        break;
      }
      before += __builtin_amdgcn_readlane(ends, 63);
    }
    few_steps<ROWS>(s, group, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
    j = (pos - before) / steps;
    begin = pos - before - j * steps;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  j = __builtin_amdgcn_readfirstlane(j);
  begin = __builtin_amdgcn_readfirstlane(begin);
  slots = __builtin_amdgcn_readfirstlane(slots);
  steps = __builtin_amdgcn_readfirstlane(steps);
  const int start = pos;

  while (pos < stop) {
    // (opaque: or all that follows from the lane, addresses above all, is kept in registers from one slot to the next)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int col = lane & 15, quarter = lane >> 4;
    const int run = min(stop - pos, steps - begin);
    Kv8Rows rw;
    rw.seq_lo = cu_seqlens[s];
    (void)kv8_rows_at(rw, s, (int64_t)j * ROWS, ROWS, group, n_tokens, max_blocks, cu_seqlens, cached_lens);
    const int end = min(rw.steps, begin + run);          // (a slot that is not the sequence's last may see fewer keys than its last row)
    const bool whole = run == steps;
    const int64_t slab = ((int64_t)share * 2 + (pos == start ? 0 : 1)) * n_kv_heads + kvh;
    if (shares > 0 && begin == 0 && threadIdx.x == 0) {
      const int64_t slot = kv8_slot(rw.seq_lo * group, s, ROWS, 1) + j;
      const int last = (int)kv8_share_of(pos + steps - 1, n_shares, total);
      list_out[slot * n_kv_heads + kvh] = i32x4{whole ? -1 : share, pos == start ? 0 : 1, last, 0};
    }

    // ---- queries (B operand): from LDS for every step, as the registers hold the codes on their way ----
    int q_pos[R];
    bf16x8 q_mine[R];
#pragma unroll
    for (int g = 0; g < R; ++g) {
      const int r = g * 16 + col, row = rw.row0 + min(r, rw.n_rows - 1), tok = row / group;
      q_pos[g] = r < rw.n_rows ? rw.cached + tok : -1;
      const int kk = wave % KK;                          // (a k-step per wave)
      q_mine[g] = *reinterpret_cast<const bf16x8*>(q + (rw.seq_lo + tok) * q_stride + (kvh * group + row % group) * D + quarter * 16 +
                                                   (kk >> 1) * 64 + (kk & 1) * 8);
    }
    static_assert(KK <= kFewWaves, "a wave brings one k-step of the queries");
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
    u32x4 kw[4][KH], vw[DC];
    float ks, vs;
    bool there;
    auto fetch_k = [&](int id) __attribute__((always_inline)) {
      const int64_t at = (int64_t)max(id, 0) * n_kv_heads + kvh;
      const uint8_t* p = k_pool + at * (kKv8Block * D) + (col & 3) * D + quarter * 16;
      ks = k_scale[at];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < KH; ++h) kw[j][h] = *reinterpret_cast<const u32x4*>(p + j * 4 * D + h * 64);
    };
    auto fetch_v = [&](int id) __attribute__((always_inline)) {
      there = id >= 0;
      const int64_t at = (int64_t)max(id, 0) * n_kv_heads + kvh;
      const uint8_t* p = v_pool + at * (kKv8Block * D) + col * kKv8Block;
      vs = v_scale[at];
#pragma unroll
      for (int i = 0; i < DC; ++i) vw[i] = *reinterpret_cast<const u32x4*>(p + i * 16 * kKv8Block);
    };

    // Block ids of a step, -1 for one that is not there: the same for the whole wave, by scalar loads.
    auto look = [&](int step) __attribute__((always_inline)) {
      i32x4 id;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int lb = step * 4 + b, i = table[min(lb, n_blocks - 1)];
        id[b] = lb < n_blocks && i < num_blocks ? max(i, -1) : -1;
      }
      return id;
    };
    auto none = [](i32x4 id) { return (id[0] & id[1] & id[2] & id[3]) < 0; };
    // The wave's first step from `step` on that has a block at all, 64 of its steps to a look.  Blocks that such a step lacks are read
    // from block 0 and masked.
    auto seek = [&](int step) __attribute__((always_inline)) {
      for (; step < end; step += 64 * kFewWaves) {
        const int mine = step + lane * kFewWaves;
        bool any = false;
        for (int b = 0; b < 4 && mine < end; ++b) {
          const int lb = mine * 4 + b, i = lb < n_blocks ? table[lb] : -1;
          any |= i >= 0 && i < num_blocks;
        }
        const uint64_t live = __ballot(any);
        if (live) return step + (int)__builtin_ctzll(live) * kFewWaves;
      }
      return end;
    };
    auto pick = [](i32x4 id, int b) { return b & 2 ? (b & 1 ? id[3] : id[2]) : (b & 1 ? id[1] : id[0]); };

    const i32x4 nothing = {-1, -1, -1, -1};
    int step = begin + wave;
    i32x4 id = step < end ? look(step) : nothing;
    if (step < end && none(id)) {
      step = seek(step);
      if (step < end) id = look(step);
    }
    if (step < end) {
      fetch_k(pick(id, col >> 2));
      fetch_v(pick(id, quarter));
    }
    int next = step + kFewWaves;
    id = next < end ? look(next) : nothing;
#pragma unroll
    for (int g = 0; g < R; ++g)
      if (wave < KK) s_q[g][wave][lane] = q_mine[g];
    lds_barrier();
    bool left_out = false;
    float factor = scale_log2, slack = 8.f;              // (with a reference beyond kFarScore: 1, and -infinity, for the block that multiplies)
    while (step < end) {
      if (next < end && none(id)) {
        next = seek(next);
        if (next < end) id = look(next);
      }
      const i32x4 later = next + kFewWaves < end ? look(next + kFewWaves) : nothing;   // (on its way while this step is multiplied)
      const int key0 = step * kKv8Step + quarter * kKv8Block;       // first key of this quarter's block
      const bool masked = __any(!there) || step * kKv8Step + kKv8Step - 1 > first_pos;

      f32x4 s[R][4];
#pragma unroll
      for (int g = 0; g < R; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[g][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        bf16x8 qf[R];
#pragma unroll
        for (int g = 0; g < R; ++g) qf[g] = s_q[g][kk][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 w = kw[j][kk >> 1];
          const bf16x8 kf = kv8_widen8(w[2 * (kk & 1)], w[2 * (kk & 1) + 1], ks);
#pragma unroll
          for (int g = 0; g < R; ++g) s[g][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[g], s[g][j], 0, 0, 0);
        }
      }
      if (next < end) fetch_k(pick(id, col >> 2));

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
        for (int j = 0; j < 4; ++j) mx = max3(max3(mx, s[g][j][0], s[g][j][1]), s[g][j][2], s[g][j][3]);
        mx *= scale_log2;
        if (__any(mx > m_ref[g] + slack)) {
          const float top = fmaxf(m_ref[g], xhalf_max(xquarter_max(mx)));
          const float alpha = m_ref[g] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref[g] - top);
          m_ref[g] = top;
          l_run[g] *= alpha;
#pragma unroll
          for (int i = 0; i < DC; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[g][i][r] *= alpha;
          if (__any(far_score(top))) factor = 1.f, slack = -INFINITY;
          if (slack < 0.f) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) s[g][j][r] = rounded_product(s[g][j][r], scale_log2);
          }
        }
        const float m = m_ref[g] == -INFINITY ? 0.f : m_ref[g];      // (a row that has seen nothing yet)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f32x8 e;
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][2 * u + (i >> 2)][i & 3], factor, -m));
          p[g][u] = __builtin_convertvector(e, bf16x8);
#pragma unroll
          for (int i = 0; i < 8; i += 2) l_run[g] = pair_sum(p[g][u][i], p[g][u][i + 1], l_run[g]);
        }
      }
      if (masked) {
        // A NaN value next to keys that some rows do not see: their weight of zero would still make NaN of them.  It stays out of the
        // product; rows that do see it get it at the end.  So would the scale of a block that nothing was ever appended to, which
        // stands in for one that is not there.
        vs = there ? vs : 1.f;
        uint32_t nan = 0;
#pragma unroll
        for (int i = 0; i < DC; ++i) nan |= nan_codes(vw[i][0]) | nan_codes(vw[i][1]) | nan_codes(vw[i][2]) | nan_codes(vw[i][3]);
        if (__any(nan)) {
          left_out = true;
#pragma unroll
          for (int i = 0; i < DC; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) vw[i][w] = without_nan(vw[i][w]);
        }
      }
#pragma unroll
      for (int i = 0; i < DC; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const bf16x8 vf = kv8_widen8(vw[i][2 * u], vw[i][2 * u + 1], vs);
#pragma unroll
          for (int g = 0; g < R; ++g) acc[g][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[g][u], acc[g][i], 0, 0, 0);
        }
      if (next < end) fetch_v(pick(id, quarter));
      step = next;
      next += kFewWaves;
      id = later;
    }

    if (left_out) {
      // For every (channel, row), how many of the NaN that were left out the row sees: a product of ones, straight from the cache.
      for (int step = begin; step < end; ++step) {
        const int lb = step * 4 + quarter;
        const int id = lb < n_blocks ? table[lb] : -1;
        const bool have = id >= 0 && id < num_blocks;
        if (!__any(!have) && step * kKv8Step + kKv8Step - 1 <= first_pos) continue;
        const uint8_t* p = v_pool + ((int64_t)(have ? id : 0) * n_kv_heads + kvh) * (kKv8Block * D) + col * kKv8Block;
#pragma unroll
        for (int i = 0; i < DC; ++i) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(p + i * 16 * kKv8Block);
#pragma unroll
          for (int g = 0; g < R; ++g) {
            f32x4 seen = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const bf16x8 is = kv8_widen8((nan_codes(w[2 * u]) >> 7) * 0x38u, (nan_codes(w[2 * u + 1]) >> 7) * 0x38u, 1.f);   // 0x38 = 1.0
              bf16x8 sees;
#pragma unroll
              for (int e = 0; e < 8; ++e) sees[e] = have && lb * kKv8Block + 8 * u + e <= q_pos[g] ? (bf16)1.0f : (bf16)0.0f;
              seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, sees, seen, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[g][i][r] = seen[r] > 0.f ? __builtin_nanf("") : acc[g][i][r];
          }
        }
      }
    }

    // ---- the four waves' results joined through LDS, 16 rows at a time, in order of the waves ----
#pragma unroll
    for (int g = 0; g < R; ++g) {
      if (g * 16 >= rw.n_rows) break;
      if (g > 0) lds_barrier();
      const float l_mine = xhalf_sum(xquarter_sum(l_run[g]));
      if (quarter == 0) { s_m[wave][col] = m_ref[g]; s_l[wave][col] = l_mine; }
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        const int piece = i * 4 + quarter;               // 16-byte piece of the row; swizzled over the banks by the row
        *reinterpret_cast<f32x4*>(&s_acc[wave][col][(piece ^ (col & 7)) * 4]) = acc[g][i];
      }
      lds_barrier();
      const int n = min(rw.n_rows - g * 16, 16);
      for (int idx = threadIdx.x; idx < n * (D / 4); idx += kFewWaves * 64) {
        const int r = idx / (D / 4), piece = idx % (D / 4);
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) m = fmaxf(m, s_m[w][r]);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
          const float f = part_weight(s_m[w][r], s_l[w][r], m);
          l += f * s_l[w][r];
          const f32x4 a = *reinterpret_cast<const f32x4*>(&s_acc[w][r][(piece ^ (r & 7)) * 4]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += f * a[e];
        }
        if (whole) {
          const float inv = 1.0f / l;
          const int row = rw.row0 + g * 16 + r;
          bf16x4 out;
#pragma unroll
          for (int e = 0; e < 4; ++e) out[e] = static_cast<bf16>(l == 0.f ? 0.f : sum[e] * inv);
          *reinterpret_cast<bf16x4*>(o + (rw.seq_lo + row / group) * o_stride + (kvh * group + row % group) * D + piece * 4) = out;
        } else {
          float* dst = part_out + slab * (ROWS * (D + 2));
          *reinterpret_cast<f32x4*>(dst + (g * 16 + r) * D + piece * 4) = sum;
          if (piece == 0) {
            dst[ROWS * D + 2 * (g * 16 + r)] = m;
            dst[ROWS * D + 2 * (g * 16 + r) + 1] = l;
          }
        }
      }
    }

    // ---- the next slot of the share ----
    pos += run;
    begin += run;
    if (begin == steps) {
      begin = 0;
      ++j;
    }
    while (pos < stop && j >= slots) {                   // (sequences without rows have no slots)
      if (++s >= n_seqs) return;
      j = 0;
      few_steps<ROWS>(s, group, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
    }
    if (pos < stop) lds_barrier();
  }
}

// ------------------------------------------------------------------------------------------
// Joins the partial results of a row: with reference m_i, sum l_i and unnormalised output O_i of the i-th and M = max m_i, the output
// is sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.  D/4 threads hold a row, SIDE such groups of them take its parts side by side: what a
// row waits for is a chain of loads, so with many parts (SIDE = 1024/D, a workgroup to a row) each link of it asks for all there is.
// A thread's parts are added in order, the groups' sums in order of the groups.  `list`: the few-rows form's shares (null: the parts
// of the tile form).  Latency bounds it with few rows: 4.6 us for one token's 64 shares a head, 5 to 6 for a batch; 512 tokens of 32
// heads in four parts, 34 MB of partial results out of the caches, 12.5.
// ------------------------------------------------------------------------------------------
template <int D, int SIDE>
__global__ __launch_bounds__(256) void kv8_attn_merge_kernel(const i32x4* __restrict__ list, const float* __restrict__ part_in,
                                                             bf16* __restrict__ o, int64_t o_stride, int rows, int parts, int part_steps,
                                                             int64_t n_tokens, int n_q_heads, int n_kv_heads, int n_seqs, int max_blocks,
                                                             const int32_t* __restrict__ cu_seqlens, const int32_t* __restrict__ cached_lens) {
  constexpr int LANES = D / 4, PER = 256 / (LANES * SIDE);          // rows of a workgroup
  static_assert(SIDE == 1 || PER == 1, "one row of many parts, or many rows of few");
  __shared__ __attribute__((aligned(16))) f32x4 s_sum[SIDE > 1 ? 256 : 1];
  __shared__ float s_top[4], s_l[SIDE];
  const int lane = threadIdx.x % LANES, side = SIDE > 1 ? threadIdx.x / LANES : 0;
  const int64_t row_all = (int64_t)blockIdx.x * PER + (PER > 1 ? threadIdx.x / LANES : 0);
  const int64_t t = row_all / n_q_heads;
  const int head = (int)(row_all - t * n_q_heads);
  const int group = n_q_heads / n_kv_heads, kvh = head / group;
  // (the rows of a wave are neighbours, of one token or two, so the wave looks for the sequence of its first and then steps on)
  const int64_t t0 = __builtin_amdgcn_readfirstlane((int)min(t, n_tokens - 1));
  int s = kv8_find_seq(cu_seqlens, n_seqs, t0, n_tokens, 1, 1, 0);
  if (s < 0 || t >= n_tokens) return;
  while (s + 1 < n_seqs && cu_seqlens[s + 1] <= t) ++s;
  const int64_t seq_lo = cu_seqlens[s];
  if (seq_lo < 0 || t >= cu_seqlens[s + 1]) return;
  const int64_t row = (t - seq_lo) * group + head % group;
  const int64_t slot = kv8_slot(seq_lo * group, s, rows, 1) + row / rows;
  const int r = (int)(row % rows);
  // Part i lies at base + (i ? second + (i - 1) * stride : 0).
  const int64_t size = (int64_t)rows * (D + 2);
  const float* base;
  int64_t second, stride;
  int used;
  if (list) {
    const i32x4 at = list[slot * n_kv_heads + kvh];
    if (at[0] < 0) return;                             // a slot that one workgroup finished
    used = at[2] - at[0] + 1;
    base = part_in + (((int64_t)at[0] * 2 + at[1]) * n_kv_heads + kvh) * size;
    stride = 2 * n_kv_heads * size;
    second = (2 - at[1]) * n_kv_heads * size;
  } else {
    Kv8Rows rw;
    rw.seq_lo = seq_lo;
    if (!kv8_rows_at(rw, s, row / rows * rows, rows, group, n_tokens, max_blocks, cu_seqlens, cached_lens)) return;
    const int each = kv8_part_steps(rw.steps, part_steps, parts);
    used = max(1, (rw.steps + each - 1) / each);
    base = part_in + (slot * n_kv_heads + kvh) * parts * size;
    second = stride = size;
  }
  auto of = [&](int i) { return base + (i > 0 ? second + (i - 1) * stride : 0); };
  const int ml = rows * D + 2 * r;
  float top = -INFINITY;
  if (SIDE > 1) {
    for (int i = threadIdx.x; i < used; i += 256) top = fmaxf(top, of(i)[ml]);
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
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
    float m[8], n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* p = of(min(i0 + i * SIDE, used - 1));
      v[i] = *reinterpret_cast<const f32x4*>(p + r * D + lane * 4);
      m[i] = p[ml];
      n[i] = p[ml + 1];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + i * SIDE >= used) break;
      const float w = part_weight(m[i], n[i], top);
      l += w * n[i];
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
  bf16x4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = static_cast<bf16>(l == 0.f ? 0.f : sum[e] * inv);
  *reinterpret_cast<bf16x4*>(o + t * o_stride + (int64_t)head * D + lane * 4) = out;
}

// ------------------------------------------------------------------------------------------
// Many rows (prompts and chunks of them).  One workgroup = 8 waves = (256 rows, kv head, part of the keys); rows are (token, head of
// the group) pairs, so four heads share a tile's keys and a workgroup's rows span 64 tokens, which leaves little of a tile behind the
// diagonal and fills the tile with a chunk of a few dozen tokens.  Each wave owns 32 rows; 64 keys at a time.
//
// The products are laid out as in the form for few rows: exp2 of the scores lies in the lanes as the operand of O^T += V^T P^T.
// Waves 0-3 load a tile's codes into registers (16 of K and 16 of V, a channel's 16 tokens, at a time) while the
// tile before is multiplied, widen them once for all eight waves, and store bf16 into the other LDS stage.  Widening
// at the reads instead would halve the LDS bytes and repeat 128 conversions in every wave.
//
// What bounds it: the chip's power with long prompts.  8192 tokens of 32/8 heads of 128 take 3600 clocks a tile, 2048 of them products, at the 1.9 GHz
// that it holds: 0.48 to 0.55 ms (1.15 to 1.0 PFLOP/s) by itself as the calls before it leave the clock, 0.61 behind a layer's
// projections, where the bf16 cache's kernel, which widens nothing, takes 0.48.  512 tokens behind 15872: 131 us
// and 144 behind others of its kind, the join included, where the bf16 cache's takes 118: four parts of 64 tiles fill the chip once, and
// widening and the start of a part are paid in full.
// Measured inside: a SIMD's two waves, w and w + 4, are not served alike, the older one is done with products and softmax in 2280
// clocks, the other in 3220; dealt to all, the widening's 640 clocks a wave held up the younger ones and the older ones waited 1110 at
// the barrier.  That gave 9 % fewer clocks and 2 % less time.  16x16x32 products draw less than 32x32x16 (16384 tokens 2.00 -> 1.94
// ms).  No gain: two or four tiles on their way instead of one, four LDS stages with a barrier every other tile, a raised priority for
// the products, all of K's fragments ahead of them.
// ------------------------------------------------------------------------------------------
namespace {

// Where 16-byte chunk c of a key's row (eight channels) lies in LDS: swizzled so that the 16 rows that are read together, tokens 4j ..
// 4j+3 of four blocks, fall on 16 slots of 256 bytes, and so do 16 threads that write, two keys' every second chunk.  (With the even
// chunks in front of the odd ones the writes of two keys shared eight slots: 29 % of LDS clocks were conflicts instead of 10; 8192 tokens
// 477 us instead of 475, 512 behind 15872 143.4 instead of 142.1.)
template <int D> __device__ __forceinline__ int k_place(int row, int c) {
  const int i = (row >> 4) << 2 | (row & 3);          // which of the 16
  return c ^ (D == 128 ? i : i >> 1);
}

}  // namespace

template <int D>
__global__ __launch_bounds__(512) void kv8_attn_tile_kernel(
    const bf16* __restrict__ q, int64_t q_stride, bf16* __restrict__ o, int64_t o_stride, float* __restrict__ part_out, int parts,
    int part_steps, int n_tiles, int64_t n_tokens, int n_q_heads, int n_kv_heads, float scale_log2,
    const uint8_t* __restrict__ k_pool, const uint8_t* __restrict__ v_pool, const float* __restrict__ k_scale,
    const float* __restrict__ v_scale, int64_t num_blocks, int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ block_tables) {
  constexpr int ROWS = kKv8TileRows;
  constexpr int CPR = D / 8;                 // 16-byte chunks of a bf16 row
  constexpr int DC = D / 16, KK = D / 32;
  constexpr int TILE = kKv8Step * D;
  constexpr int PIECES = D / 64;
  __shared__ __attribute__((aligned(1024))) bf16 s_k[2][TILE];
  __shared__ __attribute__((aligned(1024))) bf16 s_v[2][TILE];
  __shared__ uint32_t s_flags[2];            // {the part has holes, NaN was left out}

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int group = n_q_heads / n_kv_heads;
  const int kvh = blockIdx.x % n_kv_heads;
  const int part = blockIdx.x / n_kv_heads / n_tiles;
  int s, j;                                   // most keys first, where there is one sequence
  tile_from_end<ROWS>(blockIdx.x / n_kv_heads % n_tiles, group, n_tokens, n_seqs, cu_seqlens, s, j);
  if (s < 0) return;
  Kv8Rows rw;
  rw.seq_lo = cu_seqlens[s];
  if (!kv8_rows_at(rw, s, (int64_t)j * ROWS, ROWS, group, n_tokens, max_blocks, cu_seqlens, cached_lens)) return;
  const int64_t slot = kv8_slot(rw.seq_lo * group, s, ROWS, 1) + j;
  const int size = kv8_part_steps(rw.steps, part_steps, parts);
  const int begin = part * size, end = min(rw.steps, begin + size);
  if (part > 0 && begin >= end) return;

  const int32_t* table = block_tables + (int64_t)rw.s * max_blocks;
  const int n_blocks = (rw.n_keys + kKv8Block - 1) / kKv8Block;

  const int first_pos = rw.cached + rw.row0 / group;
  auto straddles = [&](int step) { return step * kKv8Step + kKv8Step - 1 > first_pos; };
  // Which of a step's four blocks are there (the same for all waves).  Looked at step by step only in a part that has holes: blocks
  // outside the pool, or rows whose positions go beyond the table.
  auto there_of = [&](int step) {
    uint32_t bits = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int lb = step * 4 + b;
      const int id = lb < n_blocks ? table[lb] : -1;
      bits |= ((uint32_t)id < (uint32_t)num_blocks ? 1u : 0u) << b;
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane(bits);
  };
  // ---- the pieces of a tile that a thread of waves 0-3 brings: 16 codes of K and 16 of V from PIECES blocks ----
  const bool loader = wave < 4;
  const int l_tid = tid & 255;
  const int k_row = D == 128 ? l_tid >> 3 : l_tid >> 2;                 // key of the tile (piece p: 32 p further)
  const int k_c16 = D == 128 ? l_tid & 7 : l_tid & 3;                   // which 16 channels
  const int v_ch = l_tid & (D - 1);
  const int l_block = D == 128 ? wave >> 1 : wave;                      // block of the tile, K and V alike (piece p: 2 p further)
  const uint32_t k_off = (uint32_t)((k_row & 15) * D + k_c16 * 16);
  const uint32_t v_off = (uint32_t)(v_ch * kKv8Block);
  bf16* k_put[PIECES][2];
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int h = 0; h < 2; ++h) k_put[p][h] = s_k[0] + (k_row + 32 * p) * D + (k_place<D>(k_row + 32 * p, 2 * k_c16 + h) << 3);
  bf16* const v_put = s_v[0] + l_block * (D * kKv8Block) + v_ch * 8;
  u32x4 raw_k[PIECES], raw_v[PIECES];
  float raw_ks[PIECES], raw_vs[PIECES];
  bool raw_there[PIECES];
  int lane_zero = 0;                         // (opaque: scales come by vector loads, as scalar ones would hold up the barrier)
  asm volatile("" : "+v"(lane_zero));
  struct Ids { uint32_t at[PIECES]; };
  auto ids_of = [&](int step) {              // wave-uniform
    Ids id;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) id.at[p] = (uint32_t)table[min(step * 4 + l_block + 2 * p, n_blocks - 1)];
    return id;
  };
  auto fetch = [&](Ids id) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {       // (of a block that is not there, block 0 is read, and masked)
      raw_there[p] = id.at[p] < (uint32_t)num_blocks;
      const uint32_t blk = raw_there[p] ? id.at[p] : 0u;
      const uint64_t at = (uint64_t)blk * (uint32_t)n_kv_heads + (uint32_t)kvh;
      raw_k[p] = *reinterpret_cast<const u32x4*>(k_pool + at * (kKv8Block * D) + k_off);
      raw_v[p] = *reinterpret_cast<const u32x4*>(v_pool + at * (kKv8Block * D) + v_off);
      raw_ks[p] = (k_scale + at)[lane_zero];
      raw_vs[p] = (v_scale + at)[lane_zero];
    }
  };
  // Widens the fetched pieces into `stage`.  `careful`: the tile has keys that some row does not see.  A NaN value among them would make
  // NaN of that row through its weight of zero; it stays out of the product, and the rows that do see it get it at the end.  So does the
  // scale of a block that nothing was ever appended to, which stands in for one that is not there.
  auto put = [&](int stage, bool careful) __attribute__((always_inline)) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = stage * TILE + p * (TILE / 2);
      *reinterpret_cast<bf16x8*>(k_put[p][0] + stage * TILE) = kv8_widen8(raw_k[p][0], raw_k[p][1], raw_ks[p]);
      *reinterpret_cast<bf16x8*>(k_put[p][1] + stage * TILE) = kv8_widen8(raw_k[p][2], raw_k[p][3], raw_ks[p]);
      u32x4 wv = raw_v[p];
      if (careful && !raw_there[p]) raw_vs[p] = 1.f;
      if (careful && __any(nan_codes(wv[0]) | nan_codes(wv[1]) | nan_codes(wv[2]) | nan_codes(wv[3]))) {
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[i] = without_nan(wv[i]);
        s_flags[1] = 1;
      }
      *reinterpret_cast<bf16x8*>(v_put + at) = kv8_widen8(wv[0], wv[1], raw_vs[p]);
      *reinterpret_cast<bf16x8*>(v_put + at + D * 8) = kv8_widen8(wv[2], wv[3], raw_vs[p]);
    }
  };

  if (tid < 2) s_flags[tid] = 0;
  if (loader && begin < end) fetch(ids_of(begin));    // (on its way while the table is looked through)
  lds_barrier();
  {
    bool hole = (int64_t)rw.cached + (rw.row0 + rw.n_rows - 1) / group >= rw.n_keys;
    for (int lb = begin * 4 + tid; lb < min(end * 4, n_blocks); lb += 512) hole |= (uint32_t)table[lb] >= (uint32_t)num_blocks;
    if (__any(hole) && lane == 0) s_flags[0] = 1;
  }

  // ---- queries ----
  const int wr0 = wave * 32;                  // first row of the wave within the slot
  int q_pos[2];
  bf16x8 qf[2][KK];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = rw.row0 + min(wr0 + g * 16 + col, rw.n_rows - 1), tok = row / group;
    q_pos[g] = rw.cached + tok;
    const bf16* src = q + (rw.seq_lo + tok) * q_stride + (kvh * group + row % group) * D + quarter * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[g][kk] = *reinterpret_cast<const bf16x8*>(src + kk * 32);
  }
  const bool wave_valid = wr0 < rw.n_rows;
  const int wave_first = rw.cached + (rw.row0 + min(wr0, rw.n_rows - 1)) / group;
  const int wave_last = rw.cached + (rw.row0 + min(wr0 + 31, rw.n_rows - 1)) / group;

  f32x4 oacc[2][DC];
  float m_ref[2], l_run[2];                   // (m_ref in units of exp2)
  float factor = scale_log2, slack = 8.f;     // (with a reference beyond kFarScore: 1, and -infinity, for the block that multiplies)
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    m_ref[g] = -INFINITY;
    l_run[g] = 0.f;
#pragma unroll
    for (int i = 0; i < DC; ++i) oacc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int k_row0 = (col >> 2) * kKv8Block + (col & 3);      // key of row `col` of score tile 0; 4 further in each

  auto multiply = [&](int step, int stage, uint32_t there) __attribute__((always_inline)) {
    const int key0 = step * kKv8Step;
    if (!wave_valid || key0 > wave_last) return;
    const bf16* ck = s_k[stage] + k_row0 * D;
    const bf16* cv = s_v[stage] + quarter * (D * kKv8Block) + col * 8;
    f32x4 s[2][4];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[g][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k2 = 0; k2 < KK; k2 += 2) {
      bf16x8 kf[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) kf[k][j] = *reinterpret_cast<const bf16x8*>(ck + j * 4 * D + (k_place<D>(k_row0, (k2 + k) * 4 + quarter) << 3));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int g = 0; g < 2; ++g) s[g][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[k][j], qf[g][k2 + k], s[g][j], 0, 0, 0);
    }
    // Register r of score tile j: token 4j + r of this quarter's block.
    if (there != 15u || key0 + kKv8Step - 1 > wave_first) {
      const bool have = there >> quarter & 1;
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[g][j][r] = have && key0 + quarter * kKv8Block + 4 * j + r <= q_pos[g] ? s[g][j][r] : -INFINITY;
    }
    bf16x8 p[2][2];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = max3(max3(mx, s[g][j][0], s[g][j][1]), s[g][j][2], s[g][j][3]);
      mx *= scale_log2;
      if (__any(mx > m_ref[g] + slack)) {
        const float top = fmaxf(m_ref[g], xhalf_max(xquarter_max(mx)));
        const float alpha = m_ref[g] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref[g] - top);
        m_ref[g] = top;
        l_run[g] *= alpha;
#pragma unroll
        for (int i = 0; i < DC; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[g][i][r] *= alpha;
        if (__any(far_score(top))) factor = 1.f, slack = -INFINITY;
        if (slack < 0.f) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[g][j][r] = rounded_product(s[g][j][r], scale_log2);
        }
      }
      const float m = m_ref[g] == -INFINITY ? 0.f : m_ref[g];          // (a row that has seen nothing yet)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 e;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][2 * u + (i >> 2)][i & 3], factor, -m));
        p[g][u] = __builtin_convertvector(e, bf16x8);
#pragma unroll
        for (int i = 0; i < 8; i += 2) l_run[g] = pair_sum(p[g][u][i], p[g][u][i + 1], l_run[g]);
      }
    }
#pragma unroll
    for (int i2 = 0; i2 < DC; i2 += 2) {
      bf16x8 vf[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) vf[i][u] = *reinterpret_cast<const bf16x8*>(cv + u * (D * 8) + (i2 + i) * 16 * 8);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int g = 0; g < 2; ++g) oacc[g][i2 + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i][u], p[g][u], oacc[g][i2 + i], 0, 0, 0);
    }
  };

  // ---- tile t is multiplied from one stage while t + 1 waits in registers; it goes to the other stage behind the products ----
  lds_barrier();
  const bool holes = __builtin_amdgcn_readfirstlane(s_flags[0]);
  if (loader && begin < end) {
    put(0, holes || straddles(begin));
    if (begin + 1 < end) fetch(ids_of(begin + 1));
  }
  lds_barrier();
  auto tile_step = [&](int t, auto stage) __attribute__((always_inline)) {
    Ids id;
    if (loader && t + 2 < end) id = ids_of(t + 2);      // (there by the time the tile is multiplied)
    multiply(t, stage(), holes ? there_of(t) : 15u);
    if (loader && t + 1 < end) {
      put(stage() ^ 1, holes || straddles(t + 1));
      if (t + 2 < end) fetch(id);
    }
    lds_barrier();
  };
  for (int t = begin; t < end; t += 2) {       // (stages as constants: their addresses are offsets of the LDS instructions)
    tile_step(t, std::integral_constant<int, 0>{});
    if (t + 1 < end) tile_step(t + 1, std::integral_constant<int, 1>{});
  }

  if (s_flags[1]) {
    // For every (channel, row), how many of the NaN that were left out the row sees: a product of ones, straight from the cache.
    for (int t = begin; t < end; ++t) {
      if (!straddles(t) && !holes) continue;
      const int lb = t * 4 + quarter;
      const int id = lb < n_blocks ? table[lb] : -1;
      const bool have = (uint32_t)id < (uint32_t)num_blocks;
      const uint8_t* src = v_pool + ((int64_t)(have ? id : 0) * n_kv_heads + kvh) * (kKv8Block * D) + col * kKv8Block;
#pragma unroll
      for (int i = 0; i < DC; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(src + i * 16 * kKv8Block);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          f32x4 seen = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const bf16x8 is = kv8_widen8((nan_codes(w[2 * u]) >> 7) * 0x38u, (nan_codes(w[2 * u + 1]) >> 7) * 0x38u, 1.f);   // 0x38 = 1.0
            bf16x8 sees;
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[e] = have && lb * kKv8Block + 8 * u + e <= q_pos[g] ? (bf16)1.0f : (bf16)0.0f;
            seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, sees, seen, 0, 0, 0);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[g][i][r] = seen[r] > 0.f ? __builtin_nanf("") : oacc[g][i][r];
        }
      }
    }
  }

  float l_tot[2];
#pragma unroll
  for (int g = 0; g < 2; ++g) l_tot[g] = xhalf_sum(xquarter_sum(l_run[g]));
  if (parts > 1) {
    // One part of the keys, rows by channels as the join reads them.
    float* const slab = part_out + ((slot * n_kv_heads + kvh) * parts + part) * (ROWS * (D + 2));
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int r = wr0 + g * 16 + col;
      if (r >= rw.n_rows) continue;
#pragma unroll
      for (int i = 0; i < DC; ++i) *reinterpret_cast<f32x4*>(slab + r * D + i * 16 + quarter * 4) = oacc[g][i];
      if (quarter < 2) slab[ROWS * D + 2 * r + quarter] = quarter ? l_tot[g] : m_ref[g];
    }
    return;
  }

  // ---- normalise, stage through LDS (all waves are past their last tile), store rows with 16-byte accesses ----
  bf16* stage = (wave < 4 ? s_k[0] : s_v[0]) + (wave & 3) * (32 * D);
  static_assert(4 * 32 * D <= 2 * TILE, "the waves' rows fit the stages");
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float inv = 1.0f / l_tot[g];
    const int r = g * 16 + col;
#pragma unroll
    for (int i = 0; i < DC; ++i) {
      bf16x4 v4;
#pragma unroll
      for (int b = 0; b < 4; ++b) v4[b] = static_cast<bf16>(l_tot[g] == 0.f ? 0.f : oacc[g][i][b] * inv);
      *reinterpret_cast<bf16x4*>(stage + r * D + (((i * 2 + (quarter >> 1)) ^ (r & 7)) << 3) + (quarter & 1) * 4) = v4;
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
                            int64_t n_tokens, int n_q_heads, float scale_log2, const Kv8Plan& p, void* workspace, hipStream_t s) {
  const int hkv = c.n_kv_heads;
  const uint8_t *kp = (const uint8_t*)c.k_pool, *vp = (const uint8_t*)c.v_pool;
  const int n_slots = (int)p.slots;
  i32x4* list = p.shares > 0 ? static_cast<i32x4*>(workspace) : nullptr;
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + (list ? ((size_t)p.slots * hkv * 16 + 255) / 256 * 256 : 0));
  if (p.few())
    launch_kernel(p.rows == 16 ? kv8_attn_few_kernel<D, 1> : kv8_attn_few_kernel<D, 2>, dim3((unsigned)((p.shares > 0 ? p.shares : n_slots) * hkv)),
                  kFewWaves * 64, 0, s, q, q_stride, o, o_stride, list, part, p.shares, n_slots, n_tokens, n_q_heads, hkv, scale_log2, kp, vp,
                  c.k_scale, c.v_scale, c.num_blocks, b.n_seqs, b.max_blocks, b.cu_seqlens, b.cached_lens, b.block_tables);
  else
    launch_kernel(kv8_attn_tile_kernel<D>, dim3((unsigned)(p.tiles * p.parts * hkv)), 512, 0, s, q, q_stride, o, o_stride, part, p.parts, p.part_steps,
                  (int)p.tiles, n_tokens, n_q_heads, hkv, scale_log2, kp, vp, c.k_scale, c.v_scale, c.num_blocks, b.n_seqs, b.max_blocks,
                  b.cu_seqlens, b.cached_lens, b.block_tables);
  if (p.cut()) {
    // A workgroup to a row where a few rows have many parts.  us, side by side | in order: one token of 32 heads behind 32767 positions
    // 20.4 | 31.2, four behind 8000 21.9 | 24.8, eight behind 4000 22.4 | 23.6 (eight shares to a slot: in order), 16 behind 2000 20.0 | 19.9,
    // 32 behind 4000 48.9 | 47.8; 40 tokens of 8/1 heads behind 30000 41.4 | 45.7, 80 behind 16000 42.5 | 43.2 (640 rows: in order).
    const int64_t rows = n_tokens * n_q_heads;
    const bool many = rows <= 512 && (list ? p.shares > 8 * n_slots : p.parts > 8);
    const int64_t per = many ? 1 : 1024 / D;
    launch_kernel(many ? kv8_attn_merge_kernel<D, 1024 / D> : kv8_attn_merge_kernel<D, 1>, dim3((unsigned)((rows + per - 1) / per)), 256, 0, s,
                  list, part, o, o_stride, p.rows, p.parts, p.part_steps, n_tokens, n_q_heads, hkv, b.n_seqs, b.max_blocks, b.cu_seqlens,
                  b.cached_lens);
  }
}

void launch_kv8_attention(const fp_kv8_cache& c, const fp_kv8_batch& b, const void* q, int64_t q_stride, void* o, int64_t o_stride,
                          int64_t n_tokens, int n_q_heads, float scale, int max_new, int max_len, void* workspace,
                          size_t workspace_bytes, hipStream_t s) {
  if (n_tokens == 0 || b.n_seqs == 0) return;
  Kv8Plan p = kv8_plan(n_tokens, b.n_seqs, n_q_heads, c.n_kv_heads, c.head_dim, max_new, max_len, workspace ? workspace_bytes : 0);
  if (p.slots * ((b.max_blocks + 3) / 4 + 1) > INT32_MAX) p.shares = 0;      // (steps are counted in 32 bits)
  const float scale_log2 = scale * 1.4426950408889634f;
  if (c.head_dim == 128)
    launch_kv8_attn<128>(c, b, (const bf16*)q, q_stride, (bf16*)o, o_stride, n_tokens, n_q_heads, scale_log2, p, workspace, s);
  else
    launch_kv8_attn<64>(c, b, (const bf16*)q, q_stride, (bf16*)o, o_stride, n_tokens, n_q_heads, scale_log2, p, workspace, s);
}

}  // namespace fp
