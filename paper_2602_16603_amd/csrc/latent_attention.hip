// Latent attention in its absorbed form: causal attention of all query heads over the paged cache of latent rows, which are keys (R + P
// numbers) and values (their first R) at once (Eq. (2) with the causal mask and the KV cache of Section 3.1).
#include "../../include/flowprefill.h"
#include "common.h"
#include "kernels.h"
#include "latent.h"
#include "launch.h"

namespace fp {

namespace {

// Slots of sequence s and the steps that are counted for each: those of its last row, and one for a sequence that sees nothing, whose
// rows are to be zero.
__device__ __forceinline__ void seq_steps(int s, int group, int rows, int64_t n_tokens, int max_blocks, const int32_t* cu_seqlens,
                                          const int32_t* cached_lens, int& slots, int& steps) {
  const int64_t lo = cu_seqlens[s], n = min((int64_t)cu_seqlens[s + 1], n_tokens) - lo, cached = cached_lens[s];
  slots = lo >= 0 && n > 0 ? (int)((n * group + rows - 1) / rows) : 0;
  const int64_t keys = cached < 0 ? 0 : min(cached + n, (int64_t)max_blocks * kLatentBlock);
  steps = (int)max((keys + kLatentStep - 1) / kLatentStep, (int64_t)1);
}
// Where the steps of sequence s (one per lane, 64 neighbours) end, counted from the first lane's.
__device__ __forceinline__ int seq_ends(int s, int group, int rows, int64_t n_tokens, int n_seqs, int max_blocks, const int32_t* cu_seqlens,
                                        const int32_t* cached_lens) {
  int slots = 0, steps = 0;
  if (s < n_seqs) seq_steps(s, group, rows, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
  return latent_scan(slots * steps);
}

// XORs of 16-byte chunks within a row, so that no read meets another on a bank.  LDS serves a 16-byte read in four turns of lanes 0-3, 12-15,
// 20-23, 24-27; 4-11, 16-19, 28-31; and the same of the upper half; an 8-byte read in two turns of 32 lanes.
// Tile rows, neighbours 128 bytes apart modulo 256: a score fragment reads one chunk of 16 rows in lanes 0-15 and its neighbour in
// lanes 16-31, a value fragment two neighbouring chunks of rows 0-3 and 8-11 (modulo 16).
__device__ __forceinline__ int tile_swizzle(int row) { return ((row >> 1) & 4) | (row & 2); }
// Rows of probabilities, 64 bytes apart.
__device__ __forceinline__ int weight_swizzle(int row) { return (0 - (row >> 2)) & 3; }

}  // namespace

// ------------------------------------------------------------------------------------------
// One workgroup = NW waves = 8 NW rows (64 or 32), a row being a (token, head) pair: all heads share the keys, so 64 heads of one token fill
// a workgroup, or a few heads of several tokens.  Keys are taken 32 at a time (two blocks) through four LDS stages that DMA fills three steps
// ahead.  Wave w computes the scores of rows 16 (w / 2) .. +15 with keys 16 (w % 2) .. +15, its queries in registers, and then the sums of rows
// 32 (w / 4) .. +31 for a quarter of the R columns; the probabilities change hands through LDS.
//
// S^T = K Q^T puts a row into lane % 16, so that reference and sum of a row are one number a lane.  O^T += V^T P^T: V^T comes out of
// the same LDS rows by reads that turn 4 x 16 elements.  The products of step t and the scores of step t + 1 lie between the same two
// barriers, one a step.
//
// The exponent reference of a row moves only when a score lies more than 2^8 above it; a wave that finds one says so beside its
// probabilities, and behind the barrier all waves agree on new references and the probabilities are written once more.
// Scores are multiplied by scale * log2(e) and rounded before the reference is taken off, so that the largest score's exponent is
// never above the 2^8, however large the numbers.  Probabilities are rounded to bf16 for the second product (the matrix cores' type),
// and the sum that divides is taken over the rounded ones.
//
// Keys that some rows of a step do not see have weight zero there, and would make NaN of an infinity or a NaN among their values.
// Values are the keys' own first R numbers, so such a key shows in the scores of every row: a step that hides a score which is not finite
// takes such values out of its tile, and the rows that do see one get their NaN at the end.  Keys of a block that is not there are zeros, and stay.
//
// What bounds it: with few heads and single tokens HBM (64 tokens of 20 heads behind 512 .. 16384 positions, 378 MB in 85 us, 4.4 TB/s, and 8 for
// the join).  With many rows the chain of a step, in which no unit is full: 512 tokens of 20 heads behind 15872, 359 GFLOP, take 370 to 396
// us with the join from card to card (0.91 to 0.97 PFLOP/s; a large library product reaches 1.4), the matrix cores are busy for 39 % of the
// clocks and LDS for 37 %.  Four waves of 32 rows by half of the columns, one to a SIMD, halve LDS reads and took 429 | eight 393.  LDS
// rows whose fragments' reads meet on a bank: 44 M of 95 M LDS clocks were conflicts, now 3 M of 84 M.  No gain: priorities, deeper prefetch.
// A few tokens' call is a chain: lengths, queries and ids, a tile, the steps, the join (one token of 128 heads behind 32767: 26 us and 11).
// ------------------------------------------------------------------------------------------
template <int R, int P, int NW>
__global__ __launch_bounds__(NW * 64, NW / 4) void latent_attn_kernel(
    const bf16* __restrict__ q, int64_t q_stride, bf16* __restrict__ o, int64_t o_stride, i32x4* __restrict__ list_out,
    float* __restrict__ part_out, int shares, int units, int head_tiles, int group, int64_t n_tokens, int n_heads, float scale_log2,
    const bf16* __restrict__ pool, int64_t num_blocks, int n_seqs, int max_blocks, const int32_t* __restrict__ cu_seqlens,
    const int32_t* __restrict__ cached_lens, const int32_t* __restrict__ block_tables) {
  constexpr int ROWS = 8 * NW, KT = kLatentStep;
  constexpr int KK = (R + P) / 32;                    // k-steps of the scores
  constexpr int W = R + 64;                           // elements of a tile row in LDS: 128 bytes beyond a multiple of 256
  constexpr int CH = W / 8;                           // its 16-byte chunks
  constexpr int IPB = CH / 4;                         // DMA instructions of a block, shared by half of the waves
  constexpr int IPW = (IPB + NW / 2 - 1) / (NW / 2);  // of a wave (where that is too many, the last ones are done twice)
  constexpr int CB = R / 64;                          // 16-column blocks of a wave
  constexpr int ROW_BYTES = (R + P) * 2;
  static_assert(CH % 8 == 0 && W * 2 % 256 == 128, "tile rows");
  __shared__ __attribute__((aligned(1024))) bf16 s_t[4][KT * W];
  __shared__ __attribute__((aligned(16))) bf16 s_p[2][ROWS * KT];
  __shared__ float s_row[2][ROWS], s_alpha[ROWS];
  __shared__ __attribute__((aligned(16))) int s_flag[2][NW];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kb = wave & 1, sr = (wave >> 1) * 16;     // scores: key block, first row
  const int vc = (wave & 3) * (R / 4), vr = (wave >> 2) * 32;   // sums: first column, first row
  // (head tiles of a unit are eight workgroups apart, that is on one XCD, whose L2 then holds their keys)
  const int head_tile = (blockIdx.x / 8) % head_tiles;
  const int unit = blockIdx.x / (8 * head_tiles) * 8 + blockIdx.x % 8;
  if (unit >= units) return;

  // ---- this workgroup's share of the steps: from step `begin` of slot j of sequence s on, as positions pos .. stop among all ----
  int s = 0, j = 0, begin = 0, slots = 0, steps = 0;
  int total = 1, n_shares = 1, pos = 0, stop = 1;
  if (shares == 0) {
    latent_tile_from_end(unit, group, ROWS, n_tokens, n_seqs, cu_seqlens, s, j);
    if (s < 0) return;
    steps = 1;                                        // (one run; its own number of steps follows from its rows)
    slots = j + 1;
  } else {
    int ends = 0;
    total = 0;
    for (int base = 0; base < n_seqs; base += 64) {
      ends = seq_ends(base + (int)(threadIdx.x & 63), group, ROWS, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens);
      total += __builtin_amdgcn_readlane(ends, 63);
    }
    n_shares = (int)latent_shares(shares, total);
    if (unit >= n_shares || total == 0) return;
    pos = (int)kv8_share(unit, n_shares, total);
    stop = (int)kv8_share(unit + 1, n_shares, total);
    int before = 0;
    for (int base = 0;; base += 64) {
      if (n_seqs > 64) ends = seq_ends(base + (int)(threadIdx.x & 63), group, ROWS, n_tokens, n_seqs, max_blocks, cu_seqlens, cached_lens);
      const uint64_t past = __ballot(before + ends > pos);
      if (past) {
        const int first = (int)__builtin_ctzll(past);
        s = base + first;
        if (first > 0) before += __builtin_amdgcn_readlane(ends, first - 1);
        break;
      }
      before += __builtin_amdgcn_readlane(ends, 63);
    }
    seq_steps(s, group, ROWS, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
    j = (pos - before) / steps;
    begin = pos - before - j * steps;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  j = __builtin_amdgcn_readfirstlane(j);
  begin = __builtin_amdgcn_readfirstlane(begin);
  slots = __builtin_amdgcn_readfirstlane(slots);
  steps = __builtin_amdgcn_readfirstlane(steps);
  const int start = pos;

  const int lane = threadIdx.x & 63, col = lane & 15, quarter = lane >> 4;
  const int head0 = head_tile * group;

  // Source offsets of this lane's chunks within a block: the tile's swizzle is in the order in which the chunks are fetched.  Chunks that
  // fill a row up to W come from beyond the block, as zeros.
  uint32_t dma_off[IPW];
  const int dma_first = min((wave >> 1) * IPW, IPB - IPW);
#pragma unroll
  for (int i = 0; i < IPW; ++i) {
    const int at = (dma_first + i) * 64 + lane, row = at / CH, c = at % CH;
    const int src = (c & ~7) | ((c & 7) ^ tile_swizzle(row));
    dma_off[i] = src < (R + P) / 8 ? (uint32_t)(row * ROW_BYTES + src * 16) : 0x40000000u;
  }
  const uint32_t dma_to = latent_lds_address(s_t[0]) + (kb * (kLatentBlock * W) + dma_first * 512) * 2;
  const int k_row = kb * 16 + col;
  int k_off[2], v_off[4];
#pragma unroll
  for (int b = 0; b < 2; ++b) k_off[b] = k_row * W + (((b * 4 + quarter) ^ tile_swizzle(k_row)) << 3);
  const int v_row = 8 * quarter + (col >> 2);
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int chunk = vc / 8 + b * 2 + ((col & 3) >> 1);
    v_off[b] = v_row * W + (((chunk & ~7) | ((chunk & 7) ^ tile_swizzle(v_row))) << 3) + (col & 1) * 4;
  }
  // Where this lane's four probabilities of a row go, and where it finds eight.
  const int p_put = (sr + col) * KT + (((kb * 2 + (quarter >> 1)) ^ weight_swizzle(col)) << 3) + (quarter & 1) * 4;
  const int p_get = (vr + col) * KT + ((quarter ^ weight_swizzle(col)) << 3);

  while (pos < stop) {
    const int run = min(stop - pos, steps - begin);
    const int64_t seq_lo = cu_seqlens[s];
    const int64_t all_rows = (min((int64_t)cu_seqlens[s + 1], n_tokens) - seq_lo) * group;
    const int64_t row0 = (int64_t)j * ROWS;
    const int n_rows = __builtin_amdgcn_readfirstlane((int)min(all_rows - row0, (int64_t)ROWS));
    const int cached = min(cached_lens[s], max_blocks * kLatentBlock);   // (from the table's end on all of it is visible)
    const int64_t last_tok = (row0 + n_rows - 1) / group;
    const int n_keys = __builtin_amdgcn_readfirstlane(cached < 0 ? 0 : (int)min((int64_t)cached + last_tok + 1, (int64_t)max_blocks * kLatentBlock));
    const int own_steps = (n_keys + KT - 1) / KT;
    const int end = shares == 0 ? own_steps : min(own_steps, begin + run);
    const bool whole = run == steps;
    const int64_t slab = ((int64_t)unit * 2 + (pos == start ? 0 : 1)) * head_tiles + head_tile;
    if (shares > 0 && begin == 0 && threadIdx.x == 0 && head_tile == 0) {
      const int64_t slot = kv8_slot(seq_lo * group, s, ROWS, 1) + j;
      list_out[slot] = i32x4{whole ? -1 : unit, pos == start ? 0 : 1, (int)kv8_share_of(pos + steps - 1, n_shares, total), 0};
    }
    // Token and head of row r; -1: none.
    auto position = [&](int r, int64_t& tok, int& head) __attribute__((always_inline)) {
      const int64_t row = row0 + min(r, n_rows - 1);
      tok = row / group;
      head = head0 + (int)(row - tok * group);
      return r < n_rows && head < n_heads ? cached + (int)tok : -1;
    };

    // ---- queries of this wave's rows (B operand) ----
    bf16x8 qf[KK];
    int64_t tok;
    int head;
    const int q_pos = position(sr + col, tok, head);
    {
      const bf16* src = q + (seq_lo + tok) * q_stride + (int64_t)min(head, n_heads - 1) * (R + P) + quarter * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(src + kk * 32);
    }
    // The position that the fewest keys are visible to.
    const int first_pos = __builtin_amdgcn_readfirstlane(cached + (int)(row0 / group));

    f32x4 acc[2][CB], sc;
    float m_ref = -INFINITY, l_run = 0.f, l_new = 0.f;
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < CB; ++i) acc[g][i] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int32_t* table = block_tables + (int64_t)s * max_blocks;
    const int n_blocks = (n_keys + kLatentBlock - 1) / kLatentBlock;
    // Ids of this wave's blocks of 64 tiles, a tile to a lane, and of the 64 behind them.
    auto ids_from = [&](int t) __attribute__((always_inline)) {
      const int lb = (t + lane) * 2 + kb;
      return lb < n_blocks ? table[lb] : -1;
    };
    uint32_t there_bits = 0;                          // of this wave's block of the last tiles
    int ids = ids_from(begin), ids_later = ids_from(begin + 64);
    // This wave's share of its block of tile t; rows behind the last key, and blocks that are not there, arrive as zeros.
    u32x4 source;
    uint32_t target = 0;
    auto aim = [&](int t) __attribute__((always_inline)) {
      const int k = t - begin;
      if (__builtin_expect(k > 0 && k % 64 == 0, 0)) {
        ids = ids_later;
        ids_later = ids_from(t + 64);
      }
      const int id = __builtin_amdgcn_readlane(ids, k % 64);
      const bool have = id >= 0 && id < num_blocks;
      there_bits = (there_bits << 1) | (have ? 1u : 0u);
      const int rows = min(max(n_keys - (t * 2 + kb) * kLatentBlock, 0), kLatentBlock);
      source = latent_source(pool + (int64_t)(have ? id : 0) * (kLatentBlock * (R + P)), have ? rows * ROW_BYTES : 0);
      target = dma_to + (k & 3) * (KT * W * 2);
    };
    auto fetch = [&](auto i) __attribute__((always_inline)) { latent_load_lds<i() * 1024>(source, target, dma_off[i()]); };
    auto fetch_all = [&](int t) __attribute__((always_inline)) {
      aim(t);
      latent_each<IPW>(fetch);
    };

    // Fragments are asked for AHEAD of their products, a read behind each product.
    constexpr int AHEAD = 6, AHEAD_V = CB < 4 ? CB : 4, TURN = KK > AHEAD ? KK - AHEAD : 0;    // (TURN: where the scores' last read is behind)
    static_assert(TURN + AHEAD_V < KK, "the sums' first reads lie behind products of the scores");
    bf16x8 kf[KK];
    auto key = [&](const bf16* tile, int kk) __attribute__((always_inline)) {
      kf[kk] = *reinterpret_cast<const bf16x8*>(tile + (kk >> 1) * 64 + k_off[kk & 1]);
    };
    auto first_keys = [&](const bf16* tile) __attribute__((always_inline)) {
#pragma unroll
      for (int kk = 0; kk < AHEAD && kk < KK; ++kk) key(tile, kk);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto scores = [&](const bf16* tile, auto&& behind) __attribute__((always_inline)) {
      sc = f32x4{0.f, 0.f, 0.f, 0.f};
      latent_each<KK>([&](auto kk) __attribute__((always_inline)) {
        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kk()], qf[kk()], sc, 0, 0, 0);
        if constexpr (kk() + AHEAD < KK) key(tile, kk() + AHEAD);
        behind(kk);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    float weight[4];
    auto weigh = [&](f32x4 x, int r) __attribute__((always_inline)) {
      const float m = m_ref == -INFINITY ? 0.f : m_ref;                // (a row that has seen nothing yet)
      weight[r] = __builtin_amdgcn_exp2f(x[r] - m);
    };
    auto put = [&](bf16* p) __attribute__((always_inline)) {
      bf16x4 e;
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = static_cast<bf16>(weight[r]);
      l_new = pair_sum(e[0], e[1], pair_sum(e[2], e[3], 0.f));
      *reinterpret_cast<bf16x4*>(p + p_put) = e;
    };
    // Masks the scores of step t; -> whether one that is hidden is not finite.  A block that is not there has values of zero, which are
    // finite whatever a query makes of them: only tiles from the first row's position on are ever cleaned, and put right at the end.
    auto mask = [&](int t, bool there) __attribute__((always_inline)) {
      bool hides = false;
      if (__builtin_expect(!there || t * KT + KT - 1 > first_pos, 0)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool sees = there && t * KT + kb * 16 + quarter * 4 + r <= q_pos;
          hides |= there && !sees && !(sc[r] - sc[r] == 0.f);
          sc[r] = sees ? sc[r] : -INFINITY;
        }
      }
      return hides;
    };
    // Scales the scores, writes their probabilities and says what their step needs, in pieces that fit behind products.
    bool moves = false;
    constexpr int PIECES = 8;
    auto soften = [&](int piece, bool hides, bf16* p, int* flag) __attribute__((always_inline)) {
      if (piece == 0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[r] = latent_product(sc[r], scale_log2);
      } else if (piece == 1) {
        moves = max3(sc[0], sc[1], __builtin_fmaxf(sc[2], sc[3])) > m_ref + 8.f;
      } else if (piece < 6) {
        weigh(sc, piece - 2);
      } else if (piece == 6) {
        put(p);
      } else if (piece == 7) {
        flag[wave] = (__any(moves) ? 1 : 0) | (__any(hides) ? 2 : 0);
      }
    };
    // New references where a score of the step before asks for them; all waves take part.
    f32x4 last_sc;
    auto move = [&](bf16* p) __attribute__((always_inline)) {
      const float top = xhalf_max(xquarter_max(max3(last_sc[0], last_sc[1], __builtin_fmaxf(last_sc[2], last_sc[3]))));
      if (quarter == 0) s_row[kb][sr + col] = top;
      latent_barrier();
      const float now = max3(m_ref, top, s_row[kb ^ 1][sr + col]);
      // (equal ones may be infinite)
      const float alpha = now == m_ref ? 1.f : m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref - now);
      m_ref = now;
      l_run = alpha == 1.f ? l_run : l_run * alpha;
      if (kb == 0 && quarter == 0) s_alpha[sr + col] = alpha;
#pragma unroll
      for (int r = 0; r < 4; ++r) weigh(last_sc, r);
      put(p);
      latent_barrier();
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float a = s_alpha[vr + g * 16 + col];
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[g][i][r] *= a;
      }
    };
    auto value = [&](const bf16* tile, int i) __attribute__((always_inline)) {
      const bf16* a = tile + (i >> 2) * 64 + v_off[i & 3];
      return latent_join(latent_turned(a), latent_turned(a + 4 * W));      // (the swizzle leaves bit 2 of the row out)
    };
    // Infinities and NaN of a tile's values become zeros; all waves take part.
    auto clean = [&](bf16* tile) __attribute__((always_inline)) {
#pragma unroll 1
      for (int at = threadIdx.x; at < KT * CH; at += NW * 64) {
        bf16x8* const chunk = reinterpret_cast<bf16x8*>(tile) + at;
        *chunk = latent_finite(*chunk);
      }
      latent_barrier();
    };
    // The accumulators stay in vector registers: held in those that matrix instructions alone address, they would leave half as many for
    // everything else and be copied there and back around the blocks that are rarely entered.
    auto pin = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < CB; ++i) asm volatile("" : "+v"(acc[g][i]));
    };

    // Behind the barrier of step t: its probabilities are there, and tile t + 1 is.
    bool cleaned = false;
    auto step = [&](int t) __attribute__((always_inline)) {
      const int k = t - begin, par = k & 1;
      bf16* const tv = s_t[k & 3];
      const bf16* const tk = s_t[(k + 1) & 3];
      constexpr int EARLY = (IPW + 1) / 2, LATE = IPW - EARLY;     // DMA instructions behind the scores' products, and behind the sums'
      bf16x8 pf[2], vf[CB];
      i32x4 f[NW / 4];
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) pf[g] = *reinterpret_cast<const bf16x8*>(s_p[par] + g * (16 * KT) + p_get);
      };
      auto values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < AHEAD_V; ++i) vf[i] = value(tv, i);
      };
      first_keys(tk);
      last_sc = sc;
      scores(tk, [&](auto kk) __attribute__((always_inline)) {
        if constexpr (kk() == 0) aim(t + 3);
        if constexpr (kk() == TURN) {
#pragma unroll
          for (int i = 0; i < NW / 4; ++i) f[i] = *reinterpret_cast<const i32x4*>(s_flag[par] + 4 * i);
          weights();
        } else if constexpr (kk() > TURN && kk() <= TURN + AHEAD_V) {
          vf[kk() - TURN - 1] = value(tv, kk() - TURN - 1);
        }
        if constexpr (kk() > 0 && kk() * EARLY / KK != (kk() + 1) * EARLY / KK) fetch(std::integral_constant<int, kk() * EARLY / KK>{});
      });
      int any = 0;
#pragma unroll
      for (int i = 0; i < NW / 4; ++i) any |= f[i][0] | f[i][1] | f[i][2] | f[i][3];
      const int flags = __builtin_amdgcn_readfirstlane(any);
      pin();
      if (__builtin_expect(flags != 0, 0)) {
        if (flags & 1) {
          latent_settle();
          pin();
          move(s_p[par]);
          weights();
          pin();
        }
        if (flags & 2) {
          clean(tv);
          cleaned = true;
          values();
        }
      }
      l_run += l_new;

      bool hides = false;
      latent_each<CB>([&](auto i) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) latent_add_product(acc[g][i()], vf[i()], pf[g]);
        if constexpr (i() + AHEAD_V < CB) vf[i() + AHEAD_V] = value(tv, i() + AHEAD_V);
        latent_each<LATE>([&](auto d) __attribute__((always_inline)) {
          if constexpr (d() * CB / (LATE > 0 ? LATE : 1) == i()) fetch(std::integral_constant<int, EARLY + d()>{});
        });
        constexpr int FROM = CB > 4 ? 1 : 0, EACH = (PIECES + CB - 1 - FROM) / (CB - FROM);
        if (i() == FROM) hides = mask(t + 1, (there_bits >> 2) & 1);   // (the scores' products have left the pipe)
#pragma unroll
        for (int e = 0; e < EACH; ++e)
          if (i() >= FROM) soften((i() - FROM) * EACH + e, hides, s_p[par ^ 1], s_flag[par ^ 1]);
        __builtin_amdgcn_sched_barrier(0);
      });
      __builtin_amdgcn_s_waitcnt(latent_wait_loads(IPW));       // tile t + 2 is there
      latent_barrier();
    };

    if (begin < end) {
      fetch_all(begin);
      fetch_all(begin + 1);
      fetch_all(begin + 2);
      __builtin_amdgcn_s_waitcnt(latent_wait_loads(2 * IPW));
      latent_barrier();
      first_keys(s_t[0]);
      scores(s_t[0], [](auto) {});
      const bool hides = mask(begin, (there_bits >> 2) & 1);
#pragma unroll
      for (int piece = 0; piece < PIECES; ++piece) soften(piece, hides, s_p[0], s_flag[0]);
      __builtin_amdgcn_s_waitcnt(latent_wait_loads(IPW));
      latent_barrier();
#pragma unroll 1
      for (int t = begin; t < end; ++t) step(t);
      latent_settle();
      pin();                                             // (no read of them moves up)
    }
    __builtin_amdgcn_s_waitcnt(latent_wait_loads(0));           // (tiles that were asked for beyond the last step: nothing writes LDS from here on)

    // ---- sums of the rows: the quarters' and the other key block's ----
    const float l_mine = xhalf_sum(xquarter_sum(l_run));
    if (quarter == 0) s_row[kb][sr + col] = l_mine;
    latent_barrier();
    float* const part = part_out + slab * (int64_t)latent_slab_floats(ROWS, R);
    if (!whole && kb == 0 && quarter == 0 && sr + col < n_rows)
      *reinterpret_cast<f32x2*>(part + ROWS * R + 2 * (sr + col)) = f32x2{m_ref, l_mine + s_row[1][sr + col]};
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int r = vr + g * 16 + col;
      if (r >= n_rows) continue;
      int64_t tok_v;
      int head_v;
      const int pos_v = position(r, tok_v, head_v);
      if (cleaned) {
        // What the tiles that hide keys lost: rows that see a value that is not finite.
#pragma unroll 1
        for (int at = max(begin * KT, first_pos / KT * KT); at < min(end * KT, n_keys); ++at) {
          const int id = table[at / kLatentBlock];
          if (id < 0 || id >= num_blocks) continue;
          const bf16* src = pool + ((int64_t)id * kLatentBlock + at % kLatentBlock) * (R + P) + vc + quarter * 4;
#pragma unroll
          for (int i = 0; i < CB; ++i) {
            const bf16x4 v = *reinterpret_cast<const bf16x4*>(src + i * 16);
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[g][i][b] = (float)v[b] - (float)v[b] == 0.f || at > pos_v ? acc[g][i][b] : __builtin_nanf("");
          }
        }
      }
      if (whole) {
        if (head_v >= n_heads) continue;
        const float l = s_row[0][r] + s_row[1][r], inv = 1.0f / l;
        bf16* dst = o + (seq_lo + tok_v) * o_stride + (int64_t)head_v * R + vc + quarter * 4;
#pragma unroll
        for (int i = 0; i < CB; ++i) {
          bf16x4 v;
#pragma unroll
          for (int b = 0; b < 4; ++b) v[b] = static_cast<bf16>(l == 0.f ? 0.f : acc[g][i][b] * inv);
          *reinterpret_cast<bf16x4*>(dst + i * 16) = v;
        }
      } else {
#pragma unroll
        for (int i = 0; i < CB; ++i) *reinterpret_cast<f32x4*>(part + r * R + vc + i * 16 + quarter * 4) = acc[g][i];
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
      seq_steps(s, group, ROWS, n_tokens, max_blocks, cu_seqlens, cached_lens, slots, steps);
    }
    if (pos < stop) latent_barrier();
  }
}

// ------------------------------------------------------------------------------------------
// Joins the shares' partial results, R/4 threads to a (token, head), or a workgroup of 1024: one token of 128 heads in 128 parts 29.5 us | 11.4
// (33 MB).  A workgroup of 1024 to 128 columns of a row: 12.7.
// ------------------------------------------------------------------------------------------
template <int R, int SIDE>
__global__ __launch_bounds__(SIDE > 1 ? 1024 : 256) void latent_attn_merge_kernel(
    const i32x4* __restrict__ list, const float* __restrict__ part_in, bf16* __restrict__ o, int64_t o_stride, int rows, int head_tiles,
    int group, int64_t n_tokens, int n_heads, int n_seqs, const int32_t* __restrict__ cu_seqlens) {
  constexpr int LANES = R / 4, PER = SIDE > 1 ? 1 : 256 / LANES;
  static_assert(SIDE == 1 || SIDE * LANES == 1024, "a workgroup to a row");
  const int64_t row_all = (int64_t)blockIdx.x * PER + (PER > 1 ? threadIdx.x / LANES : 0);
  const int64_t t = row_all / n_heads;
  const int head = (int)(row_all - t * n_heads);
  // (the rows of a wave are neighbours: it looks for the sequence of its first and then steps on)
  const int64_t t0 = __builtin_amdgcn_readfirstlane((int)min(t, n_tokens - 1));
  int s = kv8_find_seq(cu_seqlens, n_seqs, t0, n_tokens, 1, 1, 0);
  if (s < 0 || t >= n_tokens) return;
  while (s + 1 < n_seqs && cu_seqlens[s + 1] <= t) ++s;
  const int64_t seq_lo = cu_seqlens[s];
  if (seq_lo < 0 || t >= cu_seqlens[s + 1]) return;
  const int head_tile = head / group;
  const int64_t row = (t - seq_lo) * group + (head - head_tile * group);
  const int64_t slot = kv8_slot(seq_lo * group, s, rows, 1) + row / rows;
  const i32x4 at = list[slot];
  if (at[0] < 0) return;                               // a slot that one workgroup finished
  const int64_t size = (int64_t)latent_slab_floats(rows, R);
  latent_join_row<R, SIDE>(part_in + (((int64_t)at[0] * 2 + at[1]) * head_tiles + head_tile) * size, (2 - at[1]) * head_tiles * size,
                     2 * head_tiles * size, at[2] - at[0] + 1, rows, (int)(row % rows), o + t * o_stride + (int64_t)head * R);
}

namespace {

template <int R, int P>
void launch_for(const fp_latent_cache& c, const fp_latent_batch& b, const bf16* q, int64_t q_stride, bf16* o, int64_t o_stride,
                int64_t n_tokens, int n_heads, float scale_log2, const LatentPlan& p, void* workspace, hipStream_t s) {
  i32x4* list = p.shares > 0 ? static_cast<i32x4*>(workspace) : nullptr;
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + (list ? latent_list_bytes(p.slots) : 0));
  const int units = p.shares > 0 ? p.shares : (int)p.tiles;
  launch_kernel(p.rows == 32 ? latent_attn_kernel<R, P, 4> : latent_attn_kernel<R, P, 8>, dim3((unsigned)((units + 7) / 8 * 8 * p.head_tiles)),
                p.rows * 8, 0, s, q, q_stride, o, o_stride, list, part, p.shares, units, p.head_tiles, p.group, n_tokens, n_heads, scale_log2,
                (const bf16*)c.pool, c.num_blocks, b.n_seqs, b.max_blocks, b.cu_seqlens, b.cached_lens, b.block_tables);
  if (p.shares > 0) {
    constexpr int SIDE = 1024 / (R / 4), PER = 256 / (R / 4);
    const int64_t rows = n_tokens * n_heads;
    const bool many = rows <= 1024 && p.shares > 8 * p.slots;
    launch_kernel(many ? latent_attn_merge_kernel<R, SIDE> : latent_attn_merge_kernel<R, 1>,
                  dim3((unsigned)(many ? rows : (rows + PER - 1) / PER)), many ? 1024 : 256, 0, s, list, part, o, o_stride, p.rows, p.head_tiles,
                  p.group, n_tokens, n_heads, b.n_seqs, b.cu_seqlens);
  }
}

}  // namespace

void launch_latent_attention(const fp_latent_cache& c, const fp_latent_batch& b, const void* q, int64_t q_stride, void* o, int64_t o_stride,
                             int64_t n_tokens, int n_heads, float scale, int max_new, int max_len, void* workspace, size_t workspace_bytes,
                             hipStream_t s) {
  if (n_tokens == 0 || b.n_seqs == 0) return;
  const LatentPlan p = latent_plan(n_tokens, b.n_seqs, n_heads, c.latent_dim, b.max_blocks, max_new, max_len, workspace ? workspace_bytes : 0);
  const float scale_log2 = scale * 1.4426950408889634f;
  auto go = [&](auto launch) {
    launch(c, b, (const bf16*)q, q_stride, (bf16*)o, o_stride, n_tokens, n_heads, scale_log2, p, workspace, s);
  };
  const bool wide = c.rope_dim == 64;
  if (c.latent_dim == 512) go(wide ? launch_for<512, 64> : launch_for<512, 32>);
  else if (c.latent_dim == 256) go(wide ? launch_for<256, 64> : launch_for<256, 32>);
  else go(wide ? launch_for<128, 64> : launch_for<128, 32>);
}

}  // namespace fp
