// How the 8-bit cache's operators cut their work: which rows a workgroup finds by itself from the batch description in device
// memory, and how an attention call is cut over its keys.  Plain C++17 with no GPU dependency: checked on the CPU.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace fp {

constexpr int kKv8Block = 16;          // tokens per block
constexpr int kKv8Step = 64;           // keys per attention step
constexpr int kKv8FewWorkgroups = 512; // workgroups of the form for few rows that the chip holds at once (two per CU)
// Rows per (sequence, kv head) up to which the form for few rows is the faster one.  us with the join, few rows | tiles: 16 sequences of 6000
// with 8 heads to a group, 96 rows 62 | 71, 128 rows 56 | 75, 256 rows 87 | 86; one of 16000 with 4, 128 rows 29 | 36, 256 rows 39 | 51.
constexpr int kKv8FewRows = 256;
constexpr int kKv8TileRows = 256;      // rows of a workgroup of the form for many rows
constexpr int kKv8MaxBlocks = 1 << 26; // of a sequence: the kernels hold positions in 32 bits
constexpr int kKv8MinExp = -110, kKv8MaxExp = 119;   // exponents of a scale: 448 * 2^119 is the largest that bf16 holds

// A launch is sized before the lengths in device memory are known: sequence s takes the slots from kv8_slot(first row of s, s) to
// kv8_slot(first row of s + 1, s + 1), with `per` rows to a slot and `extra` slots for the rows' rounding at its two ends.  With
// extra = 1 that is at least ceil(rows / per) slots, since floor(b) - floor(a) + 1 >= ceil(b - a); with extra = 2 and rows that may
// begin inside a slot, one more.  The function of s is increasing, so a slot's sequence is the last one that begins at or before it.
constexpr int64_t kv8_slot(int64_t first_row, int64_t s, int per, int extra) { return first_row / per + extra * s; }

// A launch has fewer than 2^32 threads: at most 64 per (token, head) and 512 per (sequence, kv head), parts of the keys apart
// (kv8_plan bounds those).
constexpr bool kv8_too_large(int64_t n_tokens, int64_t n_seqs, int n_q_heads, int n_kv_heads) {
  return n_tokens > INT32_MAX || n_tokens * (2 * (int64_t)n_kv_heads + n_q_heads) + n_seqs * n_kv_heads * 16 >= 1 << 26;
}

// Number of steps of each part when `steps` are cut into parts of `size` at least, no more than `parts` of them.
constexpr int kv8_part_steps(int steps, int size, int parts) {
  const int even = (steps + parts - 1) / parts;
  return even > size ? even : size;
}

// Few rows per sequence: the steps of all slots, one after the other, are dealt in equal runs to as many workgroups as the chip
// holds at once, so that all end together whatever the lengths are.  Share i of n of `total` steps begins at kv8_share(i, ...); the
// share that has step x is the largest one that begins at or before it.
constexpr int64_t kv8_share(int64_t i, int64_t n, int64_t total) { return i * total / n; }
constexpr int64_t kv8_share_of(int64_t x, int64_t n, int64_t total) { return ((x + 1) * n + total - 1) / total - 1; }
// Shares in use: no less than kKv8ShareSteps steps to each.  us with the join, 4 | 8 | 16 steps, 32 query and 8 kv heads of 128: one token
// behind 600 positions 12.1 | 11.6 | 8.7 (with 16 it is not cut), 2000 11.3 | 12.5 | 15.3, 8000 12.2 | 13.3 | 16.4, 16000 15.1 | 14.5 | 17.4,
// 32768 20.4 | 20.4 | 21.1; 16 tokens behind 600 each 15.9 | 16.0 | 9.1 (not cut).
constexpr int kKv8ShareSteps = 8;
constexpr int64_t kv8_shares(int64_t most, int64_t total) {
  return total / kKv8ShareSteps < 1 ? 1 : total / kKv8ShareSteps < most ? total / kKv8ShareSteps : most;
}

struct Kv8Plan {
  int rows = 16;                       // rows of a slot: 16 or 32 (few-rows form), 256 (tile form)
  int64_t slots = 0;
  int64_t tiles = 0;                   // tile form: slots that can be in use
  int shares = 0;                      // few-rows form: workgroups per kv head that the steps are dealt to; 0: one for every slot
  int parts = 1, part_steps = 0;       // tile form: parts of a slot's keys at most, and steps per part at least
  size_t workspace = 0;
  bool cut() const { return shares > 0 || parts > 1; }
  bool few() const { return rows < kKv8TileRows; }
};

inline Kv8Plan kv8_plan(int64_t n_tokens, int64_t n_seqs, int n_q_heads, int n_kv_heads, int head_dim, int max_new, int max_len,
                        size_t workspace_bytes) {
  Kv8Plan p;
  const int group = n_q_heads / n_kv_heads;
  const int64_t rows = (int64_t)max_new * group;
  // One form for the whole call, by its longest sequence: single tokens beside a prompt take the tile form, a wave of eight at work.  63 single
  // tokens behind 512 .. 16384 positions take 142 us, a prompt of 512 22, all in one call 551.
  p.rows = rows <= 16 ? 16 : rows <= kKv8FewRows ? 32 : kKv8TileRows;
  p.slots = kv8_slot(n_tokens * group, n_seqs, p.rows, 1);
  const int steps = (int)std::max<int64_t>(1, ((int64_t)max_len + kKv8Step - 1) / kKv8Step);
  const size_t slab = (size_t)n_kv_heads * p.rows * (head_dim + 2) * 4;       // one partial result of every kv head
  if (p.few()) {
    // Where each slot's partial results lie (16 bytes), then two of them for every share: only a share's first and last slot
    // can be cut.
    const size_t lists = ((size_t)p.slots * n_kv_heads * 16 + 255) / 256 * 256;
    const int64_t most = std::max(1, kKv8FewWorkgroups / n_kv_heads);
    const int64_t fits = workspace_bytes < lists ? 0 : (int64_t)std::min<size_t>((workspace_bytes - lists) / (2 * slab), (size_t)most);
    if (steps > kKv8ShareSteps && fits > 1) {
      p.shares = (int)fits;
      p.workspace = lists + 2 * slab * fits;
    }
    return p;
  }
  const size_t part = slab * p.slots;
  const int64_t fits = workspace_bytes == SIZE_MAX ? 1 << 20 : (int64_t)(workspace_bytes / std::max<size_t>(part, 1));
  // Rows of S sequences fill at most this many tiles: ceil(a / n) = floor((a - 1) / n) + 1 for each.
  const int64_t full = std::min(n_seqs, n_tokens);
  p.tiles = (n_tokens * group - full) / p.rows + full;
  const int64_t want = std::max<int64_t>(1, 256 / (p.tiles * n_kv_heads));
  // At least 16 steps to a part.  us with the join, 8 | 16 | 32 steps, 32/8 heads of 128: 128 tokens behind 2000 positions 32 | 43 | 68, behind
  // 24576 64 | 63 | 73, 512 behind 1000 42 | 51 | 48, behind 4000 56 | 56 | 77; a prompt of 777, whose first tiles see few keys, 42 | 28 | 28.
  // The number of parts goes by the number of tiles, as the host does not know their lengths: a long chunk beside a prompt that fills
  // the chip with tiles stays whole.  512 tokens behind 15872 take 142, a prompt of 1024 36, the two in one call 434 (256 steps in a row, by 64
  // workgroups); 1024 behind 15360 in two parts 245, 1040 in one 435.
  p.part_steps = (int)std::max<int64_t>(16, (steps + want - 1) / want);
  // (the grids of the parts and of the merge stay below 2^31 threads)
  const int64_t wgs = p.slots * n_kv_heads, grid = (1 << 22) / std::max<int64_t>(wgs, 1);
  p.parts = (int)std::clamp<int64_t>((steps + p.part_steps - 1) / p.part_steps, 1, std::max<int64_t>(1, std::min<int64_t>({fits, grid, 256})));
  if (p.parts > 1) p.workspace = part * p.parts;
  return p;
}

}  // namespace fp
