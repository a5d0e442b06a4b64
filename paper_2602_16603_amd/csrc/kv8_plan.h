// How the 8-bit cache's operators cut their work: which rows a workgroup finds by itself from the batch description in device
// memory, and how an attention call is cut over its keys.  Plain C++17 with no GPU dependency: checked on the CPU.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace fp {

constexpr int kKv8Block = 16;          // tokens per block
constexpr int kKv8Step = 64;           // keys per attention step
constexpr int kKv8TileRows = 256;      // rows of a workgroup of the form for many rows
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

struct Kv8Plan {
  int rows = 16;                       // rows of a slot: 16 or 32 (few-rows form), 256 (tile form)
  int64_t slots = 0;
  int parts = 1, part_steps = 0;       // parts of a slot's keys at most, and steps per part at least
  size_t part_bytes = 0;               // workspace of one part of every (slot, kv head)
  size_t workspace() const { return parts > 1 ? part_bytes * parts : 0; }
};

inline Kv8Plan kv8_plan(int64_t n_tokens, int64_t n_seqs, int n_q_heads, int n_kv_heads, int head_dim, int max_new, int max_len,
                        size_t workspace_bytes) {
  Kv8Plan p;
  const int group = n_q_heads / n_kv_heads;
  const int64_t rows = (int64_t)max_new * group;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : kKv8TileRows;
  p.slots = kv8_slot(n_tokens * group, n_seqs, p.rows, 1);
  p.part_bytes = (size_t)p.slots * n_kv_heads * p.rows * (head_dim + 2) * 4;
  const int steps = (int)std::max<int64_t>(1, ((int64_t)max_len + kKv8Step - 1) / kKv8Step);
  const int64_t fits = workspace_bytes == SIZE_MAX ? 1 << 20 : (int64_t)(workspace_bytes / std::max<size_t>(p.part_bytes, 1));
  if (p.rows < kKv8TileRows) {
    const int64_t work = n_seqs * n_kv_heads * steps;
    p.part_steps = (int)std::clamp<int64_t>(work / 4096, 8, 64);
  } else {
    const int64_t tiles = std::max<int64_t>(1, (n_tokens * group + p.rows - 1) / p.rows) * n_kv_heads;
    const int64_t want = tiles >= 256 ? 1 : 256 / tiles;
    p.part_steps = (int)std::max<int64_t>(16, (steps + want - 1) / want);
  }
  // (the grids of the parts and of the merge stay below 2^31 threads)
  const int64_t wgs = p.slots * n_kv_heads, grid = wgs * p.rows < 1 << 25 ? (1 << 22) / std::max<int64_t>(wgs, 1) : 1;
  p.parts = (int)std::clamp<int64_t>((steps + p.part_steps - 1) / p.part_steps, 1, std::max<int64_t>(1, std::min<int64_t>({fits, grid, 256})));
  return p;
}

}  // namespace fp
