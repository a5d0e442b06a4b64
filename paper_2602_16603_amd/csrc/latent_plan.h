// How the operators of latent attention cut their work.  Plain C++17 with no GPU dependency: checked on the CPU.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

#include "kv8_plan.h"

namespace fp {

constexpr int kLatentBlock = 16;               // tokens per block
constexpr int kLatentStep = 32;                // keys per step of the absorbed form
constexpr int kLatentMaxBlocks = 1 << 26;      // of a sequence: the kernels hold positions in 32 bits
constexpr int kLatentWorkgroups = 256;         // one per CU
constexpr int kLatentHeads = 64;               // heads of a head tile at most: the rows of a workgroup
// Steps of a share at least, and shares for each slot that can be in use at most, but for those of kLatentLongSteps.  All at R = 512.  us with the join,
// 4 | 8 | 16 | 32 steps, one token of 128 heads behind 600 positions 25 | 29 | 35 | 32 (with 32 it is not cut), 2000 27 | 30 | 40 | 77, 8000
// 31 | 32 | 39 | 55; of 20 heads behind 600 18 | 21 | 25 | 22, 8000 20 | 22 | 27 | 40, eight such behind 4000 28 | 29 | 35 | 50.  One token in 256 | 128
// shares, 32 heads behind 32767 33 | 29, 60000 38 | 36, 120000 47 | 51; 64 heads 38 | 35, 42 | 42, 50 | 56; 32 of R = 128 17.6 | 17.9, 20 | 22, 24 | 31.
constexpr int kLatentShareSteps = 4, kLatentMaxParts = 128, kLatentLongSteps = 16;
// What a join costs, in steps (1.2 us): a launch, and writing and reading 2 MB of partial results.  20 heads, one token behind 250 positions
// whole 14 us, in shares 17; 300 behind 600 43 | 51; 512 behind 15872 whole 600, in shares 370.
constexpr int64_t kLatentJoinSteps = 4, kLatentJoinBytes = 2 << 20;
constexpr int kExpandedRows = 256;             // rows of a workgroup of the expanded form
constexpr int kExpandedStep = 64;              // keys per step

constexpr bool latent_dims(int latent, int rope) {
  return (latent == 128 || latent == 256 || latent == 512) && (rope == 32 || rope == 64);
}
constexpr bool expanded_dims(int nope, int rope, int v) {
  return (nope == 64 || nope == 128) && (rope == 32 || rope == 64) && (v == 64 || v == 128);
}

// Launches have fewer than 2^32 threads: at most 64 for a token and 32 of its heads, 8 for a (token, head), 512 for a (sequence, head).
constexpr bool latent_too_large(int64_t n_tokens, int64_t n_seqs, int n_heads) {
  return n_tokens >= 1 << 24 || n_seqs >= 1 << 24 || n_tokens * n_heads >= 1 << 27 || (n_seqs < n_tokens ? n_seqs : n_tokens) * n_heads >= 1 << 22;
}

// Absorbed form.  All heads read the same keys.  A slot is `rows` (token, head) pairs of one sequence and head tile, heads fastest; the
// head tiles of a slot have the same steps, so a share of the steps is dealt to one workgroup for each of them.
struct LatentPlan {
  int head_tiles = 1, group = 1;       // group: heads of a tile (the last tile may have fewer)
  int rows = 32;                       // 32 or 64
  int64_t slots = 0;                   // kv8_slot's, gaps included
  int64_t tiles = 0;                   // slots that can be in use
  int shares = 0;                      // 0: a workgroup walks all steps of its slot
  size_t workspace = 0;
};
constexpr size_t latent_list_bytes(int64_t slots) { return ((size_t)slots * 16 + 255) / 256 * 256; }
constexpr size_t latent_slab_floats(int rows, int latent) { return (size_t)rows * (latent + 2); }

inline LatentPlan latent_plan(int64_t n_tokens, int64_t n_seqs, int n_heads, int latent, int max_blocks, int max_new, int max_len,
                              size_t workspace_bytes) {
  LatentPlan p;
  p.head_tiles = (n_heads + kLatentHeads - 1) / kLatentHeads;
  p.group = (n_heads + p.head_tiles - 1) / p.head_tiles;
  p.rows = (int64_t)max_new * p.group <= 32 ? 32 : 64;
  p.slots = kv8_slot(n_tokens * p.group, n_seqs, p.rows, 1);
  const int64_t full = std::min(n_seqs, n_tokens);
  p.tiles = (n_tokens * p.group - full) / p.rows + full;
  const int64_t steps = std::max<int64_t>(1, ((int64_t)max_len + kLatentStep - 1) / kLatentStep);
  // Many more workgroups than CUs balance themselves, and leave no partial results.  us, whole | in shares, 128 heads behind 4000 positions, 513
  // tokens 725 | 688, 600 742 | 794, 700 897 | 939; behind 15000, 513 2500 | 2259, 600 2478 | 2443, 700 2999 | 3015, 1000 4038 | 4411; 32 heads, 2600 behind
  // 4000 1044 | 1180; 20 heads, 3300 behind 4000 913 | 1023; 128 heads, 300 behind 4000 and 500 behind 100 520 | 684.
  if (p.tiles * p.head_tiles > 4 * kLatentWorkgroups) return p;
  if (p.slots * ((max_blocks + 1) / 2 + 1) > INT32_MAX) return p;            // steps are counted in 32 bits
  const size_t lists = latent_list_bytes(p.slots);
  const size_t slab = latent_slab_floats(p.rows, latent) * 4 * p.head_tiles;
  const int64_t most = std::min<int64_t>(std::max(1, kLatentWorkgroups / p.head_tiles),
                                         std::max<int64_t>(kLatentMaxParts, steps / kLatentLongSteps) * p.tiles);
  const int64_t fits = workspace_bytes < lists ? 0 : (int64_t)std::min<size_t>((workspace_bytes - lists) / (2 * slab), (size_t)most);
  if (fits < 2) return p;
  const int64_t whole = steps * ((p.tiles * p.head_tiles + kLatentWorkgroups - 1) / kLatentWorkgroups);
  const int64_t used = std::clamp<int64_t>(p.tiles * steps / kLatentShareSteps, 1, fits), each = (p.tiles * steps + used - 1) / used;
  const int64_t joined = (used + std::min(p.tiles, used)) * (int64_t)slab;
  if (each + kLatentJoinSteps + joined / kLatentJoinBytes < whole) {
    p.shares = (int)fits;
    p.workspace = lists + 2 * slab * fits;
  }
  return p;
}
constexpr int64_t latent_shares(int64_t most, int64_t total) {
  return total / kLatentShareSteps < 1 ? 1 : total / kLatentShareSteps < most ? total / kLatentShareSteps : most;
}

// Products per head of many tokens, with W in LDS: `outputs` of a head to a workgroup, and runs of tokens of as few rounds of the eight
// waves, 16 tokens to each, as leave no more workgroups than CUs (40 heads of 64 x 256, 4096 tokens: 240 workgroups 20 us, 280 25).
constexpr int kHeadsRound = 128;
constexpr int heads_outputs(int k) { return k >= 128 ? 65536 / k : 512; }      // 128 KB of W at most; k: 64, 128, 256 or 512
constexpr int64_t heads_run(int64_t m, int64_t n_heads, int64_t n_tiles) {
  const int64_t runs = std::max<int64_t>(1, kLatentWorkgroups / (n_heads * n_tiles)), rounds = (m + kHeadsRound - 1) / kHeadsRound;
  return (rounds + runs - 1) / runs * kHeadsRound;
}
// Where the other form's blocks of 32 tokens of a head are more than there are CUs, and more than one to a head.  us, straight from memory | from LDS, 512 x 128 and 128 x 512:
// 4 heads, 2000 tokens 9.1 | 9.5 and 10.0 | 10.8, 4096 15 | 11 and 18 | 12; 20 heads, 300 9.8 | 9.2 and 10.0 | 10.8, 400 10.7 | 9.5 and 16 | 11, 700
// 15 | 11 and 17 | 11; 32 heads, 256 9.3 | 9.5 and 10.1 | 10.8, 300 11 | 10 and 17 | 11; 40 heads, 128 8.4 | 9.0 and 9.9 | 10.7, 200 10.4 | 9.4 and 15 | 11;
// 128 heads, 64 9.4 | 9.1 and 10.0 | 8.4, 96 14 | 11 and 18 | 11; 256 x 64 and 64 x 256, 40 heads, 128 4.6 | 5.3 and 4.7 | 5.5, 200 5.3 | 5.5 and 5.9 | 5.5,
// 400 7.5 | 6.1 and 8.2 | 5.8; 300 heads of 512 x 128, 32 tokens 15 | 16, 64 20 | 19.
constexpr bool heads_in_lds(int64_t m, int64_t n_heads, int64_t k) {
  return m > 32 && (m + 31) / 32 * n_heads > kLatentWorkgroups && (k == 64 || k == 128 || k == 256 || k == 512);
}

// Expanded form: tiles of 256 rows of one head, their keys in `parts` parts of at least part_steps steps.
struct ExpandedPlan {
  int64_t slots = 0, tiles = 0;
  int parts = 1, part_steps = 0;
  size_t workspace = 0;
};
inline ExpandedPlan expanded_plan(int64_t n_tokens, int64_t n_seqs, int n_heads, int v_dim, int max_new, int max_len, size_t workspace_bytes) {
  ExpandedPlan p;
  p.slots = kv8_slot(n_tokens, n_seqs, kExpandedRows, 1);
  const int64_t full = std::min(n_seqs, n_tokens);
  p.tiles = (n_tokens - full) / kExpandedRows + full;
  const int steps = (int)std::max<int64_t>(1, ((int64_t)max_len + kExpandedStep - 1) / kExpandedStep);
  const size_t part = (size_t)kExpandedRows * (v_dim + 2) * 4 * n_heads * p.slots;
  const int64_t fits = workspace_bytes == SIZE_MAX ? 1 << 20 : (int64_t)(workspace_bytes / std::max<size_t>(part, 1));
  const int64_t want = std::max<int64_t>(1, 256 / (p.tiles * n_heads));
  // At least 4 steps to a part behind a prefix, and 16 of a prompt, whose first tiles see few keys.  us with the join, 4 | 8 | 16 | 32 steps | whole, 20
  // heads: 64 tokens behind 2000 positions 20 | 22 | 32 | 51 | 50, 512 behind 1000 33 | 38 | 50 | 58 | 58, 512 behind 8000 75 | 73 | 75 | 91 |
  // 259, one behind 2000 15 | 20 | 29 | 46 | 46; a prompt of 300 26 | 19 | 19 | 19 | 19, of 777 33 | 40 | 34 | 34 | 35; 16 behind 300 (five steps)
  // 13.9 | 12.3 | 12.2 | 12.2 | 12.3.
  const bool prefix = max_len > 2 * (int64_t)max_new;
  p.part_steps = (int)std::max<int64_t>(!prefix ? 16 : steps < 8 ? 8 : 4, (steps + want - 1) / want);
  const int64_t grid = (1 << 22) / std::max<int64_t>(p.slots * n_heads, 1);
  p.parts = (int)std::clamp<int64_t>((steps + p.part_steps - 1) / p.part_steps, 1, std::max<int64_t>(1, std::min<int64_t>({fits, grid, 256})));
  if (p.parts > 1) p.workspace = part * p.parts;
  return p;
}

}  // namespace fp
