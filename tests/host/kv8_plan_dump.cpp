// Prints what the 8-bit cache's plan (csrc/kv8_plan.h) makes of the calls read from standard input, one per line:
//   plan tokens seqs q_heads kv_heads head_dim max_new max_len workspace(-1: unlimited)  -> rows slots shares parts part_steps workspace tiles
//   slot first_row s per extra                                                           -> the slot
//   part steps size parts                                                                -> steps of a part
//   shares most total; share i n total; of step n total                                  -> shares in use, a share's first step, a step's share
//   large tokens seqs q_heads kv_heads                                                   -> 1: refused
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

#include "../../paper_2602_16603_amd/csrc/kv8_plan.h"

int main() {
  std::string line, what;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    long long a, b, c, d, e, f, g, h;
    in >> what;
    if (what == "plan" && in >> a >> b >> c >> d >> e >> f >> g >> h) {
      const fp::Kv8Plan p = fp::kv8_plan(a, b, (int)c, (int)d, (int)e, (int)f, (int)g, h < 0 ? SIZE_MAX : (size_t)h);
      std::printf("%d %lld %d %d %d %zu %lld\n", p.rows, (long long)p.slots, p.shares, p.parts, p.part_steps, p.workspace, (long long)p.tiles);
    } else if (what == "slot" && in >> a >> b >> c >> d) {
      std::printf("%lld\n", (long long)fp::kv8_slot(a, b, (int)c, (int)d));
    } else if (what == "part" && in >> a >> b >> c) {
      std::printf("%d\n", fp::kv8_part_steps((int)a, (int)b, (int)c));
    } else if (what == "shares" && in >> a >> b) {
      std::printf("%lld\n", (long long)fp::kv8_shares(a, b));
    } else if (what == "share" && in >> a >> b >> c) {
      std::printf("%lld\n", (long long)fp::kv8_share(a, b, c));
    } else if (what == "of" && in >> a >> b >> c) {
      std::printf("%lld\n", (long long)fp::kv8_share_of(a, b, c));
    } else if (what == "large" && in >> a >> b >> c >> d) {
      std::printf("%d\n", fp::kv8_too_large(a, b, (int)c, (int)d) ? 1 : 0);
    }
  }
  return 0;
}
