// Prints what the plans of latent attention (csrc/latent_plan.h) make of the calls read from standard input, one per line:
//   plan tokens seqs heads latent max_blocks max_new max_len workspace(-1: unlimited)  -> head_tiles group rows slots tiles shares workspace slab
//   expanded tokens seqs heads v_dim max_new max_len workspace(-1: unlimited)          -> slots tiles parts part_steps workspace
//   shares most total                                                                  -> shares in use
//   heads tokens heads n k                                                             -> 1: in LDS; run tiles
//   large tokens seqs heads                                                            -> 1: refused
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

#include "../../paper_2602_16603_amd/csrc/latent_plan.h"

int main() {
  std::string line, what;
  while (std::getline(std::cin, line)) {
    std::istringstream in(line);
    long long a, b, c, d, e, f, g, h;
    in >> what;
    if (what == "plan" && in >> a >> b >> c >> d >> e >> f >> g >> h) {
      const fp::LatentPlan p = fp::latent_plan(a, b, (int)c, (int)d, (int)e, (int)f, (int)g, h < 0 ? SIZE_MAX : (size_t)h);
      std::printf("%d %d %d %lld %lld %d %zu %zu\n", p.head_tiles, p.group, p.rows, (long long)p.slots, (long long)p.tiles, p.shares, p.workspace,
                  fp::latent_slab_floats(p.rows, (int)d) * 4);
    } else if (what == "expanded" && in >> a >> b >> c >> d >> e >> f >> g) {
      const fp::ExpandedPlan p = fp::expanded_plan(a, b, (int)c, (int)d, (int)e, (int)f, g < 0 ? SIZE_MAX : (size_t)g);
      std::printf("%lld %lld %d %d %zu\n", (long long)p.slots, (long long)p.tiles, p.parts, p.part_steps, p.workspace);
    } else if (what == "shares" && in >> a >> b) {
      std::printf("%lld\n", (long long)fp::latent_shares(a, b));
    } else if (what == "heads" && in >> a >> b >> c >> d) {
      const long long tiles = (c + fp::heads_outputs((int)d) - 1) / fp::heads_outputs((int)d);
      std::printf("%d %lld %lld\n", fp::heads_in_lds(a, b, d) ? 1 : 0, (long long)fp::heads_run(a, b, tiles), tiles);
    } else if (what == "large" && in >> a >> b >> c) {
      std::printf("%d\n", fp::latent_too_large(a, b, (int)c) ? 1 : 0);
    }
  }
  return 0;
}
