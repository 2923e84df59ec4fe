// Host-only driver of the latent attention's planner: reads "H fp32_waves n_segments" and
// n_segments lines "row0 nrows pos0 page0 qoff" per problem; prints "plan tile n_parts",
// one line per item "item qv0 nqv row0 pos0 page0 t0 t1 part qoff", per group "group qv0
// nqv part0 nparts", then the same of the prompt form as "prompt rows n_parts", "block",
// "join".
#include <cstdio>
#include <vector>

#include "latent.h"

int main() {
  int H, waves, n;
  while (std::scanf("%d %d %d", &H, &waves, &n) == 3) {
    std::vector<spec::LatentSegment> segs(n);
    for (auto& s : segs)
      if (std::scanf("%d %d %d %d %d", &s.row0, &s.nrows, &s.pos0, &s.page0, &s.qoff) != 5) return 1;
    const spec::LatentPlan p = spec::plan_latent(segs, H, waves);
    std::printf("plan %d %d\n", p.tile, p.n_parts);
    auto items = [](const char* name, const std::vector<spec::LatentItem>& v) {
      for (const auto& i : v)
        std::printf("%s %d %d %d %d %d %d %d %d %d\n", name, i.qv0, i.nqv, i.row0, i.pos0, i.page0, i.t0, i.t1, i.part, i.qoff);
    };
    auto groups = [](const char* name, const std::vector<spec::LatentGroup>& v) {
      for (const auto& g : v) std::printf("%s %d %d %d %d\n", name, g.qv0, g.nqv, g.part0, g.nparts);
    };
    items("item", p.items);
    groups("group", p.groups);
    const spec::LatentPromptPlan x = spec::plan_latent_prompt(segs, H);
    std::printf("prompt %d %d\n", x.rows, x.n_parts);
    items("block", x.items);
    groups("join", x.groups);
  }
  return 0;
}
