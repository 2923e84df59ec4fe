// Host-only driver of the 4-bit cache's attention planner (plan_kv4): reads
// "G Hkv max_parts fp32 n_segments" and n_segments lines "seq row0 nrows pos0"
// per problem; prints "plan nt w prefill n_parts n_items n_groups", one line per
// item "item row0 nrows pos0 seq t0 t1 part" and per group "group row0 nrows
// part0 nparts".
#include <cstdio>
#include <vector>

#include "host_util.h"

int main() {
  int G, Hkv, max_parts, fp32, n;
  while (std::scanf("%d %d %d %d %d", &G, &Hkv, &max_parts, &fp32, &n) == 5) {
    std::vector<spec::AttnSegment> segs(n);
    for (auto& s : segs)
      if (std::scanf("%d %d %d %d", &s.seq, &s.row0, &s.nrows, &s.pos0) != 4) return 1;
    const spec::AttnPlan p = spec::plan_kv4(segs, G, Hkv, max_parts, fp32 != 0);
    std::printf("plan %d %d %d %d %zu %zu\n", p.nt, p.w, p.prefill ? 1 : 0, p.n_parts, p.items.size(), p.groups.size());
    for (const auto& it : p.items)
      std::printf("item %d %d %d %d %d %d %d\n", it.row0, it.nrows, it.pos0, it.seq, it.t0, it.t1, it.part);
    for (const auto& g : p.groups) std::printf("group %d %d %d %d\n", g.row0, g.nrows, g.part0, g.nparts);
  }
  return 0;
}
