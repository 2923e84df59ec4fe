// Test driver for pages that several tables hold (pure C++): reads a script of
// operations on stdin, prints the free count, the held pages and every table
// after each step.
//   "E seq length" ensure | "T seq length" truncate | "F seq new" fork of seq's
//   full pages (length 16 * pages) into the empty table new | "K 0 0" compact
#include <cstdio>
#include <map>
#include <vector>

#include "pages.h"

int main() {
  int num_pages = 0;
  if (std::scanf("%d", &num_pages) != 1) return 2;
  spec::PagePool pool(num_pages, 16);
  std::map<long long, std::vector<int32_t>> tabs;
  char op;
  long long a, b;
  while (std::scanf(" %c %lld %lld", &op, &a, &b) == 3) {
    if (op == 'E') {
      std::printf("%s", pool.ensure(tabs[a], b) ? "ok" : "oom");
    } else if (op == 'T') {
      const int before = pool.free_pages(), freed = pool.freed_by(tabs[a], b);
      pool.truncate(tabs[a], b);
      std::printf(pool.free_pages() == before + freed ? "ok" : "miscount");
    } else if (op == 'F') {
      pool.share(tabs[a], static_cast<int>(tabs[a].size()), tabs[b]);
      std::printf("ok");
    } else {
      const auto moves = pool.compact();
      std::vector<int32_t> name(num_pages);
      for (int p = 0; p < num_pages; ++p) name[p] = p;
      std::printf("moved");
      for (const auto& m : moves) {
        name[m.first] = m.second;
        std::printf(" %d>%d", m.first, m.second);
      }
      for (auto& kv : tabs)
        for (int32_t& p : kv.second) p = name[p];
    }
    std::printf(" free %d", pool.free_pages());
    for (auto& kv : tabs) {
      std::printf(" |%lld:", kv.first);
      for (int32_t p : kv.second) std::printf(" %d%s", p, pool.shared(p) ? "*" : "");
    }
    std::printf("\n");
  }
  return 0;
}
