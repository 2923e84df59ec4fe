// Test driver for cutting a table to a length (pure C++, csrc/pages.h): reads a
// script of operations on stdin, prints the outcome and every table after each.
//   "E seq length" ensure | "F seq new" fork of seq's full pages into the empty
//   table new | "C seq keep end" cut to keep positions of end | "K 0 0" compact
//   | "D 0 0" give up every table, printing how many allocations that made
#include <cstdio>
#include <cstdlib>
#include <map>
#include <new>
#include <vector>

#include "pages.h"

static long g_news = 0;
void* operator new(std::size_t n) {
  ++g_news;
  if (void* p = std::malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

int main() {
  int num_pages = 0;
  if (std::scanf("%d", &num_pages) != 1) return 2;
  spec::PagePool pool(num_pages, 16);
  std::map<long long, std::vector<int32_t>> tabs;
  char op;
  long long a, b, c = 0;
  while (std::scanf(" %c %lld %lld", &op, &a, &b) == 3) {
    if (op == 'E') {
      std::printf("%s", pool.ensure(tabs[a], b) ? "ok" : "oom");
    } else if (op == 'F') {
      pool.share(tabs[a], static_cast<int>(tabs[a].size()), tabs[b]);
      std::printf("ok");
    } else if (op == 'C') {
      if (std::scanf("%lld", &c) != 1) return 2;
      if (!pool.can_cut(tabs[a], b)) {
        std::printf("oom");
      } else {
        const spec::PagePool::Cut cut = pool.cut(tabs[a], b, c);
        std::printf("cut %d>%d", cut.from, cut.to);
        for (int32_t s : cut.clear) std::printf(" %d", s);
      }
    } else if (op == 'K') {
      const auto moves = pool.compact();
      std::vector<int32_t> name(num_pages);
      for (int p = 0; p < num_pages; ++p) name[p] = p;
      for (const auto& m : moves) name[m.first] = m.second;
      for (auto& kv : tabs)
        for (int32_t& p : kv.second) p = name[p];
      std::printf("ok");
    } else {
      const long before = g_news;
      for (auto& kv : tabs) pool.truncate(kv.second, 0);
      std::printf("allocated %ld", g_news - before);
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
