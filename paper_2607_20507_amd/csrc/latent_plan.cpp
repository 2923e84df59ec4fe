// Work of the attention over a latent cache: query tiles and key splits.

#include <algorithm>

#include "latent.h"

namespace spec {

LatentPlan plan_latent(const std::vector<LatentSegment>& segs, int H, int max_parts, bool fp32) {
  LatentPlan p;
  int64_t most = 1;
  for (const LatentSegment& s : segs) most = std::max<int64_t>(most, static_cast<int64_t>(s.nrows) * H);
  p.tile = fp32 || most <= 16 ? 16 : most <= 32 ? 32 : most <= 64 ? 64 : 128;
  struct Tile {
    int32_t qv0, nqv, row0, pos0, page0, kend, qoff;
  };
  std::vector<Tile> tiles;
  int64_t most_keys = 0;
  for (const LatentSegment& s : segs) {
    const int64_t first = static_cast<int64_t>(s.row0) * H, n = static_cast<int64_t>(s.nrows) * H;
    for (int64_t m = 0; m < n; m += p.tile) {
      const int64_t c = std::min<int64_t>(p.tile, n - m);
      const int kend = static_cast<int>(s.pos0 + (m + c - 1) / H + 1);  // keys 0 .. its last row's position
      tiles.push_back(Tile{static_cast<int32_t>(first + m), static_cast<int32_t>(c), s.row0, s.pos0, s.page0, kend, s.qoff});
      most_keys = std::max<int64_t>(most_keys, kend);
    }
  }
  const int target = 256, least = 4;
  // the least split, in chunks of 32 keys, that makes at most `target` items (or one for each tile)
  auto items = [&](int64_t sp) {
    int64_t n = 0;
    for (const Tile& t : tiles) n += (t.kend + sp - 1) / sp;
    return n;
  };
  int64_t lo = least, hi = std::max<int64_t>(least, (most_keys + 31) / 32);
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (items(32 * mid) <= std::max<int64_t>(target, static_cast<int64_t>(tiles.size()))) hi = mid;
    else lo = mid + 1;
  }
  int64_t split = 32 * lo;
  auto parts = [&](int64_t sp) {
    int64_t n = 0;
    for (const Tile& t : tiles) n += t.kend > sp ? (t.kend + sp - 1) / sp : 0;
    return n;
  };
  while (parts(split) > max_parts) split *= 2;
  for (const Tile& t : tiles) {
    const int c = static_cast<int>((t.kend + split - 1) / split);
    if (c <= 1) {
      p.items.push_back(LatentItem{t.qv0, t.nqv, t.row0, t.pos0, t.page0, 0, t.kend, -1, t.qoff});
      continue;
    }
    p.groups.push_back(LatentGroup{t.qv0, t.nqv, p.n_parts, c});
    for (int i = 0; i < c; ++i)
      p.items.push_back(LatentItem{t.qv0, t.nqv, t.row0, t.pos0, t.page0, static_cast<int32_t>(i * split),
                                   static_cast<int32_t>(std::min<int64_t>(t.kend, (i + 1) * split)), p.n_parts + i, t.qoff});
    p.n_parts += c;
  }
  // longest key ranges first, so that the short ones fill in behind them
  std::stable_sort(p.items.begin(), p.items.end(),
                   [](const LatentItem& x, const LatentItem& y) { return x.t1 - x.t0 > y.t1 - y.t0; });
  return p;
}

LatentPromptPlan plan_latent_prompt(const std::vector<LatentSegment>& segs, int H) {
  LatentPromptPlan p;
  auto blocks = [&](int rows) {
    int64_t n = 0;
    for (const LatentSegment& s : segs) n += (static_cast<int64_t>(s.nrows) + rows - 1) / rows;
    return n * H;
  };
  if (blocks(256) < 256) p.rows = 128;
  for (const LatentSegment& s : segs)
    for (int64_t r = 0; r < s.nrows; r += p.rows) {
      const int n = static_cast<int>(std::min<int64_t>(p.rows, s.nrows - r)), first = static_cast<int>(r);
      p.items.push_back(LatentItem{s.row0 + s.qoff + first, n, 0, s.pos0 + first, s.page0, 0, s.pos0 + first + n, -1, 0});
    }
  std::stable_sort(p.items.begin(), p.items.end(), [](const LatentItem& x, const LatentItem& y) { return x.t1 > y.t1; });
  return p;
}

bool latent_expands(int nrows, int pos0) { return nrows >= 256; }

}  // namespace spec
