// Work of the attention over a latent cache: query tiles and key splits.

#include <algorithm>

#include "latent.h"

namespace spec {

namespace {

// The least split of at least `lo` that makes at most `target` items (hi makes as few as
// there can be).
template <typename F>
int64_t least_split(int64_t lo, int64_t hi, int64_t target, F&& items) {
  hi = std::max(lo, hi);
  while (lo < hi) {
    const int64_t mid = (lo + hi) / 2;
    if (items(mid) <= target) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

constexpr int kCus = 256;

// Query vectors of a tile: the narrowest that holds a sequence's, at most 64 (32 heads of rank
// 512; tiles of 16 / 32 / 64, us a call): one token of 64 sequences 70 / 56 / 60, the same
// of 131000 keys 71 / 53 / 55, 4 to 8 rows of 64 sequences 201 / 172 / 128; 16 heads of rank
// 256, one token of 64 sequences 36 / 40 / 40.  (Tiles of 128, a wave with 32 query vectors
// and its SIMD to itself, took 131 for the second last.)
int tile_of(const std::vector<LatentSegment>& segs, int H, bool fp32) {
  int64_t most = 1;
  for (const LatentSegment& s : segs) most = std::max<int64_t>(most, static_cast<int64_t>(s.nrows) * H);
  return fp32 || most <= 16 ? 16 : most <= 32 ? 32 : 64;
}

}  // namespace

int64_t latent_tiles(const std::vector<LatentSegment>& segs, int H, int fp32_waves) {
  const int tile = tile_of(segs, H, fp32_waves > 0);
  int64_t n = 0;
  for (const LatentSegment& s : segs) n += (static_cast<int64_t>(s.nrows) * H + tile - 1) / tile;
  return n;
}

LatentPlan plan_latent(const std::vector<LatentSegment>& segs, int H, int fp32_waves) {
  const bool fp32 = fp32_waves > 0;
  LatentPlan p;
  p.tile = tile_of(segs, H, fp32);
  struct Tile {
    int32_t qv0, nqv, row0, pos0, page0, kend, qoff;
  };
  std::vector<Tile> tiles;
  int64_t most_keys = 0, all_keys = 0;
  for (const LatentSegment& s : segs) {
    const int64_t first = static_cast<int64_t>(s.row0) * H, n = static_cast<int64_t>(s.nrows) * H;
    for (int64_t m = 0; m < n; m += p.tile) {
      const int64_t c = std::min<int64_t>(p.tile, n - m);
      const int kend = static_cast<int>(s.pos0 + (m + c - 1) / H + 1);  // keys 0 .. its last row's position
      tiles.push_back(Tile{static_cast<int32_t>(first + m), static_cast<int32_t>(c), s.row0, s.pos0, s.page0, kend, s.qoff});
      most_keys = std::max<int64_t>(most_keys, kend);
      all_keys += kend;
    }
  }
  // Items that run at once, one a CU.  Two a CU (the 64-wide ones have the registers for it)
  // hide each other's starts and ends, but halve the keys of an item, whose parts of 2 KB a
  // query vector are written and read again: the better choice where an item has much to do
  // (keys of all tiles a CU; 256 / 384 items, us): 187 keys 48.3 / 54.2, 312 keys 53.8 / 58.5, 940
  // 83.6 / 86.4, 1300 155 / 128, 2344 158 / 145.
  const int target = p.tile == 64 && all_keys / kCus >= 1200 ? kCus * 3 / 2 : kCus;
  // Whole where a wave then has at most four chunks of 32 keys, or two fp32 pages (a join is
  // a launch): 8 sequences of 256 to 512 keys, 16 heads of rank 256, 24.8 us in parts, 17.3
  // whole.  Otherwise an item has at least four chunks, or a page for every fp32 wave.  Four
  // chunks are one for each key share of a tile of 16, but two in turn of a tile of 32, and of
  // a tile of 64 four: 6 rows of 32 heads behind 505 / 1005 / 2047 / 4000 keys are 12 / 24 / 51 /
  // 96 items on 256 CUs (25.5 / 25.3 / 28.5 / 36.4 us a call).
  // The split is one for all tiles, and makes as many items as there are tiles, or the target:
  // with that many tiles every context stays whole, however long one is.  32 heads, one row of
  // 199 sequences of 512 to 4096 keys 132 us, and of one more of 131001, in parts, 175; of 255
  // such sequences 185, and of one more of 131001, which one workgroup walks, 3629.
  const int shares = p.tile == 64 ? 1 : p.tile == 32 ? 2 : 4;
  const int whole = fp32 ? fp32_waves : 4 * shares;
  const int least = most_keys <= 32 * whole ? whole : fp32 ? fp32_waves / 2 : 4;
  const int64_t split = 32 * least_split(least, (most_keys + 31) / 32, std::max<int64_t>(target, static_cast<int64_t>(tiles.size())),
                                         [&](int64_t sp) {
                                           int64_t n = 0;
                                           for (const Tile& t : tiles) n += (t.kend + 32 * sp - 1) / (32 * sp);
                                           return n;
                                         });
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
  // Blocks of 128 rows take 0.7 of the time of 256.  Where the CUs have much to do (300 keys of
  // 128-row blocks each, or more) the form with less work in all is the faster one, else
  // the smaller blocks, which share it out (32 heads of 128, 256 / 128 rows, us): 300 rows behind 8000
  // keys 181 / 195, 4 x 300 rows 46.6 / 48.5, 512 behind 2000 78.3 / 80.8; 130 behind 500 42.6 / 39.6,
  // 4 x 200 39.6 / 35.0, 512 41.7 / 35.7; 96 behind 8000 135 / 123.
  int64_t wide = 0, narrow = 0, keys = 0;
  for (const LatentSegment& s : segs) {
    wide += (static_cast<int64_t>(s.nrows) + 255) / 256;
    narrow += (static_cast<int64_t>(s.nrows) + 127) / 128;
    for (int64_t r = 0; r < s.nrows; r += 128) keys += s.pos0 + std::min<int64_t>(r + 128, s.nrows);
  }
  p.rows = keys * H / kCus >= 300 && wide * 100 <= narrow * 70 ? 256 : 128;
  struct Block {
    int32_t row, nrows, pos, page0, kend;
  };
  std::vector<Block> tiles;
  int64_t most_keys = 0;
  for (const LatentSegment& s : segs)
    for (int64_t r = 0; r < s.nrows; r += p.rows) {
      const int n = static_cast<int>(std::min<int64_t>(p.rows, s.nrows - r)), first = static_cast<int>(r);
      tiles.push_back(Block{s.row0 + s.qoff + first, n, s.pos0 + first, s.page0, s.pos0 + first + n});
      most_keys = std::max<int64_t>(most_keys, tiles.back().kend);
    }
  // The least range of keys, in 64s and at least 256, with which the workgroups run at once.  As
  // above it is one for all blocks, and does not even them out: of 32 heads, 1024 rows behind 6000
  // keys are 4 blocks in two parts of up to 3520 keys (217 us a call); of 1025 to 1280 rows' five
  // blocks the last ones are cut at 6528, into a long and a very short part (300 to 305).
  const int64_t split = 64 * least_split(4, (most_keys + 63) / 64, std::max<int64_t>(kCus / H, static_cast<int64_t>(tiles.size())),
                                         [&](int64_t sp) {
                                           int64_t n = 0;
                                           for (const Block& t : tiles) n += (t.kend + 64 * sp - 1) / (64 * sp);
                                           return n;
                                         });
  for (const Block& t : tiles) {
    const int c = static_cast<int>((t.kend + split - 1) / split);
    if (c > 1) p.groups.push_back(LatentGroup{t.row, t.nrows, p.n_parts, c});
    for (int i = 0; i < c; ++i)
      p.items.push_back(LatentItem{t.row, t.nrows, 0, t.pos, t.page0, static_cast<int32_t>(i * split),
                                   static_cast<int32_t>(std::min<int64_t>(t.kend, (i + 1) * split)), c > 1 ? p.n_parts + i : -1, 0});
    if (c > 1) p.n_parts += c;
  }
  std::stable_sort(p.items.begin(), p.items.end(),
                   [](const LatentItem& x, const LatentItem& y) { return x.t1 - x.t0 > y.t1 - y.t0; });
  return p;
}

// The expanded form makes every head's keys and values of all pos0 + nrows tokens, whatever
// the rows, and then has a third of the absorbed form's work a row and key.  The border in
// rows grows with what is made for the keys before them.  One sequence, absorbed / expanded, us:
//   32 heads of 128 dims, rank 512 (4.2M weights): 16 rows 22 / 19, 24 21 / 17; behind 500 keys
//   (border 35) 32 rows 33 / 30, 48 41 / 32; behind 2000 (68) 48 45 / 48, 64 47 / 50, 96 54 / 51; behind
//   4000 (112) 96 66 / 73, 130 87 / 83; behind 8000 (201) 130 129 / 136, 200 184 / 142, 260 248 / 175.
//   8 of them: behind 2000 (35) 32 29 / 31, 48 40 / 31; behind 8000 (68) 64 47 / 55, 130 54 / 61, 200 65 / 65.
//   16 heads of 64 dims, rank 256 (0.5M): behind 2000 (30) 24 29 / 24, 32 30 / 24; behind 8000 (46)
//   32 34 / 39, 48 40 / 39.  32 of them: behind 2000 (35) 24 34 / 26, 48 36 / 26.
// Near the border the form that is taken is the slower one by up to 30% in places.  And it is
// the border of one sequence: several fill the chip with fewer rows each, and the absorbed form's
// range grows.  16 sequences of the first kind, 48 rows behind 500 83 / 134, 96 behind 2000 271 / 518,
// 130 behind 4000 701 / 1076, four of 96 behind 2000 117 / 130: there the expanded form is taken.
bool latent_expands(int nrows, int pos0, int64_t weights) {
  return nrows >= 24 + static_cast<double>(pos0) * static_cast<double>(weights) / 1.9e8;
}

}  // namespace spec
