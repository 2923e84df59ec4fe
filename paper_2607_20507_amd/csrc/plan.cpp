// Attention work planning: query tiles and key-range splits.

#include <algorithm>

#include "host_util.h"

namespace spec {

namespace {

// Rows [row0, row0 + nrows) of one sequence against its keys 0 .. kend - 1.
struct Tile {
  int seq, row0, nrows, pos0, kend;
};

// Tiles of at most `qt` rows.
std::vector<Tile> tiles_of(const std::vector<AttnSegment>& segs, int qt) {
  std::vector<Tile> tiles;
  for (const auto& s : segs)
    for (int r = 0; r < s.nrows; r += qt) {
      const int n = std::min(qt, s.nrows - r);
      tiles.push_back(Tile{s.seq, s.row0 + r, n, s.pos0 + r, s.pos0 + r + n});  // keys 0 .. last row's position
    }
  return tiles;
}

// The prefill form's items, if the segments allow it.
bool plan_prefill(const std::vector<AttnSegment>& segs, int G, AttnPlan& p) {
  int min_rows = 1 << 30, max_keys = 0;
  for (const auto& s : segs) {
    min_rows = std::min(min_rows, s.nrows);
    max_keys = std::max(max_keys, s.pos0 + s.nrows);
  }
  if (segs.empty() || min_rows < kPrefillMinRows || G < 1 || 256 % G != 0 || max_keys > kPrefillMaxKeys) return false;
  p.prefill = true;
  p.few_keys = max_keys <= kPrefillShortKeys;
  for (const auto& t : tiles_of(segs, 256 / G))
    p.items.push_back(AttnItem{t.row0, t.nrows, t.pos0, t.seq, 0, t.kend, -1, 0});
  // heaviest (most keys) first, so that the long blocks start in the first
  // round of workgroups
  std::stable_sort(p.items.begin(), p.items.end(), [](const AttnItem& x, const AttnItem& y) { return x.t1 > y.t1; });
  return true;
}

// Items of at most about `split` keys (at most max_parts partials).
void cut(const std::vector<Tile>& tiles, long long split, int max_parts, AttnPlan& p) {
  auto parts_for = [&](long long sp) {
    long long n = 0;
    for (const auto& t : tiles) {
      const long long c = (t.kend + sp - 1) / sp;
      if (c > 1) n += c;
    }
    return n;
  };
  while (parts_for(split) > max_parts) split *= 2;
  for (const auto& t : tiles) {
    const int c = static_cast<int>((t.kend + split - 1) / split);
    if (c <= 1) {
      p.items.push_back(AttnItem{t.row0, t.nrows, t.pos0, t.seq, 0, t.kend, -1, 0});
      continue;
    }
    p.groups.push_back(AttnGroup{t.row0, t.nrows, p.n_parts, c});
    for (int i = 0; i < c; ++i) {
      const int t0 = static_cast<int>(i * split);
      const int t1 = static_cast<int>(std::min<long long>(t.kend, (i + 1) * split));
      p.items.push_back(AttnItem{t.row0, t.nrows, t.pos0, t.seq, t0, t1, p.n_parts + i, 0});
    }
    p.n_parts += c;
  }
  // longest key ranges first: workgroups start in this order, so the short
  // items fill in behind the long ones instead of trailing after them
  std::stable_sort(p.items.begin(), p.items.end(),
                   [](const AttnItem& x, const AttnItem& y) { return x.t1 - x.t0 > y.t1 - y.t0; });
}

}  // namespace

AttnPlan plan_attention(const std::vector<AttnSegment>& segs, int G, int Hkv, int max_parts,
                        int target_wgs, bool allow_prefill) {
  AttnPlan p;
  if (allow_prefill && plan_prefill(segs, G, p)) return p;
  int max_rows = 1, max_keys = 0;
  for (const auto& s : segs) {
    max_rows = std::max(max_rows, s.nrows);
    max_keys = std::max(max_keys, s.pos0 + s.nrows);
  }
  // query vectors per tile: rows * G <= 16 * nt, nt in {1, 2, 4}
  const int want = std::min(max_rows * G, 64);
  p.nt = want <= 16 ? 1 : (want <= 32 ? 2 : 4);
  // One sequence (a batch-1 verify, draft step or tree verify: a few MB of
  // keys and values, latency-bound): twice the items with half the query
  // vectors each, when a row's query heads still fit the narrower tile (6
  // rows x 4 heads per KV head, head dim 128: 8.6 -> 7.6 us per layer; the
  // 15-node tree verify 4.76 -> 4.44 ms; halving the tree's tiles twice was
  // no better).  Several sequences keep the wider tiles, whose items read
  // their keys and values once for all rows.
  if (segs.size() == 1 && p.nt >= 2 && G <= 8 * p.nt) p.nt /= 2;
  p.w = p.nt >= 4 ? 2 : 4;  // waves per workgroup (LDS of the merge bounds it at nt = 4)
  const int qt = std::max(1, 16 * p.nt / G);

  const std::vector<Tile> tiles = tiles_of(segs, qt);
  long long total_keys = 0;
  for (const auto& t : tiles) total_keys += t.kend;
  // key range per work item: about target_wgs workgroups over all (tile, kv
  // head) pairs, at least one 32-key chunk per wave
  long long split = (total_keys * Hkv + target_wgs - 1) / std::max(1, target_wgs);
  split = std::max<long long>(32 * p.w, (split + 31) / 32 * 32);
  // Short contexts whole: a combine is a launch of 3.5 us or more, and one
  // workgroup walks 512 keys in less.  Measured on verify forwards of 6 rows a
  // sequence (12 layers 16q / 16kv head dim 64, 16 layers 32 / 8 / 64, 4 layers
  // 32 / 8 / 128; 1, 3, 8 and 24 sequences): at up to 512 keys whole is faster
  // or equal everywhere (8 sequences of up to 500 tokens 557 -> 528 us; 24: 824 ->
  // 780, 1632 -> 1542, 1021 -> 981 us).  At 1000 it is from 64 workgroups on (8
  // sequences 1268 -> 1239 and 779 -> 763 us, 24: 1679 -> 1596 and 1043 -> 1001
  // us), but not at 8 and 24 (390 -> 406 and 1126 -> 1132 us).
  // The widest tiles (64 query vectors, two waves: a wave walks twice the keys
  // at twice the work each) gain less and lose sooner: 16 rows x 4 query heads
  // of 8 sequences over 1016 keys, head dim 128 (64 workgroups), 34 us split
  // and 55 whole, 48 vectors over 506 keys (24 workgroups) 22 and 33.  Whole is
  // faster there up to 128 keys (9 to 64 workgroups: 10% on average), 192 from
  // 64 workgroups on (25%) and 512 from 256 (25-30%).
  const long long wgs = static_cast<long long>(tiles.size()) * Hkv;
  const long long whole = p.nt < 4 ? (wgs >= 64 ? 1024 : 512) : (wgs >= 256 ? 512 : wgs >= 64 ? 192 : 128);
  if (max_keys <= whole) split = std::max<long long>(split, max_keys);
  cut(tiles, split, max_parts, p);
  return p;
}

AttnPlan plan_kv4(const std::vector<AttnSegment>& segs, int G, int Hkv, int max_parts, bool fp32) {
  AttnPlan p;
  // The prompt form at plan_prefill's border, which the bf16 attention's kernels set
  // (64 rows of every sequence).  Over a 4-bit cache (8b shape, prompt form / tiles,
  // us) it is the faster one from about 2000 rows on, 8192 rows 516 / 684, 4096 142 /
  // 194, 2048 behind 8192 keys 286 / 456, and not below, where its blocks leave CUs
  // idle and every key is expanded for few rows: 2048 rows 69 / 65, 1000 40 / 31, 512
  // 27 / 13, 64 18 / 12; behind 8192 keys 1000 rows 253 / 203, 64 rows 227 / 33.
  if (!fp32 && plan_prefill(segs, G, p)) return p;
  int max_rows = 1, max_keys = 0;
  for (const auto& s : segs) {
    max_rows = std::max(max_rows, s.nrows);
    max_keys = std::max(max_keys, s.pos0 + s.nrows);
  }
  // query tiles as above
  const int want = std::min(max_rows * G, 16 * (fp32 ? kKv4MaxNtF32 : kKv4MaxNt));
  p.nt = want <= 16 ? 1 : (want <= 32 ? 2 : 4);
  if (segs.size() == 1 && p.nt >= 2 && G <= 8 * p.nt) p.nt /= 2;
  const std::vector<Tile> tiles = tiles_of(segs, std::max(1, 16 * p.nt / G));
  long long total_keys = 0;
  for (const auto& t : tiles) total_keys += t.kend;
  const long long wgs = static_cast<long long>(tiles.size()) * Hkv;
  // Eight waves share an item's keys where every CU gets at most one workgroup
  // (one sequence of 2000 keys 16.3 -> 12.9 us, 24 of 2000 26.4 -> 24.0), four where
  // there are more (64 sequences of 1000 keys, 32 / 8 heads of 64, 23.1 -> 19.6).
  // The widest tiles and fp32 have registers for one wave a SIMD.
  p.w = !fp32 && p.nt < 4 && wgs <= 256 ? 8 : 4;
  // Whole items need no combine, and where the tables are small they are a single
  // kernel.  That is as good while the longest item's waves have at most 9 chunks
  // of 32 keys, about 1 us each, more than they would if the chip's waves shared all
  // chunks evenly.  One sequence (8b shape) of 2000 / 3000 / 4000 keys: whole 12.9 /
  // 17.0 / 21.0 us, split 17.2 / 17.6 / 18.9; 24 of 4000 35.0 and 43.5, 8 of 4000
  // 33.3 and 24.9.
  constexpr int kSlack = 9;
  const long long waves = p.nt < 4 ? 2048 : 1024;
  const long long longest = (max_keys + 32 * p.w - 1) / (32 * p.w), even = total_keys * Hkv / 32 / waves;
  long long split = max_keys;
  if (longest > even + kSlack) {
    // Workgroups that run at once: 512 (two of four waves a CU), 256 of the widest
    // tiles (16 rows of 8 sequences of 2000 keys 28.4 us, with 512 40.6).  Where a
    // batch has nearly as many before any split, only its longest sequences are
    // split (64 of 512 .. 4096 keys: 300 41.4 us, 256 43.8, 512 45.2; but 131000
    // keys of one sequence 44.4 us with 300, 35.2 with 512; in even parts instead of
    // full ones and a remainder the 64 take 2 us more).  Above the border, 300 / 512: 33
    // sequences of 512 .. 4096 keys 31.9 / 34.5, 48 36.2 / 39.3; 48 of 300 .. 8000
    // 38.9 / 37.7.  Below it uneven batches would do better with 300 too (16 of 512 ..
    // 4096 keys 26 / 36, 24 28 / 30.4).
    const int target = p.nt >= 4 ? 256 : wgs < 256 ? 512 : 300;
    p.w = 4;
    split = (total_keys * Hkv + target - 1) / target;
    split = std::max<long long>(32 * p.w, (split + 31) / 32 * 32);
  }
  cut(tiles, split, max_parts, p);
  return p;
}

}  // namespace spec
