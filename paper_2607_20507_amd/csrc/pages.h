// Host page allocator of the paged KV cache.  Pure C++ (no HIP) so that it can
// be tested on a machine without a GPU.
//
// Page indices are a deterministic function of the history of lengths:
// allocation always takes the lowest-numbered free page, and a page returns
// to the pool as soon as no table holds it: with no sharing, as soon as it holds
// no position below its sequence's length.  Several tables may hold a page
// (share); whoever writes to one must hold it alone.
#pragma once

#include <algorithm>
#include <cstdint>
#include <functional>
#include <queue>
#include <utility>
#include <vector>

namespace spec {

class PagePool {
 public:
  explicit PagePool(int num_pages = 0, int page_size = 16) { reset(num_pages, page_size); }

  void reset(int num_pages, int page_size) {
    page_size_ = page_size;
    num_pages_ = num_pages;
    free_ = decltype(free_)();
    for (int p = 0; p < num_pages; ++p) free_.push(p);
    holders_.assign(num_pages, 0);
  }

  int page_size() const { return page_size_; }
  int num_pages() const { return num_pages_; }
  int free_pages() const { return static_cast<int>(free_.size()); }
  int pages_for(int64_t length) const {
    return static_cast<int>((length + page_size_ - 1) / page_size_);
  }
  // pages a table must gain to cover positions 0..length-1
  int need(const std::vector<int32_t>& table, int64_t length) const {
    const int n = pages_for(length) - static_cast<int>(table.size());
    return n > 0 ? n : 0;
  }
  // Extend `table` to cover 0..length-1; false (nothing changed) if the pool is short.
  bool ensure(std::vector<int32_t>& table, int64_t length) {
    const int n = need(table, length);
    if (n > free_pages()) return false;
    for (int i = 0; i < n; ++i) table.push_back(take());
    return true;
  }
  // Give up pages holding no position below `length`.
  void truncate(std::vector<int32_t>& table, int64_t length) {
    const int keep = pages_for(length);
    while (static_cast<int>(table.size()) > keep) {
      drop(table.back());
      table.pop_back();
    }
  }
  // The lowest-numbered free page (there is one), held once.
  int32_t take() {
    const int32_t p = free_.top();
    free_.pop();
    holders_[p] = 1;
    return p;
  }
  // Hold the first n pages of `from` in `to` (empty) too (no allocation if `to` has
  // room for them).
  void share(const std::vector<int32_t>& from, int n, std::vector<int32_t>& to) {
    to.assign(from.begin(), from.begin() + n);
    for (int32_t p : to) ++holders_[p];
  }
  bool shared(int32_t page) const { return holders_[page] > 1; }
  // One holder less; the page is free with the last.
  void drop(int32_t page) {
    if (--holders_[page] == 0) free_.push(page);
  }
  // Pages that truncate(table, length) would free.
  int freed_by(const std::vector<int32_t>& table, int64_t length) const {
    int n = 0;
    for (size_t i = pages_for(length); i < table.size(); ++i) n += holders_[table[i]] == 1;
    return n;
  }
  // A table cut to `keep` of its `end` positions.  The page that keep ends in is
  // written next: held by another table too, it is replaced by a copy.
  struct Cut {
    int32_t from = -1, to = -1;  // the page to copy and its copy (-1: none)
    std::vector<int32_t> clear;  // slots from keep on that no other table holds, those of the copy among them
  };
  bool can_cut(const std::vector<int32_t>& table, int64_t keep) const {
    return keep % page_size_ == 0 || !shared(table[keep / page_size_]) || free_pages() + freed_by(table, keep) > 0;
  }
  Cut cut(std::vector<int32_t>& table, int64_t keep, int64_t end) {
    Cut c;
    const int64_t last = keep / page_size_;
    const bool copied = keep % page_size_ != 0 && shared(table[last]);
    for (int64_t p = keep; p < end; ++p)
      if (!shared(table[p / page_size_])) c.clear.push_back(slot(table, p));
    truncate(table, keep);
    if (copied) {
      c.from = table[last];
      c.to = take();
      table[last] = c.to;
      drop(c.from);
      // (a page that this cut freed may come back as the copy: not to be cleared as such)
      c.clear.erase(std::remove_if(c.clear.begin(), c.clear.end(), [&](int32_t s) { return s / page_size_ == c.to; }),
                    c.clear.end());
      for (int64_t p = keep; p < std::min(end, page_size_ * (last + 1)); ++p) c.clear.push_back(slot(table, p));
    }
    return c;
  }
  // Renumber the held pages to 0 .. live - 1, moving as few as possible: the held
  // pages from `live` on, ascending, to the free ones below it, ascending.  Returns
  // the (from, to) pairs; the caller moves the contents and renames its tables.
  std::vector<std::pair<int32_t, int32_t>> compact() {
    const int live = num_pages_ - free_pages();
    std::vector<std::pair<int32_t, int32_t>> moves;
    int to = 0;
    for (int from = live; from < num_pages_; ++from) {
      if (holders_[from] == 0) continue;
      while (holders_[to] != 0) ++to;
      moves.emplace_back(from, to++);
    }
    std::vector<int32_t> left;
    left.reserve(num_pages_);  // (pages are given up without an allocation)
    for (int p = live; p < num_pages_; ++p) left.push_back(p);
    for (const auto& m : moves) std::swap(holders_[m.first], holders_[m.second]);
    free_ = decltype(free_)(std::greater<int32_t>(), std::move(left));
    return moves;
  }
  int32_t slot(const std::vector<int32_t>& table, int64_t pos) const {
    return table[pos / page_size_] * page_size_ + static_cast<int32_t>(pos % page_size_);
  }

 private:
  int page_size_ = 16;
  int num_pages_ = 0;
  std::vector<int32_t> holders_;  // tables that hold a page
  std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_;
};

}  // namespace spec
