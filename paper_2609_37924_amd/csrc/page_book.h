// Bookkeeping of a page pool on the host: which rows hold which page.  No device work; the
// moves it decides on are lists that the caller turns into launches.
#pragma once
#include <stdint.h>

#include <vector>

namespace tadm {

// The pages of a batch of rows: [rows, per_row] ids, -1 where a row has none yet.
struct PageTable {
  int rows = 0, per_row = 0;
  std::vector<int32_t> id;
  PageTable() = default;
  PageTable(int rows, int per_row) : rows(rows), per_row(per_row), id((size_t)rows * per_row, -1) {}
  int32_t& at(int b, int i) { return id[(size_t)b * per_row + i]; }
  int32_t at(int b, int i) const { return id[(size_t)b * per_row + i]; }
  // whether a row has a page in [from, per_row)
  bool any(int from) const {
    for (int b = 0; b < rows; ++b)
      for (int i = from; i < per_row; ++i)
        if (at(b, i) >= 0) return true;
    return false;
  }
};

// Page dst[i] takes what page src[i] has; entry at[i] of a table becomes to[i].
struct PageMoves {
  std::vector<int32_t> src, dst, at, to;
};

struct PageBook {
  std::vector<int> refs;      // rows that hold each page
  std::vector<int32_t> free;  // ids nobody holds, the next one taken at the back

  explicit PageBook(int n) : refs(n, 0) { refill(0); }
  int size() const { return (int)refs.size(); }
  int held() const { return size() - (int)free.size(); }

  // Rows of t give back their pages [from, per_row).  Never allocates.
  void drop(PageTable& t, int from) {
    for (int b = 0; b < t.rows; ++b)
      for (int i = from; i < t.per_row; ++i) {
        const int32_t p = t.at(b, i);
        if (p >= 0 && --refs[p] == 0) free.push_back(p);
        t.at(b, i) = -1;
      }
  }

  // Row b of `to` takes a share of the pages [0, n) of row `row` of `from`.
  void share(const PageTable& from, int row, PageTable& to, int b, int n) {
    for (int i = 0; i < n; ++i) {
      to.at(b, i) = from.at(row, i);
      ++refs[to.at(b, i)];
    }
  }

  // Gives every row of t pages that it alone holds in places [first, last]: a free one where it has
  // none, a copy of a page that others hold too (the last of its holders keeps it).
  // False, and nothing has changed, when too few are free.
  bool own(PageTable& t, int first, int last, PageMoves& m) {
    const size_t most = (size_t)t.rows * (last - first + 1);
    m.src.reserve(most);
    m.dst.reserve(most);
    m.at.reserve(most);
    m.to.reserve(most);
    for (int b = 0; b < t.rows; ++b)
      for (int i = first; i <= last; ++i) {
        const int32_t p = t.at(b, i);
        if (p >= 0 && refs[p] == 1) continue;
        if (p >= 0) {
          --refs[p];
          m.src.push_back(p);
        }
        m.at.push_back((int32_t)((size_t)b * t.per_row + i));
      }
    if (m.at.size() > free.size()) {
      for (int32_t p : m.src) ++refs[p];
      return false;
    }
    for (int32_t a : m.at) {
      const int32_t p = free.back();
      free.pop_back();
      refs[p] = 1;
      if (t.id[a] >= 0) m.dst.push_back(p);
      m.to.push_back(p);
      t.id[a] = p;
    }
    return true;
  }

  // Moves the held pages at and above held() to the free ones below it; to[p] = the new id of a
  // moved page, else -1.  Tables are renumbered with renumber().
  void compact(PageMoves& m, std::vector<int32_t>& to) {
    const int n = held();
    to.assign(refs.size(), -1);
    for (int i = 0, j = n; i < n; ++i)
      if (refs[i] == 0) {
        while (refs[j] == 0) ++j;
        m.src.push_back(j);
        m.dst.push_back(i);
        to[j] = i;
        refs[i] = refs[j];
        refs[j] = 0;
      }
    refill(n);
  }
  static void renumber(PageTable& t, const std::vector<int32_t>& to, PageMoves& m) {
    m.at.clear();
    m.to.clear();
    for (size_t i = 0; i < t.id.size(); ++i)
      if (t.id[i] >= 0 && to[t.id[i]] >= 0) {
        t.id[i] = to[t.id[i]];
        m.at.push_back((int32_t)i);
        m.to.push_back(t.id[i]);
      }
  }

  // n pages in all, of which the first held() are held (after compact).
  void resize(int n) {
    const int h = held();
    refs.resize(n, 0);
    refill(h);
  }

 private:
  void refill(int from) {
    free.clear();
    free.reserve(refs.size());
    for (int i = size(); i-- > from;) free.push_back(i);
  }
};

}  // namespace tadm
