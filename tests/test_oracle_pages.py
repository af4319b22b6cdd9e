"""Pins of the 8-bit page oracle, and the pool's bookkeeping (CPU).

The e4m3 conversion against torch's, the scale rule against its definition, append against
quantising whole pages; the bookkeeping of page_book.h in a C++ driver under the address and
undefined-behaviour sanitizers."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import pages as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_codes_equal_torch():
    c = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(c).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(P.decode(c)), np.isnan(ref))
    ok = ~np.isnan(ref)
    assert np.array_equal(P.decode(c)[ok], ref[ok])


def test_rounding_equals_torch():
    """Every midpoint of neighbouring values, its float32 neighbours, and random values."""
    mid = (P.POSITIVE[1:] + P.POSITIVE[:-1]) / 2
    x = np.concatenate([mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 1e9),
                        P.POSITIVE, np.random.default_rng(0).normal(size=4000) * 60]).astype(np.float32)
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 448]
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(P.encode(x), ref)
    assert np.all(P.encode(np.array([np.inf, -np.inf, np.nan])) == 0x7f)


@pytest.mark.parametrize("e", [-12, -1, 0, 5])
def test_scale_is_the_least_that_holds_the_largest(e):
    top = 448.0 * 2.0 ** e
    assert P.scale_of([0.1 * top, -top]) == 2.0 ** e
    assert P.scale_of([np.nextafter(np.float32(top), np.float32(1e30))]) == 2.0 ** (e + 1)
    assert P.scale_of([np.inf, np.nan, top]) == 2.0 ** e
    assert P.scale_of([]) == P.scale_of([0.0]) == 2.0 ** P.E_MIN


def test_append_in_pieces_equals_whole_pages():
    """A power-of-two scale that grows keeps the codes that stay normal: appending a row in pieces gives what
    quantising the page at once gives, but for values that a page's scale makes subnormal."""
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(2, 2, 150, 8)) + 3.0 * np.sign(rng.normal(size=(2, 2, 150, 8)))  # no tiny values
    one = P.Pages(np.zeros((4, 1, 2, 2, 64 * 8), np.uint8), np.ones((4, 1, 2, 2)))
    two = P.Pages(np.zeros((4, 1, 2, 2, 64 * 8), np.uint8), np.ones((4, 1, 2, 2)))
    one.append(0, [2, 0, 3], 0, k, v)
    at = 0
    for n in (1, 62, 2, 64, 21):
        two.append(0, [2, 0, 3], at, k[:, at:at + n], v[:, at:at + n])
        at += n
    assert np.array_equal(one.codes, two.codes) and np.array_equal(one.scales, two.scales)
    rk, rv, there = one.read(0, [2, 0, 3], 150)
    assert there.all()
    assert np.all(np.abs(rk - k) <= 2.0 ** -4 * np.abs(k)) and np.all(np.abs(rv - v) <= 2.0 ** -4 * np.abs(v))
    assert np.all(one.codes[1] == 0)


def test_attention_equals_torch():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(4, 5, 16)), rng.normal(size=(2, 9, 16)), rng.normal(size=(2, 9, 16))
    o, lse = P.attend(q, k, v)
    kk, vv = (torch.from_numpy(np.repeat(x, 2, axis=0)) for x in (k, v))
    s = torch.from_numpy(q) @ kk.transpose(1, 2) / 4.0
    assert np.allclose(o, (torch.softmax(s, -1) @ vv).permute(1, 0, 2).numpy(), atol=1e-12)
    assert np.allclose(lse, torch.logsumexp(s, -1).numpy(), atol=1e-12)
    o, lse = P.attend(q, k[:, :0], v[:, :0])
    assert np.all(o == 0) and np.all(np.isneginf(lse))


DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "page_book.h"
using namespace tadm;
#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

// what a page holds, as the moves say it: (row history, place); own() copies it, compact() moves it
struct World {
  PageBook book{40};
  std::vector<long> content = std::vector<long>(40, -1);
  struct Ctx { PageTable t; int held; std::vector<long> want; };
  std::vector<Ctx> ctx;
  void apply(const PageMoves& m) {
    for (size_t i = 0; i < m.src.size(); ++i) content[m.dst[i]] = content[m.src[i]];
  }
  void verify() {
    std::vector<int> refs(book.size(), 0);
    for (auto& c : ctx)
      for (int b = 0; b < c.t.rows; ++b)
        for (int i = 0; i < c.t.per_row; ++i) {
          const int p = c.t.at(b, i);
          if (p < 0) continue;
          CHECK(p < book.size());
          ++refs[p];
          if (i < c.held) CHECK(content[p] == c.want[(size_t)b * c.t.per_row + i]);
        }
    CHECK(refs == book.refs);
    std::vector<char> isfree(book.size(), 0);
    for (int p : book.free) { CHECK(refs[p] == 0 && !isfree[p]); isfree[p] = 1; }
    for (int p = 0; p < book.size(); ++p) CHECK((refs[p] == 0) == (bool)isfree[p]);
  }
};

int main() {
  std::mt19937 rng(7);
  World w;
  long stamp = 0;
  int full = 0, copied = 0, moved = 0;
  for (int step = 0; step < 20000; ++step) {
    const int what = rng() % 6;
    if (what == 0 && w.ctx.size() < 5) {
      const int rows = 1 + rng() % 3;
      w.ctx.push_back({PageTable(rows, 6), 0, std::vector<long>(rows * 6, -1)});
    } else if (w.ctx.empty()) {
      continue;
    } else if (what == 1) {  // append: the last page again or new ones
      auto& c = w.ctx[rng() % w.ctx.size()];
      const int first = c.held - (c.held && rng() % 2 ? 1 : 0), last = first + rng() % 3;
      if (last >= c.t.per_row) continue;
      PageMoves m;
      const auto refs = w.book.refs;
      const auto ids = c.t.id;
      const auto nfree = w.book.free.size();
      if (!w.book.own(c.t, first, last, m)) {
        CHECK(refs == w.book.refs && ids == c.t.id && nfree == w.book.free.size());
        ++full;
      } else {
        CHECK(m.src.size() == m.dst.size() && m.at.size() == m.to.size());
        copied += (int)m.src.size();
        w.apply(m);
        for (int b = 0; b < c.t.rows; ++b)
          for (int i = first; i <= last; ++i) {
            CHECK(w.book.refs[c.t.at(b, i)] == 1);
            if (i < c.held) CHECK(w.content[c.t.at(b, i)] == c.want[(size_t)b * c.t.per_row + i]);
            w.content[c.t.at(b, i)] = c.want[(size_t)b * c.t.per_row + i] = ++stamp;
          }
        c.held = last + 1;
      }
    } else if (what == 2) {  // truncate
      auto& c = w.ctx[rng() % w.ctx.size()];
      c.held = rng() % (c.held + 1);
      w.book.drop(c.t, c.held);
    } else if (what == 3 && w.ctx.size() < 5) {  // fork
      const size_t s = rng() % w.ctx.size();
      const int rows = 1 + rng() % 3;
      World::Ctx n{PageTable(rows, 6), w.ctx[s].held, std::vector<long>(rows * 6, -1)};
      for (int b = 0; b < rows; ++b) {
        const int from = rng() % w.ctx[s].t.rows;
        w.book.share(w.ctx[s].t, from, n.t, b, n.held);
        for (int i = 0; i < 6; ++i) n.want[b * 6 + i] = w.ctx[s].want[from * 6 + i];
      }
      // places behind held are not shared: own() gives them new pages
      w.ctx.push_back(n);
    } else if (what == 4 && rng() % 3 == 0) {  // destroy
      const size_t i = rng() % w.ctx.size();
      w.book.drop(w.ctx[i].t, 0);
      w.ctx.erase(w.ctx.begin() + i);
    } else if (what == 5) {  // compact, now and then with another size
      PageMoves m;
      std::vector<int32_t> to;
      w.book.compact(m, to);
      moved += (int)m.src.size();
      for (size_t i = 0; i < m.src.size(); ++i) {
        CHECK(m.src[i] >= w.book.held() && m.dst[i] < w.book.held());
        w.content[m.dst[i]] = w.content[m.src[i]];
      }
      for (auto& c : w.ctx) {
        const auto before = c.t.id;
        PageBook::renumber(c.t, to, m);
        auto device = before;
        for (size_t i = 0; i < m.at.size(); ++i) device[m.at[i]] = m.to[i];
        CHECK(device == c.t.id);
      }
      for (int p = 0; p < w.book.size(); ++p) CHECK((w.book.refs[p] > 0) == (p < w.book.held()));
      if (rng() % 2) {
        const int n = w.book.held() + 1 + rng() % 40;
        w.book.resize(n);
        w.content.resize(n, -1);
      }
    }
    w.verify();
  }
  CHECK(full > 50 && copied > 50 && moved > 50);
  std::printf("ok full %d copied %d moved %d\n", full, copied, moved);
}
"""


def test_bookkeeping_of_shared_pages(tmp_path):
    src, exe = tmp_path / "book.cpp", tmp_path / "book"
    src.write_text(DRIVER)
    inc = os.path.join(ROOT, "paper_2609_37924_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", inc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120,
                       env={k: v for k, v in os.environ.items() if k != "LD_PRELOAD"})
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.startswith("ok")
