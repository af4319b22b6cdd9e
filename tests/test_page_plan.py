"""Which entries of a plan of shared pages the blocks and the join of a call follow (CPU): page_plan.h in a C++ driver
under the address and undefined-behaviour sanitizers.

A plan that has not been laid out, or whose tables and lengths have changed, holds any words at all.  Whatever of
them is admitted has every place that follows from it inside the arrays of the call; a plan's own entries are admitted."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

DRIVER = r"""
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include "page_plan.h"
using namespace tadm;
#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

std::mt19937 rng(11);
int upto(int n) { return (int)(rng() % (unsigned)(n + 1)); }  // 0 to n

struct Call {
  PlanSizes p;
  int H;
};
Call call_of(bool f32, int B, int G, int Hkv, int L, int max_pages) {
  const Bounds w = bounds_of(f32, B, G * Hkv, Hkv, L);
  return {{f32, B, Hkv, G * L, L, max_pages, w.own_width, w.shared_width, w.own_columns, w.shared_columns}, G * Hkv};
}

// every place that a block takes from an item it follows
void places(const Item& i, const Call& c) {
  const PlanSizes& p = c.p;
  CHECK(i.width % 16 == 0 && 8 % i.teams == 0);
  const long first = (long)i.ct * i.width, last = first + i.width - 1;
  CHECK(last <= INT_MAX);
  for (int team = 0; team < i.teams; ++team) {
    const int h = i.h + team;
    CHECK(i.b >= 0 && i.b + i.rows <= p.B && h >= 0 && h < p.Hkv);
    for (long col : {first, first + i.width / 2, last}) {
      CHECK(column_of(p.ncol, p.Hkv, i.b, i.rows, h, (int)col) < (size_t)p.B * p.Hkv * p.ncol);
      if (col >= (long)i.rows * p.ncol) continue;  // no result
      const int row = i.b + (int)(col / p.ncol);
      CHECK(row >= 0 && row < p.B);                // whose tokens are looked up
      if (i.part < 0) {                            // the row's result
        CHECK(i.rows == 1 && col % p.max_n < p.max_n && (col / p.max_n) < p.ncol / p.max_n);
      } else {
        const size_t at = ((size_t)i.part + team) * (i.n ? i.width : p.shared_width) + (col - first);
        CHECK(at < (i.n ? p.own_columns : p.shared_columns));
      }
    }
  }
  for (int t : {i.t0, i.t0 + (i.t1 - i.t0) / 2, i.t1 - 1}) {
    if (t < i.t0 || t >= i.t1) continue;
    if (t < i.np)
      CHECK(t >= 0 && t < p.max_pages && (long)i.len - (long)t * PLAN_PAGE >= INT_MIN);
    else  // a tile of the window, whose arrays are whole tiles
      CHECK((long)(t - i.np) * PLAN_PAGE < i.n && i.n <= p.max_n);
  }
}

int garbled(int near) {
  switch (rng() % 8) {
    case 0: return 0;
    case 1: return INT_MAX - upto(3);
    case 2: return INT_MIN + upto(3);
    case 3: return (int)rng();
    case 4: return -1 - upto(3);
    case 5: return (int)((unsigned)near + upto(4) - 2);
    default: return near;
  }
}

// An item as a plan would lay it out.
Item sound(const Call& c) {
  const PlanSizes& p = c.p;
  const bool shared = p.B > 1 && rng() % 2;
  Item i{};
  i.rows = shared ? 2 + upto(p.B - 2) : 1;
  i.b = upto(p.B - i.rows);
  i.width = shared ? width_of(p.f32, i.rows * p.ncol) : p.own_width > 64 && rng() % 2 ? 64 : p.own_width;
  i.ct = upto(tiles_of(i.rows * p.ncol, i.width) - 1);
  i.teams = !shared && !p.f32 && i.width <= 32 ? (p.Hkv % 4 == 0 && rng() % 2 ? 4 : p.Hkv % 2 == 0 && rng() % 2 ? 2 : 1) : 1;
  i.h = upto(p.Hkv / i.teams - 1) * i.teams;
  i.n = shared ? 0 : 1 + upto(p.max_n - 1);
  i.np = upto(p.max_pages);
  i.len = shared ? i.np * PLAN_PAGE : i.np ? i.np * PLAN_PAGE - upto(PLAN_PAGE - 1) : 0;
  const int tiles = i.np + tiles_of(i.n, PLAN_PAGE);
  i.t0 = upto(tiles);
  i.t1 = i.t0 + upto(tiles - i.t0);
  const size_t room = shared ? p.shared_columns / p.shared_width : p.own_columns / i.width;
  i.part = !shared && rng() % 3 == 0 ? -1 : upto((int)(room - i.teams));
  return i;
}

long items_followed = 0, items_refused = 0, joins_followed = 0, joins_refused = 0;
void items(const Call& c) {
  for (int k = 0; k < 4000; ++k) {
    const Item good = sound(c);
    CHECK(item_fits(good, c.p));
    places(good, c);
    Item x = good;
    int32_t* words = reinterpret_cast<int32_t*>(&x);
    for (int n = 1 + upto(rng() % 3 ? 1 : 11); n > 0; --n) {
      const int at = upto(11);
      words[at] = garbled(words[at]);
    }
    if (item_fits(x, c.p)) {
      ++items_followed;
      places(x, c);
    } else {
      ++items_refused;
    }
  }
}

void joins(const Call& c) {
  const PlanSizes& p = c.p;
  for (int k = 0; k < 4000; ++k) {
    const int b = upto(p.B - 1), h = upto(p.Hkv - 1), col = upto(p.ncol - 1);
    RowParts r{b - upto(b), 1 + upto(p.B * p.ncol - 1), 1 + upto(7), upto(500), upto(7), upto(500), {0, 0}};
    int own_width = 16 << upto(3);
    int32_t* words = reinterpret_cast<int32_t*>(&r);
    for (int n = upto(3); n > 0; --n) {
      const int at = upto(5);
      words[at] = garbled(words[at]);
    }
    if (rng() % 4 == 0) own_width = garbled(own_width);
    size_t at = ~(size_t)0;
    if (shared_parts(r, p, b, h, col, at)) {
      ++joins_followed;
      CHECK(r.shared > 0 && at + (size_t)(r.shared - 1) * p.shared_width < p.shared_columns);
    } else {
      ++joins_refused;
    }
    if (own_parts(r, p, own_width, h, col, at)) {
      ++joins_followed;
      CHECK(own_width > 0 && r.own >= 0 && (r.own == 0 || at + (size_t)(r.own - 1) * own_width < p.own_columns));
    } else {
      ++joins_refused;
    }
  }
}

long wholes = 0;
// What a plan lays out: every part that the join looks up has its item.
void whole(const Call& c, int own_width, int so, int ss) {
  const PlanSizes& p = c.p;
  const int set = p.B * p.ncol, width = width_of(p.f32, set), n_shared = p.Hkv * tiles_of(set, width) * ss;
  const int units = p.Hkv * tiles_of(p.ncol, own_width);
  if (p.B * units * (so - 1) + (n_shared - n_shared / ss) > CHIP) return;  // a plan takes no more splits than these
  ++wholes;
  for (int b = 0; b < p.B; ++b) {
    const RowParts r{0, set, ss, 0, so, b * units * so, {0, 0}};
    for (int h = 0; h < p.Hkv; ++h)
      for (int col = 0; col < p.ncol; col += 1 + upto(6)) {
        size_t at;
        if (p.B > 1) {
          CHECK(shared_parts(r, p, b, h, col, at));
          const int x = b * p.ncol + col;
          CHECK(at == (size_t)((x / width * p.Hkv + h) * ss) * p.shared_width + x % width);
          CHECK((int)(at / p.shared_width) + ss <= n_shared);
        }
        CHECK(own_parts(r, p, own_width, h, col, at));
        CHECK(at == (size_t)((b * units + (col / own_width * p.Hkv + h)) * so) * own_width + col % own_width);
      }
  }
}

int main() {
  for (bool f32 : {false, true})
    for (int B : {1, 2, 5, 64, 1024})
      for (int G : {1, 2, 4})
        for (int Hkv : {1, 3, 4, 16})
          for (int L : {1, 3, 24, 64, 200}) {
            if ((long)B * G * Hkv * L > 1 << 20) continue;
            for (int mp : {1, 300, 1 << 24}) {
              const Call c = call_of(f32, B, G, Hkv, L, mp);
              items(c);
              joins(c);
            }
            const Call c = call_of(f32, B, G, Hkv, L, 40);
            whole(c, c.p.own_width, 1, 1);
            if (c.p.own_width > 64) whole(c, 64, 1, 1);
            whole(c, c.p.own_width, 2, 3);
            whole(c, c.p.own_width, 20, 30);
          }
  // by hand: places that 32 bits would wrap
  const Call c = call_of(false, 8, 4, 4, 3, 40);
  Item i{2, 1, 1, 0, 16, 0, 3, 100, 2, 3, -1, 1};
  CHECK(item_fits(i, c.p));
  auto without = [&](int Item::*f, int v) {
    Item x = i;
    x.*f = v;
    return !item_fits(x, c.p);
  };
  for (int ct : {1, 1 << 27, INT_MAX, -1, INT_MIN}) CHECK(without(&Item::ct, ct));
  for (int part : {INT_MAX, INT_MAX - 1, 1 << 30}) CHECK(without(&Item::part, part));
  for (int teams : {0, 3, 5, 8, -1, INT_MIN}) CHECK(without(&Item::teams, teams));
  for (int width : {0, 17, 32, 48, 256, INT_MIN}) CHECK(without(&Item::width, width));
  for (int rows : {0, 2, 7, INT_MAX, INT_MIN}) CHECK(without(&Item::rows, rows));
  for (int len : {-1, 129, INT_MIN, INT_MAX}) CHECK(without(&Item::len, len));
  for (int t1 : {-1, 4, INT_MAX}) CHECK(without(&Item::t1, t1));
  RowParts r{0, 8 * 12, 2, 0, 2, 0, {0, 0}};
  size_t at;
  CHECK(shared_parts(r, c.p, 3, 1, 5, at) && own_parts(r, c.p, 16, 1, 5, at));
  for (int lead : {4, -1, INT_MIN, INT_MAX}) CHECK((r.lead = lead, !shared_parts(r, c.p, 3, 1, 5, at)));
  r.lead = 0;
  for (int own : {INT_MAX, INT_MAX / 2, -1}) CHECK((r.own = own, !own_parts(r, c.p, 16, 1, 5, at)));
  r.own = 2;
  for (int at_own : {INT_MAX, INT_MAX - 1, -1}) CHECK((r.at_own = at_own, !own_parts(r, c.p, 16, 1, 5, at)));
  CHECK(items_followed > 10000 && items_refused > 10000 && joins_followed > 10000 && joins_refused > 10000 && wholes > 300);
  std::printf("ok %ld %ld %ld %ld %ld\n", wholes, items_followed, items_refused, joins_followed, joins_refused);
}
"""


def test_what_is_followed_stays_in_the_arrays(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2609_37924_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120,
                       env={k: v for k, v in os.environ.items() if k != "LD_PRELOAD"})
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.startswith("ok")
