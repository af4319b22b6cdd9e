// The plan of attention over shared pages: its layout, the room that it and its parts take, and which of its
// entries the blocks and the join of a call may follow.  No device work; the functions serve host and device.
//
// A plan lies in the caller's memory, and is of the tables and lengths that it was made from.  Where these have changed, or
// where it has not been laid out yet, what it holds is any words at all: item_fits, shared_parts and own_parts admit
// only those whose every access lies in the arrays of the call.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace tadm {

constexpr int PLAN_PAGE = 64;  // positions of a page

// Columns of a block by the columns of a set; 16 in float32.
constexpr int width_of(bool f32, int columns) {
  return f32 || columns <= 16 ? 16 : columns <= 32 ? 32 : columns <= 64 ? 64 : 128;
}
constexpr int tiles_of(int columns, int width) { return (columns + width - 1) / width; }

// One item of a plan.
struct Item {
  int b, rows;         // the row whose pages are read; rows whose columns are in the set
  int h, ct, width;    // K/V head, tile of columns
  int t0, t1;          // key tiles: pages, behind the last of them the window's
  int len, np, n;      // positions on pages and their tiles; the row's window (0 on shared pages)
  int part;            // the first of its units' parts, -1: it writes the result
  int teams;           // K/V heads h, h + 1, ... that the block's waves share out (few columns, short rows)
};
// What a row's columns are joined from: the group's items with h and ct 0, then the row's own.
struct RowParts {
  int lead, columns;      // first row of the group, columns of its set; no shared part: lead is the row
  int shared, at_shared;  // splits of the shared pages, and the part of their first unit
  int own, at_own;        // splits of its own keys, ...; own < 0: one, which has written the result
  int pad[2];
};
constexpr int PLAN_HEAD = 64;  // bytes before the rows; the first words are the number of items and the columns of a row's own

// Sizes of a plan and of what its items write, from what the host knows.
struct Bounds {
  int own_width, shared_width;      // the most columns of a block on a row's own keys, and on shared pages
  long own_items, shared_items;
  size_t own_columns, shared_columns;  // columns of their parts
};
constexpr int CHIP = 256;  // blocks that run at once: one a CU
constexpr Bounds bounds_of(bool f32, int B, int H, int Hkv, int L) {
  const int ncol = H / Hkv * L;
  Bounds r{};
  r.own_width = width_of(f32, ncol);
  r.shared_width = width_of(f32, B * ncol < 128 ? B * ncol : 128);
  // Splits add at most one item a CU.  The plan takes 64 or 128 columns where a row has more than 64.
  const long rows = (long)B * Hkv;
  r.own_items = rows * tiles_of(ncol, r.own_width > 64 ? 64 : r.own_width) + CHIP;
  r.own_columns = (size_t)(rows * tiles_of(ncol, r.own_width) + CHIP) * r.own_width;
  // groups have two rows or more, and each set at most one tile more than its columns fill
  r.shared_items = B < 2 ? 0 : (long)Hkv * (tiles_of(B * ncol, f32 ? 16 : 128) + B / 2) + CHIP;
  r.shared_columns = (size_t)r.shared_items * r.shared_width;
  return r;
}

// Sizes of a call.
struct PlanSizes {
  bool f32;
  int B, Hkv, ncol, max_n, max_pages;  // ncol: columns of a row, B ncol below 2^27
  int own_width, shared_width;         // as in Bounds
  size_t own_columns, shared_columns;
};

// Every block of a call asks this first, so it has no branches, and sums and products of 64 bits instead of their limits'
// differences and quotients: as a chain of returns, each behind a load, a layer took 0.4 to 1.5 us longer.
constexpr uint64_t word(int x) { return (uint32_t)x; }  // negative: more than any size here
constexpr bool item_fits(const Item& i, const PlanSizes& p) {
  const bool own = i.n != 0, few = own & (i.width <= 32) & !p.f32;
  const uint64_t width = word(i.width), rows = word(i.rows), teams = word(i.teams), b = word(i.b), h = word(i.h), ct = word(i.ct),
                 t0 = word(i.t0), t1 = word(i.t1), len = word(i.len), np = word(i.np), n = word(i.n);
  const uint64_t B = p.B, Hkv = p.Hkv, ncol = p.ncol, max_n = p.max_n, max_pages = p.max_pages;
  const uint64_t most_rows = own ? 1 : B, most_width = own ? p.own_width : p.shared_width;
  const uint64_t end = (word(i.part) + teams) * (own ? width : most_width), room = own ? p.own_columns : p.shared_columns;
  bool ok = (rows >= 1) & (rows <= most_rows) & (b + rows <= B);
  ok &= (width >= 16) & (width <= most_width) & ((width & (width - 1)) == 0) & (ct * width < rows * ncol);
  ok &= (teams == 1) | (few & ((teams == 2) | (teams == 4)));
  ok &= (h + teams <= Hkv) & (n <= max_n) & (np <= max_pages) & (len <= np * PLAN_PAGE);
  ok &= (t0 <= t1) & (t1 <= np + (n + PLAN_PAGE - 1) / PLAN_PAGE);
  return ok & (i.part < 0 ? own : end <= room);
}

// The place among all columns of column col of K/V head h in a set of `rows` rows from b on (of the last one, behind it).
constexpr size_t column_of(int ncol, int Hkv, int b, int rows, int h, int col) {
  const int c = col < rows * ncol ? col : rows * ncol - 1;
  return rows == 1 ? ((size_t)b * Hkv + h) * ncol + c : ((size_t)(b + c / ncol) * Hkv + h) * ncol + c % ncol;
}

// The first of the parts that column c of row b and head h is joined from, in columns: on shared pages, r.shared of them,
// shared_width apart; of its own keys, r.own of them, own_width apart (the plan's).  Widths are powers of two; columns fewer
// than 2^40.
constexpr bool room_for(uint64_t parts, int width, uint64_t columns) { return (parts <= columns) & (parts * width <= columns); }
constexpr bool shared_parts(const RowParts& r, const PlanSizes& p, int b, int h, int c, size_t& at) {
  const uint64_t columns = word(r.columns), all = (uint64_t)p.B * p.ncol;
  const bool ok = (r.shared >= 1) & (r.at_shared >= 0) & (r.lead >= 0) & (r.lead <= b) & (columns >= 1) & (columns <= all);
  const uint32_t col = (uint32_t)(b - (ok ? r.lead : b)) * p.ncol + c, shift = __builtin_ctz(width_of(p.f32, r.columns));
  const uint64_t first = word(r.at_shared) + ((uint64_t)(col >> shift) * p.Hkv + h) * word(r.shared);
  at = first * p.shared_width + (col & ((1u << shift) - 1));
  const bool room = room_for(first + word(r.shared), p.shared_width, p.shared_columns);
  return ok & room;
}
constexpr bool own_parts(const RowParts& r, const PlanSizes& p, int own_width, int h, int c, size_t& at) {
  const uint64_t width = word(own_width), most = p.own_width;
  const bool ok = (r.own >= 0) & (r.at_own >= 0) & (width >= 16) & (width <= most) & ((width & (width - 1)) == 0);
  const uint32_t shift = ok ? __builtin_ctz(own_width) : 4;
  const uint64_t first = word(r.at_own) + ((uint64_t)((uint32_t)c >> shift) * p.Hkv + h) * word(r.own);
  at = (first << shift) + ((uint32_t)c & ((1u << shift) - 1));
  const bool room = room_for(first + word(r.own), 1 << shift, p.own_columns);
  return ok & room;
}

}  // namespace tadm
