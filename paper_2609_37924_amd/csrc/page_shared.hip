// Attention over the paged 8-bit K/V store for rows that share their leading pages.
//
// Rows that continue one prompt name the same pages for it.  With K, V of a row cut into the shared positions and
// its own, the softmax over both is joined from the two parts: each has its maximum m_i, its sum l_i of
// 2^(s - m_i) and the unnormalised O_i; m = max m_i, l = sum l_i 2^(m_i - m), O = sum O_i 2^(m_i - m) / l.  The shared
// part is attention with the columns (queries of the heads that share a K/V head) of every row of the group in one
// set, so that its pages are read once for all of them, and by the kernels for many columns.
//
// What the blocks do follows from the tables and lengths, which are on the device: a plan, laid out by one
// block before the layers of a pass, lists the items (a tile of columns, a K/V head, a run of key tiles) that the
// blocks of each layer's launch take, their tiles balanced over the chip.  A second launch joins
// the parts of each column in the order of their keys.
//
// Sharing saves bytes, and the tiles of blocks that a row's columns do not fill; where they do, a plan shares nothing, and what it
// adds is the join.  us a layer on one MI355X, each row by itself and by a plan:
// 64 rows x 1 token over 8 192 shared and up to 512 other positions, 32/16 heads x 128: 204 and 46; 16 rows: 55 and 25; 32
// rows of four prompts: 104 and 41; 32 rows of two over 4 096, 16 heads x 128: 61 and 29, 12 heads x 64: 24 and 15; 16 x 16 over 8 192,
// 32/16 heads: 64 and 65.  Nothing shared: 8 x 1 over 1 000, 12 heads x 64: 7.7 and 9.8; 16 x 64 over 1 024, 16/4 heads x
// 128: 25.5 and 28.1, over 4 096 64 and 59 (58 and 56 with pages of each row's own, so no gain of sharing).
#include "page_plan.h"
#include "page_tiles.h"

namespace tadm {
namespace {

static_assert(PLAN_PAGE == PAGE, "positions of a page");

struct PlanArgs {
  PageRows r;
  DType dt;
  int Hkv, ncol, dh, min_pages;
  int own_items, shared_items;  // room for
  int own_width;
  int32_t* plan;
  int32_t *lead, *pages;  // nullable
};

// What a block needs for a tile and for everything around its tiles, in 0.1 us, as measured with every CU at work: the slope
// and the rest of times over prompts of 1 024 to 8 192 positions (16 rows x 64 tokens, 16/4 heads x 128; 8 x 128, 12 x 64).
// With few columns a tile's bytes come at a CU's share of HBM, or from an L2 where rows read the same pages.
struct Cost {
  float tile, again, item;  // again: of a tile that other rows read too
  int least;                // tiles of a split at least
};
__device__ __forceinline__ Cost cost_of(DType dt, int dh, int width) {
  if (dt == F32) return Cost{4.f, 4.f, 20.f, 4};
  if (width > 64) return dh > 64 ? Cost{10.f, 10.f, 110.f, 4} : Cost{5.f, 5.f, 85.f, 4};
  if (width > 32) return dh > 64 ? Cost{8.9f, 8.9f, 45.f, 4} : Cost{3.5f, 3.5f, 40.f, 4};
  return dh > 64 ? Cost{8.f, 4.2f, 30.f, 2} : Cost{4.f, 2.1f, 30.f, 4};
}
// Of the join, where there are parts.  With 60 or 80, 8 rows x 1 token over 2 048 shared positions (32/16 heads x 128) are taken one by
// one, 17.8 us instead of 11.3; of 26 other calls none chose otherwise.
constexpr float JOIN = 40.f;
// Splits of a unit's tiles that a budget of time for a block's tiles asks for.
__device__ __forceinline__ int splits_of(int tiles, const Cost& c, float budget) {
  return max(1, min((int)ceilf(tiles * c.tile / budget), tiles / c.least));
}

// The threads that plan, one a row: a wave, which needs no barriers, or a block.
template <int N>
struct Team {
  float* red;
  __device__ __forceinline__ void sync() const {
    if constexpr (N > 64)
      __syncthreads();
    else
      __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  }
  template <bool MAX>
  __device__ __forceinline__ float over(float v) const {
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (N > 64) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = red[0];
      for (int w = 1; w < N / 64; ++w) v = MAX ? fmaxf(v, red[w]) : v + red[w];
    }
    return v;
  }
  __device__ __forceinline__ float sum(float v) const { return over<false>(v); }
  __device__ __forceinline__ float max(float v) const { return over<true>(v); }
  // sum over the threads before this one, and over all
  __device__ __forceinline__ int scan(int v, int& all) const {
    int upto = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int t = __shfl_up(upto, o, 64);
      if ((int)(threadIdx.x & 63) >= o) upto += t;
    }
    all = __builtin_amdgcn_readlane(upto, 63);
    if constexpr (N > 64) {
      int* r = reinterpret_cast<int*>(red);
      const int wave = threadIdx.x >> 6;
      __syncthreads();
      if ((threadIdx.x & 63) == 63) r[wave] = upto;
      __syncthreads();
      all = 0;
      for (int w = 0; w < N / 64; ++w) {
        if (w < wave) upto += r[w];
        all += r[w];
      }
    }
    return upto - v;
  }
};

struct PlanRow {  // of a row; of a group in its first row's place
  int len, n, common, lead, rows, set, shared, set_units, own, shared_splits, at_shared, own_splits, at_own;
};

// A way to cut the work of the rows (one a thread of the team) into items, and its time: the longest's where each has a CU
// of its own, else the larger of the work's share a CU (and half of a shortest item, which come last) and of the rounds
// that the longer items need; the shorter ones fill the gaps.
struct Choice {
  int width, teams, units, own_splits, shared_splits;
  float time;
};
constexpr int SPLITS = 12;  // 1, 2, 3, 4, 6, 8, 12, ... 64 splits of the longest unit
template <int N>
__device__ __forceinline__ Choice choice_of(const Team<N>& team, const PlanArgs& a, const PlanRow& r, int width, int j) {
  Choice c{width, 1, r.n > 0 ? a.Hkv * tiles_of(a.ncol, width) : 0, 0, 0, 0.f};
  const Cost co = cost_of(a.dt, a.dh, width), cs = cost_of(a.dt, a.dh, width_of(a.dt == F32, r.set));
  // few columns and more rows than blocks: the waves of a block share out several heads, so that each has several tiles
  const float units = team.sum((float)c.units);
  if (a.dt == BF16 && width <= 32)
    c.teams = units >= 4 * CHIP && a.Hkv % 4 == 0 ? 4 : units >= 2 * CHIP && a.Hkv % 2 == 0 ? 2 : 1;
  const float own_cost = r.own * co.tile * c.teams, shared_cost = r.shared * cs.tile, blocks = (float)(c.units / c.teams);
  const float longest = fmaxf(team.max(fmaxf(c.units ? own_cost : 0.f, r.set_units ? shared_cost : 0.f)), 1.f);
  const float budget = longest / (j < 2 ? j + 1 : j & 1 ? 1 << (j + 1) / 2 : 3 << (j - 2) / 2);
  const int o = c.teams > 1 ? 1 : splits_of(r.own, co, budget), s = splits_of(r.shared, cs, budget);
  const float to = own_cost / o + co.item, ts = shared_cost / s + cs.item;
  const float more = team.sum((float)c.units * (o - 1) + (float)r.set_units * (s - 1));
  const float work = team.sum(blocks * o * to + r.set_units * s * ts);
  const float top = team.max(fmaxf(c.units ? to : 0.f, r.set_units ? ts : 0.f));
  const float large = team.sum((to > 0.5f * top ? blocks * o : 0.f) + (ts > 0.5f * top ? r.set_units * s : 0.f));
  const float items = team.sum(blocks * o + r.set_units * s);
  const float least = -team.max(-fminf(c.units ? to : INFINITY, r.set_units ? ts : INFINITY));
  const bool joins = team.max(r.set_units || (c.units && o > 1) ? 1.f : 0.f) > 0.f;
  c.own_splits = c.units ? o : 0;
  c.shared_splits = r.set_units ? s : 0;
  // no more items than one a CU beside the units: there is room for no more
  const float rounds = ceilf(large / CHIP) * top;
  c.time = more > CHIP ? INFINITY : (items > CHIP ? fmaxf(work / CHIP + 0.5f * least, rounds) : top) + (joins ? JOIN : 0.f);
  return c;
}

// One block; ROWS threads (at least the rows) plan.  Bound by steps behind one another, loads first:
// 7.6 us a call in the smallest of the measured cases, 12.8 for 64 rows of up to 136 pages.  Planned by 1 024 threads for
// every number of rows, with barriers in every step, 16 to 22.
template <int ROWS>
__global__ __launch_bounds__(1024) void plan_kernel(PlanArgs a) {
  constexpr int THREADS = 1024;
  __shared__ PlanRow row[ROWS];
  __shared__ float red[THREADS / 64];
  __shared__ int s_alive, s_shared_items, s_own_items, s_teams, s_own_width;
  const int tid = threadIdx.x, B = a.r.B;
  if (tid < ROWS) {
    row[tid].len = tid < B ? row_len(a.r, tid) : 0;
    row[tid].n = tid < B ? row_new(a.r, tid) : 0;
  }
  if (tid == 0) s_alive = 0;
  __syncthreads();
  // whole pages that each row and the one before it could share, and those that they do: pages [p0, p0 + width) of
  // all rows at once, until no two share any further
  int most = 0;
  if (tid < ROWS) {
    most = tid > 0 && tid < B ? min(row[tid].len, row[tid - 1].len) / PAGE : 0;
    row[tid].common = most;
    if (most) atomicMax(&s_alive, most);
  }
  __syncthreads();
  constexpr int AHEAD = 8;
  int bits = 6;
  while ((1 << bits) < s_alive && (B << bits) < 2 * AHEAD * THREADS) ++bits;
  __syncthreads();
  for (int p0 = 0; p0 < s_alive;) {
    for (int i0 = tid; i0 < (B - 1) << bits; i0 += AHEAD * THREADS) {
      int x[AHEAD], y[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * THREADS, b = 1 + (i >> bits), p = p0 + (i & ((1 << bits) - 1));
        x[u] = y[u] = 0;
        if (b < B && p < row[b].common) {
          const int32_t* t = a.r.table + (size_t)b * a.r.max_pages + p;
          x[u] = t[0];
          y[u] = t[-(long)a.r.max_pages];
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int i = i0 + u * THREADS;
        if (x[u] != y[u]) atomicMin(&row[1 + (i >> bits)].common, p0 + (i & ((1 << bits) - 1)));
      }
    }
    __syncthreads();
    p0 += 1 << bits;
    if (tid == 0) s_alive = 0;
    __syncthreads();
    if (tid < ROWS && most > p0 && row[tid].common == most) atomicMax(&s_alive, most);
    __syncthreads();
  }

  if (tid < ROWS) {
    const Team<ROWS> team{red};
    const int b = tid;
    const bool mine = b < B;
    const int len = row[b].len, n = row[b].n;
    // groups: runs of rows that share min_pages pages or more with the row before
    const int common = mine && row[b].common >= a.min_pages ? row[b].common : 0;
    row[b].lead = common ? 0 : b;
    row[b].shared = 1 << 30;
    row[b].rows = 0;
    team.sync();
    for (int o = 1; o < ROWS && o < B; o <<= 1) {  // the last row at or before this one that begins a group
      const int v = b >= o ? max(row[b].lead, row[b - o].lead) : row[b].lead;
      team.sync();
      row[b].lead = v;
      team.sync();
    }
    const int lead = row[b].lead;
    if (mine) atomicAdd(&row[lead].rows, 1);
    if (common) atomicMin(&row[lead].shared, common);
    team.sync();
    const int rows = row[lead].rows, found = mine && rows > 1 ? row[lead].shared : 0;
    if (mine && a.lead) a.lead[b] = lead;
    if (mine && a.pages) a.pages[b] = found;

    // Units (K/V head x tile of columns): the row's, and those of its group.  A group's together where that takes less than
    // its rows apart, which it does not once a row's columns fill the tiles of a block, and all groups if the work of
    // the whole call gets less by more than a join.
    const int set = rows * a.ncol, set_width = width_of(a.dt == F32, set);
    const Cost cs = cost_of(a.dt, a.dh, set_width);
    const int pages = (len + PAGE - 1) / PAGE, news = (n + PAGE - 1) / PAGE;
    const int set_units = a.Hkv * tiles_of(set, set_width);
    int shared = found, shared_units = 0;
    {
      const Cost co = cost_of(a.dt, a.dh, a.own_width);
      const float row_units = a.Hkv * tiles_of(a.ncol, a.own_width);
      if (set_units * (found * cs.tile + cs.item) >= rows * row_units * found * co.again) shared = 0;
      shared_units = mine && lead == b && shared ? set_units : 0;
      const float apart = n > 0 ? row_units * ((pages - shared + news) * co.tile + shared * co.again + co.item) : 0.f;
      const float together = (n > 0 ? row_units * ((pages - shared + news) * co.tile + co.item) : 0.f) +
                             shared_units * (shared * cs.tile + cs.item);
      if (team.sum(together) + CHIP * JOIN > team.sum(apart)) shared = shared_units = 0;
    }
    row[b].own = n > 0 ? pages - shared + news : 0;
    row[b].set_units = shared_units;
    team.sync();  // the group's pages and rows have been read
    row[b].shared = shared;
    row[b].rows = rows;
    row[b].set = set;
  }
  // Columns of a block on a row's own keys (64 or 128 where it has more than 64) and splits: the choice whose estimate is
  // best; where a wave holds the rows, a wave for each number of splits.
  __shared__ float s_time[2][SPLITS];
  const int widths = a.own_width > 64 ? 2 : 1;
  if constexpr (ROWS == 64) {
    __syncthreads();
    const int j = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (j < SPLITS)
      for (int v = 0; v < widths; ++v) {
        const float time = choice_of(Team<64>{red}, a, row[tid & 63], v ? 64 : a.own_width, j).time;
        if ((tid & 63) == 0) s_time[v][j] = time;
      }
    __syncthreads();
  } else {
    for (int v = 0; v < widths; ++v)
      for (int j = 0; j < SPLITS; ++j) {
        const float time = choice_of(Team<ROWS>{red}, a, row[tid], v ? 64 : a.own_width, j).time;
        if (tid == 0) s_time[v][j] = time;
      }
    __syncthreads();
  }

  RowParts* parts = reinterpret_cast<RowParts*>(a.plan + PLAN_HEAD / 4);
  if (tid < ROWS) {
    const Team<ROWS> team{red};
    const int b = tid;
    const bool mine = b < B;
    // the first of the best, in every wave: lane i looks at the i-th
    const int lane = tid & 63, at = lane < widths * SPLITS ? lane : 0;
    const float time = (&s_time[0][0])[at];
    const int first = __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64(time == -wave_max(-time))) - 1;
    const int v = first / SPLITS, j = first % SPLITS;
    const PlanRow mine_row = row[b];
    const int lead = mine_row.lead, shared = mine_row.shared, shared_units = mine_row.set_units;
    const Choice c = choice_of(team, a, mine_row, v ? 64 : a.own_width, j);
    const int own_width = c.width, teams = c.teams, own_units = c.units, so = c.own_splits, ss = c.shared_splits;
    int n_shared, n_own;
    const int at_shared = team.scan(shared_units * ss, n_shared), at_own = team.scan(own_units * so, n_own);
    row[b].shared_splits = ss;
    row[b].at_shared = at_shared;
    row[b].own_splits = so;
    row[b].at_own = at_own;
    team.sync();
    if (b == 0) {
      s_shared_items = min(n_shared, a.shared_items);
      s_own_items = min(n_own, a.own_items) / teams;
      s_teams = teams;
      s_own_width = own_width;
      a.plan[0] = s_shared_items + s_own_items;
      a.plan[1] = own_width;
    }
    if (mine) {
      const int gs = shared ? row[lead].shared_splits : 0;
      parts[b] = RowParts{shared ? lead : b, mine_row.set, gs, row[lead].at_shared, so == 1 && gs == 0 ? -1 : so, at_own, {0, 0}};
    }
  }
  __syncthreads();
  // the items: shared pages first, being the longest; in a row or group, tiles of columns last (items of one head
  // and run of keys are a multiple of 8 apart where heads x splits is, and then run on one XCD)
  Item* items = reinterpret_cast<Item*>(parts + B);
  const int n_shared = s_shared_items, n_own = s_own_items, teams = s_teams, own_width = s_own_width;
  auto owner = [&](auto at, int i) {  // the last row whose first unit is at or before i
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (at(row[mid]) <= i)
        lo = mid;
      else
        hi = mid;
    }
    return lo;
  };
  for (int i = tid; i < n_shared; i += THREADS) {
    const int b = owner([](const PlanRow& r) { return r.at_shared; }, i);
    const PlanRow& g = row[b];
    const int splits = g.shared_splits, x = i - g.at_shared, s = x % splits, h = x / splits % a.Hkv, ct = x / splits / a.Hkv;
    items[i] = Item{b, g.rows, h, ct, width_of(a.dt == F32, g.rows * a.ncol), (int)((long)g.shared * s / splits),
                    (int)((long)g.shared * (s + 1) / splits), g.shared * PAGE, g.shared, 0, i, 1};
  }
  for (int j = tid; j < n_own; j += THREADS) {
    const int i = j * teams, b = owner([](const PlanRow& r) { return r.at_own; }, i);
    const PlanRow& g = row[b];
    const int splits = g.own_splits, x = i - g.at_own, s = x % splits, h = x / splits % a.Hkv, ct = x / splits / a.Hkv;
    const int pages = (g.len + PAGE - 1) / PAGE, tiles = pages - g.shared + (g.n + PAGE - 1) / PAGE;
    items[n_shared + j] = Item{b, 1, h, ct, own_width, g.shared + (int)((long)tiles * s / splits),
                               g.shared + (int)((long)tiles * (s + 1) / splits), g.len, pages, g.n,
                               splits == 1 && g.shared == 0 ? -1 : i, teams};
  }
}

// Where the parts lie: O of the shared items, (m, l) of them, then those of the rows' own.
struct Parts {
  float *o_shared, *ml_shared, *o_own, *ml_own;
};

// An item as a block's work.
struct Strip {
  int b, rows, h, ct, n, len, np, t0, t1;
  size_t head;
  float *po, *pml;  // of the columns from the item's first on; null: the result
  int col0;
  __device__ __forceinline__ size_t column(const Args& a, int col) const {
    return column_of(a.G * a.r.max_n, a.p.Hkv, b, rows, h, col);
  }
  __device__ __forceinline__ bool wanted(const Args& a, int col) const {
    const int L = a.r.max_n, ncol = a.G * L;
    return rows == 1 ? col < ncol && col % L < n : col < rows * ncol && col % L < row_new(a.r, b + col / ncol);
  }
  __device__ __forceinline__ bool parts(const Args&) const { return po != nullptr; }
  __device__ __forceinline__ float* part_o(const Args& a, int col) const { return po + (size_t)(col - col0) * a.p.dh; }
  __device__ __forceinline__ float* part_ml(const Args&, int col) const { return pml + 2 * (col - col0); }
};
struct SharedArgs {
  Args a;
  const int32_t* plan;
  Parts parts;
  PlanSizes sizes;
};
// (parts of a row's own keys are as wide as their items, those of shared pages as the widest of them)
__device__ __forceinline__ Strip strip_of(const SharedArgs& x, const Item& i, bool shared, int team = 0) {
  const Args& a = x.a;
  const Parts& p = x.parts;
  const int h = i.h + team;
  Strip s{i.b, i.rows, h, i.ct, i.n, i.len, i.np, i.t0, a.k ? i.t1 : min(i.t1, i.np), (size_t)i.b * a.p.Hkv + h,
          nullptr, nullptr, i.ct * i.width};
  const size_t at = (size_t)(i.part + team) * (shared ? x.sizes.shared_width : i.width);
  if (i.part >= 0) {
    s.po = (shared ? p.o_shared : p.o_own) + at * a.p.dh;
    s.pml = (shared ? p.ml_shared : p.ml_own) + at * 2;
  }
  return s;
}

// The block's item; false where there is none, or words by which a block would leave the arrays.
__device__ __forceinline__ bool item_of(const SharedArgs& s, Item& i) {
  // every load on its way at once: no branch on the number of items before the item's words are there
  const int items = s.plan[0];
  i = reinterpret_cast<const Item*>(s.plan + PLAN_HEAD / 4 + (sizeof(RowParts) / 4) * s.a.r.B)[blockIdx.x];
  const bool fits = item_fits(i, s.sizes);
  return ((int)blockIdx.x < items) & fits;
}

template <int NB>
__global__ __launch_bounds__(64 * F32_WAVES) void shared_f32_kernel(SharedArgs s) {
  __shared__ float xs[F32_WAVES * (2 + 4 * NB) * 64];
  Item i;
  if (item_of(s, i)) f32_tiles<NB>(s.a, strip_of(s, i, i.n == 0), xs);
}

constexpr int WAVES = 8;
// An item's work.  Bound by what bounds the tiles: the pages' bytes with few columns, the products and exponentials
// with many (283 Gflop of 4 rows x 256 tokens over 16 640 positions in 278 us with its join, 1.0 PFLOP/s).  A tile of 128 columns
// takes 1.0 us, what is around an item 11; 64 columns 0.89 and 4.5.  WIDE: sets of more than 32 columns occur.
// One item a block: blocks that took several in turns spilled registers and took 1.4 to 1.5 times as long.  The grid
// is the most that there may be; blocks without an item cost nothing that could be measured.
template <int DH, bool WIDE>
__device__ __forceinline__ void work_on(const SharedArgs& s, const Item& i, char* smem) {
  float* const xs = reinterpret_cast<float*>(smem);
  if (i.teams > 1) {
    const int waves = WAVES / i.teams, team = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / waves;
    const Strip x = strip_of(s, i, false, team);
    float* const mine = xs + team * waves * (2 + DH / 4) * 64;
    if (i.width == 16 && waves == 2) return narrow_tiles<DH, 1, 2>(s.a, x, mine);
    if (i.width == 16 && waves == 4) return narrow_tiles<DH, 1, 4>(s.a, x, mine);
    if (i.width == 32 && waves == 2) return narrow_tiles<DH, 2, 2>(s.a, x, mine);
    if (i.width == 32 && waves == 4) return narrow_tiles<DH, 2, 4>(s.a, x, mine);
    return;
  }
  const Strip x = strip_of(s, i, i.n == 0);
  if (i.width == 16) return narrow_tiles<DH, 1, WAVES>(s.a, x, xs);
  if (i.width == 32) return narrow_tiles<DH, 2, WAVES>(s.a, x, xs);
  if constexpr (WIDE) {
    if (i.width == 64) return wide_tiles<DH, 1, 4>(s.a, x, smem);
    if (i.width == 128) return wide_tiles<DH, 2, 4>(s.a, x, smem);
  }
}
template <int DH, bool WIDE>
__global__ __launch_bounds__(64 * WAVES, 2) void shared_bf16_kernel(SharedArgs s) {
  constexpr int FEW = WAVES * (2 + DH / 4) * 64 * 4;
  __shared__ __attribute__((aligned(16))) char smem[WIDE ? wide_lds<DH>() : FEW];
  static_assert(FEW <= wide_lds<DH>(), "the LDS of a block");
  Item i;
  if (item_of(s, i)) work_on<DH, WIDE>(s, i, smem);
}

// Joins the parts of a column: 32 lanes, four values of the head width each.  Bound by its launch and the bytes of the parts:
// 2 048 columns 5.1 us, 16 384 of two parts 6.1.
template <class T>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs s) {
  const Args& a = s.a;
  const int i = threadIdx.x & 31, L = a.r.max_n, ncol = a.G * L, dh = a.p.dh, Hkv = a.p.Hkv;
  const size_t id = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (id >= (size_t)a.r.B * Hkv * ncol) return;
  const int c = (int)(id % ncol), h = (int)(id / ncol % Hkv), b = (int)(id / ncol / Hkv), g = c / L, j = c % L;
  if (j >= row_new(a.r, b)) return;
  const RowParts p = reinterpret_cast<const RowParts*>(s.plan + PLAN_HEAD / 4)[b];
  const int own_width = s.plan[1];
  const PlanSizes& z = s.sizes;  // on their way beside the row's words: loaded behind the branch, 2 048 blocks took 7.2 us, not 6.2
  asm volatile("" ::"s"(own_width), "s"(z.Hkv), "s"(z.own_width), "s"(z.shared_width), "s"(z.own_columns), "s"(z.shared_columns));
  if (p.own < 0) return;  // one item has written the result
  size_t shared_at, own_at;
  const bool shared = shared_parts(p, s.sizes, b, h, c, shared_at), own = own_parts(p, s.sizes, own_width, h, c, own_at);
  if (!own | (!shared & (p.shared > 0))) return;  // parts of no such plan
  const int d = 4 * i < dh ? 4 * i : 0;
  float m = M_NONE, sum = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const float* ml, const float* o) {
    const float mi = ml[0], top = fmaxf(m, mi), f = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(mi - top);
    const f32x4 v = *reinterpret_cast<const f32x4*>(o);
    sum = sum * f + ml[1] * w;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = r[e] * f + v[e] * w;
    m = top;
  };
#pragma unroll 4
  for (int k = 0; k < p.shared; ++k, shared_at += s.sizes.shared_width)
    add(s.parts.ml_shared + 2 * shared_at, s.parts.o_shared + shared_at * dh + d);
#pragma unroll 4
  for (int k = 0; k < p.own; ++k, own_at += own_width) add(s.parts.ml_own + 2 * own_at, s.parts.o_own + own_at * dh + d);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.o) + (((size_t)b * L + j) * Hkv * a.G + h * a.G + g) * dh;
  if (4 * i < dh) store4(out + 4 * i, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
  if (i == 0 && a.lse) a.lse[id] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}

}  // namespace

size_t page_plan_bytes(DType dt, int B, int H, int Hkv, int L) {
  const Bounds w = bounds_of(dt == F32, B, H, Hkv, L);
  return PLAN_HEAD + (size_t)B * sizeof(RowParts) + (size_t)(w.own_items + w.shared_items) * sizeof(Item);
}

size_t page_shared_threads(DType dt, int B, int H, int Hkv, int L) {
  const Bounds w = bounds_of(dt == F32, B, H, Hkv, L);
  const size_t items = (size_t)(w.own_items + w.shared_items) * (dt == BF16 ? 64 * WAVES : 64 * F32_WAVES);
  const size_t join = (size_t)B * H * L * 32 + 256;
  return items > join ? items : join;
}

size_t page_shared_work(DType dt, int B, int H, int Hkv, int dh, int L) {
  const Bounds w = bounds_of(dt == F32, B, H, Hkv, L);
  return (w.own_columns + w.shared_columns) * (dh + 2) * sizeof(float);
}

hipError_t page_plan(DType dt, const PageRows& r, int H, int Hkv, int dh, int min_pages, int32_t* plan, int32_t* lead,
                     int32_t* pages, hipStream_t s) {
  const Bounds w = bounds_of(dt == F32, r.B, H, Hkv, r.max_n);
  const PlanArgs a{r, dt, Hkv, H / Hkv * r.max_n, dh, min_pages, (int)w.own_items, (int)w.shared_items, w.own_width, plan, lead, pages};
  if (r.B <= 64)
    hipLaunchKernelGGL(plan_kernel<64>, dim3(1), dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL(plan_kernel<PAGE_SHARE_ROWS>, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

hipError_t page_attend_shared(DType dt, const PageAttend& c, const int32_t* plan, hipStream_t s) {
  const int dh = c.p.dh, G = c.H / c.p.Hkv;
  const Bounds w = bounds_of(dt == F32, c.r.B, c.H, c.p.Hkv, c.r.max_n);
  float* work = static_cast<float*>(c.work);
  const size_t shared = w.shared_columns, own = w.own_columns;
  SharedArgs a{Args{c.p, c.r, c.q, c.k, c.vt, c.o, c.lse, nullptr, G, c.cap, 1, 1.4426950408889634f / sqrtf((float)dh)}, plan,
               Parts{work, work + (shared + own) * dh, work + shared * dh, work + (shared + own) * dh + 2 * shared},
               PlanSizes{dt == F32, c.r.B, c.p.Hkv, G * c.r.max_n, c.r.max_n, c.r.max_pages, w.own_width, w.shared_width, own, shared}};
  const dim3 grid((unsigned)(w.own_items + w.shared_items));
  if (dt == BF16) {
    const bool wide = c.r.B * G * c.r.max_n > 32;
    if (dh == 128 && wide)
      launch_timed(shared_bf16_kernel<128, true>, grid, dim3(64 * WAVES), 0, s, a);
    else if (dh == 128)
      launch_timed(shared_bf16_kernel<128, false>, grid, dim3(64 * WAVES), 0, s, a);
    else if (dh == 64 && wide)
      launch_timed(shared_bf16_kernel<64, true>, grid, dim3(64 * WAVES), 0, s, a);
    else if (dh == 64)
      launch_timed(shared_bf16_kernel<64, false>, grid, dim3(64 * WAVES), 0, s, a);
    else
      return hipErrorInvalidValue;
  } else {
    const dim3 threads(64 * F32_WAVES);
    switch ((dh + 15) / 16) {
      case 1: launch_timed(shared_f32_kernel<1>, grid, threads, 0, s, a); break;
      case 2: launch_timed(shared_f32_kernel<2>, grid, threads, 0, s, a); break;
      case 3: launch_timed(shared_f32_kernel<3>, grid, threads, 0, s, a); break;
      case 4: launch_timed(shared_f32_kernel<4>, grid, threads, 0, s, a); break;
      case 5: launch_timed(shared_f32_kernel<5>, grid, threads, 0, s, a); break;
      case 6: launch_timed(shared_f32_kernel<6>, grid, threads, 0, s, a); break;
      case 7: launch_timed(shared_f32_kernel<7>, grid, threads, 0, s, a); break;
      case 8: launch_timed(shared_f32_kernel<8>, grid, threads, 0, s, a); break;
      default: return hipErrorInvalidValue;
    }
  }
  const unsigned joins = (unsigned)(((size_t)c.r.B * c.H * c.r.max_n + 7) / 8);
  if (dt == BF16)
    hipLaunchKernelGGL(shared_join_kernel<bf16>, dim3(joins), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(shared_join_kernel<float>, dim3(joins), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace tadm
