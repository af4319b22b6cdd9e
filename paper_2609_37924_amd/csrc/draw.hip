// One token of each row of logits, from a uniform number and settings of the row's own.
//
// With l' = l (1 / temperature) and m the row's maximum, entry v weighs q_v = rint(exp(l'_v - m) 2^40), the float32
// exponential of the samplers (sampler_math.h): whole numbers, so that every order of summation gives the
// same draw.  The entries' order is l' descending, then v ascending; what is kept of them:
//   K  the first top_k, Q = sum of their q;
//   P  the shortest prefix of K that weighs ceil(p Q 2^-24) or more, p = ceil(top_p 2^24);
//   F  those of P with q >= ceil(min_p 2^40), T = sum of their q.
// The token is the least v at which the running sum of F over v exceeds floor(floor(u 2^24) T 2^-24).
//
// K and P are prefixes of the order, so each is one entry, its last (a cut).  Entries fall into 2 048 bins of
// m - l' (bin_of), which order as they do.  Where the running count or weight over the bins reaches its mark is the
// bin of the cut; what lies in the bins before is kept for sure and summed as it is read, and the entries of
// the bins that a cut may be in go to a list, which is ranked entry by entry.  For a small top_k the bins of the maxima of
// disjoint parts of the row do: the k-th of those bounds the k-th entry, and the list has a few more than k entries.
// A list that overflows leaves the row to digits of z, of l' and of v, one after the other, and to one block: where many entries are
// equal, and where a bin of 1 / 192 at a cut has more than 2 048, as in rows that are nearly flat for their width.
// us with top-p 0.5 and normal l' of deviation 2, then flatter: 1 x 262 144 30, 628 at 0.25, 734 at 0.02, 4 399 all equal;
// 64 x 128 256 56, 403 at 0.1, 2 320 all equal; 1 024 x 32 768 120, 366 at 0.02, 2 083 all equal.  With top-k too the bins of
// both cuts are listed, and 262 144 entries overflow from 0.5 on (610).
//
// A row takes one block, or where that leaves the chip empty several in four launches: maxima of its parts; bins;
// sure weights and list; the draw.
//
// Large calls are bound by the exponential, whose float32 operations are each rounded by themselves, and by sums in LDS; small
// ones by their launches, one after the other.  A row without top-k and top-p takes one exponential an entry, top-p two.
// us a call on one MI355X with none of the settings, with top-k, with top-p and with all of them mixed: 1 024 x 32 768 (134 MB)
// 55, 89, 118, 89; 64 x 128 256 26, 44, 57, 47; 1 x 262 144 13, 23, 27, 27.  The first form, one block a row for all: 1 x 262 144
// with top-p 264, 64 x 128 256 mixed 180.
#include "common.h"
#include "kernels.h"
#include "sampler_math.h"

#pragma clang fp contract(off)

namespace tadm {
namespace {

typedef unsigned long long u64;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows may begin at any float

constexpr int T = 512, NW = T / 64;  // threads and waves of a block; two blocks a CU
constexpr int BINS = 2048, LIST = 2048;
constexpr int BPT = BINS / T;             // bins of a thread
constexpr int CELL = 1024, CELLS = DRAW_MAX_VOCAB / CELL;  // a cell: sixteen entries of each lane of a wave
constexpr int PART = 64, PARTS = DRAW_MAX_VOCAB / PART;   // a part of a row that several blocks share: 16 lanes
constexpr int FEW = 256;                                  // top_k up to here by the maxima of parts
constexpr int LEVELS = 7;

struct Settings {
  float inv;    // 1 / temperature
  int k;        // entries of K; 1 at temperature 0
  uint32_t p;   // ceil(top_p 2^24), 2^24: all
  float q_min;  // ceil(min_p 2^40)
};
__device__ __forceinline__ Settings settings_of(const DrawRows& d, int r) {
  const float t = d.temperature ? d.temperature[r] : 1.f;
  const int k = d.top_k ? d.top_k[r] : 0;
  const float p = d.top_p ? d.top_p[r] : 1.f, q = d.min_p ? d.min_p[r] : 0.f;
  Settings s{1.f, 1, 1u << 24, 0.f};
  if (t > 0.f) {
    s.inv = 1.f / t;
    s.k = k > 0 && k < d.V ? k : d.V;
  }
  if (p < 1.f) s.p = p > 0.f ? (uint32_t)ceilf(p * 0x1p24f) : 1u;
  if (q > 0.f) s.q_min = fminf(ceilf(q * 0x1p40f), 0x1p40f);
  return s;
}

// a x / 2^24 for a <= 2^24, rounded up or down
__device__ __forceinline__ u64 share_of(u64 a, u64 x, bool up) {
  return a * (x >> 24) + ((a * (x & 0xFFFFFF) + (up ? 0xFFFFFF : 0)) >> 24);
}

// A row's entries by y = l' - m <= 0: 2 048 bins, the number before the point, that order as l' does (each operation
// is monotonic): 192 to the unit down to -8, where a flat row's mass is, 32 to -16 and 16 to -30, below
// which nothing weighs.  Eleven binary places behind the point are the next digit.
__device__ __forceinline__ float bin_of(float y) {
  const float z = -y;
  return z < 8.f ? z * 192.f : z < 16.f ? z * 32.f + 1280.f : z * 16.f + 1536.f;
}

// Digit `level` of an entry in the order, ascending.
__device__ __forceinline__ uint32_t digit(int level, float x, float y, int v) {
  const float z = bin_of(y);
  if (level == 0) return (uint32_t)z;
  if (level == 1) return (uint32_t)((z - floorf(z)) * 2048.f);
  if (level >= 5) return ((uint32_t)v >> (level == 5 ? 9 : 0)) & 511u;
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 is 0
  const uint32_t key = b & 0x80000000u ? b : ~b & 0x7FFFFFFFu;
  return level == 2 ? key >> 21 : level == 3 ? (key >> 10) & 2047u : key & 1023u;
}

// The last entry of a prefix of the order.
struct Cut {
  float x;
  int v;
  __device__ __forceinline__ bool has(float xv, int v_) const { return xv > x || (xv == x && v_ <= v); }
};

struct BinsShared {
  u64 mass[BINS];
  uint32_t count[BINS];
  u64 wave[NW];
  float wave_f[NW];
  u64 through;  // the weight of a prefix
  u64 before;   // what comes before the chosen bin: entries or weight
  uint32_t bin, n;  // the chosen bin; entries in the list
};
struct Shared : BinsShared {
  u64 sub[BINS];  // bins of the list
  float list_x[LIST];
  int list_v[LIST];
  u64 list_q[LIST];
  uint16_t few[LIST];
  u64 cell[CELLS];
  Cut cut;
  uint32_t n_few;           // of the list, the few that a cut is among
  uint32_t prefix[LEVELS];  // digits chosen so far
  int token;
  u64 rest;
  __device__ __forceinline__ void put(float x, int v, u64 q) {
    const uint32_t at = atomicAdd(&n, 1u);
    if (at < LIST) {
      list_x[at] = x;
      list_v[at] = v;
      list_q[at] = q;
    }
  }
};
// Of a block that lists entries for another: three blocks a CU.
struct ListShared : BinsShared {
  float list_x[LIST];
  int list_v[LIST];
  uint32_t at;
  __device__ __forceinline__ void put(float x, int v) {
    const uint32_t i = atomicAdd(&n, 1u);
    if (i < LIST) {
      list_x[i] = x;
      list_v[i] = v;
    }
  }
};

__device__ __forceinline__ float block_max(float v, BinsShared& s) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s.wave_f[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s.wave_f[0];
  for (int w = 1; w < NW; ++w) v = fmaxf(v, s.wave_f[w]);
  return v;
}

// Sum over the lanes up to and with this one: within 16 lanes by shifts, then the row before and the half before.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 add_dpp(u64 v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
  return v + ((u64)hi << 32 | lo);
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
  v = add_dpp<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v = add_dpp<0x112, 0xF>(v);
  v = add_dpp<0x114, 0xF>(v);
  v = add_dpp<0x118, 0xF>(v);
  v = add_dpp<0x142, 0xA>(v);  // row_bcast 15 into rows 1 and 3
  return add_dpp<0x143, 0xC>(v);  // row_bcast 31 into rows 2 and 3
}
// Sum over the threads before this one; all: over every one.
__device__ __forceinline__ u64 block_scan(u64 v, u64* wave, u64* all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const u64 sum = wave_scan(v);
  __syncthreads();
  if (lane == 63) wave[w] = sum;
  __syncthreads();
  u64 before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const u64 x = wave[i];
    before += i < w ? x : 0;
    total += x;
  }
  *all = total;
  return before + sum - v;
}
// The thread's bins.
struct Bins {
  u64 v[BPT];
  template <class H>
  __device__ __forceinline__ explicit Bins(const H* hist) {
#pragma unroll
    for (int i = 0; i < BPT; ++i) v[i] = hist[BPT * threadIdx.x + i];
  }
  __device__ __forceinline__ u64 sum() const {
    u64 r = 0;
#pragma unroll
    for (int i = 0; i < BPT; ++i) r += v[i];
    return r;
  }
};

// The bin at which the running sum over the bins reaches `mark` >= 1 (no more than the sum of all); s.bin and
// s.before (the sum of the bins before it).  before: the sum of those before the thread's.
__device__ __forceinline__ void pick_bin(u64 before, const Bins& x, u64 mark, BinsShared& s) {
  __syncthreads();
  if (before < mark && before + x.sum() >= mark) {
    uint32_t bin = BPT * threadIdx.x;
#pragma unroll
    for (int i = 0; i + 1 < BPT; ++i)
      if (before + x.v[i] < mark && bin == BPT * threadIdx.x + i) {
        before += x.v[i];
        ++bin;
      }
    s.bin = bin;
    s.before = before;
  }
  __syncthreads();
}
template <class H>
__device__ __forceinline__ void choose_bin(const H* hist, u64 mark, BinsShared& s) {
  const Bins x(hist);
  u64 all;
  const u64 before = block_scan(x.sum(), s.wave, &all);
  pick_bin(before, x, mark, s);
}

// A row of logits, or a block's share [first, end) of one; first is a multiple of CELL NW.  A wave has every NW-th
// cell: its lane l the quads at 256 i + 4 l, i < 4.  The next cell's are on their way while one is worked on.
struct Row {
  const float* lg;
  int V;
  float inv;
  int first, end;
  f32x4 head[4];  // the quads of the wave's first cell, on their way since start()

  __device__ __forceinline__ int first_cell() const { return first / CELL + (int)(threadIdx.x >> 6); }
  __device__ __forceinline__ void load_cell(int c, f32x4 (&a)[4]) const {
    const int v = c * CELL + 4 * (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = load(v + 256 * i);
  }
  __device__ __forceinline__ void start() {
    if (first_cell() * CELL < end) load_cell(first_cell(), head);
  }
  __device__ __forceinline__ f32x4 load(int v) const {
    f32x4 a;
    if (v + 3 < V) {
      a = *reinterpret_cast<const f32x4u*>(lg + v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = v + e < V ? lg[v + e] : -INFINITY;
    }
    return a;
  }
  __device__ __forceinline__ f32x4 scaled(const f32x4& a) const {
    f32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = a[e] * inv;
    return r;
  }
  // f(cell, the lane's first entry, l' of its quads) for the wave's cells
  template <class F>
  __device__ __forceinline__ void cells(F f) const {
    f32x4 next[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = head[i];
    for (int c = first_cell(); c * CELL < end; c += NW) {
      f32x4 a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = scaled(next[i]);
      if ((c + NW) * CELL < end) load_cell(c + NW, next);
      f(c, c * CELL + 4 * (int)(threadIdx.x & 63), a);
    }
  }
  // f(quad of the cell, the lane's first entry, its four l'), and at a cell's end done(cell)
  template <class F, class D>
  __device__ __forceinline__ void quads(F f, D done) const {
    cells([&](int c, int v, const f32x4 (&a)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) f(i, v + 256 * i, a[i]);
      done(c);
    });
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    quads(
        [&](int, int v, const f32x4& a) {
#pragma unroll
          for (int e = 0; e < 4; ++e) f(a[e], v + e);
        },
        [](int) {});
  }
};
// Sum over the wave of whole numbers, none of the partial sums above 2^53: exact.
__device__ __forceinline__ double wave_whole(double q) {
  q = row16_sum(q);
  q += xor16(q);
  return q + xor32(q);
}

// l' - m; entries that are -inf or lie past the row weigh nothing, nor does a NaN, which fails every comparison here, and
// which a maximum passes over
__device__ __forceinline__ float below(float x, float m) { return x == m ? 0.f : x - m; }
constexpr float Y_MIN = -30.f;  // own_exp_term is 0 at and below

__device__ __forceinline__ void clear(u64* a, int n) {
  for (int i = threadIdx.x; i < n; i += T) a[i] = 0;
}

// Of the list's entries in `bin` (BINS: of all), the one at which the running count or weight over their order reaches
// mark (s.cut).  Longer lists by their bins (unless they are of one) and the next digit first, then entry by entry
// (a step of that loop waits for LDS, some 0.19 us each).
__device__ __forceinline__ void cut_in_list(Shared& s, float m, bool count, u64 mark, uint32_t bin, bool one_bin) {
  constexpr int DIRECT = 8;
  const int n = min((int)s.n, LIST), tid = threadIdx.x;
  uint32_t next = BINS;  // the next digit of the entries left
  auto left = [&](float x, int v) {
    const float y = below(x, m);
    return (bin == BINS || digit(0, x, y, v) == bin) && (next == BINS || digit(1, x, y, v) == next);
  };
  if (n > DIRECT)
#pragma unroll 1
    for (int level = one_bin ? 1 : 0; level < 2; ++level) {
      clear(s.sub, BINS);
      __syncthreads();
      for (int i = tid; i < n; i += T) {
        const float x = s.list_x[i];
        const int v = s.list_v[i];
        if (left(x, v)) atomicAdd(&s.sub[digit(level, x, below(x, m), v)], count ? 1 : s.list_q[i]);
      }
      __syncthreads();
      choose_bin(s.sub, mark, s);
      (level ? next : bin) = s.bin;
      mark -= s.before;
    }
  if (tid == 0) s.n_few = 0;
  __syncthreads();
  for (int i = tid; i < n; i += T)
    if (left(s.list_x[i], s.list_v[i])) s.few[atomicAdd(&s.n_few, 1u)] = (uint16_t)i;
  __syncthreads();
  const int few = s.n_few;
  for (int i = tid; i < few; i += T) {
    const Cut mine{s.list_x[s.few[i]], s.list_v[s.few[i]]};
    const u64 q = s.list_q[s.few[i]];
    u64 before = 0;
    for (int j = 0; j < few; ++j) {
      const int at = s.few[j];
      if (j != i && mine.has(s.list_x[at], s.list_v[at])) before += count ? 1 : s.list_q[at];
    }
    if (before < mark && before + (count ? 1 : q) >= mark) s.cut = mine;
  }
  __syncthreads();
}
// The weight of the list's entries up to the cut, in `bin` (BINS: in all).
__device__ __forceinline__ u64 weigh_list(Shared& s, float m, const Cut& cut, uint32_t bin) {
  const int n = min((int)s.n, LIST);
  u64 sum = 0, all;
  for (int i = threadIdx.x; i < n; i += T) {
    const float x = s.list_x[i];
    if (cut.has(x, s.list_v[i]) && (bin == BINS || (uint32_t)bin_of(below(x, m)) == bin)) sum += s.list_q[i];
  }
  block_scan(sum, s.wave, &all);
  return all;
}

// What a row's settings leave to do.
enum Kind { NOTHING, FIRST, SMALL_K, BY_BINS, ALL };
__device__ __forceinline__ Kind kind_of(const Settings& s, float m, int V, int small) {
  if (m == -INFINITY) return NOTHING;
  if (s.k == 1) return FIRST;
  if (s.k < V && s.k <= small) return SMALL_K;
  return s.k < V || s.p < 1u << 24 ? BY_BINS : ALL;
}

// Which bins are kept for sure, and which hold a cut or may.
struct Marks {
  uint32_t sure;             // bins below are kept
  uint32_t lo, hi;           // the cut of P is in one of these
  uint32_t k_bin;            // that of K; BINS: K is everything
  u64 k_left;                // entries of k_bin that K has
  u64 k_mass, lo_mass, mass; // weight before k_bin, before lo, and of all
  __device__ __forceinline__ bool listed(uint32_t bin) const { return (bin >= lo && bin <= hi) || bin == k_bin; }
};
// From the bins in s (counts where top_k is on, weights where top_p is).
__device__ __forceinline__ Marks marks_of(const Settings& set, int V, BinsShared& s) {
  const int tid = threadIdx.x;
  Marks r{BINS, BINS, BINS, BINS, 0, 0, 0, 0};
  if (set.k < V) {
    const Bins x(s.count);
    u64 all;
    const u64 before = block_scan(x.sum(), s.wave, &all);
    if (all > (u64)set.k) {
      pick_bin(before, x, set.k, s);
      r.k_bin = s.bin;
      r.k_left = set.k - s.before;
    }
  }
  if (set.p < 1u << 24) {
    const Bins x(s.mass);
    const u64 before = block_scan(x.sum(), s.wave, &r.mass);
    u64 least = r.mass, most = r.mass;
    if (r.k_bin < BINS) {
      if (r.k_bin / BPT == (uint32_t)tid) {
        u64 sum = before;
#pragma unroll
        for (int i = 0; i < BPT; ++i) sum += BPT * tid + i < (int)r.k_bin ? x.v[i] : 0;
        s.through = sum;
      }
      __syncthreads();
      r.k_mass = least = s.through;
      most = least + s.mass[r.k_bin];
    }
    const u64 low = share_of(set.p, least, true), high = share_of(set.p, most, true);
    pick_bin(before, x, low ? low : 1, s);
    r.lo = r.hi = s.bin;
    r.lo_mass = s.before;
    if (high > low) {
      pick_bin(before, x, high, s);
      r.hi = s.bin;
    }
    r.sure = r.lo;
  } else {
    r.sure = r.lo = r.hi = r.k_bin;
  }
  return r;
}

// The list holds every entry that a cut may be: the cut of P (or of K).  SMALL_K: no bins, the list has all of K.
// lo < hi: the bins' weights are in s.
__device__ __forceinline__ Cut cut_of(const Settings& set, Kind kind, const Marks& k, float m, int V, Shared& s) {
  Cut cut{-INFINITY, V};
  u64 Q = k.mass;
#pragma unroll 1
  for (int step = 0; step < 2; ++step) {  // the cut of K, that of P
    uint32_t bin = BINS;
    u64 mark;
    if (step == 0) {
      if (kind == SMALL_K ? (int)s.n < set.k : k.k_bin == BINS) continue;  // K is everything
      mark = kind == SMALL_K ? set.k : k.k_left;
      if (kind == BY_BINS) bin = k.k_bin;
    } else {
      if (set.p == 1u << 24) break;
      if (kind == SMALL_K) {
        Q = weigh_list(s, m, cut, BINS);
      } else if (k.k_bin < BINS) {
        Q = k.k_mass + weigh_list(s, m, cut, k.k_bin);
      }
      mark = share_of(set.p, Q, true);
      if (kind == BY_BINS) {
        bin = k.lo;
        u64 base = k.lo_mass;
        if (k.k_bin < BINS && mark > k.k_mass) {
          bin = k.k_bin;
          base = k.k_mass;
        } else if (k.lo < k.hi) {
          choose_bin(s.mass, mark, s);
          bin = s.bin;
          base = s.before;
        }
        mark -= base;
      }
    }
    cut_in_list(s, m, step == 0, mark, bin, kind == BY_BINS);
    cut = s.cut;
  }
  return cut;
}

// An entry's weight in F.
__device__ __forceinline__ float kept_weight(float x, int v, float m, const Cut& cut, const Settings& set) {
  const float q = cut.has(x, v) ? own_exp_term(below(x, m)) : 0.f;
  return q >= set.q_min ? q : 0.f;
}

// The token, from F's weight by cells (s.cell).
__device__ __forceinline__ void draw_token(const DrawRows& d, int r, const Row& row, float m, const Cut& cut, const Settings& set, Shared& s) {
  const int tid = threadIdx.x, lane = tid & 63;
  static_assert(CELLS <= T, "a thread a cell");
  __syncthreads();
  const u64 mine = tid < CELLS ? s.cell[tid] : 0;
  u64 total;
  const u64 before = block_scan(mine, s.wave, &total);
  const float u = d.u[r];
  const u64 mark = share_of(u > 0.f ? (u64)fminf(floorf(u * 0x1p24f), 0x1p24f - 1.f) : 0ull, total, false);
  if (before <= mark && before + mine > mark) {
    s.token = tid * CELL;
    s.rest = mark - before;
  }
  __syncthreads();
  if (tid >= 64) return;
  const int v = s.token + 4 * lane;
  u64 rest = s.rest;
  f32x4 next = row.load(v);
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const f32x4 a = row.scaled(next);
    if (i < 3) next = row.load(v + 256 * (i + 1));
    u64 q[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += q[e] = (u64)kept_weight(a[e], v + 256 * i + e, m, cut, set);
    const u64 upto = wave_scan(sum);
    u64 run = upto - sum, chosen = 0;
    if (run <= rest && upto > rest) {
      int at = -1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        run += q[e];
        if (at < 0 && run > rest) {
          at = v + 256 * i + e;
          chosen = q[e];
        }
      }
      d.token[r] = at;
      if (d.logp) d.logp[r] = (float)log((double)chosen / (double)total);
    }
    const u64 all = __shfl(upto, 63, 64);
    if (all > rest) return;  // the whole wave
    rest -= all;
  }
}

__device__ __forceinline__ void answer(const DrawRows& d, int r, int token, float logp) {
  if (threadIdx.x == 0) {
    d.token[r] = token;
    if (d.logp) d.logp[r] = logp;
  }
}

// F's weight in the cells of a block, every entry against the cut.
template <class Put>
__device__ __forceinline__ void weigh_cells(const Row& row, float m, const Cut& cut, const Settings& set, Put put) {
  double sum = 0.0;
  row.quads(
      [&](int i, int v, const f32x4& a) {
        if (i == 0) sum = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += (double)kept_weight(a[e], v + e, m, cut, set);
      },
      [&](int c) {
        const double q = wave_whole(sum);
        if ((threadIdx.x & 63) == 0) put(c, q);
      });
}

// A row whose list overflowed, by digits: for the cut of K and that of P, the bins of the entries that the digits
// chosen so far have left, until these fit a list.
__device__ __noinline__ Cut cut_by_digits(Settings set, const float* lg, int V, float m, Shared& s) {
  const int tid = threadIdx.x;
  Row row{lg, V, set.inv, 0, V, {}};
  Cut cut{-INFINITY, V};
#pragma unroll 1
  for (int step = 0; step < 2; ++step) {
    const bool count = step == 0;
    if (count ? set.k >= V : set.p == 1u << 24) continue;
    u64 mark = set.k;
    int level = 0;
    for (;; ++level) {
      // an entry that takes part: its weight if its first n digits are those chosen, else 0
      auto weight = [&](float x, int v, int n) {
        const float y = below(x, m);
        if (!(y > Y_MIN) || !cut.has(x, v)) return (u64)0;
        for (int l = 0; l < n; ++l)
          if (digit(l, x, y, v) != s.prefix[l]) return (u64)0;
        return (u64)own_exp_term(y);
      };
      clear(s.mass, BINS);
      row.start();
      __syncthreads();
      row.each([&](float x, int v) {
        const u64 q = weight(x, v, level);
        if (q) atomicAdd(&s.mass[digit(level, x, below(x, m), v)], count ? 1 : q);
      });
      __syncthreads();
      const Bins x(s.mass);
      u64 all;
      const u64 before = block_scan(x.sum(), s.wave, &all);
      if (level == 0 && !count) mark = share_of(set.p, all, true);
      if (all < mark) break;  // K is everything
      pick_bin(before, x, mark, s);
      mark -= s.before;
      if (tid == 0) {
        s.prefix[level] = s.bin;
        s.n = 0;
      }
      __syncthreads();
      row.each([&](float x, int v) {
        const u64 q = weight(x, v, level + 1);
        if (q) s.put(x, v, q);
      });
      __syncthreads();
      if (s.n <= LIST) {
        cut_in_list(s, m, count, mark, BINS, level > 0);
        cut = s.cut;
        break;
      }
    }
    __syncthreads();
  }
  return cut;
}

// The list and the sure weights of a block's entries.  SMALL_K: every entry of the bins up to `last`.
template <class Put>
__device__ __forceinline__ void gather_small(const Row& row, float m, uint32_t last, Put put) {
  const float end = (float)(last + 1);
  row.quads([&](int, int v, const f32x4& a) {
    const float top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
    if (!(bin_of(below(top, m)) < end)) return;
#pragma unroll 1
    for (int e = 0; e < 4; ++e) {
      const float x = e == 0 ? a[0] : e == 1 ? a[1] : e == 2 ? a[2] : a[3], y = below(x, m);
      if (!(y > Y_MIN) || !(bin_of(y) < end)) continue;
      const u64 q = (u64)own_exp_term(y);
      if (q) put(x, v + e, q);
    }
  }, [](int) {});
}
template <class Put, class Cell>
__device__ __forceinline__ void gather_bins(const Row& row, float m, const Marks& k, const Settings& set, Put put, Cell cell) {
  double sum = 0.0;
  row.quads([&](int i, int v, const f32x4& a) {
    if (i == 0) sum = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = below(a[e], m);
      const float q = own_exp_term(y);
      const uint32_t bin = y > Y_MIN ? (uint32_t)bin_of(y) : BINS;
      sum += bin < k.sure && q >= set.q_min ? (double)q : 0.0;
      if (bin < BINS && k.listed(bin) && q > 0.f) put(a[e], v + e, (u64)q);
    }
  }, [&](int c) {
    const double q = wave_whole(sum);
    if ((threadIdx.x & 63) == 0) cell(c, q);
  });
}
// Adds a block's entries to the bins in s.
__device__ __forceinline__ void fill_bins(const Row& row, float m, const Settings& set, BinsShared& s) {
  const bool top_k = set.k < row.V, top_p = set.p < 1u << 24;
  for (int i = threadIdx.x; i < BINS; i += T) {
    s.mass[i] = 0;
    s.count[i] = 0;
  }
  __syncthreads();
  row.each([&](float x, int) {
    const float y = below(x, m);
    if (!(y > Y_MIN)) return;
    const float q = own_exp_term(y);
    if (q == 0.f) return;
    const uint32_t bin = (uint32_t)bin_of(y);
    if (top_k) atomicAdd(&s.count[bin], 1u);
    if (top_p) atomicAdd(&s.mass[bin], (u64)q);
  });
  __syncthreads();
}
// The kept entries of the list that are not sure, into their cells.
__device__ __forceinline__ void add_list(const Cut& cut, const Settings& set, Shared& s) {
  const int n = min((int)s.n, LIST);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += T) {
    const u64 q = s.list_q[i];
    if (cut.has(s.list_x[i], s.list_v[i]) && (float)q >= set.q_min) atomicAdd(&s.cell[s.list_v[i] / CELL], q);
  }
}
// The bin at which the maxima of parts are as many as k; all bins where they are too few.
__device__ __forceinline__ uint32_t small_bin(int k, BinsShared& s) {
  const Bins x(s.count);
  u64 all;
  const u64 before = block_scan(x.sum(), s.wave, &all);
  if (all < (u64)k) return BINS - 1;
  pick_bin(before, x, k, s);
  return s.bin;
}

// One block a row.
__global__ __launch_bounds__(T, 4) void draw_kernel(DrawRows d) {
  __shared__ Shared s;
  const int r = blockIdx.x, tid = threadIdx.x;
  const Settings set = settings_of(d, r);
  Row row{d.logits + (size_t)r * d.ld, d.V, set.inv, 0, d.V, {}};
  row.start();
  float own = -INFINITY;
  row.cells([&](int, int, const f32x4 (&a)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) own = fmaxf(own, fmaxf(fmaxf(a[i][0], a[i][1]), fmaxf(a[i][2], a[i][3])));
  });
  const float m = block_max(own, s);
  // the parts are the threads' entries here; a row that fits the list has none too many
  const Kind kind = kind_of(set, m, d.V, d.V <= LIST ? FEW : min(FEW, d.V / CELL * 32));
  if (kind == NOTHING) return answer(d, r, -1, -INFINITY);
  if (tid == 0) {
    s.token = d.V;
    s.n = 0;
  }
  clear(s.cell, CELLS);
  __syncthreads();
  if (kind == FIRST) {
    int first = d.V;
    row.each([&](float x, int v) {
      if (x == m) first = min(first, v);
    });
    if (first < d.V) atomicMin(&s.token, first);
    __syncthreads();
    return answer(d, r, s.token, 0.f);
  }
  Cut cut{-INFINITY, d.V};
  Marks k{};
  const auto put = [&](float x, int v, u64 q) { s.put(x, v, q); };
  const auto cell = [&](int c, double q) { s.cell[c] = (u64)q; };
  if (kind == SMALL_K) {
    for (int i = tid; i < BINS; i += T) s.count[i] = 0;
    __syncthreads();
    if (below(own, m) > Y_MIN) atomicAdd(&s.count[(uint32_t)bin_of(below(own, m))], 1u);
    __syncthreads();
    gather_small(row, m, small_bin(set.k, s), put);
  } else if (kind == BY_BINS) {
    fill_bins(row, m, set, s);
    k = marks_of(set, d.V, s);
    gather_bins(row, m, k, set, put, cell);
  } else {
    weigh_cells(row, m, cut, set, cell);
  }
  __syncthreads();
  if (s.n > LIST) {
    cut = cut_by_digits(set, row.lg, d.V, m, s);
    weigh_cells(row, m, cut, set, cell);
  } else if (kind != ALL) {
    cut = cut_of(set, kind, k, m, d.V, s);
    add_list(cut, set, s);
  }
  draw_token(d, r, row, m, cut, set, s);
}

// ---- a row in several blocks
// What the launches of a row hand on.
struct alignas(16) Work {
  float part_max[PARTS];
  u64 mass[BINS];
  uint32_t count[BINS];
  double cell[CELLS];
  float x[LIST];
  int v[LIST];
  Marks marks;
  float m;
  uint32_t n;
  int first;
};
struct Split {
  DrawRows d;
  Work* work;
  int share;  // entries of a block, a multiple of CELL NW
};
__device__ __forceinline__ Row share_of_row(const Split& a, float inv) {
  const int first = blockIdx.x * a.share;
  Row row{a.d.logits + (size_t)blockIdx.y * a.d.ld, a.d.V, inv, first, min(first + a.share, a.d.V), {}};
  row.start();
  return row;
}
// The row's maximum, from those of its parts; own: the thread's.
struct OwnParts {
  static constexpr int N = PARTS / T;
  float v[N];
};
__device__ __forceinline__ float row_max(const Split& a, const Work& w, BinsShared& s, OwnParts& own) {
  const int parts = (a.d.V + PART - 1) / PART;
  float m = -INFINITY;
#pragma unroll
  for (int e = 0; e < OwnParts::N; ++e) {
    const int i = threadIdx.x + T * e;
    own.v[e] = i < parts ? w.part_max[i] : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < OwnParts::N; ++e) m = fmaxf(m, own.v[e]);
  return block_max(m, s);
}
__device__ __forceinline__ Kind kind_split(const Split& a, const Settings& set, float m) {
  return kind_of(set, m, a.d.V, min(FEW, a.d.V / PART / 2));
}
__device__ __forceinline__ void load_bins(const Work& w, BinsShared& s) {
  for (int i = threadIdx.x; i < BINS; i += T) {
    s.mass[i] = w.mass[i];
    s.count[i] = w.count[i];
  }
  __syncthreads();
}

__global__ __launch_bounds__(T, 4) void parts_kernel(Split a) {
  const int tid = threadIdx.x;
  Work& w = a.work[blockIdx.y];
  const Row row = share_of_row(a, settings_of(a.d, blockIdx.y).inv);
  for (int i = blockIdx.x * T + tid; i < BINS; i += gridDim.x * T) {
    w.mass[i] = 0;
    w.count[i] = 0;
  }
  if (blockIdx.x == 0 && tid == 0) {
    w.n = 0;
    w.first = a.d.V;
  }
  row.cells([&](int, int v, const f32x4 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float m = row16_max(fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3])));
      if ((tid & 15) == 0 && v + 256 * i < a.d.V) w.part_max[(v + 256 * i) / PART] = m;
    }
  });
}

__global__ __launch_bounds__(T, 4) void bins_kernel(Split a) {
  __shared__ BinsShared s;
  Work& w = a.work[blockIdx.y];
  const Settings set = settings_of(a.d, blockIdx.y);
  const Row row = share_of_row(a, set.inv);
  OwnParts own;
  const float m = row_max(a, w, s, own);
  if (kind_split(a, set, m) != BY_BINS) return;
  fill_bins(row, m, set, s);
  for (int i = threadIdx.x; i < BINS; i += T) {
    if (s.count[i]) atomicAdd(&w.count[i], s.count[i]);
    if (s.mass[i]) atomicAdd(&w.mass[i], s.mass[i]);
  }
}

__global__ __launch_bounds__(T, 4) void gather_kernel(Split a) {
  __shared__ ListShared s;
  const int tid = threadIdx.x;
  Work& w = a.work[blockIdx.y];
  const Settings set = settings_of(a.d, blockIdx.y);
  const Row row = share_of_row(a, set.inv);
  OwnParts own;
  const float m = row_max(a, w, s, own);
  if (blockIdx.x == 0 && tid == 0) w.m = m;
  const Kind kind = kind_split(a, set, m);
  if (kind == NOTHING) return;
  if (kind == FIRST) {
    int first = a.d.V;
    row.each([&](float x, int v) {
      if (x == m) first = min(first, v);
    });
    if (first < a.d.V) atomicMin(&w.first, first);
    return;
  }
  if (tid == 0) s.n = 0;
  const auto put = [&](float x, int v, u64) { s.put(x, v); };
  const auto cell = [&](int c, double q) { w.cell[c] = q; };
  if (kind == ALL) return weigh_cells(row, m, Cut{-INFINITY, a.d.V}, set, cell);
  if (kind == SMALL_K) {
    for (int i = tid; i < BINS; i += T) s.count[i] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < OwnParts::N; ++e)
      if (below(own.v[e], m) > Y_MIN) atomicAdd(&s.count[(uint32_t)bin_of(below(own.v[e], m))], 1u);
    __syncthreads();
    gather_small(row, m, small_bin(set.k, s), put);
  } else {
    load_bins(w, s);
    const Marks k = marks_of(set, a.d.V, s);
    if (blockIdx.x == 0 && tid == 0) w.marks = k;
    gather_bins(row, m, k, set, put, cell);
  }
  __syncthreads();
  if (tid == 0 && s.n) s.at = atomicAdd(&w.n, s.n);
  __syncthreads();
  for (int i = tid; i < min((int)s.n, LIST); i += T)
    if (s.at + i < LIST) {
      w.x[s.at + i] = s.list_x[i];
      w.v[s.at + i] = s.list_v[i];
    }
}

__global__ __launch_bounds__(T, 4) void finish_kernel(Split a) {
  __shared__ Shared s;
  const int r = blockIdx.x, tid = threadIdx.x;
  const DrawRows& d = a.d;
  const Work& w = a.work[r];
  const Settings set = settings_of(d, r);
  // every load is on its way before the first is waited for
  constexpr int N = LIST / T;
  float x[N];
  int v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = w.x[tid + T * i];
    v[i] = w.v[tid + T * i];
  }
  const double mine = tid < CELLS ? w.cell[tid] : 0.0;
  const float m = w.m;
  const uint32_t listed = w.n;
  const int first = w.first;
  const Marks marks = w.marks;
  const Kind kind = kind_split(a, set, m);
  if (kind == NOTHING) return answer(d, r, -1, -INFINITY);
  if (kind == FIRST) return answer(d, r, first, 0.f);
  Row row{d.logits + (size_t)r * d.ld, d.V, set.inv, 0, d.V, {}};
  const uint32_t n = kind == ALL ? 0 : listed;
  Cut cut{-INFINITY, d.V};
  if (n > LIST) {
    cut = cut_by_digits(set, row.lg, d.V, m, s);
    clear(s.cell, CELLS);
    row.start();
    __syncthreads();
    weigh_cells(row, m, cut, set, [&](int c, double q) { s.cell[c] = (u64)q; });
  } else {
    if (tid == 0) s.n = n;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((uint32_t)(tid + T * i) < n) {
        s.list_x[tid + T * i] = x[i];
        s.list_v[tid + T * i] = v[i];
        s.list_q[tid + T * i] = (u64)own_exp_term(below(x[i], m));
      }
    if (tid < CELLS) s.cell[tid] = kind != SMALL_K && tid * CELL < d.V ? (u64)mine : 0;
    if (kind == BY_BINS && marks.lo < marks.hi) load_bins(w, s);
    __syncthreads();
    if (kind != ALL) {
      cut = cut_of(set, kind, marks, m, d.V, s);
      add_list(cut, set, s);
    }
  }
  draw_token(d, r, row, m, cut, set, s);
}

// Entries of a block where a row takes several; 0: one block a row.  Up to 1 024 blocks in all: rows differ in what they need, so
// that 512 blocks of twice the entries took 132 us for 256 mixed rows of 128 256 where these take 114 (with top-p alone 139 and
// 134; calls of up to 64 rows within 5 us of each other).
int share_for(int R, int V) {
  constexpr int UNIT = CELL * NW;
  const int most = (V + UNIT - 1) / UNIT, blocks = 1024 / R < most ? 1024 / R : most;
  if (blocks < 2) return 0;
  return ((V + blocks - 1) / blocks + UNIT - 1) / UNIT * UNIT;
}

}  // namespace

size_t draw_work(int R, int V) { return share_for(R, V) ? (size_t)R * sizeof(Work) : 0; }

hipError_t draw_rows(const DrawRows& d, void* work, hipStream_t s) {
  if (const int share = share_for(d.R, d.V)) {
    const Split a{d, static_cast<Work*>(work), share};
    const dim3 grid((d.V + share - 1) / share, d.R);
    hipLaunchKernelGGL(parts_kernel, grid, dim3(T), 0, s, a);
    if (d.top_k || d.top_p) hipLaunchKernelGGL(bins_kernel, grid, dim3(T), 0, s, a);
    hipLaunchKernelGGL(gather_kernel, grid, dim3(T), 0, s, a);
    hipLaunchKernelGGL(finish_kernel, dim3(d.R), dim3(T), 0, s, a);
  } else {
    hipLaunchKernelGGL(draw_kernel, dim3(d.R), dim3(T), 0, s, d);
  }
  return hipGetLastError();
}

}  // namespace tadm
