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
#include "page_tiles.h"

namespace tadm {
namespace {

// Columns of a block by the columns of a set; 16 in float32.
__host__ __device__ __forceinline__ int width_of(DType dt, int columns) {
  return dt == F32 || columns <= 16 ? 16 : columns <= 32 ? 32 : columns <= 64 ? 64 : 128;
}
__host__ __device__ __forceinline__ int tiles_of(int columns, int width) { return (columns + width - 1) / width; }

// One item of a plan.
struct Item {
  int b, rows;         // the row whose pages are read; rows whose columns are in the set
  int h, ct, width;    // K/V head, tile of columns
  int t0, t1;          // key tiles: pages, behind the last of them the window's
  int len, np, n;      // positions on pages and their tiles; the row's window (0 on shared pages)
  int part;            // where its columns' parts begin, -1: it writes the result
  int pad;
};
// What a row's columns are joined from: the group's items with h and ct 0, then the row's own.
struct RowParts {
  int lead, columns;      // first row of the group, columns of its set; no shared part: lead is the row
  int shared, at_shared;  // splits of the shared pages, and the part of their first item
  int own, at_own;        // splits of its own keys, ...; own < 0: one, which has written the result
  int pad[2];
};
constexpr int PLAN_HEAD = 64;  // bytes before the rows; the first word is the number of items

// Sizes of a plan and of what its items write, from what the host knows.
struct Bounds {
  int own_width, own_tiles;   // columns of a block on a row's own keys, tiles of them per head
  int shared_width;           // the most columns of a block on shared pages
  long own_items, shared_items;
};
constexpr int CHIP = 256;  // blocks that run at once: one a CU
Bounds bounds_of(DType dt, int B, int H, int Hkv, int L) {
  const int ncol = H / Hkv * L;
  Bounds r;
  r.own_width = width_of(dt, ncol);
  r.own_tiles = tiles_of(ncol, r.own_width);
  r.shared_width = width_of(dt, B * ncol < 128 ? B * ncol : 128);
  const long own = (long)B * Hkv * r.own_tiles;
  // groups have two rows or more, and each set at most one tile more than its columns fill
  const long shared = B < 2 ? 0 : (long)Hkv * (tiles_of(B * ncol, dt == F32 ? 16 : 128) + B / 2);
  r.own_items = own + CHIP;  // splits add at most one item a CU
  r.shared_items = B < 2 ? 0 : shared + CHIP;
  return r;
}

struct PlanArgs {
  PageRows r;
  DType dt;
  int Hkv, ncol, min_pages;
  int own_items, shared_items;  // room for
  int own_width, shared_width;
  int32_t* plan;
  int32_t *lead, *pages;  // nullable
};

constexpr int PLAN_THREADS = PAGE_SHARE_ROWS;  // a thread a row

template <class V>
__device__ __forceinline__ V plan_sum(V v, int* red) {
  V* r = reinterpret_cast<V*>(red);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 64; ++w) v += r[w];
  return v;
}
__device__ __forceinline__ int plan_scan(int v, int* red) {  // over the threads before this one
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(sum, o, 64);
    if (lane >= o) sum += t;
  }
  __syncthreads();
  if (lane == 63) red[wave] = sum;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 64; ++w) before += w < wave ? red[w] : 0;
  return before + sum - v;
}

// Key tiles of an item for a budget of q: the least number of equal runs of at most q.
__device__ __forceinline__ int splits_of(int tiles, int q) { return tiles > 0 ? (tiles + q - 1) / q : 0; }

// One block, a thread a row.
__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(PlanArgs a) {
  __shared__ int red[PLAN_THREADS / 64];
  __shared__ int s_common[PLAN_THREADS + 1], s_lead[PLAN_THREADS], s_least[PLAN_THREADS], s_rows[PLAN_THREADS];
  __shared__ int s_at_shared[PLAN_THREADS + 1], s_at_own[PLAN_THREADS + 1], s_alive;
  const int b = threadIdx.x, B = a.r.B;
  const bool mine = b < B;
  const int len = mine ? row_len(a.r, b) : 0, n = mine ? row_new(a.r, b) : 0;
  // whole pages that the row and the one before it could share, and those that they do
  s_rows[b] = len / PAGE;
  __syncthreads();
  const int most = mine && b > 0 ? min(s_rows[b], s_rows[b - 1]) : 0;
  s_common[b] = most;
  if (b == 0) s_alive = 0;
  __syncthreads();
  atomicMax(&s_alive, most);
  __syncthreads();
  // pages [p0, p0 + step) of every row at once, until no two rows share any further
  const int step = max(8 * PLAN_THREADS / B, 64);
  for (int p0 = 0; p0 < s_alive;) {
    const int width = min(step, s_alive - p0), total = (B - 1) * width;
    for (int i = b; i < total; i += PLAN_THREADS) {
      const int row = 1 + i / width, p = p0 + i % width;
      if (p < s_common[row]) {
        const int32_t* t = a.r.table + (size_t)row * a.r.max_pages + p;
        if (t[0] != t[-(long)a.r.max_pages]) atomicMin(&s_common[row], p);
      }
    }
    __syncthreads();
    p0 += width;
    if (b == 0) s_alive = 0;
    __syncthreads();
    if (s_common[b] >= p0 && mine && b > 0 && s_common[b] == most) atomicMax(&s_alive, most);
    __syncthreads();
  }
  // groups: runs of rows that share min_pages pages or more with the row before
  const int common = mine && s_common[b] >= a.min_pages ? s_common[b] : 0;
  s_lead[b] = common ? 0 : b;
  s_least[b] = 1 << 30;
  s_rows[b] = 0;
  __syncthreads();
  for (int o = 1; o < PLAN_THREADS; o <<= 1) {  // the last row at or before this one that begins a group
    const int v = b >= o ? max(s_lead[b], s_lead[b - o]) : s_lead[b];
    __syncthreads();
    s_lead[b] = v;
    __syncthreads();
  }
  const int lead = s_lead[b];
  if (mine) atomicAdd(&s_rows[lead], 1);
  if (common) atomicMin(&s_least[lead], common);
  __syncthreads();
  const int rows = mine ? s_rows[lead] : 0, shared = rows > 1 ? s_least[lead] : 0;
  if (mine && a.lead) a.lead[b] = lead;
  if (mine && a.pages) a.pages[b] = shared;

  // units (K/V head x tile of columns) and their key tiles, of the group (its first row's thread) and of the row
  const int np = (len + PAGE - 1) / PAGE;
  const int own_tiles = n > 0 ? np - shared + (n + PAGE - 1) / PAGE : 0;
  const int own_units = n > 0 ? a.Hkv * tiles_of(a.ncol, a.own_width) : 0;
  const int set = rows * a.ncol, set_width = width_of(a.dt, set);
  const int shared_units = mine && lead == b && shared > 0 ? a.Hkv * tiles_of(set, set_width) : 0;
  // the least budget of tiles an item that makes no more items than run at once, where the units allow that
  constexpr int LEAST = 4;
  const int units = plan_sum(own_units + shared_units, red);
  const float work = plan_sum((float)own_units * own_tiles + (float)shared_units * shared, red);
  const int longest = [&] {
    __syncthreads();
    if (b == 0) s_alive = LEAST;
    __syncthreads();
    atomicMax(&s_alive, max(own_tiles, shared_units ? shared : 0));
    __syncthreads();
    return s_alive;
  }();
  int q = max(LEAST, (int)fminf(ceilf(work / CHIP), 0x1p30f));
  if (units <= CHIP) {
    int lo = q, hi = max(q, longest);  // hi is enough
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      const int items = plan_sum(own_units * splits_of(own_tiles, mid) + shared_units * splits_of(shared, mid), red);
      if (items <= CHIP)
        hi = mid;
      else
        lo = mid + 1;
    }
    q = lo;
  }
  const int sp = shared_units ? splits_of(shared, q) : 0, so = own_units ? splits_of(own_tiles, q) : 0;
  const int at_shared = plan_scan(shared_units * sp, red), at_own = plan_scan(own_units * so, red);
  s_at_shared[b] = at_shared;
  s_at_own[b] = at_own;
  s_common[b] = sp;
  if (b == PLAN_THREADS - 1) {
    s_at_shared[b + 1] = at_shared + shared_units * sp;
    s_at_own[b + 1] = at_own + own_units * so;
  }
  __syncthreads();
  const int n_shared = min(s_at_shared[PLAN_THREADS], a.shared_items), n_own = min(s_at_own[PLAN_THREADS], a.own_items);
  if (b == 0) a.plan[0] = n_shared + n_own;
  const int group_splits = s_common[lead], group_at = s_at_shared[lead];
  RowParts* parts = reinterpret_cast<RowParts*>(a.plan + PLAN_HEAD / 4);
  if (mine)
    parts[b] = RowParts{group_splits ? lead : b, group_splits ? set : a.ncol, group_splits, group_at,
                        so == 1 && group_splits == 0 ? -1 : so, at_own, {0, 0}};
  s_lead[b] = shared;
  s_least[b] = so;
  // the items: shared pages first, being the longest; in a row or group, tiles of columns last (items of one head
  // and run of keys are a multiple of 8 apart where heads x splits is, and then run on one XCD)
  Item* items = reinterpret_cast<Item*>(parts + B);
  __syncthreads();
  for (int i = b; i < n_shared; i += PLAN_THREADS) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_at_shared[mid] <= i)
        lo = mid;
      else
        hi = mid;
    }
    const int splits = s_common[lo], tiles = s_lead[lo], x = i - s_at_shared[lo], per = a.Hkv * splits;
    const int s = x % splits, h = x / splits % a.Hkv;
    items[i] = Item{lo, s_rows[lo], h, x / per, width_of(a.dt, s_rows[lo] * a.ncol), (int)((long)tiles * s / splits),
                    (int)((long)tiles * (s + 1) / splits), tiles * PAGE, tiles, 0, i, 0};
  }
  for (int i = b; i < n_own; i += PLAN_THREADS) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_at_own[mid] <= i)
        lo = mid;
      else
        hi = mid;
    }
    const int splits = s_least[lo], x = i - s_at_own[lo], per = a.Hkv * splits;
    const int s = x % splits, h = x / splits % a.Hkv, row_l = row_len(a.r, lo), row_n = row_new(a.r, lo);
    const int first = s_lead[lo], pages = (row_l + PAGE - 1) / PAGE, tiles = pages - first + (row_n + PAGE - 1) / PAGE;
    const bool whole = splits == 1 && s_common[lo] == 0 && first == 0;
    items[n_shared + i] = Item{lo, 1, h, x / per, a.own_width, first + (int)((long)tiles * s / splits),
                               first + (int)((long)tiles * (s + 1) / splits), row_l, pages, row_n, whole ? -1 : i, 0};
  }
}

// Where the parts lie: O of the shared items, (m, l) of them, then those of the rows' own.
struct Parts {
  float *o_shared, *ml_shared, *o_own, *ml_own;
  int shared_width, own_width;
};

// An item as a block's work.
struct Strip {
  int b, rows, h, ct, n, len, np, t0, t1;
  size_t head;
  float *po, *pml;  // of the columns from the item's first on; null: the result
  int col0;
  __device__ __forceinline__ size_t column(const Args& a, int col) const {
    const int ncol = a.G * a.r.max_n, c = min(col, rows * ncol - 1);
    return rows == 1 ? head * ncol + c : ((size_t)(b + c / ncol) * a.p.Hkv + h) * ncol + c % ncol;
  }
  __device__ __forceinline__ bool wanted(const Args& a, int col) const {
    const int L = a.r.max_n, ncol = a.G * L;
    return rows == 1 ? col < ncol && col % L < n : col < rows * ncol && col % L < row_new(a.r, b + col / ncol);
  }
  __device__ __forceinline__ bool parts(const Args&) const { return po != nullptr; }
  __device__ __forceinline__ float* part_o(const Args& a, int col) const { return po + (size_t)(col - col0) * a.p.dh; }
  __device__ __forceinline__ float* part_ml(const Args&, int col) const { return pml + 2 * (col - col0); }
};
__device__ __forceinline__ Strip strip_of(const Args& a, const Item& i, const Parts& p, bool shared) {
  Strip s{i.b, i.rows, i.h, i.ct, i.n, i.len, i.np, i.t0, a.k ? i.t1 : min(i.t1, i.np), (size_t)i.b * a.p.Hkv + i.h,
          nullptr, nullptr, i.ct * i.width};
  const size_t at = (size_t)i.part * (shared ? p.shared_width : p.own_width);
  if (i.part >= 0) {
    s.po = (shared ? p.o_shared : p.o_own) + at * a.p.dh;
    s.pml = (shared ? p.ml_shared : p.ml_own) + at * 2;
  }
  return s;
}

struct SharedArgs {
  Args a;
  const int32_t* plan;
  Parts parts;
  int shared_items, own_items;
};

// The block's item; false for none, and for one that could not have come from a plan of such rows.
__device__ __forceinline__ bool item_of(const SharedArgs& s, Item& i) {
  if ((int)blockIdx.x >= s.plan[0]) return false;
  i = reinterpret_cast<const Item*>(s.plan + PLAN_HEAD / 4 + (sizeof(RowParts) / 4) * s.a.r.B)[blockIdx.x];
  const PageRows& r = s.a.r;
  const bool row = i.b >= 0 && i.rows >= 1 && i.rows <= r.B && i.b <= r.B - i.rows && (unsigned)i.h < (unsigned)s.a.p.Hkv;
  const bool keys = i.n >= 0 && i.n <= r.max_n && i.np >= 0 && i.np <= r.max_pages && i.t0 >= 0 && i.t1 <= i.np + (i.n + PAGE - 1) / PAGE;
  const bool part = i.part < (i.n ? s.own_items : s.shared_items) && i.width <= (i.n ? s.parts.own_width : s.parts.shared_width);
  return row && keys && part && i.ct >= 0 && (i.part >= 0 || i.rows == 1);
}

template <int NB>
__global__ __launch_bounds__(64 * F32_WAVES) void shared_f32_kernel(SharedArgs s) {
  __shared__ float xs[F32_WAVES * (2 + 4 * NB) * 64];
  Item i;
  if (!item_of(s, i)) return;
  f32_tiles<NB>(s.a, strip_of(s.a, i, s.parts, i.n == 0), xs);
}

constexpr int WAVES = 8;
// WIDE: sets of more than 32 columns occur.
template <int DH, bool WIDE>
__global__ __launch_bounds__(64 * WAVES, 2) void shared_bf16_kernel(SharedArgs s) {
  constexpr int FEW = WAVES * (2 + DH / 4) * 64 * 4;
  __shared__ __attribute__((aligned(16))) char smem[WIDE ? wide_lds<DH>() : FEW];
  static_assert(FEW <= wide_lds<DH>(), "the LDS of a block");
  Item i;
  if (!item_of(s, i)) return;
  const Strip x = strip_of(s.a, i, s.parts, i.n == 0);
  if (i.width == 16) return narrow_tiles<DH, 1, WAVES>(s.a, x, reinterpret_cast<float*>(smem));
  if (i.width == 32) return narrow_tiles<DH, 2, WAVES>(s.a, x, reinterpret_cast<float*>(smem));
  if constexpr (WIDE) {
    if (i.width == 64)
      wide_tiles<DH, 1, 4>(s.a, x, smem);
    else
      wide_tiles<DH, 2, 4>(s.a, x, smem);
  }
}

// Joins the parts of a column: 32 lanes, four values of the head width each.
template <class T>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs s) {
  const Args& a = s.a;
  const int i = threadIdx.x & 31, L = a.r.max_n, ncol = a.G * L, dh = a.p.dh, Hkv = a.p.Hkv;
  const size_t id = (size_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (id >= (size_t)a.r.B * Hkv * ncol) return;
  const int c = (int)(id % ncol), h = (int)(id / ncol % Hkv), b = (int)(id / ncol / Hkv), g = c / L, j = c % L;
  if (j >= row_new(a.r, b)) return;
  const RowParts p = reinterpret_cast<const RowParts*>(s.plan + PLAN_HEAD / 4)[b];
  if (p.own < 0) return;  // one item has written the result
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
  if (p.shared > 0) {
    const int at = (b - p.lead) * ncol + c, width = width_of(sizeof(T) == 2 ? BF16 : F32, p.columns);
    const int first = p.at_shared + (at / width * Hkv + h) * p.shared;
    if (first < 0 || first > s.shared_items - p.shared) return;
    size_t x = (size_t)first * s.parts.shared_width + at % width;
    for (int k = 0; k < p.shared; ++k, x += s.parts.shared_width) add(s.parts.ml_shared + 2 * x, s.parts.o_shared + x * dh + d);
  }
  const int first = p.at_own + (c / s.parts.own_width * Hkv + h) * p.own;
  if (first < 0 || first > s.own_items - p.own) return;
  size_t x = (size_t)first * s.parts.own_width + c % s.parts.own_width;
  for (int k = 0; k < p.own; ++k, x += s.parts.own_width) add(s.parts.ml_own + 2 * x, s.parts.o_own + x * dh + d);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.o) + (((size_t)b * L + j) * Hkv * a.G + h * a.G + g) * dh;
  if (4 * i < dh) store4(out + 4 * i, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
  if (i == 0 && a.lse) a.lse[id] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}

}  // namespace

size_t page_plan_bytes(DType dt, int B, int H, int Hkv, int L) {
  const Bounds w = bounds_of(dt, B, H, Hkv, L);
  return PLAN_HEAD + (size_t)B * sizeof(RowParts) + (size_t)(w.own_items + w.shared_items) * sizeof(Item);
}

size_t page_shared_threads(DType dt, int B, int H, int Hkv, int L) {
  const Bounds w = bounds_of(dt, B, H, Hkv, L);
  const size_t items = (size_t)(w.own_items + w.shared_items) * (dt == BF16 ? 64 * WAVES : 64 * F32_WAVES);
  const size_t join = (size_t)B * H * L * 32 + 256;
  return items > join ? items : join;
}

size_t page_shared_work(DType dt, int B, int H, int Hkv, int dh, int L) {
  const Bounds w = bounds_of(dt, B, H, Hkv, L);
  return (size_t)(w.own_items * w.own_width + w.shared_items * w.shared_width) * (dh + 2) * sizeof(float);
}

hipError_t page_plan(DType dt, const PageRows& r, int H, int Hkv, int min_pages, int32_t* plan, int32_t* lead,
                     int32_t* pages, hipStream_t s) {
  const Bounds w = bounds_of(dt, r.B, H, Hkv, r.max_n);
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s,
                     PlanArgs{r, dt, Hkv, H / Hkv * r.max_n, min_pages, (int)w.own_items, (int)w.shared_items, w.own_width,
                              w.shared_width, plan, lead, pages});
  return hipGetLastError();
}

hipError_t page_attend_shared(DType dt, const PageAttend& c, const int32_t* plan, hipStream_t s) {
  const int dh = c.p.dh, G = c.H / c.p.Hkv;
  const Bounds w = bounds_of(dt, c.r.B, c.H, c.p.Hkv, c.r.max_n);
  float* work = static_cast<float*>(c.work);
  const size_t shared = (size_t)w.shared_items * w.shared_width, own = (size_t)w.own_items * w.own_width;
  SharedArgs a{Args{c.p, c.r, c.q, c.k, c.vt, c.o, c.lse, nullptr, G, c.cap, 1, 1.4426950408889634f / sqrtf((float)dh)}, plan,
               Parts{work, work + (shared + own) * dh, work + shared * dh, work + (shared + own) * dh + 2 * shared, w.shared_width,
                     w.own_width},
               (int)w.shared_items, (int)w.own_items};
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
