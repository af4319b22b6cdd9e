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
// K and P are prefixes of the order, so each is one entry, its last (a cut).  It is found by digits: 2 048
// bins of z = 64 (m - l') first, of which the one where the running count or weight reaches its mark is looked
// into further, until what is left of it fits a list that is ranked entry by entry.
#include "common.h"
#include "kernels.h"
#include "sampler_math.h"

#pragma clang fp contract(off)

namespace tadm {
namespace {

typedef unsigned long long u64;
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // rows may begin at any float

constexpr int T = 1024, NW = T / 64;  // threads and waves of a block
constexpr int BINS = 2048, LIST = 1024;
constexpr int CELL = 256, CELLS = DRAW_MAX_VOCAB / CELL;  // a cell: the four entries of each lane of a wave
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

// m - l' as a number >= 0 with six binary places before the bins and eleven behind; its bins order as l' does
__device__ __forceinline__ float bin_of(float y) { return y * -64.f; }

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

struct Shared {
  u64 mass[BINS];
  uint32_t count[BINS];
  float list_x[LIST];
  int list_v[LIST];
  u64 list_q[LIST];
  u64 wave[NW];
  float wave_f[NW];
  Cut cut;
  u64 through;            // the weight of a prefix
  u64 before;             // what comes before the chosen bin: entries or weight
  uint32_t bin, size;     // the chosen bin, entries gathered
  int token;
  u64 chosen, total, rest;
};

__device__ __forceinline__ float block_max(float v, Shared& s) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) s.wave_f[threadIdx.x >> 6] = v;
  __syncthreads();
  v = s.wave_f[0];
  for (int w = 1; w < NW; ++w) v = fmaxf(v, s.wave_f[w]);
  return v;
}

// Sum over the threads before this one; all: over every one.
__device__ __forceinline__ u64 block_scan(u64 v, u64* wave, u64* all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  u64 sum = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 t = __shfl_up(sum, o, 64);
    if (lane >= o) sum += t;
  }
  __syncthreads();
  if (lane == 63) wave[w] = sum;
  __syncthreads();
  u64 before = 0, total = 0;
  for (int i = 0; i < NW; ++i) {
    before += i < w ? wave[i] : 0;
    total += wave[i];
  }
  *all = total;
  return before + sum - v;
}

// The bin at which the running sum over the bins reaches `mark` >= 1 (no more than the sum of all); s.bin and
// s.before (the sum of the bins before it).
template <class H>
__device__ __forceinline__ void choose_bin(const H* hist, u64 mark, Shared& s) {
  const int i = 2 * threadIdx.x;
  const u64 a = hist[i], b = hist[i + 1];
  u64 all;
  const u64 before = block_scan(a + b, s.wave, &all);
  if (before < mark && before + a + b >= mark) {
    const bool second = before + a < mark;
    s.bin = i + second;
    s.before = before + (second ? a : 0);
  }
  __syncthreads();
}

// A row of logits.  PER > 0: V <= T PER, each thread keeps its PER entries l' in registers; else every pass
// reads them again.  Thread t has the quads t, t + T, ...: a wave's quads of one round are a cell.
template <int PER>
struct Row {
  const float* lg;
  int V;
  float inv;
  float x[PER > 0 ? PER : 1];

  __device__ __forceinline__ f32x4 load(int v) const {
    f32x4 a;
    if (v + 3 < V) {
      a = *reinterpret_cast<const f32x4u*>(lg + v);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = v + e < V ? lg[v + e] : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = a[e] * inv;
      a[e] = p == p ? p : -INFINITY;
    }
    return a;
  }
  __device__ __forceinline__ void read() {
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER / 4; ++j) {
        const f32x4 a = load(4 * ((int)threadIdx.x + T * j));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * j + e] = a[e];
      }
    }
  }
  // f(cell, first entry, four l') for the thread's quads; every thread of the block goes through the same rounds
  template <class F>
  __device__ __forceinline__ void quads(F f) const {
    const int wave = threadIdx.x >> 6;
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER / 4; ++j)
        if (4 * T * j < V)
          f(NW * j + wave, 4 * ((int)threadIdx.x + T * j), f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]});
    } else {
      constexpr int AHEAD = 4;
      for (int j0 = 0; 4 * T * j0 < V; j0 += AHEAD) {
        f32x4 a[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) a[i] = load(4 * ((int)threadIdx.x + T * (j0 + i)));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          if (4 * T * (j0 + i) < V) f(NW * (j0 + i) + wave, 4 * ((int)threadIdx.x + T * (j0 + i)), a[i]);
      }
    }
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    quads([&](int, int v, const f32x4& a) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(a[e], v + e);
    });
  }
};

// l' - m; entries that are -inf or lie past the row weigh nothing
__device__ __forceinline__ float below(float x, float m) { return x == m ? 0.f : x - m; }
constexpr float Y_MIN = -30.f;  // own_exp_term is 0 at and below

// The cut at which the running count (COUNT) or weight over the order reaches `mark`; s.cut, and s.through the
// weight of the prefix that it ends (only if `masses`).  The bins of level 0 are filled; `in` tells the entries that take part.
template <bool COUNT, class R, class In>
__device__ void find_cut(const R& row, float m, u64 mark, bool masses, In in, Shared& s) {
  const int tid = threadIdx.x;
  uint32_t prefix[LEVELS];
  u64 before_mass = 0;
  for (int level = 0;; ++level) {
    if (level > 0) {  // the bins of what the digits so far have left
      for (int i = tid; i < BINS; i += T) {
        s.mass[i] = 0;
        s.count[i] = 0;
      }
      __syncthreads();
      row.each([&](float x, int v) {
        const float y = below(x, m);
        if (!(y > Y_MIN) || !in(x, v)) return;
        for (int l = 0; l < level; ++l)
          if (digit(l, x, y, v) != prefix[l]) return;
        const u64 q = (u64)own_exp_term(y);
        if (q == 0) return;
        const uint32_t d = digit(level, x, y, v);
        if (COUNT) atomicAdd(&s.count[d], 1u);
        if (masses) atomicAdd(&s.mass[d], q);
      });
      __syncthreads();
    }
    if (COUNT)
      choose_bin(s.count, mark, s);
    else
      choose_bin(s.mass, mark, s);
    const uint32_t bin = s.bin;
    prefix[level] = bin;
    mark -= s.before;
    if (masses) {
      u64 sum = 0, all;
      for (int i = tid; i < BINS; i += T) sum += (uint32_t)i < bin ? s.mass[i] : 0;
      block_scan(sum, s.wave, &all);
      before_mass += all;
    }
    if (tid == 0) s.size = 0;
    __syncthreads();
    row.each([&](float x, int v) {
      const float y = below(x, m);
      if (!(y > Y_MIN) || !in(x, v)) return;
      for (int l = 0; l <= level; ++l)
        if (digit(l, x, y, v) != prefix[l]) return;
      const u64 q = (u64)own_exp_term(y);
      if (q == 0) return;
      const uint32_t at = atomicAdd(&s.size, 1u);
      if (at < LIST) {
        s.list_x[at] = x;
        s.list_v[at] = v;
        s.list_q[at] = q;
      }
    });
    __syncthreads();
    if (s.size <= LIST || level == LEVELS - 1) break;
  }
  const int n = min((int)s.size, LIST);
  if (tid < n) {
    const Cut mine{s.list_x[tid], s.list_v[tid]};
    u64 weight = 0;
    uint32_t rank = 0;
    for (int i = 0; i < n; ++i)
      if (i != tid && mine.has(s.list_x[i], s.list_v[i])) {
        ++rank;
        weight += s.list_q[i];
      }
    const u64 q = s.list_q[tid];
    if (COUNT ? rank + 1 == mark : weight < mark && weight + q >= mark) {
      s.cut = mine;
      s.through = before_mass + weight + q;
    }
  }
  __syncthreads();
}

// One block a row.
template <int PER>
__global__ __launch_bounds__(T) void draw_kernel(DrawRows d) {
  __shared__ Shared s;
  __shared__ double cell[CELLS];
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Settings set = settings_of(d, r);
  Row<PER> row{d.logits + (size_t)r * d.ld, d.V, set.inv, {}};
  row.read();
  float m = -INFINITY;
  row.each([&](float x, int) { m = fmaxf(m, x); });
  m = block_max(m, s);
  if (m == -INFINITY) {  // nothing to draw from
    if (tid == 0) {
      d.token[r] = -1;
      if (d.logp) d.logp[r] = -INFINITY;
    }
    return;
  }
  if (set.k == 1) {  // the first entry of the order
    if (tid == 0) s.token = d.V;
    __syncthreads();
    int first = d.V;
    row.each([&](float x, int v) {
      if (x == m) first = min(first, v);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
    if (lane == 0) atomicMin(&s.token, first);
    __syncthreads();
    if (tid == 0) {
      d.token[r] = s.token;
      if (d.logp) d.logp[r] = 0.f;
    }
    return;
  }
  const bool top_k = set.k < d.V, top_p = set.p < 1u << 24;
  Cut cut{-INFINITY, d.V};
  if (top_k || top_p) {
    for (int i = tid; i < BINS; i += T) {
      s.mass[i] = 0;
      s.count[i] = 0;
    }
    __syncthreads();
    row.each([&](float x, int) {
      const float y = below(x, m);
      if (!(y > Y_MIN)) return;
      const u64 q = (u64)own_exp_term(y);
      if (q == 0) return;
      const uint32_t bin = (uint32_t)bin_of(y);
      if (top_k) atomicAdd(&s.count[bin], 1u);
      if (top_p) atomicAdd(&s.mass[bin], q);
    });
    __syncthreads();
    u64 entries, Q;
    block_scan((u64)s.count[2 * tid] + s.count[2 * tid + 1], s.wave, &entries);
    block_scan(s.mass[2 * tid] + s.mass[2 * tid + 1], s.wave, &Q);
    if (top_k && entries > (u64)set.k) {
      find_cut<true>(row, m, (u64)set.k, top_p, [](float, int) { return true; }, s);
      cut = s.cut;
      Q = s.through;
      __syncthreads();
    }
    if (top_p) {
      const Cut k = cut;
      if (k.x > -INFINITY) {  // the bins of K: find_cut has used them
        for (int i = tid; i < BINS; i += T) s.mass[i] = 0;
        __syncthreads();
        row.each([&](float x, int v) {
          const float y = below(x, m);
          if (!(y > Y_MIN) || !k.has(x, v)) return;
          const u64 q = (u64)own_exp_term(y);
          if (q) atomicAdd(&s.mass[(uint32_t)bin_of(y)], q);
        });
        __syncthreads();
      }
      find_cut<false>(row, m, share_of(set.p, Q, true), true, [&](float x, int v) { return k.has(x, v); }, s);
      cut = s.cut;
    }
  }
  // F's weight by cells of 256 entries, then the cell and the entry at which it reaches the mark
  auto weight = [&](float x, int v) {
    const float y = below(x, m);
    const float q = cut.has(x, v) ? own_exp_term(y) : 0.f;
    return q >= set.q_min ? q : 0.f;
  };
  for (int i = tid; i < CELLS; i += T) cell[i] = 0.0;
  __syncthreads();
  row.quads([&](int c, int v, const f32x4& a) {
    double q = 0.0;  // whole numbers up to 2^48: exact
#pragma unroll
    for (int e = 0; e < 4; ++e) q += (double)weight(a[e], v + e);
    q = row16_sum(q);
    q += xor16(q);
    q += xor32(q);
    if (lane == 0) cell[c] = q;
  });
  __syncthreads();
  static_assert(CELLS == T, "a thread a cell");
  const u64 mine = (u64)cell[tid];
  u64 total;
  const u64 before = block_scan(mine, s.wave, &total);
  const float u = d.u[r];
  const u64 mark = share_of(u > 0.f ? (u64)fminf(floorf(u * 0x1p24f), 0x1p24f - 1.f) : 0ull, total, false);
  if (before <= mark && before + mine > mark) {
    s.token = tid * CELL;
    s.rest = mark - before;
  }
  __syncthreads();
  if (wave == 0) {
    const int v = s.token + 4 * lane;
    f32x4 a = row.load(v);
    u64 q[4], sum = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[e] = (u64)weight(a[e], v + e);
      sum += q[e];
    }
    u64 upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const u64 t = __shfl_up(upto, o, 64);
      if (lane >= o) upto += t;
    }
    u64 run = upto - sum;
    const u64 rest = s.rest;
    if (run <= rest && upto > rest) {
      int e = 0;
      while (run + q[e] <= rest) run += q[e++];
      u64 chosen = q[0];
      for (int i = 1; i < 4; ++i) chosen = i == e ? q[i] : chosen;
      d.token[r] = v + e;
      if (d.logp) d.logp[r] = (float)log((double)chosen / (double)total);
    }
  }
}

}  // namespace

hipError_t draw_rows(const DrawRows& d, hipStream_t s) {
  if (d.V <= 16 * T)
    hipLaunchKernelGGL(draw_kernel<16>, dim3(d.R), dim3(T), 0, s, d);
  else if (d.V <= 32 * T)
    hipLaunchKernelGGL(draw_kernel<32>, dim3(d.R), dim3(T), 0, s, d);
  else
    hipLaunchKernelGGL(draw_kernel<0>, dim3(d.R), dim3(T), 0, s, d);
  return hipGetLastError();
}

}  // namespace tadm
