// Attention of a window of queries over the paged 8-bit K/V store.
//
//   O = softmax(q K^T / sqrt(dh)) V over the committed positions of a row (e4m3 codes with
//   one scale per page and head) followed by the window's own keys in the model type.
//
// The queries of the G = H / Hkv heads that share a K/V head are one set of G L columns (they
// lie one after the other in memory), so that a page is read once for all of them.  Scores
// are computed transposed, S^T = K Q^T, a lane owning one column; the running maximum and sum
// of the softmax live in the lane, and the probabilities feed O^T = V^T P^T from registers.
// The order of the keys within a page is free (a sum over them), and so is that of the head
// width within a score: each kernel takes the orders that its loads of K and V^T like best.
//
// Three kernels: float32 models; bf16 with few columns, where each wave takes tiles of 64 keys
// of its own straight from memory (the pages' bytes bound it); bf16 with many, where tiles
// go through LDS for the waves of a block (the matrix cores and the exponentials bound it).
// The key axis is split over S blocks when the columns alone leave the chip empty; the
// partial results (m, l, unnormalised O) are joined in the order of the splits.
#include "page_tiles.h"

namespace tadm {
namespace {

__device__ __forceinline__ float* part_o(const Args& a, size_t col, int split) {
  return a.part + (col * a.S + split) * a.p.dh;
}
__device__ __forceinline__ float* part_ml(const Args& a, size_t col, int split) {
  const size_t cols = (size_t)a.r.B * a.p.Hkv * a.G * a.r.max_n;
  return a.part + cols * a.S * a.p.dh + (col * a.S + split) * 2;
}

// What a block works on: columns [ct * width, ...) of K/V head h of row b, split sp of its tiles.
// Column tiles are fastest, so that the blocks that read the same pages run on one XCD.
struct Block {
  int b, h, ct, sp, n, len, np, t0, t1;  // tiles [t0, t1): pages below np, the window's from np on
  size_t head;
  __device__ __forceinline__ size_t column(const Args& a, int col) const {
    const int ncol = a.G * a.r.max_n;
    return head * ncol + min(col, ncol - 1);
  }
  __device__ __forceinline__ bool wanted(const Args& a, int col) const {
    const int L = a.r.max_n;
    return col < a.G * L && col % L < n;
  }
  __device__ __forceinline__ bool parts(const Args& a) const { return a.S > 1; }
  __device__ __forceinline__ float* part_o(const Args& a, int col) const {
    return tadm::part_o(a, head * (a.G * a.r.max_n) + col, sp);
  }
  __device__ __forceinline__ float* part_ml(const Args& a, int col) const {
    return tadm::part_ml(a, head * (a.G * a.r.max_n) + col, sp);
  }
};
__device__ __forceinline__ Block block_of(const Args& a, int width) {
  const int nct = (a.G * a.r.max_n + width - 1) / width, id = xcd_contiguous(blockIdx.x, gridDim.x);
  Block x;
  x.ct = id % nct;
  x.sp = (id / nct) % a.S;
  x.h = (id / nct / a.S) % a.p.Hkv;
  x.b = id / nct / a.S / a.p.Hkv;
  x.n = row_new(a.r, x.b);
  x.len = row_len(a.r, x.b);
  x.np = (x.len + PAGE - 1) / PAGE;
  const int nt = x.np + (a.k ? (x.n + PAGE - 1) / PAGE : 0);
  x.t0 = (int)((long)nt * x.sp / a.S);
  x.t1 = (int)((long)nt * (x.sp + 1) / a.S);
  x.head = (size_t)x.b * a.p.Hkv + x.h;
  return x;
}

template <int NB>
__global__ __launch_bounds__(64 * F32_WAVES) void attend_f32_kernel(Args a) {
  __shared__ float xs[F32_WAVES * (2 + 4 * NB) * 64];
  const Block x = block_of(a, 16);
  if (x.n) f32_tiles<NB>(a, x, xs);
}
template <int DH, int QS, int NW>
__global__ __launch_bounds__(64 * NW) void attend_narrow_kernel(Args a) {
  __shared__ float xs[NW * (2 + DH / 4) * 64];
  const Block x = block_of(a, 16 * QS);
  if (x.n) narrow_tiles<DH, QS, NW>(a, x, xs);
}
template <int DH, int QS, int CW>
__global__ __launch_bounds__(128 * CW, 2) void attend_wide_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char smem[wide_lds<DH>()];
  const Block x = block_of(a, 16 * QS * CW);
  if (x.n) wide_tiles<DH, QS, CW>(a, x, smem);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
// Joins the splits of a column: GROUPS groups of 32 lanes, four values of the head width a lane, take every
// GROUPS-th split and are summed in order; a block has eight groups.
template <class T, int GROUPS>
__global__ __launch_bounds__(256) void join_kernel(Args a) {
  __shared__ float xs[GROUPS > 1 ? GROUPS : 1][132];
  const int i = threadIdx.x & 31, g8 = threadIdx.x / 32 % GROUPS;
  const int L = a.r.max_n, ncol = a.G * L, dh = a.p.dh;
  const size_t cols = (size_t)a.r.B * a.p.Hkv * ncol, id = (size_t)blockIdx.x * (8 / GROUPS) + threadIdx.x / (32 * GROUPS);
  const size_t col_id = id < cols ? id : cols - 1;
  const int col = (int)(col_id % ncol), g = col / L, j = col % L;
  const int b = (int)(col_id / ncol / a.p.Hkv), h = (int)(col_id / ncol % a.p.Hkv);
  const bool mine = id < cols && j < row_new(a.r, b);
  if (GROUPS == 8 && !mine) return;  // the whole block
  const float* ml = part_ml(a, col_id, 0);
  const float* po = part_o(a, col_id, 0) + (4 * i < dh ? 4 * i : 0);
  // the group's first splits are on their way while the maximum waits for its loads
  constexpr int AHEAD = 4;
  f32x4 v[AHEAD];
  f32x2 w[AHEAD];
#pragma unroll
  for (int e = 0; e < AHEAD; ++e) {
    const int s = min(g8 + GROUPS * e, a.S - 1);
    v[e] = *reinterpret_cast<const f32x4*>(po + (size_t)s * dh);
    w[e] = *reinterpret_cast<const f32x2*>(ml + 2 * s);
  }
  float m = M_NONE;
  for (int s = i; s < a.S; s += 32) m = fmaxf(m, ml[2 * s]);
  m = row16_max(m);
  m = fmaxf(m, xor16(m));
  float r[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
  auto add = [&](const f32x4& v, const f32x2& w) {
    const float f = __builtin_amdgcn_exp2f(w[0] - m);
    sum += w[1] * f;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] += v[e] * f;
  };
#pragma unroll
  for (int e = 0; e < AHEAD; ++e)
    if (g8 + GROUPS * e < a.S) add(v[e], w[e]);
#pragma unroll 4
  for (int s = g8 + GROUPS * AHEAD; s < a.S; s += GROUPS)
    add(*reinterpret_cast<const f32x4*>(po + (size_t)s * dh), *reinterpret_cast<const f32x2*>(ml + 2 * s));
  if constexpr (GROUPS > 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) xs[g8][4 * i + e] = r[e];
    if (i == 0) xs[g8][128] = sum;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = 0.f;
#pragma unroll
    for (int v = 0; v < GROUPS; ++v) {
      sum += xs[v][128];
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] += xs[v][4 * i + e];
    }
  }
  if (!mine) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(a.o) + (((size_t)b * L + j) * a.p.Hkv * a.G + h * a.G + g) * dh;
  if (4 * i < dh) store4(out + 4 * i, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
  if (i == 0 && a.lse) a.lse[col_id] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}
// Eight groups a column from 9 splits on, where the loads of one group in a row are what takes time (96 columns
// of 16 splits: 15.3 us with one group, 14.6 with eight, the attention included); else one, which
// needs an eighth of the blocks (2 048 columns of 8 splits: 18.5 with one, 20.8 with eight; 16 columns of 8:
// 10.0 and 9.9).  Bound by its launch and two loads behind one another.
template <class T>
void start_join(const Args& a, hipStream_t s) {
  const size_t cols = (size_t)a.r.B * a.p.Hkv * a.G * a.r.max_n;
  if (a.S > 8)
    hipLaunchKernelGGL((join_kernel<T, 8>), dim3((unsigned)cols), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((join_kernel<T, 1>), dim3((unsigned)((cols + 7) / 8)), dim3(256), 0, s, a);
}

constexpr int NARROW_WAVES = 8;  // of a block with few columns, as of one with many

// Which kernel a call takes: columns of a block, splits of the key axis, and the blocks in all.
struct Plan {
  int width, S;
  long blocks;
};

// Measured on one MI355X, in us a call with everything around it:
//  - Many columns: blocks of 128 or of 64, whichever needs less for its rounds of 256 blocks.  With 128 elements a key
//    a round of 128 columns takes as long as one and a half of 64 (16 heads, over 1 000 positions, in
//    rounds of 128 against of 64: 5 rows x 192 tokens, 1 : 1, 30.7 and 21.6; 10 x 100, 1 : 2, 28.2 and 37.9; 9 x 160,
//    2 : 2, 59 and 41; 16 x 192, 2 : 3, 60.3 and 60.7; 12 x 320, 3 : 4, 93 and 85; 16 x 320, 3 : 5, 96 and 106);
//    with 64, where a CU holds two of the narrower, as long as two (12 heads: 8 x 128, 1 : 1, 21.5 and 13.7; 16 x 128,
//    1 : 2, 19.5 and 20.7; 16 x 256, 2 : 3, 39.3 and 32.5; 10 x 512, 2 : 4, 45 and 46; 15 x 340, 3 : 5, 62 and 52).
//  - At most a block per CU in all: 16 tokens over 8 192 positions (256 blocks) take 81, and 95 in two splits;
//    1 token over 131 000 29 in 64 splits of 4 blocks, 33 in 32, and 34 in 128.  All with 128 elements a key; with
//    64 a CU has room for two blocks, and with 129 to 255 blocks a part of the chip is left empty: neither was
//    tried with more splits.
//  - Few columns: a split has two tiles of 128 or four of 64 elements a key, from 9 and 25 tiles on (1 token,
//    16/4 heads x 128, over 8 000 positions: 12.7 in 16 splits, 10.7 in 32 and 64; over 1 000, 13.7 in one and
//    10.2 in 8; over 300, 8.5 in one and 10.2 in two;
//    12 heads x 64 over 1 000 positions, 17 tiles: 8.0 in one, 9.3 in 16).
//  - Many: a split has four tiles, two steps of its two groups, from 13 tiles on (64 tokens, 16/4 heads x 128, over
//    750 positions: 16.3 in one split, 14.7 in four; over 500, 13.4 and 13.9; 32/16 heads over 4 000: 51 in
//    one, 25.6 in four, 22.5 in 8; 12 heads x 64 over 4 000: 35 in one, 13.8 in 16; 2 rows over 500: 9.7
//    in one, 12.4 in four).
Plan plan(DType dt, int B, int H, int Hkv, int dh, int L, int max_len) {
  const int ncol = H / Hkv * L;
  const int tiles = (max_len + PAGE - 1) / PAGE + (L + PAGE - 1) / PAGE;
  auto blocks = [&](int width) { return (long)B * Hkv * ((ncol + width - 1) / width); };
  Plan p{16, 1, 0};
  long most = tiles > 8 ? tiles / 4 : 1;  // float32
  if (dt == BF16 && ncol > 32) {
    auto rounds = [&](int width) { return (blocks(width) + 255) / 256; };
    p.width = dh > 64 ? (3 * rounds(128) <= 2 * rounds(64) ? 128 : 64) : (2 * rounds(128) <= rounds(64) ? 128 : 64);
    most = tiles > 12 ? tiles / 4 : 1;
  } else if (dt == BF16) {
    p.width = ncol > 16 ? 32 : 16;
    most = dh > 64 ? (tiles > 8 ? tiles / 2 : 1) : (tiles > 24 ? tiles / 4 : 1);
  }
  long S = 256 / blocks(p.width);
  S = S < most ? S : most;
  p.S = S < 1 ? 1 : (int)S;
  p.blocks = blocks(p.width) * p.S;
  return p;
}

template <typename K>
void start(K kernel, const Args& a, const Plan& p, int threads, hipStream_t s) {
  launch_timed(kernel, dim3((unsigned)p.blocks), dim3(threads), 0, s, a);
}

template <int DH>
void start_bf16(const Args& a, const Plan& p, hipStream_t s) {
  switch (p.width) {
    case 128: return start(attend_wide_kernel<DH, 2, 4>, a, p, 512, s);
    case 64: return start(attend_wide_kernel<DH, 1, 4>, a, p, 512, s);
    case 32: return start(attend_narrow_kernel<DH, 2, NARROW_WAVES>, a, p, 64 * NARROW_WAVES, s);
    default: return start(attend_narrow_kernel<DH, 1, NARROW_WAVES>, a, p, 64 * NARROW_WAVES, s);
  }
}

}  // namespace

size_t page_attend_threads(DType dt, int B, int H, int Hkv, int dh, int L, int max_len) {
  return (size_t)plan(dt, B, H, Hkv, dh, L, max_len).blocks * (dt == BF16 ? 64 * NARROW_WAVES : 256);
}

size_t page_attend_work(DType dt, int B, int H, int Hkv, int dh, int L, int max_len) {
  const Plan pl = plan(dt, B, H, Hkv, dh, L, max_len);
  return pl.S > 1 ? (size_t)B * H * L * pl.S * (dh + 2) * sizeof(float) : 0;
}

hipError_t page_attend(DType dt, const PageAttend& c, hipStream_t s) {
  const int dh = c.p.dh;
  const Plan pl = plan(dt, c.r.B, c.H, c.p.Hkv, dh, c.r.max_n, c.r.max_len);
  Args a{c.p, c.r, c.q, c.k, c.vt, c.o, c.lse, static_cast<float*>(c.work), c.H / c.p.Hkv, c.cap, pl.S,
         1.4426950408889634f / sqrtf((float)dh)};
  if (dt == BF16) {
    if (dh == 128)
      start_bf16<128>(a, pl, s);
    else if (dh == 64)
      start_bf16<64>(a, pl, s);
    else
      return hipErrorInvalidValue;
  } else {
    switch ((dh + 15) / 16) {
      case 1: start(attend_f32_kernel<1>, a, pl, 256, s); break;
      case 2: start(attend_f32_kernel<2>, a, pl, 256, s); break;
      case 3: start(attend_f32_kernel<3>, a, pl, 256, s); break;
      case 4: start(attend_f32_kernel<4>, a, pl, 256, s); break;
      case 5: start(attend_f32_kernel<5>, a, pl, 256, s); break;
      case 6: start(attend_f32_kernel<6>, a, pl, 256, s); break;
      case 7: start(attend_f32_kernel<7>, a, pl, 256, s); break;
      case 8: start(attend_f32_kernel<8>, a, pl, 256, s); break;
      default: return hipErrorInvalidValue;
    }
  }
  if (pl.S > 1) {
    if (dt == BF16)
      start_join<bf16>(a, s);
    else
      start_join<float>(a, s);
  }
  return hipGetLastError();
}

}  // namespace tadm
