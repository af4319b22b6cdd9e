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
#include "common.h"
#include "pages.h"

namespace tadm {
namespace {

constexpr float LN2 = 0.6931471805599453f;
constexpr int VM_DONE = 7 << 4 | 15 << 8;                      // s_waitcnt: no load outstanding
constexpr int SCHED_MFMA = 0x8, SCHED_LDS_READ = 0x100;        // instruction kinds of a schedule group

struct Args {
  PageLayer p;
  PageRows r;
  const void *q, *k, *vt;
  void* o;
  float* lse;
  float* part;  // S > 1: O [row, K/V head, column, split, dh], then (m, l) [row, K/V head, column, split, 2]
  int G, cap, S;
  float scale_log2;
};

__device__ __forceinline__ int row_len(const PageRows& r, int b) {
  return r.len ? min(max(r.len[b], 0), r.max_len) : r.max_len;
}
__device__ __forceinline__ int row_new(const PageRows& r, int b) {
  return r.n ? min(max(r.n[b], 0), r.max_n) : r.max_n;
}
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

// The key of a tile that row 4 grp + j of its i-th block of 16 scores stands for.  RUN: 16 keys in a row
// for a lane, one 16-byte load of the codes of a V^T row; else two runs of 8, 32 apart.
template <bool RUN>
__device__ __forceinline__ int key_of(int i, int grp, int j) {
  return RUN ? 16 * grp + 4 * i + j : 32 * (i >> 1) + 8 * grp + 4 * (i & 1) + j;
}

// One tile of a strip's softmax, in base 2.  s[i][j]: the score of key_of(i, grp, j), unscaled; on return
// its probability relative to a reference m of the column, that moves only when a score of the
// tile exceeds it by more than 8 (in base 2): until then the probabilities stay at 2^8 or below, and
// neither the sum l nor O need rescaling.  So most tiles need no maximum over the lanes of a column.
// M_NONE, below every finite score, is the reference before the first.
constexpr float M_NONE = -3.402823466e38f;
template <bool RUN, int NB>
__device__ __forceinline__ void softmax_tile(f32x4 (&s)[4], int keys, int grp, float scale_log2, float& m, float& l,
                                             f32x4 (&o)[NB]) {
  if (keys < PAGE) {
    asm volatile("" : "+s"(keys));  // the comparisons stay in here
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (key_of<RUN>(i, grp, j) >= keys) s[i][j] = -INFINITY;
  }
  float mt = s[0][0];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) mt = fmaxf(mt, s[i][j]);
  if (__builtin_amdgcn_ballot_w64(mt * scale_log2 > m + 8.f)) {
    mt = fmaxf(mt, xor16(mt));
    mt = fmaxf(mt, xor32(mt)) * scale_log2;
    const float m_new = mt > m + 8.f ? mt : m, alpha = __builtin_amdgcn_exp2f(m - m_new);
    l *= alpha;
    m = m_new;
#pragma unroll
    for (int d = 0; d < NB; ++d) o[d] *= alpha;
  }
  float ps = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][j], scale_log2, -m));
      ps += s[i][j];
    }
  l += ps;
}

// Stores 4 values of column col (head width d0 + [0, 4)) of a strip: part of a split, or the result.
template <class T>
__device__ __forceinline__ void put4(const Args& a, const Block& x, int col, int d0, float inv, const float* r) {
  if (a.S > 1) {
    store4(part_o(a, x.head * (a.G * a.r.max_n) + col, x.sp) + d0, r[0], r[1], r[2], r[3]);
  } else {
    const int L = a.r.max_n, g = col / L, j = col % L;
    T* out = static_cast<T*>(a.o) + (((size_t)x.b * L + j) * a.p.Hkv * a.G + x.h * a.G + g) * a.p.dh;
    store4(out + d0, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
  }
}
__device__ __forceinline__ void put_ml(const Args& a, const Block& x, int col, float m, float sum) {
  const size_t at = x.head * (a.G * a.r.max_n) + col;
  if (a.S > 1)
    store2(part_ml(a, at, x.sp), m, sum);
  else if (a.lse)
    a.lse[at] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}
__device__ __forceinline__ float inverse(const Args& a, float sum) { return a.S > 1 || sum == 0.f ? 0.f : 1.f / sum; }

// Joins NW waves that hold the same strip of 16 columns, in the order of the waves: per lane m,
// l and O in [wave][value][lane] floats; wave w sums the head-width blocks w, w + NW, ...
template <class T, int NB, int NW>
__device__ __forceinline__ void join_waves(const Args& a, const Block& x, int col, float m_run, float l_run,
                                           const f32x4 (&o)[NB], float* xs, int wave) {
  constexpr int NV = 2 + 4 * NB;
  const int lane = threadIdx.x & 63, grp = lane >> 4;
  float l = l_run + xor16(l_run);
  l += xor32(l);
  float* w = xs + wave * NV * 64 + lane;
  w[0] = m_run;
  w[64] = l;
#pragma unroll
  for (int d = 0; d < NB; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) w[(2 + 4 * d + j) * 64] = o[d][j];
  __syncthreads();
  const float* y = xs + lane;
  float m = M_NONE, f[NW], sum = 0.f;
#pragma unroll
  for (int v = 0; v < NW; ++v) m = fmaxf(m, y[v * NV * 64]);
#pragma unroll
  for (int v = 0; v < NW; ++v) {
    f[v] = __builtin_amdgcn_exp2f(y[v * NV * 64] - m);
    sum += y[v * NV * 64 + 64] * f[v];
  }
  const int L = a.r.max_n;
  if (col < a.G * L && col % L < x.n) {
    const float inv = inverse(a, sum);
    for (int d = wave; d < NB; d += NW) {
      float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < NW; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] += y[(v * NV + 2 + 4 * d + e) * 64] * f[v];
      if (16 * d + 4 * grp < a.p.dh) put4<T>(a, x, col, 16 * d + 4 * grp, inv, r);
    }
    if (wave == 0 && grp == 0) put_ml(a, x, col, m, sum);
  }
  __syncthreads();  // xs is free again
}

// bytes [0, keep) of a dword (keep may be negative or above 4)
__device__ __forceinline__ uint32_t keep_bytes(uint32_t v, int keep) {
  return keep >= 4 ? v : keep <= 0 ? 0u : v & ((1u << (8 * keep)) - 1u);
}

// ---------------------------------------------------------------- float32 models
// 4 codes (a dword) as floats times the scale
__device__ __forceinline__ f32x4 f32_codes(uint32_t c, float s) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
}

// Four waves on a strip of 16 columns, each taking every fourth tile; NB: head width in blocks of
// 16, the last of which may be partial.  Products and probabilities stay in float32.  float32 models are small
// (at most 4 096 positions of a window), and what bounds them is a launch and one tile's latency: 5 rows of
// 24 tokens over up to 333 positions, 4 heads x 16, 7.4 us, of which an empty launch takes 3.6.
template <int NB>
__global__ __launch_bounds__(256) void attend_f32_kernel(Args a) {
  constexpr int NW = 4;
  __shared__ float xs[NW * (2 + 4 * NB) * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15;
  const Block x = block_of(a, 16);
  if (x.n == 0) return;
  const int dh = a.p.dh, ncol = a.G * a.r.max_n, col = x.ct * 16 + fr;
  f32x4 qx[NB], o[NB];
  const float* q = static_cast<const float*>(a.q) + (x.head * ncol + min(col, ncol - 1)) * dh;
#pragma unroll
  for (int c = 0; c < NB; ++c) {
    qx[c] = 16 * c + 4 * grp < dh ? *reinterpret_cast<const f32x4*>(q + 16 * c + 4 * grp) : f32x4{0.f, 0.f, 0.f, 0.f};
    o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float m_run = M_NONE, l_run = 0.f;
  for (int t = x.t0 + wave; t < x.t1; t += NW) {
    const bool paged = t < x.np;
    const int keys = paged ? min(PAGE, x.len - t * PAGE) : min(PAGE, x.n - (t - x.np) * PAGE);
    const uint8_t* codes = nullptr;
    const float *sc = nullptr, *kw = nullptr, *vw = nullptr;
    if (paged) {
      const int page = a.r.table[(size_t)x.b * a.r.max_pages + t];
      if ((unsigned)page >= (unsigned)a.p.n_pages) continue;
      codes = a.p.data + (size_t)page * a.p.page_bytes + (size_t)x.h * 2 * PAGE * dh;
      sc = a.p.scale + (size_t)page * a.p.page_scales + 2 * x.h;
    } else {
      kw = static_cast<const float*>(a.k) + (x.head * a.cap + (size_t)(t - x.np) * PAGE) * dh;
      vw = static_cast<const float*>(a.vt) + x.head * dh * a.cap + (size_t)(t - x.np) * PAGE;
    }
    const float sk = paged ? sc[0] : 1.f, sv = paged ? sc[1] : 1.f;
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key_of<true>(i, fr >> 2, fr & 3);
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NB; ++c) {
        f32x4 kf = f32x4{0.f, 0.f, 0.f, 0.f};
        if (16 * c + 4 * grp < dh)
          kf = paged ? f32_codes(*reinterpret_cast<const uint32_t*>(codes + key * dh + 16 * c + 4 * grp), sk)
                     : *reinterpret_cast<const f32x4*>(kw + (size_t)key * dh + 16 * c + 4 * grp);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qx[c][e], s[i], 0, 0, 0);
      }
    }
    softmax_tile<true>(s, keys, grp, a.scale_log2, m_run, l_run, o);
    // V^T row 16 d + fr, keys 16 grp + [0, 16); what lies behind the last key is taken as 0, so
    // that p = 0 meets a finite value
#pragma unroll
    for (int d = 0; d < NB; ++d) {
      const int row = min(16 * d + fr, dh - 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 vf = paged ? f32_codes(*reinterpret_cast<const uint32_t*>(codes + PAGE * dh + row * PAGE + 16 * grp + 4 * i), sv)
                         : *reinterpret_cast<const f32x4*>(vw + (size_t)row * a.cap + 16 * grp + 4 * i);
        if (keys < PAGE)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (16 * grp + 4 * i + j >= keys) vf[j] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j], s[i][j], o[d], 0, 0, 0);
      }
    }
  }
  join_waves<float, NB, NW>(a, x, col, m_run, l_run, o, xs, wave);
}

// ---------------------------------------------------------------- bf16 models
// 8 codes as bf16 times the scale, exactly
__device__ __forceinline__ bf16x8 bf16_codes(uint32_t a, uint32_t b, float s) {
  const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false),
             p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true),
             p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false),
             p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true);
  return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
// A column's query.  RUN: a lane has DH / 4 elements in a row; else runs of 8, 32 apart.
template <int DH>
struct Query {
  bf16x8 op[DH / 32];
};
template <int DH, bool RUN>
__device__ __forceinline__ Query<DH> load_query(const bf16* q, int grp) {
  Query<DH> r;
#pragma unroll
  for (int c = 0; c < DH / 32; ++c)
    r.op[c] = *reinterpret_cast<const bf16x8*>(q + (RUN ? DH / 4 * grp + 8 * c : 32 * c + 8 * grp));
  return r;
}
// Waits for a query's loads here.  Left to its first use, inside the loop over the tiles, the wait would
// be for the tile's loads too, in every step.
template <int DH>
__device__ __forceinline__ void settle(Query<DH>& q) {
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) asm volatile("" : "+v"(q.op[c]));
}
// Scores of QS strips of 16 columns and 16 keys, from the lane's DH / 4 codes of the row it stands for.
// The codes become bf16, exactly, for the bf16 products: the 8-bit ones, twice as fast, drop
// what lies 2^-12 below the largest product of a sum.
template <int DH, int QS>
__device__ __forceinline__ void scores(const uint4 (&c)[DH / 64], float scale, const Query<DH> (&q)[QS], int i,
                                       f32x4 (&s)[QS][4]) {
#pragma unroll
  for (int u = 0; u < QS; ++u) s[u][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < DH / 32; ++e) {
    const uint4 w = c[e / 2];
    const bf16x8 k = e % 2 ? bf16_codes(w.z, w.w, scale) : bf16_codes(w.x, w.y, scale);
#pragma unroll
    for (int u = 0; u < QS; ++u) s[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[u].op[e], s[u][i], 0, 0, 0);
  }
}

// The tiles of pages that a wave takes, 64 at a time: lane l has the page, the keys and the scales
// of the (64 i + l)-th, so that a step finds them in a register.
struct TileBatch {
  int page, keys;
  float sk, sv;
};
__device__ __forceinline__ TileBatch tile_batch(const Args& a, const Block& x, int tile, int t1) {
  TileBatch r{0, 0, 1.f, 1.f};  // no keys: a tile of an absent page, or none (page 0 is read)
  if (tile < t1) {
    const int page = a.r.table[(size_t)x.b * a.r.max_pages + tile];
    if ((unsigned)page < (unsigned)a.p.n_pages) {
      const float* sc = a.p.scale + (size_t)page * a.p.page_scales + 2 * x.h;
      r = TileBatch{page, min(PAGE, x.len - tile * PAGE), sc[0], sc[1]};
    }
  }
  return r;
}
// Waits for a batch's loads here, as for a query's.
__device__ __forceinline__ void settle(TileBatch& b) {
  asm volatile("" : "+v"(b.page), "+v"(b.keys), "+v"(b.sk), "+v"(b.sv));
}
__device__ __forceinline__ int at_lane(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float at_lane(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Probabilities are rounded to bf16 here (at most 2^-8 of each, like the rounding of the result; the sum l has
// them unrounded), as attention over a bf16 context rounds them: against 64 bits the result's error is 0.0021 to
// 0.0023 of its norm where rounding the result alone leaves 0.0017.  float32 products are sixteen times
// slower.  f16 ones, as fast, would round a probability eight times finer, but their V would have to be f16 too: the
// window's bf16 values have a range that it lacks, and so have the scales (2^-110 to 2^120), which would
// have to meet the probabilities (out of their range as well) or, tile by tile, every element of O.
// Probabilities of a tile as the operand of O^T = V^T P^T: k index 8 grp + j of product c is the key of
// score row 4 grp + j % 4 of block 2 c + j / 4.
__device__ __forceinline__ void p_operand(const f32x4 (&s)[4], bf16x8 (&p)[2]) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) p[c][j] = (bf16)s[2 * c + j / 4][j % 4];
}

// A tile of the window's own keys (bf16), read from memory by the wave itself, for QS strips.
template <int DH, int QS>
__device__ __forceinline__ void window_tile(const Args& a, const Block& x, int w, const bf16* const (&q)[QS],
                                            f32x4 (&o)[QS][DH / 16], float (&m_run)[QS], float (&l_run)[QS]) {
  constexpr int NB = DH / 16;
  const int lane = threadIdx.x & 63, grp = lane >> 4, fr = lane & 15, keys = min(PAGE, x.n - w * PAGE);
  const bf16* kw = static_cast<const bf16*>(a.k) + (x.head * a.cap + (size_t)w * PAGE) * DH;
  const bf16* vw = static_cast<const bf16*>(a.vt) + x.head * DH * a.cap + (size_t)w * PAGE;
  f32x4 s[QS][4];
#pragma unroll
  for (int u = 0; u < QS; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[u][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < NB / 2; ++c) {
    bf16x8 qf[QS];
#pragma unroll
    for (int u = 0; u < QS; ++u) qf[u] = *reinterpret_cast<const bf16x8*>(q[u] + 32 * c + 8 * grp);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = key_of<true>(i, fr >> 2, fr & 3);
      const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kw + (size_t)key * DH + 32 * c + 8 * grp);
#pragma unroll
      for (int u = 0; u < QS; ++u) s[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[u], s[u][i], 0, 0, 0);
    }
  }
  // one strip: the values are on their way while the scores wait for theirs
  constexpr bool AHEAD = QS == 1;
  bf16x8 v[AHEAD ? NB : 1][2];
  if constexpr (AHEAD)
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        v[d][c] = *reinterpret_cast<const bf16x8*>(vw + (size_t)(16 * d + fr) * a.cap + 16 * grp + 8 * c);
  bf16x8 p[QS][2];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    softmax_tile<true>(s[u], keys, grp, a.scale_log2, m_run[u], l_run[u], o[u]);
    p_operand(s[u], p[u]);
  }
#pragma unroll
  for (int d = 0; d < NB; ++d)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      bf16x8 vf = v[AHEAD ? d : 0][c];
      if (!AHEAD) vf = *reinterpret_cast<const bf16x8*>(vw + (size_t)(16 * d + fr) * a.cap + 16 * grp + 8 * c);
      if (keys < PAGE)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (16 * grp + 8 * c + j >= keys) vf[j] = (bf16)0.f;
#pragma unroll
      for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[u][c], o[u][d], 0, 0, 0);
    }
}

// Few columns: NW waves on the same 16 QS columns, each taking every NW-th tile straight from
// memory into registers; the codes of the next tile are on their way while one is computed.
//
// Bound by the pages' bytes: no wave reads what another does, so LDS would only add a way, and
// with a tile on its way per wave eight waves keep 128 KB a CU outstanding (128 elements a key).  16 tokens
// over up to 8 192 positions, 32/16 heads x 128 (412 MB): 81 us, 5.1 TB/s, the rate of a copy of 1 GiB
// on the same card (row kernels that write less reach 6.0) (blocks of four waves took 101 where those of eight took 85).  1 token over 131 071
// positions, 16/4 heads x 128 (134 MB): 32 with the join of its splits, 26 at the copy's rate.  1 token over
// 200 positions: 7.7, of which an empty launch takes 3.6; the rest is loads that wait for one
// another (lengths and table, scales, codes, the window) and the join of the waves.
template <int DH, int QS, int NW>
__global__ __launch_bounds__(64 * NW) void attend_narrow_kernel(Args a) {
  constexpr int NB = DH / 16;
  __shared__ float xs[NW * (2 + 4 * NB) * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15;
  const Block x = block_of(a, 16 * QS);
  if (x.n == 0) return;
  const int ncol = a.G * a.r.max_n, tp = min(x.t1, x.np), first = x.t0 + wave;
  const int steps = first < tp ? (tp - first + NW - 1) / NW : 0;
  const bf16* q[QS];
  Query<DH> qs[QS];
  f32x4 o[QS][NB];
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    q[u] = static_cast<const bf16*>(a.q) + (x.head * ncol + min(x.ct * 16 * QS + 16 * u + fr, ncol - 1)) * DH;
    m_run[u] = M_NONE;
    l_run[u] = 0.f;
#pragma unroll
    for (int d = 0; d < NB; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  TileBatch tb = tile_batch(a, x, first + NW * lane, tp);
  const uint8_t* base = a.p.data + (size_t)x.h * 2 * PAGE * DH;
  const int koff = key_of<true>(0, fr >> 2, fr & 3) * DH + DH / 4 * grp;
  const int voff = PAGE * DH + fr * PAGE + 16 * grp;
  uint4 kc[4][DH / 64], vc[NB];
  auto load_k = [&](int page) {
    const uint8_t* c = base + (size_t)page * a.p.page_bytes + koff;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DH / 64; ++e) kc[i][e] = *reinterpret_cast<const uint4*>(c + 4 * i * DH + 16 * e);
  };
  auto load_v = [&](int page) {
    const uint8_t* c = base + (size_t)page * a.p.page_bytes + voff;
#pragma unroll
    for (int d = 0; d < NB; ++d) vc[d] = *reinterpret_cast<const uint4*>(c + 16 * d * PAGE);
  };
  if (steps) {
#pragma unroll
    for (int u = 0; u < QS; ++u) qs[u] = load_query<DH, true>(q[u], grp);
    const int first_page = at_lane(tb.page, 0);
    load_k(first_page);
    load_v(first_page);
#pragma unroll
    for (int u = 0; u < QS; ++u) settle<DH>(qs[u]);
    settle(tb);
    __builtin_amdgcn_s_waitcnt(VM_DONE);  // so that the waits in the loop count its own loads alone
    for (int st = 0; st < steps; ++st) {
      const int keys = at_lane(tb.keys, st & 63);
      const float sk = at_lane(tb.sk, st & 63), sv = at_lane(tb.sv, st & 63);
      if (((st + 1) & 63) == 0) {
        tb = tile_batch(a, x, first + NW * (st + 1 + lane), tp);
        settle(tb);
      }
      const int page = at_lane(tb.page, (st + 1) & 63);  // behind the last tile: page 0
      f32x4 s[QS][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) scores<DH, QS>(kc[i], sk, qs, i, s);
      load_k(page);
      bf16x8 p[QS][2];
#pragma unroll
      for (int u = 0; u < QS; ++u) {
        softmax_tile<true>(s[u], keys, grp, a.scale_log2, m_run[u], l_run[u], o[u]);
        p_operand(s[u], p[u]);
      }
      // V^T row 16 d + fr, keys 16 grp + [0, 16); what lies behind the last key is taken as 0, so
      // that p = 0 meets a finite value
      if (keys < PAGE)
#pragma unroll
        for (int d = 0; d < NB; ++d) {
          vc[d].x = keep_bytes(vc[d].x, keys - 16 * grp);
          vc[d].y = keep_bytes(vc[d].y, keys - 16 * grp - 4);
          vc[d].z = keep_bytes(vc[d].z, keys - 16 * grp - 8);
          vc[d].w = keep_bytes(vc[d].w, keys - 16 * grp - 12);
        }
#pragma unroll
      for (int d = 0; d < NB; ++d)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const bf16x8 vf = c ? bf16_codes(vc[d].z, vc[d].w, sv) : bf16_codes(vc[d].x, vc[d].y, sv);
#pragma unroll
          for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[u][c], o[u][d], 0, 0, 0);
        }
      load_v(page);
    }
  }
  for (int t = max(x.t0, x.np); t < x.t1; ++t)
    if ((t - x.t0) % NW == wave) window_tile<DH, QS>(a, x, t - x.np, q, o, m_run, l_run);
#pragma unroll
  for (int u = 0; u < QS; ++u)
    join_waves<bf16, NB, NW>(a, x, x.ct * 16 * QS + 16 * u + fr, m_run[u], l_run[u], o[u], xs, wave);
}

// Slot of chunk c (16 bytes) of a row of 128 or 256 bytes in LDS: c ^ swizzle(row).  With it, and lane
// group g at chunk 4 c + g, reads of 16 rows meet the banks evenly (4 cycles a wave, 8 with
// the groups' chunks side by side), and so do writes of a row's chunks by neighbouring lanes.
template <int ROW>
__device__ __forceinline__ int swizzle(int row) {
  static_assert(ROW == 128 || ROW == 256, "bytes of a row");
  return row & (ROW / 16 - 1);
}

// Many columns: two groups of CW waves work on the same 16 QS CW columns, each on every second tile of
// 64 keys, which its waves share through LDS.  The groups take turns: while one is at its
// matrix products (O += V^T P of the tile before, S = K Q^T of this one), the other is at its
// exponentials, so that each SIMD has a wave for its matrix core and one for its vector unit.
// A barrier of the whole block ends every such half step.  A step's V and the next one's K go to
// LDS beside the matrix products.
//
// Bound by the half steps, the products' against the exponentials': 4 rows of 256 tokens over 16 384
// positions, 32/16 heads x 128 (279 Gflop): 279 to 286 us, 979 to 1 000 TFLOP/s; at the 1 318 of a large
// library product 212.  A half step of products takes 2 060 to 2 340 cycles for 1 024 of matrix instructions a
// wave, one of exponentials 1 050 to 1 600, both stretched by the other group's instructions.
// Both groups at the same step took 331 where turns took 307, K placed beside the exponentials 296 where beside
// the products 290, a second tile ahead in registers 327 to 353.
//
// With 64 columns (QS = 1) a step takes 3 100 cycles, the moves to LDS alone 800 to 1 100: 16 rows x 64 tokens over
// up to 1 024 positions, 16/4 heads x 128: 19.6 us.  Keys of a tile halved between waves of 32
// columns (half the reads of LDS), a second tile ahead and K beside the exponentials: 20.2 to 21.9.
//
// The codes of a tile are converted to bf16, scaled, on their way to LDS, once for all waves
// (with codes in LDS, converted by every wave, the step took 8 % more), the values 0 behind the
// last key, so that p = 0 meets a finite value.  K row r has the key that score row r % 16 of
// block r / 16 stands for.
template <int DH, int QS, int CW>
__global__ __launch_bounds__(128 * CW, 2) void attend_wide_kernel(Args a) {
  constexpr int NB = DH / 16, KC = DH / 8, NV = 2 + 4 * NB, GT = 64 * CW;
  constexpr int SIDE = PAGE * DH, BUF = 2 * SIDE, GROUP = 4 * BUF;  // codes of a side, and its bf16; K, K, V, V
  constexpr int PER = SIDE / 8 / GT;                               // chunks (8 codes) of a side that a lane moves per tile
  constexpr int KROWS = GT / KC, VROWS = GT / 8;                   // rows of K and V^T that a group moves at once
  static_assert(PER * 8 * GT == SIDE && CW == 4, "a tile splits over the lanes of a group in whole blocks of 16 keys");
  static_assert(2 * CW * NV * 64 * 4 <= 2 * GROUP, "the groups are joined in the space of the tiles");
  __shared__ __attribute__((aligned(16))) char smem[2 * GROUP];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15, cw = wave % CW, kw = wave / CW, gl = cw * 64 + lane;
  const Block x = block_of(a, 16 * QS * CW);
  if (x.n == 0) return;
  const int ncol = a.G * a.r.max_n, col0 = (x.ct * CW + cw) * 16 * QS;
  const int tp = min(x.t1, x.np);
  const int steps = x.t0 < tp ? (tp - x.t0 + 1) / 2 : 0;  // of both groups; the second may have no tile in the last
  Query<DH> qs[QS];
  f32x4 o[QS][NB], s[QS][4];
  bf16x8 p[QS][2];
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    m_run[u] = M_NONE;
    l_run[u] = 0.f;
#pragma unroll
    for (int d = 0; d < NB; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // the lane's chunks of a tile: the j-th is KROWS j rows of K, VROWS j rows of V^T after the first
  const uint8_t* base = a.p.data + (size_t)x.h * 2 * PAGE * DH;
  char* const sb = smem + kw * GROUP;
  const int kr = gl / KC, vr = gl / 8;
  auto k_first = [&](int l) { return key_of<false>(l / KC >> 4, l / KC >> 2 & 3, l / KC & 3) * DH + l % KC * 8; };
  const int k_src = k_first(gl);
  const int k_dst = kr * 2 * DH + (gl % KC ^ swizzle<2 * DH>(kr)) * 16;
  const int v_dst = 2 * BUF + vr * 128 + (gl % 8 ^ swizzle<128>(vr)) * 16;
  auto k_next = [&](int j) { return key_of<false>(KROWS * j >> 4, 0, 0) * DH; };
  TileBatch tb = tile_batch(a, x, x.t0 + kw + 2 * lane, tp);
  struct Tile {
    int page, keys;
    float sk, sv;
  };
  auto tile = [&](int st) {  // of step st; places behind the last tile read page 0, with no keys
    const int l = st & 63;
    return Tile{at_lane(tb.page, l), at_lane(tb.keys, l), at_lane(tb.sk, l), at_lane(tb.sv, l)};
  };
  uint2 kc[PER], vc[PER];  // codes of the tiles kt and vt
  Tile kt, vt;
  auto load_k = [&](const Tile& t) {
    const uint8_t* c = base + (size_t)t.page * a.p.page_bytes + k_src;
#pragma unroll
    for (int j = 0; j < PER; ++j) kc[j] = *reinterpret_cast<const uint2*>(c + k_next(j));
    kt = t;
  };
  auto load_v = [&](const Tile& t) {
    const uint8_t* c = base + (size_t)t.page * a.p.page_bytes + SIDE;
#pragma unroll
    for (int j = 0; j < PER; ++j) vc[j] = *reinterpret_cast<const uint2*>(c + (gl + GT * j) * 8);
    vt = t;
  };
  auto place_k = [&](int st) {
    char* to = sb + (st & 1) * BUF + k_dst;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      *reinterpret_cast<bf16x8*>(to + KROWS * j * 2 * DH) = bf16_codes(kc[j].x, kc[j].y, kt.sk);
  };
  auto place_v = [&](int st) {
    char* to = sb + (st & 1) * BUF + v_dst;
    if (vt.keys < PAGE)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        vc[j] = uint2{keep_bytes(vc[j].x, vt.keys - gl % 8 * 8), keep_bytes(vc[j].y, vt.keys - gl % 8 * 8 - 4)};
#pragma unroll
    for (int j = 0; j < PER; ++j)
      *reinterpret_cast<bf16x8*>(to + VROWS * j * 128) = bf16_codes(vc[j].x, vc[j].y, vt.sv);
  };
  // the lane's places in a buffer: K row fr, chunks 4 e + grp; V^T row fr, chunks (8 keys) 4 c + grp
  int kofs[DH / 32], vofs[2];
  auto places = [&](int fr) {
#pragma unroll
    for (int e = 0; e < DH / 32; ++e) kofs[e] = fr * 2 * DH + ((4 * e + grp) ^ swizzle<2 * DH>(fr)) * 16;
#pragma unroll
    for (int e = 0; e < 2; ++e) vofs[e] = 2 * BUF + fr * 128 + ((4 * e + grp) ^ swizzle<128>(fr)) * 16;
  };
  places(fr);
  auto add_pv = [&](int st) {  // O += V^T P of step st
    const char* from = sb + (st & 1) * BUF;
#pragma unroll
    for (int c = 0; c < 2; ++c)  // a product's sum is not taken up again before NB QS others
#pragma unroll
      for (int d = 0; d < NB; ++d) {
        const bf16x8 vf = *reinterpret_cast<const bf16x8*>(from + d * 16 * 128 + vofs[c]);
#pragma unroll
        for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, p[u][c], o[u][d], 0, 0, 0);
      }
  };
  auto score = [&](int st) {  // S = K Q^T of step st
    const char* from = sb + (st & 1) * BUF;
#pragma unroll
    for (int e = 0; e < DH / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x8 k = *reinterpret_cast<const bf16x8*>(from + i * 32 * DH + kofs[e]);
#pragma unroll
        for (int u = 0; u < QS; ++u)
          s[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qs[u].op[e], e ? s[u][i] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
      }
  };
  int keys = 0;
  // Beside the products of step st: the next K and this V go to LDS, those after them to registers.
  auto move = [&](int st, const Tile& after) {
    const Tile next = kt;
    place_k(st + 1);
    load_k(after);
    place_v(st);
    keys = vt.keys;
    load_v(next);
  };
  auto soften = [&]() {  // P of the step
#pragma unroll
    for (int u = 0; u < QS; ++u) {
      softmax_tile<false>(s[u], keys, grp, a.scale_log2, m_run[u], l_run[u], o[u]);
      p_operand(s[u], p[u]);
    }
  };
#pragma unroll
  for (int u = 0; u < QS; ++u)
    qs[u] = load_query<DH, false>(
        static_cast<const bf16*>(a.q) + (x.head * ncol + min(col0 + 16 * u + fr, ncol - 1)) * DH, grp);
  if (steps) {
    const int page0 = at_lane(tb.page, 0);
    load_k(Tile{page0});  // before the scales are there
    load_v(Tile{page0});
    settle(tb);
    kt = vt = tile(0);
    place_k(0);
    load_k(tile(1));
#pragma unroll
    for (int u = 0; u < QS; ++u) settle<DH>(qs[u]);
    __builtin_amdgcn_s_waitcnt(VM_DONE);  // so that the waits in the loop count its own loads alone
    if (kw) __syncthreads();              // the second group is half a step behind
    __syncthreads();
    move(0, tile(2));
    score(0);
    __syncthreads();
    soften();
    for (int st = 1; st < steps; ++st) {
      if (((st + 2) & 63) == 0) {
        tb = tile_batch(a, x, x.t0 + kw + 2 * (st + 2 + lane), tp);
        settle(tb);
      }
      const Tile after = tile(st + 2);
      __syncthreads();  // the group's K of this step and V of the one before are in LDS
      move(st, after);
      add_pv(st - 1);
      score(st);
      // reads of LDS run 8 ahead of the products that take them: left to itself the compiler has
      // two in flight, and waits out their latency 16 times a step
      constexpr int READS = 2 * NB + DH / 8, AHEAD = 8;
      __builtin_amdgcn_sched_group_barrier(SCHED_LDS_READ, AHEAD, 0);
#pragma unroll
      for (int r = AHEAD; r < READS; ++r) {
        __builtin_amdgcn_sched_group_barrier(SCHED_MFMA, QS, 0);
        __builtin_amdgcn_sched_group_barrier(SCHED_LDS_READ, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(SCHED_MFMA, QS * AHEAD, 0);
      __syncthreads();  // the group is done with V of the step before
      soften();
    }
  }
  // The window's tiles: as steps behind those of the pages, the groups side by side, their elements through
  // registers to the same places in LDS.  The first are on their way beside the last product of the pages.
  const int w0 = max(x.t0, x.np), wsteps = x.t1 > w0 ? (x.t1 - w0 + 1) / 2 : 0;
  const int mine = w0 + (kw ^ ((w0 - x.t0) & 1));
  bf16x8 wk[PER], wv[PER];
  auto load_window = [&](int t) {  // behind the last: the first one's, with no keys
    const size_t w = (size_t)(t < x.t1 ? t - x.np : 0) * PAGE;
    int l = gl;
    asm volatile("" : "+v"(l));  // the addresses are made here, and take no registers in the loops
    const bf16* k = static_cast<const bf16*>(a.k) + (x.head * a.cap + w) * DH + k_first(l);
    const bf16* v = static_cast<const bf16*>(a.vt) + (x.head * DH + l / 8) * a.cap + w + l % 8 * 8;
#pragma unroll
    for (int j = 0; j < PER; ++j) wk[j] = *reinterpret_cast<const bf16x8*>(k + k_next(j));
#pragma unroll
    for (int j = 0; j < PER; ++j) wv[j] = *reinterpret_cast<const bf16x8*>(v + (size_t)(VROWS * j) * a.cap);
  };
  if (wsteps) load_window(mine);
  if (steps) {
    __syncthreads();
    add_pv(steps - 1);
    if (!kw) __syncthreads();
  }
  for (int i = 0; i < wsteps; ++i) {
    int f = fr;
    asm volatile("" : "+v"(f));  // as in load_window
    places(f);
    const int st = steps + i, t = mine + 2 * i;
    keys = t < x.t1 ? min(PAGE, x.n - (t - x.np) * PAGE) : 0;
    if (keys < PAGE)
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (gl % 8 * 8 + e >= keys) wv[j][e] = (bf16)0.f;
    char* to = sb + (st & 1) * BUF;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      *reinterpret_cast<bf16x8*>(to + k_dst + KROWS * j * 2 * DH) = wk[j];
      *reinterpret_cast<bf16x8*>(to + v_dst + VROWS * j * 128) = wv[j];
    }
    __syncthreads();  // also: the group is done with the step before the last, whose buffers come next
    if (i + 1 < wsteps) load_window(t + 2);
    if (keys > 0) {
      score(st);
      soften();
      add_pv(st);
    }
  }
  __syncthreads();  // every wave is done with the tiles
  float* xs = reinterpret_cast<float*>(smem) + cw * 2 * NV * 64;  // of the two waves of a strip
#pragma unroll
  for (int u = 0; u < QS; ++u)
    join_waves<bf16, NB, 2>(a, x, col0 + 16 * u + fr, m_run[u], l_run[u], o[u], xs, kw);
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
