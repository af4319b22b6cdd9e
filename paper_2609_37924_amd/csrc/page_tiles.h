// Tiles of the paged 8-bit K/V store in attention: the work of a block on a run of 64-key tiles, for
// the kernels of page_attention.hip (each row by itself) and page_shared.hip (rows that share pages).
//
// A block type X says what the block works on.  Its columns (queries) are numbered from 0; x.ct is the tile of them
// that the block has, and x.column(a, col) the place of a column among those of q (any valid one behind the last);
// x.b, x.len, x.np: the row whose pages are read, its positions and their tiles; tiles [x.t0, x.t1), pages below x.np,
// the window's (x.n tokens of K/V head x.head) from there on; x.wanted(a, col): whether the column has a result;
// x.parts(a): whether that is a part, at x.part_o and x.part_ml, rather than the whole of it.
#pragma once
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
template <class T, class X>
__device__ __forceinline__ void put4(const Args& a, const X& x, int col, int d0, float inv, const float* r) {
  if (x.parts(a)) {
    store4(x.part_o(a, col) + d0, r[0], r[1], r[2], r[3]);
  } else {
    const int L = a.r.max_n, g = col / L, j = col % L;
    T* out = static_cast<T*>(a.o) + (((size_t)x.b * L + j) * a.p.Hkv * a.G + x.h * a.G + g) * a.p.dh;
    store4(out + d0, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
  }
}
template <class X>
__device__ __forceinline__ void put_ml(const Args& a, const X& x, int col, float m, float sum) {
  if (x.parts(a))
    store2(x.part_ml(a, col), m, sum);
  else if (a.lse)
    a.lse[x.head * (a.G * a.r.max_n) + col] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}
template <class X>
__device__ __forceinline__ float inverse(const Args& a, const X& x, float sum) {
  return x.parts(a) || sum == 0.f ? 0.f : 1.f / sum;
}

// Joins NW waves that hold the same strip of 16 columns, in the order of the waves: per lane m,
// l and O in [wave][value][lane] floats; wave w sums the head-width blocks w, w + NW, ...
template <class T, int NB, int NW, class X>
__device__ __forceinline__ void join_waves(const Args& a, const X& x, int col, float m_run, float l_run,
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
  if (x.wanted(a, col)) {
    const float inv = inverse(a, x, sum);
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
constexpr int F32_WAVES = 4;
// 4 codes (a dword) as floats times the scale
__device__ __forceinline__ f32x4 f32_codes(uint32_t c, float s) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
}

// Four waves on a strip of 16 columns, each taking every fourth tile; NB: head width in blocks of
// 16, the last of which may be partial.  Products and probabilities stay in float32.  float32 models are small
// (at most 4 096 positions of a window), and what bounds them is a launch and one tile's latency: 5 rows of
// 24 tokens over up to 333 positions, 4 heads x 16, 7.4 us, of which an empty launch takes 3.6.
template <int NB, class X>
__device__ __forceinline__ void f32_tiles(const Args& a, const X& x, float* xs) {
  constexpr int NW = F32_WAVES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15;
  const int dh = a.p.dh, col = x.ct * 16 + fr;
  f32x4 qx[NB], o[NB];
  const float* q = static_cast<const float*>(a.q) + x.column(a, col) * dh;
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
template <class X>
__device__ __forceinline__ TileBatch tile_batch(const Args& a, const X& x, int tile, int t1) {
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
template <int DH, int QS, class X>
__device__ __forceinline__ void window_tile(const Args& a, const X& x, int w, const bf16* const (&q)[QS],
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
template <int DH, int QS, int NW, class X>
__device__ __forceinline__ void narrow_tiles(const Args& a, const X& x, float* xs) {
  constexpr int NB = DH / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW, grp = lane >> 4,
            fr = lane & 15;
  const int tp = min(x.t1, x.np), first = x.t0 + wave;
  const int steps = first < tp ? (tp - first + NW - 1) / NW : 0;
  const bf16* q[QS];
  Query<DH> qs[QS];
  f32x4 o[QS][NB];
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    q[u] = static_cast<const bf16*>(a.q) + x.column(a, x.ct * 16 * QS + 16 * u + fr) * DH;
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
template <int DH>
constexpr int wide_lds() { return 16 * PAGE * DH; }  // bytes
template <int DH, int QS, int CW, class X>
__device__ __forceinline__ void wide_tiles(const Args& a, const X& x, char* smem) {
  constexpr int NB = DH / 16, KC = DH / 8, NV = 2 + 4 * NB, GT = 64 * CW;
  constexpr int SIDE = PAGE * DH, BUF = 2 * SIDE, GROUP = 4 * BUF;  // codes of a side, and its bf16; K, K, V, V
  constexpr int PER = SIDE / 8 / GT;                               // chunks (8 codes) of a side that a lane moves per tile
  constexpr int KROWS = GT / KC, VROWS = GT / 8;                   // rows of K and V^T that a group moves at once
  static_assert(PER * 8 * GT == SIDE && CW == 4, "a tile splits over the lanes of a group in whole blocks of 16 keys");
  static_assert(2 * CW * NV * 64 * 4 <= 2 * GROUP, "the groups are joined in the space of the tiles");
  static_assert(2 * GROUP == wide_lds<DH>(), "the LDS of a block");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15, cw = wave % CW, kw = wave / CW, gl = cw * 64 + lane;
  const int col0 = (x.ct * CW + cw) * 16 * QS;
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
        static_cast<const bf16*>(a.q) + x.column(a, col0 + 16 * u + fr) * DH, grp);
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

}  // namespace
}  // namespace tadm
