// Attention of a window of queries over the paged 8-bit K/V store.
//
//   O = softmax(q K^T / sqrt(dh)) V over the committed positions of a row (e4m3 codes with
//   one scale per page and head) followed by the window's own keys in the model type.
//
// The queries of the G = H / Hkv heads that share a K/V head are one set of G L columns (they
// lie one after the other in memory), so that a page is read once for all of them.  Scores
// are computed transposed, S^T = K Q^T, a lane owning one column; the running maximum and sum
// of the softmax live in the lane, and the probabilities feed O^T = V^T P^T from registers.
// The order of the keys within a page is free (a sum over them): score row 4 g + j of the
// 16-key block i stands for key 16 g + 4 i + j, so that a lane's 16 probabilities of a page
// are those of 16 consecutive keys, one 16-byte load of a V^T row.
//
// A block is 4 waves on the same columns, each taking every fourth tile of 64 keys; the key
// axis is split over S blocks when the columns alone leave the chip empty, and the partial
// results (m, l, unnormalised O) are joined in the order of the splits.
#include "common.h"
#include "pages.h"

namespace tadm {
namespace {

constexpr int NW = 4;  // waves of a block
constexpr float LN2 = 0.6931471805599453f;

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

// 4 codes (a dword) as floats times the scale
__device__ __forceinline__ f32x4 f32_codes(uint32_t c, float s) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
}
__device__ __forceinline__ float* part_o(const Args& a, size_t col, int split) {
  return a.part + (col * a.S + split) * a.p.dh;
}
__device__ __forceinline__ float* part_ml(const Args& a, size_t col, int split) {
  const size_t cols = (size_t)a.r.B * a.p.Hkv * a.G * a.r.max_n;
  return a.part + cols * a.S * a.p.dh + (col * a.S + split) * 2;
}
// 8 codes as bf16 times the scale, exactly
__device__ __forceinline__ bf16x8 bf16_codes(uint32_t a, uint32_t b, float s) {
  const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false),
             p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true),
             p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false),
             p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true);
  return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
// bytes [0, keep) of a dword (keep may be negative or above 4)
__device__ __forceinline__ uint32_t keep_bytes(uint32_t v, int keep) {
  return keep >= 4 ? v : keep <= 0 ? 0u : v & ((1u << (8 * keep)) - 1u);
}

// NB: head width in blocks of 16 (the last may be partial for float), QS: strips of 16 columns.
template <class T, int NB, int QS>
__global__ __launch_bounds__(64 * NW) void attend_kernel(Args a) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NV = 2 + 4 * NB;  // floats a lane keeps per strip: m, l and its part of O
  __shared__ float xs[NW * NV * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4,
            fr = lane & 15;
  const int dh = BF ? 16 * NB : a.p.dh, L = a.r.max_n, ncol = a.G * L, nct = (ncol + 16 * QS - 1) / (16 * QS);
  const int id = xcd_contiguous(blockIdx.x, gridDim.x);
  const int ct = id % nct, sp = (id / nct) % a.S, h = (id / nct / a.S) % a.p.Hkv, b = id / nct / a.S / a.p.Hkv;
  const int n = row_new(a.r, b);
  if (n == 0) return;
  const int len = row_len(a.r, b), np = (len + PAGE - 1) / PAGE, nt = np + (a.k ? (n + PAGE - 1) / PAGE : 0);
  const int t0 = (int)((long)nt * sp / a.S), t1 = (int)((long)nt * (sp + 1) / a.S);

  // queries: lane's column of strip u, the head-width elements that its k index of a product has
  const size_t head = (size_t)b * a.p.Hkv + h;
  bf16x8 qb[QS][BF ? NB / 2 : 1];
  f32x4 qx[QS][BF ? 1 : NB];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    const int col = min(ct * 16 * QS + 16 * u + fr, ncol - 1);
    const T* q = static_cast<const T*>(a.q) + (head * ncol + col) * dh;
    if constexpr (BF) {
#pragma unroll
      for (int c = 0; c < NB / 2; ++c) qb[u][c] = *reinterpret_cast<const bf16x8*>(q + grp * (4 * NB) + 8 * c);
    } else {
#pragma unroll
      for (int c = 0; c < NB; ++c)
        qx[u][c] = 16 * c + 4 * grp < dh ? *reinterpret_cast<const f32x4*>(q + 16 * c + 4 * grp) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  f32x4 o[QS][NB];
  float m_run[QS], l_run[QS];
#pragma unroll
  for (int u = 0; u < QS; ++u) {
#pragma unroll
    for (int d = 0; d < NB; ++d) o[u][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[u] = -INFINITY;
    l_run[u] = 0.f;
  }

  for (int t = t0 + wave; t < t1; t += NW) {
    const bool paged = t < np;
    const int kv = paged ? min(PAGE, len - t * PAGE) : min(PAGE, n - (t - np) * PAGE);  // keys of this tile
    const uint8_t* codes = nullptr;
    float sk = 1.f, sv = 1.f;
    const T *kw = nullptr, *vw = nullptr;
    if (paged) {
      const int page = a.r.table[(size_t)b * a.r.max_pages + t];
      if ((unsigned)page >= (unsigned)a.p.n_pages) continue;
      codes = a.p.data + (size_t)page * a.p.page_bytes + (size_t)h * 2 * PAGE * dh;
      const float* sc = a.p.scale + (size_t)page * a.p.page_scales + 2 * h;
      sk = sc[0];
      sv = sc[1];
    } else {
      kw = static_cast<const T*>(a.k) + (head * a.cap + (size_t)(t - np) * PAGE) * dh;
      vw = static_cast<const T*>(a.vt) + head * dh * a.cap + (size_t)(t - np) * PAGE;
    }
    f32x4 s[QS][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = 16 * (fr >> 2) + 4 * i + (fr & 3);
#pragma unroll
      for (int u = 0; u < QS; ++u) s[u][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (BF) {
        bf16x8 kf[NB / 2];
        if (paged) {
          uint32_t w[NB];
          const uint4* src = reinterpret_cast<const uint4*>(codes + key * dh + grp * (4 * NB));
#pragma unroll
          for (int c = 0; c < NB / 4; ++c) *reinterpret_cast<uint4*>(w + 4 * c) = src[c];
#pragma unroll
          for (int c = 0; c < NB / 2; ++c) kf[c] = bf16_codes(w[2 * c], w[2 * c + 1], sk);
        } else {
          const bf16x8* src = reinterpret_cast<const bf16x8*>(kw + (size_t)key * dh + grp * (4 * NB));
#pragma unroll
          for (int c = 0; c < NB / 2; ++c) kf[c] = src[c];
        }
#pragma unroll
        for (int c = 0; c < NB / 2; ++c)
#pragma unroll
          for (int u = 0; u < QS; ++u) s[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qb[u][c], s[u][i], 0, 0, 0);
      } else {
#pragma unroll
        for (int c = 0; c < NB; ++c) {
          f32x4 kf = f32x4{0.f, 0.f, 0.f, 0.f};
          if (16 * c + 4 * grp < dh)
            kf = paged ? f32_codes(*reinterpret_cast<const uint32_t*>(codes + key * dh + 16 * c + 4 * grp), sk)
                       : *reinterpret_cast<const f32x4*>(kw + (size_t)key * dh + 16 * c + 4 * grp);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int u = 0; u < QS; ++u) s[u][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qx[u][c][e], s[u][i], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < QS; ++u) {
      // s[u][i][j]: key 16 grp + 4 i + j of the tile, unscaled; the softmax runs in base 2 on
      // s * scale_log2, relative to a reference that moves only when the tile's maximum
      // exceeds it by more than 2^8: until then the probabilities stay below 256 and the
      // accumulators need no rescaling
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (16 * grp + 4 * i + j >= kv) s[u][i][j] = -INFINITY;
          mt = fmaxf(mt, s[u][i][j]);
        }
      mt = fmaxf(mt, xor16(mt));
      mt = fmaxf(mt, xor32(mt));
      const float mt2 = mt * a.scale_log2;
      const float m_new = mt2 > m_run[u] + 8.f ? mt2 : m_run[u];
      const float ref = m_new == -INFINITY ? 0.f : m_new;  // no finite score yet: every p is 0
      const float alpha = __builtin_amdgcn_exp2f(m_run[u] - ref);
      float ps = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[u][i][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i][j], a.scale_log2, -ref));
          ps += s[u][i][j];
        }
      l_run[u] = l_run[u] * alpha + ps;
      m_run[u] = m_new;
#pragma unroll
      for (int d = 0; d < NB; ++d) o[u][d] *= alpha;
    }
    bf16x8 pf[QS][BF ? 2 : 1];
    if constexpr (BF) {
#pragma unroll
      for (int u = 0; u < QS; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int j = 0; j < 8; ++j) pf[u][c][j] = (bf16)s[u][2 * c + j / 4][j % 4];
    }
    // V^T row 16 d + fr, keys 16 grp + [0, 16) of the tile; what lies behind the last key is
    // taken as 0, so that p = 0 meets a finite value
#pragma unroll
    for (int d = 0; d < NB; ++d) {
      const int row = min(16 * d + fr, dh - 1);
      if (paged) {
        uint32_t w[4];
        *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(codes + PAGE * dh + row * PAGE + 16 * grp);
        if (kv < PAGE)
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = keep_bytes(w[c], kv - 16 * grp - 4 * c);
        if constexpr (BF) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const bf16x8 vf = bf16_codes(w[2 * c], w[2 * c + 1], sv);
#pragma unroll
            for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][c], o[u][d], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 vf = f32_codes(w[i], sv);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j], s[u][i][j], o[u][d], 0, 0, 0);
          }
        }
      } else if constexpr (BF) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          bf16x8 vf = *reinterpret_cast<const bf16x8*>(vw + (size_t)row * a.cap + 16 * grp + 8 * c);
          if (kv < PAGE)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (16 * grp + 8 * c + j >= kv) vf[j] = (bf16)0.f;
#pragma unroll
          for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[u][c], o[u][d], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 vf = *reinterpret_cast<const f32x4*>(vw + (size_t)row * a.cap + 16 * grp + 4 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float v = 16 * grp + 4 * i + j < kv ? vf[j] : 0.f;
#pragma unroll
            for (int u = 0; u < QS; ++u) o[u][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[u][i][j], o[u][d], 0, 0, 0);
          }
        }
      }
    }
  }

  // Join the waves, a strip at a time, in the order of the waves: per lane m, l and O in
  // [wave][value][lane] floats; wave w sums the head-width blocks w, w + 4, ...
#pragma unroll
  for (int u = 0; u < QS; ++u) {
    if (u) __syncthreads();  // the previous strip has been read
    float l = l_run[u] + xor16(l_run[u]);
    l += xor32(l);
    float* w = xs + wave * NV * 64 + lane;
    w[0] = m_run[u];
    w[64] = l;
#pragma unroll
    for (int d = 0; d < NB; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) w[(2 + 4 * d + j) * 64] = o[u][d][j];
    __syncthreads();
    const float* x = xs + lane;
    float m = -INFINITY, f[NW], sum = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v) m = fmaxf(m, x[v * NV * 64]);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      f[v] = __builtin_amdgcn_exp2f(x[v * NV * 64] - ref);
      sum += x[v * NV * 64 + 64] * f[v];
    }
    const int col = ct * 16 * QS + 16 * u + fr, g = col / L, j = col % L;
    if (col >= ncol || j >= n) continue;
    const float inv = a.S > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
    float* part = part_o(a, head * ncol + col, sp);
    T* out = static_cast<T*>(a.o) + (((size_t)b * L + j) * a.p.Hkv * a.G + h * a.G + g) * dh;
    for (int d = wave; d < NB; d += NW) {
      float r[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < NW; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] += x[(v * NV + 2 + 4 * d + e) * 64] * f[v];
      if (16 * d + 4 * grp < dh) {
        if (a.S > 1) {
          store4(part + 16 * d + 4 * grp, r[0], r[1], r[2], r[3]);
        } else {
          store4(out + 16 * d + 4 * grp, r[0] * inv, r[1] * inv, r[2] * inv, r[3] * inv);
        }
      }
    }
    if (wave == 0 && grp == 0) {
      if (a.S > 1) {
        store2(part_ml(a, head * ncol + col, sp), m, sum);
      } else if (a.lse) {
        a.lse[head * ncol + col] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
      }
    }
  }
}

// Joins the splits of a column, one block each: eight groups of 32 lanes take every eighth
// split, four values of the head width a lane, and are summed in order.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Args a) {
  __shared__ float xs[8][132];
  const int lane = threadIdx.x & 63, g8 = threadIdx.x >> 5, i = threadIdx.x & 31;
  const int L = a.r.max_n, ncol = a.G * L, dh = a.p.dh;
  const size_t col_id = blockIdx.x;
  const int col = (int)(col_id % ncol), g = col / L, j = col % L;
  const int b = (int)(col_id / ncol / a.p.Hkv), h = (int)(col_id / ncol % a.p.Hkv);
  if (j >= row_new(a.r, b)) return;
  const float* ml = part_ml(a, col_id, 0);
  float m = -INFINITY;
  for (int s = lane; s < a.S; s += 64) m = fmaxf(m, ml[2 * s]);
  m = wave_max(m);
  const float ref = m == -INFINITY ? 0.f : m;
  const float* po = part_o(a, col_id, 0) + 4 * i;
  float r[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
#pragma unroll 4
  for (int s = g8; s < a.S; s += 8) {
    const float f = __builtin_amdgcn_exp2f(ml[2 * s] - ref);
    sum += ml[2 * s + 1] * f;
    if (4 * i < dh) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(po + (size_t)s * dh);
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] += v[e] * f;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) xs[g8][4 * i + e] = r[e];
  if (i == 0) xs[g8][128] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int v = 0; v < 8; ++v) sum += xs[v][128];
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (threadIdx.x < dh) {
    float o = 0.f;
#pragma unroll
    for (int v = 0; v < 8; ++v) o += xs[v][threadIdx.x];
    static_cast<T*>(a.o)[(((size_t)b * L + j) * a.p.Hkv * a.G + h * a.G + g) * dh + threadIdx.x] = from_f32<T>(o * inv);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[col_id] = sum == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * LN2;
}

struct Plan {
  int qs, S;
};

// Strips per wave and splits of the key axis.
Plan plan(DType dt, int B, int H, int Hkv, int L, int max_len) {
  (void)dt;
  const int ncol = H / Hkv * L;
  const int qs = ncol > 16 ? 2 : 1;
  const long blocks = (long)B * Hkv * ((ncol + 16 * qs - 1) / (16 * qs));
  const int tiles = (max_len + PAGE - 1) / PAGE + (L + PAGE - 1) / PAGE;
  long S = 1024 / blocks;                          // a block per CU and more
  S = S < (tiles + 7) / 8 ? S : (tiles + 7) / 8;   // two tiles per wave at least
  return Plan{qs, S < 1 ? 1 : (int)S};
}

template <class T, int NB>
hipError_t launch(const Args& a, const Plan& pl, hipStream_t s) {
  const int ncol = a.G * a.r.max_n;
  const long blocks = (long)a.r.B * a.p.Hkv * pl.S * ((ncol + 16 * pl.qs - 1) / (16 * pl.qs));
  if (blocks > 0x7fffffffL) return hipErrorInvalidValue;
  if (pl.qs == 2)
    launch_timed(attend_kernel<T, NB, 2>, dim3((unsigned)blocks), dim3(64 * NW), 0, s, a);
  else
    launch_timed(attend_kernel<T, NB, 1>, dim3((unsigned)blocks), dim3(64 * NW), 0, s, a);
  if (pl.S > 1) {
    hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)(a.r.B * a.p.Hkv * ncol)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace

size_t page_attend_work(DType dt, int B, int H, int Hkv, int dh, int L, int max_len) {
  const Plan pl = plan(dt, B, H, Hkv, L, max_len);
  return pl.S > 1 ? (size_t)B * H * L * pl.S * (dh + 2) * sizeof(float) : 0;
}

hipError_t page_attend(DType dt, const PageAttend& c, hipStream_t s) {
  const int dh = c.p.dh;
  const Plan pl = plan(dt, c.r.B, c.H, c.p.Hkv, c.r.max_n, c.r.max_len);
  Args a{c.p, c.r, c.q, c.k, c.vt, c.o, c.lse, static_cast<float*>(c.work), c.H / c.p.Hkv, c.cap, pl.S,
         1.4426950408889634f / sqrtf((float)dh)};
  if (dt == BF16) {
    if (dh == 64) return launch<bf16, 4>(a, pl, s);
    if (dh == 128) return launch<bf16, 8>(a, pl, s);
    return hipErrorInvalidValue;
  }
  switch ((dh + 15) / 16) {
    case 1: return launch<float, 1>(a, pl, s);
    case 2: return launch<float, 2>(a, pl, s);
    case 3: return launch<float, 3>(a, pl, s);
    case 4: return launch<float, 4>(a, pl, s);
    case 5: return launch<float, 5>(a, pl, s);
    case 6: return launch<float, 6>(a, pl, s);
    case 7: return launch<float, 7>(a, pl, s);
    case 8: return launch<float, 8>(a, pl, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace tadm
