// Append, read and copy of the paged 8-bit K/V store.
//
// Quantisation of one page, head and side: with M the largest finite |x| among the new values,
// e = the least exponent with M <= 448 2^e (448 is the largest e4m3), cut to [-110, 120]; a
// page that holds earlier positions of the row keeps the larger of its scale and 2^e, and if
// it grew its codes are rounded again to the new scale.  code(x) = x 2^-e rounded to nearest
// even, at e = 120 at most 240, so that what is read back is finite; values that are not finite get the
// NaN code.  A power of two costs no precision: the codes are floating point, and 2^-e x is exact.
#include "common.h"
#include "pages.h"

namespace tadm {
namespace {

__device__ __forceinline__ int row_len(const PageRows& r, int b) {
  return r.len ? min(max(r.len[b], 0), r.max_len) : r.max_len;
}
__device__ __forceinline__ int row_new(const PageRows& r, int b) {
  return r.n ? min(max(r.n[b], 0), r.max_n) : r.max_n;
}

// 2^e of the least e in [PAGE_E_MIN, PAGE_E_MAX] with top <= 448 2^e = 1.75 2^(e + 8)
__device__ __forceinline__ float scale_of(float top) {
  const uint32_t bits = __float_as_uint(top);
  int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = min(max(e, PAGE_E_MIN), PAGE_E_MAX);
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
// The largest finite magnitude of values, by their bits: without the sign they order as the
// values do, and adding one to the exponent makes those of infinities and NaN negative, which
// a signed maximum that starts at 0 passes over.  bf16: two values a step.
typedef short i16x2 __attribute__((ext_vector_type(2)));
struct Top16 {
  i16x2 m = {0x80, 0x80};
  __device__ __forceinline__ void add(uint32_t two) {
    const uint32_t t = two & 0x7fff7fffu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(i16x2, t) + i16x2{0x80, 0x80});
  }
  __device__ __forceinline__ float value() const {
    return __uint_as_float((uint32_t)(max((int)m[0], (int)m[1]) - 0x80) << 16);
  }
};
struct Top32 {
  int m = 0x800000;
  __device__ __forceinline__ void add(uint32_t x) { m = max(m, (int)((x & 0x7fffffffu) + 0x800000u)); }
  __device__ __forceinline__ float value() const { return __int_as_float(m - 0x800000); }
};

// 16 values as they lie in memory, of any alignment.
template <class T>
struct Raw16;
template <>
struct Raw16<bf16> {
  typedef Top16 Top;
  uint32_t w[8];
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ __forceinline__ void set(int e, bf16 x) {
    const uint32_t b = __builtin_bit_cast(uint16_t, x);
    w[e / 2] = e % 2 ? (w[e / 2] & 0xffffu) | b << 16 : (w[e / 2] & 0xffff0000u) | b;
  }
};
template <>
struct Raw16<float> {
  typedef Top32 Top;
  uint32_t w[16];
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(w[e]); }
  __device__ __forceinline__ void set(int e, float x) { w[e] = __float_as_uint(x); }
};

// Codes of 4 values; one that is not finite gets a NaN code (nothing finite is above 448 here).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, v, true);
}
__device__ __forceinline__ uint8_t code_of(float x, float inv) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x * inv, 0.f, 0, false) & 255);
}
// Four codes of the scale 2^120 with 256 (0x78), the only one above 240 that a finite number rounds to, taken to 240:
// of 0x80 less the difference of two codes without signs, bit 7 is set where they are equal.
__device__ __forceinline__ uint32_t capped(uint32_t w) {
  const uint32_t d = (w & 0x7f7f7f7fu) ^ 0x78787878u;
  return w - (((0x80808080u - d) & 0x80808080u) >> 7);
}
__device__ __forceinline__ float value_of(uint8_t c) { return __builtin_amdgcn_cvt_f32_fp8((int)c, 0); }

// One block per (page of a row, K/V head, row).  Up to 15 new positions a thread takes single
// elements; from 16 on it takes units of 16 codes, all of a page in registers between the
// search for the maximum and the rounding, so that the window is read once.  A unit
// that holds other positions as well keeps theirs.
//
// HBM's for prompts, but not at its rate: 1 024 tokens in 4 rows, 16 heads x 128, from position 37 on (50 MB): 17.2 us,
// 2.9 TB/s, against 9.8 at the rate of a large copy.  Every block waits for the whole of its window before it
// may round, and keys that start inside a page make the unit loads of V^T straddle lines, each of which two
// pages read; which of these costs what was not measured.  With single elements throughout 48.7.  One token in each of 16 rows: 5.1, of which an empty launch takes 3.6.
template <class T>
__global__ __launch_bounds__(256) void append_kernel(PageLayer p, PageRows r, const T* k, const T* vt, int cap) {
  __shared__ float red[2][4];
  const int b = blockIdx.z, h = blockIdx.y, dh = p.dh;
  const int len = row_len(r, b);
  const int slot = len / PAGE + blockIdx.x, start = slot * PAGE;
  if (slot >= r.max_pages) return;
  const int lo = max(len, start) - start, hi = min(len + row_new(r, b), start + PAGE) - start;  // new places of the page
  if (hi <= lo) return;
  const int page = r.table[(size_t)b * r.max_pages + slot];
  if ((unsigned)page >= (unsigned)p.n_pages) return;
  // the window as the page sees it: place i of the page is token start - len + i
  const T* ks = k + ((size_t)b * p.Hkv + h) * cap * dh + (ptrdiff_t)(start - len) * dh;
  const T* vs = vt + ((size_t)b * p.Hkv + h) * dh * cap + (start - len);
  uint8_t* codes = p.data + (size_t)page * p.page_bytes + (size_t)h * 2 * PAGE * dh;
  float* scale = p.scale + (size_t)page * p.page_scales + 2 * h;
  const float old[2] = {scale[0], scale[1]};
  const int m = hi - lo, units = 4 * dh;  // of a side; at most two a thread
  const bool whole = m >= 16;
  Raw16<T> x[2][2];  // [keys, values][unit]
  typename Raw16<T>::Top tops[2];
  if (whole) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int u = threadIdx.x + 256 * j;
      if (u >= units) continue;
      const int k0 = 16 * u / dh, k1 = (16 * u + 15) / dh;  // the unit's places
      if (k0 >= lo && k1 < hi) {
        __builtin_memcpy(x[0][j].w, ks + 16 * u, sizeof x[0][j].w);
      } else {
        x[0][j] = Raw16<T>{};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int at = (16 * u + e) / dh;
          if (at >= lo && at < hi) x[0][j].set(e, ks[16 * u + e]);
        }
      }
      const int d = u / 4, v0 = 16 * (u % 4);
      if (v0 >= lo && v0 + 16 <= hi) {
        __builtin_memcpy(x[1][j].w, vs + (size_t)d * cap + v0, sizeof x[1][j].w);
      } else {
        x[1][j] = Raw16<T>{};
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (v0 + e >= lo && v0 + e < hi) x[1][j].set(e, vs[(size_t)d * cap + v0 + e]);
      }
#pragma unroll
      for (int side = 0; side < 2; ++side)
#pragma unroll
        for (uint32_t w : x[side][j].w) tops[side].add(w);
    }
  } else {
    for (int i = threadIdx.x; i < m * dh; i += 256) {
      Raw16<T> one{};
      one.set(0, ks[lo * dh + i]);
      tops[0].add(one.w[0]);
      one.set(0, vs[(size_t)(i / m) * cap + lo + i % m]);
      tops[1].add(one.w[0]);
    }
  }
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const float top = wave_max(tops[side].value());
    if (threadIdx.x % 64 == 0) red[side][threadIdx.x / 64] = top;
  }
  __syncthreads();  // also: every thread has the old scales
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    float s = scale_of(fmaxf(fmaxf(red[side][0], red[side][1]), fmaxf(red[side][2], red[side][3])));
    uint8_t* c = codes + side * PAGE * dh;
    const bool grown = lo > 0 && s > old[side];  // the codes of the earlier places change
    if (lo > 0 && !grown) s = old[side];
    const float inv = 1.f / s, f = old[side] * inv;
    const bool at_top = __builtin_amdgcn_readfirstlane(__float_as_int(s)) == __float_as_int(PAGE_SCALE_MAX);
    auto again = [&](uint8_t b) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(value_of(b) * f, 0.f, 0, false) & 255); };
    if (whole) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int u = threadIdx.x + 256 * j;
        if (u >= units) continue;
        const int first = side ? 16 * (u % 4) : 16 * u / dh, last = side ? first + 15 : (16 * u + 15) / dh;
        const bool all = first >= lo && last < hi, none = last < lo || first >= hi;
        if (none && !(grown && first < lo)) continue;
        const Raw16<T>& v = x[side][j];
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = codes4(v.get(4 * e), v.get(4 * e + 1), v.get(4 * e + 2), v.get(4 * e + 3), inv);
        if (at_top)
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = capped(w[e]);
        if (!all) {
          uint32_t had[4];
          *reinterpret_cast<uint4*>(had) = *reinterpret_cast<const uint4*>(c + 16 * u);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = side ? first + e : (16 * u + e) / dh, sh = 8 * (e % 4);
            if (at >= lo && at < hi) continue;
            uint32_t b = (had[e / 4] >> sh) & 255u;
            if (grown && at < lo) b = again((uint8_t)b);
            w[e / 4] = (w[e / 4] & ~(255u << sh)) | (b << sh);
          }
        }
        *reinterpret_cast<uint4*>(c + 16 * u) = *reinterpret_cast<const uint4*>(w);
      }
    } else {
      if (grown)
        for (int i = threadIdx.x; i < lo * dh; i += 256) {
          uint8_t* at = side == 0 ? c + i : c + (i / lo) * PAGE + i % lo;
          *at = again(*at);
        }
      for (int i = threadIdx.x; i < m * dh; i += 256) {
        const float y = f32_of(side == 0 ? ks[lo * dh + i] : vs[(size_t)(i / m) * cap + lo + i % m]);
        const uint8_t b = code_of(y, inv);
        uint8_t* at = side == 0 ? c + lo * dh + i : c + (i / m) * PAGE + lo + i % m;
        *at = at_top ? (uint8_t)capped(b) : b;
      }
    }
    if (threadIdx.x == 0) scale[side] = s;
  }
}

// W codes as values times the scale, 16 bytes of the model type: 8 for bf16, 4 for float
__device__ __forceinline__ void values(const uint8_t* c, float s, bf16x8& v) {
  const uint2 w = *reinterpret_cast<const uint2*>(c);
  const auto p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, false),
             p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, s, true),
             p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, false),
             p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, s, true);
  v = bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
__device__ __forceinline__ void values(const uint8_t* c, float s, f32x4& v) {
  const int w = *reinterpret_cast<const int*>(c);
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  v = f32x4{lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
}

// One block per (page of a row, K/V head, row); a thread takes pieces of 16 bytes of the result, so
// that both sides move whole lines.  Bound by HBM, by its writes above all: 4 rows of 16 384 positions, 16 heads x 128
// (805 MB): 167 us, 4.8 TB/s (157 at the rate of a large copy); element by element 393.  8 rows of up to
// 777, 12 heads x 64 (22 MB): 5.8.
template <class T, class V>
__global__ __launch_bounds__(256) void read_kernel(PageLayer p, PageRows r, T* k, T* vt, int cap) {
  constexpr int W = 16 / sizeof(T);
  const int b = blockIdx.z, h = blockIdx.y, dh = p.dh;
  const int start = blockIdx.x * PAGE, m = min(row_len(r, b) - start, PAGE);
  if (m <= 0) return;
  const int page = r.table[(size_t)b * r.max_pages + blockIdx.x];
  const bool there = (unsigned)page < (unsigned)p.n_pages;
  const uint8_t* codes = p.data + (size_t)(there ? page : 0) * p.page_bytes + (size_t)h * 2 * PAGE * dh;
  const float* scale = p.scale + (size_t)(there ? page : 0) * p.page_scales + 2 * h;
  const float sk = scale[0], sv = scale[1];
  T* kd = k + (((size_t)b * p.Hkv + h) * cap + start) * dh;
  T* vd = vt + ((size_t)b * p.Hkv + h) * dh * cap + start;
#pragma unroll 4
  for (int u = threadIdx.x; u < PAGE * dh / W; u += 256) {
    V x, y;
    values(codes + W * u, sk, x);
    values(codes + PAGE * dh + W * u, sv, y);
    if (!there) x = y = V(0);
    T* ko = kd + W * u;
    if (W * u + W <= m * dh) {
      *reinterpret_cast<V*>(ko) = x;
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (W * u + e < m * dh) ko[e] = x[e];
    }
    const int d = W * u / PAGE, j = W * u % PAGE;
    T* vo = vd + (size_t)d * cap + j;
    if (j + W <= m) {
      *reinterpret_cast<V*>(vo) = y;
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (j + e < m) vo[e] = y[e];
    }
  }
}

constexpr int COPY_PAIRS = 448;  // pairs of a launch: they travel in its arguments (4 KB)
struct CopyPairs {
  int32_t src[COPY_PAIRS], dst[COPY_PAIRS];
};

// grid: x = 16 KB pieces of a page, y = pairs.  Bound by HBM: 96 pages of 46 layers of 16 heads x 128 (2.3 GB):
// 420 us, 5.5 TB/s; 4 pages of 24 layers of 4 heads x 128 (12.6 MB): 6.7, an empty launch's 3.6 and 2.5 at the rate of a
// large copy (with fewer bytes of arguments 6.9).
__global__ __launch_bounds__(256) void copy_pages_kernel(uint8_t* data, float* scale, size_t page_bytes,
                                                         size_t page_scales, CopyPairs pairs) {
  const int src = pairs.src[blockIdx.y], dst = pairs.dst[blockIdx.y];
  const uint4* a = reinterpret_cast<const uint4*>(data + (size_t)src * page_bytes);
  uint4* o = reinterpret_cast<uint4*>(data + (size_t)dst * page_bytes);
  const size_t n = page_bytes / 16, first = (size_t)blockIdx.x * 1024 + threadIdx.x;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (first + 256 * i < n) o[first + 256 * i] = a[first + 256 * i];
  if (blockIdx.x == 0)
    for (size_t i = threadIdx.x; i < page_scales; i += 256)
      scale[(size_t)dst * page_scales + i] = scale[(size_t)src * page_scales + i];
}

__global__ __launch_bounds__(512) void table_set_kernel(int32_t* table, CopyPairs pairs, int n) {
  const int i = threadIdx.x;
  if (i < n) table[pairs.src[i]] = pairs.dst[i];
}

__global__ __launch_bounds__(256) void table_clear_kernel(int32_t* table, int rows, int per_row, int from) {
  const int i = blockIdx.x * 256 + threadIdx.x, w = per_row - from;
  if (i < rows * w) table[(size_t)(i / w) * per_row + from + i % w] = -1;
}

// pairs [i, i + COPY_PAIRS) of two lists of n, unused places 0
CopyPairs some_pairs(const int32_t* a, const int32_t* b, int i, int n, int* m) {
  CopyPairs pairs{};
  *m = n - i < COPY_PAIRS ? n - i : COPY_PAIRS;
  for (int j = 0; j < *m; ++j) {
    pairs.src[j] = a[i + j];
    pairs.dst[j] = b[i + j];
  }
  return pairs;
}

}  // namespace

hipError_t table_set(int32_t* table, const int32_t* at, const int32_t* id, int n, hipStream_t s) {
  for (int i = 0, m; i < n; i += COPY_PAIRS) {
    const CopyPairs pairs = some_pairs(at, id, i, n, &m);
    hipLaunchKernelGGL(table_set_kernel, dim3(1), dim3(512), 0, s, table, pairs, m);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t table_clear(int32_t* table, int rows, int per_row, int from, hipStream_t s) {
  if (from >= per_row) return hipSuccess;
  const unsigned blocks = ((unsigned)rows * (per_row - from) + 255) / 256;
  hipLaunchKernelGGL(table_clear_kernel, dim3(blocks), dim3(256), 0, s, table, rows, per_row, from);
  return hipGetLastError();
}

hipError_t pages_append(DType dt, const PageLayer& p, const PageRows& r, const void* k, const void* vt, int cap,
                        hipStream_t s) {
  const dim3 grid((r.max_n + PAGE - 1) / PAGE + 1, p.Hkv, r.B);
  if (dt == BF16)
    hipLaunchKernelGGL(append_kernel<bf16>, grid, dim3(256), 0, s, p, r, static_cast<const bf16*>(k),
                       static_cast<const bf16*>(vt), cap);
  else
    hipLaunchKernelGGL(append_kernel<float>, grid, dim3(256), 0, s, p, r, static_cast<const float*>(k),
                       static_cast<const float*>(vt), cap);
  return hipGetLastError();
}

hipError_t pages_read(DType dt, const PageLayer& p, const PageRows& r, void* k, void* vt, int cap, hipStream_t s) {
  const dim3 grid((r.max_len + PAGE - 1) / PAGE, p.Hkv, r.B);
  if (grid.x == 0) return hipSuccess;
  if (dt == BF16)
    hipLaunchKernelGGL((read_kernel<bf16, bf16x8>), grid, dim3(256), 0, s, p, r, static_cast<bf16*>(k), static_cast<bf16*>(vt),
                       cap);
  else
    hipLaunchKernelGGL((read_kernel<float, f32x4>), grid, dim3(256), 0, s, p, r, static_cast<float*>(k),
                       static_cast<float*>(vt), cap);
  return hipGetLastError();
}

hipError_t pages_copy(void* data, float* scale, size_t page_bytes, size_t page_scales, const int32_t* src,
                      const int32_t* dst, int n, hipStream_t s) {
  const unsigned pieces = (unsigned)((page_bytes + 16383) / 16384);
  for (int i = 0, m; i < n; i += COPY_PAIRS) {
    const CopyPairs pairs = some_pairs(src, dst, i, n, &m);
    hipLaunchKernelGGL(copy_pages_kernel, dim3(pieces, m), dim3(256), 0, s, static_cast<uint8_t*>(data), scale,
                       page_bytes, page_scales, pairs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace tadm
