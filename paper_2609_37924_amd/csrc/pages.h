// Paged 8-bit K/V store: geometry and host-side launchers (pages.hip, page_attention.hip).
//
// A page holds 64 positions of every layer.  Per page, layer and K/V head it has the keys,
// [64][dh] e4m3 codes, then the values transposed, [dh][64] codes, and one float32 scale for
// each of the two: the value of a code c is c * scale.  Scales are powers of two, so a
// code's value is exact in bf16 and a page whose scale grows keeps its codes up to those
// that become subnormal.
#pragma once
#include "kernels.h"

namespace tadm {

constexpr int PAGE = 64;
// exponents a scale may have: every value of a code is a normal bf16, at the largest of the codes up
// to 240, where append stops (the next, 256, would be 2^128)
constexpr int PAGE_E_MIN = -110, PAGE_E_MAX = 120;
constexpr float PAGE_SCALE_MAX = 0x1p120f;

// One layer of a page set: page p, head h at data + p * page_bytes + h * 128 * dh, its two
// scales at scale + p * page_scales + 2 h.
struct PageLayer {
  uint8_t* data;
  float* scale;
  size_t page_bytes;
  size_t page_scales;
  int n_pages, Hkv, dh;
};

// The rows of a call: row b's pages are table[b * max_pages ...], an id outside [0, n_pages)
// being an absent page; it holds the positions [0, len_b), len_b = max_len or, with len,
// len[b] cut to [0, max_len]; its window has n_b tokens, max_n or n[b] cut to [0, max_n].
struct PageRows {
  const int32_t* table;
  const int32_t* len;
  const int32_t* n;
  int B, max_pages, max_len, max_n;
};
__device__ __forceinline__ int row_len(const PageRows& r, int b) {
  return r.len ? min(max(r.len[b], 0), r.max_len) : r.max_len;
}
__device__ __forceinline__ int row_new(const PageRows& r, int b) {
  return r.n ? min(max(r.n[b], 0), r.max_n) : r.max_n;
}

// Quantises the window's keys [B, Hkv, cap, dh] and values [B, Hkv, dh, cap] (columns
// [0, n_b)) into positions [len_b, len_b + n_b) of each row.
hipError_t pages_append(DType dt, const PageLayer& p, const PageRows& r, const void* k, const void* vt, int cap,
                        hipStream_t s);
// Positions [0, len_b) of each row as keys and values of the model type (zero on absent pages).
hipError_t pages_read(DType dt, const PageLayer& p, const PageRows& r, void* k, void* vt, int cap, hipStream_t s);
// Page dst[i] <- page src[i], whole pages (src, dst: host arrays, copied into the launch).
hipError_t pages_copy(void* data, float* scale, size_t page_bytes, size_t page_scales, const int32_t* src,
                      const int32_t* dst, int n, hipStream_t s);

// A stack of free pages in device memory: id[0, free) with free = state[0], the next one taken at the back;
// size: the pages in all and the entries of id; the other three words of state are 0 outside of a launch.
struct PageStack {
  int32_t* id;
  int32_t* state;
  int size;
};
constexpr int PAGE_STACK_ROWS = 4096;  // rows of a call: the block that takes pages back holds a word of each
// Pages for the positions [len_b, len_b + n_b) of the rows of `table` (r.table), in the order of the rows; granted [B]
// tokens that got theirs (n_b or 0), slot (nullable) [B, max_n] their places page * 64 + offset, -1 for the others.
hipError_t pages_assign(const PageStack& st, const PageRows& r, int32_t* table, int32_t* granted, int64_t* slot,
                        hipStream_t s);
// Takes those pages back and clears their entries.
hipError_t pages_release(const PageStack& st, const PageRows& r, int32_t* table, hipStream_t s);

// table[at[i]] = id[i] (host arrays, copied into the launches).
hipError_t table_set(int32_t* table, const int32_t* at, const int32_t* id, int n, hipStream_t s);
// The entries [from, per_row) of every row name no page (-1).
hipError_t table_clear(int32_t* table, int rows, int per_row, int from, hipStream_t s);

// Attention of the window's queries q [B, H, L, dh] (L = r.max_n) over the committed positions
// and, with k, the window's own keys: o [B, L, H dh], lse (nullable) [B, H, L].  Rows at and
// behind n_b are left as they are; a query without keys gives 0 and -inf.
struct PageAttend {
  PageLayer p;
  PageRows r;
  const void *q, *k, *vt;
  void* o;
  float* lse;
  int H, cap;
  void* work;  // page_attend_work() bytes
};
// The bytes of partial results that a call of this shape keeps between its kernels, the threads of its
// launch (below 2^32, or it fails), and the launch.
size_t page_attend_work(DType dt, int B, int H, int Hkv, int dh, int L, int max_len);
size_t page_attend_threads(DType dt, int B, int H, int Hkv, int dh, int L, int max_len);
hipError_t page_attend(DType dt, const PageAttend& a, hipStream_t s);

// The same for rows of which neighbours may share their leading pages (page_shared.hip): those are read once for all
// that share them.  page_plan finds the groups, runs of rows that have min_pages whole leading pages or more in
// common with the row before, and lays out what the blocks of page_attend_shared do with these rows' tables and
// lengths (plan: page_plan_bytes(), 16-byte aligned); lead, pages (nullable, [B]): each row's group by its first row, and the
// pages that the group has in common.
constexpr int PAGE_SHARE_ROWS = 1024;  // rows of a plan: a thread of a block each
size_t page_plan_bytes(DType dt, int B, int H, int Hkv, int L);
size_t page_shared_work(DType dt, int B, int H, int Hkv, int dh, int L);
size_t page_shared_threads(DType dt, int B, int H, int Hkv, int L);
hipError_t page_plan(DType dt, const PageRows& r, int H, int Hkv, int dh, int min_pages, int32_t* plan, int32_t* lead,
                     int32_t* pages, hipStream_t s);
hipError_t page_attend_shared(DType dt, const PageAttend& a, const int32_t* plan, hipStream_t s);

}  // namespace tadm
