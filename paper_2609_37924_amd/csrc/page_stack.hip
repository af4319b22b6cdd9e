// Page tables kept on the device: rows take pages from a stack of free ones and give them back.
//
// A row of len positions uses the entries [0, ceil(len / 64)) of its table.  n more tokens need the entries
// [ceil(len / 64), ceil((len + n) / 64)), which follow from the lengths alone, so that every block of a
// launch finds by itself where its row's pages stand in the stack: a sum over the rows before it.  Both calls
// are a launch; nothing visits the host.
#include "common.h"
#include "pages.h"

namespace tadm {
namespace {

// state: free pages, an unused word, and between the blocks of a launch 64 bits, pages taken above blocks done (0 outside of one)
enum { FREE = 0, PROGRESS = 2 };

__device__ __forceinline__ int up(int x) { return (x + PAGE - 1) / PAGE; }

// A row's new tokens: the positions [len, len + n) and the entries [first, first + need) that they need.
struct Span {
  int len, n, first, need;
};
__device__ __forceinline__ Span span_of(const PageRows& r, int b) {
  Span s{row_len(r, b), row_new(r, b), 0, 0};
  if (s.len + s.n > r.max_pages * PAGE) s.n = 0;  // past the table: none of them
  s.first = up(s.len);
  s.need = up(s.len + s.n) - s.first;
  return s;
}

// Sum over the block's threads, every one receiving it (256 threads).
__device__ __forceinline__ int block_total(int v, int* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0] + red[1] + red[2] + red[3];
  __syncthreads();
  return v;
}

constexpr int CHUNK = 2048;  // tokens of a block

// grid (chunks of the window, rows).  Bound by its launch and the atomic that counts the blocks: 64 rows x 1 token 3.9 us,
// x 4 096 tokens with their slots (2.1 MB) 5.9; in chunks of 512, four times the blocks, 3 us more.
__global__ __launch_bounds__(256) void assign_kernel(PageStack st, PageRows r, int32_t* table, int32_t* granted,
                                                     int64_t* slot) {
  __shared__ int red[4];
  __shared__ int s_free;
  const int b = blockIdx.y, tid = threadIdx.x;
  if (tid == 0) s_free = min(max(st.state[FREE], 0), st.size);
  int before = 0;
  for (int a = tid; a < b; a += 256) before += span_of(r, a).need;
  const Span s = span_of(r, b);
  before = block_total(before, red);
  const int free = s_free;
  const bool all = s.need == 0 || before + s.need <= free;
  const int n = all ? s.n : 0, need = all ? s.need : 0;
  int32_t* row = table + (size_t)b * r.max_pages;
  const int32_t* top = st.id + (free - 1 - before);  // the row's k-th page is top[-k]
  // the chunk's entries are those that begin at one of its tokens
  const int j0 = blockIdx.x * CHUNK, j1 = min(j0 + CHUNK, r.max_n);
  if (tid <= CHUNK / PAGE) {
    const int e = max(up(s.len + j0), s.first) + tid;
    if (e - s.first < need && e * PAGE < s.len + j1) row[e] = top[s.first - e];
  }
  if (blockIdx.x == 0 && tid == 0) granted[b] = n;
  if (slot) {
    int64_t* out = slot + (size_t)b * r.max_n;
    for (int j = j0 + tid; j < j1; j += 256) {
      const int p = s.len + j, e = p / PAGE;
      int id = -1;
      if (j < n) id = e >= s.first ? top[s.first - e] : row[e];
      out[j] = (unsigned)id < (unsigned)st.size ? (int64_t)id * PAGE + p % PAGE : -1;
    }
  }
  if (tid == 0) {  // the last block, when every other has read the count, sets it; what each took rides on the same atomic
    unsigned long long* progress = reinterpret_cast<unsigned long long*>(st.state + PROGRESS);
    const unsigned long long mine = (unsigned long long)(blockIdx.x == 0 ? need : 0) << 32 | 1, old = atomicAdd(progress, mine);
    if ((uint32_t)old == gridDim.x * gridDim.y - 1) {
      st.state[FREE] = free - (int)((old + mine) >> 32);
      *progress = 0;
    }
  }
}

constexpr int RELEASE_THREADS = 1024, PER_ROW = PAGE_STACK_ROWS / RELEASE_THREADS, PER = 4;

// The sum of v over the threads before this one, and over all (RELEASE_THREADS threads).
__device__ __forceinline__ int scan_before(int v, int* red, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(sum, o, 64);
    if (lane >= o) sum += t;
  }
  if (lane == 63) red[wave] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < RELEASE_THREADS / 64; ++w) {
    before += w < wave ? red[w] : 0;
    all += red[w];
  }
  __syncthreads();
  *total = all;
  return before + sum - v;
}

// One block: the rows' entries one after the other, PER of them a thread, the present ones packed
// behind the free pages in that order.  Bound by its launch and the way lengths -> entries -> table -> place in the stack:
// 64 rows x 1 token 4.2 us, x 4 096 tokens 7.4.
__global__ __launch_bounds__(RELEASE_THREADS) void release_kernel(PageStack st, PageRows r, int32_t* table) {
  __shared__ int at[PAGE_STACK_ROWS + 1];  // the first of each row's entries among all
  __shared__ int red[RELEASE_THREADS / 64];
  const int tid = threadIdx.x;
  int need[PER_ROW], mine = 0, total;
#pragma unroll
  for (int i = 0; i < PER_ROW; ++i) {
    const int b = tid * PER_ROW + i;
    need[i] = b < r.B ? span_of(r, b).need : 0;
    mine += need[i];
  }
  int sum = scan_before(mine, red, &total);
#pragma unroll
  for (int i = 0; i < PER_ROW; ++i) {
    at[tid * PER_ROW + i] = sum;
    sum += need[i];
  }
  if (tid == RELEASE_THREADS - 1) at[PAGE_STACK_ROWS] = total;
  int top = min(max(st.state[FREE], 0), st.size);
  __syncthreads();
  for (int base = 0; base < total; base += RELEASE_THREADS * PER) {
    int32_t id[PER];
    int count = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = base + tid * PER + i;
      id[i] = -1;
      if (x < total) {
        int lo = 0, hi = r.B;  // the last row whose first entry is at or before x has it
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (at[mid] <= x)
            lo = mid;
          else
            hi = mid;
        }
        int32_t* e = table + (size_t)lo * r.max_pages + up(row_len(r, lo)) + (x - at[lo]);
        id[i] = *e;
        *e = -1;
      }
      if ((unsigned)id[i] < (unsigned)st.size) ++count;
    }
    int all, to = top + scan_before(count, red, &all);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((unsigned)id[i] < (unsigned)st.size) {
        if (to < st.size) st.id[to] = id[i];  // more than the stack holds: a page that came back twice
        ++to;
      }
    top += all;
  }
  if (tid == 0) st.state[FREE] = min(top, st.size);
}

}  // namespace

hipError_t pages_assign(const PageStack& st, const PageRows& r, int32_t* table, int32_t* granted, int64_t* slot,
                        hipStream_t s) {
  hipLaunchKernelGGL(assign_kernel, dim3((r.max_n + CHUNK - 1) / CHUNK, r.B), dim3(256), 0, s, st, r, table, granted, slot);
  return hipGetLastError();
}

hipError_t pages_release(const PageStack& st, const PageRows& r, int32_t* table, hipStream_t s) {
  hipLaunchKernelGGL(release_kernel, dim3(1), dim3(RELEASE_THREADS), 0, s, st, r, table);
  return hipGetLastError();
}

}  // namespace tadm
