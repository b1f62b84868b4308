// Pages handed out to new tokens and taken back, from lengths in device memory.
#include "dcl_internal.h"
#include "pages_index.h"

namespace dcl {

// Who gets what is three running sums over the sequences, each of what the one before let pass: tokens that fit the T rows,
// pages that the list still holds, tokens granted. One workgroup walks the sequences in windows with the sums carried along; the
// sums stop at 2^31 - 1, so that they never wrap: what a thread adds is at most 2^30 tokens or 2^26 pages, so that a sum that
// stopped stays past the limits it is compared with (2^22 rows, 2^30 pages) when the thread's own share is taken off it. Rows are
// then independent: each looks its sequence up among the borders. Every index formed from device data is clamped before it is
// used.
constexpr int kSmall = 256, kWindow = 1024;  // threads of the workgroup: few sequences and rows, or any
constexpr int kItems = 4;                    // sequences of a thread where there are many
constexpr uint32_t kMost = 0x7FFFFFFFu;

__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// Inclusive running sum over the workgroup's W threads, on top of `before`. `sh`: W / 64 words.
template <int W>
__device__ __forceinline__ uint32_t running_sum(uint32_t v, uint32_t before, uint32_t* sh) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = (uint32_t)__shfl_up((int)v, o, 64);
    if (lane >= o) v = add_up(v, x);
  }
  __syncthreads();
  if (lane == 63) sh[w] = v;
  __syncthreads();
  uint32_t base = before;
#pragma unroll
  for (int i = 0; i < W / 64; ++i)
    if (i < w) base = add_up(base, sh[i]);
  return add_up(base, v);
}
// What the last thread has, for all.
template <int W>
__device__ __forceinline__ uint32_t last_of(uint32_t v, uint32_t* sh) {
  __syncthreads();
  if (threadIdx.x == W - 1) sh[0] = v;
  __syncthreads();
  const uint32_t r = sh[0];
  __syncthreads();
  return r;
}

__device__ __forceinline__ int pages_for(int n, int shift) { return (int)(((long)n + (1 << shift) - 1) >> shift); }

// Largest b in [lo, hi) with at[b] <= x (at[lo] <= x).
__device__ __forceinline__ int find_last(const int32_t* at, int lo, int hi, int x) {
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Workspace: [0] the list's length before the call, [1] pages that go back at most, [2 + b] pages before sequence b,
// [2 + B + b] its first page that goes back, [2 + 2 B + g] pages that come back through workgroup g.
constexpr int kBackGroups = 64;
size_t pages_turn_ws_ints(int B) { return 2 + 2 * (size_t)B + kBackGroups; }

// ---------------------------------------------------------------- extend
// One packed row: its position, its place, and, where it is a new page's first, the page into the table. start: pages that the
// sequences before b took; list: free pages before the call.
__device__ __forceinline__ void extend_row(const PagesTurn& a, int t, int b, int first, int n, int length, int start, int list) {
  const int mask = (1 << a.shift) - 1, x = length - n + (t - first), j = x >> a.shift;
  const int fresh = j - pages_for(length - n, a.shift);  // which of the sequence's new pages
  int32_t* entry = a.table + (size_t)b * a.max_pages + j;
  const int page = fresh >= 0 ? a.free_pages[list - 1 - start - fresh] : *entry;
  if (fresh >= 0 && (x & mask) == 0) *entry = page;
  if (a.pos) a.pos[t] = x;
  if (a.slot) a.slot[t] = page >= 0 && page < a.n_pages ? ((int64_t)page << a.shift) + (x & mask) : -1;
}
__device__ __forceinline__ void no_row(const PagesTurn& a, int t) {
  if (a.pos) a.pos[t] = -1;
  if (a.slot) a.slot[t] = -1;
}

// Borders, lengths, the list's length, and into the workspace what the rows need. ROWS: the rows too, for up to W sequences.
template <int W, bool ROWS>
__global__ void __launch_bounds__(W) extend_kernel(PagesTurn a) {
  constexpr int IT = ROWS ? 1 : kItems;
  __shared__ uint32_t sh[W / 64];
  __shared__ int32_t s_cu[ROWS ? W + 1 : 1], s_n[ROWS ? W : 1], s_start[ROWS ? W : 1];
  const int tid = threadIdx.x;
  const int list = max(0, min(*a.n_free, a.n_pages));
  const long capacity = (long)a.max_pages << a.shift;
  uint32_t asked = 0, wanted = 0, granted = 0, used = 0;
  for (int w = 0; w < a.B; w += W * IT) {
    const int b0 = w + tid * IT;
    int n[IT], c[IT];
    uint32_t need[IT], sum;
    bool ok[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int b = b0 + i;
      n[i] = c[i] = 0;
      ok[i] = false;
      if (b < a.B) {
        n[i] = a.len[b];
        c[i] = a.ask ? a.ask[b] : 1;
        ok[i] = n[i] >= 0 && c[i] >= 0 && (long)n[i] + c[i] <= capacity;
      }
    }
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) sum += ok[i] ? c[i] : 0;
    const uint32_t rows = running_sum<W>(sum, asked, sh);
    uint32_t upto = rows - sum;
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      upto += ok[i] ? c[i] : 0;
      ok[i] = ok[i] && upto <= (uint32_t)a.T;
      need[i] = ok[i] ? pages_for(n[i] + c[i], a.shift) - pages_for(n[i], a.shift) : 0;
      sum += need[i];
    }
    const uint32_t pages = running_sum<W>(sum, wanted, sh);
    uint32_t start = pages - sum;
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      start += need[i];
      ok[i] = ok[i] && (need[i] == 0 || start <= (uint32_t)list);
      if (ok[i] && need[i]) used = start;
      sum += ok[i] ? c[i] : 0;
    }
    const uint32_t ends = running_sum<W>(sum, granted, sh);
    uint32_t end = ends - sum;
    start = pages;
#pragma unroll
    for (int i = 0; i < IT; ++i) start -= need[i];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int b = b0 + i;
      end += ok[i] ? c[i] : 0;
      if (b < a.B) {
        a.cu[b + 1] = (int)end;
        if (ok[i] && c[i]) a.len[b] = n[i] + c[i];
        if (ROWS) {
          s_cu[b + 1] = (int)end;
          s_n[b] = n[i] + c[i];
          s_start[b] = (int)start;
        } else {
          a.ws[2 + b] = (int)start;
        }
      }
      start += need[i];
    }
    if (!ROWS) {
      asked = last_of<W>(rows, sh);
      wanted = last_of<W>(pages, sh);
      granted = last_of<W>(ends, sh);
    }
  }
  // the sequences that take pages are the first of those that need some: the last one's sum is what the list loses
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) used = max(used, (uint32_t)__shfl_xor((int)used, o, 64));
  __syncthreads();
  if ((tid & 63) == 0) sh[tid >> 6] = used;
  if (ROWS && tid == 0) s_cu[0] = 0;
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < W / 64; ++i) used = max(used, sh[i]);
    a.cu[0] = 0;
    *a.n_free = list - (int)used;
    if (!ROWS) a.ws[0] = list;
  }
  if constexpr (ROWS) {
    const int end = s_cu[a.B];
    for (int t = tid; t < a.T; t += W) {
      if (t >= end) {
        no_row(a, t);
        continue;
      }
      const int b = find_last(s_cu, 0, a.B, t);
      extend_row(a, t, b, s_cu[b], s_cu[b + 1] - s_cu[b], s_n[b], s_start[b], list);
    }
  }
}

__global__ void __launch_bounds__(256) extend_rows_kernel(PagesTurn a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= a.T) return;
  if (t >= a.cu[a.B]) {
    no_row(a, t);
    return;
  }
  const int b = find_last(a.cu, 0, a.B, t), first = a.cu[b];
  extend_row(a, t, b, first, a.cu[b + 1] - first, a.len[b], a.ws[2 + b], a.ws[0]);
}

void launch_pages_extend(const PagesTurn& a, hipStream_t s) {
  if (a.B <= kSmall && a.T <= 4 * kSmall) {
    hipLaunchKernelGGL((extend_kernel<kSmall, true>), dim3(1), dim3(kSmall), 0, s, a);
    return;
  }
  if (a.B <= kWindow && a.T <= 16 * kWindow) {
    hipLaunchKernelGGL((extend_kernel<kWindow, true>), dim3(1), dim3(kWindow), 0, s, a);
    return;
  }
  hipLaunchKernelGGL((extend_kernel<kWindow, false>), dim3(1), dim3(kWindow), 0, s, a);
  if (a.T > 0) hipLaunchKernelGGL(extend_rows_kernel, dim3((a.T + 255) / 256), dim3(256), 0, s, a);
}

// ---------------------------------------------------------------- shrink
// Entries that may go back are numbered through, sequence by sequence; those that name a page are counted, and the i-th of
// `all` goes to place list + all - 1 - i.
__device__ __forceinline__ int32_t* back_entry(const PagesTurn& a, const int32_t* start, const int32_t* first, int i) {
  const int b = find_last(start, 0, a.B, i);
  return a.table + (size_t)b * a.max_pages + first[b] + (i - start[b]);
}
__device__ __forceinline__ bool names_page(const PagesTurn& a, int page) { return page >= 0 && page < a.n_pages; }

// Entries [from, to) of the numbering, in windows of the workgroup: how many name a page.
template <int W>
__device__ uint32_t back_count(const PagesTurn& a, const int32_t* start, const int32_t* first, int from, int to, uint32_t* sh) {
  uint32_t n = 0;
  for (long i = (long)from + threadIdx.x; i < to; i += W) n += names_page(a, *back_entry(a, start, first, (int)i));
  return last_of<W>(running_sum<W>(n, 0, sh), sh);
}
// The same entries onto the list, `before` of `all` being those of entries before them.
template <int W>
__device__ void back_write(const PagesTurn& a, const int32_t* start, const int32_t* first, int from, int to, uint32_t before,
                           uint32_t all, int list, uint32_t* sh) {
  for (long w = from; w < to; w += W) {
    const long i = w + threadIdx.x;
    int page = -1;
    if (i < to) {
      int32_t* entry = back_entry(a, start, first, (int)i);
      page = *entry;
      *entry = -1;
    }
    const bool real = names_page(a, page);
    const uint32_t upto = running_sum<W>(real, before, sh);
    const long place = (long)list + all - upto;
    if (real && place < a.n_pages) a.free_pages[place] = page;
    before = last_of<W>(upto, sh);
  }
}

template <int W, bool WHOLE>
__global__ void __launch_bounds__(W) shrink_kernel(PagesTurn a) {
  constexpr int IT = WHOLE ? 1 : kItems;
  __shared__ uint32_t sh[W / 64];
  __shared__ int32_t s_start[WHOLE ? W : 1], s_first[WHOLE ? W : 1];
  const int tid = threadIdx.x;
  const int list = max(0, min(*a.n_free, a.n_pages));
  const long capacity = (long)a.max_pages << a.shift;
  uint32_t total = 0;
  for (int w = 0; w < a.B; w += W * IT) {
    const int b0 = w + tid * IT;
    uint32_t n[IT], sum = 0;
    int first[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int b = b0 + i;
      n[i] = 0;
      first[i] = 0;
      if (b < a.B) {
        const int len = a.len[b], keep = a.ask[b];
        if (keep >= 0 && keep < len && len <= capacity) {
          first[i] = pages_for(keep, a.shift);
          n[i] = pages_for(len, a.shift) - first[i];
          a.len[b] = keep;
        }
      }
      sum += n[i];
    }
    const uint32_t upto = running_sum<W>(sum, total, sh);
    uint32_t at = upto - sum;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int b = b0 + i;
      if (b < a.B) {
        (WHOLE ? s_start : a.ws + 2)[b] = (int)at;
        (WHOLE ? s_first : a.ws + 2 + a.B)[b] = first[i];
      }
      at += n[i];
    }
    total = last_of<W>(upto, sh);
  }
  if constexpr (WHOLE) {
    const uint32_t all = back_count<W>(a, s_start, s_first, 0, (int)total, sh);
    back_write<W>(a, s_start, s_first, 0, (int)total, 0, all, list, sh);
    if (tid == 0) *a.n_free = (int)min((long)list + all, (long)a.n_pages);
  } else if (tid == 0) {
    a.ws[0] = list;
    a.ws[1] = (int)total;
  }
}

__device__ __forceinline__ void back_span(const PagesTurn& a, int* from, int* to) {
  const long total = a.ws[1], per = (total + kBackGroups - 1) / kBackGroups;
  *from = (int)min(per * blockIdx.x, total);
  *to = (int)min(per * (blockIdx.x + 1), total);
}

__global__ void __launch_bounds__(kWindow) back_count_kernel(PagesTurn a) {
  __shared__ uint32_t sh[kWindow / 64];
  int from, to;
  back_span(a, &from, &to);
  const uint32_t n = back_count<kWindow>(a, a.ws + 2, a.ws + 2 + a.B, from, to, sh);
  if (threadIdx.x == 0) a.ws[2 + 2 * a.B + blockIdx.x] = (int)n;
}

__global__ void __launch_bounds__(kWindow) back_write_kernel(PagesTurn a) {
  __shared__ uint32_t sh[kWindow / 64];
  __shared__ uint32_t s_before;
  int from, to;
  back_span(a, &from, &to);
  const int tid = threadIdx.x, list = a.ws[0];
  const uint32_t n = tid < kBackGroups ? (uint32_t)a.ws[2 + 2 * a.B + tid] : 0, upto = running_sum<kWindow>(n, 0, sh);
  if (tid == (int)blockIdx.x) s_before = upto - n;
  const uint32_t all = last_of<kWindow>(upto, sh);
  back_write<kWindow>(a, a.ws + 2, a.ws + 2 + a.B, from, to, s_before, all, list, sh);
  if (blockIdx.x == 0 && tid == 0) *a.n_free = (int)min((long)list + all, (long)a.n_pages);
}

void launch_pages_shrink(const PagesTurn& a, hipStream_t s) {
  if (a.B <= kSmall && (long)a.B * a.max_pages <= 32 * kSmall) {
    hipLaunchKernelGGL((shrink_kernel<kSmall, true>), dim3(1), dim3(kSmall), 0, s, a);
    return;
  }
  if (a.B <= kWindow && (long)a.B * a.max_pages <= 16 * kWindow) {
    hipLaunchKernelGGL((shrink_kernel<kWindow, true>), dim3(1), dim3(kWindow), 0, s, a);
    return;
  }
  hipLaunchKernelGGL((shrink_kernel<kWindow, false>), dim3(1), dim3(kWindow), 0, s, a);
  hipLaunchKernelGGL(back_count_kernel, dim3(kBackGroups), dim3(kWindow), 0, s, a);
  hipLaunchKernelGGL(back_write_kernel, dim3(kBackGroups), dim3(kWindow), 0, s, a);
}

}  // namespace dcl
