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
//
// These are launches and chains of loads, not bytes: 64 sequences with a token each 2.9 us to extend and 1.6 to shrink; 3000 with 257000
// rows 6.2 (the sums, one workgroup) and 5.3 (the rows), and back 5.5 (sums and counts) and 4.4 (pages and lengths); 65536 sequences 98
// and 71 for the sums, 6 and 4 us a window of 4096, whose strided loads and stores one CU makes alone.
constexpr int kSmall = 256, kWindow = 1024;  // threads of the workgroup: few sequences and rows, or any
constexpr int kItems = 4;                    // sequences of a thread where there are many
constexpr uint32_t kMost = 0x7FFFFFFFu;

__device__ __forceinline__ uint32_t add_up(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// What these workgroups' threads exchange goes through LDS alone, so that a barrier need not wait for loads and stores on their way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Inclusive running sum over the wave: inside rows of 16 lanes, then the rows' last lanes on the rows behind them.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t plus_shifted(uint32_t v) {
  return add_up(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
  v = plus_shifted<0x111, 0xF>(v);
  v = plus_shifted<0x112, 0xF>(v);
  v = plus_shifted<0x114, 0xF>(v);
  v = plus_shifted<0x118, 0xF>(v);
  v = plus_shifted<0x142, 0xA>(v);
  return plus_shifted<0x143, 0xC>(v);
}

// Inclusive running sum over the workgroup's W threads, on top of `all`, which becomes the sum of all. `sh`: W / 64 words, which
// nothing before the last barrier reads.
template <int W>
__device__ __forceinline__ uint32_t running_sum(uint32_t v, uint32_t& all, uint32_t* sh) {
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  v = wave_sum(v);
  if (lane == 63) sh[w] = v;
  lds_barrier();
  // the waves' sums again in a row of 16 lanes
  uint32_t x = (lane & 15) < W / 64 ? sh[lane & 15] : 0;
  x = plus_shifted<0x111, 0xF>(x);
  x = plus_shifted<0x112, 0xF>(x);
  x = plus_shifted<0x114, 0xF>(x);
  x = plus_shifted<0x118, 0xF>(x);
  const uint32_t before = all;
  all = add_up(all, (uint32_t)__builtin_amdgcn_readlane((int)x, 15));
  const uint32_t base = w ? add_up(before, (uint32_t)__builtin_amdgcn_readlane((int)x, w - 1)) : before;
  return add_up(base, v);
}

__device__ __forceinline__ int pages_for(int n, int shift) { return (n + (1 << shift) - 1) >> shift; }  // n <= 2^28

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

// The same for the values x, not falling, of a wave's lanes, by all lanes together: 64 borders a look, for the first lane's place and
// the last one's at once (three looks for 2^16 sequences, where a lane alone waits for sixteen loads one after the other), then
// each lane between the two.
__device__ __forceinline__ int find_rising(const int32_t* at, int n, int x) {
  const int lane = threadIdx.x & 63, x0 = __builtin_amdgcn_readfirstlane(x), x1 = __builtin_amdgcn_readlane(x, 63);
  int lo0 = 0, hi0 = n, lo1 = 0, hi1 = n;
  while (max(hi0 - lo0, hi1 - lo1) > 1) {  // a range of one stays as it is
    const int step0 = (hi0 - lo0 + 63) >> 6, i0 = lo0 + step0 * lane, step1 = (hi1 - lo1 + 63) >> 6, i1 = lo1 + step1 * lane;
    const int v0 = at[min(i0, hi0 - 1)], v1 = at[min(i1, hi1 - 1)];
    lo0 += step0 * (__popcll(__builtin_amdgcn_ballot_w64(i0 < hi0 && v0 <= x0)) - 1);
    lo1 += step1 * (__popcll(__builtin_amdgcn_ballot_w64(i1 < hi1 && v1 <= x1)) - 1);
    hi0 = min(lo0 + step0, hi0);
    hi1 = min(lo1 + step1, hi1);
  }
  return find_last(at, lo0, lo1 + 1, x);
}

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
  __shared__ uint32_t sh[3][W / 64];
  __shared__ int32_t s_cu[ROWS ? W + 1 : 1], s_n[ROWS ? W : 1], s_start[ROWS ? W : 1];
  const int tid = threadIdx.x;
  const int list = max(0, min(*a.n_free, a.n_pages));
  const int capacity = a.max_pages << a.shift;  // at most 2^28
  uint32_t asked = 0, wanted = 0, granted = 0, used = 0;
  int n[IT], c[IT], n_next[IT], c_next[IT];
  auto ahead = [&](int b0) {  // the window after this one
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      n_next[i] = b0 + i < a.B ? a.len[b0 + i] : -1;
      c_next[i] = b0 + i < a.B && a.ask ? a.ask[b0 + i] : 1;
    }
  };
  ahead(tid * IT);
  for (int w = 0; w < a.B; w += W * IT) {
    const int b0 = w + tid * IT;
    uint32_t need[IT], sum;
    bool ok[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      n[i] = n_next[i];
      c[i] = c_next[i];
      ok[i] = n[i] >= 0 && n[i] <= capacity && c[i] >= 0 && c[i] <= capacity - n[i];
    }
    if (!ROWS) ahead(b0 + W * IT);
    asm volatile("" ::"v"(list));  // every wave has read it before the barriers behind which it is written
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) sum += ok[i] ? c[i] : 0;
    uint32_t upto = running_sum<W>(sum, asked, sh[0]) - sum;
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      upto += ok[i] ? c[i] : 0;
      ok[i] = ok[i] && upto <= (uint32_t)a.T;
      need[i] = ok[i] ? pages_for(n[i] + c[i], a.shift) - pages_for(n[i], a.shift) : 0;
      sum += need[i];
    }
    const uint32_t first = running_sum<W>(sum, wanted, sh[1]) - sum;
    uint32_t start = first;
    sum = 0;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      start += need[i];
      ok[i] = ok[i] && (need[i] == 0 || start <= (uint32_t)list);
      if (ok[i] && need[i]) used = start;
      sum += ok[i] ? c[i] : 0;
    }
    uint32_t end = running_sum<W>(sum, granted, sh[2]) - sum;
    start = first;
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
    if (!ROWS) lds_barrier();  // before sh is written again
  }
  // the sequences that take pages are the first of those that need some: the last one's sum is what the list loses
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) used = max(used, (uint32_t)__shfl_xor((int)used, o, 64));
  if ((tid & 63) == 0) sh[0][tid >> 6] = used;  // read last before the third sum's barrier
  if (ROWS && tid == 0) s_cu[0] = 0;
  lds_barrier();
  if (tid == 0) {
    for (int i = 1; i < W / 64; ++i) used = max(used, sh[0][i]);
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
  const int t = blockIdx.x * 256 + threadIdx.x, end = a.cu[a.B], list = a.ws[0];
  const int b = find_rising(a.cu, a.B, t);  // every lane of the wave takes part
  if (t >= a.T) return;
  if (t >= end) {
    no_row(a, t);
    return;
  }
  const int first = a.cu[b];
  extend_row(a, t, b, first, a.cu[b + 1] - first, a.len[b], a.ws[2 + b], list);
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
template <bool WHOLE>
__device__ __forceinline__ int32_t* back_entry(const PagesTurn& a, const int32_t* start, const int32_t* first, int i) {
  const int b = WHOLE ? find_last(start, 0, a.B, i) : find_rising(start, a.B, i);
  return a.table + (size_t)b * a.max_pages + first[b] + (i - start[b]);
}
__device__ __forceinline__ bool names_page(const PagesTurn& a, int page) { return page >= 0 && page < a.n_pages; }

// Entries [from, to) of the numbering, in windows of the workgroup: how many name a page. WHOLE: start and first in LDS. What a
// thread past the end would look at is the last entry.
template <int W, bool WHOLE>
__device__ uint32_t back_count(const PagesTurn& a, const int32_t* start, const int32_t* first, int from, int to, uint32_t* sh) {
  uint32_t n = 0, all = 0;
  for (long w = from; w < to; w += W) {
    const long i = w + threadIdx.x;
    const int32_t* entry = back_entry<WHOLE>(a, start, first, (int)min(i, (long)to - 1));
    if (i < to) n += names_page(a, *entry);
  }
  running_sum<W>(n, all, sh);
  return all;
}
// The same entries onto the list, `before` of `all` being those of entries before them. sh: two times W / 64 words.
template <int W, bool WHOLE>
__device__ void back_write(const PagesTurn& a, const int32_t* start, const int32_t* first, int from, int to, uint32_t before,
                           uint32_t all, int list, uint32_t* sh) {
  int turn = 0;
  for (long w = from; w < to; w += W, turn ^= W / 64) {  // a barrier lies between a window's reads of sh and the next but one's writes
    const long i = w + threadIdx.x;
    int32_t* entry = back_entry<WHOLE>(a, start, first, (int)min(i, (long)to - 1));
    int page = -1;
    if (i < to) {
      page = *entry;
      *entry = -1;
    }
    const bool real = names_page(a, page);
    const long place = (long)list + all - running_sum<W>(real, before, sh + turn);
    if (real && place < a.n_pages) a.free_pages[place] = page;
  }
}

__device__ __forceinline__ void back_span(long total, int* from, int* to) {
  const long per = (total + kBackGroups - 1) / kBackGroups;
  *from = (int)min(per * blockIdx.x, total);
  *to = (int)min(per * (blockIdx.x + 1), total);
}

// WHOLE: one workgroup does it all. SPREAD: the sequences are one window, whose sums each of the workgroups makes for itself, so that it
// can count its share of the entries in the same launch; lengths stay until the next one, since others may still read them.
// ALONE: one workgroup for any number of sequences, before two launches.
enum { WHOLE, SPREAD, ALONE };
template <int W, int MODE>
__global__ void __launch_bounds__(W) shrink_kernel(PagesTurn a) {
  constexpr int IT = MODE == WHOLE ? 1 : kItems;
  __shared__ uint32_t sh[4][W / 64];
  __shared__ int32_t s_start[MODE == ALONE ? 1 : W * IT], s_first[MODE == ALONE ? 1 : W * IT];
  const int tid = threadIdx.x;
  const int list = max(0, min(*a.n_free, a.n_pages));
  const int capacity = a.max_pages << a.shift;  // at most 2^28
  uint32_t total = 0;
  int len_next[IT], keep_next[IT];
  auto ahead = [&](int b0) {  // the window after this one
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      len_next[i] = b0 + i < a.B ? a.len[b0 + i] : 0;
      keep_next[i] = b0 + i < a.B ? a.ask[b0 + i] : -1;
    }
  };
  ahead(tid * IT);
  for (int w = 0; w < a.B; w += W * IT) {
    const int b0 = w + tid * IT;
    uint32_t n[IT], sum = 0;
    int first[IT], len[IT], keep[IT];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      len[i] = len_next[i];
      keep[i] = keep_next[i];
    }
    if (MODE == ALONE) ahead(b0 + W * IT);
    asm volatile("" ::"v"(list));  // every wave has read it before the barriers behind which it is written
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      n[i] = 0;
      first[i] = 0;
      if (keep[i] >= 0 && keep[i] < len[i] && len[i] <= capacity) {
        first[i] = pages_for(keep[i], a.shift);
        n[i] = pages_for(len[i], a.shift) - first[i];
        if (MODE != SPREAD) a.len[b0 + i] = keep[i];
      }
      sum += n[i];
    }
    uint32_t at = running_sum<W>(sum, total, sh[0]) - sum;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int b = b0 + i;
      if (b < a.B) {
        if (MODE != ALONE) {
          s_start[b] = (int)at;
          s_first[b] = first[i];
        }
        if (MODE == ALONE || (MODE == SPREAD && blockIdx.x == 0)) {
          a.ws[2 + b] = (int)at;
          a.ws[2 + a.B + b] = first[i];
        }
      }
      at += n[i];
    }
    lds_barrier();  // before sh is written again, and s_start read
  }
  // How many come back the host does not know, only what the table could name: a few under a wide one are done with here by one
  // workgroup, and nothing but the lengths is left to the next launch (extend and shrink of 1000 sequences by up to 32 tokens, tables
  // of 2048 pages of 16: 17.1 us from a graph).
  const bool here = MODE == WHOLE || (MODE == SPREAD && total <= 2 * W);
  int after = list;
  if (here && blockIdx.x == 0) {
    const uint32_t all = back_count<W, true>(a, s_start, s_first, 0, (int)total, sh[1]);
    back_write<W, true>(a, s_start, s_first, 0, (int)total, 0, all, list, sh[2]);
    after = (int)min((long)list + all, (long)a.n_pages);
  }
  if (MODE == SPREAD) {
    int from, to;
    back_span(here ? 0 : total, &from, &to);
    const uint32_t n = back_count<W, true>(a, s_start, s_first, from, to, sh[0]);
    if (tid == 0) a.ws[2 + 2 * a.B + blockIdx.x] = (int)n;
  }
  if (tid == 0 && blockIdx.x == 0) {
    if (MODE == WHOLE) {
      *a.n_free = after;
    } else {
      a.ws[0] = after;
      a.ws[1] = here ? 0 : (int)total;
    }
  }
}

__global__ void __launch_bounds__(kWindow) back_count_kernel(PagesTurn a) {
  __shared__ uint32_t sh[kWindow / 64];
  int from, to;
  back_span(a.ws[1], &from, &to);
  const uint32_t n = back_count<kWindow, false>(a, a.ws + 2, a.ws + 2 + a.B, from, to, sh);
  if (threadIdx.x == 0) a.ws[2 + 2 * a.B + blockIdx.x] = (int)n;
}

template <bool LENGTHS>  // the lengths are cut here
__global__ void __launch_bounds__(kWindow) back_write_kernel(PagesTurn a) {
  __shared__ uint32_t sh[3][kWindow / 64];
  __shared__ uint32_t s_before;
  int from, to;
  back_span(a.ws[1], &from, &to);
  const int tid = threadIdx.x, list = a.ws[0], b = blockIdx.x * kWindow + tid;
  if (LENGTHS && b < a.B) {
    const int len = a.len[b], keep = a.ask[b];
    if (keep >= 0 && keep < len && len <= a.max_pages << a.shift) a.len[b] = keep;
  }
  const uint32_t n = tid < kBackGroups ? (uint32_t)a.ws[2 + 2 * a.B + tid] : 0;
  uint32_t all = 0;
  const uint32_t upto = running_sum<kWindow>(n, all, sh[0]);
  if (tid == (int)blockIdx.x) s_before = upto - n;
  lds_barrier();
  back_write<kWindow, false>(a, a.ws + 2, a.ws + 2 + a.B, from, to, s_before, all, list, sh[1]);
  if (blockIdx.x == 0 && tid == 0) *a.n_free = (int)min((long)list + all, (long)a.n_pages);
}

void launch_pages_shrink(const PagesTurn& a, hipStream_t s) {
  if (a.B <= kSmall && (long)a.B * a.max_pages <= 32 * kSmall) {
    hipLaunchKernelGGL((shrink_kernel<kSmall, WHOLE>), dim3(1), dim3(kSmall), 0, s, a);
    return;
  }
  if (a.B <= kWindow && (long)a.B * a.max_pages <= 16 * kWindow) {
    hipLaunchKernelGGL((shrink_kernel<kWindow, WHOLE>), dim3(1), dim3(kWindow), 0, s, a);
    return;
  }
  if (a.B <= kWindow * kItems) {
    hipLaunchKernelGGL((shrink_kernel<kWindow, SPREAD>), dim3(kBackGroups), dim3(kWindow), 0, s, a);
    hipLaunchKernelGGL(back_write_kernel<true>, dim3(kBackGroups), dim3(kWindow), 0, s, a);
    return;
  }
  hipLaunchKernelGGL((shrink_kernel<kWindow, ALONE>), dim3(1), dim3(kWindow), 0, s, a);
  hipLaunchKernelGGL(back_count_kernel, dim3(kBackGroups), dim3(kWindow), 0, s, a);
  hipLaunchKernelGGL(back_write_kernel<false>, dim3(kBackGroups), dim3(kWindow), 0, s, a);
}

}  // namespace dcl
