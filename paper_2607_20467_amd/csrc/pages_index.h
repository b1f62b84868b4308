// Where a packed call's rows and a sequence's keys are: every index that a kernel forms from device data (sequence
// borders, lengths, page numbers) goes through these functions, which never leave the caller's buffers whatever that
// data holds. Plain C++, so that they also compile for the host.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define DCL_HD __host__ __device__ __forceinline__
#else
#define DCL_HD inline
#endif

namespace dcl {

// Rows [first, first + n) of a packed [T, ...] operand that belong to sequence b: borders outside [0, T] are moved
// inside, a border below the one before it gives no rows.
struct SeqRows {
  int first, n;
};
DCL_HD SeqRows rows_between(int lo, int hi, int T) {
  lo = lo < 0 ? 0 : lo > T ? T : lo;
  hi = hi < lo ? lo : hi > T ? T : hi;
  return {lo, hi - lo};
}
DCL_HD SeqRows seq_rows(const int32_t* cu, int b, int T) { return rows_between(cu[b], cu[b + 1], T); }

// Length of a sequence as the kernels use it: [0, 2^30], so that positions and their sums stay in 32 bits.
DCL_HD int length_of(int n) { return n < 0 ? 0 : n > (1 << 30) ? (1 << 30) : n; }
DCL_HD int seq_len(const int32_t* len, int b) { return length_of(len[b]); }

// Page that holds positions [16 c, 16 c + 16) of a sequence whose table row is `row` (max_pages entries, pages of
// 2^shift positions), or -1: past the table, or an entry outside [0, n_pages).
DCL_HD int page_of(const int32_t* row, int max_pages, int n_pages, int shift, int c) {
  const int slot = c >> (shift - 4);
  if (c < 0 || slot >= max_pages) return -1;
  const int page = row[slot];
  return page >= 0 && page < n_pages ? page : -1;
}

// The same in two steps, for a load that nothing waits for: the entry to look at (of a row of max_pages >= 1), and the page that
// what was found there stands for.
DCL_HD int page_entry(int max_pages, int shift, int c) {
  const int slot = c >> (shift - 4);
  return slot < 0 ? 0 : slot < max_pages ? slot : max_pages - 1;
}
DCL_HD int page_found(int page, int max_pages, int n_pages, int shift, int c) {
  return c >= 0 && (c >> (shift - 4)) < max_pages && page >= 0 && page < n_pages ? page : -1;
}

}  // namespace dcl
