// Drawing one token per row of logits: temperature, top-k, top-p, min-p, one given uniform number per row.
//
// The ids of a row in order of (logit descending, id ascending) have weights w = exp((x - M) / T), M the row's maximum.
// Every filter keeps a prefix of that order, and the draw asks for the element at which the running sum passes
// u * total, so all of them are one question: at which element does the running count or the running sum of weights
// pass a value? It is answered without sorting the row: a histogram over the weights (32 bins per factor of 2, their sums, and
// their counts where top-k asks) says in which bin, and only that bin's elements (or, where they are few, all up to it) are
// collected into LDS, put in order and summed. A bin with more elements than fit is split again by value; equal values are answered by arithmetic.
//
// Weights are exponentials to 1e-13, held as whole numbers of 2^-shift, so every sum is exact in any order: results do not
// depend on timing, and a border falls as exact arithmetic on the weights has it (a float32 sum's error of 1e-7 would move
// one border in a hundred rows of a flat distribution over 10^5 ids).
//
// A workgroup per row: one kernel finds the row's maximum and answers rows that need no more (the top-1 alone) or little
// more (top-k with the ids down to its border in LDS: nothing else of the row needs a weight), one answers bfloat16 rows by a
// count of each value, and one the others from the histogram. Few rows are shared by several workgroups, in three kernels:
// maxima, then the parts' elements or histograms, then one workgroup a row for the answer. Rows of up to 2048 ids are lists as
// a whole, in one kernel.
//
// 512 rows of 152064 bfloat16 logits, each row with its own settings: 100 us. The first kernel (52) is bound by memory: 156 MB,
// and the rows with a top-k once more, mostly from the last cache; the second (45) by two passes over a row by one CU. The
// same in float32 without a filter: 200 us (211 with logits not in the caches), 57 of a row's time in the last kernel, 35 of them additions to the histogram in
// LDS (with the arithmetic of four elements interleaved 32, and low temperatures slower). 4 rows of 126464 float32, top-k 50
// and top-p 0.95: 22 us, three kernels of 6 to 9 us: chains of dependent loads, barriers and instruction fetches. Without
// sharing they took 35, rows without a filter 55 instead of 38.
#include <limits.h>

#include "dcl_internal.h"

namespace dcl {

constexpr int kBins = 2048, kList = 2048, kSampleThreads = 1024, kWaves = kSampleThreads / 64;
constexpr int kTable = 256;              // steps of a factor of 2: weights come from a table of 2^(i / 256)
constexpr int kTop = 64 * kTable;        // the maximum's step, which leaves those that count above 0
constexpr int kFar = 47 * 32;            // 32 bins per factor of 2; 2^-47 rounds to 0 of 2^-45 and more, so this bin is the last
constexpr double kMagic = 6755399441055744.0 + kTop;  // 1.5 * 2^52: the sum's last bit is 1, its low word the step
constexpr int kMaxParts = 16;

typedef unsigned long long u64;

// float as an unsigned number of the same order, -0 and +0 alike
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

struct Row {
  const char* base;
  const double* table;
  int V, head;       // vocabulary; elements before the row's first 16-byte line
  int p0, p1;        // the 16-byte pieces that this workgroup looks at
  bool edges;        // and whether the elements before and behind them all
  int drop;          // low bits that all order_keys have alike, or their complements
  float M;
  double rate;       // steps per unit of logit: 256 log2(e) / T

  // M finite
  __device__ __forceinline__ void set(float top, float T) {
    M = top;
    rate = kTable * 1.4426950408889634 / (double)T;
  }
  // A logit's step, added to kMagic - kTop: rises with x (as every operation in it does), kMagic for x = M.
  __device__ __forceinline__ double step(float x) const { return fma((double)x - (double)M, rate, kMagic); }
  __device__ __forceinline__ static uint32_t low_word(double t) { return (uint32_t)__double_as_longlong(t); }
  __device__ __forceinline__ static bool near(double t) { return t > kMagic - 8 * kFar; }
  // place in the histogram of a near one: 0 for x = M
  __device__ __forceinline__ static int place(double t) { return (int)((kTop - low_word(t)) >> 3); }
  __device__ __forceinline__ int bin(float x) const {
    const double t = step(x);
    return near(t) ? place(t) : kFar;
  }
  // 2^shift times the weight of a logit x <= M is 2^(shift - 64) 2^(step / 256) 2^(z / 256), z the rest that `step` rounds
  // off, |z| <= 1/2: the first two are table[step % 256] with step * 2^12 added to its high word (the entry has its index
  // taken off there, so that this leaves step / 256 in the exponent), the third is its series to the third power (the next
  // term is 1.4e-13). For steps above -200 * 256.
  struct Factors {
    double scale, rest;
  };
  __device__ __forceinline__ Factors factors(float x, double t) const {
    const double z = fma((double)x - (double)M, rate, kMagic - t);
    constexpr double c = 0.6931471805599453 / kTable;
    double p = fma(z, c * c * c / 6.0, c * c / 2.0);
    p = fma(z, p, c);
    p = fma(z, p, 1.0);
    const uint32_t k = low_word(t);
    const u64 bits = (u64)__double_as_longlong(table[k & (kTable - 1)]) + ((u64)(k << 12) << 32);
    return {__longlong_as_double((long long)bits), p};
  }
  __device__ __forceinline__ double weight(float x) const {
    const double t = step(x);
    if (!(t > kMagic - 200.0 * kTable)) return 0.0;
    const Factors f = factors(x, t);
    return f.scale * f.rest;
  }
  // the weight as a whole number (below 2^52), of a near logit and of any
  __device__ __forceinline__ u64 near_mass(float x, double t) const {
    const Factors f = factors(x, t);
    return (u64)__double_as_longlong(fma(f.scale, f.rest, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ u64 mass(float x) const {
    const double t = step(x);
    return near(t) ? near_mass(x, t) : 0;
  }
  // Every logit of bin b or above it is at least the first, every one of at least the second lies above bin b: a first look
  // in float, with a step's margin for what `step` rounds.
  __device__ __forceinline__ float floor_of(int b) const {
    return nextafterf((float)((double)M - (8.0 * (b + 1) + 1.0) / rate), -INFINITY);
  }
  __device__ __forceinline__ float ceiling_of(int b) const {
    return nextafterf((float)((double)M - (8.0 * b - 1.0) / rate), INFINITY);
  }
};

template <bool BF>
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row, const double* table, int part = 0, int parts = 1) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES;
  Row r;
  r.base = static_cast<const char*>(a.logits) + (size_t)row * a.stride * ES;
  r.table = table;
  r.V = a.V;
  const int at = (int)((reinterpret_cast<uintptr_t>(r.base) & 15) / ES);
  r.head = at ? min(VEC - at, a.V) : 0;
  const int pieces = (a.V - r.head) / VEC, each = (pieces + parts - 1) / parts;
  r.p0 = min(part * each, pieces);
  r.p1 = min(r.p0 + each, pieces);
  r.edges = part == 0;
  r.drop = BF ? 16 : 0;
  return r;
}
template <bool BF>
__device__ __forceinline__ float logit(const Row& r, int id) {
  return BF ? bf2f(reinterpret_cast<const bf16_t*>(r.base)[id]) : reinterpret_cast<const float*>(r.base)[id];
}

template <bool BF>
__device__ __forceinline__ void unpack(const uint4& w, float (&x)[BF ? 8 : 4]) {
  const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < (BF ? 8 : 4); ++e)
    x[e] = BF ? __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16) : __uint_as_float(v[e & 3]);
}

// piece(x, id0) for the aligned 16 bytes of logits x[0 .. VEC) of ids id0 .., U loads of a thread in flight (past the last
// one: NaN, which every caller passes over), and one(x, id) for the row's few elements before and behind them.
template <bool BF, int U, class P, class O>
__device__ __forceinline__ void each_piece(const Row& r, P piece, O one) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES;
  const int tail = r.head + (r.V - r.head) / VEC * VEC;
  const int edge = (int)threadIdx.x < r.head ? (int)threadIdx.x : tail + (int)threadIdx.x - r.head;
  if (r.edges && edge < r.V && (int)threadIdx.x < 2 * VEC) one(logit<BF>(r, edge), edge);
  const uint4* src = reinterpret_cast<const uint4*>(r.base + (size_t)r.head * ES);
  auto take = [&](const uint4& w, int p) {
    float x[VEC];
    unpack<BF>(w, x);
    piece(x, r.head + p * VEC);
  };
#pragma unroll 1
  for (int p = r.p0 + (int)threadIdx.x; p < r.p1; p += kSampleThreads * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = make_uint4(~0u, ~0u, ~0u, ~0u);
      if (p + u * kSampleThreads < r.p1) w[u] = src[p + u * kSampleThreads];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) take(w[u], p + u * kSampleThreads);
  }
}
template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {  // NaN aside
  float m = x[0];
#pragma unroll
  for (int e = 1; e < N; ++e) m = fmaxf(m, x[e]);
  return m;
}
template <bool BF, class F>
__device__ __forceinline__ void each_logit(const Row& r, F f) {
  each_piece<BF, 1>(
      r,
      [&](const auto& x, int id0) {
#pragma unroll
        for (int e = 0; e < (BF ? 8 : 4); ++e) f(x[e], id0 + e);
      },
      f);
}
// f(id) for the elements of [lo, hi), taken to be few: what stands in the loop over the row is short, f outside of it and
// once (a kernel's instructions come from memory every time it starts, some 64 bytes in 0.1 us). `above` counts those from hi
// on, each wave's in its lane 0.
template <bool BF, class F>
__device__ __forceinline__ void each_between(const Row& r, float lo, float hi, uint32_t& above, F f) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES, U = 4;
  const int tid = threadIdx.x, tail = r.head + (r.V - r.head) / VEC * VEC;
  const uint4* src = reinterpret_cast<const uint4*>(r.base + (size_t)r.head * ES);
  uint32_t from_hi = 0;
#pragma unroll 1
  for (int p = r.edges ? r.p0 - kSampleThreads * U : r.p0; p < r.p0 || p < r.p1; p += kSampleThreads * U) {
    uint32_t hits = 0;  // bit u * VEC + e: element e of the thread's piece u
    int id0;
    auto look = [&](float x, int bit) {
      from_hi += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x >= hi));
      hits |= x >= lo && x < hi ? 1u << bit : 0u;
    };
    if (p < r.p0) {  // the elements before and behind the pieces
      id0 = tid < r.head ? tid : tail + tid - r.head;
      look(id0 < r.V && tid < 2 * VEC ? logit<BF>(r, id0) : __uint_as_float(~0u), 0);
    } else {
      id0 = r.head + (p + tid) * VEC;
      uint4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u] = make_uint4(~0u, ~0u, ~0u, ~0u);  // NaN
        if (p + tid + u * kSampleThreads < r.p1) w[u] = src[p + tid + u * kSampleThreads];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[VEC];
        unpack<BF>(w[u], x);
        if (!__any(largest(x) >= lo)) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) look(x[e], u * VEC + e);
      }
    }
#pragma unroll 1
    for (; hits; hits &= hits - 1) {
      const int bit = __builtin_ctz(hits);
      f(id0 + bit / VEC * (kSampleThreads * VEC) + bit % VEC);
    }
  }
  if ((tid & 63) == 0) above += from_hi;
}
// f(x, id) for the logits of at least lo, below +inf
template <bool BF, class F>
__device__ __forceinline__ void each_from(const Row& r, float lo, F f) {
  uint32_t above = 0;
  each_between<BF>(r, lo, INFINITY, above, [&](int id) { f(logit<BF>(r, id), id); });
}

// Element at which a running value passes a target.
struct Found {
  u64 incl, weight;  // sum up to and with it, its own
  int count, id;     // elements up to and with it, its id
};

// The part of LDS that both kernels have.
struct ListShared {
  double table[kTable];
  u64 list[kList];
  u64 sum[kList];
  uint32_t start[kList + 1];
  u64 red64[kWaves];
  uint32_t red32[kWaves];
  float red_x[kWaves];
  uint32_t above;
  int n, n_ids, found;
};
struct FullShared : ListShared {
  u64 mass[kBins + 1];
  uint32_t cnt[kBins + 1];
  uint32_t lo, hi, m_cnt, dead;
  u64 m_mass;
};

// The row's settings and what follows from them.
struct How {
  float T, pf, uf, m_log;
  int k;
  bool by_p, by_m;
  double m_least;
  __device__ __forceinline__ How(const SampleArgs& a, int row) {
    T = a.temperature ? a.temperature[row] : 1.f;
    k = a.top_k ? a.top_k[row] : 0;
    pf = a.top_p ? a.top_p[row] : 1.f;
    uf = a.uniform[row];
    const float mf = a.min_p ? a.min_p[row] : 0.f;
    by_p = pf < 1.f;
    by_m = mf > 0.f;
    m_least = ldexp(mf < 1.f ? (double)mf : 1.0, a.shift);
    m_log = log2f(fminf(mf, 1.f));
  }
  // every logit that min-p keeps is at least this: two steps' margin
  __device__ __forceinline__ float m_floor(const Row& r) const {
    return nextafterf((float)((double)r.M + ((double)m_log * kTable - 2.0) / r.rate), -INFINITY);
  }
  // targets for the running sum: the prefix ends, the draw lies at the first element whose sum is above them
  __device__ __forceinline__ u64 p_target(u64 total) const {  // elements whose sum before them is below p * total
    const double y = ceil((double)pf * (double)total);
    const u64 t = y >= 1.0 ? (u64)y - 1 : 0;
    return t < total ? t : total - 1;
  }
  __device__ __forceinline__ u64 u_target(u64 total) const {
    const double y = floor((uf > 0.f ? (double)uf : 0.0) * (double)total);
    const u64 t = y < (double)total ? (u64)y : total - 1;
    return t < total ? t : total - 1;
  }
};
__device__ __forceinline__ void answer(const SampleArgs& a, int row, int token, double conf, int kept) {
  if (threadIdx.x != 0) return;
  a.token[row] = token;
  if (a.conf) a.conf[row] = (float)conf;
  if (a.kept) a.kept[row] = kept;
}
__device__ __forceinline__ void fill_table(double* table, int shift) {
  const int i = threadIdx.x;
  if (i >= kTable) return;
  const u64 bits = (u64)__double_as_longlong(ldexp(exp2(i * (1.0 / kTable)), shift - kTop / kTable));
  table[i] = __longlong_as_double((long long)(bits - ((u64)i << 44)));
}

// Exclusive prefix sums of 2048 counts or sums in place, the total behind the last; `red`: a word a wave. All threads; ends
// with a barrier.
template <class T>
__device__ __forceinline__ void scan_bins(T* v, T* red) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  static_assert(kBins == 2 * kSampleThreads, "two bins a thread");
  const T v0 = v[2 * tid], v1 = v[2 * tid + 1];
  T s = v0 + v1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) red[wid] = s;
  __syncthreads();
  for (int w = 0; w < wid; ++w) s += red[w];
  v[2 * tid] = s - v0 - v1;
  v[2 * tid + 1] = s - v1;
  if (tid == kSampleThreads - 1) v[kBins] = s;
  __syncthreads();
}

// The bin in which the running value passes t, below the total of the scanned ones: every thread looks at its two. All
// threads; ends with a barrier.
template <class T>
__device__ __forceinline__ int bin_of(const T* excl, T t, ListShared& sh) {
  const int i = 2 * threadIdx.x;
  if (excl[i] <= t && t < excl[i + 1]) sh.found = i;
  if (excl[i + 1] <= t && t < excl[i + 2]) sh.found = i + 1;
  __syncthreads();
  const int b = sh.found;
  __syncthreads();
  return b;
}

// The elements x of [lo, hi) for which side(x) is 0 into the list as (~key, id), if those of [lo, hi) fit it; sh.n counts
// them, sh.above those for which side is negative and those from hi on. All threads.
template <bool BF, class P>
__device__ __forceinline__ bool collect(const Row& r, float lo, float hi, ListShared& sh, P side) {
  const int tid = threadIdx.x;
  uint32_t* ids = sh.start;
  __syncthreads();
  if (tid == 0) sh.n = sh.n_ids = 0, sh.above = 0;
  __syncthreads();
  uint32_t above = 0;
  each_between<BF>(r, lo, hi, above, [&](int id) {
    const int at = atomicAdd(&sh.n_ids, 1);
    if (at < kList) ids[at] = (uint32_t)id;
  });
  if (above) atomicAdd(&sh.above, above);
  __syncthreads();
  const int n = sh.n_ids;
  if (n <= kList) {
#pragma unroll 1
    for (int i = tid; i < n; i += kSampleThreads) {
      const float x = logit<BF>(r, (int)ids[i]);
      const int at = side(x);
      if (at < 0) atomicAdd(&sh.above, 1u);
      if (at == 0) sh.list[atomicAdd(&sh.n, 1)] = ((u64)~order_key(x) << 32) | ids[i];
    }
  }
  __syncthreads();
  return n <= kList;
}
// those of bins from .. b
template <bool BF>
__device__ __forceinline__ bool collect_bins(const Row& r, int from, int b, ListShared& sh) {
  return collect<BF>(r, r.floor_of(b), from > 0 ? r.ceiling_of(from) : INFINITY, sh, [&](float x) {
    const int at = r.bin(x);
    return at < from ? -1 : at > b;
  });
}

// The sh.n collected pairs in order, and the running sums of their weights from `above`. All threads.
// More than 128 are first put into up to 2048 groups by value and id, as if those lay evenly between the extremes (as they
// do in one bin, or among equal values); the elements of a group are then ranked one against the other. (Sorted by a network,
// 1000 took 20 us and more: 55 steps that wait.)
__device__ __forceinline__ void order_list(const Row& r, u64 above, ListShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = sh.n;
  u64 v[2];
  int at[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 2; ++e) v[e] = e * kSampleThreads + tid < n ? sh.list[e * kSampleThreads + tid] : ~0ull;
  const bool grouped = n > 128;
  if (grouped) {
    uint32_t lo = min((uint32_t)(v[0] >> 32), (uint32_t)(v[1] >> 32));
    uint32_t hi = max(tid < n ? (uint32_t)(v[0] >> 32) : 0u, kSampleThreads + tid < n ? (uint32_t)(v[1] >> 32) : 0u);
    for (int o = 32; o >= 1; o >>= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64)), hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    if (lane == 0) sh.red32[wid] = lo, sh.red64[wid] = hi;
    for (int i = tid; i <= kList; i += kSampleThreads) sh.start[i] = 0;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) lo = min(lo, sh.red32[w]), hi = max(hi, (uint32_t)sh.red64[w]);
    const int drop = r.drop;  // bits that all keys have alike
    const double ids = (double)r.V, scale = (kList - 0.5) / ((double)((hi - lo) >> drop) * ids + ids);
    int slot[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e * kSampleThreads + tid < n) {
        at[e] = (int)(fma((double)(((uint32_t)(v[e] >> 32) - lo) >> drop), ids, (double)(uint32_t)v[e]) * scale);
        slot[e] = (int)atomicAdd(&sh.start[at[e]], 1u);
      }
    __syncthreads();
    scan_bins(sh.start, sh.red32);
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (e * kSampleThreads + tid < n) sh.sum[sh.start[at[e]] + slot[e]] = v[e];
  }
  __syncthreads();
  const u64* from = grouped ? sh.sum : sh.list;
  int rank[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (e * kSampleThreads + tid >= n) continue;
    int i = grouped ? (int)sh.start[at[e]] : 0;
    const int end = grouped ? (int)sh.start[at[e] + 1] : n;
    rank[e] = i;
    for (; i < end; ++i) rank[e] += from[i] < v[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (e * kSampleThreads + tid < n) sh.list[rank[e]] = v[e];
  __syncthreads();
  static_assert(kList == 2 * kSampleThreads, "two elements a thread");
  u64 w0 = 0, w1 = 0;
  if (2 * tid < n) w0 = r.mass(key_value(~(uint32_t)(sh.list[2 * tid] >> 32)));
  if (2 * tid + 1 < n) w1 = r.mass(key_value(~(uint32_t)(sh.list[2 * tid + 1] >> 32)));
  u64 s = w0 + w1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 u = __shfl_up(s, o, 64);
    if (lane >= o) s += u;
  }
  if (lane == 63) sh.red64[wid] = s;
  __syncthreads();
  s += above;
  for (int w = 0; w < wid; ++w) s += sh.red64[w];
  if (2 * tid < n) sh.sum[2 * tid] = s - w1;
  if (2 * tid + 1 < n) sh.sum[2 * tid + 1] = s;
  __syncthreads();
}

// In the ordered list, whose elements follow `above` (sum) and `before` (count): by count (0-based index) or by a sum below
// the list's last. All threads.
__device__ __forceinline__ Found in_list(bool by_count, u64 t, u64 above, uint32_t before, ListShared& sh) {
  if (by_count) {
    if (threadIdx.x == 0) sh.found = (int)((uint32_t)t - before);
  } else {
#pragma unroll
    for (int i = threadIdx.x; i < kList; i += kSampleThreads)
      if (i < sh.n && sh.sum[i] > t && (i == 0 || sh.sum[i - 1] <= t)) sh.found = i;
  }
  __syncthreads();
  const int i = sh.found;
  __syncthreads();
  const u64 prev = i > 0 ? sh.sum[i - 1] : above;
  return {sh.sum[i], sh.sum[i] - prev, (int)before + i + 1, (int)(uint32_t)sh.list[i]};
}

// Id of the j-th of the elements equal to v, in order of ids: the pieces are cut into one range per wave, the waves count, and
// the range that holds it is cut again. `red`: a word a wave. All threads, of which each gets it.
template <bool BF>
__device__ __forceinline__ int equal_id(const Row& r, float v, u64 j, uint32_t* red) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES, U = 4;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const uint4* src = reinterpret_cast<const uint4*>(r.base + (size_t)r.head * ES);
  const int pieces = (r.V - r.head) / VEC;
  auto count = [&](const uint4& w) {
    float x[VEC];
    unpack<BF>(w, x);
    int n = 0;
#pragma unroll
    for (int e = 0; e < VEC; ++e) n += x[e] == v;
    return n;
  };
  auto edge = [&](int first, int n) {  // of the n elements from `first` on, every wave alike; j counts on where it is not there
    u64 m = __builtin_amdgcn_ballot_w64(lane < n && logit<BF>(r, lane < n ? first + lane : 0) == v);
    for (; m && j; m &= m - 1) --j;
    return m ? first + (int)__builtin_ctzll(m) : -1;
  };
  const int before = edge(0, r.head);
  if (before >= 0) return before;
  int lo = 0, len = pieces;
#pragma unroll 1
  while (len > 64) {
    const int part = (len + kWaves - 1) / kWaves, to = min(lo + (wid + 1) * part, lo + len);
    int n = 0;
#pragma unroll 1
    for (int i = lo + wid * part + lane; i < to; i += 64 * U) {
      uint4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u] = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (i + 64 * u < to) w[u] = src[i + 64 * u];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) n += count(w[u]);
    }
    for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
    __syncthreads();
    if (lane == 0) red[wid] = (uint32_t)n;
    __syncthreads();
    int w = 0;
    while (w < kWaves && j >= red[w]) j -= red[w++];
    const int end = lo + len;
    lo = min(lo + w * part, end);
    len = w < kWaves ? min(part, end - lo) : 0;  // in none of them: behind the pieces
  }
  // a piece a lane, every wave alike
  const uint4 last = lane < len ? src[lo + lane] : make_uint4(~0u, ~0u, ~0u, ~0u);
  const int own = count(last);
  int upto = own;
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(upto, o, 64);
    if (lane >= o) upto += u;
  }
  const u64 past = __builtin_amdgcn_ballot_w64((u64)upto > j);
  if (!past) {
    j -= (u64)__shfl(upto, 63, 64);
    return edge(r.head + pieces * VEC, r.V - r.head - pieces * VEC);
  }
  const int at = (int)__builtin_ctzll(past);
  float x[VEC];
  unpack<BF>(last, x);
  int left = (int)j - (upto - own), id = -1;
#pragma unroll
  for (int e = 0; e < VEC; ++e)
    if (x[e] == v && left-- == 0) id = r.head + (lo + lane) * VEC + e;
  return __shfl(id, at, 64);
}

// What a row's kernels leave for the next ones, in the workspace: of rows that are not shared their maximum, NaN where the row
// is answered, for the next kernel (n floats) and the one after it (n more); of shared rows all this.
struct RowState {
  float M;             // as above
  uint32_t n_list;     // elements that reach top-k's bound, collected if they fit; ~0: no bound was set
  uint32_t m_cnt;      // elements that min-p keeps
  uint32_t dead;       // elements that are -inf or NaN
  u64 m_mass;          // the sum of those that min-p keeps
};
// A row that several workgroups share: its parts' maxima, 1024 maxima of groups that cover it, the collected elements, the
// histogram.
struct SplitRow {
  float part_max[kMaxParts];
  int part_id[kMaxParts];
  float group_max[kSampleThreads];
  u64 list[kList];
  u64 mass[kBins];
  uint32_t cnt[kBins];
};

// The open rows of 1024 go to the first of their 1024 workgroups, so that they spread over the XCDs and CUs whichever rows
// they are (512 rows, 213 of them open: 74 us with a row to its own workgroup, 45 so). The row of this one, or -1. All threads.
__device__ __forceinline__ int open_row(const float* M, int n, uint32_t* red, int* found) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, i = (int)(blockIdx.x & ~(kSampleThreads - 1u)) + (int)threadIdx.x;
  const bool open = i < n && M[i] > -INFINITY;
  const u64 b = __builtin_amdgcn_ballot_w64(open);
  if (lane == 0) red[wid] = (uint32_t)__builtin_popcountll(b);
  if (threadIdx.x == 0) *found = -1;
  __syncthreads();
  uint32_t before = (uint32_t)__builtin_popcountll(b & ((1ull << lane) - 1));
  for (int w = 0; w < wid; ++w) before += red[w];
  if (open && before == (blockIdx.x & (kSampleThreads - 1u))) *found = i;
  __syncthreads();
  return *found;
}

// Rows whose logits are +inf somewhere: those ids share the weight alike, all others have none.
template <bool BF>
__device__ __forceinline__ void infinite_row(const SampleArgs& a, int row, const Row& r, const How& how, ListShared& sh) {
  __syncthreads();
  if (threadIdx.x == 0) sh.red32[0] = sh.red32[1] = 0;
  __syncthreads();
  uint32_t top = 0, alive = 0;
  each_logit<BF>(r, [&](float x, int) {
    top += x == INFINITY;
    alive += x > -INFINITY;
  });
  if (alive) atomicAdd(&sh.red32[0], top), atomicAdd(&sh.red32[1], alive);
  __syncthreads();
  top = sh.red32[0];
  alive = sh.red32[1];
  uint32_t count = how.k > 0 ? min((uint32_t)how.k, alive) : alive;
  const uint32_t in_k = min(count, top);
  if (how.by_p) count = min(count, (uint32_t)how.p_target(in_k) + 1);  // weight 1 each: a sum is a count
  if (how.by_m) count = min(count, top);
  const uint32_t total = min(count, top);
  const int id = equal_id<BF>(r, INFINITY, how.u_target(total), sh.red32);
  answer(a, row, id, 1.0 / (double)total, (int)count);
}

// How many of the ordered list's first `count` elements min-p keeps: weights fall along it. All threads.
__device__ __forceinline__ int in_list_by_weight(const Row& r, const How& how, int count, const ListShared& sh) {
  int kept = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < count; i0 += kSampleThreads) {
    const int i = i0 + (int)threadIdx.x;
    kept += __syncthreads_count(i < count && r.weight(key_value(~(uint32_t)(sh.list[i] >> 32))) >= how.m_least);
  }
  return kept;
}

// The answer from the list of all elements that reach some bound, at least k of them. All threads.
__device__ __forceinline__ void answer_from_list(const SampleArgs& a, int row, const Row& r, const How& how, ListShared& sh) {
  order_list(r, 0, sh);
  int count = how.k;
  if (how.by_p) count = min(count, in_list(false, how.p_target(sh.sum[count - 1]), 0, 0, sh).count);
  if (how.by_m) count = in_list_by_weight(r, how, count, sh);
  const u64 total = sh.sum[count - 1];
  const Found f = in_list(false, how.u_target(total), 0, 0, sh);
  answer(a, row, f.id, (double)f.weight / (double)total, count);
}

// A lower bound for the k-th largest element, k up to 512: with 1024 groups that cover the row, the k-th largest of their
// maxima is one, and not many more elements reach it (about 710 for 512 of 152064 in no order). To within 1 / 1000 of the
// maxima's range, from a histogram of them. `own`: the thread's group's maximum, `least`: the smallest above -inf. False
// where fewer than k groups have any element. All threads; cnt is all zeros.
__device__ __forceinline__ bool bound_of(const Row& r, int k, float own, float least, uint32_t* cnt, ListShared& sh, float& lo) {
  const float step = fminf(2047.f / (r.M - least), 1e30f);
  auto bin = [&](float x) { return (int)fminf((r.M - x) * step, 2047.f); };  // does not decrease while x falls
  if (own > -INFINITY) atomicAdd(&cnt[bin(own)], 1u);
  __syncthreads();
  scan_bins(cnt, sh.red32);
  if (cnt[kBins] < (uint32_t)k) return false;
  // the k-th lies in this bin, within (b + 1) / step of M but for the rounding of `bin`; none lies below the least
  lo = fmaxf(least, r.M - (float)(bin_of(cnt, (uint32_t)(k - 1), sh) + 2) / step);
  return true;
}
__device__ __forceinline__ bool takes_bound(const How& how) { return how.k > 0 && how.k <= kSampleThreads / 2; }

__device__ __forceinline__ void lower_id(float x, int id, float& best, int& best_id) {  // the larger, then the lower id
  if (x > best || (x == best && id < best_id)) best = x, best_id = id;
}
// The largest logit of the workgroup's pieces and its lowest id: the thread's own.
template <bool BF>
__device__ __forceinline__ void thread_max(const Row& r, float& best, int& best_id) {
  best = -INFINITY;
  best_id = INT_MAX;
  each_piece<BF, 4>(
      r,
      [&](const auto& x, int id0) {
        if (!(largest(x) >= best)) return;  // an equal one may have a lower id than an edge element's
#pragma unroll
        for (int e = 0; e < (BF ? 8 : 4); ++e) lower_id(x[e], id0 + e, best, best_id);
      },
      [&](float x, int id) { lower_id(x, id, best, best_id); });
  if (best == -INFINITY) best_id = INT_MAX;
}

template <bool BF>
__global__ void __launch_bounds__(kSampleThreads, 8) sample_top_kernel(SampleArgs a) {
  __shared__ ListShared sh;
  __shared__ uint32_t cnt[kBins + 1];
  __shared__ int red_id[kWaves];
  __shared__ float red_least[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, row = blockIdx.x;
  Row r = row_of<BF>(a, row, sh.table);
  float* left = static_cast<float*>(a.ws) + row;
  float best;
  int best_id;
  thread_max<BF>(r, best, best_id);
  const float own = best;
  float least = own > -INFINITY ? own : INFINITY;
  for (int o = 32; o >= 1; o >>= 1) {
    const float x = __shfl_xor(best, o, 64);
    const int id = __shfl_xor(best_id, o, 64);
    lower_id(x, id, best, best_id);
    least = fminf(least, __shfl_xor(least, o, 64));
  }
  if (lane == 0) sh.red_x[wid] = best, red_id[wid] = best_id, red_least[wid] = least;
  fill_table(sh.table, a.shift);
  for (int i = tid; i <= kBins; i += kSampleThreads) cnt[i] = 0;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) lower_id(sh.red_x[w], red_id[w], best, best_id), least = fminf(least, red_least[w]);
  const How how(a, row);
  if (tid == 0) left[0] = left[a.n] = __uint_as_float(0x7FC00000u);
  if (best == -INFINITY) return answer(a, row, -1, 0.0, 0);  // nothing but -inf and NaN
  if (!(how.T > 0.f) || how.k == 1) return answer(a, row, best_id, 1.0, 1);
  if (best == INFINITY) return infinite_row<BF>(a, row, r, how, sh);
  r.set(best, how.T);
  float lo;
  if (takes_bound(how) && bound_of(r, how.k, own, least, cnt, sh, lo) && collect<BF>(r, lo, INFINITY, sh, [](float) { return 0; }))
    return answer_from_list(a, row, r, how, sh);
  if (tid == 0) left[0] = left[a.n] = best;
}

// Rows that `parts` workgroups share (few rows: one CU reads 30 GB/s, a row of 126464 float32 in 16 us). First the parts'
// maxima and those of 1024 groups of threads, and zeros where the next kernel counts.
template <bool BF>
__global__ void __launch_bounds__(kSampleThreads, 8) sample_part_kernel(SampleArgs a, int parts) {
  __shared__ float red_x[kWaves];
  __shared__ int red_id[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, row = blockIdx.x / parts, part = blockIdx.x % parts;
  RowState* state = static_cast<RowState*>(a.ws) + row;
  SplitRow* split = reinterpret_cast<SplitRow*>(static_cast<RowState*>(a.ws) + a.n) + row;
  for (int i = part * kSampleThreads + tid; i < kBins; i += parts * kSampleThreads) split->cnt[i] = 0, split->mass[i] = 0;
  if (part == 0 && tid == 0) *state = RowState{};
  const Row r = row_of<BF>(a, row, nullptr, part, parts);
  float best;
  int best_id;
  thread_max<BF>(r, best, best_id);
  float group = best;  // of `parts` neighbouring threads (a power of two)
  for (int o = 1; o < parts; o <<= 1) group = fmaxf(group, __shfl_xor(group, o, 64));
  if (tid % parts == 0) split->group_max[(part * kSampleThreads + tid) / parts] = group;
  for (int o = 32; o >= 1; o >>= 1) {
    const float x = __shfl_xor(best, o, 64);
    const int id = __shfl_xor(best_id, o, 64);
    lower_id(x, id, best, best_id);
  }
  if (lane == 0) red_x[wid] = best, red_id[wid] = best_id;
  __syncthreads();
  if (tid != 0) return;
  for (int w = 1; w < kWaves; ++w) lower_id(red_x[w], red_id[w], best, best_id);
  split->part_max[part] = best;
  split->part_id[part] = best_id;
}

// The question inside one bin with more elements than the list holds. All threads; the list is overwritten.
template <bool BF>
__device__ __forceinline__ Found in_large_bin(const Row& r, int b, bool by_count, u64 t, u64 above, FullShared& sh) {
  const int tid = threadIdx.x;
  constexpr int PARTS = 1024;
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.sum);
  u64* mass = sh.list;
  static_assert(PARTS <= kList, "counts and sums of the parts lie in the list's memory");
  // the values that are left, in order_key's terms
  uint32_t before = 0;  // elements above them
  uint32_t klo = order_key(fmaxf(r.floor_of(b), -3.4028234663852886e38f)), khi = order_key(r.M);
#pragma unroll 1
  for (bool whole = true;; whole = false) {  // the whole bin at first
    // the range that they really take
    __syncthreads();
    if (tid == 0) sh.lo = 0xFFFFFFFFu, sh.hi = 0, sh.n = 0, sh.above = 0;
    __syncthreads();
    uint32_t lo = 0xFFFFFFFFu, hi = 0, n = 0, higher = 0;
    each_from<BF>(r, key_value(klo), [&](float x, int) {
      const uint32_t k = order_key(x);
      const int at = whole ? r.bin(x) : k <= khi ? b : b - 1;
      if (at == b) lo = min(lo, k), hi = max(hi, k), ++n;
      higher += at < b;
    });
    if (whole && higher) atomicAdd(&sh.above, higher);
    if (n) {
      atomicMin(&sh.lo, lo);
      atomicMax(&sh.hi, hi);
      atomicAdd(&sh.n, (int)n);
    }
    __syncthreads();
    klo = sh.lo;
    khi = sh.hi;
    const int left = sh.n;
    if (whole) before = sh.above;
    __syncthreads();
    if (klo == khi) {  // equal values: element j of them, by arithmetic; its id by counting in order
      const u64 w = r.mass(key_value(klo));
      const u64 j = by_count ? (uint32_t)t - before : w ? (t - above) / w : 0;
      const int id = equal_id<BF>(r, key_value(klo), j, sh.red32);
      return {above + (j + 1) * w, w, (int)(before + (uint32_t)j + 1), id};
    }
    if (left <= kList) {
      collect<BF>(r, key_value(klo), key_value(khi + 1), sh, [](float) { return 0; });
      order_list(r, above, sh);
      return in_list(by_count, t, above, before, sh);
    }
    // split [klo, khi] into ranges of keys, from the top
    const u64 width = (u64)(khi - klo) + 1;
    auto part = [&](uint32_t k) { return (int)((u64)(khi - k) * PARTS / width); };
    for (int i = tid; i < PARTS; i += kSampleThreads) cnt[i] = 0, mass[i] = 0;
    __syncthreads();
    each_from<BF>(r, key_value(klo), [&](float x, int) {
      const uint32_t k = order_key(x);
      if (k > khi) return;
      atomicAdd(&cnt[part(k)], 1u);
      atomicAdd(&mass[part(k)], r.mass(x));
    });
    __syncthreads();
    // running sums by one thread: this path is for rows of many nearly equal values
    if (tid == 0) {
      uint32_t c = before;
      u64 m = above;
      int i = 0;
      for (; i < PARTS - 1; ++i) {
        if (by_count ? c + cnt[i] > (uint32_t)t : m + mass[i] > t) break;
        c += cnt[i];
        m += mass[i];
      }
      sh.red32[0] = c;
      sh.red64[0] = m;
      sh.red32[1] = (uint32_t)i;
    }
    __syncthreads();
    before = sh.red32[0];
    above = sh.red64[0];
    const u64 i = sh.red32[1];
    __syncthreads();
    // keys k with (khi - k) * PARTS / width == i
    const u64 first = (i * width + PARTS - 1) / PARTS, last = ((i + 1) * width + PARTS - 1) / PARTS - 1;
    const uint32_t top = khi;
    khi = top - (uint32_t)first;
    klo = top - (uint32_t)last;
  }
}

// The histogram over the workgroup's pieces, all zeros before: the bins' counts into sh.cnt where top-k asks by count, their
// sums into sh.mass. An atomic addition in LDS costs about as much as the arithmetic of an element, so the passes do not
// take both at once, and the far elements (most of a row at a low temperature) take none. All threads; ends with a barrier.
template <bool BF>
__device__ __forceinline__ void count_bins(const Row& r, FullShared& sh) {
  uint32_t far = 0;
  each_logit<BF>(r, [&](float x, int) {
    const double t = r.step(x);
    if (Row::near(t)) atomicAdd(&sh.cnt[Row::place(t)], 1u);
    else far += x > -INFINITY;
  });
  if (far) atomicAdd(&sh.cnt[kFar], far);
  __syncthreads();
}
// Also counts the dead elements, and count and sum of those that min-p keeps (by a pass of their own: they are few).
template <bool BF>
__device__ __forceinline__ void sum_bins(const Row& r, const How& how, FullShared& sh) {
  uint32_t dead = 0;
  each_logit<BF>(r, [&](float x, int) {
    const double t = r.step(x);
    if (Row::near(t)) atomicAdd(&sh.mass[Row::place(t)], r.near_mass(x, t));
    else dead += !(x > -INFINITY);
  });
  if (dead) atomicAdd(&sh.dead, dead);
  if (how.by_m) {
    u64 m_mass = 0;
    uint32_t m_cnt = 0;
    each_from<BF>(r, how.m_floor(r), [&](float x, int) {
      if (r.weight(x) >= how.m_least) ++m_cnt, m_mass += r.mass(x);
    });
    if (m_cnt) atomicAdd(&sh.m_cnt, m_cnt), atomicAdd(&sh.m_mass, m_mass);
  }
  __syncthreads();
}
__device__ __forceinline__ void clear_histogram(FullShared& sh) {
  for (int i = threadIdx.x; i <= kBins; i += kSampleThreads) sh.cnt[i] = 0, sh.mass[i] = 0;
  if (threadIdx.x == 0) sh.m_mass = 0, sh.m_cnt = 0, sh.dead = 0;
}

// Second kernel of shared rows: the parts' elements that reach top-k's bound go to the row's list, or the parts' histograms
// to the row's.
template <bool BF>
__global__ void __launch_bounds__(kSampleThreads, 8) sample_gather_kernel(SampleArgs a, int parts) {
  __shared__ FullShared sh;
  __shared__ int base;
  const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x / parts, part = blockIdx.x % parts;
  RowState* state = static_cast<RowState*>(a.ws) + row;
  SplitRow* split = reinterpret_cast<SplitRow*>(static_cast<RowState*>(a.ws) + a.n) + row;
  Row r = row_of<BF>(a, row, sh.table, part, parts);
  const How how(a, row);
  float best = split->part_max[0];
  int best_id = split->part_id[0];
  for (int p = 1; p < parts; ++p) lower_id(split->part_max[p], split->part_id[p], best, best_id);
  const bool answered = best == -INFINITY || !(how.T > 0.f) || how.k == 1;
  if (answered || best == INFINITY) {
    if (part == 0) {
      if (tid == 0) state->M = answered ? __uint_as_float(0x7FC00000u) : best;
      if (best == -INFINITY) answer(a, row, -1, 0.0, 0);
      else if (answered) answer(a, row, best_id, 1.0, 1);
    }
    return;
  }
  if (part == 0 && tid == 0) state->M = best;
  r.set(best, how.T);
  fill_table(sh.table, a.shift);
  clear_histogram(sh);
  const float own = split->group_max[tid];
  float least = own > -INFINITY ? own : INFINITY;
  for (int o = 32; o >= 1; o >>= 1) least = fminf(least, __shfl_xor(least, o, 64));
  if (lane == 0) sh.red_x[tid >> 6] = least;
  __syncthreads();
  if (takes_bound(how)) {
    for (int w = 0; w < kWaves; ++w) least = fminf(least, sh.red_x[w]);
    float lo;
    if (bound_of(r, how.k, own, least, sh.cnt, sh, lo)) {
      const bool fits = collect<BF>(r, lo, INFINITY, sh, [](float) { return 0; });
      if (tid == 0) base = (int)atomicAdd(&state->n_list, (uint32_t)(fits ? sh.n : kList + 1));
      __syncthreads();
      if (fits && base + sh.n <= kList)
        for (int i = tid; i < sh.n; i += kSampleThreads) split->list[base + i] = sh.list[i];
      return;
    }
    if (part == 0 && tid == 0) state->n_list = ~0u;  // the same in every part: none of them adds to it
    return;
  }
  if (how.k > 0) count_bins<BF>(r, sh);
  sum_bins<BF>(r, how, sh);
  for (int i = tid; i <= kFar; i += kSampleThreads) {
    if (sh.cnt[i]) atomicAdd(&split->cnt[i], sh.cnt[i]);
    if (sh.mass[i]) atomicAdd(&split->mass[i], sh.mass[i]);
  }
  if (tid != 0) return;
  if (sh.m_cnt) atomicAdd(&state->m_cnt, sh.m_cnt), atomicAdd(&state->m_mass, sh.m_mass);
  if (sh.dead) atomicAdd(&state->dead, sh.dead);
}

// bfloat16 rows that are not answered yet: their values are few enough for a count of each, between the maximum and 47
// factors of 2 below it, so that no element needs an exponential or a place in a list: 42 us a row of 152064 (one row a CU), of
// which the two passes over it take 12 and 13, near a CU's share of the memory's rate. Slabs of 64 values go round the waves. Rows
// whose values reach further (the biased exponents of the first and the last would have to sum to more than 290: magnitudes
// of 2^18 and more, of either sign) are left to the next kernel.
constexpr int kSlabs = 592, kValues = 64 * kSlabs;
static_assert(kSlabs % kWaves == 0 && kSlabs <= kSampleThreads, "a slab a thread in the sums");
struct ValueShared {
  alignas(16) uint32_t cnt[kValues];
  double table[kTable];
  u64 slab_mass[kSlabs];
  uint32_t slab_cnt[kSlabs];
  u64 red64[kWaves];
  uint32_t red32[kWaves];
  u64 m_mass, above;
  uint32_t m_cnt, dead, before;
  int owner;
};
__global__ void __launch_bounds__(kSampleThreads, 4) sample_values_kernel(SampleArgs a) {
  __shared__ ValueShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  float* left = static_cast<float*>(a.ws);
  const int row = open_row(left, a.n, sh.red32, &sh.owner);
  if (row < 0) return;
  const float M = left[row];
  Row r = row_of<true>(a, row, sh.table);
  const How how(a, row);
  r.set(M, how.T);
  // a value by its place: order_key has 16 bits of it
  const uint32_t top = order_key(M) >> 16;
  const uint32_t limit = top - (order_key(fmaxf(r.floor_of(kFar - 1), -3.4028234663852886e38f)) >> 16) + 1;
  if (limit > (uint32_t)kValues) return;
  auto value = [&](int i) { return key_value((top - (uint32_t)i) << 16 | ((top - (uint32_t)i) & 0x8000u ? 0u : 0xFFFFu)); };
  fill_table(sh.table, a.shift);
  if (tid == 0) sh.m_mass = 0, sh.m_cnt = 0, sh.dead = 0;
  if (tid < kSlabs) sh.slab_cnt[tid] = 0, sh.slab_mass[tid] = 0;
  for (uint32_t i = 4 * tid; i < limit; i += 4 * kSampleThreads) *reinterpret_cast<uint4*>(sh.cnt + i) = make_uint4(0, 0, 0, 0);
  __syncthreads();

  const uint32_t lowest = top - 0x80u;  // the place of the least finite value; -inf and NaN are past it, modulo 2^16
  uint32_t dead = 0;
  auto add = [&](uint32_t i) {
    if (i < limit) atomicAdd(&sh.cnt[i], 1u);
    else dead += i > lowest;
  };
  {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const u16x2 tops = {(unsigned short)top, (unsigned short)top}, flip = {0x8000, 0x8000};
    auto places = [&](uint32_t two) {
      const u16x2 w = __builtin_bit_cast(u16x2, two);
      const u16x2 sign = __builtin_bit_cast(u16x2, __builtin_bit_cast(s16x2, two) >> 15);
      return __builtin_bit_cast(uint32_t, (u16x2)(tops - (w ^ (sign | flip))));
    };
    constexpr int U = 4;
    const int tail = r.head + (r.V - r.head) / 8 * 8, edge = tid < r.head ? tid : tail + tid - r.head;
    if (edge < r.V && tid < 16) add(places(reinterpret_cast<const bf16_t*>(r.base)[edge]) & 0xFFFFu);
    const uint4* src = reinterpret_cast<const uint4*>(r.base + (size_t)r.head * 2);
#pragma unroll 1
    for (int p = tid; p < r.p1; p += kSampleThreads * U) {
      uint4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = src[min(p + u * kSampleThreads, r.p1 - 1)];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p + u * kSampleThreads >= r.p1) break;
        const uint32_t two[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t i = places(two[e]);
          add(i & 0xFFFFu);
          add(i >> 16);
        }
      }
    }
  }
  if (dead) atomicAdd(&sh.dead, dead);
  __syncthreads();
  if (tid == 0 && top >= 0x8000u && top - 0x7FFFu < limit) {  // -0 is +0
    sh.cnt[top - 0x8000u] += sh.cnt[top - 0x7FFFu];
    sh.cnt[top - 0x7FFFu] = 0;
  }
  __syncthreads();

  uint32_t m_cnt = 0;
  u64 m_mass = 0;
  constexpr int G = 8;  // slabs looked at together: most are empty
#pragma unroll 1
  for (int s0 = wid; s0 < kSlabs; s0 += G * kWaves) {
    uint32_t n[G], all = 0;
#pragma unroll
    for (int e = 0; e < G; ++e) {
      const int i = 64 * (s0 + e * kWaves) + lane;
      n[e] = i < (int)limit ? sh.cnt[i] : 0;
      all |= n[e];
    }
    if (!__any(all != 0)) continue;
#pragma unroll 1
    for (int slab = s0; slab < kSlabs && slab < s0 + G * kWaves; slab += kWaves) {
      const uint32_t c = n[0];
#pragma unroll
      for (int e = 0; e + 1 < G; ++e) n[e] = n[e + 1];
      if (c == 0) continue;
      const float x = value(64 * slab + lane);
      const u64 mass = c * r.mass(x);
      if (how.by_m && r.weight(x) >= how.m_least) m_cnt += c, m_mass += mass;
      atomicAdd(&sh.slab_cnt[slab], c);
      atomicAdd(&sh.slab_mass[slab], mass);
    }
  }
  if (m_cnt) atomicAdd(&sh.m_cnt, m_cnt), atomicAdd(&sh.m_mass, m_mass);
  __syncthreads();
  const uint32_t c = tid < kSlabs ? sh.slab_cnt[tid] : 0;
  const u64 mass = tid < kSlabs ? sh.slab_mass[tid] : 0;
  // sums up to the thread's slab
  uint32_t cs = c;
  u64 ms = mass;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(cs, o, 64);
    const u64 v = __shfl_up(ms, o, 64);
    if (lane >= o) cs += u, ms += v;
  }
  if (lane == 63) sh.red32[wid] = cs, sh.red64[wid] = ms;
  __syncthreads();
  cs -= c;
  ms -= mass;
  uint32_t near = 0;
  u64 total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wid) cs += sh.red32[w], ms += sh.red64[w];
    near += sh.red32[w];
    total += sh.red64[w];
  }
  uint32_t count = (uint32_t)r.V - sh.dead;
  u64 k_total = total;
  Found f{};
  u64 j = 0;  // which of the elements of the found value
#pragma unroll 1
  for (int q = 0; q < 3; ++q) {  // the border of top-k, that of top-p, the draw
    if (q == 0 ? how.k <= 0 || (uint32_t)how.k >= count : q == 1 && !how.by_p) continue;
    if (q == 0 && (uint32_t)how.k > near) {  // past every id with a weight: the sum is all there is
      count = (uint32_t)how.k;
      continue;
    }
    if (q == 2 && how.by_m && sh.m_cnt < count) count = sh.m_cnt, total = sh.m_mass;
    const u64 t = q == 0 ? (u64)(how.k - 1) : q == 1 ? how.p_target(k_total) : how.u_target(total);
    if (q == 0 ? cs <= t && t < cs + c : ms <= t && t < ms + mass) sh.owner = 64 * tid, sh.before = cs, sh.above = ms;
    __syncthreads();
    // that slab's values, one a lane, every wave alike
    const int i = sh.owner + lane;
    const uint32_t n = i < (int)limit ? sh.cnt[i] : 0;
    const u64 w = n ? r.mass(value(i)) : 0;
    uint32_t upto = n;
    u64 sum = n * w;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u = __shfl_up(upto, o, 64);
      const u64 v = __shfl_up(sum, o, 64);
      if (lane >= o) upto += u, sum += v;
    }
    upto += sh.before;
    sum += sh.above;
    const int at = (int)__builtin_ctzll(__builtin_amdgcn_ballot_w64(q == 0 ? upto > t : sum > t));
    const uint32_t before = (uint32_t)__shfl((int)(upto - n), at, 64);
    const u64 above = __shfl(sum - n * w, at, 64), weight = __shfl(w, at, 64);
    j = q == 0 ? t - before : (t - above) / weight;
    f = {above + (j + 1) * weight, weight, (int)(before + (uint32_t)j + 1), __shfl(i, at, 64)};
    __syncthreads();
    if (q == 0) count = (uint32_t)how.k, total = k_total = f.incl;
    if (q == 1 && (uint32_t)f.count < count) count = (uint32_t)f.count, total = f.incl;
  }
  const int id = equal_id<true>(r, value(f.id), j, sh.red32);
  answer(a, row, id, (double)f.weight / (double)total, (int)count);
  if (tid == 0) left[a.n + row] = __uint_as_float(0x7FC00000u);
}

// The rows that are not answered yet, one workgroup each; of shared rows the list or the histogram is there.
template <bool BF, bool SHARED>
__global__ void __launch_bounds__(kSampleThreads, 4) sample_full_kernel(SampleArgs a) {
  __shared__ FullShared sh;
  const int tid = threadIdx.x;
  const float* left = static_cast<const float*>(a.ws) + a.n;
  const int row = SHARED ? (int)blockIdx.x : open_row(left, a.n, sh.red32, &sh.found);
  if (row < 0) return;
  RowState state{};
  if (SHARED) state = static_cast<const RowState*>(a.ws)[row];
  else state.M = left[row];
  if (!(state.M > -INFINITY)) return;  // answered
  Row r = row_of<BF>(a, row, sh.table);
  const How how(a, row);
  fill_table(sh.table, a.shift);
  const SplitRow* split = reinterpret_cast<const SplitRow*>(static_cast<const RowState*>(a.ws) + a.n) + row;
  if (SHARED && takes_bound(how) && state.M < INFINITY && state.n_list <= kList) {  // the list is in the workspace
    r.set(state.M, how.T);
    for (int i = tid; i < (int)state.n_list; i += kSampleThreads) sh.list[i] = split->list[i];
    if (tid == 0) sh.n = (int)state.n_list;
    __syncthreads();
    return answer_from_list(a, row, r, how, sh);
  }
  clear_histogram(sh);
  __syncthreads();
  if (SHARED && state.M == INFINITY) return infinite_row<BF>(a, row, r, how, sh);
  r.set(state.M, how.T);
  const bool summed = SHARED && !takes_bound(how);  // the histogram is in the workspace
  if (summed) {
    for (int i = tid; i <= kFar; i += kSampleThreads) sh.cnt[i] = split->cnt[i], sh.mass[i] = split->mass[i];
    if (tid == 0) sh.m_cnt = state.m_cnt, sh.m_mass = state.m_mass, sh.dead = state.dead;
    __syncthreads();
  }
  if (how.k > 0) {
    if (!summed) count_bins<BF>(r, sh);
    scan_bins(sh.cnt, sh.red32);
  }

  // The bins' sums are there; the list holds all that top-k keeps (while it is asked for: all that it has to); a list of
  // several bins is worth asking for.
  bool sums = false, whole = false, several = true;
  int list_lo = 1, list_hi = 0;      // bins that the list holds
  uint32_t list_before = 0;          // elements above them
  uint32_t count = 0;
  u64 total = 0, k_total = 0;
  Found f;
#pragma unroll 1
  for (int q = 0; q < 3; ++q) {  // the border of top-k, that of top-p, the draw: one copy of the search
    int b = kFar;
    bool fresh = false;  // the list was collected just now
    if (q == 0) {
      if (how.k <= 0 || (uint32_t)how.k >= sh.cnt[kBins]) continue;
      b = bin_of(sh.cnt, (uint32_t)(how.k - 1), sh);
      whole = several && b < kFar && sh.cnt[b + 2] <= kList;  // all that `collect` looks at should fit
    }
    if (!whole && !sums) {
      if (!summed) sum_bins<BF>(r, how, sh);
      if (how.k <= 0) {
        // not counted: from the sums, whose weights all but agree in a bin. Only says what is collected.
        for (int i = tid; i < kFar; i += kSampleThreads)
          sh.cnt[i] = (uint32_t)((float)sh.mass[i] * exp2f((float)(i + 1) * (1 / 32.f) - (float)a.shift)) + (sh.mass[i] > 0);
        __syncthreads();
        scan_bins(sh.cnt, sh.red32);
      }
      scan_bins(sh.mass, sh.red64);
      sums = true;
      count = (uint32_t)r.V - sh.dead;
      total = k_total = sh.mass[kBins];
    }
    if (q == 0 && !whole && b == kFar) {  // past every id with a weight: the sum is all there is
      count = (uint32_t)how.k;
      continue;
    }
    if (q == 1 && !how.by_p) continue;
    if (q == 2 && how.by_m) {
      if (whole) count = (uint32_t)in_list_by_weight(r, how, (int)count, sh), total = sh.sum[count - 1];
      else if (sh.m_cnt < count) count = sh.m_cnt, total = sh.m_mass;
    }
    const u64 t = q == 0 ? (u64)(how.k - 1) : q == 1 ? how.p_target(k_total) : how.u_target(total);
    if (q > 0 && !whole) b = bin_of(sh.mass, t, sh);
    if (q == 0 || (!whole && (b < list_lo || b > list_hi))) {
      list_hi = b;
      for (list_lo = several && sh.cnt[b + 2] <= kList ? 0 : b;; list_lo = b) {
        fresh = collect_bins<BF>(r, list_lo, b, sh);
        if (fresh || whole || list_lo == b) break;
      }
      list_before = sh.above;
      if (!fresh) list_lo = 1, list_hi = 0;
      // Where the next float below a logit lies more than a bin away (low temperatures, logits far from 0), more elements than
      // the bins up to b + 1 have can reach floor_of(b). Then the sums are needed: once more, without that list.
      if (whole && !fresh) {
        whole = several = false;
        q = -1;
        continue;
      }
    }
    const u64 above = sums && list_lo <= list_hi ? sh.mass[list_lo] : 0;
    if (fresh) order_list(r, above, sh);
    if (whole || list_lo <= list_hi) f = in_list(q == 0, t, above, list_before, sh);
    else f = in_large_bin<BF>(r, b, q == 0, t, sh.mass[b], sh);
    if (q == 0) count = (uint32_t)how.k, total = k_total = f.incl;
    if (q == 1 && (uint32_t)f.count < count) count = (uint32_t)f.count, total = f.incl;
  }
  answer(a, row, f.id, (double)f.weight / (double)total, (int)count);
}

// Rows of up to CAP ids: all of them are the list, in one kernel, several rows a CU. 1500 rows of 1000 float32 logits without a
// filter: 95 us by the kernels above, whose passes and barriers wait for each other, 17 so; 1500 rows of 2000: 99 and 31 (37 with
// 256 threads); 1000 rows of 4000, with a top-k of 50: 78 and 71, 39 and 71, so that longer rows are left to those.
template <int CAP, int NT>
struct SmallShared {
  double table[kTable];
  u64 list[CAP], sum[CAP];
  uint32_t start[CAP + 1];
  u64 red64[NT / 64];
  uint32_t red32[NT / 64], red_hi[NT / 64];
  float red_x[NT / 64];
  int red_id[NT / 64];
  int found, kept;
};
template <bool BF, int CAP, int NT>
__global__ void __launch_bounds__(NT) sample_small_kernel(SampleArgs a) {
  constexpr int WAVES = NT / 64, E = CAP / NT;
  __shared__ SmallShared<CAP, NT> sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, row = blockIdx.x;
  Row r = row_of<BF>(a, row, sh.table);
  const How how(a, row);
  float x[E], best = -INFINITY;
  int best_id = INT_MAX;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int id = e * NT + tid;
    x[e] = id < r.V ? logit<BF>(r, id) : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (x[e] > best) best = x[e], best_id = e * NT + tid;
  uint32_t lo = 0xFFFFFFFFu, hi = 0;  // of the complements of the keys, smallest first
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (x[e] > -INFINITY) lo = min(lo, ~order_key(x[e])), hi = max(hi, ~order_key(x[e]));
  for (int o = 32; o >= 1; o >>= 1) {
    const float y = __shfl_xor(best, o, 64);
    const int id = __shfl_xor(best_id, o, 64);
    lower_id(y, id, best, best_id);
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
  if (lane == 0) sh.red_x[wid] = best, sh.red_id[wid] = best_id, sh.red32[wid] = lo, sh.red_hi[wid] = hi;
  fill_table(sh.table, a.shift);
  for (int i = tid; i <= CAP; i += NT) sh.start[i] = 0;
  if (tid == 0) sh.kept = 0;
  __syncthreads();
  for (int w = 0; w < WAVES; ++w) {
    lower_id(sh.red_x[w], sh.red_id[w], best, best_id);
    lo = min(lo, sh.red32[w]);
    hi = max(hi, sh.red_hi[w]);
  }
  if (best == -INFINITY) return answer(a, row, -1, 0.0, 0);
  if (!(how.T > 0.f) || how.k == 1) return answer(a, row, best_id, 1.0, 1);
  const bool infinite = best == INFINITY;  // those ids share the weight alike, all others have none
  r.set(infinite ? 0.f : best, how.T);

  // in order, as order_list has it, but half of the groups lie evenly over the values: a whole row's keys are dense around 0
  const double ids = (double)r.V, scale = (CAP / 2 - 0.25) / ((double)((hi - lo) >> r.drop) * ids + ids);
  const float range = best - key_value(~hi);  // its quotient stays finite, and its products below CAP / 2
  const float even = range > 0.f && range < INFINITY ? fminf((CAP / 2 - 0.25f) / range, 1e30f) : 0.f;
  u64 v[E];
  int at[E], slot[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    at[e] = -1;
    if (!(x[e] > -INFINITY)) continue;
    const uint32_t key = ~order_key(x[e]), id = (uint32_t)(e * NT + tid);
    v[e] = (u64)key << 32 | id;
    at[e] = (int)(fma((double)((key - lo) >> r.drop), ids, (double)id) * scale);
    if (even > 0.f) at[e] += (int)((best - x[e]) * even);
    slot[e] = (int)atomicAdd(&sh.start[at[e]], 1u);
  }
  __syncthreads();
  uint32_t c[E], all = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) c[e] = sh.start[E * tid + e], all += c[e];
  uint32_t cs = all;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t u = __shfl_up(cs, o, 64);
    if (lane >= o) cs += u;
  }
  if (lane == 63) sh.red32[wid] = cs;
  __syncthreads();
  int n = 0;
  cs -= all;
  for (int w = 0; w < WAVES; ++w) {
    if (w < wid) cs += sh.red32[w];
    n += (int)sh.red32[w];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sh.start[E * tid + e] = cs, cs += c[e];
  if (tid == NT - 1) sh.start[CAP] = cs;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (at[e] >= 0) sh.sum[sh.start[at[e]] + slot[e]] = v[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (at[e] < 0) continue;
    const int from = (int)sh.start[at[e]], to = (int)sh.start[at[e] + 1];
    int rank = from;
    for (int i = from; i < to; ++i) rank += sh.sum[i] < v[e];
    sh.list[rank] = v[e];
  }
  __syncthreads();
  // running sums, and how many min-p keeps
  u64 w[E], mine = 0;
  int kept = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    w[e] = 0;
    if (E * tid + e < n) {
      const float y = key_value(~(uint32_t)(sh.list[E * tid + e] >> 32));
      w[e] = infinite ? (u64)(y == INFINITY) : r.mass(y);
      if (how.by_m) kept += infinite ? y == INFINITY : r.weight(y) >= how.m_least;
    }
    mine += w[e];
  }
  u64 ms = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 u = __shfl_up(ms, o, 64);
    if (lane >= o) ms += u;
  }
  if (lane == 63) sh.red64[wid] = ms;
  if (kept) atomicAdd(&sh.kept, kept);
  __syncthreads();
  ms -= mine;
  for (int i = 0; i < wid; ++i) ms += sh.red64[i];
#pragma unroll
  for (int e = 0; e < E; ++e) sh.sum[E * tid + e] = ms += w[e];
  __syncthreads();
  auto find = [&](u64 t) {  // the place at which the running sum passes t, below the last one
#pragma unroll
    for (int i = tid; i < CAP; i += NT)
      if (i < n && sh.sum[i] > t && (i == 0 || sh.sum[i - 1] <= t)) sh.found = i;
    __syncthreads();
    const int i = sh.found;
    __syncthreads();
    return i;
  };
  int count = how.k > 0 && how.k < n ? how.k : n;
  if (how.by_p) count = min(count, find(how.p_target(sh.sum[count - 1])) + 1);
  if (how.by_m) count = min(count, sh.kept);
  const u64 total = sh.sum[count - 1];
  const int i = find(how.u_target(total));
  answer(a, row, (int)(uint32_t)sh.list[i], (double)(sh.sum[i] - (i > 0 ? sh.sum[i - 1] : 0)) / (double)total, count);
}

// Workgroups that share a row: a power of two, together up to one a CU, and at least 4096 ids each. Rows of fewer than 20000 ids
// stay whole (us shared and whole, 3 rows of float32 without a filter and with a top-k of 1000: 9000 ids 23 / 27 and 20 / 23,
// 17000 25 / 29 and 24 / 26, 31000 27 / 30 and 29 / 28, 60000 31 / 34 and, in two parts, 36 / 40).
constexpr int kShares = 256, kShare = 4096, kSharedFrom = 20000;
static int sample_parts(int n, int V) {
  int parts = 1;
  while (V >= kSharedFrom && parts < kMaxParts && (long)n * parts * 2 <= kShares && V / (parts * 2) >= kShare) parts *= 2;
  return parts;
}

size_t sample_ws_bytes(int n, int V) {  // enough for fewer rows and ids too
  const size_t shared = V >= kSharedFrom ? (n < kShares / 2 ? n : kShares / 2) : 0;
  return (size_t)n * sizeof(RowState) + shared * sizeof(SplitRow);
}

template <bool BF>
static void run_sample(const SampleArgs& a, hipStream_t s) {
  const int parts = sample_parts(a.n, a.V);
  const dim3 rows(a.n), shares((unsigned)a.n * parts), threads(kSampleThreads);
  if (a.V <= 1024) {
    hipLaunchKernelGGL((sample_small_kernel<BF, 1024, 256>), rows, dim3(256), 0, s, a);
  } else if (a.V <= 2048) {
    hipLaunchKernelGGL((sample_small_kernel<BF, 2048, 512>), rows, dim3(512), 0, s, a);
  } else if (parts > 1) {
    hipLaunchKernelGGL(sample_part_kernel<BF>, shares, threads, 0, s, a, parts);
    hipLaunchKernelGGL(sample_gather_kernel<BF>, shares, threads, 0, s, a, parts);
    hipLaunchKernelGGL((sample_full_kernel<BF, true>), rows, threads, 0, s, a);
  } else {
    hipLaunchKernelGGL(sample_top_kernel<BF>, rows, threads, 0, s, a);
    if (BF) hipLaunchKernelGGL(sample_values_kernel, rows, threads, 0, s, a);
    hipLaunchKernelGGL((sample_full_kernel<BF, false>), rows, threads, 0, s, a);
  }
}

void launch_sample(const SampleArgs& a, hipStream_t s) {
  constexpr int MOST = 1 << 21;  // rows of a launch: 2^32 threads are too many
  for (int first = 0; first < a.n; first += MOST) {
    SampleArgs b = a;
    b.n = a.n - first < MOST ? a.n - first : MOST;
    b.logits = static_cast<const char*>(a.logits) + (size_t)first * a.stride * (a.bf16 ? 2 : 4);
    auto from = [&](auto*& p) {
      if (p) p += first;
    };
    from(b.temperature), from(b.top_k), from(b.top_p), from(b.min_p), from(b.uniform), from(b.token), from(b.conf), from(b.kept);
    a.bf16 ? run_sample<true>(b, s) : run_sample<false>(b, s);  // in turn, over the same workspace
  }
}

}  // namespace dcl
