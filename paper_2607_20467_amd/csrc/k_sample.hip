// Drawing one token per row of logits: temperature, top-k, top-p, min-p, one given uniform number per row.
//
// The ids of a row in order of (logit descending, id ascending) have weights w = exp((x - M) / T), M the row's maximum.
// Every filter keeps a prefix of that order, and the draw asks for the element at which the running sum passes
// u * total, so all of them are one question: at which element does the running count or the running sum of weights
// pass a value? It is answered without sorting the row: a histogram of 2048 bins over (M - x) / T (count and sum per bin)
// says in which bin, and only that bin's elements (or, where they are few, all up to it) are collected into LDS, sorted and
// summed. A bin with more elements than fit is split again by value; equal values are answered by arithmetic.
//
// Weights are exponentials to 1e-13, held as whole numbers of 2^-shift, so every sum is exact in any order: results do not
// depend on timing, and a border falls as exact arithmetic on the weights has it (a float32 sum's error of 1e-7 would move
// one border in a hundred rows of a flat distribution over 10^5 ids).
//
// Two kernels. The first finds the maximum of every row and answers those that need no more (the top-1 alone) or little
// more (top-k with the ids down to its border in LDS: nothing else of the row needs a weight). The second answers the
// others from the histogram; it is another kernel because its arithmetic takes twice the registers.
#include <limits.h>

#include "dcl_internal.h"

namespace dcl {

constexpr int kBins = 2048, kList = 2048, kSampleThreads = 1024, kWaves = kSampleThreads / 64;
// The last bin starts 31.98 nats below the maximum: weights there are below 2^-46, which rounds to 0 of 2^-45 and more.
constexpr float kBinsPerNat = 64.f;
constexpr int kTable = 256;  // 2^(i / 256)

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
  int shift;
  float M, bin_scale;
  double rate;       // log2(e) / T

  // M finite
  __device__ __forceinline__ void set(float top, float T) {
    M = top;
    rate = 1.4426950408889634 / (double)T;
    bin_scale = fminf(fmaxf(kBinsPerNat / T, 1e-36f), 1e38f);
  }
  // 2^shift times the weight of a logit x <= M: 2^(shift + y), y = (x - M) / T log2(e), with y rounded to a multiple of
  // 1 / 256 from the table and 2^r of the rest, |r| <= 2^-9, by its series to the third power (the next term is 1.4e-13).
  // Of no use past the histogram's range (where the weight rounds to 0).
  __device__ __forceinline__ double weight_near(float x) const {
    const double y = ((double)x - (double)M) * rate;
    const double magic = 26388279066624.0;  // 1.5 * 2^44: the sum's last bit is 2^-8
    const double t = y + magic;
    const int k = (int)(uint32_t)__double_as_longlong(t);
    const double z = (y - (t - magic)) * 0.6931471805599453;
    double p = fma(z, 1.0 / 6.0, 0.5);
    p = fma(z, p, 1.0);
    p = fma(z, p, 1.0);
    return __builtin_amdgcn_ldexp(table[k & (kTable - 1)] * p, (k >> 8) + shift);
  }
  __device__ __forceinline__ double weight(float x) const {  // any x <= M
    return ((double)x - (double)M) * rate > -200.0 ? weight_near(x) : 0.0;
  }
  __device__ __forceinline__ static u64 fixed(double w) {  // 0 <= w < 2^52, to the nearest whole number
    return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
  }
  // place in the histogram: does not decrease while x falls; 0 for x = M
  __device__ __forceinline__ float place(float x) const { return (M - x) * bin_scale; }
  __device__ __forceinline__ int bin(float x) const { return (int)fminf(place(x), (float)(kBins - 1)); }
  // the least logit above -inf for which `keep` holds; keep(M) does, and for whatever lies above one for which it does
  template <class P>
  __device__ __forceinline__ float least(P keep) const {
    uint32_t lo = order_key(-3.4028234663852886e38f), hi = order_key(M);
#pragma unroll 1
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (keep(key_value(mid))) hi = mid;
      else lo = mid + 1;
    }
    return key_value(hi);
  }
};

template <bool BF>
__device__ __forceinline__ Row row_of(const SampleArgs& a, int row, const double* table) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES;
  Row r;
  r.base = static_cast<const char*>(a.logits) + (size_t)row * a.stride * ES;
  r.table = table;
  r.V = a.V;
  const int at = (int)((reinterpret_cast<uintptr_t>(r.base) & 15) / ES);
  r.head = at ? min(VEC - at, a.V) : 0;
  r.shift = a.shift;
  return r;
}
template <bool BF>
__device__ __forceinline__ float logit(const Row& r, int id) {
  return BF ? bf2f(reinterpret_cast<const bf16_t*>(r.base)[id]) : reinterpret_cast<const float*>(r.base)[id];
}

// piece(x, id0) for the aligned 16 bytes of logits x[0 .. VEC) of ids id0 .., U loads of a thread in flight (past the last
// one: NaN, which every caller passes over), and one(x, id) for the row's few elements before and behind them.
template <bool BF, int U, class P, class O>
__device__ __forceinline__ void each_piece(const Row& r, P piece, O one) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES;
  const int pieces = (r.V - r.head) / VEC, tail = r.head + pieces * VEC;
  const int edge = (int)threadIdx.x < r.head ? (int)threadIdx.x : tail + (int)threadIdx.x - r.head;
  if (edge < r.V && (int)threadIdx.x < 2 * VEC) one(logit<BF>(r, edge), edge);
  const uint4* src = reinterpret_cast<const uint4*>(r.base + (size_t)r.head * ES);
  auto take = [&](const uint4& w, int p) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    float x[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      x[e] = BF ? __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16) : __uint_as_float(v[e & 3]);
    piece(x, r.head + p * VEC);
  };
#pragma unroll 1
  for (int p = threadIdx.x; p < pieces; p += kSampleThreads * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = make_uint4(~0u, ~0u, ~0u, ~0u);
      if (p + u * kSampleThreads < pieces) w[u] = src[p + u * kSampleThreads];
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
// f(x, id) for the logits of at least lo, which are taken to be few
template <bool BF, class F>
__device__ __forceinline__ void each_from(const Row& r, float lo, F f) {
  each_piece<BF, 4>(
      r,
      [&](const auto& x, int id0) {
        if (!(largest(x) >= lo)) return;
#pragma unroll
        for (int e = 0; e < (BF ? 8 : 4); ++e)
          if (x[e] >= lo) f(x[e], id0 + e);
      },
      [&](float x, int id) {
        if (x >= lo) f(x, id);
      });
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
  u64 red64[kWaves];
  uint32_t red32[kWaves];
  float red_x[kWaves];
  int n;
};
struct FullShared : ListShared {
  u64 mass[kBins + 1];
  uint32_t cnt[kBins + 1];
  uint32_t lo, hi, m_cnt;
  u64 m_mass;
};

// The row's settings and what follows from them.
struct How {
  float T, pf, uf;
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
__device__ __forceinline__ void fill_table(double* table) {
  if (threadIdx.x < kTable) table[threadIdx.x] = exp2((int)threadIdx.x * (1.0 / kTable));
}

// Exclusive prefix sums of 2048 counts (and sums) in place, totals behind the last. All threads; ends with a barrier.
template <bool MASS>
__device__ __forceinline__ void scan_bins(uint32_t* cnt, u64* mass, ListShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  static_assert(kBins == 2 * kSampleThreads, "two bins a thread");
  const uint32_t c0 = cnt[2 * tid], c1 = cnt[2 * tid + 1];
  const u64 m0 = MASS ? mass[2 * tid] : 0, m1 = MASS ? mass[2 * tid + 1] : 0;
  uint32_t c = c0 + c1;
  u64 m = m0 + m1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t cu = __shfl_up(c, o, 64);
    if (lane >= o) c += cu;
    if constexpr (MASS) {
      const u64 mu = __shfl_up(m, o, 64);
      if (lane >= o) m += mu;
    }
  }
  if (lane == 63) sh.red32[wid] = c, sh.red64[wid] = m;
  __syncthreads();
  for (int w = 0; w < wid; ++w) {
    c += sh.red32[w];
    if constexpr (MASS) m += sh.red64[w];
  }
  cnt[2 * tid] = c - c0 - c1;
  cnt[2 * tid + 1] = c - c1;
  if (tid == kSampleThreads - 1) cnt[kBins] = c;
  if constexpr (MASS) {
    mass[2 * tid] = m - m0 - m1;
    mass[2 * tid + 1] = m - m1;
    if (tid == kSampleThreads - 1) mass[kBins] = m;
  }
  __syncthreads();
}

// Last bin whose exclusive prefix is at most t.
template <class T>
__device__ __forceinline__ int bin_of(const T* excl, T t) {
  int lo = 0, hi = kBins - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (excl[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The elements with lo <= x < hi into the list as (~key, id), if they fit it; sh.n counts them. All threads.
template <bool BF>
__device__ __forceinline__ bool collect_between(const Row& r, float lo, float hi, ListShared& sh) {
  __syncthreads();
  if (threadIdx.x == 0) sh.n = 0;
  __syncthreads();
  each_from<BF>(r, lo, [&](float x, int id) {
    if (!(x < hi)) return;
    const int i = atomicAdd(&sh.n, 1);
    if (i < kList) sh.list[i] = ((u64)~order_key(x) << 32) | (uint32_t)id;
  });
  __syncthreads();
  return sh.n <= kList;
}

// The sh.n collected pairs in order, and the running sums of their weights from `above`. All threads.
__device__ __forceinline__ void order_list(const Row& r, u64 above, ListShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = sh.n;
  // A bitonic network, element e * 1024 + thread in register e: partners 1024 apart meet in a thread, those less than 64
  // apart in a wave, and only the rest through LDS, two buffers in turn and so one barrier each.
  int m = 64;
  while (m < n) m <<= 1;
  u64 v[2] = {tid < n ? sh.list[tid] : ~0ull, tid + kSampleThreads < n ? sh.list[tid + kSampleThreads] : ~0ull};
  auto order = [&](int e, u64 other, int size, int step) {
    const int i = e * kSampleThreads + tid;
    const bool low = ((i & step) == 0) == ((i & size) == 0);  // this place takes the smaller one
    v[e] = low ? (v[e] < other ? v[e] : other) : (v[e] < other ? other : v[e]);
  };
  int turn = 0;
  __syncthreads();
#pragma unroll 1
  for (int size = 2; size <= m; size <<= 1)
#pragma unroll 1
    for (int step = size >> 1; step > 0; step >>= 1) {
      if (step == kSampleThreads) {
        const u64 x = v[0], y = v[1];
        order(0, y, size, step);
        order(1, x, size, step);
      } else if (step < 64) {
        const u64 x = __shfl_xor(v[0], step, 64);
        order(0, x, size, step);
        if (m > kSampleThreads) {
          const u64 y = __shfl_xor(v[1], step, 64);
          order(1, y, size, step);
        }
      } else {
        u64* buf = turn ? sh.list : sh.sum;
        turn ^= 1;
        buf[tid] = v[0];
        buf[tid + kSampleThreads] = v[1];
        __syncthreads();
        order(0, buf[tid ^ step], size, step);
        order(1, buf[kSampleThreads + (tid ^ step)], size, step);
      }
    }
  __syncthreads();
  sh.list[tid] = v[0];
  sh.list[tid + kSampleThreads] = v[1];
  __syncthreads();
  static_assert(kList == 2 * kSampleThreads, "two elements a thread");
  u64 w0 = 0, w1 = 0;
  if (2 * tid < n) w0 = Row::fixed(r.weight(key_value(~(uint32_t)(sh.list[2 * tid] >> 32))));
  if (2 * tid + 1 < n) w1 = Row::fixed(r.weight(key_value(~(uint32_t)(sh.list[2 * tid + 1] >> 32))));
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

// In the ordered list, whose elements follow `above` (sum) and `before` (count): by count (0-based index) or sum.
__device__ __forceinline__ Found in_list(bool by_count, u64 t, u64 above, uint32_t before, const ListShared& sh) {
  int i;
  if (by_count) {
    i = (int)((uint32_t)t - before);
  } else {
    int lo = 0, hi = sh.n - 1;  // first running sum above t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sh.sum[mid] > t) hi = mid;
      else lo = mid + 1;
    }
    i = lo;
  }
  const u64 prev = i > 0 ? sh.sum[i - 1] : above;
  return {sh.sum[i], sh.sum[i] - prev, (int)before + i + 1, (int)(uint32_t)sh.list[i]};
}

// Id of the j-th of the elements equal to the value of `k`, in order of ids: a range of ids is cut into one part per wave,
// the waves count, and the part that holds it is cut again. All threads.
template <bool BF>
__device__ __forceinline__ int equal_id(const Row& r, uint32_t k, u64 j, ListShared& sh) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  auto hit = [&](int id) {
    const float x = logit<BF>(r, id);
    return x > -INFINITY && order_key(x) == k;
  };
  int lo = 0, len = r.V;
#pragma unroll 1
  while (len > 64) {
    const int part = (len + kWaves - 1) / kWaves, from = lo + wid * part, to = min(from + part, lo + len);
    int n = 0;
    constexpr int U = 8;
#pragma unroll 1
    for (int i = from + lane; i < to; i += 64 * U) {
      bool h[U];
#pragma unroll
      for (int u = 0; u < U; ++u) h[u] = i + 64 * u < to && hit(i + 64 * u);
#pragma unroll
      for (int u = 0; u < U; ++u) n += h[u];
    }
    for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
    __syncthreads();
    if (lane == 0) sh.red32[wid] = (uint32_t)n;
    __syncthreads();
    int w = 0;
    while (w < kWaves - 1 && j >= sh.red32[w]) j -= sh.red32[w++];
    const int end = lo + len;
    lo += w * part;
    len = min(part, end - lo);
    if (len <= 0) return -1;  // fewer than j + 1 such elements: not reached
  }
  u64 m = __builtin_amdgcn_ballot_w64(lane < len && hit(lo + lane));  // every wave alike
  for (u64 i = 0; i < j && m; ++i) m &= m - 1;
  return m ? lo + (int)__builtin_ctzll(m) : -1;
}

// What the first kernel leaves for the second: the row's maximum, NaN where the row is answered.
struct RowTop {
  float M;
};

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
  const int id = equal_id<BF>(r, order_key(INFINITY), how.u_target(total), sh);
  answer(a, row, id, 1.0 / (double)total, (int)count);
}

template <bool BF>
__global__ void __launch_bounds__(kSampleThreads, 8) sample_top_kernel(SampleArgs a) {
  __shared__ ListShared sh;
  __shared__ uint32_t cnt[kBins + 1];
  __shared__ int red_id[kWaves];
  __shared__ float red_least[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, row = blockIdx.x;
  Row r = row_of<BF>(a, row, sh.table);
  RowTop* left = static_cast<RowTop*>(a.ws) + row;
  // the maximum and its lowest id; the threads' own maxima
  float best = -INFINITY;
  int best_id = INT_MAX;
  auto lower = [](float x, int id, float& bx, int& bid) {
    if (x > bx || (x == bx && id < bid)) bx = x, bid = id;
  };
  each_piece<BF, 4>(
      r,
      [&](const auto& x, int id0) {
        if (!(largest(x) >= best)) return;  // an equal one may have a lower id than an edge element's
#pragma unroll
        for (int e = 0; e < (BF ? 8 : 4); ++e) lower(x[e], id0 + e, best, best_id);
      },
      [&](float x, int id) { lower(x, id, best, best_id); });
  if (best == -INFINITY) best_id = INT_MAX;
  const float own = best;
  for (int o = 32; o >= 1; o >>= 1) {
    const float x = __shfl_xor(best, o, 64);
    const int id = __shfl_xor(best_id, o, 64);
    lower(x, id, best, best_id);
  }
  float least = own > -INFINITY ? own : INFINITY;  // of the threads' maxima
  for (int o = 32; o >= 1; o >>= 1) least = fminf(least, __shfl_xor(least, o, 64));
  if (lane == 0) sh.red_x[wid] = best, red_id[wid] = best_id, red_least[wid] = least;
  fill_table(sh.table);
  for (int i = tid; i <= kBins; i += kSampleThreads) cnt[i] = 0;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) lower(sh.red_x[w], red_id[w], best, best_id);
  const How how(a, row);
  if (tid == 0) left->M = __uint_as_float(0x7FC00000u);
  if (best == -INFINITY) return answer(a, row, -1, 0.0, 0);  // nothing but -inf and NaN
  if (!(how.T > 0.f) || how.k == 1) return answer(a, row, best_id, 1.0, 1);
  if (best == INFINITY) return infinite_row<BF>(a, row, r, how, sh);
  r.set(best, how.T);
  // Top-k: the k-th largest of the threads' maxima is a lower bound for the k-th largest element, and for k up to half the
  // threads not many more elements reach it (about 710 for 512 of 152064 in no order). The bound to within 1 / 2047 of the
  // maxima's range, from a histogram of them.
  if (how.k > 0 && how.k <= kSampleThreads / 2) {
    for (int w = 0; w < kWaves; ++w) least = fminf(least, red_least[w]);
    const float step = fminf(2047.f / (best - least), 1e30f);
    auto bin = [&](float x) { return (int)fminf((best - x) * step, 2047.f); };  // does not decrease while x falls
    if (own > -INFINITY) atomicAdd(&cnt[bin(own)], 1u);
    __syncthreads();
    scan_bins<false>(cnt, nullptr, sh);
    if (cnt[kBins] >= (uint32_t)how.k) {
      const int b = bin_of<uint32_t>(cnt, (uint32_t)(how.k - 1));
      if (collect_between<BF>(r, r.least([&](float x) { return bin(x) <= b; }), INFINITY, sh)) {
        order_list(r, 0, sh);
        int count = how.k;
        if (how.by_p) count = min(count, in_list(false, how.p_target(sh.sum[count - 1]), 0, 0, sh).count);
        if (how.by_m) {  // weights fall along the list: the first one below min-p
          int lo = 1, hi = count;
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (r.weight(key_value(~(uint32_t)(sh.list[mid] >> 32))) >= how.m_least) lo = mid + 1;
            else hi = mid;
          }
          count = lo;
        }
        const u64 total = sh.sum[count - 1];
        const Found f = in_list(false, how.u_target(total), 0, 0, sh);
        return answer(a, row, f.id, (double)f.weight / (double)total, count);
      }
    }
  }
  if (tid == 0) left->M = best;
}

// The question inside one bin with more elements than the list holds. All threads; the list is overwritten.
template <bool BF>
__device__ Found in_large_bin(const Row& r, int b, bool by_count, u64 t, u64 above, uint32_t before, FullShared& sh) {
  const int tid = threadIdx.x;
  constexpr int PARTS = 1024;
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.sum);
  u64* mass = sh.list;
  static_assert(PARTS <= kList, "counts and sums of the parts lie in the list's memory");
  // the values that are left, in order_key's terms
  uint32_t klo = order_key(r.least([&](float x) { return r.bin(x) <= b; }));
  uint32_t khi = b == 0 ? order_key(r.M) : order_key(r.least([&](float x) { return r.bin(x) < b; })) - 1;
#pragma unroll 1
  for (;;) {
    // the range that they really take
    __syncthreads();
    if (tid == 0) sh.lo = 0xFFFFFFFFu, sh.hi = 0, sh.n = 0;
    __syncthreads();
    uint32_t lo = 0xFFFFFFFFu, hi = 0, n = 0;
    each_from<BF>(r, key_value(klo), [&](float x, int) {
      const uint32_t k = order_key(x);
      if (k <= khi) lo = min(lo, k), hi = max(hi, k), ++n;
    });
    if (n) {
      atomicMin(&sh.lo, lo);
      atomicMax(&sh.hi, hi);
      atomicAdd(&sh.n, (int)n);
    }
    __syncthreads();
    klo = sh.lo;
    khi = sh.hi;
    const int left = sh.n;
    __syncthreads();
    if (klo == khi) {  // equal values: element j of them, by arithmetic; its id by counting in order
      const u64 w = Row::fixed(r.weight(key_value(klo)));
      const u64 j = by_count ? (uint32_t)t - before : w ? (t - above) / w : 0;
      const int id = equal_id<BF>(r, klo, j, sh);
      return {above + (j + 1) * w, w, (int)(before + (uint32_t)j + 1), id};
    }
    if (left <= kList) {
      collect_between<BF>(r, key_value(klo), key_value(khi + 1), sh);
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
      atomicAdd(&mass[part(k)], Row::fixed(r.weight(x)));
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

template <bool BF>
__global__ void __launch_bounds__(kSampleThreads, 8) sample_full_kernel(SampleArgs a) {
  __shared__ FullShared sh;
  const int tid = threadIdx.x, row = blockIdx.x;
  const float top = static_cast<const RowTop*>(a.ws)[row].M;
  if (!(top > -INFINITY)) return;  // answered
  Row r = row_of<BF>(a, row, sh.table);
  const How how(a, row);
  r.set(top, how.T);
  fill_table(sh.table);
  for (int i = tid; i <= kBins; i += kSampleThreads) sh.cnt[i] = 0, sh.mass[i] = 0;
  if (tid == 0) sh.m_mass = 0, sh.m_cnt = 0;
  __syncthreads();

  // counts and sums of the bins, and of the elements that min-p keeps (few, as a rule)
  const float m_lo = how.by_m ? r.least([&](float x) { return r.weight(x) >= how.m_least; }) : INFINITY;
  u64 m_mass = 0;
  uint32_t far = 0, m_cnt = 0;
  auto count_in = [&](float x, float at, u64 f) {
    if (x >= m_lo) ++m_cnt, m_mass += at < (float)(kBins - 1) ? f : 0;
    if (at < (float)(kBins - 1)) {
      atomicAdd(&sh.cnt[(int)at], 1u);
      atomicAdd(&sh.mass[(int)at], f);
    }
    far += x > -INFINITY && !(at < (float)(kBins - 1));  // most of a row at a low temperature: no atomics on one word
  };
  each_piece<BF, 1>(
      r,
      [&](const auto& x, int) {
        constexpr int N = BF ? 8 : 4, H = 2;  // elements whose arithmetic overlaps
#pragma unroll
        for (int e0 = 0; e0 < N; e0 += H) {
          float at[H];
          u64 f[H];
#pragma unroll
          for (int e = 0; e < H; ++e) at[e] = r.place(x[e0 + e]), f[e] = Row::fixed(r.weight_near(x[e0 + e]));
#pragma unroll
          for (int e = 0; e < H; ++e) count_in(x[e0 + e], at[e], f[e]);
        }
      },
      [&](float x, int) { count_in(x, r.place(x), Row::fixed(r.weight_near(x))); });
  if (far) atomicAdd(&sh.cnt[kBins - 1], far);
  if (m_cnt) atomicAdd(&sh.m_cnt, m_cnt), atomicAdd(&sh.m_mass, m_mass);
  __syncthreads();
  scan_bins<true>(sh.cnt, sh.mass, sh);

  int list_lo = 1, list_hi = 0;  // bins that the list holds
  uint32_t count = sh.cnt[kBins];
  u64 total = sh.mass[kBins], k_total = total;
  Found f;
#pragma unroll 1
  for (int q = 0; q < 3; ++q) {  // the border of top-k, that of top-p, the draw: one copy of the search
    if (q == 0 ? how.k <= 0 || (uint32_t)how.k >= count : q == 1 && !how.by_p) continue;
    if (q == 2 && how.by_m && sh.m_cnt < count) count = sh.m_cnt, total = sh.m_mass;
    const bool by_count = q == 0;
    const u64 t = q == 0 ? (u64)(how.k - 1) : q == 1 ? how.p_target(k_total) : how.u_target(total);
    const int b = by_count ? bin_of<uint32_t>(sh.cnt, (uint32_t)t) : bin_of<u64>(sh.mass, t);
    if (by_count && b == kBins - 1) {  // past every id with a weight: the sum is all there is
      count = (uint32_t)how.k;
      continue;
    }
    const int from = sh.cnt[b + 1] <= kList ? 0 : b;
    if (b >= list_lo && b <= list_hi) {
      f = in_list(by_count, t, sh.mass[list_lo], sh.cnt[list_lo], sh);
    } else if (sh.cnt[b + 1] - sh.cnt[from] > kList) {
      list_lo = 1, list_hi = 0;
      f = in_large_bin<BF>(r, b, by_count, t, sh.mass[b], sh.cnt[b], sh);
    } else {
      collect_between<BF>(r, r.least([&](float x) { return r.bin(x) <= b; }),
                          from > 0 ? r.least([&](float x) { return r.bin(x) < from; }) : INFINITY, sh);
      order_list(r, sh.mass[from], sh);
      list_lo = from;
      list_hi = b;
      f = in_list(by_count, t, sh.mass[from], sh.cnt[from], sh);
    }
    if (q == 0) count = (uint32_t)how.k, total = k_total = f.incl;
    if (q == 1 && (uint32_t)f.count < count) count = (uint32_t)f.count, total = f.incl;
  }
  answer(a, row, f.id, (double)f.weight / (double)total, (int)count);
}

size_t sample_ws_bytes(int n, int V) { return (size_t)n * sizeof(RowTop); }

void launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.n == 0) return;
  auto go = [&](auto top, auto full) {
    hipLaunchKernelGGL(top, dim3(a.n), dim3(kSampleThreads), 0, s, a);
    hipLaunchKernelGGL(full, dim3(a.n), dim3(kSampleThreads), 0, s, a);
  };
  if (a.bf16) go(sample_top_kernel<true>, sample_full_kernel<true>);
  else go(sample_top_kernel<false>, sample_full_kernel<false>);
}

}  // namespace dcl
