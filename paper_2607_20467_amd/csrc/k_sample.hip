// Drawing one token per row of logits: temperature, top-k, top-p, min-p, one given uniform number per row.
//
// The ids of a row in order of (logit descending, id ascending) have weights w = exp((x - M) / T), M the row's maximum.
// Every filter keeps a prefix of that order, and the draw asks for the element at which the running sum passes
// u * total, so all of them are one question: at which element does the running count or the running sum of weights
// pass a value? It is answered without sorting the row: a histogram of 2048 bins over (M - x) / T (count and sum per bin)
// says in which bin, and only that bin's elements (or, where they are few, all up to it) are collected into LDS, sorted and
// summed. A bin with more elements than fit is split again by value; equal values are answered by arithmetic.
//
// Weights are float64 exponentials held as whole numbers of 2^-shift (shift = 62 - bits of the vocabulary), so every sum is
// exact in any order: results do not depend on timing, and a border is decided as exact arithmetic on the weights does.
#include <limits.h>

#include "dcl_internal.h"

namespace dcl {

constexpr int kBins = 2048, kList = 2048, kSampleThreads = 1024, kWaves = kSampleThreads / 64;
constexpr float kBinsPerNat = 64.f;  // 32 nats: weights past the last bin's edge are below 2^-46

typedef unsigned long long u64;

// float as an unsigned number of the same order
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

struct Row {
  const char* base;
  int V, mis;        // vocabulary; elements between the 16-byte line before the row and the row
  float M, bin_scale;
  double inv_t, one;  // 1 / T, 2^shift

  // weight of a finite or +inf logit x <= M in units of 2^-shift
  __device__ __forceinline__ double weight(float x) const {
    if (x == M) return 1.0;
    const double w = exp(((double)x - (double)M) * inv_t);
    return w > 0.0 ? w : 0.0;  // NaN (M and T infinite): none
  }
  __device__ __forceinline__ u64 fixed(double w) const { return (u64)__double2ull_rn(w * one); }
  __device__ __forceinline__ int bin(float x) const {  // does not decrease while x falls
    if (x == M) return 0;
    return (int)fminf((M - x) * bin_scale, (float)(kBins - 1));
  }
};

// f(x, id) for every logit that is not -inf or NaN; a thread's ids increase.
template <bool BF, class F>
__device__ __forceinline__ void each_logit(const Row& r, F f) {
  constexpr int ES = BF ? 2 : 4, VEC = 16 / ES, U = 4;
  const int pieces = (r.mis + r.V + VEC - 1) / VEC;
  auto one = [&](float x, int id) {
    x += 0.f;  // -0 and +0 are one value
    if (x > -INFINITY) f(x, id);
  };
  for (int p0 = threadIdx.x; p0 < pieces; p0 += kSampleThreads * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int id0 = (p0 + u * kSampleThreads) * VEC - r.mis;
      if (id0 >= 0 && id0 + VEC <= r.V) w[u] = *reinterpret_cast<const uint4*>(r.base + (size_t)id0 * ES);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int id0 = (p0 + u * kSampleThreads) * VEC - r.mis;
      if (id0 >= 0 && id0 + VEC <= r.V) {
        const uint32_t v[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          one(BF ? __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16) : __uint_as_float(v[e & 3]), id0 + e);
      } else {
        for (int e = 0; e < VEC; ++e) {
          const int id = id0 + e;
          if (id < 0 || id >= r.V) continue;
          one(BF ? bf2f(reinterpret_cast<const bf16_t*>(r.base)[id]) : reinterpret_cast<const float*>(r.base)[id], id);
        }
      }
    }
  }
}

// Element at which a running value passes a target.
struct Found {
  u64 incl, weight;  // sum up to and with it, its own
  int count, id;     // elements up to and with it, its id
};

struct SampleShared {
  u64 mass[kBins + 1];
  u64 list[kList];
  u64 sum[kList];
  uint32_t cnt[kBins + 1];
  u64 red64[kWaves];
  uint32_t red32[kWaves];
  int n;
  uint32_t lo, hi;
  u64 m_mass;
  uint32_t m_cnt;
};

// Exclusive prefix sums of cnt and mass in place, totals behind the last bin. All threads.
__device__ void scan_bins(uint32_t* cnt, u64* mass, SampleShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  static_assert(kBins == 2 * kSampleThreads, "two bins a thread");
  const uint32_t c0 = cnt[2 * tid], c1 = cnt[2 * tid + 1];
  const u64 m0 = mass[2 * tid], m1 = mass[2 * tid + 1];
  uint32_t c = c0 + c1;
  u64 m = m0 + m1;
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t cu = __shfl_up(c, o, 64);
    const u64 mu = __shfl_up(m, o, 64);
    if (lane >= o) c += cu, m += mu;
  }
  if (lane == 63) sh.red32[wid] = c, sh.red64[wid] = m;
  __syncthreads();
  for (int w = 0; w < wid; ++w) c += sh.red32[w], m += sh.red64[w];
  cnt[2 * tid] = c - c0 - c1;
  mass[2 * tid] = m - m0 - m1;
  cnt[2 * tid + 1] = c - c1;
  mass[2 * tid + 1] = m - m1;
  if (tid == kSampleThreads - 1) cnt[kBins] = c, mass[kBins] = m;
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

// The sh.n collected (~key, id) pairs in order, and the running sums of their weights from `above`. All threads.
__device__ void order_list(const Row& r, u64 above, SampleShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, n = sh.n;
  int m = 2;
  while (m < n) m <<= 1;
  for (int i = n + tid; i < m; i += kSampleThreads) sh.list[i] = ~0ull;
  __syncthreads();
  for (int size = 2; size <= m; size <<= 1)
    for (int step = size >> 1; step > 0; step >>= 1) {
      for (int i = tid; i < m / 2; i += kSampleThreads) {
        const int a = 2 * i - (i & (step - 1)), b = a + step;
        const u64 x = sh.list[a], y = sh.list[b];
        if ((x > y) == ((a & size) == 0)) sh.list[a] = y, sh.list[b] = x;
      }
      __syncthreads();
    }
  static_assert(kList == 2 * kSampleThreads, "two elements a thread");
  u64 w0 = 0, w1 = 0;
  if (2 * tid < n) w0 = r.fixed(r.weight(key_value(~(uint32_t)(sh.list[2 * tid] >> 32))));
  if (2 * tid + 1 < n) w1 = r.fixed(r.weight(key_value(~(uint32_t)(sh.list[2 * tid + 1] >> 32))));
  u64 s = w0 + w1;
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
__device__ Found in_list(bool by_count, u64 t, u64 above, uint32_t before, const SampleShared& sh) {
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

// The question inside one bin with more elements than the list holds. All threads; the list is overwritten.
template <bool BF>
__device__ Found in_large_bin(const Row& r, int b, bool by_count, u64 t, u64 above, uint32_t before, SampleShared& sh) {
  const int tid = threadIdx.x;
  constexpr int PARTS = 1024;
  uint32_t* cnt = reinterpret_cast<uint32_t*>(sh.sum);
  u64* mass = sh.list;
  static_assert(PARTS <= kList, "counts and sums of the parts lie in the list's memory");
  uint32_t klo = 0, khi = 0xFFFFFFFFu;
  for (;;) {
    // the range of the values that are left
    __syncthreads();
    if (tid == 0) sh.lo = 0xFFFFFFFFu, sh.hi = 0, sh.n = 0;
    __syncthreads();
    uint32_t lo = 0xFFFFFFFFu, hi = 0, n = 0;
    each_logit<BF>(r, [&](float x, int) {
      const uint32_t k = order_key(x);
      if (k >= klo && k <= khi && r.bin(x) == b) lo = min(lo, k), hi = max(hi, k), ++n;
    });
    atomicMin(&sh.lo, lo);
    atomicMax(&sh.hi, hi);
    atomicAdd(&sh.n, (int)n);
    __syncthreads();
    klo = sh.lo;
    khi = sh.hi;
    const int left = sh.n;
    __syncthreads();
    if (klo == khi) {  // equal values: element j of them, by arithmetic; its id by counting in order
      const u64 w = r.fixed(r.weight(key_value(klo)));
      const u64 j = by_count ? (uint32_t)t - before : w ? (t - above) / w : 0;
      if (tid == 0) sh.n = -1;
      __syncthreads();
      // Ids in blocks of consecutive ones per wave: a wave counts its block, the workgroup adds up in order.
      u64 seen = 0;
      for (int at = 0; at < r.V; at += kSampleThreads) {
        const int id = at + tid;
        bool hit = false;
        if (id < r.V) {
          float x = BF ? bf2f(reinterpret_cast<const bf16_t*>(r.base)[id]) : reinterpret_cast<const float*>(r.base)[id];
          x += 0.f;
          hit = x > -INFINITY && order_key(x) == klo;
        }
        const u64 mask = __builtin_amdgcn_ballot_w64(hit);
        if ((tid & 63) == 0) sh.red32[tid >> 6] = (uint32_t)__popcll(mask);
        __syncthreads();
        u64 mine = seen + __popcll(mask & ((1ull << (tid & 63)) - 1ull));
        uint32_t all = 0;
        for (int v = 0; v < kWaves; ++v) {
          if (v < (tid >> 6)) mine += sh.red32[v];
          all += sh.red32[v];
        }
        if (hit && mine == j) sh.n = id;
        seen += all;
        __syncthreads();
        if (seen > j) break;
      }
      const int id = sh.n;
      __syncthreads();
      return {above + (j + 1) * w, w, (int)(before + (uint32_t)j + 1), id};
    }
    if (left <= kList) {
      if (tid == 0) sh.n = 0;
      __syncthreads();
      each_logit<BF>(r, [&](float x, int id) {
        const uint32_t k = order_key(x);
        if (k >= klo && k <= khi && r.bin(x) == b) sh.list[atomicAdd(&sh.n, 1)] = ((u64)~k << 32) | (uint32_t)id;
      });
      __syncthreads();
      order_list(r, above, sh);
      return in_list(by_count, t, above, before, sh);
    }
    // split [klo, khi] into ranges of keys, from the top
    const u64 width = (u64)(khi - klo) + 1;
    auto part = [&](uint32_t k) { return (int)((u64)(khi - k) * PARTS / width); };
    for (int i = tid; i < PARTS; i += kSampleThreads) cnt[i] = 0, mass[i] = 0;
    __syncthreads();
    each_logit<BF>(r, [&](float x, int) {
      const uint32_t k = order_key(x);
      if (k < klo || k > khi || r.bin(x) != b) return;
      atomicAdd(&cnt[part(k)], 1u);
      atomicAdd(&mass[part(k)], r.fixed(r.weight(x)));
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
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6, row = blockIdx.x;
  Row r;
  r.base = static_cast<const char*>(a.logits) + (size_t)row * a.stride * (BF ? 2 : 4);
  r.V = a.V;
  r.mis = (int)((reinterpret_cast<uintptr_t>(r.base) & 15) / (BF ? 2 : 4));
  r.one = (double)(1ull << a.shift);
  auto answer = [&](int token, float conf, int kept) {
    if (tid != 0) return;
    a.token[row] = token;
    if (a.conf) a.conf[row] = conf;
    if (a.kept) a.kept[row] = kept;
  };

  // the maximum and its lowest id
  u64 best = 0;
  each_logit<BF>(r, [&](float x, int id) {
    const u64 k = ((u64)order_key(x) << 32) | (uint32_t)~id;
    best = k > best ? k : best;
  });
  for (int o = 32; o >= 1; o >>= 1) {
    const u64 v = __shfl_xor(best, o, 64);
    best = v > best ? v : best;
  }
  if (lane == 0) sh.red64[wid] = best;
  for (int i = tid; i <= kBins; i += kSampleThreads) sh.cnt[i] = 0, sh.mass[i] = 0;
  if (tid == 0) sh.m_mass = 0, sh.m_cnt = 0;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) best = sh.red64[w] > best ? sh.red64[w] : best;
  if (best == 0) return answer(-1, 0.f, 0);  // nothing but -inf and NaN
  const int top_id = (int)~(uint32_t)best;
  const float T = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  if (!(T > 0.f) || k == 1) return answer(top_id, 1.f, 1);
  r.M = key_value((uint32_t)(best >> 32));
  r.inv_t = 1.0 / (double)T;
  r.bin_scale = fmaxf(kBinsPerNat / T, 1e-30f);
  const float pf = a.top_p ? a.top_p[row] : 1.f, mf = a.min_p ? a.min_p[row] : 0.f;
  const bool by_p = pf < 1.f, by_m = mf > 0.f;
  const double m_least = mf < 1.f ? (double)mf : 1.0;

  // counts and sums of the bins, and of the elements that min-p keeps
  u64 m_mass = 0;
  uint32_t m_cnt = 0;
  __syncthreads();
  each_logit<BF>(r, [&](float x, int) {
    const int b = r.bin(x);
    const double w = r.weight(x);
    const u64 f = r.fixed(w);
    atomicAdd(&sh.cnt[b], 1u);
    if (f) atomicAdd(&sh.mass[b], f);
    if (w >= m_least) ++m_cnt, m_mass += f;
  });
  if (by_m && m_cnt) atomicAdd(&sh.m_cnt, m_cnt), atomicAdd(&sh.m_mass, m_mass);
  __syncthreads();
  scan_bins(sh.cnt, sh.mass, sh);

  int list_lo = 1, list_hi = 0;  // bins that the list holds
  auto find = [&](bool by_count, u64 t) -> Found {
    const int b = by_count ? bin_of<uint32_t>(sh.cnt, (uint32_t)t) : bin_of<u64>(sh.mass, t);
    if (b < list_lo || b > list_hi) {
      const int from = sh.cnt[b + 1] <= kList ? 0 : b;
      if (sh.cnt[b + 1] - sh.cnt[from] > kList) {
        list_lo = 1, list_hi = 0;
        return in_large_bin<BF>(r, b, by_count, t, sh.mass[b], sh.cnt[b], sh);
      }
      __syncthreads();
      if (tid == 0) sh.n = 0;
      __syncthreads();
      each_logit<BF>(r, [&](float x, int id) {
        const int at = r.bin(x);
        if (at >= from && at <= b) sh.list[atomicAdd(&sh.n, 1)] = ((u64)~order_key(x) << 32) | (uint32_t)id;
      });
      __syncthreads();
      order_list(r, sh.mass[from], sh);
      list_lo = from;
      list_hi = b;
    }
    return in_list(by_count, t, sh.mass[list_lo], sh.cnt[list_lo], sh);
  };

  uint32_t count = sh.cnt[kBins];
  u64 total = sh.mass[kBins];
  if (k > 0 && (uint32_t)k < count) {
    count = (uint32_t)k;
    total = find(true, (u64)(k - 1)).incl;
  }
  const uint32_t k_count = count;
  const u64 k_total = total;
  if (by_p) {
    // elements whose sum before them is below p * k_total: up to the one at which it reaches that
    const double y = ceil((double)pf * (double)k_total);
    u64 t = y >= 1.0 ? (u64)y - 1 : 0;
    if (t >= k_total) t = k_total - 1;
    const Found f = find(false, t);
    if ((uint32_t)f.count < count) count = (uint32_t)f.count, total = f.incl;
  }
  if (by_m && sh.m_cnt < count) count = sh.m_cnt, total = sh.m_mass;
  const float uf = a.uniform[row];
  const double y = floor((uf > 0.f ? (double)uf : 0.0) * (double)total);
  u64 t = y < (double)total ? (u64)y : total - 1;
  if (t >= total) t = total - 1;
  const Found f = find(false, t);
  answer(f.id, (float)((double)f.weight / (double)total), (int)count);
}

void launch_sample(const SampleArgs& a, hipStream_t s) {
  if (a.n == 0) return;
  if (a.bf16) hipLaunchKernelGGL(sample_kernel<true>, dim3(a.n), dim3(kSampleThreads), 0, s, a);
  else hipLaunchKernelGGL(sample_kernel<false>, dim3(a.n), dim3(kSampleThreads), 0, s, a);
}

}  // namespace dcl
