// Pages of 4 bits: keys and values of packed tokens into them and back, and attention from a sequence's newest tokens.
#include <type_traits>

#include "dcl_internal.h"
#include "pages_index.h"

namespace dcl {

// ---------------------------------------------------------------- 4-bit rows
// 32 dimensions of a row are stored as e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) times one scale 2^(e - 127):
// the least power of two with amax <= 6 * scale. As with 8 bits, a power of two makes x / scale exact and keeps every stored
// value a bfloat16 number. 32 values share a scale because 12 to 1 is all that the format spans: keys after the rotation have a
// few large dimensions, which cost only their own group its precision. The format has no infinity and no NaN: a group that
// holds one has scale byte 255, for which gfx950's conversions and scaled matrix products give NaN (checked there for every
// byte under every scale). What would round to 2^128 is stored as 3 * 2^126, so that no finite number becomes an infinity, which
// as a value that a row does not see would meet that row's probability of 0.
__device__ __forceinline__ int e2m1_exponent(uint32_t amax_bits) {  // bfloat16 bits of amax, sign cleared
  // amax = 1.f * 2^(E - 127), 6 = 1.5 * 2^2
  const int e = (int)(amax_bits >> 7) - 2 + ((amax_bits & 127) > 64 ? 1 : 0);
  return e < 1 ? 1 : e;  // at most 253
}
__device__ __forceinline__ float scale4(uint32_t e) { return __uint_as_float(e << 23); }  // 255: no finite number

// Largest magnitude of N pairs of bfloat16, as bits: 0x7F80 and more for infinities and NaN.
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
template <int N>
__device__ __forceinline__ uint32_t magnitude(const uint32_t (&w)[N]) {
  u16x2_t m = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, w[i] & 0x7FFF7FFFu));
  return max((uint32_t)m[0], (uint32_t)m[1]);
}
__device__ __forceinline__ uint32_t magnitude8(const uint4& x) { return magnitude({x.x, x.y, x.z, x.w}); }
// The largest numbers' magnitudes cut to the last one below 3.5 * 2^126.
constexpr uint32_t kTop4 = 0x7F5Fu;
__device__ __forceinline__ void cut8(uint4& x) {
  uint32_t* w[4] = {&x.x, &x.y, &x.z, &x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *w[i] = (*w[i] & 0x80008000u) | min(*w[i] & 0x7FFFu, kTop4) | min((*w[i] >> 16) & 0x7FFFu, kTop4) << 16;
}
// Eight bfloat16 over `scale` (a power of two) to eight codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t codes8(const uint4& x, float scale) {
  uint32_t o = 0;
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2_t, x.x), scale, 0);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2_t, x.y), scale, 1);
  o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2_t, x.z), scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2_t, x.w), scale, 3);
}
// The reverse.
__device__ __forceinline__ uint4 widen_codes8(uint32_t w, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}
// Four codes to the low halves of four bytes, and back.
__device__ __forceinline__ uint32_t spread4(uint32_t x) {
  x = (x | x << 8) & 0x00FF00FFu;
  return (x | x << 4) & 0x0F0F0F0Fu;
}

static Divisor divisor(uint32_t d) {  // d >= 1
  const int l = d < 2 ? 0 : 32 - __builtin_clz(d - 1);
  return {(uint32_t)((((1ull << l) - d) << 32) / d + 1), l < 1 ? 0u : 1u, l < 1 ? 0u : (uint32_t)l - 1};
}

// A sequence's rows and its length, asked for together.
__device__ __forceinline__ SeqRows rows_and_length(const Pages& p, int b, int& len) {
  int first = p.cu[b], end = p.cu[b + 1], length = p.len[b];
  asm volatile("" : "+s"(first), "+s"(end), "+s"(length));  // none is waited for before all are
  len = length_of(length);
  return rows_between(first, end, p.T);
}

// Streams that pass the caches by.
typedef uint32_t u32x4p_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void stream_store(void* p, const uint4& x) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4p_t, x), static_cast<u32x4p_t*>(p));
}
__device__ __forceinline__ uint4 stream_load(const void* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(static_cast<const u32x4p_t*>(p)));
}

// ---------------------------------------------------------------- write
// One workgroup takes 64 positions (aligned to 64 in the sequence) of one KV head, eight dimensions a lane. Keys go out as they
// come, through LDS so that they are stored in 16-byte pieces; a value's dimensions i and i + 16 of a group, which share a byte, are
// two lanes apart, and values and scales turn position-innermost in LDS, in chunks of 16 positions that never straddle a page.
// Memory-bound: ten prompts of 400 to 6000 tokens x 32 heads, 325 MB: 60 us, 5.4 TB/s (70 with keys stored by the four bytes of a
// lane, 63 with page numbers looked up behind the rows); one token of each of 48 sequences x 8 heads: 5.4 us, a chain of loads.
// Rows are read past the caches (62 us with plain loads), pages stored through them, for what reads them next: the ten prompts written
// and read back 128.8 -> 108.7 us. Heads of 64: the same prompts, 162 MB, 34 us, 4.7 TB/s.
constexpr int kGroup4 = 64;

template <int DH>
__global__ void __launch_bounds__(256) pages4_write_kernel(Pages p, const bf16_t* __restrict__ k, long kst,
                                                          const bf16_t* __restrict__ v, long vst, int groups, Divisor by_heads,
                                                          Divisor by_groups) {
  constexpr int L = DH / 8, TPR = 256 / L, R = kGroup4 / TPR, G = DH / 32, HB = DH / 2;
  constexpr int PITCH = HB + 4;
  __shared__ __attribute__((aligned(16))) uint8_t sv[kGroup4 * PITCH], sk[kGroup4 * HB], ss[2][G][kGroup4];
  const int gb = by_heads(blockIdx.x), h = blockIdx.x - gb * p.Hkv, b = by_groups(gb), grp = gb - b * groups;
  int len;
  const SeqRows r = rows_and_length(p, b, len);
  const int n = min(r.n, p.max_new), start = len - r.n;  // position of the first row
  const int g0 = (start & ~(kGroup4 - 1)) + grp * kGroup4;
  if (g0 >= start + n) return;
  const int32_t* row = p.table + (size_t)b * p.max_pages;
  const int plen = 1 << p.shift, tid = threadIdx.x, c = tid % L;
  // the pages of what the thread stores, on their way with the rows: of its key, and of its chunk of rows of positions
  static_assert(kGroup4 * (HB / 16) <= 256, "a thread stores one piece of keys");
  const int chunk_k = (g0 + tid / (HB / 16)) >> 4, chunk_v = (g0 >> 4) + (tid & 3);
  const int entry_k = row[page_entry(p.max_pages, p.shift, chunk_k)], entry_v = row[page_entry(p.max_pages, p.shift, chunk_v)];
  uint4 xk[R], xv[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int t = g0 + i * TPR + tid / L - start;
    xk[i] = xv[i] = make_uint4(0, 0, 0, 0);
    if (t >= 0 && t < n) {
      const size_t at = (size_t)(r.first + t);
      xk[i] = stream_load(k + at * kst + (size_t)h * DH + 8 * c);
      xv[i] = stream_load(v + at * vst + (size_t)h * DH + 8 * c);
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L;
    uint32_t ak = magnitude8(xk[i]), av = magnitude8(xv[i]);
#pragma unroll
    for (int o = 2; o >= 1; o >>= 1) {  // four lanes hold a group
      ak = max(ak, (uint32_t)__shfl_xor((int)ak, o, 64));
      av = max(av, (uint32_t)__shfl_xor((int)av, o, 64));
    }
    const bool odd_k = ak >= 0x7F80u, odd_v = av >= 0x7F80u;
    if (max(ak, av) > kTop4) {
      cut8(xk[i]);
      cut8(xv[i]);
    }
    const int ek = odd_k ? 255 : e2m1_exponent(ak), ev = odd_v ? 255 : e2m1_exponent(av);
    const uint32_t qk = odd_k ? 0u : codes8(xk[i], scale4(ek)), qv = odd_v ? 0u : codes8(xv[i], scale4(ev));
    *reinterpret_cast<uint32_t*>(sk + local * HB + 4 * c) = qk;
    const uint32_t other = (uint32_t)__shfl_xor((int)qv, 2, 64);
    const bool upper = (c & 2) != 0;
    // the lower lane makes the bytes of its first four dimensions, the upper one those of its last four
    const uint32_t lo = upper ? other >> 16 : qv & 0xFFFFu, hi = upper ? qv >> 16 : other & 0xFFFFu;
    *reinterpret_cast<uint32_t*>(sv + local * PITCH + 16 * (c >> 2) + 8 * (c & 1) + (upper ? 4 : 0)) = spread4(lo) | spread4(hi) << 4;
    if ((c & 3) == 0) {
      ss[0][c >> 2][local] = (uint8_t)ek;
      ss[1][c >> 2][local] = (uint8_t)ev;
    }
  }
  __syncthreads();
  // keys in pieces of 16 bytes, those of a page one behind the other
  if (tid < kGroup4 * (HB / 16)) {
    const int x = g0 + tid / (HB / 16), page = page_found(entry_k, p.max_pages, p.n_pages, p.shift, chunk_k);
    if (x >= start && x < start + n && page >= 0)
      *reinterpret_cast<uint4*>(p.k + (((size_t)page * p.Hkv + h) * plen + (x & (plen - 1))) * HB + 16 * (tid % (HB / 16))) =
          *reinterpret_cast<const uint4*>(sk + 16 * tid);
  }
  // rows of positions: HB of values, 2 G of scales
  for (int u = tid; u < (HB + 2 * G) * 4; u += 256) {
    const int ch = u & 3, d = u >> 2, p0 = g0 + 16 * ch;
    const int lo = max(0, start - p0), hi = min(16, start + n - p0);
    if (lo >= hi) continue;
    const int page = page_found(entry_v, p.max_pages, p.n_pages, p.shift, chunk_v);
    if (page < 0) continue;
    const size_t ph = (size_t)page * p.Hkv + h;
    const int off = p0 & (plen - 1);
    uint8_t* dst;
    const uint8_t* src;
    int step;
    if (d < HB) {
      dst = p.v + (ph * HB + d) * plen + off;
      src = sv + 16 * ch * PITCH + d;
      step = PITCH;
    } else {
      const int which = (d - HB) / G, g = (d - HB) % G;
      dst = (which ? p.vs : p.ks) + (ph * G + g) * plen + off;
      src = &ss[which][g][16 * ch];
      step = 1;
    }
    if (hi - lo == 16) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = src[4 * j * step] | src[(4 * j + 1) * step] << 8 | src[(4 * j + 2) * step] << 16 |
               (uint32_t)src[(4 * j + 3) * step] << 24;
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      for (int j = lo; j < hi; ++j) dst[j] = src[j * step];
    }
  }
}

// ---------------------------------------------------------------- read
// The reverse, in the same groups. A row whose position no page holds is zeros. The same ten prompts: 69 us, 4.7 TB/s, four fifths of
// it stores of 256 bytes a row and head (48 us behind the call that wrote them: the pages are in the last cache); nine sequences of 300 to 5000 positions x 8 heads, 99 MB: 17.4 us, 5.7 TB/s
// (heads of 64, 50 MB: 10.5 us, 4.7 TB/s).
template <int DH>
__global__ void __launch_bounds__(256) pages4_read_kernel(Pages p, bf16_t* __restrict__ k, long kst, bf16_t* __restrict__ v,
                                                         long vst, int groups, Divisor by_heads, Divisor by_groups) {
  constexpr int L = DH / 8, TPR = 256 / L, R = kGroup4 / TPR, G = DH / 32, HB = DH / 2;
  constexpr int PITCH = kGroup4 + 4;
  __shared__ __attribute__((aligned(16))) uint8_t sv[HB * PITCH], sk[kGroup4 * HB];
  const int gb = by_heads(blockIdx.x), h = blockIdx.x - gb * p.Hkv, b = by_groups(gb), grp = gb - b * groups;
  int len;
  const SeqRows r = rows_and_length(p, b, len);
  const int n = min(r.n, p.max_new), start = len - r.n;
  const int g0 = (start & ~(kGroup4 - 1)) + grp * kGroup4;
  if (g0 >= start + n) return;
  const int32_t* row = p.table + (size_t)b * p.max_pages;
  const int plen = 1 << p.shift, tid = threadIdx.x, c = tid % L;
  uint32_t ks[R], vs[R], held = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L, t = g0 + local - start;
    const int page = t >= 0 && t < n ? page_of(row, p.max_pages, p.n_pages, p.shift, (g0 + local) >> 4) : -1;
    const size_t ph = (size_t)max(page, 0) * p.Hkv + h;
    const int off = (g0 + local) & (plen - 1);
    ks[i] = vs[i] = 0;
    if (page >= 0) {
      held |= 1u << i;
      ks[i] = p.ks[(ph * G + (c >> 2)) * plen + off];
      vs[i] = p.vs[(ph * G + (c >> 2)) * plen + off];
    }
  }
#pragma unroll
  for (int u = tid; u < kGroup4 * (HB / 16); u += 256) {
    const int x = g0 + u / (HB / 16);
    const int page = x >= start && x < start + n ? page_of(row, p.max_pages, p.n_pages, p.shift, x >> 4) : -1;
    if (page >= 0)
      *reinterpret_cast<uint4*>(sk + 16 * u) =
          *reinterpret_cast<const uint4*>(p.k + (((size_t)page * p.Hkv + h) * plen + (x & (plen - 1))) * HB + 16 * (u % (HB / 16)));
  }
#pragma unroll
  for (int u = tid; u < HB * 4; u += 256) {
    const int ch = u & 3, d = u >> 2, p0 = g0 + 16 * ch;
    const int page = p0 < start + n && p0 + 16 > start ? page_of(row, p.max_pages, p.n_pages, p.shift, p0 >> 4) : -1;
    if (page < 0) continue;
    const uint4 x = *reinterpret_cast<const uint4*>(p.v + (((size_t)page * p.Hkv + h) * HB + d) * plen + (p0 & (plen - 1)));
    uint32_t* dst = reinterpret_cast<uint32_t*>(sv + d * PITCH + 16 * ch);
    dst[0] = x.x;
    dst[1] = x.y;
    dst[2] = x.z;
    dst[3] = x.w;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L, t = g0 + local - start;
    if (t < 0 || t >= n) continue;
    const size_t at = (size_t)(r.first + t);
    uint4 ok = make_uint4(0, 0, 0, 0), ov = ok;
    if (held >> i & 1) {
      const uint8_t* s = sv + (16 * (c >> 2) + 8 * (c & 1)) * PITCH + local;
      const int half = c & 2 ? 4 : 0;  // which half of the bytes the lane's dimensions have
      uint32_t w = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) w |= ((uint32_t)(s[e * PITCH] >> half) & 15u) << (4 * e);
      ok = widen_codes8(*reinterpret_cast<const uint32_t*>(sk + local * HB + 4 * c), scale4(ks[i]));
      ov = widen_codes8(w, scale4(vs[i]));
    }
    stream_store(k + at * kst + (size_t)h * DH + 8 * c, ok);
    stream_store(v + at * vst + (size_t)h * DH + 8 * c, ov);
  }
}

// Groups of kGroup4 positions that `n` consecutive positions can touch.
static int groups4_of(int n) { return (n + kGroup4 - 2) / kGroup4 + 1; }

void launch_pages4_write(const Pages& p, const bf16_t* k, long ks, const bf16_t* v, long vs, hipStream_t s) {
  if (p.T == 0 || p.max_new == 0) return;
  const int groups = groups4_of(p.max_new);
  const dim3 grid((unsigned)groups * p.Hkv * p.B);
  if (p.dh == 128) hipLaunchKernelGGL((pages4_write_kernel<128>), grid, dim3(256), 0, s, p, k, ks, v, vs, groups, divisor(p.Hkv), divisor(groups));
  else hipLaunchKernelGGL((pages4_write_kernel<64>), grid, dim3(256), 0, s, p, k, ks, v, vs, groups, divisor(p.Hkv), divisor(groups));
}

void launch_pages4_read(const Pages& p, bf16_t* k, long ks, bf16_t* v, long vs, hipStream_t s) {
  if (p.T == 0 || p.max_new == 0) return;
  const int groups = groups4_of(p.max_new);
  const dim3 grid((unsigned)groups * p.Hkv * p.B);
  if (p.dh == 128) hipLaunchKernelGGL((pages4_read_kernel<128>), grid, dim3(256), 0, s, p, k, ks, v, vs, groups, divisor(p.Hkv), divisor(groups));
  else hipLaunchKernelGGL((pages4_read_kernel<64>), grid, dim3(256), 0, s, p, k, ks, v, vs, groups, divisor(p.Hkv), divisor(groups));
}

// ---------------------------------------------------------------- attention over pages
// o = sum_j softmax_j(scale q.k_j) v_j. A workgroup takes one tile of 16 QF rows of one KV head (its g = H / Hkv query heads times the
// new tokens) and one part of the sequence's keys, its NW waves every NW-th tile of 64 keys of those, which come straight from memory
// into the registers of the matrix instructions. Where a sequence has more than one part they are joined in order.
//
// Row 4 a + r of score step kt is key 16 a + 4 kt + r of the tile, so that lane group a (= lane / 16) ends up with the
// probabilities of 16 adjacent keys, which lie in one page, and loads their values as one 16-byte piece of each row of two
// dimensions.
//
// With one token it is bound by HBM behind its starts: 2 sequences of 100000 to 131072 keys, 28 / 4 heads, 133 MB: 29 us with the join
// (4.5), the kernel alone 5.3 TB/s; 80 of 250 to 9000, 32 / 8 heads, 204 MB: 46 us, 4.4 TB/s. A tile of 64 keys under one fragment takes 300
// vector instructions (160 convert its values, 90 are the softmax's) and 40 matrix ones, 0.8 us of a SIMD where HBM brings one in
// 1.7. Under blocks the two add up: 512 tokens of 4 sequences over 4096 keys, 32 / 8 heads: vector pipes busy 3/4 of the time,
// matrix pipes 2/5 of it, 181 us, 0.69 PFLOP/s; 64 tokens of 8 over 1280, 32 heads: 21.8 us. Sharing the converted values between waves
// through LDS saved a quarter of the vector instructions and lost it again to barriers and LDS reads (8 x 64 tokens 28 to 32 us,
// 4 x 512 205 to 264, where this form took 27 and 202); four fragments a wave spill (44 us).
__device__ __forceinline__ f32x4_t mfma16q(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float max_over_groups(float v) {  // over the lanes l, l ^ 16, l ^ 32, l ^ 48
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_over_groups(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
__device__ __forceinline__ float reference_of(float m) { return m == -INFINITY ? 0.f : m; }

// A query against keys that stay in their 4 bits: gfx950's scaled product takes 128 dimensions of e2m1 times e4m3, every 32 of either
// side under a power-of-two scale of their own, which is how the keys lie in their pages. The query enters as two e4m3 parts,
// the nearest and the nearest to what it leaves under a 16th of its scale. Their eight significant bits are a bfloat16's, down
// to 2^-14 of the group's largest; below, the step is 2^-13 of the scale, which the largest is more than 224 times: an error below
// 2^-21.8 of it. (e4m3 reaches from 2^-9 to 448; the scale is the least power of two with the group's largest at most 448 times it, and
// not below 2^-122, from where on the step is 2^-135 at most and every bfloat16, a multiple of 2^-133, is kept whole.)
//
// The product's own order (found by one-hot operands): lane group g holds dimensions 32 g .. of the e2m1 operand, 16 g .. and 64 +
// 16 g .. of the e4m3 one; a scale operand's lane group g is that of dimensions 32 g .. on both sides.
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
struct QueryParts {
  i32x8_t part[2];
  int scale;  // bytes 0 and 1: the parts' scales of the lane's logical group; 255 where the query is no number
};
struct RawQuery {
  uint4 x[4];  // the lane's elements as loaded: dimensions 16 lg .. and 64 + 16 lg ..
};
__device__ __forceinline__ RawQuery load_query(const bf16_t* q, int lg) {
  RawQuery r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.x[i] = *reinterpret_cast<const uint4*>(q + 64 * (i >> 1) + 16 * lg + 8 * (i & 1));
  return r;
}
// Four elements in two words: x = s1 p1 + s2 p2. The conversions divide and multiply by the scales themselves (exact to the nearest
// e4m3, ties to even, found so for every bfloat16 under ten scales from 2^-122 up), and what the first part leaves is a float32.
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void four_parts(uint32_t a, uint32_t b, float s1, float s2, i32x8_t (&part)[2], int at) {
  s16x2_t one = {0, 0}, two = {0, 0};
  one = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(one, __builtin_bit_cast(bf16x2_t, a), s1, false);
  one = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(one, __builtin_bit_cast(bf16x2_t, b), s1, true);
  const uint32_t p1 = __builtin_bit_cast(uint32_t, one);
  const auto ra = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(p1, s1, false), rb = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(p1, s1, true);
  two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(two, __uint_as_float(a << 16) - ra[0], __uint_as_float(a & 0xFFFF0000u) - ra[1], s2, false);
  two = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(two, __uint_as_float(b << 16) - rb[0], __uint_as_float(b & 0xFFFF0000u) - rb[1], s2, true);
  part[0][at] = (int)p1;
  part[1][at] = __builtin_bit_cast(int, two);
}
__device__ __forceinline__ QueryParts query_parts(RawQuery& q, int lq, int lg, uint32_t sign) {
  if (sign) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q.x[i].x ^= sign, q.x[i].y ^= sign, q.x[i].z ^= sign, q.x[i].w ^= sign;
  }
  int e[2];  // exponents of the groups that the lane's two halves belong to
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint4 &x = q.x[2 * half], &y = q.x[2 * half + 1];
    uint32_t m = magnitude({x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w});
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    const int b = (int)(m >> 7) - 8 + ((m & 127) > 96 ? 1 : 0);  // m = 1.f * 2^(E - 127), 448 = 1.75 * 2^8
    e[half] = m >= 0x7F80u ? 255 : max(b, 5);                    // the second part's is 4 less
  }
  QueryParts r;
  const int from = lq + 32 * (lg & 1), e0 = __shfl(e[0], from, 64), e1 = __shfl(e[1], from, 64), es = lg < 2 ? e0 : e1;
  r.scale = es == 255 ? 0xFFFF : es | (es - 4) << 8;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const float s1 = scale4(e[half]), s2 = scale4(e[half] - 4);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 x = q.x[2 * half + i];
      four_parts(x.x, x.y, s1, s2, r.part, 4 * half + 2 * i);
      four_parts(x.z, x.w, s1, s2, r.part, 4 * half + 2 * i + 1);
    }
  }
  return r;
}

// One fragment's scores of a tile (C layout: key 16 lg + 4 kt + r, query lq). The reference point m (log2 units) moves only when a
// score passes it by more than 2^8 (any reference gives the same quotient), so that most tiles need no maximum across the lanes
// and no rescaling. Returns whether it moved for some lane; then alpha is what the row's sum and output are worth.
__device__ __forceinline__ bool move_reference(const f32x4_t (&sc)[4], float scale, float& m, float& alpha) {
  float top = -INFINITY;
#pragma unroll
  for (int kt = 0; kt < 4; ++kt)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) top = fmaxf(top, sc[kt][rr]);
  if (__builtin_amdgcn_ballot_w64(top * scale > m + 8.f) == 0) return false;
  const float ts = max_over_groups(top) * scale;
  const float mn = ts > m + 8.f ? ts : m;
  alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
  m = mn;
  return true;
}
// The probabilities, as two bfloat16 parts: the nearest and the nearest to what it leaves (2^-16 of each together); the sum l that
// divides takes them unrounded.
__device__ __forceinline__ void probabilities(f32x4_t (&sc)[4], float scale, float m, float& l, bf16x8_t (&pf)[2], bf16x8_t (&rest)[2]) {
  const float mr = -reference_of(m);
  uint32_t first = 0xBF80u;
  asm("" : "+v"(first));  // kept in a register: as an inline -1.0 the product would take it as 0xBF800000
#pragma unroll
  for (int kt = 0; kt < 4; ++kt)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      sc[kt][rr] = __builtin_amdgcn_exp2f(fmaf(sc[kt][rr], scale, mr));
      l += sc[kt][rr];
    }
#pragma unroll
  for (int s2 = 0; s2 < 2; ++s2) {
    const f32x4_t &x = sc[2 * s2], &y = sc[2 * s2 + 1];
    const uint4 w = make_uint4(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
    // p minus its part by products with (-1, 0) and (0, -1): one instruction where taking the part out and subtracting are two (8 x 64
    // tokens 22.4 -> 22.0 us); exact, found so for four million numbers below 2^9
    auto left = [&](uint32_t two, float p0, float p1) {
      const bf16x2_t t = __builtin_bit_cast(bf16x2_t, two);
      return f2bf2(__builtin_amdgcn_fdot2_f32_bf16(t, __builtin_bit_cast(bf16x2_t, first), p0, false),
                   __builtin_amdgcn_fdot2_f32_bf16(t, __builtin_bit_cast(bf16x2_t, 0xBF800000u), p1, false));
    };
    pf[s2] = __builtin_bit_cast(bf16x8_t, w);
    rest[s2] = __builtin_bit_cast(bf16x8_t, make_uint4(left(w.x, x[0], x[1]), left(w.y, x[2], x[3]),
                                                       left(w.z, y[0], y[1]), left(w.w, y[2], y[3])));
  }
}

// Eight keys of the two dimensions that share a byte: converted under each key's scale, then two keys of a dimension side by side.
// w, e: two words of bytes and of scale bytes. A conversion takes its scale's exponent bits alone (found so for all of them): the
// byte is shifted there, with what comes along, for two words at once (the compiler makes two instructions of such a shift: 8 x 64
// tokens 22.0 us, 21.8 so, 80 x 1 token 46.4 and 45.8).
__device__ __forceinline__ void widen_values8(const uint32_t (&w)[2], const uint32_t (&e)[2], uint4& lo, uint4& hi) {
  uint32_t l[4], h[4];
  const uint64_t both = (uint64_t)e[1] << 32 | e[0];
  uint64_t es[4];
  asm("v_lshlrev_b64 %0, 23, %1" : "=v"(es[0]) : "v"(both));
  asm("v_lshlrev_b64 %0, 15, %1" : "=v"(es[1]) : "v"(both));
  asm("v_lshlrev_b64 %0, 7, %1" : "=v"(es[2]) : "v"(both));
  asm("v_lshrrev_b64 %0, 1, %1" : "=v"(es[3]) : "v"(both));
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    auto scale = [&](int i) { return __uint_as_float((uint32_t)(j ? es[i] >> 32 : es[i])); };
    const uint32_t a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale(0), 0));
    const uint32_t b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale(1), 1));
    const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale(2), 2));
    const uint32_t d = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale(3), 3));
    l[2 * j] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    h[2 * j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    l[2 * j + 1] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    h[2 * j + 1] = __builtin_amdgcn_perm(d, c, 0x07060302u);
  }
  lo = make_uint4(l[0], l[1], l[2], l[3]);
  hi = make_uint4(h[0], h[1], h[2], h[3]);
}

// Scale bytes of four keys: those that are not there (`keep` masks the ones that are) become 1, so that any code is a number. The return
// value marks bytes of 253 and more, under which a code can stand for an infinity (4 and 6 under 253, 2 to 6 under 254) or NaN.
__device__ __forceinline__ uint32_t sane_scales(uint32_t& s, uint32_t keep) {
  s = (s & keep) | (0x7F7F7F7Fu & ~keep);
  return ((s & 0x7F7F7F7Fu) + 0x03030303u) & s & 0x80808080u;
}
// Those codes made finite; the rows that see them are given NaN apart. s, w: scales and codes of four keys, odd: the marks.
__device__ __forceinline__ void finite_codes(uint32_t& s, uint32_t& w, uint32_t odd) {
  const uint32_t from_2 = odd & (s << 6), from_4 = odd & ~(s << 6);  // 254 and 255; 253
  w &= ~((w & 0x44444444u & (from_2 >> 7) * 255u) | (w & (w << 1) & 0x44444444u & (from_4 >> 7) * 255u));
  s ^= odd & (s << 6) & (s << 7);                                     // 255 -> 127
}
__device__ __forceinline__ uint32_t first_bytes(int n) {  // a mask of the first n bytes of a word
  return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

template <int DH, int QF, int NW>
__global__ void __launch_bounds__(64 * NW, QF == 1 && NW == 4 ? 3 : 2) pages4_attn_kernel(PagesAttn a) {
  // heads of 64 would leave half of the scaled product empty: their keys are converted to bfloat16
  constexpr bool SCALED = DH == 128;
  constexpr int KT = 64, NKT = 4, HB = DH / 2, G = DH / 32, KS = DH / 32, DT = DH / 16;
  constexpr int KW = DH / 32;  // words of a lane's dimensions of one key
  __shared__ f32x4_t xo[NW][DT][64];
  __shared__ float2 xml[NW][64];
  const Pages& p = a.p;
  // units: row tiles of one (part, sequence, KV head) follow each other on one XCD and share its L2
  const int u = blockIdx.x, eight = u >> 3, group = a.by_tiles(eight), item = 8 * group + (u & 7), tile = eight - group * a.row_tiles;
  if (item >= a.nsplit * p.B * p.Hkv) return;
  const int hb = a.by_heads(item), h = item - hb * p.Hkv, part = a.by_seqs(hb), b = hb - part * p.B;
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* row = p.table + (size_t)b * p.max_pages;
  // The part's i-th tile: every nsplit-th run of 2^run tiles is its own.
  auto tile_of = [&](int i) { return (((i >> a.run) * a.nsplit + part) << a.run) + (i & ((1 << a.run) - 1)); };
  // Pages of the 64 chunks of 16 keys from the part's tile `base` on, one a lane, and of the 64 after those: asked for together with the
  // borders and the length, which they do not depend on, and what is needed of the arguments behind those (the empty assembly keeps
  // all of these loads before the first wait: 64 tokens of 8 sequences over 1280 22.86 -> 22.73 us).
  int base = 0;
  auto chunk_of = [&](int i) { return 4 * tile_of(i + (lane >> 2)) + (lane & 3); };
  auto entry = [&](int i) { return row[page_entry(p.max_pages, p.shift, chunk_of(i))]; };
  auto page_in = [&](int found, int i) { return page_found(found, p.max_pages, p.n_pages, p.shift, chunk_of(i)); };
  int ids = entry(0), ids_next = entry(16);
  int border = p.cu[b], end = p.cu[b + 1], length = p.len[b];
  asm volatile("" : "+v"(ids), "+v"(ids_next), "+s"(border), "+s"(end), "+s"(length)
               : "s"(p.k), "s"(p.v), "s"(p.ks), "s"(p.vs), "s"(a.q), "s"(a.q_stride), "s"(a.g), "s"(a.causal), "s"(p.max_new),
                 "s"(a.by_parts.mul), "s"(a.by_parts.shift1), "s"(a.by_parts.shift2), "s"(a.by_group.mul), "s"(a.by_group.shift1), "s"(a.by_group.shift2));
  const SeqRows r = rows_between(border, end, p.T);
  const int len = __builtin_amdgcn_readfirstlane(length_of(length));
  const int n = min(r.n, p.max_new), rows = n * a.g, row0 = tile * 16 * QF, plen = 1 << p.shift;
  const int kend = min(len, p.max_pages << p.shift);  // keys that the table can name
  // the part's tiles: whole runs, and what the last run has of one
  const int tiles = (kend + KT - 1) / KT, runs = tiles >> a.run, each = a.by_parts(runs), over = runs - each * a.nsplit;
  const int t1 = ((each + (part < over)) << a.run) + (part == over ? tiles & ((1 << a.run) - 1) : 0);
  if (row0 >= rows || (part > 0 && t1 == 0)) return;  // part 0 always answers
  const bool kept = a.nsplit > 1 && tiles > 1 << a.run;  // more than this part: for the join
  ids = page_in(ids, 0);
  const int lq = lane & 15, lg = lane >> 4, la = lq >> 2, lr = lq & 3;

  const float scale = a.scale_log2;
  f32x4_t o[QF][DT];
  float m[QF], l[QF];
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    m[f] = -INFINITY;
    l[f] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[f][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  typedef uint32_t words_t __attribute__((ext_vector_type(KW)));
  typedef uint32_t u32x4q_t __attribute__((ext_vector_type(4)));
  words_t kr[NKT];           // the tile's keys, values and scales, as loaded
  u32x4q_t vr[G], vsr[G], ksr;
  int pid_v = -1;            // page of the lane group's 16 keys of the tile whose values are in vr
  // With one fragment a KV head's rows are one tile, and pages are read once: past the caches, so that they keep what is not (2 x 1
  // token over 131072 keys 33.9 -> 30.5 us, 80 x 1 55.4 -> 50.4).
  auto fetch = [](auto* src) {
    if constexpr (QF == 1) return __builtin_nontemporal_load(src);
    else return *src;
  };
  auto load_keys = [&](int t, int pid) {  // pid: page of keys 64 t + 16 la ..
    const int off = (KT * t + 16 * la) & (plen - 1);
    const size_t ph = (size_t)((unsigned)max(pid, 0)) * p.Hkv + h;
    const uint8_t* base = p.k + ((ph << p.shift) + (off + lr)) * HB + lg * (HB / 4);
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) kr[kt] = fetch(reinterpret_cast<const words_t*>(base + 4 * kt * HB));
    ksr = *reinterpret_cast<const u32x4q_t*>(p.ks + ((ph * G + lg * G / 4) << p.shift) + off);  // byte lr of word kt
  };
  auto load_values = [&](int t, int pid) {  // pid: page of keys 64 t + 16 lg ..
    const int off = (KT * t + 16 * lg) & (plen - 1);
    const size_t ph = (size_t)((unsigned)max(pid, 0)) * p.Hkv + h;
    const uint8_t *vb = p.v + ((ph * HB + lq) << p.shift) + off, *sb = p.vs + ((ph * G) << p.shift) + off;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      vr[g] = fetch(reinterpret_cast<const u32x4q_t*>(vb + ((size_t)(16 * g) << p.shift)));
      vsr[g] = *reinterpret_cast<const u32x4q_t*>(sb + ((size_t)g << p.shift));
    }
    pid_v = pid;
  };

  int pk = -1, pv = -1;
  auto find_pages = [&](int i) {  // of the part's tile i, at most sixteen further than the last one asked for
    if (i - base >= 16) {
      base += 16;
      ids = page_in(ids_next, base);
      ids_next = entry(base + 16);
    }
    pk = __shfl(ids, 4 * (i - base) + la, 64);
    pv = __shfl(ids, 4 * (i - base) + lg, 64);
  };

  // The wave's queries, and how many keys each may see (rows past the last one: like any other, never written). They are asked for
  // behind the pages' numbers and before the first tile, and made ready while that is on its way.
  bf16x8_t qf[SCALED ? 1 : QF][KS];
  QueryParts qp[SCALED ? QF : 1];
  RawQuery raw[SCALED ? QF : 1];
  int lim[QF], lim_min = kend;
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    const int rr = min(row0 + 16 * f + lq, rows - 1), i = a.by_group(rr), head = h * a.g + rr - i * a.g;
    const bf16_t* q = a.q + (size_t)(r.first + i) * a.q_stride + (size_t)head * DH;
    if constexpr (SCALED) {
      raw[f] = load_query(q, lg);
    } else {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        uint4 x = *reinterpret_cast<const uint4*>(q + (DH / 4) * lg + 8 * ks);
        x.x ^= a.q_sign, x.y ^= a.q_sign, x.z ^= a.q_sign, x.w ^= a.q_sign;  // a negative scale is a sign of the query
        qf[f][ks] = __builtin_bit_cast(bf16x8_t, x);
      }
    }
    lim[f] = a.causal ? min(kend, max(0, len - r.n + i + 1)) : kend;
  }
  if (a.causal) lim_min = min(kend, max(0, len - r.n + a.by_group(row0) + 1));
  int i = wid, t = tile_of(i), t_next = t;  // the part's tile, and which of the sequence it is
  if (i < t1) {
    find_pages(i);
    load_keys(t, pk);
    load_values(t, pv);
  }
  if constexpr (SCALED) {
#pragma unroll
    for (int f = 0; f < QF; ++f) qp[f] = query_parts(raw[f], lq, lg, a.q_sign);
  }

  // MORE: a tile of this wave follows, whose loads are issued here. The last tile is a call of its own: behind a branch around the
  // loads, the waits for older ones are counted as if they had not been issued, and wait for them too.
  auto one_tile = [&](auto more) {
    constexpr bool MORE = decltype(more)::value;
    const int k0 = KT * t + 16 * lg;  // the lane group's first key
    f32x4_t sc[QF][NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      const uint32_t key_scale = ksr[kt] >> (8 * lr);  // in the lowest byte
      if constexpr (SCALED) {
        i32x8_t kf = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < KW; ++x) kf[x] = (int)kr[kt][x];
#pragma unroll
        for (int f = 0; f < QF; ++f) {
          sc[f][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          sc[f][kt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp[f].part[0], sc[f][kt], 4, 0, 0, (int)key_scale, 0, qp[f].scale);
          sc[f][kt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp[f].part[1], sc[f][kt], 4, 0, 0, (int)key_scale, 1, qp[f].scale);
        }
      } else {
        bf16x8_t kf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = __builtin_bit_cast(bf16x8_t, widen_codes8(kr[kt][ks], __uint_as_float(key_scale << 23)));
#pragma unroll
        for (int f = 0; f < QF; ++f) {
          sc[f][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) sc[f][kt] = mfma16q(kf[ks], qf[f][ks], sc[f][kt]);
        }
      }
    }
    if constexpr (MORE) {
      find_pages(i + NW);
      t_next = tile_of(i + NW);
      load_keys(t_next, pk);
    }

    // the keys that a row does not see: past its limit, past the last key, in no page
    const bool whole = KT * t + KT <= lim_min && __builtin_amdgcn_ballot_w64(pid_v < 0) == 0;
    if (!whole) {
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        const int seen = pid_v < 0 ? 0 : lim[f] - k0;  // of the lane group's keys
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) sc[f][kt][rr] = 4 * kt + rr < seen ? sc[f][kt][rr] : -INFINITY;
      }
    }
    bf16x8_t pf[QF][2], rest[QF][2];
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      float alpha;
      if (move_reference(sc[f], scale, m[f], alpha)) {
        l[f] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[f][dt] *= alpha;
      }
      probabilities(sc[f], scale, m[f], l[f], pf[f], rest[f]);
    }
    // values: in a tile that some row does not see whole, a probability of 0 must meet no NaN
    if (!whole) {
      const int nv = pid_v < 0 ? 0 : kend - k0;  // the lane group's keys that are there
      uint32_t odd = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          uint32_t e = vsr[g][j];
          odd |= sane_scales(e, first_bytes(nv - 4 * j));
          vsr[g][j] = e;
        }
      if (__builtin_amdgcn_ballot_w64(odd != 0)) {  // rare
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int g = 0; g < G; ++g) {
            uint32_t e = vsr[g][j], w = vr[g][j];
            finite_codes(e, w, sane_scales(e, ~0u));
            vsr[g][j] = e;
            vr[g][j] = w;
          }
#pragma unroll 1
        for (int y = 0; y < KT; ++y) {
          const int key = KT * t + y, pid = page_of(row, p.max_pages, p.n_pages, p.shift, key >> 4);
          if (pid < 0 || key >= kend) continue;
          const size_t ph = (size_t)pid * p.Hkv + h;
          const int off = key & (plen - 1);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const uint32_t e = p.vs[((ph * G + g) << p.shift) + off];
            if (e < 253) continue;
            const uint32_t least = e == 253 ? 0x66u : e == 254 ? 0x44u : 0u;  // bits of the codes that are no numbers
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t miss = ~p.v[((ph * HB + 16 * g + 4 * lg + x) << p.shift) + off] & least;
#pragma unroll
              for (int f = 0; f < QF; ++f) {
                if (key < lim[f] && (miss & 15) == 0) o[f][2 * g][x] = __uint_as_float(0x7FC00000u);
                if (key < lim[f] && (miss & 0xF0) == 0) o[f][2 * g + 1][x] = __uint_as_float(0x7FC00000u);
              }
            }
          }
        }
      }
    }
    __builtin_amdgcn_s_setprio(1);  // ahead of a wave in its softmax: 1 to 2 % under blocks
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        uint4 lo, hi;
        widen_values8({vr[g][2 * s2], vr[g][2 * s2 + 1]}, {vsr[g][2 * s2], vsr[g][2 * s2 + 1]}, lo, hi);
        const bf16x8_t vl = __builtin_bit_cast(bf16x8_t, lo), vh = __builtin_bit_cast(bf16x8_t, hi);
#pragma unroll
        for (int f = 0; f < QF; ++f) {
          o[f][2 * g] = mfma16q(vl, pf[f][s2], o[f][2 * g]);
          o[f][2 * g] = mfma16q(vl, rest[f][s2], o[f][2 * g]);
          o[f][2 * g + 1] = mfma16q(vh, pf[f][s2], o[f][2 * g + 1]);
          o[f][2 * g + 1] = mfma16q(vh, rest[f][s2], o[f][2 * g + 1]);
        }
      }
    // the conversions of the next eight keys between the products of these (left to itself the compiler groups each kind; the shifts
    // before them are not counted)
    __builtin_amdgcn_sched_group_barrier(0x002, 16, 0);
#pragma unroll
    for (int i = 0; i < (2 * G - 1) * 4 * QF; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 4 / QF, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4 * QF, 0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
    if constexpr (MORE) {
      load_values(t_next, pv);
      t = t_next;
    }
  };
  for (; i + NW < t1; i += NW) one_tile(std::true_type());
  if (i < t1) one_tile(std::false_type());

  // The waves' (m, l, o) joined in wave order, query fragment by query fragment: each wave takes every NW-th group of dimensions.
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    if (f) __syncthreads();
    l[f] = sum_over_groups(l[f]);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) xo[wid][dt][lane] = o[f][dt];
    xml[wid][lane] = make_float2(m[f], l[f]);
    __syncthreads();
    const int rr = row0 + 16 * f + lq;
    if (wid >= DT || rr >= rows) continue;
    float e[NW], mm = -INFINITY, lt = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) mm = fmaxf(mm, xml[w][lane].x);
    const float ref = reference_of(mm);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 ml = xml[w][lane];
      e[w] = __builtin_amdgcn_exp2f(ml.x - ref);  // a wave without keys: (-inf, 0), and zeros for an output
      lt += ml.y * e[w];
    }
    const int i = a.by_group(rr);
    const size_t at = (size_t)(r.first + i) * a.H + h * a.g + rr - i * a.g;
    const float inv = lt == 0.f ? 0.f : 1.0f / lt;  // a row without keys is zeros
#pragma unroll
    for (int dt = wid; dt < DT; dt += NW) {
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) x += xo[w][dt][lane] * e[w];
      if (kept)
        *reinterpret_cast<f32x4_t*>(a.po + ((size_t)part * p.T * a.H + at) * DH + 16 * dt + 4 * lg) = x;
      else
        *reinterpret_cast<uint2*>(a.out + at * DH + 16 * dt + 4 * lg) = make_uint2(f2bf2(x[0] * inv, x[1] * inv), f2bf2(x[2] * inv, x[3] * inv));
    }
    if (wid == 0 && lg == 0) {
      if (kept) a.pml[(size_t)part * p.T * a.H + at] = make_float2(mm, lt);
      else if (a.lse) a.lse[at] = lt == 0.f ? -INFINITY : mm * 0.6931471805599453f + logf(lt);
    }
  }
}

// The parts of a (row, head) joined: DH / 4 lanes take its dimensions, G such groups every G-th part, eight of them asked for at
// once, with their references; then the groups in order. One pass, so that two loads follow each other, the lengths and the parts.
template <int DH, int G>
__global__ void __launch_bounds__(256) pages4_join_kernel(PagesAttn a, int head_blocks, Divisor by_blocks, Divisor by_new) {
  constexpr int L = DH / 4, PER = 256 / L, AT = 8;
  __shared__ float4 xo[PER][L];
  __shared__ float2 xml[PER];
  const Pages& p = a.p;
  const int bi = by_blocks(blockIdx.x), hb = blockIdx.x - bi * head_blocks, b = by_new(bi), i = bi - b * p.max_new;
  int len;
  const SeqRows r = rows_and_length(p, b, len);
  const int grp = threadIdx.x / L, c = threadIdx.x % L, head = G > 1 ? hb : hb * PER + grp;
  if (i >= r.n) return;
  const bool mine = head < a.H;  // uniform over the workgroup where groups meet
  const int kend = min(len, p.max_pages << p.shift);
  const int runs = (kend + (64 << a.run) - 1) >> (a.run + 6), parts = mine ? min(a.nsplit, runs) : 0;
  if (runs < 2) return;  // answered by its only part
  const size_t at = (size_t)(r.first + i) * a.H + head, step = (size_t)p.T * a.H;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = G > 1 ? grp : 0; s0 < parts; s0 += AT * G) {
    float2 ml[AT];
    float4 x[AT];
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      const int s = s0 + j * G;
      ml[j] = make_float2(-INFINITY, 0.f);
      x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s < parts) {
        ml[j] = a.pml[s * step + at];
        x[j] = *reinterpret_cast<const float4*>(a.po + (s * step + at) * DH + 4 * c);
      }
    }
    float mn = m;
#pragma unroll
    for (int j = 0; j < AT; ++j) mn = fmaxf(mn, ml[j].x);
    const float ref = reference_of(mn), old = __builtin_amdgcn_exp2f(m - ref);
    l *= old;
    o.x *= old, o.y *= old, o.z *= old, o.w *= old;
#pragma unroll
    for (int j = 0; j < AT; ++j) {
      // a part without keys that the row sees: (-inf, 0), and zeros for an output
      const float e = __builtin_amdgcn_exp2f(ml[j].x - ref);
      l += ml[j].y * e;
      o.x += x[j].x * e, o.y += x[j].y * e, o.z += x[j].z * e, o.w += x[j].w * e;
    }
    m = mn;
  }
  if constexpr (G > 1) {
    xo[grp][c] = o;
    if (c == 0) xml[grp] = make_float2(m, l);
    __syncthreads();
    if (grp > 0) return;
    float mn = m;
#pragma unroll
    for (int s = 1; s < G; ++s) mn = fmaxf(mn, xml[s].x);
    const float ref = reference_of(mn);
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < G; ++s) {
      const float2 ml = xml[s];
      const float e = __builtin_amdgcn_exp2f(ml.x - ref);
      const float4 x = xo[s][c];
      l += ml.y * e;
      o.x += x.x * e, o.y += x.y * e, o.z += x.z * e, o.w += x.w * e;
    }
    m = mn;
  }
  if (!mine) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  *reinterpret_cast<uint2*>(a.out + at * DH + 4 * c) = make_uint2(f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv));
  if (a.lse && c == 0) a.lse[at] = l == 0.f ? -INFINITY : m * 0.6931471805599453f + logf(l);
}

static int query_fragments4(int g, int max_new) { return (long)g * max_new <= 16 ? 1 : 2; }

// How many parts, and how long the runs of keys that they take in turn. The host knows no lengths, only what the table could name;
// runs in turn give every part its share at any length, so that a wide table costs no more than a tight one that has as many parts (80 x 1
// token over 250 to 9000 keys, 32 / 8 heads, tables of 9000 / 131072: 46.5 / 46.2 us; parts of 1536 adjoining keys 50.3 / 105, when runs in turn
// took 47.9). Where the tight one has fewer, the wide one adds workgroups, the join and its workspace: 128 x 1 over 200 to 600: 18.6 / 20.3 us
// (adjoining keys: 130); 64 tokens of 8 sequences over 1280, 32 heads: 23.2 / 24.6.
//
// The tables below were measured when the rules were made, each line with one draw of lengths: their figures compare within a line. (Now:
// 32 x 1 with 320000 keys in all 76 us, 80 x 1 with 186000 46, 200 x 1 with 473000 102, 64 tokens of 8 over 500 to 20000 with 58000 122.)
//
// From a workgroup a CU on (units: sequences x KV heads x row tiles): runs of 2048 keys, since a sequence cut further pays more starts, and
// parts for three rounds of the three workgroups that a CU holds, at least three, to even out the lengths. us by parts, runs of 2048:
// 32 x 1 over 1000 to 32000 (256 units): 3 / 6 / 8 / 10: 123 / 83.7 / 82.9 / 77.4; 80 x 1 (640): 1 / 2 / 3 / 4 / 8: 52.7 / 52.5 / 47.9 / 49.6 /
// 49.6; 200 x 1 (1600): 1 / 2 / 3 / 4: 120 / 110 / 108 / 110; 80 x 1 in 3 by runs of 1024 / 2048 / 4096: 51.0 / 47.9 / 54.4. Under two
// fragments, whose outputs are larger, runs of 16384 and two rounds of two: 8 x 64 over 500 to 20000 (512): 1 / 2 / 4 / 8: 132 / 114 / 113 / 127;
// 4 x 256 over 200 to 20000 (1024): 160 / 173 / - / 176.
//
// Below that, as many parts as cost least if the table were filled: the workgroups of the fullest CU, each its keys and 300 more for
// its start, and 900 for a join (a workgroup of eight waves takes about 5 ns a key), over one part and the numbers from as many as
// all CUs take at once. us: 28 / 4 heads, 2 x 1 over 131072: 16 / 32 (256 workgroups) / 64: 43.0 / 29.0 / 29.4; 32 / 8 heads, 1 x 1 over 20000:
// 16 / 32 / 64: 14.8 / 12.7 / 13.3; 24 x 1 over 2000 to 6000: 1 / 2 / 4: 30.8 / 31.9 / 27.3; 32 / 32 heads, 4 x 1 over 80 to 720: 1 / 2: 8.9 /
// 11.5. Runs of 256 keys, a tile of half of the waves: 1 x 1 over 20000 in runs of 128 / 256 / 512 / 1024: 12.8 / 12.7 / 13.9 / 13.5.
void pages4_attention_parts(int Hkv, int g, int B, int max_new, int capacity, int* parts, int* run) {
  const int qf = query_fragments4(g, max_new);
  const long rows = (long)g * max_new, units = ((rows + 16 * qf - 1) / (16 * qf)) * Hkv * B;
  long n = 1, r = 2;
  if (units >= 256) {
    r = qf == 1 ? 5 : 8;
    n = qf == 1 ? 2304 / units : 1024 / units;
    n = qf == 1 && n < 3 ? 3 : n;
    const long all = (capacity + (64L << r) - 1) >> (r + 6);
    n = n > all ? all : n;
  } else {
    long best = capacity + 300;
    for (long k = 256 / units, i = 0; i < 8; ++k, ++i) {
      const long cost = (units * k + 255) / 256 * (capacity / k + 300) + 900;
      if (k > 1 && cost < best) best = cost, n = k;
    }
  }
  *parts = (int)(n < 1 ? 1 : n > 128 ? 128 : n);
  *run = (int)r;
}

template <int DH>
static void run_pages4_attention(PagesAttn& a, hipStream_t s) {
  const int qf = query_fragments4(a.g, a.p.max_new);
  a.row_tiles = (int)(((long)a.g * a.p.max_new + 16 * qf - 1) / (16 * qf));
  a.by_tiles = divisor(a.row_tiles);
  a.by_heads = divisor(a.p.Hkv);
  a.by_seqs = divisor(a.p.B);
  a.by_parts = divisor(a.nsplit);
  a.by_group = divisor(a.g);
  const long items = (long)a.nsplit * a.p.B * a.p.Hkv;
  const dim3 grid((unsigned)((items + 7) / 8 * 8 * a.row_tiles));
  const bool wide_groups = items * a.row_tiles <= 256;  // one a CU: eight waves take its keys (1 x 1 token over 20000: 13.1 / 12.7 us with four / eight)
  if (qf == 1 && wide_groups) hipLaunchKernelGGL((pages4_attn_kernel<DH, 1, 8>), grid, dim3(512), 0, s, a);
  else if (qf == 1) hipLaunchKernelGGL((pages4_attn_kernel<DH, 1, 4>), grid, dim3(256), 0, s, a);
  else if (wide_groups) hipLaunchKernelGGL((pages4_attn_kernel<DH, 2, 8>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((pages4_attn_kernel<DH, 2, 4>), grid, dim3(256), 0, s, a);
  if (a.nsplit > 1) {
    constexpr int PER = 1024 / DH;  // groups of lanes in a workgroup
    const bool wide = a.nsplit > 16;
    const int blocks = wide ? a.H : (a.H + PER - 1) / PER;
    const dim3 all((unsigned)blocks * a.p.max_new * a.p.B);
    if (wide) hipLaunchKernelGGL((pages4_join_kernel<DH, PER>), all, dim3(256), 0, s, a, blocks, divisor(blocks), divisor(a.p.max_new));
    else hipLaunchKernelGGL((pages4_join_kernel<DH, 1>), all, dim3(256), 0, s, a, blocks, divisor(blocks), divisor(a.p.max_new));
  }
}

void launch_pages4_attention(PagesAttn a, hipStream_t s) {  // T and max_new above 0
  a.p.dh == 128 ? run_pages4_attention<128>(a, s) : run_pages4_attention<64>(a, s);
}

}  // namespace dcl
