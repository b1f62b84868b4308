// The paged cache: keys and values of packed tokens into pages and back (bfloat16, or 8 bits with a scale), and
// attention from a sequence's newest tokens to its pages, split over the cache's length and joined.
#include <type_traits>

#include "dcl_internal.h"
#include "pages_index.h"

namespace dcl {

// ---------------------------------------------------------------- 8-bit rows
// A row of head_dim elements is stored as e4m3 values (4 significant bits, 2^-6 to 448, subnormals down to 2^-9) times
// one scale 2^(e - 127), e a byte in [1, 254]: the least power of two with amax <= 448 * scale. A power of two costs a
// floating-point format no precision (only the subnormal end moves), makes x / scale exact, so that e4m3's rounding to
// nearest even is the only one, and keeps every stored value a bfloat16 number, so that the products of attention see
// exactly what is stored. amax is the largest finite magnitude; infinities and NaN are stored as e4m3 NaN (the format
// has no infinity), with their sign.
__device__ __forceinline__ int e4m3_exponent(uint32_t amax_bits) {  // bfloat16 bits of amax, sign cleared
  // amax = 1.f * 2^(E - 127), 448 = 1.75 * 2^8
  const int e = (int)(amax_bits >> 7) - 8 + ((amax_bits & 127) > 96 ? 1 : 0);
  return e < 1 ? 1 : e;  // at most 247
}
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// Eight bfloat16 (as loaded) to eight e4m3 bytes, times `inv` (a power of two).
__device__ __forceinline__ uint2 quantise8(const uint4& x, float inv) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t o[2];
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int p = 0;
    p = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w[2 * i] << 16) * inv,
                                        __uint_as_float(w[2 * i] & 0xFFFF0000u) * inv, p, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(w[2 * i + 1] << 16) * inv,
                                        __uint_as_float(w[2 * i + 1] & 0xFFFF0000u) * inv, p, true);
    o[i] = (uint32_t)p;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
  if (odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t h = (w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
      if ((h & 0x7F80u) == 0x7F80u) {
        const uint32_t b = 0x7Fu | ((h >> 8) & 0x80u);
        o[i >> 2] = (o[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | (b << (8 * (i & 3)));
      }
    }
  }
  return make_uint2(o[0], o[1]);
}
// Largest finite magnitude of eight bfloat16, as bits.
__device__ __forceinline__ uint32_t amax8(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = w[i] & 0x7FFFu, b = (w[i] >> 16) & 0x7FFFu;
    m = max(m, a < 0x7F80u ? a : 0u);
    m = max(m, b < 0x7F80u ? b : 0u);
  }
  return m;
}

// Streams that pass the caches by, where it measured faster: stores of whole rows and pages (the read measured below 23.5 -> 16.9
// us, write 127 -> 122.5) and the rows that are written to pages (119.3). Pages are read through the caches: their lines are
// asked for in pieces (read 21.7 otherwise, attention over two long sequences 111 instead of 102).
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store_past(void* p, const uint4& x) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, x), static_cast<u32x4_t*>(p));
}
__device__ __forceinline__ uint4 load_past(const void* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(static_cast<const u32x4_t*>(p)));
}
__device__ __forceinline__ void store_past(void* p, const uint2& x) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x2_t, x), static_cast<u32x2_t*>(p));
}

// ---------------------------------------------------------------- write
// One workgroup takes 64 positions (aligned to 64 in the sequence) of one KV head. Rows arrive with the dimension
// innermost; keys go out the same way, values through LDS with the position innermost, in chunks of 16 positions that
// never straddle a page. Memory-bound: each row is read once and each byte of the pages written once. Nine prompts of 500 to
// 7000 tokens x 32 heads into 8-bit pages, 592 MB: 119 us, 5.0 TB/s (a copy reaches 5.1); one token of each of 64 sequences
// x 8 heads: 7.7 us, the chain of border, length, page number and row, one load after the other.
constexpr int kGroup = 64;

template <int DH, bool E4>
__global__ void __launch_bounds__(256) pages_write_kernel(Pages p, const bf16_t* __restrict__ k, long kst,
                                                         const bf16_t* __restrict__ v, long vst, int groups) {
  constexpr int ES = E4 ? 1 : 2, L = DH / 8, TPR = 256 / L, R = kGroup / TPR;
  constexpr int PITCH = DH * ES + 4;  // four chunks of 16 rows apart: other banks
  __shared__ __attribute__((aligned(16))) uint8_t sv[kGroup * PITCH];
  const int h = blockIdx.x % p.Hkv, gb = blockIdx.x / p.Hkv, grp = gb % groups, b = gb / groups;
  const SeqRows r = seq_rows(p.cu, b, p.T);
  const int n = min(r.n, p.max_new), start = seq_len(p.len, b) - r.n;  // position of the first row
  const int g0 = (start & ~(kGroup - 1)) + grp * kGroup;
  if (g0 >= start + n) return;
  const int32_t* row = p.table + (size_t)b * p.max_pages;
  const int plen = 1 << p.shift, tid = threadIdx.x, c = tid % L;
  uint4 xk[R], xv[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int t = g0 + i * TPR + tid / L - start;
    xk[i] = xv[i] = make_uint4(0, 0, 0, 0);
    if (t >= 0 && t < n) {
      const size_t at = (size_t)(r.first + t);
      xk[i] = load_past(k + at * kst + (size_t)h * DH + 8 * c);
      xv[i] = load_past(v + at * vst + (size_t)h * DH + 8 * c);
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L, t = g0 + local - start;
    const int page = t >= 0 && t < n ? page_of(row, p.max_pages, p.n_pages, p.shift, (g0 + local) >> 4) : -1;
    const int off = (g0 + local) & (plen - 1);
    const size_t slot = ((size_t)max(page, 0) * p.Hkv + h) * plen + off;
    if constexpr (E4) {
      uint32_t ak = amax8(xk[i]), av = amax8(xv[i]);
#pragma unroll
      for (int o = L / 2; o >= 1; o >>= 1) {
        ak = max(ak, (uint32_t)__shfl_xor((int)ak, o, 64));
        av = max(av, (uint32_t)__shfl_xor((int)av, o, 64));
      }
      const int ek = e4m3_exponent(ak), ev = e4m3_exponent(av);
      const uint2 qk = quantise8(xk[i], scale_of(254 - ek)), qv = quantise8(xv[i], scale_of(254 - ev));
      uint32_t* d = reinterpret_cast<uint32_t*>(sv + local * PITCH + 8 * c);
      d[0] = qv.x;
      d[1] = qv.y;
      if (page >= 0) {
        store_past(p.k + slot * DH + 8 * c, qk);
        if (c == 0) {
          p.ks[slot] = (uint8_t)ek;
          p.vs[slot] = (uint8_t)ev;
        }
      }
    } else {
      uint32_t* d = reinterpret_cast<uint32_t*>(sv + local * PITCH + 16 * c);
      d[0] = xv[i].x;
      d[1] = xv[i].y;
      d[2] = xv[i].z;
      d[3] = xv[i].w;
      if (page >= 0) store_past(p.k + (slot * DH + 8 * c) * 2, xk[i]);
    }
  }
  __syncthreads();
  for (int u = tid; u < DH * 4; u += 256) {
    const int ch = u & 3, d = u >> 2, p0 = g0 + 16 * ch;
    const int lo = max(0, start - p0), hi = min(16, start + n - p0);
    if (lo >= hi) continue;
    const int page = page_of(row, p.max_pages, p.n_pages, p.shift, p0 >> 4);
    if (page < 0) continue;
    uint8_t* dst = p.v + ((((size_t)page * p.Hkv + h) * DH + d) * plen + (p0 & (plen - 1))) * ES;
    const uint8_t* src = sv + 16 * ch * PITCH + d * ES;
    if (hi - lo == 16) {
      uint32_t w[4 * ES];
#pragma unroll
      for (int j = 0; j < 4 * ES; ++j) {
        if constexpr (E4) {
          w[j] = src[4 * j * PITCH] | src[(4 * j + 1) * PITCH] << 8 | src[(4 * j + 2) * PITCH] << 16 |
                 (uint32_t)src[(4 * j + 3) * PITCH] << 24;
        } else {
          w[j] = *reinterpret_cast<const uint16_t*>(src + 2 * j * PITCH) |
                 (uint32_t)*reinterpret_cast<const uint16_t*>(src + (2 * j + 1) * PITCH) << 16;
        }
      }
#pragma unroll
      for (int j = 0; j < ES; ++j)
        store_past(dst + 16 * j, make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]));
    } else {
      for (int j = lo; j < hi; ++j) {
        if constexpr (E4) dst[j] = src[j * PITCH];
        else reinterpret_cast<uint16_t*>(dst)[j] = *reinterpret_cast<const uint16_t*>(src + j * PITCH);
      }
    }
  }
}

// ---------------------------------------------------------------- read
// The reverse, in the same groups: values come in by rows of positions and leave by rows of dimensions. A row whose
// position no page holds is zeros. Seven sequences of 300 to 5000 positions x 8 heads of 8 bits, 96 MB: 17 us, 5.7 TB/s
// (28 with the heads of a group in workgroups far apart, the keys read after the values and stores that stay in the caches).
template <int DH, bool E4>
__global__ void __launch_bounds__(256) pages_read_kernel(Pages p, bf16_t* __restrict__ k, long kst,
                                                        bf16_t* __restrict__ v, long vst, int groups) {
  constexpr int ES = E4 ? 1 : 2, L = DH / 8, TPR = 256 / L, R = kGroup / TPR;
  constexpr int PITCH = kGroup * ES + 4;
  __shared__ __attribute__((aligned(16))) uint8_t sv[DH * PITCH];
  const int h = blockIdx.x % p.Hkv, gb = blockIdx.x / p.Hkv, grp = gb % groups, b = gb / groups;
  const SeqRows r = seq_rows(p.cu, b, p.T);
  const int n = min(r.n, p.max_new), start = seq_len(p.len, b) - r.n;
  const int g0 = (start & ~(kGroup - 1)) + grp * kGroup;
  if (g0 >= start + n) return;
  const int32_t* row = p.table + (size_t)b * p.max_pages;
  const int plen = 1 << p.shift, tid = threadIdx.x, c = tid % L;
  typedef std::conditional_t<E4, uint2, uint4> Piece;
  Piece xk[R];
  uint32_t held = 0, ks[R], vs[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L, t = g0 + local - start;
    const int page = t >= 0 && t < n ? page_of(row, p.max_pages, p.n_pages, p.shift, (g0 + local) >> 4) : -1;
    const size_t slot = ((size_t)max(page, 0) * p.Hkv + h) * plen + ((g0 + local) & (plen - 1));
    xk[i] = Piece{};
    ks[i] = vs[i] = 0;
    if (page >= 0) {
      held |= 1u << i;
      xk[i] = *reinterpret_cast<const Piece*>(p.k + (slot * DH + 8 * c) * ES);
      if constexpr (E4) ks[i] = p.ks[slot], vs[i] = p.vs[slot];
    }
  }
#pragma unroll
  for (int i = 0; i < DH * 4 / 256; ++i) {
    const int u = tid + 256 * i, ch = u & 3, d = u >> 2, p0 = g0 + 16 * ch;
    const int page = p0 < start + n && p0 + 16 > start ? page_of(row, p.max_pages, p.n_pages, p.shift, p0 >> 4) : -1;
    if (page < 0) continue;
    const uint4* src = reinterpret_cast<const uint4*>(
        p.v + ((((size_t)page * p.Hkv + h) * DH + d) * plen + (p0 & (plen - 1))) * ES);
    uint32_t* dst = reinterpret_cast<uint32_t*>(sv + d * PITCH + 16 * ch * ES);
#pragma unroll
    for (int j = 0; j < ES; ++j) {
      const uint4 x = src[j];
      dst[4 * j] = x.x;
      dst[4 * j + 1] = x.y;
      dst[4 * j + 2] = x.z;
      dst[4 * j + 3] = x.w;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int local = i * TPR + tid / L, t = g0 + local - start;
    if (t < 0 || t >= n) continue;
    const size_t at = (size_t)(r.first + t);
    uint4 ok = make_uint4(0, 0, 0, 0), ov = ok;
    if (held >> i & 1) {
      if constexpr (E4) {
        const uint2 x = xk[i];
        const float fk = scale_of(ks[i]), fv = scale_of(vs[i]);
        uint32_t y[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint8_t* s = sv + (8 * c + 4 * j) * PITCH + local;
          y[j] = s[0] | s[PITCH] << 8 | s[2 * PITCH] << 16 | (uint32_t)s[3 * PITCH] << 24;
        }
        auto pair = [](uint32_t w, bool hi, float f) -> uint32_t {
          const auto q = hi ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
          return f2bf2(q[0] * f, q[1] * f);
        };
        ok = make_uint4(pair(x.x, false, fk), pair(x.x, true, fk), pair(x.y, false, fk), pair(x.y, true, fk));
        ov = make_uint4(pair(y[0], false, fv), pair(y[0], true, fv), pair(y[1], false, fv), pair(y[1], true, fv));
      } else {
        ok = xk[i];
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint8_t* s = sv + (8 * c + 2 * j) * PITCH + 2 * local;
          y[j] = *reinterpret_cast<const uint16_t*>(s) | (uint32_t)*reinterpret_cast<const uint16_t*>(s + PITCH) << 16;
        }
        ov = make_uint4(y[0], y[1], y[2], y[3]);
      }
    }
    store_past(k + at * kst + (size_t)h * DH + 8 * c, ok);
    store_past(v + at * vst + (size_t)h * DH + 8 * c, ov);
  }
}

// Groups of kGroup positions that `n` consecutive positions can touch.
static int groups_of(int n) { return (n + kGroup - 2) / kGroup + 1; }

void launch_pages_write(const Pages& p, const bf16_t* k, long ks, const bf16_t* v, long vs, hipStream_t s) {
  if (p.T == 0 || p.max_new == 0) return;
  const int groups = groups_of(p.max_new);
  const dim3 grid((unsigned)groups * p.Hkv * p.B);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p, k, ks, v, vs, groups); };
  if (p.dh == 128) p.e4m3 ? go(pages_write_kernel<128, true>) : go(pages_write_kernel<128, false>);
  else p.e4m3 ? go(pages_write_kernel<64, true>) : go(pages_write_kernel<64, false>);
}

void launch_pages_read(const Pages& p, bf16_t* k, long ks, bf16_t* v, long vs, hipStream_t s) {
  if (p.T == 0 || p.max_new == 0) return;
  const int groups = groups_of(p.max_new);
  const dim3 grid((unsigned)groups * p.Hkv * p.B);
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, s, p, k, ks, v, vs, groups); };
  if (p.dh == 128) p.e4m3 ? go(pages_read_kernel<128, true>) : go(pages_read_kernel<128, false>);
  else p.e4m3 ? go(pages_read_kernel<64, true>) : go(pages_read_kernel<64, false>);
}

// ---------------------------------------------------------------- attention over pages
// o = sum_j softmax_j(scale q.k_j) v_j over the keys j of the sequence, per query row one running maximum and sum.
// The rows of one KV head (its g = H / Hkv query heads times the sequence's new tokens) are tiles of 16 QF; a workgroup
// takes one tile and `span` keys of the sequence, its four waves every fourth tile of KT of them. The cache is
// read once from HBM straight into the registers of the matrix instructions (no LDS: with one new token nothing is
// shared between waves), the scores are S^T = K Q^T and the probabilities feed O^T = V^T P^T from the same lanes.
//
// Which key sits in which row of a matrix instruction is free as long as scores and values agree: with PK = KT / 4, row
// 4 a + r of score step kt is key PK a + 4 kt + r, so that lane group a (= lane / 16) ends up with the probabilities of PK
// adjacent keys, which lie in one page, and reads its values as whole pieces of the position-innermost rows. In the same
// way the dimensions of a step are those of one 16-byte piece of a key per lane, so that a load covers 64 adjacent bytes of
// each of 16 keys: 8 dimensions of bfloat16, or 16 of 8 bits, which are two steps. KT is 64 for 8-bit pages (16-byte pieces
// of values) and 32 for bfloat16 ones, and for 8-bit ones under several query fragments, whose registers a larger tile
// would spill.
//
// 8-bit rows become bfloat16, exactly: a key with its scale (the conversion takes one; all of a lane's piece is one key),
// a value without, since its piece is many keys; that scale multiplies the key's probability in float32. That product goes
// to the matrix instructions as two bfloat16, the nearest and the nearest to what it leaves, which keep it to 2^-16 of itself;
// the sum that divides takes the probability unrounded. With the first alone (2^-8) the error against 64 bits was 1.8e-3 to
// 2.3e-3 where the output's own rounding gives 1.6e-3 to 1.7e-3, on 90000 keys as on 90: where values of both signs cancel,
// their roundings do no better. The second costs least where memory bounds (one / two parts: 64 x 1 token 78.1 / 78.7 us, 2 x
// 1 long 102.6 / 102.5, 8 x 64 tokens x 32 heads 31.8 / 34.0, x 28 / 4 heads in bfloat16 32.8 / 35.2).
//
// With one token it is bound by HBM: two sequences of 90000 to 131072 keys, 28 / 4 heads, bfloat16, 516 MB: 102 us with the
// join, 5.05 TB/s; 64 sequences of 200 to 8000 8-bit keys, 32 / 8 heads, 323 MB: 79 us, 4.1 TB/s, the rest being the first
// loads and the ragged end. Four sequences of 90 to 700 keys x 32 heads take 12 us, the latency of their loads. Under
// a block of 64 tokens (8 sequences, 1280 8-bit keys, 32 heads: 34 us, 2.7 TB/s) the vector pipes are busy half of the time with
// conversions and exponentials, the matrix pipes a fifth, and a wave has one tile of keys on its way at a time.
__device__ __forceinline__ f32x4_t mfma16p(const bf16x8_t& a, const bf16x8_t& b, const f32x4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float max_groups(float v) {  // over the lanes l, l ^ 16, l ^ 32, l ^ 48
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_groups(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
// eight e4m3 bytes times a power of two
__device__ __forceinline__ bf16x8_t widen8(uint32_t lo, uint32_t hi, float scale = 1.0f) {
  uint4 o;
  o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return __builtin_bit_cast(bf16x8_t, o);
}

// A reference point, and what a row without keys (reference -inf) is taken relative to.
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.f : m; }

template <int DH, bool E4, int QF>
__global__ void __launch_bounds__(256, QF <= 2 ? 2 : 1) pages_attn_kernel(PagesAttn a) {
  constexpr int ES = E4 ? 1 : 2, KT = E4 && QF == 1 ? 64 : 32, PK = KT / 4, NKT = KT / 16, S2 = KT / 32;
  constexpr int KS = DH / 32, DT = DH / 16;
  constexpr int NK = DH * ES / 64;  // 16-byte pieces of a lane's dimensions of one key
  constexpr int VW = PK * ES / 4;   // words of a lane's keys of one dimension
  constexpr int SW = PK / 4;        // words of their scales
  __shared__ f32x4_t xo[3][DT][64];
  __shared__ float2 xml[3][64];
  const Pages& p = a.p;
  // units: row tiles of one (part, sequence, KV head) follow each other on one XCD and share its L2
  const int u = blockIdx.x, item = (u / (8 * a.row_tiles)) * 8 + (u & 7), tile = (u >> 3) % a.row_tiles;
  if (item >= a.nsplit * p.B * p.Hkv) return;
  const int h = item % p.Hkv, b = (item / p.Hkv) % p.B, part = item / (p.Hkv * p.B);
  const SeqRows r = seq_rows(p.cu, b, p.T);
  const int n = min(r.n, p.max_new), rows = n * a.g, row0 = tile * 16 * QF;
  if (row0 >= rows) return;
  const int len = seq_len(p.len, b), plen = 1 << p.shift;
  const int kend = min(len, p.max_pages << p.shift);  // keys that the table can name
  const int t0 = part * (a.span / KT), t1 = min(t0 + a.span / KT, (kend + KT - 1) / KT);
  if (part > 0 && t0 >= t1) return;  // part 0 always answers
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 15, lg = lane >> 4, la = lq >> 2, lr = lq & 3;
  const int32_t* row = p.table + (size_t)b * p.max_pages;

  // the wave's queries, and how many keys each may see (rows past the last one: like any other, never written)
  bf16x8_t qf[QF][KS];
  int lim[QF], lim_min = kend;
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    const int rr = min(row0 + 16 * f + lq, rows - 1), i = rr / a.g, head = h * a.g + rr % a.g;
    const bf16_t* qp = a.q + (size_t)(r.first + i) * a.q_stride + (size_t)head * DH + (E4 ? 16 : 8) * lg;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4 x = *reinterpret_cast<const uint4*>(qp + (E4 ? 64 * (ks >> 1) + 8 * (ks & 1) : 32 * ks));
      x.x ^= a.q_sign, x.y ^= a.q_sign, x.z ^= a.q_sign, x.w ^= a.q_sign;  // a negative scale is a sign of the query
      qf[f][ks] = __builtin_bit_cast(bf16x8_t, x);
    }
    lim[f] = a.causal ? min(kend, max(0, len - r.n + i + 1)) : kend;
  }
  if (a.causal) lim_min = min(kend, max(0, len - r.n + row0 / a.g + 1));

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

  uint4 kr[NKT][NK];                 // the tile's keys, values and scales, as loaded
  typedef uint32_t words_t __attribute__((ext_vector_type(VW)));
  words_t vr[DT];
  uint32_t ksr[SW], vsr[SW];
  int pid_v = -1;                    // page of the lane group's PK keys of the tile whose values are in vr
  const size_t page_bytes = (size_t)p.Hkv * plen * DH * ES, head_bytes = (size_t)h * plen * DH * ES;
  auto load_words = [](uint32_t* w, const uint8_t* src, auto words) {
    if constexpr (decltype(words)::value == 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(src);
      w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(src);
      w[0] = x.x, w[1] = x.y;
    }
  };
  auto load_keys = [&](int t, int pid) {  // pid: page of keys KT t + PK la ..
    const int off = ((KT * t + PK * la) & (plen - 1)) + lr;
    const uint8_t* base = p.k + (size_t)max(pid, 0) * page_bytes + head_bytes + (size_t)off * (DH * ES) + lg * 16;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int x = 0; x < NK; ++x)
        kr[kt][x] = *reinterpret_cast<const uint4*>(base + kt * 4 * DH * ES + 64 * x);
    if constexpr (E4) {  // byte lr of word kt
      const size_t at = ((size_t)max(pid, 0) * p.Hkv + h) * plen + ((KT * t + PK * la) & (plen - 1));
      load_words(ksr, p.ks + at, std::integral_constant<int, SW>());
    }
  };
  auto load_values = [&](int t, int pid) {  // pid: page of keys KT t + PK lg ..
    const int off = (KT * t + PK * lg) & (plen - 1);
    const uint8_t* base = p.v + (size_t)max(pid, 0) * page_bytes + head_bytes + ((size_t)lq * plen + off) * ES;
    const size_t step = (size_t)16 * plen * ES;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) vr[dt] = *reinterpret_cast<const words_t*>(base + dt * step);
    if constexpr (E4) {
      const size_t at = ((size_t)max(pid, 0) * p.Hkv + h) * plen + off;
      load_words(vsr, p.vs + at, std::integral_constant<int, SW>());
    }
    pid_v = pid;
  };
  // eight values of one dimension, of score steps 2 s2 and 2 s2 + 1
  auto value_fragment = [&](int dt, int s2) -> bf16x8_t {
    if constexpr (E4) return widen8(vr[dt][2 * s2], vr[dt][2 * s2 + 1]);
    else return __builtin_bit_cast(bf16x8_t, vr[dt]);
  };
  auto page_at = [&](int t, int grp) { return page_of(row, p.max_pages, p.n_pages, p.shift, (KT * t + PK * grp) >> 4); };

  // Pages of the 64 chunks of 16 keys from `base` on, one a lane, and of the 64 after those: a look-up is then an exchange
  // between lanes. Loaded tile by tile they come back in order with the values before them, so that the next keys are
  // asked for only when this tile's values have arrived (8 x 64 tokens over 1280 keys, 28 / 4 heads, bfloat16: 36.4 us, so
  // 33.2; 32 heads, 8 bits: 41 and 37).
  int base = t0 * (KT / 16);
  int ids = page_of(row, p.max_pages, p.n_pages, p.shift, base + lane);
  int ids_next = page_of(row, p.max_pages, p.n_pages, p.shift, base + 64 + lane);
  int pk = -1, pv = -1;
  auto find_pages = [&](int t) {  // of tile t, at most four further than the last one asked for
    if (t * (KT / 16) - base >= 64) {
      base += 64;
      ids = ids_next;
      ids_next = page_of(row, p.max_pages, p.n_pages, p.shift, base + 64 + lane);
    }
    pk = __shfl(ids, (KT * t + PK * la) / 16 - base, 64);
    pv = __shfl(ids, (KT * t + PK * lg) / 16 - base, 64);
  };

  int t = t0 + wid;
  if (t < t1) {
    find_pages(t);
    load_keys(t, pk);
    load_values(t, pv);
  }
  for (; t < t1; t += 4) {
    const int k0 = KT * t + PK * lg;  // the lane group's first key
    f32x4_t sc[QF][NKT];
#pragma unroll
    for (int f = 0; f < QF; ++f)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) sc[f][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      bf16x8_t kf[KS];
      const float key_scale = E4 ? scale_of((ksr[E4 ? kt : 0] >> (8 * lr)) & 255u) : 1.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (E4) {
          const uint4 x = kr[kt][ks >> 1];
          kf[ks] = ks & 1 ? widen8(x.z, x.w, key_scale) : widen8(x.x, x.y, key_scale);
        } else {
          kf[ks] = __builtin_bit_cast(bf16x8_t, kr[kt][ks]);
        }
      }
#pragma unroll
      for (int f = 0; f < QF; ++f)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sc[f][kt] = mfma16p(kf[ks], qf[f][ks], sc[f][kt]);
    }
    if (t + 4 < t1) {
      find_pages(t + 4);
      load_keys(t + 4, pk);
    }

    // the keys that a row does not see: past its limit, past the last key, in no page
    const bool whole = KT * t + KT <= lim_min && __builtin_amdgcn_ballot_w64(pid_v < 0) == 0;
    auto dead = [&](int f, int kt, int rr) { return pid_v < 0 || k0 + 4 * kt + rr >= lim[f]; };
    if (!whole) {
#pragma unroll
      for (int f = 0; f < QF; ++f)
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int rr = 0; rr < 4; ++rr)
            if (dead(f, kt, rr)) sc[f][kt][rr] = -INFINITY;
    }
    // The reference point m (log2 units) moves only when a score passes it by more than 2^8 (any reference gives the same
    // quotient), so that most tiles need no maximum across the lanes and no rescaling.
    float tmax[QF];
    bool move = false;
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      tmax[f] = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) tmax[f] = fmaxf(tmax[f], sc[f][kt][rr]);
      move |= tmax[f] * scale > m[f] + 8.f;
    }
    if (__builtin_amdgcn_ballot_w64(move)) {
#pragma unroll
      for (int f = 0; f < QF; ++f) {
        const float ts = max_groups(tmax[f]) * scale;
        const float mn = ts > m[f] + 8.f ? ts : m[f];
        const float alpha = mn == m[f] ? 1.f : __builtin_amdgcn_exp2f(m[f] - mn);
        l[f] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[f][dt] *= alpha;
        m[f] = mn;
      }
    }
    bf16x8_t pf[QF][S2], rest[QF][S2];  // the probabilities as bfloat16, and what that leaves
#pragma unroll
    for (int f = 0; f < QF; ++f) {
      const float mr = -finite_ref(m[f]);
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const float pv1 = __builtin_amdgcn_exp2f(fmaf(sc[f][kt][rr], scale, mr));
          l[f] += pv1;
          sc[f][kt][rr] = pv1;
          if constexpr (E4) {
            const float w = pv1 * scale_of((vsr[kt] >> (8 * rr)) & 255u);
            sc[f][kt][rr] = whole || !dead(f, kt, rr) ? w : 0.f;  // the scale of an unused slot may be infinite
          }
        }
#pragma unroll
      for (int s2 = 0; s2 < S2; ++s2) {
        const f32x4_t &x = sc[f][2 * s2], &y = sc[f][2 * s2 + 1];
        const uint4 w = make_uint4(f2bf2(x[0], x[1]), f2bf2(x[2], x[3]), f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
        auto left = [](uint32_t two, float p0, float p1) {
          return f2bf2(p0 - __uint_as_float(two << 16), p1 - __uint_as_float(two & 0xFFFF0000u));
        };
        pf[f][s2] = __builtin_bit_cast(bf16x8_t, w);
        rest[f][s2] = __builtin_bit_cast(bf16x8_t, make_uint4(left(w.x, x[0], x[1]), left(w.y, x[2], x[3]),
                                                              left(w.z, y[0], y[1]), left(w.w, y[2], y[3])));
      }
    }
    // Values. In a tile that some row does not see whole, a probability of 0 must meet no infinity or NaN: what lies in
    // a slot past the last key becomes 0, and a key that only some rows see gives infinities and NaN to just those.
    if (!whole) {
      const int nv = pid_v < 0 ? 0 : kend - k0;  // the lane group's keys that are there
      uint32_t odd = 0;
      words_t keep;
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        const int bits = E4 ? 8 * (nv - 4 * j) : 16 * (nv - 2 * j);
        keep[j] = bits >= 32 ? ~0u : bits <= 0 ? 0u : (1u << bits) - 1u;
      }
      // Each group of registers is changed as one and pinned as one (the empty assembly): changed word by word, this
      // compiler gave the product registers of other words (ROCm 7.2, two fragments, bfloat16).
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        vr[dt] &= keep;
        asm volatile("" : "+v"(vr[dt]));
#pragma unroll
        for (int j = 0; j < VW; ++j)
          odd |= E4 ? ((vr[dt][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u
                    : ((vr[dt][j] & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u;
      }
      if (__builtin_amdgcn_ballot_w64(odd != 0)) {
        // rare, and written for few registers: such values leave the product and are added key by key, from the page
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          words_t m;
#pragma unroll
          for (int j = 0; j < VW; ++j)
            m[j] = E4 ? ((((vr[dt][j] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xFFu
                      : ((((vr[dt][j] & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u) >> 15) * 0xFFFFu;
          vr[dt] &= ~m;
          asm volatile("" : "+v"(vr[dt]));
        }
#pragma unroll 1
        for (int y = 0; y < KT; ++y) {
          const int key = KT * t + y, pid = page_at(t, y / PK);
          if (pid < 0 || key >= kend) continue;
          const uint8_t* at = p.v + (size_t)pid * page_bytes + head_bytes + ((size_t)4 * lg * plen + (key & (plen - 1))) * ES;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
              const uint8_t* e = at + (size_t)(16 * dt + rr) * plen * ES;
              const uint32_t v = E4 ? ((*e & 0x7Fu) == 0x7Fu ? 0x7FC00000u : 0u) : (uint32_t)*reinterpret_cast<const uint16_t*>(e) << 16;
              if ((v & 0x7F800000u) != 0x7F800000u) continue;
#pragma unroll
              for (int f = 0; f < QF; ++f)
                if (key < lim[f]) o[f][dt][rr] += __uint_as_float(v);
            }
        }
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int s2 = 0; s2 < S2; ++s2) {
        const bf16x8_t vf = value_fragment(dt, s2);
#pragma unroll
        for (int f = 0; f < QF; ++f) {
          o[f][dt] = mfma16p(vf, pf[f][s2], o[f][dt]);
          o[f][dt] = mfma16p(vf, rest[f][s2], o[f][dt]);
        }
      }
    if (t + 4 < t1) load_values(t + 4, pv);
  }

  // the waves' (m, l, o) joined in wave order, query fragment by query fragment
#pragma unroll
  for (int f = 0; f < QF; ++f) {
    if (f) __syncthreads();
    l[f] = sum_groups(l[f]);
    if (wid > 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) xo[wid - 1][dt][lane] = o[f][dt];
      xml[wid - 1][lane] = make_float2(m[f], l[f]);
    }
    __syncthreads();
    if (wid > 0) continue;
    float mm = m[f];
#pragma unroll
    for (int w = 0; w < 3; ++w) mm = fmaxf(mm, xml[w][lane].x);
    const float ref = finite_ref(mm), e0 = __builtin_amdgcn_exp2f(m[f] - ref);
    float lt = l[f] * e0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[f][dt] *= e0;
#pragma unroll
    for (int w = 0; w < 3; ++w) {
      const float2 ml = xml[w][lane];
      if (ml.x == -INFINITY && ml.y == 0.f) continue;  // a wave without keys
      const float e = __builtin_amdgcn_exp2f(ml.x - ref);
      lt += ml.y * e;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[f][dt] += xo[w][dt][lane] * e;
    }
    const int rr = row0 + 16 * f + lq;
    if (rr >= rows) continue;
    const size_t at = (size_t)(r.first + rr / a.g) * a.H + h * a.g + rr % a.g;
    if (a.nsplit > 1) {  // uniform: the join reads all of them
      float* dst = a.po + ((size_t)part * p.T * a.H + at) * DH + 4 * lg;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(dst + 16 * dt) = o[f][dt];
      if (lg == 0) a.pml[(size_t)part * p.T * a.H + at] = make_float2(mm, lt);
    } else {
      const float inv = lt == 0.f ? 0.f : 1.0f / lt;  // a row without keys is zeros
      bf16_t* dst = a.out + at * DH + 4 * lg;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
        *reinterpret_cast<uint2*>(dst + 16 * dt) =
            make_uint2(f2bf2(o[f][dt][0] * inv, o[f][dt][1] * inv), f2bf2(o[f][dt][2] * inv, o[f][dt][3] * inv));
      if (a.lse && lg == 0) a.lse[at] = lt == 0.f ? -INFINITY : mm * 0.6931471805599453f + logf(lt);
    }
  }
}

// The parts of a (row, head) joined: DH / 4 lanes take its dimensions, G such groups every G-th part, then the groups' sums
// in order. One group (and 8 or 16 (row, head)s a workgroup) is enough for up to 16 parts; 128 parts of 131072 keys took
// 100 us so, a load after the other, and take 5 us with all of a workgroup's groups on one row.
template <int DH, bool WIDE>
__global__ void __launch_bounds__(256) pages_join_kernel(PagesAttn a, int head_blocks) {
  constexpr int L = DH / 4, PER = 256 / L, G = WIDE ? PER : 1;
  __shared__ float4 xo[PER][L];
  __shared__ float xl[PER];
  const Pages& p = a.p;
  const int hb = blockIdx.x % head_blocks, bi = blockIdx.x / head_blocks, i = bi % p.max_new, b = bi / p.max_new;
  const SeqRows r = seq_rows(p.cu, b, p.T);
  const int grp = threadIdx.x / L, c = threadIdx.x % L, head = WIDE ? hb : hb * PER + grp;
  if (i >= r.n) return;
  const bool mine = head < a.H;  // uniform over the workgroup where groups meet
  const int kend = min(seq_len(p.len, b), p.max_pages << p.shift);
  const int parts = !mine ? 0 : kend == 0 ? 1 : (kend + a.span - 1) / a.span;
  const size_t at = (size_t)(r.first + i) * a.H + head, step = (size_t)p.T * a.H;
  float mm = -INFINITY;
  for (int s = c; s < parts; s += L) mm = fmaxf(mm, a.pml[s * step + at].x);
#pragma unroll
  for (int x = L / 2; x >= 1; x >>= 1) mm = fmaxf(mm, __shfl_xor(mm, x, 64));
  const float ref = finite_ref(mm);
  float lt = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float4& s, const float4& x, float e) {
    s.x += x.x * e;
    s.y += x.y * e;
    s.z += x.z * e;
    s.w += x.w * e;
  };
#pragma unroll 4
  for (int s = WIDE ? grp : 0; s < parts; s += G) {
    const float2 ml = a.pml[s * step + at];
    const float4 x = *reinterpret_cast<const float4*>(a.po + (s * step + at) * DH + 4 * c);
    // a part without keys that the row sees: (-inf, 0), and zeros for an output
    const float e = __builtin_amdgcn_exp2f(ml.x - ref);
    lt += ml.y * e;
    add(o, x, e);
  }
  if constexpr (WIDE) {
    xo[grp][c] = o;
    if (c == 0) xl[grp] = lt;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int s = 1; s < PER; ++s) {
      lt += xl[s];
      add(o, xo[s][c], 1.f);
    }
  }
  if (!mine) return;
  const float inv = lt == 0.f ? 0.f : 1.0f / lt;
  *reinterpret_cast<uint2*>(a.out + at * DH + 4 * c) = make_uint2(f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv));
  if (a.lse && c == 0) a.lse[at] = lt == 0.f ? -INFINITY : mm * 0.6931471805599453f + logf(lt);
}

// Query fragments (16 rows each) per wave. With two, two workgroups share a CU; four read a KV head's bfloat16 cache once for
// 64 rows, which pays where the rows are more and the workgroups of two would not all have a CU of their own. us with 1 / 2 /
// 4 over 1280 keys, three sets of operands in turn: 28 / 4 heads, bfloat16: 8 x 64 tokens (224 workgroups of four) 76 / 43 /
// 33, 5 x 64 (140) - / 43 / 33, 8 x 32 (128) 49 / 25 / 32, 8 x 16 (64) 29 / 25 / 32. 8-bit rows are bound by their conversions,
// for which one workgroup a CU is too few: 8 x 64 tokens x 32 / 32 heads 44 / 37 / 49, 28 / 4 heads - / 32 / 45, over 6000 keys
// - / 127 / 158.
static int query_fragments(int Hkv, int g, int B, int max_new, int e4m3) {
  const long rows = (long)g * max_new;
  return rows <= 16 ? 1 : e4m3 || rows <= 64 || (rows + 63) / 64 * Hkv * B <= 128 ? 2 : 4;
}

// Keys of a part: about 2048 workgroups if every sequence filled its row of the table (fewer leave CUs idle and the longest
// sequence's parts last; more spend their time on their first loads: one token of 64 sequences of 200 to 8000, 2048 / 4096 /
// 8192 workgroups 81 / 85 / 90 us), at most 128 parts. A part's output costs 8 bytes an element of memory traffic: at most
// a sixteenth of the part's keys and values, unless there are too few workgroups for that to matter. Up to 768 keys under one
// fragment stay whole: a join costs more than three parts save (4 x 1 token, 32 heads, 500 / 700 bfloat16 keys: 14.4 / 15.9 us in
// parts of 256, 12.3 / 14.2 whole; 32 / 8 heads, 8 bits: 12.7 / 12.8 and 12.0 / 12.3).
int pages_attention_span(int Hkv, int g, int B, int max_new, int capacity, int e4m3) {
  const int qf = query_fragments(Hkv, g, B, max_new, e4m3);
  const long rows = (long)g * max_new, units = ((rows + 16 * qf - 1) / (16 * qf)) * Hkv * B;
  if (qf == 1 && capacity <= 768) return (capacity + 63) / 64 * 64;
  const long tile = rows < 16 * qf ? rows : 16 * qf, cheap = 64 * tile / (e4m3 ? 1 : 2);
  long span = ((long)capacity * units + 2047) / 2048;
  if (span < cheap && units * ((capacity + span - 1) / span) > 256) span = cheap;
  if (span < 256) span = 256;
  long parts = (capacity + span / 2) / span;
  parts = parts < 1 ? 1 : parts > 128 ? 128 : parts;
  return (int)(((capacity + parts - 1) / parts + 63) / 64 * 64);
}

template <int DH, bool E4>
static void run_pages_attention(PagesAttn& a, hipStream_t s) {
  const int qf = query_fragments(a.p.Hkv, a.g, a.p.B, a.p.max_new, E4);
  a.row_tiles = (int)(((long)a.g * a.p.max_new + 16 * qf - 1) / (16 * qf));
  const long items = (long)a.nsplit * a.p.B * a.p.Hkv;
  const dim3 grid((unsigned)((items + 7) / 8 * 8 * a.row_tiles));
  if (qf == 1) hipLaunchKernelGGL((pages_attn_kernel<DH, E4, 1>), grid, dim3(256), 0, s, a);
  else if (E4 || qf == 2) hipLaunchKernelGGL((pages_attn_kernel<DH, E4, 2>), grid, dim3(256), 0, s, a);
  else if constexpr (!E4) hipLaunchKernelGGL((pages_attn_kernel<DH, false, 4>), grid, dim3(256), 0, s, a);
  if (a.nsplit > 1) {
    const bool wide = a.nsplit > 16;
    const int blocks = wide ? a.H : (a.H + 1024 / DH - 1) / (1024 / DH);
    const dim3 all((unsigned)blocks * a.p.max_new * a.p.B);
    if (wide) hipLaunchKernelGGL((pages_join_kernel<DH, true>), all, dim3(256), 0, s, a, blocks);
    else hipLaunchKernelGGL((pages_join_kernel<DH, false>), all, dim3(256), 0, s, a, blocks);
  }
}

void launch_pages_attention(PagesAttn a, hipStream_t s) {  // T and max_new above 0
  if (a.p.dh == 128) a.p.e4m3 ? run_pages_attention<128, true>(a, s) : run_pages_attention<128, false>(a, s);
  else a.p.e4m3 ? run_pages_attention<64, true>(a, s) : run_pages_attention<64, false>(a, s);
}

}  // namespace dcl
