// Attention over whole prompts: packed sequences of different lengths, causal or bidirectional, grouped heads.
//
// o_i = sum_j softmax_j(scale q_i.k_j) v_j with one running maximum and sum per query and the score tile in registers.
// One workgroup takes 128 queries of one head, a wave 32 of them; keys and values pass through LDS in tiles of 64, two
// stages, copied there directly (global_load_lds). The scores are S^T = K Q^T (32 x 32 tiles), so that a lane holds 32
// of the 64 scores of one query and its probabilities feed O^T = V^T P^T as they are; the values, which lie with the
// dimension innermost, reach that product's lanes through the transposing LDS read (ds_read_b64_tr_b16: of 16 lanes'
// 8 bytes, four rows of 16 elements, lane i gets column i). Both tiles are XOR-swizzled in 16-byte chunks so that the
// rows that one read touches lie in different banks.
//
// The probabilities are rounded to bfloat16 once, 2^-8 of each at most; the sum that divides takes them unrounded. That rounding
// is about as large as the output's own: the error against 64 bits is 1.9e-3 to 2.1e-3 where the output alone gives 1.6e-3. A
// second part for what it leaves, as the attention over pages has, takes that away and costs half as many matrix
// instructions again, here where they bound: 8192 tokens 506 / 684 us, the eight prompts below 90 / 119.
//
// Bound by the matrix and vector pipes together: one causal prompt of 8192 tokens x 32 heads of 128 takes 506 to 533 us, 1.03 to
// 1.09 PFLOP/s of the 1.21 that a large matrix product reaches (520 to 620 each where nothing but such calls runs, at the clock
// that the power leaves). Eight prompts of 78 to 1531 tokens, 28 / 4 heads: 90 us, 0.59 PFLOP/s: the two tiles on the diagonal
// are half masked, and a workgroup of seven tiles starts and ends three times as often as it would in the long prompt.
// Bidirectional, 32 heads: 8 prompts of 512 tokens 67 us, of 1024 190, one of 4096 263 (1.04 PFLOP/s).
#include <type_traits>

#include "dcl_internal.h"
#include "pages_index.h"

namespace dcl {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16_t mfma32(const bf16x8_t& a, const bf16x8_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint2 read_transposed(const uint8_t* lds) {
  typedef __attribute__((address_space(3))) s16x4_t lds_vec;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)(lds)));
}
template <int N>
__device__ __forceinline__ void prompt_wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
// A wave-uniform address in scalar registers.
__device__ __forceinline__ const bf16_t* prompt_uniform(const bf16_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const bf16_t*>(((uint64_t)hi << 32) | lo);
}

constexpr int kPromptQ = 128, kPromptK = 64;  // queries and keys of a tile

template <int DH>
__global__ void __launch_bounds__(256, 2) prompt_attn_kernel(PromptAttn a) {
  constexpr int KT = kPromptK, KC = DH / 8, CH = KT * KC, NL = CH / 256;  // chunks per row, per tile, copies per wave
  constexpr int STAGE = 2 * CH * 16;                                      // bytes: keys, then values
  __shared__ __attribute__((aligned(1024))) uint8_t sm[2 * STAGE];
  // (sequence, head) pairs go round the XCDs: a head's query tiles share one L2, every sequence spreads over all of
  // them; the tiles with the most keys come first
  const int heads = a.B * a.H, j = blockIdx.x >> 3;
  const int hx = (heads + 7) / 8, bh = (blockIdx.x & 7) + 8 * (j % hx), qt = a.q_tiles - 1 - j / hx;
  if (bh >= heads) return;
  const int b = __builtin_amdgcn_readfirstlane(bh / a.H), h = __builtin_amdgcn_readfirstlane(bh % a.H), g = h / (a.H / a.Hkv);
  const SeqRows r = seq_rows(a.cu, b, a.T);
  const int n = r.n, q0 = qt * kPromptQ;
  if (q0 >= min(n, a.max_len)) return;
  const int tid = threadIdx.x, lane = tid & 63, wid = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, hi = lane >> 5;
  const int qw = q0 + 32 * wid, query = qw + lq;
  const int lim = a.causal ? min(n, query + 1) : n;       // keys that the lane's query sees
  const int nkeys = a.causal ? min(n, q0 + kPromptQ) : n;  // that the workgroup's queries see
  const int wopen = a.causal ? min(n, qw + 1) : n;        // that all of the wave's queries see
  const int wkeys = qw >= n ? 0 : a.causal ? min(n, qw + 32) : n;
  const int tiles = (nkeys + KT - 1) / KT;

  const bf16_t* kbase = a.k + (size_t)r.first * a.k_stride + (size_t)g * DH;
  const bf16_t* vbase = a.v + (size_t)r.first * a.v_stride + (size_t)g * DH;

  // copy i of wave w fills the 64 chunks from (i * 4 + w) * 64: slot c of row y holds chunk c ^ f(y). A tile that lies
  // whole in the sequence is a scalar base plus a per-lane offset that never changes.
  auto key_swizzle = [](int y) { return DH == 128 ? y & 15 : (y >> 1) & 7; };
  auto value_swizzle = [](int y) { return DH == 128 ? (y & 3) << 2 : ((y >> 1) & 1) << 2; };
  auto slot_row = [&](int i) { return ((i * 4 + wid) * 64 + lane) / KC; };
  auto key_chunk = [&](int i) { return 8 * ((lane % KC) ^ key_swizzle(slot_row(i))); };
  auto value_chunk = [&](int i) { return 8 * ((lane % KC) ^ value_swizzle(slot_row(i))); };
  uint32_t koff[NL], voff[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    koff[i] = ((uint32_t)slot_row(i) * (uint32_t)a.k_stride + (uint32_t)key_chunk(i)) * 2u;
    voff[i] = ((uint32_t)slot_row(i) * (uint32_t)a.v_stride + (uint32_t)value_chunk(i)) * 2u;
  }
  const bool near = a.k_stride <= (1 << 24) && a.v_stride <= (1 << 24);  // a tile's offsets stay in 32 bits
  const uint32_t lds = lds_addr_of(sm) + (uint32_t)wid * 1024u;
  auto issue = [&](int t, uint32_t stage) {
    const uint32_t dst = lds + stage;
    const int k0 = t * KT;
    if (near && k0 + KT <= n) {
      const bf16_t* kb = prompt_uniform(kbase + (size_t)k0 * a.k_stride);
      const bf16_t* vb = prompt_uniform(vbase + (size_t)k0 * a.v_stride);
#pragma unroll
      for (int i = 0; i < NL; ++i) dma16_sv(kb, koff[i], dst + i * 4096u);
#pragma unroll
      for (int i = 0; i < NL; ++i) dma16_sv(vb, voff[i], dst + CH * 16u + i * 4096u);
    } else {  // a row past the last key repeats that key: no query sees it there
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        const int y = min(k0 + slot_row(i), n - 1);
        dma16_at(kbase + (size_t)y * a.k_stride + key_chunk(i), dst + i * 4096u);
        dma16_at(vbase + (size_t)y * a.v_stride + value_chunk(i), dst + CH * 16u + i * 4096u);
      }
    }
  };
  issue(0, 0);  // first of all: the queries arrive beside it
  bf16x8_t qf[DH / 16];
  {
    const bf16_t* qp = a.q + (size_t)(r.first + min(query, n - 1)) * a.q_stride + (size_t)h * DH + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks) {
      uint4 x = *reinterpret_cast<const uint4*>(qp + 16 * ks);
      x.x ^= a.q_sign, x.y ^= a.q_sign, x.z ^= a.q_sign, x.w ^= a.q_sign;  // a negative scale is a sign of the query
      qf[ks] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  // where the lane's fragments lie in a stage (see the reads below)
  const int key_at = lq * KC * 16 + ((hi ^ key_swizzle(lq)) * 16);
  int value_at[DH / 32];
  {
    const int lr = (lane & 15) >> 2, piece = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), y = 4 * hi + lr;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) value_at[d] = CH * 16 + (y * KC + ((4 * d + piece) ^ value_swizzle(y))) * 16 + 8 * (lane & 1);
  }

  f32x16_t o[DH / 32];
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float scale = a.scale_log2;

  // Tile t in the stage at byte STG. `masked`: some query of the workgroup does not see all of it.
  auto step = [&](int t, auto stage_of, auto masked_of) {
    const int STG = stage_of;  // a constant where the tile is whole
    constexpr bool masked = decltype(masked_of)::value;
    prompt_wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < tiles) issue(t + 1, STAGE - STG);
    const int k0 = t * KT;
    if (masked && k0 >= wkeys) return;  // none of the wave's queries sees this tile
    const uint8_t* sv = sm + STG + CH * 16;

    // Keys: step ks takes chunk 2 ks + hi of row y at slot (2 ks + hi) ^ f(y), that is (hi ^ f(y)) ^ 2 ks.
    f32x16_t sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
#pragma unroll
    for (int ks = 0; ks < DH / 16; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const uint4 x = *reinterpret_cast<const uint4*>(sm + (key_at ^ (32 * ks)) + STG + kb * 32 * KC * 16);
        sc[kb] = mfma32(__builtin_bit_cast(bf16x8_t, x), qf[ks], sc[kb]);
      }
    // register i of step kb is key k0 + 32 kb + 8 (i / 4) + 4 hi + i % 4
    const bool cut = masked && k0 + KT > wopen;  // some query of the wave does not see all of the tile
    if (cut) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (k0 + 32 * kb + 8 * (i >> 2) + 4 * hi + (i & 3) >= lim) sc[kb][i] = -INFINITY;
    }
    // Values of 16 keys (step s) and 32 dimensions: lanes 0-15 / 16-31 take 16 dimensions each of keys 16 s + 0..3 and
    // + 8..11, lanes 32-63 the four keys after those, as the probabilities lie.
    auto value_fragment = [&](int s, int d) -> uint4 {
      const uint2 x = read_transposed(sm + value_at[d] + STG + s * 16 * KC * 16);
      const uint2 z = read_transposed(sm + value_at[d] + STG + (s * 16 + 8) * KC * 16);
      return make_uint4(x.x, x.y, z.x, z.y);
    };
    // the reference point (log2 units) moves only when a score passes it by more than 2^8
    float tmax = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, sc[kb][i]);
    if (__builtin_amdgcn_ballot_w64(tmax * scale > m + 8.f)) {
      const float ts = fmaxf(tmax, __shfl_xor(tmax, 32, 64)) * scale;
      const float mn = ts > m + 8.f ? ts : m;
      const float alpha = mn == m ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DH / 32; ++d) o[d] *= alpha;
      m = mn;
    }
    const float mr = m == -INFINITY ? 0.f : -m;
    bf16x8_t pf[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint32_t w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[s >> 1][8 * (s & 1) + 2 * x], scale, mr));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[s >> 1][8 * (s & 1) + 2 * x + 1], scale, mr));
        l += p0;
        l += p1;
        w[x] = f2bf2(p0, p1);
      }
      pf[s] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
    }
    bool odd_tile = false;
    if (cut) {  // an infinity or NaN in a value that only some of the queries see must meet no probability of 0
      uint32_t odd = 0;
#pragma unroll 4
      for (int c = lane; c < CH; c += 64) {
        const uint4 x = *reinterpret_cast<const uint4*>(sv + c * 16);
        odd |= (((x.x & 0x7FFF7FFFu) + 0x00800080u) | ((x.y & 0x7FFF7FFFu) + 0x00800080u) |
                ((x.z & 0x7FFF7FFFu) + 0x00800080u) | ((x.w & 0x7FFF7FFFu) + 0x00800080u)) & 0x80008000u;
      }
      odd_tile = __builtin_amdgcn_ballot_w64(odd != 0) != 0;
    }
    if (!masked || !odd_tile) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int d = 0; d < DH / 32; ++d) o[d] = mfma32(__builtin_bit_cast(bf16x8_t, value_fragment(s, d)), pf[s], o[d]);
    } else {
      // rare, and written for few registers: the product without such values, then they alone, key by key
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int d = 0; d < DH / 32; ++d) {
          __builtin_amdgcn_sched_barrier(0);
          uint4 x = value_fragment(s, d);
          uint32_t* w = &x.x;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] &= ((w[e] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w[e] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
          o[d] = mfma32(__builtin_bit_cast(bf16x8_t, x), pf[s], o[d]);
        }
#pragma unroll 1
      for (int y = 0; y < KT; ++y) {
        if (k0 + y >= lim) break;
#pragma unroll
        for (int d = 0; d < DH / 32; ++d)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint2 x = *reinterpret_cast<const uint2*>(sv + (y * KC + ((4 * d + c) ^ value_swizzle(y))) * 16 + 8 * hi);
            const uint32_t w[4] = {x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if ((w[e] & 0x7F800000u) == 0x7F800000u) o[d][4 * c + e] += __uint_as_float(w[e]);
          }
      }
    }
  };
  const int open = (a.causal ? min(n, q0 + 1) : n) / KT;  // tiles that every query of the workgroup sees whole
  int t = 0;
  for (; t + 1 < open; t += 2) {
    step(t, std::integral_constant<int, 0>(), std::false_type());
    step(t + 1, std::integral_constant<int, STAGE>(), std::false_type());
  }
  for (; t < tiles; ++t) step(t, (t & 1) * STAGE, std::true_type());

  const float lt = l + __shfl_xor(l, 32, 64);
  if (query >= min(n, a.max_len)) return;
  const float inv = lt == 0.f ? 0.f : 1.0f / lt;
  const size_t at = (size_t)(r.first + query) * a.H + h;
  bf16_t* dst = a.out + at * DH + 4 * hi;
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<uint2*>(dst + 32 * d + 8 * i) = make_uint2(f2bf2(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                                                                  f2bf2(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
  if (a.lse && hi == 0) a.lse[at] = lt == 0.f ? -INFINITY : m * 0.6931471805599453f + logf(lt);
}

void launch_prompt_attention(PromptAttn a, hipStream_t s) {
  const int most = a.max_len < a.T ? a.max_len : a.T;
  if (most == 0) return;
  a.q_tiles = (most + kPromptQ - 1) / kPromptQ;
  const dim3 grid((unsigned)((long)(a.B * (long)a.H + 7) / 8 * 8 * a.q_tiles));
  if (a.dh == 128) hipLaunchKernelGGL(prompt_attn_kernel<128>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(prompt_attn_kernel<64>, grid, dim3(256), 0, s, a);
}

}  // namespace dcl
