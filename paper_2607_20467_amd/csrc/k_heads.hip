// Each head's RMSNorm and rotate-half RoPE, queries and keys in one pass.
#include "dcl_internal.h"

namespace dcl {

// dh / 8 lanes hold a head, so that a wave takes 64 / (dh / 8) heads of a row at a time. A lane has both dimensions of its four
// pairs, 4 c .. and r / 2 + 4 c .. (behind the rotated ones, eight that follow each other): nothing is exchanged but the sum
// of squares, and a wave, which stays with its row, works each angle out once for all of its heads.
//
// The angle: pos * turns[i] in float64, below 2^31 / (2 pi) < 2^29 turns. Two roundings, of the turns a position (half a step 2^-56 and
// less, 2^31 times) and of the product (half a step of 2^-24), leave 2^-24 of a turn at the farthest position; as float32 in [-0.5, 0.5]
// the fraction keeps 2^-26.
//
// Memory-bound for many rows: 8192 of 32 + 8 heads of 128, 168 MB: 31 us, 5.4 TB/s (with pairs in different lanes, which an exchange
// brings together, 43 to 74: its twelve LDS-crossbar instructions a head group and twice the angles). Four rows: 3.5 us, a chain of
// position, angle, head.
//
// Gains and angles meet before the heads do: with x and z a pair's elements times 1 / sqrt(mean + eps), the outputs are
// x (g_x cos) - z (g_z sin) and z (g_z cos) + x (g_x sin).

// Sum over the L lanes (8 or 16, aligned) of a head, by exchanges inside a row of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float plus_lane(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int L>
__device__ __forceinline__ float sum_head(float v) {
  v = plus_lane<0xB1>(v);                          // quads 1 0 3 2
  v = plus_lane<0x4E>(v);                          // quads 2 3 0 1
  v = plus_lane<0x141>(v);                         // lane 7 - i of eight
  return L == 16 ? plus_lane<0x140>(v) : v;        // lane 15 - i of sixteen
}

// Read once: past the caches, so that they keep what is written (8192 rows 36.5 us with plain loads, 31.1 so, 32.1 with the stores past
// them too).
__device__ __forceinline__ uint2 load_once(const bf16_t* p) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(p)));
}

template <int DH>
__global__ void __launch_bounds__(256) heads_kernel(HeadsArgs a, int groups_q, int groups, int per) {
  constexpr int L = DH / 8, HW = 64 / L;  // lanes of a head, heads of a wave
  const int lane = threadIdx.x & 63, c = lane % L, sub = lane / L;
  const int t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (t >= a.T) return;
  const int pos = a.pos[t];
  if (pos < 0) return;
  const bool turned = c < a.rot / 8;
  const int dx = turned ? 4 * c : a.rot + 8 * (c - a.rot / 8), dz = turned ? a.rot / 2 + 4 * c : dx + 4;
  float cs[4], sn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (turned) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double turns = (double)pos * a.turns[dx + e];
      sincospif(2.0f * (float)(turns - rint(turns)), &sn[e], &cs[e]);
    }
  }
  // groups of HW heads: those of the queries, then those of the keys
  auto some = [&](const bf16_t* in, bf16_t* out, int heads, const float* gain, int g0, int g1) {
    if (g0 >= g1) return;
    float gx[4], gz[4], xs[4], zs[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) gx[e] = gz[e] = 1.f;
    if (gain) {
      const float4 p = *reinterpret_cast<const float4*>(gain + dx), q = *reinterpret_cast<const float4*>(gain + dz);
      gx[0] = p.x, gx[1] = p.y, gx[2] = p.z, gx[3] = p.w;
      gz[0] = q.x, gz[1] = q.y, gz[2] = q.z, gz[3] = q.w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      xs[e] = gx[e] * sn[e];
      zs[e] = gz[e] * sn[e];
      gx[e] *= cs[e];
      gz[e] *= cs[e];
    }
    for (int g = g0; g < g1; ++g) {
      const int h = g * HW + sub;
      if (h >= heads) continue;  // a head's lanes together
      const bf16_t* src = in + (size_t)h * DH;
      const uint2 ux = load_once(src + dx), uz = load_once(src + dz);
      float x[4] = {__uint_as_float(ux.x << 16), __uint_as_float(ux.x & 0xFFFF0000u), __uint_as_float(ux.y << 16),
                    __uint_as_float(ux.y & 0xFFFF0000u)};
      float z[4] = {__uint_as_float(uz.x << 16), __uint_as_float(uz.x & 0xFFFF0000u), __uint_as_float(uz.y << 16),
                    __uint_as_float(uz.y & 0xFFFF0000u)};
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) ss = fmaf(x[e], x[e], fmaf(z[e], z[e], ss));
        const float inv = rsqrtf(sum_head<L>(ss) * (1.0f / DH) + a.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] *= inv;
          z[e] *= inv;
        }
      }
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[e] = fmaf(x[e], gx[e], -(z[e] * zs[e]));
        y[4 + e] = fmaf(z[e], gz[e], x[e] * xs[e]);
      }
      if (!turned) {  // an infinity of the one is nothing to the other
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = x[e] * gx[e];
          y[4 + e] = z[e] * gz[e];
        }
      }
      bf16_t* dst = out + (size_t)h * DH;
      *reinterpret_cast<uint2*>(dst + dx) = make_uint2(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]));
      *reinterpret_cast<uint2*>(dst + dz) = make_uint2(f2bf2(y[4], y[5]), f2bf2(y[6], y[7]));
    }
  };
  const int g0 = blockIdx.y * per, g1 = min(g0 + per, groups);
  some(a.q + t * a.q_stride, a.q_out + t * a.q_out_stride, a.H, a.g_q, g0, min(g1, groups_q));
  some(a.k + t * a.k_stride, a.k_out + t * a.k_out_stride, a.Hkv, a.g_k, max(g0, groups_q) - groups_q, g1 - groups_q);
}

void launch_heads_norm_rope(const HeadsArgs& a, hipStream_t s) {  // T above 0
  const int HW = 512 / a.dh, gq = (a.H + HW - 1) / HW, groups = gq + (a.Hkv + HW - 1) / HW;
  // A wave per group of heads while that leaves CUs idle, otherwise about 16384 of them, that share a row evenly (8192 rows of ten
  // groups, waves at most 4096 / 8192 / 16384 / 32768: 32.2 / 32.3 / 31.1 / 32.0 us).
  const long waves = (long)a.T * groups;
  int chunks = (int)(waves <= 16384 ? groups : 16384 / a.T);
  chunks = chunks < 1 ? 1 : chunks;
  const int per = (groups + chunks - 1) / chunks;
  const dim3 grid((unsigned)((a.T + 3) / 4), (unsigned)((groups + per - 1) / per));
  if (a.dh == 128) hipLaunchKernelGGL((heads_kernel<128>), grid, dim3(256), 0, s, a, gq, groups, per);
  else hipLaunchKernelGGL((heads_kernel<64>), grid, dim3(256), 0, s, a, gq, groups, per);
}

}  // namespace dcl
