// Each head's RMSNorm and rotate-half RoPE, queries and keys in one pass.
#include "dcl_internal.h"

namespace dcl {

// dh / 8 lanes hold a head, eight dimensions each, so that a wave takes 64 / (dh / 8) heads of a row at a time; the squares are
// summed over those lanes, and the partner of a rotated dimension, r / 2 further, comes from the lane that holds it. A wave
// stays with its row, so that angles are worked out once for all of its heads.
//
// The angle: pos * turns[i] in float64 is exact to 2^-52 of itself, at most 2^31 / (2 pi) turns, so that its fraction is exact to
// 2^-23 of a turn at the farthest position and to 2^-24 below 2^28; as float32 in [-0.5, 0.5] it keeps 2^-25.
template <int DH>
__global__ void __launch_bounds__(256) heads_kernel(HeadsArgs a, int chunks, int per) {
  constexpr int L = DH / 8, HW = 64 / L;  // lanes of a head, heads of a wave
  const int lane = threadIdx.x & 63, c = lane % L, sub = lane / L;
  const long unit = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t = (int)(unit / chunks), chunk = (int)(unit % chunks);
  if (t >= a.T) return;
  const int pos = a.pos[t];
  if (pos < 0) return;
  const int half = a.rot / 2, d0 = 8 * c;
  const bool turned = d0 < a.rot, upper = d0 >= half;
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (turned) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double turns = (double)pos * a.turns[(upper ? d0 - half : d0) + e];
      sincospif(2.0f * (float)(turns - rint(turns)), &sn[e], &cs[e]);
      if (!upper) sn[e] = -sn[e];
    }
  }
  const int partner = turned ? sub * L + c + (upper ? -half / 8 : half / 8) : lane;
  const int total = a.H + a.Hkv, h1 = min((chunk + 1) * per * HW, total);
  for (int h0 = chunk * per * HW; h0 < h1; h0 += HW) {
    const int h = h0 + sub;
    const bool mine = h < h1, key = h >= a.H;
    const int hh = key ? h - a.H : h;
    const float* gain = key ? a.g_k : a.g_q;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (mine) w = *reinterpret_cast<const uint4*>((key ? a.k + t * a.k_stride : a.q + t * a.q_stride) + (size_t)hh * DH + d0);
    float x[8];
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
    for (int o = L / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
    if (mine && gain) {
      const float inv = 1.0f / sqrtf(ss * (1.0f / DH) + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * inv * gain[d0 + e];
    }
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = __shfl(x[e], partner, 64);
      y[e] = turned ? fmaf(other, sn[e], x[e] * cs[e]) : x[e];
    }
    if (mine)
      *reinterpret_cast<uint4*>((key ? a.k_out + t * a.k_out_stride : a.q_out + t * a.q_out_stride) + (size_t)hh * DH + d0) =
          make_uint4(f2bf2(y[0], y[1]), f2bf2(y[2], y[3]), f2bf2(y[4], y[5]), f2bf2(y[6], y[7]));
  }
}

void launch_heads_norm_rope(const HeadsArgs& a, hipStream_t s) {  // T above 0
  const int HW = 512 / a.dh, groups = (a.H + a.Hkv + HW - 1) / HW;
  // a wave per group of heads while that leaves CUs idle, otherwise a wave per row
  const long waves = (long)a.T * groups;
  int per = 1;
  while (per < groups && waves / (2 * per) >= 8192) per *= 2;
  const int chunks = (groups + per - 1) / per;
  const dim3 grid((unsigned)(((long)a.T * chunks + 3) / 4));
  if (a.dh == 128) hipLaunchKernelGGL((heads_kernel<128>), grid, dim3(256), 0, s, a, chunks, per);
  else hipLaunchKernelGGL((heads_kernel<64>), grid, dim3(256), 0, s, a, chunks, per);
}

}  // namespace dcl
