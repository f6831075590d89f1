// Rotary positions with several axes (time, height, width of image and video
// tokens): pair i = (x_i, x_{i + d/2}) of a head belongs to one axis, and its
// angle is that axis' position of the token times the pair's frequency. The
// tables hold cos and sin of every (position, pair), so the frequencies are
// theirs alone and the rotation only picks, per pair, the row of its axis.
#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

__global__ __launch_bounds__(256) void rope_axes_table_k(RopeFreqs f, int rows, int half,
                                                         float* __restrict__ cos_t,
                                                         float* __restrict__ sin_t) {
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  if (id >= (long)rows * half) return;
  const int p = (int)(id / half), i = (int)(id % half);
  // far positions: the angle in fp64, rounded once after cos and sin
  const double ang = (double)p * f.w[i];
  cos_t[id] = (float)cos(ang);
  sin_t[id] = (float)sin(ang);
}

// One thread per (token, head, eight pairs), lanes in that order from the pairs up: a
// wave reads and writes whole heads, and a token's cos and sin come from the caches
// for all its heads. WHOLE: no chunk of eight pairs is shared by axes, and its cos and
// sin are 16-byte loads from one row. Else the workgroup first collects its tokens'
// cos and sin in LDS, a lane to a pair (as eight loads each of a thread's own pairs,
// 4095 tokens x 24 heads of 128 took 15.0 us, now 12.6; a chunk to an axis 12.2).
// Bound by HBM: 16384 x 40 heads of 128, 61 us for 336 MB (5.5 TB/s). Threads that
// keep a chunk's cos and sin for 2, 4 or 8 heads are no faster (61.5, 63.4, 65.9).
// (tokens that 256 threads touch, of d / 16 threads a token and more: at most
// 256 / (d / 16) + 2, with d / 2 pairs each)
constexpr int kTableFloats = 8 * (256 + 2 * kRopeMaxPairs / 8);
template <bool WHOLE>
__global__ __launch_bounds__(256) void rope_axes_k(RopeAxes ax, const bf16_t* x, long ldx,
                                                   bf16_t* y, long ldy,
                                                   const float* __restrict__ cos_t,
                                                   const float* __restrict__ sin_t,
                                                   const int32_t* __restrict__ pos, uint32_t T,
                                                   int rows, uint32_t nrot, uint32_t d,
                                                   float sign) {
  const uint32_t half = d / 2, cpr = half / 8;
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t c = id % cpr, th = id / cpr, hd = th % nrot, t = th / nrot;
  const float4 *cp, *sp;
  if constexpr (WHOLE) {
    if (t >= T) return;
    const uint32_t a = (ax.axis[c >> 1] >> ((c & 1) * 16)) & 3;   // two bits a pair
    const int p = min(max(pos[(size_t)a * T + t], 0), rows - 1);
    cp = reinterpret_cast<const float4*>(cos_t + (size_t)p * half + c * 8);
    sp = reinterpret_cast<const float4*>(sin_t + (size_t)p * half + c * 8);
  } else {
    __shared__ __attribute__((aligned(16))) float tab[2][kTableFloats];
    const uint32_t t0 = blockIdx.x * 256u / cpr / nrot;
    const uint32_t t1 = min((blockIdx.x * 256u + 255u) / cpr / nrot, T - 1);
    for (uint32_t k = threadIdx.x; k < (t1 - t0 + 1) * half; k += 256) {
      const uint32_t i = k % half, tk = t0 + k / half;
      const uint32_t a = (ax.axis[i >> 4] >> (2 * (i & 15))) & 3;
      const int p = min(max(pos[(size_t)a * T + tk], 0), rows - 1);
      tab[0][k] = cos_t[(size_t)p * half + i];
      tab[1][k] = sin_t[(size_t)p * half + i];
    }
    __syncthreads();
    if (t >= T) return;
    cp = reinterpret_cast<const float4*>(&tab[0][(t - t0) * half + c * 8]);
    sp = reinterpret_cast<const float4*>(&tab[1][(t - t0) * half + c * 8]);
  }
  const float4 c0 = cp[0], c1 = cp[1], s0 = sp[0], s1 = sp[1];
  const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
  const float sn[8] = {s0.x * sign, s0.y * sign, s0.z * sign, s0.w * sign,
                       s1.x * sign, s1.y * sign, s1.z * sign, s1.w * sign};
  const bf16_t* xr = x + (size_t)t * ldx + (size_t)hd * d + c * 8;
  bf16_t* yr = y + (size_t)t * ldy + (size_t)hd * d + c * 8;
  float x1[8], x2[8], y1[8], y2[8];
  unpack8(*reinterpret_cast<const uint4*>(xr), x1);
  unpack8(*reinterpret_cast<const uint4*>(xr + half), x2);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y1[e] = x1[e] * cs[e] - x2[e] * sn[e];
    y2[e] = x2[e] * cs[e] + x1[e] * sn[e];
  }
  *reinterpret_cast<uint4*>(yr) = pack8(y1);
  *reinterpret_cast<uint4*>(yr + half) = pack8(y2);
}

}  // namespace

hipError_t rope_axes_table(const RopeFreqs& f, int rows, int d, float* cos_t, float* sin_t,
                           hipStream_t s) {
  const long n = (long)rows * (d / 2);
  hipLaunchKernelGGL(rope_axes_table_k, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, f,
                     rows, d / 2, cos_t, sin_t);
  return hipGetLastError();
}

hipError_t rope_axes(const RopeAxes& ax, const uint16_t* x, long ldx, uint16_t* y, long ldy,
                     const float* cos_t, const float* sin_t, const int32_t* pos, int T, int rows,
                     int nrot, int d, bool inverse, hipStream_t s) {
  bool whole = true;
  for (int i = 0; i < d / 2; ++i) whole = whole && ax.at(i) == ax.at(i / 8 * 8);
  const long n = (long)T * nrot * (d / 16);
  const dim3 grid((unsigned)((n + 255) / 256)), block(256);
  const float sign = inverse ? -1.0f : 1.0f;
  hipLaunchKernelGGL((whole ? rope_axes_k<true> : rope_axes_k<false>), grid, block, 0, s, ax, x,
                     ldx, y, ldy, cos_t, sin_t, pos, (uint32_t)T, rows, (uint32_t)nrot,
                     (uint32_t)d, sign);
  return hipGetLastError();
}

}  // namespace forge
