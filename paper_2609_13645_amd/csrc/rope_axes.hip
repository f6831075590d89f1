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

// One thread per (token, head, 8-pair chunk).
__global__ __launch_bounds__(256) void rope_axes_k(RopeAxes ax, const bf16_t* x, long ldx,
                                                   bf16_t* y, long ldy,
                                                   const float* __restrict__ cos_t,
                                                   const float* __restrict__ sin_t,
                                                   const int32_t* __restrict__ pos, int T, int rows,
                                                   int nrot, int d, float sign) {
  const int half = d / 2, cpr = half / 8;
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  if (id >= (long)T * nrot * cpr) return;
  const int c = (int)(id % cpr);
  const long th = id / cpr;
  const int hd = (int)(th % nrot);
  const long t = th / nrot;
  const uint32_t axes = ax.axis[c >> 1] >> ((c & 1) * 16);   // two bits a pair
  float cs[8], sn[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int a = (axes >> (2 * e)) & 3;
    const int p = min(max(pos[(long)a * T + t], 0), rows - 1);
    cs[e] = cos_t[(long)p * half + c * 8 + e];
    sn[e] = sin_t[(long)p * half + c * 8 + e] * sign;
  }
  const long col = (long)hd * d + c * 8;
  float x1[8], x2[8], y1[8], y2[8];
  unpack8(*reinterpret_cast<const uint4*>(x + t * ldx + col), x1);
  unpack8(*reinterpret_cast<const uint4*>(x + t * ldx + col + half), x2);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y1[e] = x1[e] * cs[e] - x2[e] * sn[e];
    y2[e] = x2[e] * cs[e] + x1[e] * sn[e];
  }
  *reinterpret_cast<uint4*>(y + t * ldy + col) = pack8(y1);
  *reinterpret_cast<uint4*>(y + t * ldy + col + half) = pack8(y2);
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
  const long n = (long)T * nrot * (d / 16);
  hipLaunchKernelGGL(rope_axes_k, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, ax, x, ldx,
                     y, ldy, cos_t, sin_t, pos, T, rows, nrot, d, inverse ? -1.0f : 1.0f);
  return hipGetLastError();
}

}  // namespace forge
