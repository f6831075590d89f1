// Rotary positions on a part of each head: r pairs of its columns, in halves
// (i, i + r) or interleaved (2i, 2i + 1), turned by amplitude * rotation of the
// token's position times the pair's frequency, the rest passed through. How the
// frequencies are scaled for a longer context is the tables' alone.
#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

__global__ __launch_bounds__(256) void rope_part_table_k(RopeFreqs f, float amplitude, int rows,
                                                         int half, float* __restrict__ cos_t,
                                                         float* __restrict__ sin_t) {
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  if (id >= (long)rows * half) return;
  const int p = (int)(id / half), i = (int)(id % half);
  // far positions: the angle in fp64, rounded once after cos and sin
  const double ang = (double)p * f.w[i];
  cos_t[id] = (float)(amplitude * cos(ang));
  sin_t[id] = (float)(amplitude * sin(ang));
}

// One pair turned: explicit multiply-adds, so that every form of the kernel has the
// same roundings (and those of forge_rope_apply).
__device__ __forceinline__ void turn(float x1, float x2, float c, float s, float& y1, float& y2) {
#pragma clang fp contract(off)
  y1 = __builtin_fmaf(x1, c, -(x2 * s));
  y2 = __builtin_fmaf(x2, c, x1 * s);
}

// One thread per (token, head, pair), and behind a head's pairs one per passed
// column (none in place).
__global__ __launch_bounds__(256) void rope_part_k(RopePart a) {
  const uint32_t half = a.rot / 2;
  const uint32_t per_head = half + (a.copy ? a.d - a.rot : 0);
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t u = id % per_head, th = id / per_head, hd = th % a.nrot, t = th / a.nrot;
  if (t >= a.T) return;
  const bf16_t* xr = a.x + (size_t)t * a.ldx + (size_t)hd * a.d;
  bf16_t* yr = a.y + (size_t)t * a.ldy + (size_t)hd * a.d;
  if (u >= half) {
    const uint32_t c = u - half < a.offset ? u - half : u - half + a.rot;
    yr[c] = xr[c];
    return;
  }
  const int p = a.pos ? min(max(a.pos[t], 0), a.rows - 1) : (int)(t % (uint32_t)a.rows);
  const float c = a.cos_t[(size_t)p * half + u], s = a.sin_t[(size_t)p * half + u] * a.sign;
  const uint32_t i = a.offset + (a.interleaved ? 2 * u : u), j = i + (a.interleaved ? 1 : half);
  float y1, y2;
  turn(bf2f(xr[i]), bf2f(xr[j]), c, s, y1, y2);
  yr[i] = f2bf(y1);
  yr[j] = f2bf(y2);
}

}  // namespace

hipError_t rope_part_table(const RopeFreqs& f, float amplitude, int rows, int half, float* cos_t,
                           float* sin_t, hipStream_t s) {
  const long n = (long)rows * half;
  hipLaunchKernelGGL(rope_part_table_k, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, f,
                     amplitude, rows, half, cos_t, sin_t);
  return hipGetLastError();
}

hipError_t rope_part(const RopePart& a, hipStream_t s) {
  const long n = (long)a.T * a.nrot * (a.rot / 2 + (a.copy ? a.d - a.rot : 0));
  hipLaunchKernelGGL(rope_part_k, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace forge
