// LayerNorm over rows, forward and backward: HBM-bound kernels.
//
// Forward: m = mean(x), v = mean((x - m)^2), r = (v + eps)^(-1/2), xh = (x - m) r,
// y = xh g + b. The row stays in registers between the two sums, so the variance
// is that of the centred values (no difference of two large sums) and x is read
// once. All sums are fp32.
// Backward, with u = g dy: dx = r (u - mean(u) - xh mean(u xh)) (+ resid),
// dg = sum_rows dy xh, db = sum_rows dy. One pass over x, dy (and resid): each
// lane keeps its columns' shares of dg and db in registers over all rows of its
// workgroup; the workgroups' sums are added by a second kernel in a fixed order
// (no atomics, so the gradients repeat bit for bit).
#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

// One wave per row, MAXCH 16-byte chunks per lane.
template <int MAXCH>
__global__ __launch_bounds__(256) void layernorm_fwd_k(const bf16_t* __restrict__ x,
                                                       const bf16_t* __restrict__ g,
                                                       const bf16_t* __restrict__ b,
                                                       bf16_t* __restrict__ y,
                                                       float* __restrict__ mean,
                                                       float* __restrict__ rstd, int T, int h,
                                                       float eps) {
  const int lane = threadIdx.x & 63;
  const long row = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= T) return;
  const int nch = h / 8;
  const uint4* xr = reinterpret_cast<const uint4*>(x + row * h);
  float f[MAXCH][8];
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < MAXCH; ++i) {
    const int c = lane + i * 64;
    if (c < nch) {
      unpack8(xr[c], f[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += f[i][e];
    }
  }
  const float m = wave_sum(s) / (float)h;
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < MAXCH; ++i) {
    if (lane + i * 64 < nch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[i][e] -= m;
        ss += f[i][e] * f[i][e];
      }
    }
  }
  const float r = 1.0f / sqrtf(wave_sum(ss) / (float)h + eps);
  if (lane == 0) {
    mean[row] = m;
    rstd[row] = r;
  }
  uint4* yr = reinterpret_cast<uint4*>(y + row * h);
  const uint4* gr = reinterpret_cast<const uint4*>(g);
  const uint4* br = reinterpret_cast<const uint4*>(b);
#pragma unroll
  for (int i = 0; i < MAXCH; ++i) {
    const int c = lane + i * 64;
    if (c < nch) {
      float w[8], a[8] = {};
      unpack8(gr[c], w);
      if (br) unpack8(br[c], a);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[i][e] = __builtin_fmaf(f[i][e] * r, w[e], a[e]);
      yr[c] = pack8(f[i]);
    }
  }
}

// One wave per row, rows strided over the waves of the grid; the workgroup's
// gain and bias sums go to part [gridDim.x][2][h].
constexpr int kBwdWaves = 4, kBwdMaxBlocks = 512;

template <int MAXCH>
__global__ __launch_bounds__(64 * kBwdWaves) void layernorm_bwd_k(
    const bf16_t* __restrict__ x, const bf16_t* __restrict__ g, const float* __restrict__ mean,
    const float* __restrict__ rstd, const bf16_t* __restrict__ dy,
    const bf16_t* __restrict__ resid, bf16_t* __restrict__ dx, float* __restrict__ part, int T,
    int h) {
  __shared__ float red[kBwdWaves][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nch = h / 8;
  const uint4* gr = reinterpret_cast<const uint4*>(g);
  float dga[MAXCH][8], dba[MAXCH][8];
#pragma unroll
  for (int i = 0; i < MAXCH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) dga[i][e] = dba[i][e] = 0.0f;

  for (long row = (long)blockIdx.x * kBwdWaves + wave; row < T;
       row += (long)gridDim.x * kBwdWaves) {
    const uint4* xr = reinterpret_cast<const uint4*>(x + row * h);
    const uint4* dyr = reinterpret_cast<const uint4*>(dy + row * h);
    const uint4* rr = resid ? reinterpret_cast<const uint4*>(resid + row * h) : nullptr;
    const float m = mean[row], r = rstd[row];
    uint4 xv[MAXCH], dv[MAXCH];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < MAXCH; ++i) {
      const int c = lane + i * 64;
      if (c < nch) {
        xv[i] = xr[c];
        dv[i] = dyr[c];
        float xf[8], df[8], w[8];
        unpack8(xv[i], xf);
        unpack8(dv[i], df);
        unpack8(gr[c], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float xh = (xf[e] - m) * r, u = w[e] * df[e];
          s1 += u;
          s2 += u * xh;
          dga[i][e] += df[e] * xh;
          dba[i][e] += df[e];
        }
      }
    }
    const float c1 = wave_sum(s1) / (float)h, c2 = wave_sum(s2) / (float)h;
    uint4* dxr = reinterpret_cast<uint4*>(dx + row * h);
#pragma unroll
    for (int i = 0; i < MAXCH; ++i) {
      const int c = lane + i * 64;
      if (c < nch) {
        float xf[8], df[8], w[8], o[8];
        unpack8(xv[i], xf);
        unpack8(dv[i], df);
        unpack8(gr[c], w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = r * (w[e] * df[e] - c1 - (xf[e] - m) * r * c2);
        if (rr) {
          float rf[8];
          unpack8(rr[c], rf);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += rf[e];
        }
        dxr[c] = pack8(o);
      }
    }
  }
  float* pg = part + (long)blockIdx.x * 2 * h;
#pragma unroll
  for (int i = 0; i < MAXCH; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int e = 0; e < 8; ++e) red[wave][lane * 8 + e] = k ? dba[i][e] : dga[i][e];
      __syncthreads();
      for (int j = threadIdx.x; j < 512; j += 64 * kBwdWaves) {
        if (i * 512 + j < h) {
          float s = 0.0f;
#pragma unroll
          for (int w = 0; w < kBwdWaves; ++w) s += red[w][j];
          pg[k * h + i * 512 + j] = s;
        }
      }
      __syncthreads();
    }
}

// dg[c] (and db[c], grid.y 1) = or += the sum over the workgroups' partial rows:
// 64 columns per workgroup, 16 stripes of 16-byte loads, stripe sums added in order.
template <bool ACC>
__global__ __launch_bounds__(256) void layernorm_grad_sum_k(const float* __restrict__ part,
                                                            int nblk, float* __restrict__ dg,
                                                            float* __restrict__ db, int h) {
  __shared__ float4 red[16][16];
  const int cg = threadIdx.x & 15, stripe = threadIdx.x >> 4;
  const int col = blockIdx.x * 64 + cg * 4;
  const float* src = part + (long)blockIdx.y * h;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (col < h) {
#pragma unroll 8
    for (int b = stripe; b < nblk; b += 16) {
      const float4 v = *reinterpret_cast<const float4*>(src + (long)b * 2 * h + col);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  }
  red[stripe][cg] = s;
  __syncthreads();
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x < 64 && c < h) {
    const float* rf = reinterpret_cast<const float*>(red);
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += rf[w * 64 + threadIdx.x];
    float* out = blockIdx.y ? db : dg;
    out[c] = ACC ? out[c] + t : t;
  }
}

}  // namespace

hipError_t layernorm_fwd(const uint16_t* x, const uint16_t* g, const uint16_t* b, uint16_t* y,
                         float* mean, float* rstd, int T, int h, float eps, hipStream_t s) {
  const dim3 grid((unsigned)(((long)T + 3) / 4)), block(256);
  const int ch = (h / 8 + 63) / 64;
#define FORGE_LNF(N) \
  hipLaunchKernelGGL(layernorm_fwd_k<N>, grid, block, 0, s, x, g, b, y, mean, rstd, T, h, eps)
  if (ch <= 1) FORGE_LNF(1);
  else if (ch <= 2) FORGE_LNF(2);
  else if (ch <= 4) FORGE_LNF(4);
  else if (ch <= 8) FORGE_LNF(8);
  else if (ch <= 16) FORGE_LNF(16);
  else return hipErrorInvalidValue;
#undef FORGE_LNF
  return hipGetLastError();
}

int layernorm_bwd_blocks(int T, int h) {
  const long need = ((long)T + kBwdWaves - 1) / kBwdWaves;
  return need < kBwdMaxBlocks ? (int)need : kBwdMaxBlocks;
}

hipError_t layernorm_bwd(const uint16_t* x, const uint16_t* g, const float* mean,
                         const float* rstd, const uint16_t* dy, const uint16_t* resid,
                         uint16_t* dx, float* dg, float* db, bool accumulate, float* part, int T,
                         int h, hipStream_t s) {
  const int nblk = T > 0 ? layernorm_bwd_blocks(T, h) : 0;
  if (nblk > 0) {
    const dim3 grid(nblk), block(64 * kBwdWaves);
    const int ch = (h / 8 + 63) / 64;
#define FORGE_LNB(N)                                                                       \
  hipLaunchKernelGGL(layernorm_bwd_k<N>, grid, block, 0, s, x, g, mean, rstd, dy, resid, dx, \
                     part, T, h)
    if (ch <= 1) FORGE_LNB(1);
    else if (ch <= 2) FORGE_LNB(2);
    else if (ch <= 4) FORGE_LNB(4);
    else if (ch <= 8) FORGE_LNB(8);
    else if (ch <= 16) FORGE_LNB(16);
    else return hipErrorInvalidValue;
#undef FORGE_LNB
  }
  const dim3 sgrid((h + 63) / 64, db ? 2 : 1);
  if (accumulate)
    hipLaunchKernelGGL(layernorm_grad_sum_k<true>, sgrid, dim3(256), 0, s, part, nblk, dg, db, h);
  else
    hipLaunchKernelGGL(layernorm_grad_sum_k<false>, sgrid, dim3(256), 0, s, part, nblk, dg, db, h);
  return hipGetLastError();
}

}  // namespace forge
