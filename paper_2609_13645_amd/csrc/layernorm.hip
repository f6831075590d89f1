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
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

// A row belongs to WPR waves with CH 16-byte chunks per lane. Bound by memory:
// 16384 x 4096 50 us for 268 MB (5.4 TB/s, above a large copy's 4.9: the memory-side
// cache has a part; with one wave to a row 60), 16384 x 2048 26.7 (28.9); few rows by
// the latency of a row: 64 x 4096 3.5 us (6.0), 1 x 8192 4.1 (8.3).
template <int CH, int WPR>
__global__ __launch_bounds__(256) void layernorm_fwd_k(const bf16_t* __restrict__ x,
                                                       const bf16_t* __restrict__ g,
                                                       const bf16_t* __restrict__ b,
                                                       bf16_t* __restrict__ y,
                                                       float* __restrict__ mean,
                                                       float* __restrict__ rstd, int T, int h,
                                                       float eps) {
  constexpr int RG = 4 / WPR, LANES = 64 * WPR;
  __shared__ float part[2][4];
  const int grp = threadIdx.x / LANES, col = threadIdx.x % LANES, wave = threadIdx.x >> 6;
  // sum over the row's waves, in order
  const auto row_sum = [&](float v, int k) {
    v = wave_sum(v);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) part[k][wave] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) v += part[k][grp * WPR + w];
    }
    return v;
  };
  // (grid.y: more rows than one dimension of a launch has threads for)
  const long row = ((long)blockIdx.y * gridDim.x + blockIdx.x) * RG + grp;
  const int nch = row < T ? h / 8 : 0;   // (no chunks past the last row)
  const uint4* xr = reinterpret_cast<const uint4*>(x + row * h);
  float f[CH][8];
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = col + i * LANES;
    if (c < nch) {
      unpack8(xr[c], f[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += f[i][e];
    }
  }
  const float m = row_sum(s, 0) / (float)h;
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (col + i * LANES < nch) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        f[i][e] -= m;
        ss += f[i][e] * f[i][e];
      }
    }
  }
  const float r = 1.0f / sqrtf(row_sum(ss, 1) / (float)h + eps);
  if (col == 0 && row < T) {
    mean[row] = m;
    rstd[row] = r;
  }
  uint4* yr = reinterpret_cast<uint4*>(y + row * h);
  const uint4* gr = reinterpret_cast<const uint4*>(g);
  const uint4* br = reinterpret_cast<const uint4*>(b);
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = col + i * LANES;
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

// A row belongs to WPR waves with CH chunks per lane, so that a row of any width
// keeps few registers (the columns' shares of dg and db, the row and the next one,
// whose loads are in flight while this one is reduced); a workgroup's NW / WPR row
// groups take rows grid-strided and end with their sums in part [gridDim.x][2][h].
// Bound by memory: 16384 x 4096, residual included, 102 us for 537 MB (5.3 TB/s; with a
// wave per row, whose 8 chunks a lane left one row's loads in flight, 233 us).
// Narrow rows come near the vector units, 13 operations an element (x r - m r as one
// fma, a 13th less, is no faster at any of 11 shapes and off by 2^-24 |m| r where x - m
// is exact: rows of one value, whose r is eps^(-1/2)).
template <int CH, int WPR, int NW>
__global__ __launch_bounds__(64 * NW) void layernorm_bwd_k(
    const bf16_t* __restrict__ x, const bf16_t* __restrict__ g, const float* __restrict__ mean,
    const float* __restrict__ rstd, const bf16_t* __restrict__ dy,
    const bf16_t* __restrict__ resid, bf16_t* __restrict__ dx, float* __restrict__ part, int T,
    int h, float* __restrict__ dg, float* __restrict__ db, bool accumulate) {
  constexpr int RG = NW / WPR, LANES = 64 * WPR;
  __shared__ float2 sums[2][NW];
  __shared__ float red[RG > 1 ? RG : 1][RG > 1 ? LANES * 8 : 1];
  const int grp = threadIdx.x / LANES, col = threadIdx.x % LANES;
  const int nch = h / 8;
  const float inv_h = 1.0f / (float)h;
  float w[CH][8], dga[CH][8], dba[CH][8];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = col + i * LANES;
    uint4 gv = make_uint4(0, 0, 0, 0);
    if (c < nch) gv = reinterpret_cast<const uint4*>(g)[c];
    unpack8(gv, w[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dga[i][e] = dba[i][e] = 0.0f;
  }
  struct Row {
    uint4 x[CH], dy[CH], res[CH];
    float m, r;
  };
  // (a row past the end, and chunks past the width, read as zeros)
  const auto load = [&](long row) {
    Row v;
    const bool ok = row < T;
    v.m = ok ? mean[row] : 0.0f;
    v.r = ok ? rstd[row] : 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = col + i * LANES;
      const bool in = ok && c < nch;
      v.x[i] = v.dy[i] = v.res[i] = make_uint4(0, 0, 0, 0);
      if (in) {
        v.x[i] = reinterpret_cast<const uint4*>(x + row * h)[c];
        v.dy[i] = reinterpret_cast<const uint4*>(dy + row * h)[c];
        if (resid) v.res[i] = reinterpret_cast<const uint4*>(resid + row * h)[c];
      }
    }
    return v;
  };
  const long step = (long)gridDim.x * RG;
  int buf = 0;
  long row = (long)blockIdx.x * RG + grp;
  Row v = load(row);
  // (every wave of a workgroup makes the same number of turns: the barriers)
  for (long base = (long)blockIdx.x * RG; base < T; base += step, row += step) {
    const Row next = load(row + step);
    float xh[CH][8], u[CH][8], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      float df[8];
      unpack8(v.x[i], xh[i]);
      unpack8(v.dy[i], df);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[i][e] = (xh[i][e] - v.m) * v.r;
        u[i][e] = w[i][e] * df[e];
        s1 += u[i][e];
        s2 = __builtin_fmaf(u[i][e], xh[i][e], s2);
        dga[i][e] = __builtin_fmaf(df[e], xh[i][e], dga[i][e]);
        dba[i][e] += df[e];
      }
    }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) sums[buf][threadIdx.x >> 6] = make_float2(s1, s2);
      __syncthreads();
      s1 = s2 = 0.0f;
#pragma unroll
      for (int k = 0; k < WPR; ++k) {
        const float2 t = sums[buf][grp * WPR + k];
        s1 += t.x;
        s2 += t.y;
      }
      buf ^= 1;
    }
    const float c1 = -s1 * inv_h * v.r, c2 = -s2 * inv_h * v.r;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = col + i * LANES;
      if (row < T && c < nch) {
        float o[8];
        unpack8(v.res[i], o);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = __builtin_fmaf(u[i][e], v.r, __builtin_fmaf(xh[i][e], c2, c1)) + o[e];
        reinterpret_cast<uint4*>(dx + row * h)[c] = pack8(o);
      }
    }
    v = next;
  }
  // (a workgroup alone: its sums are the gradients)
  const bool alone = gridDim.x == 1;
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float* out = !alone ? part + ((long)blockIdx.x * 2 + k) * h : k ? db : dg;
      float a[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = k ? dba[i][e] : dga[i][e];
      if constexpr (RG == 1) {
        const int c = col + i * LANES;
        if (c < nch && out) {
          float4* p = reinterpret_cast<float4*>(out + c * 8);
          float4 u = make_float4(a[0], a[1], a[2], a[3]), v = make_float4(a[4], a[5], a[6], a[7]);
          if (alone && accumulate) {
            const float4 s = p[0], t = p[1];
            u = make_float4(s.x + u.x, s.y + u.y, s.z + u.z, s.w + u.w);
            v = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
          }
          p[0] = u;
          p[1] = v;
        }
      } else {
        float4* p = reinterpret_cast<float4*>(&red[grp][col * 8]);
        p[0] = make_float4(a[0], a[1], a[2], a[3]);
        p[1] = make_float4(a[4], a[5], a[6], a[7]);
        __syncthreads();
        for (int j = threadIdx.x; j < LANES * 8; j += 64 * NW) {
          if (i * LANES * 8 + j < h && out) {
            float s = 0.0f;
#pragma unroll
            for (int q = 0; q < RG; ++q) s += red[q][j];
            if (alone && accumulate) s = out[i * LANES * 8 + j] + s;
            out[i * LANES * 8 + j] = s;
          }
        }
        __syncthreads();
      }
    }
}

// dg[c] (and db[c], grid.y 1) = or += the sum over the workgroups' partial rows:
// 64 columns per workgroup, 64 stripes of 16-byte loads, stripe sums added in order.
template <bool ACC>
__global__ __launch_bounds__(1024) void layernorm_grad_sum_k(const float* __restrict__ part,
                                                             int nblk, float* __restrict__ dg,
                                                             float* __restrict__ db, int h) {
  __shared__ float4 red[64][16];
  __shared__ float quarter[4][64];
  const int cg = threadIdx.x & 15, stripe = threadIdx.x >> 4;
  const int col = blockIdx.x * 64 + cg * 4;
  const float* src = part + (long)blockIdx.y * h;
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (col < h) {
#pragma unroll 8
    for (int b = stripe; b < nblk; b += 64) {
      const float4 v = *reinterpret_cast<const float4*>(src + (long)b * 2 * h + col);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  }
  red[stripe][cg] = s;
  __syncthreads();
  if (threadIdx.x < 256) {
    const int c = threadIdx.x & 63, q = threadIdx.x >> 6;
    const float* rf = reinterpret_cast<const float*>(&red[q * 16][0]);
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) t += rf[w * 64 + c];
    quarter[q][c] = t;
  }
  __syncthreads();
  const int c = blockIdx.x * 64 + threadIdx.x;
  if (threadIdx.x < 64 && c < h) {
    const float t = (quarter[0][threadIdx.x] + quarter[1][threadIdx.x]) +
                    (quarter[2][threadIdx.x] + quarter[3][threadIdx.x]);
    float* out = blockIdx.y ? db : dg;
    out[c] = ACC ? out[c] + t : t;
  }
}

}  // namespace

hipError_t layernorm_fwd(const uint16_t* x, const uint16_t* g, const uint16_t* b, uint16_t* y,
                         float* mean, float* rstd, int T, int h, float eps, hipStream_t s) {
  const auto grid = [&](int rows) {
    const long n = ((long)T + rows - 1) / rows, most = 1L << 23;
    return dim3((unsigned)std::min(n, most), (unsigned)((n + most - 1) / most));
  };
#define FORGE_LNF(CH, WPR)                                                              \
  hipLaunchKernelGGL((layernorm_fwd_k<CH, WPR>), grid(4 / WPR), dim3(256), 0, s, x, g, b, y, \
                     mean, rstd, T, h, eps)
  if (h <= 512) FORGE_LNF(1, 1);
  else if (h <= 1024) FORGE_LNF(2, 1);
  else if (h <= 2048) FORGE_LNF(2, 2);
  else if (h <= 4096) FORGE_LNF(2, 4);
  else if (h <= 8192) FORGE_LNF(4, 4);
  else return hipErrorInvalidValue;
#undef FORGE_LNF
  return hipGetLastError();
}

namespace {
// Eight waves a workgroup and one workgroup a CU: enough loads in flight for the
// HBM's rate, and no more partial rows to write and add than CUs (16384 x 4096 with
// resid: 192 workgroups 114 us, 256 103, 512 108; 999 x 2056: 256 12.5 us, 500 19).
constexpr int kBwdWaves = 8, kBwdMaxBlocks = 256;
// Waves of a row, two chunks of 512 columns each.
int row_waves(int h) { return h <= 1024 ? 1 : h <= 2048 ? 2 : h <= 4096 ? 4 : 8; }
}  // namespace

int layernorm_bwd_blocks(int T, int h) {
  const int groups = kBwdWaves / row_waves(h);
  // few rows: one workgroup, whose sums are the gradients, and no second launch, while its
  // turns take no longer than that (16 x 1024, two turns: 6.3 us, so 5.1; four: 6.3, 7.1)
  if (T <= 3 * groups) return 1;
  return (int)std::min(((long)T + groups - 1) / groups, (long)kBwdMaxBlocks);
}

hipError_t layernorm_bwd(const uint16_t* x, const uint16_t* g, const float* mean,
                         const float* rstd, const uint16_t* dy, const uint16_t* resid,
                         uint16_t* dx, float* dg, float* db, bool accumulate, float* part, int T,
                         int h, hipStream_t s) {
  const int nblk = T > 0 ? layernorm_bwd_blocks(T, h) : 0;
  if (nblk > 0) {
    const dim3 grid(nblk), block(64 * kBwdWaves);
#define FORGE_LNB(CH, WPR)                                                                     \
  hipLaunchKernelGGL((layernorm_bwd_k<CH, WPR, kBwdWaves>), grid, block, 0, s, x, g, mean, rstd, \
                     dy, resid, dx, part, T, h, dg, db, accumulate)
    if (h <= 512) FORGE_LNB(1, 1);
    else if (h <= 1024) FORGE_LNB(2, 1);
    else if (h <= 2048) FORGE_LNB(2, 2);
    else if (h <= 4096) FORGE_LNB(2, 4);
    else if (h <= 8192) FORGE_LNB(2, 8);
    else return hipErrorInvalidValue;
#undef FORGE_LNB
  }
  if (nblk == 1) return hipGetLastError();
  const dim3 sgrid((h + 63) / 64, db ? 2 : 1);
  if (accumulate)
    hipLaunchKernelGGL(layernorm_grad_sum_k<true>, sgrid, dim3(1024), 0, s, part, nblk, dg, db, h);
  else
    hipLaunchKernelGGL(layernorm_grad_sum_k<false>, sgrid, dim3(1024), 0, s, part, nblk, dg, db, h);
  return hipGetLastError();
}

}  // namespace forge
