// AdamW over many tensors, moments in 32 or 8 bits, gradients in fp32 or bf16.
//
// Moments of 8 bits. 256 neighbouring elements share an fp32 scale, the largest
// magnitude among them. m keeps q = sqrt of its share of it in 127ths, v the fourth
// root of its in 255ths: roots spread the codes over 1.6e4 : 1 of m and 4e9 : 1 of
// v (6.5e4 : 1 of its root, which the step divides by), with steps of 1.6 % at the
// top, where a format with three bits of mantissa has 12 %. A decoded moment is an
// integer's square times a scale; the code of a value is the floor of a root, and one
// more with a probability that keeps the mean.
// (The codes are a matter of borders: every operation on the way to them is rounded
// once, in the order written here, so that the same state gives the same codes
// whatever computes it. The roots are the hardware's, one step of the last bit off at
// most: at a border the code below has probability 2^-17 or less of being taken,
// which no drawn number reaches.)
#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

constexpr int kBlock = 256;             // elements that share a scale
constexpr float kTiny = 0x1p-94f;       // blocks below are kept as zeros (255^4 / kTiny is finite)

__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xE699D49Du;
  x = (x ^ (x >> 15)) * 0xC570DA33u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float decode_m(int q, float unit) {
  return (float)(q * abs(q)) * unit;
}
__device__ __forceinline__ float decode_v(int q, float scale) {
#pragma clang fp contract(off)
  const float c = (float)(q * q) * (1.0f / 65025.0f);
  return (c * c) * scale;
}
// Code of |m|: a = |m| / scale * 127^2 lies between q^2 and (q + 1)^2.
__device__ __forceinline__ int encode_m(float m, float inv, float u) {
#pragma clang fp contract(off)
  const float a = fabsf(m) * inv;
  const float q = floorf(__builtin_amdgcn_sqrtf(a));
  const float up = u * (2.0f * q + 1.0f) < a - q * q ? 1.0f : 0.0f;
  const int c = (int)fminf(q + up, 127.0f);
  return m < 0.0f ? -c : c;
}
// Code of v: x = v / scale * 255^4 lies between q^4 and (q + 1)^4.
__device__ __forceinline__ int encode_v(float v, float inv, float u) {
#pragma clang fp contract(off)
  const float x = v * inv;
  const float q = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(x)));
  const float lo2 = q * q, hi2 = (q + 1.0f) * (q + 1.0f);
  const float lo = lo2 * lo2, hi = hi2 * hi2;
  const float up = u * (hi - lo) < x - lo ? 1.0f : 0.0f;
  const float c = fminf(fmaxf(q + up, 1.0f), 255.0f);
  return x > 0.0f ? (int)c : 0;
}

__device__ __forceinline__ float grad_at(const void* g, int64_t i, bool bf16) {
  return bf16 ? bf2f(static_cast<const bf16_t*>(g)[i]) : static_cast<const float*>(g)[i];
}

// Moments in 32 bits: a thread an element.
__global__ __launch_bounds__(256) void adamw_multi_32_k(AdamTensor t, AdamHyper h, bool bf16) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= t.n) return;
  float p = t.master[i], m = static_cast<float*>(t.m)[i], v = static_cast<float*>(t.v)[i];
  adam1(p, m, v, grad_at(t.grad, i, bf16), h.b1, h.b2, h.eps, h.wd * t.decay_scale,
        h.sc[0] * t.lr_scale, 1.0f / h.sc[1], 1.0f / h.sc[2], h.sc[3]);
  t.master[i] = p;
  static_cast<float*>(t.m)[i] = m;
  static_cast<float*>(t.v)[i] = v;
  t.param[i] = f2bf(p);
}

// Moments in 8 bits: a wave a block of 256, four neighbours to a lane.
__global__ __launch_bounds__(256) void adamw_multi_8_k(AdamTensor t, AdamHyper h, bool bf16) {
#pragma clang fp contract(off)
  const int lane = threadIdx.x & 63;
  const int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t i0 = b * kBlock + lane * 4;
  if (b * kBlock >= t.n) return;
  const float lr = h.sc[0] * t.lr_scale, ibc1 = 1.0f / h.sc[1], ibc2 = 1.0f / h.sc[2];
  const float unit_m = t.m_scale[b] * (1.0f / 16129.0f), sv = t.v_scale[b];
  const uint32_t key = h.seed ? mixed(mixed((uint32_t)*h.seed) + t.index) : 0;
  float m[4], v[4];
  float top_m = 0.0f, top_v = 0.0f;
  bool bad = false;
  for (int e = 0; e < 4; ++e) {
    m[e] = v[e] = 0.0f;
    const int64_t i = i0 + e;
    if (i >= t.n) continue;
    const float g = grad_at(t.grad, i, bf16) * h.sc[3];
    m[e] = decode_m(static_cast<int8_t*>(t.m)[i], unit_m) * h.b1 + (1.0f - h.b1) * g;
    v[e] = decode_v(static_cast<uint8_t*>(t.v)[i], sv) * h.b2 + ((1.0f - h.b2) * g) * g;
    bad = bad || !(fabsf(m[e]) < INFINITY) || !(v[e] < INFINITY);
    top_m = fmaxf(top_m, fabsf(m[e]));
    top_v = fmaxf(top_v, v[e]);
    const float p = t.master[i];
    const float upd = __builtin_fmaf(h.wd * t.decay_scale, p,
                                     (m[e] * ibc1) / (sqrtf(v[e] * ibc2) + h.eps));
    const float q = __builtin_fmaf(-lr, upd, p);
    t.master[i] = q;
    t.param[i] = f2bf(q);
  }
  top_m = wave_max(top_m);
  top_v = wave_max(top_v);
  bad = __any(bad);
  const float inv_m = top_m < kTiny ? 0.0f : 16129.0f * (1.0f / top_m);
  const float inv_v = top_v < kTiny ? 0.0f : 4228250625.0f * (1.0f / top_v);
  for (int e = 0; e < 4; ++e) {
    const int64_t i = i0 + e;
    if (i >= t.n) continue;
    const uint32_t r = mixed((uint32_t)i ^ key);
    const float um = h.seed ? ((float)(r & 0xFFFF) + 0.5f) * 0x1p-16f : 0.5f;
    const float uv = h.seed ? ((float)(r >> 16) + 0.5f) * 0x1p-16f : 0.5f;
    static_cast<int8_t*>(t.m)[i] = (int8_t)(bad ? 0 : encode_m(m[e], inv_m, um));
    static_cast<uint8_t*>(t.v)[i] = (uint8_t)(bad ? 0 : encode_v(v[e], inv_v, uv));
  }
  if (lane == 0) {
    t.m_scale[b] = bad ? NAN : top_m < kTiny ? 0.0f : top_m;
    t.v_scale[b] = bad ? NAN : top_v < kTiny ? 0.0f : top_v;
  }
}

// A thread an element's values.
__global__ __launch_bounds__(256) void adamw_multi_read_k(AdamTensor t, bool bf16) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= t.n) return;
  const auto put = [&](void* out, float x) {
    if (bf16) static_cast<bf16_t*>(out)[i] = f2bf(x);
    else static_cast<float*>(out)[i] = x;
  };
  if (t.m_out)
    put(t.m_out,
        decode_m(static_cast<int8_t*>(t.m)[i], t.m_scale[i / kBlock] * (1.0f / 16129.0f)));
  if (t.v_out) put(t.v_out, decode_v(static_cast<uint8_t*>(t.v)[i], t.v_scale[i / kBlock]));
}

}  // namespace

hipError_t adamw_multi(const AdamTensor* t, int n, int bits, bool grad_bf16, const AdamHyper& h,
                       hipStream_t s) {
  for (int i = 0; i < n; ++i) {
    if (bits == 32) {
      hipLaunchKernelGGL(adamw_multi_32_k, dim3((unsigned)((t[i].n + 255) / 256)), dim3(256), 0, s,
                         t[i], h, grad_bf16);
    } else {
      hipLaunchKernelGGL(adamw_multi_8_k, dim3((unsigned)((t[i].n + 1023) / 1024)), dim3(256), 0,
                         s, t[i], h, grad_bf16);
    }
  }
  return hipGetLastError();
}

hipError_t adamw_multi_read(const AdamTensor* t, int n, bool out_bf16, hipStream_t s) {
  for (int i = 0; i < n; ++i)
    hipLaunchKernelGGL(adamw_multi_read_k, dim3((unsigned)((t[i].n + 255) / 256)), dim3(256), 0, s,
                       t[i], out_bf16);
  return hipGetLastError();
}

}  // namespace forge
