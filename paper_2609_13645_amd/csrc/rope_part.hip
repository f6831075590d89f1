// Rotary positions on a part of each head: r pairs of its columns, in halves
// (i, i + r) or interleaved (2i, 2i + 1), turned by amplitude * rotation of the
// token's position times the pair's frequency, the rest passed through. How the
// frequencies are scaled for a longer context is the tables' alone.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

// A thread takes kRows rows of a pair: the first row's angle in fp64 through sine and
// cosine, the next ones by turning it on by one position (four fp64 multiply-adds, each
// off by 2^-53: nothing of the fp32 that is kept). 32768 positions x 64 pairs, 16.8 MB:
// 6.6 us, as a sine and a cosine for each entry 15.8; with 8 or 4 rows 7.2 and 7.6.
constexpr int kRows = 16;
__global__ __launch_bounds__(256) void rope_part_table_k(RopeFreqs f, float amplitude, int rows,
                                                         int half, float* __restrict__ cos_t,
                                                         float* __restrict__ sin_t) {
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  const int i = (int)(id % half);
  const long p0 = id / half * kRows;
  if (p0 >= rows) return;
  const double w = f.w[i];
  double c, s, cw, sw;
  sincos((double)p0 * w, &s, &c);
  sincos(w, &sw, &cw);
#pragma unroll 4
  for (int r = 0; r < kRows; ++r) {
    if (p0 + r >= rows) return;
    cos_t[(p0 + r) * half + i] = (float)(amplitude * c);
    sin_t[(p0 + r) * half + i] = (float)(amplitude * s);
    const double x = c * cw - s * sw;
    s = s * cw + c * sw;
    c = x;
  }
}

// One pair turned: explicit multiply-adds, so that every form of the kernel has the
// same roundings (and those of forge_rope_apply).
__device__ __forceinline__ void turn(float x1, float x2, float c, float s, float& y1, float& y2) {
#pragma clang fp contract(off)
  y1 = __builtin_fmaf(x1, c, -(x2 * s));
  y2 = __builtin_fmaf(x2, c, x1 * s);
}

// N bf16 from p (aligned to their size) as floats, and back.
template <int N>
__device__ __forceinline__ void load_bf16(const bf16_t* p, float* f) {
  if constexpr (N == 8) {
    unpack8(*reinterpret_cast<const uint4*>(p), f);
  } else if constexpr (N == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    f[0] = lo_f(u.x); f[1] = hi_f(u.x); f[2] = lo_f(u.y); f[3] = hi_f(u.y);
  } else if constexpr (N == 2) {
    const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
    f[0] = lo_f(u); f[1] = hi_f(u);
  } else {
    f[0] = bf2f(*p);
  }
}
template <int N>
__device__ __forceinline__ void store_bf16(bf16_t* p, const float* f) {
  if constexpr (N == 8) *reinterpret_cast<uint4*>(p) = pack8(f);
  else if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
  else if constexpr (N == 2) *reinterpret_cast<uint32_t*>(p) = pack2(f[0], f[1]);
  else *p = f2bf(f[0]);
}
template <int N>
struct Bits;
template <> struct Bits<8> { typedef uint4 type; };
template <> struct Bits<4> { typedef uint2 type; };
template <> struct Bits<2> { typedef uint32_t type; };
template <> struct Bits<1> { typedef uint16_t type; };
template <int N>
__device__ __forceinline__ void load_f32(const float* p, float* f) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<float4*>(f + i) = *reinterpret_cast<const float4*>(p + i);
  } else if constexpr (N == 2) {
    *reinterpret_cast<float2*>(f) = *reinterpret_cast<const float2*>(p);
  } else {
    f[0] = p[0];
  }
}

// One thread per (token, head, V pairs), which also takes the C passed columns of its
// number (none in place): accesses as wide as the part's place in the head lets them be
// aligned. Bound by HBM: 16384 x 40 heads of 128, half of each interleaved, apart, 63 us
// for 336 MB (5.4 TB/s). With threads of their own for the passed columns 73, those two
// bytes at a time as the pairs 242; threads that take 2 or 4 tokens 72, 75.
template <int V, bool INTER>
constexpr uint32_t passed = INTER ? 2 * V : V;
template <int V, bool INTER>
__global__ __launch_bounds__(256) void rope_part_k(RopePart a) {
  constexpr uint32_t C = passed<V, INTER>;
  typedef typename Bits<C>::type B;
  const uint32_t half = a.rot / 2, units = half / V, copies = a.copy ? (a.d - a.rot) / C : 0;
  const uint32_t per_head = max(units, copies);
  const uint32_t id = blockIdx.x * 256u + threadIdx.x;
  const uint32_t u = id % per_head, th = id / per_head, hd = th % a.nrot, t = th / a.nrot;
  if (t >= a.T) return;
  const bf16_t* xr = a.x + (size_t)t * a.ldx + (size_t)hd * a.d;
  bf16_t* yr = a.y + (size_t)t * a.ldy + (size_t)hd * a.d;
  const uint32_t c0 = u * C, c = c0 < a.offset ? c0 : c0 + a.rot;
  B rest;
  if (u < copies) rest = *reinterpret_cast<const B*>(xr + c);
  if (u < units) {
    const int p = a.pos ? min(max(a.pos[t], 0), a.rows - 1) : (int)(t % (uint32_t)a.rows);
    float cs[V], sn[V], x[2 * V], y[2 * V];
    load_f32<V>(a.cos_t + (size_t)p * half + u * V, cs);
    load_f32<V>(a.sin_t + (size_t)p * half + u * V, sn);
    const uint32_t i = a.offset + c0, j = i + half;
    if constexpr (INTER) {
      load_bf16<2 * V>(xr + i, x);
#pragma unroll
      for (int e = 0; e < V; ++e)
        turn(x[2 * e], x[2 * e + 1], cs[e], sn[e] * a.sign, y[2 * e], y[2 * e + 1]);
      store_bf16<2 * V>(yr + i, y);
    } else {
      load_bf16<V>(xr + i, x);
      load_bf16<V>(xr + j, x + V);
#pragma unroll
      for (int e = 0; e < V; ++e)
        turn(x[e], x[V + e], cs[e], sn[e] * a.sign, y[e], y[V + e]);
      store_bf16<V>(yr + i, y);
      store_bf16<V>(yr + j, y + V);
    }
  }
  if (u < copies) *reinterpret_cast<B*>(yr + c) = rest;
}

}  // namespace

hipError_t rope_part_table(const RopeFreqs& f, float amplitude, int rows, int half, float* cos_t,
                           float* sin_t, hipStream_t s) {
  const long n = (rows + kRows - 1L) / kRows * half;
  hipLaunchKernelGGL(rope_part_table_k, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, f,
                     amplitude, rows, half, cos_t, sin_t);
  return hipGetLastError();
}

hipError_t rope_part(const RopePart& a, hipStream_t s) {
  // V divides what its accesses start at and the pairs; interleaved it also has to
  // divide the part's pairs as two columns each
  const uint32_t at = a.interleaved ? a.offset | a.rot : a.offset | a.rot / 2;
  const auto go = [&](auto v, auto inter) {
    constexpr int V = decltype(v)::value;
    constexpr bool I = decltype(inter)::value;
    const long copies = a.copy ? (a.d - a.rot) / passed<V, I> : 0;
    const long n = (long)a.T * a.nrot * std::max(a.rot / 2L / V, copies);
    hipLaunchKernelGGL((rope_part_k<V, I>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
    return hipGetLastError();
  };
  using std::integral_constant;
  if (a.interleaved) {
    if (at % 8 == 0) return go(integral_constant<int, 4>{}, std::true_type{});
    if (at % 4 == 0) return go(integral_constant<int, 2>{}, std::true_type{});
    return go(integral_constant<int, 1>{}, std::true_type{});
  }
  if (at % 8 == 0) return go(integral_constant<int, 8>{}, std::false_type{});
  if (at % 4 == 0) return go(integral_constant<int, 4>{}, std::false_type{});
  if (at % 2 == 0) return go(integral_constant<int, 2>{}, std::false_type{});
  return go(integral_constant<int, 1>{}, std::false_type{});
}

}  // namespace forge
