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
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

constexpr int kBlock = 256;             // elements that share a scale
// Blocks below are kept as zeros (255^4 / kTiny is finite); eps, FORGE_ADAMW_MIN_EPS_8BIT at
// least, stands in for the roots of such a v.
constexpr float kTiny = 0x1p-94f;

// A permutation of 32 bits (odd multipliers, chosen by test: over 2^20 drawn x and over x below
// 2^20 each bit of x, flipped, flips each bit of the result in 0.497 to 0.503 of the cases).
__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xE699D49Du;
  x = (x ^ (x >> 15)) * 0xC570DA33u;
  return x ^ (x >> 16);
}

// (Multiply-adds below stand where the product is exact, so that they round once as the
// operations that they join.)
__device__ __forceinline__ float decode_m(int8_t code, float unit) {
#pragma clang fp contract(off)
  const float q = (float)code;
  return (q * fabsf(q)) * unit;
}
__device__ __forceinline__ float decode_v(uint8_t code, float scale) {
#pragma clang fp contract(off)
  const float q = (float)code, c = (q * q) * (1.0f / 65025.0f);
  return (c * c) * scale;
}
// Code of |m|: a = |m| / scale * 127^2 lies between q^2 and (q + 1)^2.
__device__ __forceinline__ int encode_m(float m, float inv, float u) {
#pragma clang fp contract(off)
  const float a = fabsf(m) * inv, q = floorf(__builtin_amdgcn_sqrtf(a));
  const bool up = u * __builtin_fmaf(2.0f, q, 1.0f) < __builtin_fmaf(-q, q, a);
  const int c = (int)fminf(q, up ? 126.0f : 127.0f) + up;
  return m < 0.0f ? -c : c;
}
// Code of v: x = v / scale * 255^4 lies between q^4 and (q + 1)^4. Above zero, also where x is
// too small for fp32, for a v > least (0; where the block is kept as zeros infinity).
__device__ __forceinline__ float encode_v(float v, float inv, float least, float u) {
#pragma clang fp contract(off)
  const float x = v * inv, q = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(x)));
  const float q1 = q + 1.0f, lo2 = q * q, hi2 = q1 * q1, lo = lo2 * lo2, hi = hi2 * hi2;
  const float c = u * (hi - lo) < x - lo ? q1 : q;
  return v > least ? __builtin_amdgcn_fmed3f(c, 1.0f, 255.0f) : 0.0f;
}

// Largest of the wave's 64 unsigned values, in every lane: the rows of 16 by shifted
// moves on the VALU, then across rows; lane 63 has it.
__device__ __forceinline__ uint32_t wave_top(uint32_t x) {
  const auto step = [&](auto ctrl) {
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF,
                                                             0xF, false);
    x = x > y ? x : y;
  };
  using std::integral_constant;
  step(integral_constant<int, 0x111>{});   // from 1, 2, 4, 8 lanes before, in the row
  step(integral_constant<int, 0x112>{});
  step(integral_constant<int, 0x114>{});
  step(integral_constant<int, 0x118>{});
  step(integral_constant<int, 0x142>{});   // the row before's last lane
  step(integral_constant<int, 0x143>{});   // lane 31
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

// The workgroup's tensor and its first element there.
__device__ __forceinline__ const AdamTensor& tensor_of(const AdamBatch& b, int64_t& first) {
  int i = 0;
#pragma unroll
  for (int step = 32; step; step /= 2)
    if (i + step <= kAdamBatch && (int)blockIdx.x >= b.end[min(i + step, kAdamBatch) - 1]) i += step;
  first = (int64_t)((int)blockIdx.x - (i ? b.end[i - 1] : 0)) * b.chunk;
  return b.t[i];
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// Four neighbours from element i on, as floats; those at or past n are zeros. Every buffer
// is read and written once in a step: nontemporal, as in the plain update.
template <typename T>
__device__ __forceinline__ T load_nt(const void* p, int64_t i) {
  return __builtin_nontemporal_load(reinterpret_cast<const T*>(static_cast<const char*>(p)) + i);
}
template <typename T>
__device__ __forceinline__ void store_nt(void* p, int64_t i, T x) {
  __builtin_nontemporal_store(x, reinterpret_cast<T*>(p) + i);
}
__device__ __forceinline__ f32x4_t load4(const float* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return load_nt<f32x4_t>(p, i / 4);
  f32x4_t x = {};
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x[e] = p[i + e];
  return x;
}
__device__ __forceinline__ void store4(float* p, int64_t i, int64_t n, f32x4_t x) {
  if (i + 4 <= n) return store_nt<f32x4_t>(p, i / 4, x);
  for (int e = 0; e < 4; ++e)
    if (i + e < n) p[i + e] = x[e];
}
// (bf16 and codes stay packed until they are used)
__device__ __forceinline__ u32x2_t load4(const bf16_t* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return load_nt<u32x2_t>(p, i / 4);
  u32x2_t x = {};
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x[e / 2] |= (uint32_t)p[i + e] << 16 * (e % 2);
  return x;
}
__device__ __forceinline__ void store4(bf16_t* p, int64_t i, int64_t n, f32x4_t f) {
  const u32x2_t x = {pack2(f[0], f[1]), pack2(f[2], f[3])};
  if (i + 4 <= n) return store_nt<u32x2_t>(p, i / 4, x);
  for (int e = 0; e < 4; ++e)
    if (i + e < n) p[i + e] = (bf16_t)(x[e / 2] >> 16 * (e % 2));
}
__device__ __forceinline__ uint32_t load4(const uint8_t* p, int64_t i, int64_t n) {
  if (i + 4 <= n) return load_nt<uint32_t>(p, i / 4);
  uint32_t x = 0;
  for (int e = 0; e < 4; ++e)
    if (i + e < n) x |= (uint32_t)p[i + e] << 8 * e;
  return x;
}
__device__ __forceinline__ void store4(uint8_t* p, int64_t i, int64_t n, uint32_t x) {
  if (i + 4 <= n) return store_nt<uint32_t>(p, i / 4, x);
  for (int e = 0; e < 4; ++e)
    if (i + e < n) p[i + e] = (uint8_t)(x >> 8 * e);
}
// Gradients of four neighbours.
template <bool BF16>
struct Grad;
template <>
struct Grad<false> {
  f32x4_t x;
  __device__ __forceinline__ Grad(const void* p, int64_t i, int64_t n)
      : x(load4(static_cast<const float*>(p), i, n)) {}
  __device__ __forceinline__ float operator[](int e) const { return x[e]; }
};
template <>
struct Grad<true> {
  u32x2_t x;
  __device__ __forceinline__ Grad(const void* p, int64_t i, int64_t n)
      : x(load4(static_cast<const bf16_t*>(p), i, n)) {}
  __device__ __forceinline__ float operator[](int e) const {
    return e % 2 ? hi_f(x[e / 2]) : lo_f(x[e / 2]);
  }
};

// Moments in 32 bits: four neighbours to a thread. 218 M parameters in five tensors: 1088 us,
// 6.0 TB/s; as four times four to a thread 1165.
template <bool BF16>
__global__ __launch_bounds__(256) void adamw_multi_32_k(AdamBatch b, AdamHyper h) {
  int64_t i;
  const AdamTensor& t = tensor_of(b, i);
  const float lr = h.sc[0] * t.lr_scale, ibc1 = 1.0f / h.sc[1], ibc2 = 1.0f / h.sc[2];
  const float clip = h.sc[3], wd = h.wd * t.decay_scale;
  i += threadIdx.x * 4;
  if (i >= t.n) return;
  f32x4_t p = load4(t.master, i, t.n), m = load4(static_cast<float*>(t.m), i, t.n);
  f32x4_t v = load4(static_cast<float*>(t.v), i, t.n);
  const Grad<BF16> g(t.grad, i, t.n);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float pe = p[e], me = m[e], ve = v[e];
    adam1(pe, me, ve, g[e], h.b1, h.b2, h.eps, wd, lr, ibc1, ibc2, clip);
    p[e] = pe;
    m[e] = me;
    v[e] = ve;
  }
  store4(t.master, i, t.n, p);
  store4(static_cast<float*>(t.m), i, t.n, m);
  store4(static_cast<float*>(t.v), i, t.n, v);
  store4(t.param, i, t.n, p);
}

// Moments in 8 bits: a wave a block of 256, four neighbours to a lane. 18 bytes a parameter
// move in the time of some 110 vector operations, and the codes take most of that: the
// update's root and quotient are the hardware's (off by the last bit or two; with IEEE's, and
// magnitudes and codes by selects, 218 M parameters took 824 us, now 660 to 680, 5.9 TB/s). A wave
// that takes four blocks one behind another, all loaded first: 678, and 4 M 18.3 us for 16.1.
template <bool BF16>
__global__ __launch_bounds__(256) void adamw_multi_8_k(AdamBatch bt, AdamHyper h) {
#pragma clang fp contract(off)
  int64_t i0;
  const AdamTensor& t = tensor_of(bt, i0);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n = t.n, b = i0 / kBlock + wave, i = b * kBlock + lane * 4;
  if (b * kBlock >= n) return;
  const float lr = h.sc[0] * t.lr_scale, ibc1 = 1.0f / h.sc[1], ibc2 = 1.0f / h.sc[2];
  const float clip = h.sc[3], wd = h.wd * t.decay_scale;
  const float c1 = 1.0f - h.b1, c2 = 1.0f - h.b2;
  // u = (16 bits + 1/2) / 2^16, or 1/2
  const uint32_t key = h.seed ? mixed(mixed((uint32_t)*h.seed) + t.index) : 0;
  const float u_step = h.seed ? 0x1p-16f : 0.0f, u_first = h.seed ? 0x1p-17f : 0.5f;
  f32x4_t p = load4(t.master, i, n);
  const Grad<BF16> g(t.grad, i, n);
  uint32_t qm = load4(static_cast<uint8_t*>(t.m), i, n);
  uint32_t qv = load4(static_cast<uint8_t*>(t.v), i, n);
  const float unit_m = t.m_scale[b] * (1.0f / 16129.0f), sv = t.v_scale[b];
  float m[4], v[4];
  uint32_t bits_m = 0, bits_v = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = g[e] * clip;
    m[e] = decode_m((int8_t)(qm >> 8 * e), unit_m) * h.b1 + c1 * x;
    v[e] = decode_v((uint8_t)(qv >> 8 * e), sv) * h.b2 + (c2 * x) * x;
    // (as integers the magnitudes order as they do, what is not finite above them)
    bits_m = max(bits_m, __builtin_bit_cast(uint32_t, m[e]) << 1);
    bits_v = max(bits_v, __builtin_bit_cast(uint32_t, v[e]) << 1);
    const float upd =
        (m[e] * ibc1) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[e] * ibc2) + h.eps);
    p[e] = __builtin_fmaf(-lr, __builtin_fmaf(wd, p[e], upd), p[e]);
  }
  store4(t.master, i, n, p);
  store4(t.param, i, n, p);
  bits_m = wave_top(bits_m);
  bits_v = wave_top(bits_v);
  const bool bad = max(bits_m, bits_v) >= 0xFF000000u;
  const float top_m = __builtin_bit_cast(float, bits_m >> 1);
  const float top_v = __builtin_bit_cast(float, bits_v >> 1);
  const float inv_m = top_m < kTiny ? 0.0f : 16129.0f * (1.0f / top_m);
  const float inv_v = top_v < kTiny ? 0.0f : 4228250625.0f * (1.0f / top_v);
  const float least_v = top_v < kTiny ? INFINITY : 0.0f;
  qm = qv = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t r = mixed((uint32_t)(i + e) ^ key);
    const float um = __builtin_fmaf((float)(r & 0xFFFF), u_step, u_first);
    const float uv = __builtin_fmaf((float)(r >> 16), u_step, u_first);
    qm |= (uint32_t)(encode_m(m[e], inv_m, um) & 255) << 8 * e;
    qv = __builtin_amdgcn_cvt_pk_u8_f32(encode_v(v[e], inv_v, least_v, uv), e, qv);
  }
  store4(static_cast<uint8_t*>(t.m), i, n, bad ? 0u : qm);
  store4(static_cast<uint8_t*>(t.v), i, n, bad ? 0u : qv);
  if (lane == 0) {
    t.m_scale[b] = bad ? NAN : top_m < kTiny ? 0.0f : top_m;
    t.v_scale[b] = bad ? NAN : top_v < kTiny ? 0.0f : top_v;
  }
}

// Values of eight neighbours to a thread: 218 M parameters' in bf16 225 us (5.8 TB/s); four neighbours
// to a thread, four times, 249.
template <bool BF16>
__global__ __launch_bounds__(256) void adamw_multi_read_k(AdamBatch bt) {
  int64_t i;
  const AdamTensor& t = tensor_of(bt, i);
  const int64_t n = t.n;
  i += threadIdx.x * 8;
  if (i >= n) return;
  const auto codes = [&](const void* p) {
    const uint8_t* q = static_cast<const uint8_t*>(p);
    if (i + 8 <= n) return load_nt<u32x2_t>(q, i / 8);
    return u32x2_t{load4(q, i, n), load4(q, i + 4, n)};
  };
  const auto put = [&](void* out, const float* f) {
    if constexpr (BF16) {
      if (i + 8 <= n) {
        const uint4 x = pack8(f);
        return store_nt<u32x4_t>(out, i / 8, u32x4_t{x.x, x.y, x.z, x.w});
      }
      store4(static_cast<bf16_t*>(out), i, n, f32x4_t{f[0], f[1], f[2], f[3]});
      store4(static_cast<bf16_t*>(out), i + 4, n, f32x4_t{f[4], f[5], f[6], f[7]});
    } else {
      store4(static_cast<float*>(out), i, n, f32x4_t{f[0], f[1], f[2], f[3]});
      store4(static_cast<float*>(out), i + 4, n, f32x4_t{f[4], f[5], f[6], f[7]});
    }
  };
  u32x2_t qm, qv;
  float unit, scale, f[8];
  if (t.m_out) {
    qm = codes(t.m);
    unit = t.m_scale[i / kBlock] * (1.0f / 16129.0f);
  }
  if (t.v_out) {
    qv = codes(t.v);
    scale = t.v_scale[i / kBlock];
  }
  if (t.m_out) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = decode_m((int8_t)(qm[e / 4] >> 8 * (e % 4)), unit);
    put(t.m_out, f);
  }
  if (t.v_out) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = decode_v((uint8_t)(qv[e / 4] >> 8 * (e % 4)), scale);
    put(t.v_out, f);
  }
}

}  // namespace

// The launch of kernel on a batch that is not empty, which is empty behind it.
template <typename K, typename... A>
static hipError_t launch(K kernel, AdamBatch& b, hipStream_t s, A... rest) {
  if (b.count == 0) return hipSuccess;
  for (int i = b.count; i < kAdamBatch; ++i) b.end[i] = INT32_MAX;   // (for the search)
  hipLaunchKernelGGL(kernel, dim3((unsigned)b.chunks), dim3(256), 0, s, b, rest...);
  b.count = b.chunks = 0;
  return hipGetLastError();
}

hipError_t adamw_multi(AdamBatch& b, int bits, bool grad_bf16, const AdamHyper& h, hipStream_t s) {
  if (bits == 32) return launch(grad_bf16 ? adamw_multi_32_k<true> : adamw_multi_32_k<false>, b, s, h);
  return launch(grad_bf16 ? adamw_multi_8_k<true> : adamw_multi_8_k<false>, b, s, h);
}
hipError_t adamw_multi_read(AdamBatch& b, bool out_bf16, hipStream_t s) {
  return launch(out_bf16 ? adamw_multi_read_k<true> : adamw_multi_read_k<false>, b, s);
}

}  // namespace forge
