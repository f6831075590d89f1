// The plan of a packed batch (PackedPlan, kernels.h): which tiles its sequences have,
// built on the device from their offsets.
#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Inclusive sum (or maximum) over the workgroup's threads; every thread gets the total too.
template <bool MAX>
__device__ __forceinline__ int scan(int x, int* lds, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const auto join = [](int a, int b) { return MAX ? max(a, b) : a + b; };
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x = join(x, y);
  }
  __syncthreads();   // (lds may still be read by the scan before)
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  int before = MAX ? INT32_MIN : 0;
  total = before;
  for (int w = 0; w < kWaves; ++w) {
    const int y = lds[w];
    if (w < wave) before = join(before, y);
    total = join(total, y);
  }
  return join(before, x);
}

// One workgroup, a thread to a sequence, kThreads of them at a time.
__global__ __launch_bounds__(kThreads) void packed_plan_k(PackedPlan p,
                                                          const int32_t* __restrict__ offsets,
                                                          char* plan) {
  __shared__ int lds[kWaves];
  int first = 0, base = 0, done[3] = {0, 0, 0};
  for (int s0 = 0; s0 < p.n_seqs; s0 += kThreads) {
    const int s = s0 + (int)threadIdx.x;
    const auto offset = [&](int i) { return min(max(offsets[min(i, p.n_seqs)], 0), p.tokens); };
    // running maximum of the offsets, the sequence's end among them
    int total;
    const int end = scan<true>(max(offset(s + 1), max(s0 == 0 ? offset(0) : 0, first)), lds, total);
    int start = __shfl_up(end, 1, 64);
    __shared__ int edge[kWaves];
    if ((threadIdx.x & 63) == 63) edge[threadIdx.x >> 6] = end;
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
      start = threadIdx.x ? edge[(threadIdx.x >> 6) - 1] : max(s0 == 0 ? offset(0) : 0, first);
    first = total;
    const int len = s < p.n_seqs ? min(end - start, p.max_seq) : 0;
    const int blocks = len > 0 ? (int)DsPacked(len, p.window, 0, 0).blocks() : 0;
    const int my_base = base + scan<false>(blocks, lds, total) - blocks;
    base += total;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const int nt = (len + (64 << k) - 1) >> (6 + k);
      const int at = done[k] + scan<false>(nt, lds, total) - nt;
      done[k] += total;
      PackedTile* list = reinterpret_cast<PackedTile*>(plan + p.tiles[k]);
      for (int t = 0; t < nt && at + t < p.cap[k]; ++t)
        list[at + t] = PackedTile{start, len, t, my_base};
    }
  }
  if (threadIdx.x == 0) {
    PackedHeader* h = reinterpret_cast<PackedHeader*>(plan);
    *h = PackedHeader{p.tokens, p.n_seqs, p.max_seq, p.window, {}, 0};
    for (int k = 0; k < 3; ++k) h->count[k] = min(done[k], p.cap[k]);
  }
}

__global__ __launch_bounds__(64) void packed_positions_k(PackedPlan p, const char* plan,
                                                         int32_t* __restrict__ pos) {
  if ((int)blockIdx.x >= reinterpret_cast<const PackedHeader*>(plan)->count[0]) return;
  const PackedTile t = reinterpret_cast<const PackedTile*>(plan + p.tiles[0])[blockIdx.x];
  const int r = t.tile * 64 + (int)threadIdx.x;
  if (r < t.len) pos[t.start + r] = r;
}

}  // namespace

PackedPlan::PackedPlan(int tokens_, int n_seqs_, int max_seq_, int window_)
    : tokens(tokens_), n_seqs(n_seqs_), max_seq(max_seq_ < tokens_ ? max_seq_ : tokens_),
      window(window_ > 0 && window_ < tokens_ ? window_ : tokens_) {
  const long n = n_seqs < tokens ? n_seqs : tokens;   // sequences with a row
  bytes = 256;
  for (int k = 0; k < 3; ++k) {
    const long rows = 64L << k;
    cap[k] = (int)((tokens + (rows - 1) * n) / rows);
    tiles[k] = bytes;
    bytes += ((size_t)cap[k] * sizeof(PackedTile) + 255) / 256 * 256;
  }
  // a tile has on average no more blocks than one of a sequence of max_seq, whose later
  // tiles the end cuts least
  const long nt = (max_seq + 63) / 64;
  const long full = DsPacked((int)(nt * 64), window, 0, 0).blocks();
  ds_blocks = cap[0] * ((full + nt - 1) / nt);
}

hipError_t attn_packed_plan(const PackedPlan& p, const int32_t* offsets, void* plan, int32_t* pos,
                            hipStream_t s) {
  hipLaunchKernelGGL(packed_plan_k, dim3(1), dim3(kThreads), 0, s, p, offsets,
                     static_cast<char*>(plan));
  if (pos)
    hipLaunchKernelGGL(packed_positions_k, dim3((unsigned)p.cap[0]), dim3(64), 0, s, p,
                       static_cast<const char*>(plan), pos);
  return hipGetLastError();
}

}  // namespace forge
