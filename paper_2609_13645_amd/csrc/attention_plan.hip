// The plan of a packed batch (PackedPlan, kernels.h): which tiles its sequences have,
// built on the device from their offsets, and in which order blocks take them: those with
// the most keys first, so that no long block starts when the others have ended.
//  * The query passes: the longest sequences first, of each the last tile first. The blocks
//    that run at once are then of few sequences, whose keys an XCD's L2 holds.
//  * The kv pass, whose blocks are few and long: by the tiles' places, across all sequences
//    (4 documents of 4096 tokens, 32/8 heads of 64: backward 1267 us in the other order,
//    so 1141).
// With the sequences in order of their tiles neither needs a sort: in the first order those
// of k tiles stand behind the tiles of all longer ones, k to a sequence; in the second tile j
// of the r-th sequence stands r behind all tiles further in.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace forge {
namespace {

constexpr int kLdsBins = 4096;   // tiles of a sequence whose counts fit LDS

// Inclusive sum (or maximum) over the workgroup's threads; every thread gets the total too.
template <int THREADS, bool MAX>
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
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) {
    const int y = lds[w];
    if (w < wave) before = join(before, y);
    total = join(total, y);
  }
  return join(before, x);
}

// The sequences, THREADS at a time, a thread to each.
template <int THREADS>
struct Sequences {
  const PackedPlan& p;
  const int32_t* offsets;
  int* lds;
  int end = 0, base = 0;   // of those before
  __device__ __forceinline__ int offset(int i) const {
    return min(max(offsets[min(i, p.n_seqs)], 0), p.tokens);
  }
  // sequence s0 + thread: its rows and its first block of dS
  __device__ __forceinline__ PackedTile next(int s0) {
    const int s = s0 + (int)threadIdx.x;
    // the offsets' running maximum; a sequence starts where that before it ends
    if (s0 == 0) end = offset(0);
    const int last = end;
    const int e = scan<THREADS, true>(max(offset(s + 1), last), lds, end);
    int start = __shfl_up(e, 1, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = e;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) start = threadIdx.x ? lds[(threadIdx.x >> 6) - 1] : last;
    const int len = s < p.n_seqs ? min(e - start, p.max_seq) : 0;
    const int blocks = len > 0 ? (int)DsPacked(len, p.window, 0, 0).blocks() : 0;
    int total;
    const int b = base + scan<THREADS, false>(blocks, lds, total) - blocks;
    base += total;
    return PackedTile{start, len, 0, b};
  }
};

// One workgroup for each kind of tile. BINS, ORDER: the counts, the sequences in their order
// lie in LDS and not behind the lists. Bound by latencies: a dozen barriers, the offsets'
// load and the lists' stores.
template <int THREADS, bool BINS, bool ORDER>
__global__ __launch_bounds__(THREADS) void packed_plan_k(PackedPlan p,
                                                          const int32_t* __restrict__ offsets,
                                                          char* plan) {
  __shared__ int lds[THREADS / 64];
  __shared__ int bins[BINS ? 2 * (kLdsBins + 1) : 1];
  __shared__ PackedTile by_tiles[ORDER ? THREADS : 1];
  const int kind = (int)blockIdx.x, rows = packed_rows(kind), shift = 31 - __builtin_clz(rows);
  const bool by_place = kind == 4;
  const int nt = (p.max_seq + rows - 1) >> shift;   // tiles of a sequence, at most
  // per number of tiles k: how many sequences have exactly k, then how many have more;
  // the entries before those of k tiles (by_place: before tile k of any sequence)
  int* count = BINS ? bins : reinterpret_cast<int*>(plan + p.bins[kind]);
  int* first = count + nt + 1;
  PackedTile* order = ORDER ? by_tiles : reinterpret_cast<PackedTile*>(plan + p.order[kind]);
  PackedTile* list = reinterpret_cast<PackedTile*>(plan + p.tiles[kind]);
  // (in memory the atomics pass the vector cache, and so must what reads after them)
  const auto counted = [&](int k) {
    if constexpr (BINS) return count[k];
    else return __hip_atomic_load(&count[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  for (int j = (int)threadIdx.x; j <= nt; j += THREADS) count[j] = 0;
  __syncthreads();
  PackedTile mine{};
  {
    Sequences<THREADS> seqs{p, offsets, lds};
    for (int s0 = 0; s0 < p.n_seqs; s0 += THREADS) {
      mine = seqs.next(s0);
      if (mine.len > 0) atomicAdd(&count[(mine.len + rows - 1) >> shift], 1);
    }
  }
  __syncthreads();
  // from the most tiles down: the sequences with more, and the entries before
  int longer = 0, entries = 0;
  for (int k0 = 0; k0 <= nt; k0 += THREADS) {
    const int k = nt - k0 - (int)threadIdx.x;
    const int exactly = k >= 0 ? counted(k) : 0;
    int total;
    const int more = longer + scan<THREADS, false>(exactly, lds, total) - exactly;
    longer += total;
    const int tiles = k < 0 ? 0 : by_place ? more : exactly * k;
    const int before = entries + scan<THREADS, false>(tiles, lds, total) - tiles;
    entries += total;
    if (k >= 0) {
      count[k] = more;
      first[k] = before;
    }
  }
  __syncthreads();
  // the sequences in that order (which of equals comes first decides nothing but the
  // blocks' order)
  {
    Sequences<THREADS> seqs{p, offsets, lds};
    for (int s0 = 0; s0 < p.n_seqs; s0 += THREADS) {
      if (p.n_seqs > THREADS) mine = seqs.next(s0);
      if (mine.len > 0) order[atomicAdd(&count[(mine.len + rows - 1) >> shift], 1)] = mine;
    }
  }
  __syncthreads();
  // (count[k] is now the sequences with k tiles and more: those with exactly k end there)
  const int total = min(entries, p.cap[kind]);
  for (int e = (int)threadIdx.x; e < total; e += THREADS) {
    int lo = by_place ? 0 : 1, hi = nt;   // the smallest k with first[k] <= e
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (first[mid] <= e) hi = mid;
      else lo = mid + 1;
    }
    const int at = e - first[lo];
    PackedTile t;
    if (by_place) {
      t = order[at];
      t.tile = lo;
    } else {
      t = order[(lo < nt ? counted(lo + 1) : 0) + at / lo];
      t.tile = lo - 1 - at % lo;
    }
    list[e] = t;
  }
  if (threadIdx.x == 0) {
    PackedHeader* h = reinterpret_cast<PackedHeader*>(plan);
    h->count[kind] = total;
    if (kind == 0) {
      h->tokens = p.tokens;
      h->n_seqs = p.n_seqs;
      h->max_seq = p.max_seq;
      h->window = p.window;
    }
  }
}

__global__ __launch_bounds__(64) void packed_positions_k(PackedPlan p, const char* plan,
                                                         int32_t* __restrict__ pos) {
  if ((int)blockIdx.x >= reinterpret_cast<const PackedHeader*>(plan)->count[1]) return;
  const PackedTile t = reinterpret_cast<const PackedTile*>(plan + p.tiles[1])[blockIdx.x];
  const int r = t.tile * 64 + (int)threadIdx.x;
  if (r < t.len) pos[t.start + r] = r;
}

}  // namespace

// Blocks of dS of a head that n sequences of at most max_seq rows can come to in `tokens` rows.
// One of s slabs of 32 queries has f(s) blocks and 32 (s - 1) + 1 rows or more. f(s + 1) - f(s)
// does not fall with s where a window's keys are seen by an even number of slabs (else one more
// is taken): a slab of a shorter sequence is worth no less in a longer one. So the most come of
// as many sequences of max_seq as fit, one of the slabs that are left, and a block for each
// of the others.
static long most_ds_blocks(int tokens, long n, int max_seq, int window) {
  const int even = (62 + window) / 32 % 2 ? window : window + 32;
  const auto more = [&](long slabs) {   // f(slabs + 1) - f(1)
    return DsPacked((int)(32 * (slabs + 1)), even, 0, 0).blocks() - 1;
  };
  const long each = (max_seq - 1) / 32;   // slabs beyond the first
  const long full = std::min(n, tokens / (32 * each + 1)), rows = tokens - full * (32 * each + 1);
  const long rest = full < n && rows > 0 ? (rows - 1) / 32 : 0;
  return n + full * more(each) + more(rest);
}

PackedPlan::PackedPlan(int tokens_, int n_seqs_, int max_seq_, int window_)
    : tokens(tokens_), n_seqs(n_seqs_), max_seq(max_seq_ < tokens_ ? max_seq_ : tokens_),
      window(window_ > 0 && window_ < tokens_ ? window_ : tokens_) {
  const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  const long n = n_seqs < tokens ? n_seqs : tokens;   // sequences with a row
  bytes = 256;
  for (int k = 0; k < kPackedKinds; ++k) {
    const long rows = packed_rows(k), nt = (max_seq + rows - 1) / rows;
    cap[k] = (int)((tokens + (rows - 1) * n) / rows);
    tiles[k] = bytes;
    order[k] = tiles[k] + up((size_t)cap[k] * sizeof(PackedTile));
    bins[k] = order[k] + up((size_t)n * sizeof(PackedTile));
    bytes = bins[k] + up((size_t)(nt + 1) * 8);
  }
  // (nor more than those of every tile at the average of a sequence of max_seq, whose later
  // tiles the end cuts least)
  const long nt = (max_seq + 63) / 64;
  const long full = DsPacked((int)(nt * 64), window, 0, 0).blocks();
  ds_blocks = std::min(most_ds_blocks(tokens, n, max_seq, window), cap[1] * ((full + nt - 1) / nt));
}

hipError_t attn_packed_plan(const PackedPlan& p, const int32_t* offsets, void* plan, int32_t* pos,
                            hipStream_t s) {
  char* out = static_cast<char*>(plan);
  const bool bins = p.max_seq <= 32 * (kLdsBins - 1);
  const auto build = [&](auto kernel, int threads) {
    hipLaunchKernelGGL(kernel, dim3(kPackedKinds), dim3(threads), 0, s, p, offsets, out);
  };
  // Fewer threads wait less for each other, more fill long lists sooner: 5 sequences of 611
  // rows 3.8 us (of 1024 threads 5.4), 41 of 16384 5.0 (5.6), 4 of 32768 6.8 (5.8).
  if (bins && p.n_seqs <= 256 && p.cap[0] <= 768) build(packed_plan_k<256, true, true>, 256);
  else if (bins && p.n_seqs <= 1024) build(packed_plan_k<1024, true, true>, 1024);
  else if (bins) build(packed_plan_k<1024, true, false>, 1024);
  else if (p.n_seqs <= 1024) build(packed_plan_k<1024, false, true>, 1024);
  else build(packed_plan_k<1024, false, false>, 1024);
  if (pos)
    hipLaunchKernelGGL(packed_positions_k, dim3((unsigned)p.cap[1]), dim3(64), 0, s, p,
                       static_cast<const char*>(plan), pos);
  return hipGetLastError();
}

}  // namespace forge
