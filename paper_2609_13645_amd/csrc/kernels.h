// Internal launchers of libforge's gfx950 kernels (not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace forge {

// ---------------------------------------------------------------- GEMM ----
// C[m][n] (op)= sum_k A(m,k) B(k,n), bf16 operands, fp32 accumulation.
//   A layout KC: A(m,k) = A[m*lda + k]     MC: A(m,k) = A[k*lda + m]
//   B layout KC: B(k,n) = B[n*ldb + k]     MC: B(k,n) = B[k*ldb + n]
// so y = x W^T is (KC, KC), dX = dY W is (KC, MC), dW = dY^T X is (MC, MC).
enum GemmLayout { kKC = 0, kMC = 1 };
enum GemmEpilogue {
  kStoreBF16 = 0,     // C bf16 = acc
  kResidBF16 = 1,     // C bf16 = acc + R (bf16), one rounding
  kAccF32 = 2,        // C fp32 += acc
  kStoreF32 = 3,      // C fp32 = acc
  // weight gradient and its AdamW update in one epilogue (per-group weight
  // gradients, gemm_grouped_k): g = acc (kStoreF32Adam) or C + acc
  // (kAccF32Adam) is stored to C and then applied to the optimizer state at
  // the same position
  kStoreF32Adam = 4,
  kAccF32Adam = 5,
};

struct GemmArgs {
  const uint16_t* A;
  const uint16_t* B;
  void* C;
  const uint16_t* R;
  int M, N, K;
  long lda, ldb, ldc, ldr;
  // every epilogue takes alpha * acc in place of acc (a residual branch's
  // scale, App. B muP); 1 leaves every result bit-identical
  float alpha = 1.0f;
  // grouped products (MoE experts): g_off[E + 1] device row offsets of the
  // groups; strideB / strideC elements between consecutive groups' B / C.
  const int* g_off = nullptr;
  int groups = 0;
  long strideB = 0, strideC = 0;
  // split last round (GEMM tile order 4): the full 256-wide tiles from this
  // one on in the band order, each run as two BN-wide halves
  int tile_base = 0;
  // AdamW epilogues: fp32 master, moments m and v and the bf16 parameter,
  // laid out like C (leading dimension ldc; grouped: strideC apart), device
  // step scalars {lr, 1 - b1^t, 1 - b2^t, clip} and the hyper-parameters
  float* o_master = nullptr;
  float* o_m = nullptr;
  float* o_v = nullptr;
  uint16_t* o_param = nullptr;
  const float* o_sc = nullptr;
  float o_b1 = 0.0f, o_b2 = 0.0f, o_eps = 0.0f, o_wd = 0.0f;
};

// Host-side shape rules (checked by the caller): K-contiguous operands need
// K % 8 == 0; M/N-contiguous operands need that dimension % 8 == 0; leading
// dimensions % 8 == 0; base pointers 16-byte aligned.
// part (16-byte aligned, part_bytes): scratch that lets a product of few output
// tiles and a long reduction split the reduction over more workgroups, fp32
// partials added in a fixed order; gemm_split_bytes is what the product would
// use (0: it does not split). With less scratch it splits into fewer parts.
size_t gemm_split_bytes(GemmLayout la, GemmLayout lb, long M, long N, long K);
// How a product runs, and the tile of one over row groups (host only).
struct GemmPlan {
  int tile_m, tile_n, splits;
  size_t bytes;  // of partial products
};
GemmPlan gemm_plan(GemmLayout la, GemmLayout lb, long M, long N, long K, size_t part_bytes);
GemmPlan gemm_grouped_m_plan(GemmLayout lb, long rows, long groups, long N, long K);
hipError_t gemm(GemmLayout la, GemmLayout lb, GemmEpilogue epi, const GemmArgs& a,
                hipStream_t stream, float* part = nullptr, size_t part_bytes = 0);
// Grouped forms, one product per group e with rows [g_off[e], g_off[e+1]):
//   M-grouped (KC or MC B): C rows g_off[e].. = A rows g_off[e].. x B_e, where
//     B_e = B + e * strideB; M is an upper bound of the total rows (T * k).
//   K-grouped (MC, MC): C_e (+)= sum over rows g_off[e].. of A^T B, C_e = C + e * strideC.
hipError_t gemm_grouped_m(GemmLayout lb, GemmEpilogue epi, const GemmArgs& a, hipStream_t s);
hipError_t gemm_grouped_k(GemmEpilogue epi, const GemmArgs& a, hipStream_t s);

// --------------------------------------------------------- elementwise ----
hipError_t rmsnorm_fwd(const uint16_t* x, const uint16_t* g, uint16_t* y, float* rstd,
                       int T, int h, float eps, hipStream_t s);
// dx = RMSNorm backward (+ resid if non-null); dg_partial [nblk, h] per-block
// partial sums of dy*x*rstd, reduced into dg (+=, or = when !accumulate)
// by rmsnorm_dg_reduce.
int rmsnorm_bwd_blocks(int T);
hipError_t rmsnorm_bwd(const uint16_t* x, const uint16_t* g, const float* rstd,
                       const uint16_t* dy, const uint16_t* resid, uint16_t* dx,
                       float* dg_partial, int T, int h, hipStream_t s);
hipError_t rmsnorm_dg_reduce(const float* dg_partial, int nblk, float* dg, int h, bool accumulate,
                             hipStream_t s);
hipError_t rope_table(int seq, int d, float base, float* cos_t, float* sin_t,
                      hipStream_t s);
// pos: RoPE position of every token (NULL: index within its batch row).
hipError_t rope_apply(uint16_t* qkv, long row_stride, const float* cos_t,
                      const float* sin_t, const int32_t* pos, int T, int seq, int n_heads_rot,
                      int d, bool inverse, hipStream_t s);
// QK-Norm then RoPE on the nh q heads and nkv k heads of the qkv buffer, in
// place; raw [T, (nh + nkv) * d] keeps the un-normalised rows, rstd
// [T, nh + nkv] their rstd. The backward turns the post-RoPE gradient rows
// into the pre-norm gradient in place and writes gain-gradient partials
// [2][qknorm_bwd_blocks][d] (q, then k) for rmsnorm_dg_reduce.
hipError_t qknorm_rope_fwd(uint16_t* qkv, long ld, uint16_t* raw, float* rstd, const uint16_t* gq,
                           const uint16_t* gk, const float* cos_t, const float* sin_t,
                           const int32_t* pos, int T, int seq, int nh, int nkv, int d, float eps,
                           hipStream_t s);
int qknorm_bwd_blocks(int T, int nrot, int d);
hipError_t qknorm_rope_bwd(uint16_t* dqkv, long ld, const uint16_t* raw, const float* rstd,
                           const uint16_t* gq, const uint16_t* gk, const float* cos_t,
                           const float* sin_t, const int32_t* pos, int T, int seq, int nh, int nkv,
                           int d, float* dg_partial, hipStream_t s);
hipError_t swiglu_fwd(const uint16_t* gu, uint16_t* a, int T, int f, hipStream_t s);
hipError_t swiglu_bwd(const uint16_t* gu, const uint16_t* da, uint16_t* dgu, int T,
                      int f, hipStream_t s);
hipError_t embed_fwd(const int32_t* ids, const uint16_t* emb, uint16_t* x, int T,
                     int h, int V, float scale, hipStream_t s);
hipError_t embed_bwd(const int32_t* ids, const uint16_t* dx, float* demb, int T,
                     int h, int V, float scale, hipStream_t s);
// In place: z [T, V] bf16 logits -> dz = scale (softmax(scale z) - onehot)
// * inv_T; row_loss[t] of the scaled logits.
hipError_t ce_fwd_bwd(uint16_t* z, const int32_t* targets, float* row_loss, int T,
                      int V, float inv_T, float scale, hipStream_t s);
hipError_t mean_reduce(const float* v, int n, float scale, float* out, hipStream_t s);
hipError_t adamw(float* master, uint16_t* param, const float* grad, float* m, float* v,
                 int64_t n, float b1, float b2, float eps, float wd,
                 const float* scalars, hipStream_t s);
hipError_t adamw_advance(float* scalars, int32_t* step, float lr, double b1, double b2,
                         hipStream_t s);
constexpr int kNormPartials = 1024;
hipError_t sumsq_partials(const float* g, int64_t n, float* partials, hipStream_t s);
hipError_t sumsq_finish(const float* partials, float* accum, hipStream_t s);
hipError_t clip_coeff(const float* norm_sq, float max_norm, float eps, float* scalars,
                      hipStream_t s);

// ------------------------------------------- AdamW over many tensors ----
// (the members of forge_adamw_multi_tensor, and the tensor's place in the list)
struct AdamTensor {
  // (of a read: where the moments' values go; NULL: nowhere)
  union { float* master; void* m_out; };
  union { const void* grad; void* v_out; };   // fp32 or bf16
  uint16_t* param;
  void *m, *v;          // fp32, or int8 and uint8
  float *m_scale, *v_scale;
  int64_t n;
  float lr_scale, decay_scale;
  uint32_t index;
};
struct AdamHyper {
  float b1, b2, eps, wd;
  const float* sc;      // device {lr, 1 - b1^t, 1 - b2^t, clip}
  const int32_t* seed;  // device, NULL: codes to the nearest
};
// The tensors of a launch, which takes them by value (4 KB of arguments): tensor i has the
// workgroups from end[i - 1] (0) to end[i], one for `chunk` of its elements. (70 tensors of 19
// M elements in 8 bits, step and read: 96.5 us in launches of 32 tensors, so 90.1.)
constexpr int kAdamBatch = 48, kAdamStep = 1024, kAdamRead = 2048;
struct AdamBatch {
  AdamTensor t[kAdamBatch];
  int32_t end[kAdamBatch];
  int32_t count = 0, chunks = 0, chunk;
  // chunk_: kAdamStep or kAdamRead, by what takes the batch
  explicit AdamBatch(int chunk_) : chunk(chunk_) {}
  // false: the launch is full (n <= 2^33, threads of a launch below 2^32)
  bool add(const AdamTensor& x) {
    const int32_t c = (int32_t)((x.n + chunk - 1) / chunk);
    if (count == kAdamBatch || (count > 0 && chunks + c > 1 << 23)) return false;
    t[count] = x;
    end[count++] = chunks += c;
    return true;
  }
};
static_assert(sizeof(AdamBatch) + sizeof(AdamHyper) <= 4096);
// Launches of the batch's tensors, which is empty again behind them; bits 32 or 8.
hipError_t adamw_multi(AdamBatch& b, int bits, bool grad_bf16, const AdamHyper& h, hipStream_t s);
hipError_t adamw_multi_read(AdamBatch& b, bool out_bf16, hipStream_t s);

// ----------------------------------------------------------- LayerNorm ----
hipError_t layernorm_fwd(const uint16_t* x, const uint16_t* g, const uint16_t* b, uint16_t* y,
                         float* mean, float* rstd, int T, int h, float eps, hipStream_t s);
// dx (+ resid if non-null), dg and db (db may be null), added to or stored; part:
// layernorm_bwd_blocks(T, h) * 2 * h floats of scratch. T == 0: dg and db alone.
int layernorm_bwd_blocks(int T, int h);
hipError_t layernorm_bwd(const uint16_t* x, const uint16_t* g, const float* mean,
                         const float* rstd, const uint16_t* dy, const uint16_t* resid,
                         uint16_t* dx, float* dg, float* db, bool accumulate, float* part, int T,
                         int h, hipStream_t s);

// ----------------------------------------- rotary positions, several axes ----
constexpr int kRopeMaxPairs = 256;
struct RopeFreqs {
  double w[kRopeMaxPairs];            // angle of pair i per position
};
struct RopeAxes {
  uint32_t axis[kRopeMaxPairs / 16];  // the axis of pair i: bits 2 (i % 16) of word i / 16
  int at(int i) const { return axis[i / 16] >> 2 * (i % 16) & 3; }
};
hipError_t rope_axes_table(const RopeFreqs& f, int rows, int d, float* cos_t, float* sin_t,
                           hipStream_t s);
// y = x rotated on the first nrot heads of each row (y may be x); pos [axes][T].
hipError_t rope_axes(const RopeAxes& ax, const uint16_t* x, long ldx, uint16_t* y, long ldy,
                     const float* cos_t, const float* sin_t, const int32_t* pos, int T, int rows,
                     int nrot, int d, bool inverse, hipStream_t s);

// --------------------------- rotary positions, a part of each head ----
// Tables of amplitude cos and amplitude sin of `half` pairs.
hipError_t rope_part_table(const RopeFreqs& f, float amplitude, int rows, int half, float* cos_t,
                           float* sin_t, hipStream_t s);
struct RopePart {
  const uint16_t* x;
  uint16_t* y;                  // may be x
  long ldx, ldy;
  const float *cos_t, *sin_t;   // [rows, rot / 2]
  const int32_t* pos;           // [T], NULL: index modulo rows
  uint32_t T;
  int rows;
  uint32_t nrot, d, rot, offset;
  bool interleaved, copy;       // copy: y is not x, the other columns go with the part
  float sign;                   // of the sine: -1 backward
};
// (T * nrot * d < 2^31)
hipError_t rope_part(const RopePart& a, hipStream_t s);

// ----------------------------------------------------------- attention ----
struct AttnArgs {
  const uint16_t* q;    // [T, *] rows, head n at column n*d, row stride ld_qkv
  const uint16_t* k;
  const uint16_t* v;
  long ld_qkv;
  int batch, seq, n_heads, n_kv_heads, d;
  float scale;          // 1/sqrt(d)
  // (what AttnWindowArgs adds; the causal kernels have no such arguments)
  static constexpr int window = 0, sinks = 0;
  static constexpr const int32_t* lens = nullptr;
};
// Where a sliding window's backward keeps dS, of each (batch, head): for every key tile
// kt of 64 a block of 2048 elements for each slab of 32 queries from 2 kt on that is
// stored, and no more: of a sink tile (kt < nst) all ns - 2 kt, of the others the nwin
// slabs that its keys' windows can reach, from tile cut on fewer, as the sequence ends.
struct DsWindow {
  int ns = 0, nst = 0, nwin = 0, cut = 0;
  long band = 0, tail = 0;   // added by tile() from tile nst and from tile cut on
  long head = 0;             // elements of a (batch, head)
  __host__ __device__ long tile(int kt) const {
    const bool full = kt > nst && kt <= cut;
    return 2048L * ((long)kt * (full ? nwin : ns + 1 - kt) + (kt <= nst ? 0 : full ? band : tail));
  }
  __host__ __device__ long block(int kt, int j) const { return tile(kt) + 2048L * (j - 2 * kt); }
};
// Sliding window: key j is visible to query i iff j <= i and (j > i - window or
// j < sinks); 1 <= window <= seq, 0 <= sinks <= seq. lens (device int32 [batch],
// may be NULL): tokens of each batch row, clamped to [0, seq]; the rows behind
// them are neither read nor visible, and their outputs are zeros (lse -inf).
struct AttnWindowArgs : AttnArgs {
  int window, sinks;
  const int32_t* lens;
  // set by the backward: where dS lies; chunks of the sink tiles' slabs behind their own
  // windows (0: none), slabs of each, and the sink tiles' partial sums; whether a key
  // tile's slabs are walked round
  DsWindow ds;
  int sink_chunks = 0, chunk_slabs = 0, go_round = 0;
  float *sink_pk = nullptr, *sink_pv = nullptr;
  // the other key tiles' splits and their partial sums; units of the sums, of the splits'
  // and in all; where the sums go
  float *pk = nullptr, *pv = nullptr;
  int splits = 1, part_units = 0, sum_units = 0;
  uint16_t *dk = nullptr, *dv = nullptr;
  // the forward's outputs
  const uint16_t* o = nullptr;
  const float* lse = nullptr;
};
// Packed sequences: rows [start, start + len) of a packed row, one sequence of many.
struct PackedTile {
  int32_t start, len;   // the sequence's
  int32_t tile;         // which of its tiles
  int32_t base;         // its first block of dS (DsPacked)
};
// Where a sequence's dS lies within a head's: as that of a window over one batch row,
// from block `base` on.
struct DsPacked : DsWindow {
  long base = 0;
  __host__ __device__ DsPacked(int len, int window, long base_, long head_) : base(base_) {
    ns = (len + 31) / 32;
    nwin = min((62 + window) / 32 + 1, ns);
    cut = (ns - nwin + 1) / 2;
    tail = (long)cut * nwin - (long)cut * (ns + 1 - cut);
    head = head_;
  }
  __host__ __device__ static int min(int a, int b) { return a < b ? a : b; }
  __host__ __device__ long blocks() const { return DsWindow::tile((ns + 1) / 2) / 2048; }
  __host__ __device__ long tile(int kt) const { return 2048L * base + DsWindow::tile(kt); }
  __host__ __device__ long block(int kt, int j) const { return tile(kt) + 2048L * (j - 2 * kt); }
};
// The plan of a packed batch: a header (for which sizes it was made; how many tiles of
// each kind there are), a list of each kind of tile, and what the builder keeps of the
// sequences. All of it from the host's bounds alone: each list has room for what the
// sequences can come to.
// Lists of tiles of 32, 64, 128 and 256 rows, the longest sequences first; and of 64 rows,
// the tiles furthest into their sequence first.
constexpr int kPackedKinds = 5;
constexpr int packed_rows(int kind) { return kind == 4 ? 64 : 32 << kind; }
struct PackedHeader {
  int32_t tokens, n_seqs, max_seq, window;
  int32_t count[kPackedKinds], pad[3];
};
struct PackedPlan {
  int tokens, n_seqs, max_seq, window;   // max_seq and window cut to tokens
  int cap[kPackedKinds];                 // entries of each list
  // bytes: where the lists lie, the sequences by their tiles, and how many have them
  size_t tiles[kPackedKinds], order[kPackedKinds], bins[kPackedKinds], bytes;
  long ds_blocks;                        // blocks of dS of a head, at most
  __host__ PackedPlan(int tokens_, int n_seqs_, int max_seq_, int window_);
};
// batch 1, seq the tokens of the packed row.
struct AttnPackedArgs : AttnArgs {
  int window;
  const PackedHeader* plan;
  const PackedTile* tiles[kPackedKinds];
  int n_seqs, max_seq;
  long ds_head;                          // elements of a head's dS
  // the forward's outputs
  const uint16_t* o = nullptr;
  const float* lse = nullptr;
};
// pos (may be NULL): every token's place in its sequence.
hipError_t attn_packed_plan(const PackedPlan& p, const int32_t* offsets, void* plan, int32_t* pos,
                            hipStream_t s);
// o [T, n_heads*d] bf16; lse [batch, n_heads, seq] fp32 (natural log).
hipError_t attn_fwd(const AttnArgs& a, uint16_t* o, float* lse, hipStream_t s);
hipError_t attn_window_fwd(const AttnWindowArgs& a, uint16_t* o, float* lse, hipStream_t s);
hipError_t attn_packed_fwd(const AttnPackedArgs& a, const PackedPlan& p, uint16_t* o, float* lse,
                           hipStream_t s);
// Backward. delta: 2 * batch * n_heads * seq fp32 scratch ([b,n,i] =
// -sum_d dO*O, then [b,n,i] = -lse * log2(e)); ds: attn_bwd_ds_bytes scratch
// (dS in bf16, the causal half per (batch, head)); part: attn_bwd_part_bytes
// scratch (fp32 partial sums of dk and dv where the launch would leave CUs
// idle, else 0 bytes and may be NULL). dq [T, n_heads*d] and
// dk, dv [T, n_kv*d] are column blocks of the dqkv buffer (row stride
// ld_dqkv); dk and dv hold each kv head's sums over its GQA group.
size_t attn_bwd_ds_bytes(const AttnArgs& a);
size_t attn_bwd_part_bytes(const AttnArgs& a);
hipError_t attn_bwd(const AttnArgs& a, const uint16_t* o, const uint16_t* dout, const float* lse,
                    float* delta, uint16_t* ds, float* part, uint16_t* dq, uint16_t* dk,
                    uint16_t* dv, long ld_dqkv, hipStream_t s);
// The same of a sliding window, its dS a band (and, for the sinks, whole rows).
size_t attn_window_bwd_ds_bytes(const AttnWindowArgs& a);
size_t attn_window_bwd_part_bytes(const AttnWindowArgs& a);
hipError_t attn_window_bwd(const AttnWindowArgs& a, const uint16_t* o, const uint16_t* dout,
                           const float* lse, float* delta, uint16_t* ds, float* part, uint16_t* dq,
                           uint16_t* dk, uint16_t* dv, long ld_dqkv, hipStream_t s);
// The same of packed sequences; dS: 4096 * n_heads * p.ds_blocks bytes.
hipError_t attn_packed_bwd(const AttnPackedArgs& a, const PackedPlan& p, const uint16_t* o,
                           const uint16_t* dout, const float* lse, float* delta, uint16_t* ds,
                           uint16_t* dq, uint16_t* dk, uint16_t* dv, long ld_dqkv, hipStream_t s);

// ----------------------------------------------------------------- MoE ----
// Routing of fp32 logits [T, E] (E <= 256): idx / gates [T, k], probs [T, E];
// every idx entry lies in [0, E) (NaN logits rank below -inf).
hipError_t moe_route(const float* logits, int T, int E, int k, int32_t* idx, float* gates,
                     float* probs, hipStream_t s);
// Blocks of the counting sort; block_counts needs moe_sort_blocks(T) * E ints.
int moe_sort_blocks(int T);
// counts [E], offsets [E + 1], perm / pos_of [T k] (canonical order). With aux,
// the layer's load-balance loss over probs [T, E] is added to it (colsum:
// moe_sort_blocks(T) * E floats of scratch).
hipError_t moe_sort(const int32_t* idx, int T, int E, int k, int32_t* block_counts,
                    int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* pos_of,
                    hipStream_t s, const float* probs = nullptr, float alpha = 0.0f,
                    float* colsum = nullptr, float* aux = nullptr);
hipError_t moe_gather(const uint16_t* b, const int32_t* perm, long rows, int h, int k,
                      uint16_t* xs, hipStream_t s);
// out = h1 + scale * sum_j gate_j ys_j; backward with the same scale.
hipError_t moe_combine(const uint16_t* ys, const float* gates, const int32_t* pos_of,
                       const uint16_t* h1, long T, int h, int k, float scale, uint16_t* out,
                       hipStream_t s);
hipError_t moe_combine_bwd(const uint16_t* ys, const float* gates, const int32_t* pos_of,
                           const uint16_t* dy, long T, int h, int k, float scale, float* dgate,
                           uint16_t* dys, hipStream_t s);
hipError_t moe_scatter_back(const uint16_t* dxs, const int32_t* pos_of, long T, int h, int k,
                            uint16_t* db, hipStream_t s);
hipError_t moe_router_bwd(const float* probs, const int32_t* idx, const float* dgate,
                          const int32_t* counts, int T, int E, int k, float alpha, uint16_t* dl,
                          hipStream_t s);

}  // namespace forge
