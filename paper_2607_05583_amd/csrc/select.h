// Launch interface of the selective layer's kernels and of the token probabilities: the
// short causal convolution (conv.hip), the selective scan (selective.hip) and the log
// probabilities (logprobs.hip), between their C entry points (api_select.hip) and the kernels.
#pragma once

#include <algorithm>

#include "layer.h"

namespace res {

// N elements at the alignment of one: the unit takes vector accesses at any address.
template <typename T, int N> using AnyVec = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));

// The first n (at most V) of V consecutive elements; zeros behind them.
template <typename T, int V>
__device__ __forceinline__ void load_part(const T* p, int n, T (&v)[V]) {
  if (n >= V) {
    const AnyVec<T, V> q = *reinterpret_cast<const AnyVec<T, V>*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = q[e];
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e < n ? p[e] : T(0);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, int n, const T (&v)[V]) {
  if (n >= V) {
    AnyVec<T, V> q;
#pragma unroll
    for (int e = 0; e < V; ++e) q[e] = v[e];
    *reinterpret_cast<AnyVec<T, V>*>(p) = q;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = v[e];
  }
}

// ---------------------------------------------------------------------------
// Short causal convolution
// ---------------------------------------------------------------------------
constexpr int CONV_TAPS = 16;       // taps at most
constexpr int CONV_THREADS = 256;
constexpr int CONV_SHIFT = 5;       // steps of a thread at most: 32 forward
constexpr int CONV_BWD_SHIFT = 6;   // and 64 backward
constexpr int CONV_LEAST = 3;       // 8 at least (16 forward with more than nine taps where the state is overwritten)
constexpr int CONV_ENOUGH = 512;    // work-groups that are enough for the chip: with fewer, threads take fewer steps
constexpr int CONV_BWD_ROWS = 4;    // tiles of a work-group of the backward, whose weight gradients are summed in it
constexpr int CONV_BWD_CHANNELS = 128;

struct ConvArgs {
  Rows x, dy;
  RowsOut dx;
  const float* w;        // [D][K]
  const float* bias;     // [D] or null
  const void* state;     // [B][K - 1][D] or null (zeros)
  const int* lengths;    // [B] or null
  void* y;               // [B][L][D]
  void* state_out;       // [B][K - 1][D] or null
  const void* dstate_out;
  void* dstate;
  float* part;           // backward: [row blocks][K + 1][D], the sums of a block's dw and dbias
  float *dw, *dbias;
  int64_t B, L, D, b0;   // b0: the launch's first batch row
  int K, act;
  int tile, shift;       // steps of a thread, and their binary logarithm
};
inline int64_t conv_tiles(int64_t L, int shift) { return ((L + (1 << shift) - 1) >> shift) + (L == 0); }
// Where the forward writes the state over (state_out is the state), its tiles have K - 1 steps at least: then no tile but the first needs
// an input before the call, and the first tile's threads have read theirs when they write.  Other calls take tiles of 8 steps with any
// number of taps (2 x 512 steps of 640 channels, bf16, 10 and 16 taps: 12.0 and 16.5 us; 16.6 and 21.1 with tiles of 16, in place).
inline int conv_least(int K) {
  int shift = CONV_LEAST;
  while (1 << shift < K - 1) ++shift;
  return shift;
}
static_assert(CONV_TAPS - 1 <= 1 << CONV_SHIFT, "a tile of the most steps reaches over the taps");
template <typename F> int conv_shift(int most, int least, int64_t L, F&& work_groups) {
  int shift = most;
  while (shift > least && work_groups(conv_tiles(L, shift)) < CONV_ENOUGH) --shift;
  return shift;
}
inline int64_t conv_row_blocks(int64_t B, int64_t L, int shift) { return (B * conv_tiles(L, shift) + CONV_BWD_ROWS - 1) / CONV_BWD_ROWS; }
inline int conv_bwd_shift(int64_t B, int64_t L, int64_t D) {
  const int64_t across = (D + CONV_BWD_CHANNELS - 1) / CONV_BWD_CHANNELS;
  return conv_shift(CONV_BWD_SHIFT, CONV_LEAST, L, [&](int64_t tiles) { return (B * tiles + CONV_BWD_ROWS - 1) / CONV_BWD_ROWS * across; });
}
// Floats of the sums of all blocks, of the largest call of up to these sizes.  A call with CONV_ENOUGH work-groups of the most steps has
// as many blocks as these make.  Any other takes half the steps only while the work-groups were fewer than CONV_ENOUGH, so that it has
// fewer than 2 CONV_ENOUGH work-groups of CONV_BWD_CHANNELS channels each, and no more blocks than tiles of the least steps make.
inline int64_t conv_part_floats(int64_t B, int64_t L, int64_t D, int64_t K) {
  const int64_t most = 2 * (CONV_ENOUGH - 1) * CONV_BWD_CHANNELS;
  return (K + 1) * std::max(conv_row_blocks(B, L, CONV_BWD_SHIFT) * D, std::min(conv_row_blocks(B, L, CONV_LEAST) * D, most));
}
template <typename T> hipError_t launch_conv_fwd(ConvArgs a, hipStream_t st);
template <typename T> hipError_t launch_conv_bwd(const ConvArgs& a, hipStream_t st);
template <typename T> hipError_t launch_conv_step(ConvArgs a, hipStream_t st);

// ---------------------------------------------------------------------------
// Selective scan.  The time axis goes in chunks of SEL_Q steps; a segment is a number of
// consecutive chunks that one work-group takes in turn.  A head's P rows go in blocks of
// SEL_P: a "row block" (b, head, block) holds a state [SEL_P][NP], NP = N padded.
// ---------------------------------------------------------------------------
constexpr int SEL_Q = 64, SEL_P = 64, SEL_THREADS = 256;
constexpr int SEL_MAX = 128;   // P and N at most
constexpr int SEL_BWD_HEADS = 4;  // row blocks of a work-group of the backward at most

struct SelPlan {
  int NT;            // tiles of 16 states, padded: 2, 4 or 8
  int PB, PS;        // row blocks of a head: 1 or 2; PB - 1
  int HV, HG;        // row blocks of a batch row, of a group
  int HF, HR;        // row blocks of a work-group, forward and backward
  int64_t chunks, seg, segs;  // chunks of a row; chunks of a segment; segments
};
SelPlan sel_plan(bool bf16, int64_t B, int64_t L, int64_t H, int64_t P, int64_t G, int64_t N);

struct SelArgs {
  Rows x, dt, b, c, dy;     // x, dy: [H][P] a step; dt: [H]; b, c: [G][N]
  RowsOut dx, ddt, db, dc;
  const float *gamma, *dt_bias, *skip;  // [H]; the last two or null
  const float *h0, *dh_out;             // [B][H][P][N] or null
  const int* lengths;                   // [B] or null
  void* y;                              // [B][L][H][P]
  float *h_out, *dh0;                   // [B][H][P][N] or null
  float* enter;   // [B][HV][segs][SEL_P][NP]: the state before each segment (with several)
  float* leave;   // the gradient of the state behind each segment, likewise
  float* decay;   // [B][HV][segs]: a segment's sum of gamma D in units of ln 2
  f4* hs;         // backward: a work-group's states before each chunk
  f4* gs;         // backward: its states' gradients
  float* part;    // backward: db and dc of each block of heads of a group [blocks][2][B][L][G N], with more than one
  float* params;  // backward: [B][segs][HV][3], sums for dgamma, ddt_bias, dskip
  float *dgamma, *ddt_bias, *dskip;     // [H]; the last two or null
  int64_t B, L, wg0;                    // wg0: the launch's first work-group
  int H, P, G, N;
  SelPlan p;
};
template <typename T> hipError_t launch_selective_fwd(const SelArgs& a, hipStream_t st);
template <typename T> hipError_t launch_selective_bwd(const SelArgs& a, hipStream_t st);
template <typename T> hipError_t launch_selective_step(const SelArgs& a, const float* h, hipStream_t st);

// ---------------------------------------------------------------------------
// Token log probabilities
// ---------------------------------------------------------------------------
constexpr int LOGPROBS_TOP = 64;  // alternatives at most: one lane of a wave each

struct LogprobsArgs {
  const void* logits;     // rows at distance ld
  int64_t ld, ldd;
  const int64_t* tokens;  // [R]
  int64_t R, V, r0;       // r0: the launch's first row
  float scale;
  float* logp;            // [R]
  float* stats;           // [R][2]: the largest logit, and the logarithm of the sum of exp(scale (logit - largest))
  float* entropy;         // [R] or null
  int top;
  int64_t* top_ids;       // [R][top]
  float* top_logp;
  const float* dlogp;     // [R] or null
  const float* dentropy;  // [R] or null
  void* dlogits;          // rows at distance ldd
};
template <typename T> hipError_t launch_logprobs_fwd(LogprobsArgs a, hipStream_t st);
template <typename T> hipError_t launch_logprobs_bwd(LogprobsArgs a, hipStream_t st);

}  // namespace res
