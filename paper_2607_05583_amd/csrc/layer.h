// Launch interface of the gated recurrent layer's kernels: the gated scan
// (gated.hip), the linear product with its epilogue (linear.hip) and the AdamW
// step (adamw.hip), between their C entry points (api_layer.hip) and the kernels.
#pragma once

#include "../../include/resonator.h"
#include "common.h"

namespace res {

// Records the text resonator_last_error returns and gives the code back (api.hip).
int api_error(int code, const char* fmt, ...);

// Rows of D consecutive elements at p + b sb + t st (strides in elements).
struct Rows {
  const void* p;
  int64_t sb, st;
};
struct RowsOut {
  void* p;
  int64_t sb, st;
};

// Threads of one launch: more are not refused, their last work-groups are left out without an error.
constexpr int64_t LAUNCH_THREADS = (1LL << 32) - 1;

// ---------------------------------------------------------------------------
// Device mathematics shared by the operators
// ---------------------------------------------------------------------------
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float sigmoid_fast(float v) {
  return __builtin_amdgcn_rcpf(1.0f + exp2_fast(-LOG2E * v));  // exp2 = inf gives 0
}

// Activations of the linear product (codes RES_ACT_*): none, relu, silu = v sigmoid(v),
// gelu_tanh = v/2 (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))), which is v sigmoid(2 sqrt(2/pi) (...)).
enum { ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_GELU_TANH = 3 };
constexpr float GELU_2C = 1.59576912160573071176f;  // 2 sqrt(2 / pi)
constexpr float GELU_K = 0.044715f;
__device__ __forceinline__ float gelu_sigmoid(float v) {  // sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3))
  return __builtin_amdgcn_rcpf(1.0f + exp2_fast(v * fmaf(-LOG2E * GELU_2C * GELU_K * v, v, -LOG2E * GELU_2C)));
}

__device__ __forceinline__ float act_value(float v, int act) {
  if (act == ACT_RELU) return v > 0.0f ? v : (v != v ? v : 0.0f);
  if (act == ACT_SILU) return v * sigmoid_fast(v);
  if (act == ACT_GELU_TANH) return v * gelu_sigmoid(v);
  return v;
}
__device__ __forceinline__ float act_slope(float v, int act) {
  if (act == ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
  if (act == ACT_SILU) {
    const float q = sigmoid_fast(v);
    return q * fmaf(v, 1.0f - q, 1.0f);
  }
  if (act == ACT_GELU_TANH) {
    const float q = gelu_sigmoid(v), d = q * (1.0f - q);
    // far out d is 0 and the polynomial may be infinite
    return d == 0.0f ? q : fmaf(d * GELU_2C * v, fmaf(3.0f * GELU_K * v, v, 1.0f), q);
  }
  return 1.0f;
}

// ---------------------------------------------------------------------------
// Gated scan.  A chain is one batch row and one block of GATED_CW channels.
// ---------------------------------------------------------------------------
constexpr int GATED_CW = 64;      // channels of a chain: 128-byte rows of bf16
constexpr int GATED_CARRY = 128;  // steps between the states that a forward keeps for its backward
constexpr int GATED_FWD_TILE = 256, GATED_BWD_TILE = 128;  // steps of a tile (of 512 threads)
constexpr int GATED_TILE_WORDS = 3 * GATED_CW;             // words that a tile publishes

constexpr int GATED_THREADS = 512;  // of a work-group, at most

// tiles of a chain: one where there is no step, which hands the state through
__host__ __device__ inline int64_t gated_tiles(int64_t L, int64_t tile) { return L > 0 ? (L + tile - 1) / tile : 1; }

struct GatedArgs {
  Rows x, r, i, dy;
  void* y;              // [B][L][D] or null (states only)
  RowsOut dx, dr, di;
  int64_t B, L;
  int D, NB;            // channels; blocks of GATED_CW channels
  int vec;              // every row starts at a multiple of its vector's bytes, and D is a multiple of the vector
  const float* gamma;   // [D]
  const float* h0;      // [B][D] or null
  const int* lengths;   // [B] or null
  float* h_out;         // [B][D] or null
  float* carry;         // [B][ceil(L / GATED_CARRY)][D]: the state before each such step (forward: written where not null)
  const float* dh_out;  // [B][D] or null
  float* dh0;           // [B][D] or null
  uint32_t* hdr;        // [0] status (a wait gave up), [1] number of calls so far, [2] next ticket, [3] work-groups done
  uint64_t* words;      // published maps and end values: [chain][tile][A, H or C, end][GATED_CW]
  uint64_t* part;       // backward: partial sums of dgamma [B][tiles][NB * GATED_CW]
};

template <typename T>
hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t st);
template <typename T>
hipError_t launch_gated_bwd(const GatedArgs& a, float* dgamma, hipStream_t st);
template <typename T>
hipError_t launch_gated_step(const Rows& x, const Rows& r, const Rows& i, void* y, int64_t B, int64_t D,
                             const float* gamma, const float* h, float* h_out, hipStream_t st);


// ---------------------------------------------------------------------------
// Linear product with epilogue: C[m][n] = sum_k A(m, k) B(k, n), then out =
// act(C + bias[n]) + res[m][n]; pre receives C + bias[n].
// ---------------------------------------------------------------------------
// 64 x 64, 128 x 128, 128 x 256 (bf16) outputs of a work-group; 64 x 64 with the K axis spread over its waves
enum { TILE_SMALL = 0, TILE_SQUARE = 1, TILE_WIDE = 2, TILE_DEEP = 3 };

struct GemmArgs {
  const void* A;      // ak: A(m, k) = A[m lda + k], else A[k lda + m]
  const void* B;      // bk: B(k, n) = B[n ldb + k], else B[k ldb + n]
  int64_t lda, ldb;   // 16-byte aligned operands with rows of whole 16-byte pieces (behind K: zeros)
  int64_t xa, xb;     // rows (ak, bk) or columns that the operands hold: M, N, or padded to whole pieces
  bool ak, bk;
  int64_t M, N, K;
  const float* bias;  // [N] or null
  const void* res;    // [M][N] or null
  float* pre;         // [M][N] or null
  void* out;          // [M][N]
  int act;
  const void* dy;     // [M][N]: out = dy act'(C + bias) instead, and
  float* colpart;     // [linear_col_blocks][N] or null: the sums of its columns over blocks of rows
  bool loose;         // out, res, pre, bias or dy not 16-byte aligned, or N not a whole number of 16-byte pieces
  int tile;           // TILE_*
  int splits;         // parts of the K axis; more than one leave float32 partial sums in `part` [splits][M][N]
  float* part;
};
struct LinearPlan {
  int tile, splits;
};
// whole: the K axis is not cut and dy is taken; wide: the widest tile, which takes neither dy nor `loose`, may be taken
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, size_t es, bool whole, bool wide);
int64_t linear_col_blocks(int tile, int64_t M);  // rows of colpart: one for each wave's rows
template <typename T>
hipError_t launch_gemm(const GemmArgs& a, hipStream_t st);
template <typename T>
hipError_t launch_pack(const void* src, int64_t ld, int64_t rows, int64_t cols, void* dst, int64_t to, hipStream_t st);
// out [R][to] (or none) = dy act'(pre) (pre null: dy), zero from column N on, and, where part is not null, the sums of its
// columns over blocks of rows [linear_row_blocks(R)][N]
int64_t linear_row_blocks(int64_t R);
template <typename T>
hipError_t launch_act_bwd(const void* dy, const float* pre, int act, void* out, int64_t to, float* part, int64_t R, int64_t N,
                          bool loose, hipStream_t st);
hipError_t launch_col_sum(const float* part, int64_t blocks, int64_t N, float* db, hipStream_t st);

// ---------------------------------------------------------------------------
// AdamW over many tensors (states: flat buffers, RES_ADAMW_BLOCK elements a scale)
// ---------------------------------------------------------------------------
struct AdamWArgs {
  const void *m, *v;
  const float *sm, *sv, *master;
  void *m_out, *v_out;
  float *sm_out, *sv_out, *master_out;
  const float* grad_scale;  // [1] or null
  float b1, b1c, b2, b2c, eps;
  float decay;              // 1 - lr weight_decay
  float step;               // lr / (1 - beta1^t)
  float root;               // 1 / sqrt(1 - beta2^t)
};
hipError_t launch_adamw(const AdamWArgs& a, const res_adamw_tensor_t* tensors, int64_t count, bool p_bf16, bool g_bf16,
                        int bits, hipStream_t st);
hipError_t launch_adamw_values(const void* m, const void* v, const float* sm, const float* sv, int64_t n, float* mo,
                               float* vo, hipStream_t st);

}  // namespace res
