// Launch interface of the gated recurrent layer's kernels: the gated scan
// (gated.hip), the linear product with its epilogue (linear.hip) and the AdamW
// step (adamw.hip), between their C entry points (api_layer.hip) and the kernels.
#pragma once

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

// ---------------------------------------------------------------------------
// Gated scan.  A chain is one batch row and one block of GATED_CW channels.
// ---------------------------------------------------------------------------
constexpr int GATED_CW = 64;      // channels of a chain: 128-byte rows of bf16
constexpr int GATED_CARRY = 128;  // steps between the states that a forward keeps for its backward

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
  float* part;          // [B][NB * GATED_CW] partial sums of dgamma
};

template <typename T>
hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t st);
template <typename T>
hipError_t launch_gated_bwd(const GatedArgs& a, float* dgamma, hipStream_t st);
template <typename T>
hipError_t launch_gated_step(const Rows& x, const Rows& r, const Rows& i, void* y, int64_t B, int64_t D,
                             const float* gamma, const float* h, float* h_out, hipStream_t st);

}  // namespace res
