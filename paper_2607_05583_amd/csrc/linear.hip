// Linear product with bias, activation and residual, and its gradients:
//   pre = x W + b, y = act(pre) + residual;
//   dpre = dy act'(pre), dx = dpre W^T, dW = x^T dpre, db = sum over rows of dpre.
// All three products are one kernel over strided operands; sums are float32 (MFMA).
#include "layer.h"

namespace res {
namespace {

// What a product's element becomes: the epilogue of its row m and column n.
template <typename T>
__device__ __forceinline__ void finish(const GemmArgs& g, int64_t m, int64_t n, float c) {
  const int64_t at = m * g.N + n;
  if (g.bias != nullptr) c += g.bias[n];
  if (g.pre != nullptr) g.pre[at] = c;
  c = act_value(c, g.act);
  if (g.res != nullptr) c += to_f32(((const T*)g.res)[at]);
  ((T*)g.out)[at] = from_f32<T>(c);
}

// Any sizes, strides and alignments: 64 x 64 outputs of a work-group of four waves
// (32 x 32 each), 32 terms of the sum at a time through LDS, both operands with the
// terms of a row or column side by side.
template <typename T>
__global__ __launch_bounds__(256) void gemm_any_kernel(GemmArgs g) {
  constexpr int BM = 64, BK = 32, PAD = 16 / sizeof(T), LD = BK + PAD;
  __shared__ __align__(16) T sa[BM * LD], sb[BM * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int li = lane & 15, lq = lane >> 4;
  const int64_t tn = (g.N + BM - 1) / BM;
  const int64_t m0 = (blockIdx.x / tn) * BM, n0 = (blockIdx.x % tn) * BM;
  const int64_t per = ((g.K + g.splits - 1) / g.splits + BK - 1) / BK * BK;
  const int64_t k0 = blockIdx.y * per, k1 = k0 + per < g.K ? k0 + per : g.K;
  f4 acc[2][2] = {};
  for (int64_t k = k0; k < k1; k += BK) {
#pragma unroll
    for (int e = 0; e < BM * BK / 256; ++e) {
      const int id = e * 256 + tid;
      const int am = g.sak == 1 ? id / BK : id % BM, ak = g.sak == 1 ? id % BK : id / BM;
      const int bn = g.sbk == 1 ? id / BK : id % BM, bk = g.sbk == 1 ? id % BK : id / BM;
      sa[am * LD + ak] = m0 + am < g.M && k + ak < k1 ? ((const T*)g.A)[(m0 + am) * g.sam + (k + ak) * g.sak] : T(0);
      sb[bn * LD + bk] = n0 + bn < g.N && k + bk < k1 ? ((const T*)g.B)[(k + bk) * g.sbk + (n0 + bn) * g.sbn] : T(0);
    }
    __syncthreads();
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bf8 a = *reinterpret_cast<const bf8*>(&sa[(wm + i * 16 + li) * LD + lq * 8]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf8 b = *reinterpret_cast<const bf8*>(&sb[(wn + j * 16 + li) * LD + lq * 8]);
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc[i][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < BK; h += 16)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f4 a = *reinterpret_cast<const f4*>(&sa[(wm + i * 16 + li) * LD + h + lq * 4]);
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = mma_f32(a, *reinterpret_cast<const f4*>(&sb[(wn + j * 16 + li) * LD + h + lq * 4]), acc[i][j]);
        }
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + (wave >> 1) * 32 + i * 16 + lq * 4 + r, n = n0 + (wave & 1) * 32 + j * 16 + li;
        if (m < g.M && n < g.N) {
          if (g.splits > 1)
            g.part[(blockIdx.y * g.M + m) * g.N + n] = acc[i][j][r];
          else
            finish<T>(g, m, n, acc[i][j][r]);
        }
      }
}

// the parts of a split sum, in order, then the epilogue
template <typename T>
__global__ __launch_bounds__(256) void gemm_join_kernel(GemmArgs g) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, n = g.M * g.N;
  if (id >= n) return;
  float c = 0.0f;
  for (int s = 0; s < g.splits; ++s) c += g.part[s * n + id];
  finish<T>(g, id / g.N, id % g.N, c);
}

// dpre and the sums of its columns: a work-group takes ACT_ROWS rows of 256 columns
constexpr int ACT_ROWS = 128;
template <typename T>
__global__ __launch_bounds__(256) void act_bwd_kernel(const T* dy, const float* pre, int act, T* out, float* part, int64_t R,
                                                      int64_t N) {
  const int64_t cols = (N + 255) / 256, block = blockIdx.x / cols;
  const int64_t n = (blockIdx.x % cols) * 256 + threadIdx.x, r0 = block * ACT_ROWS;
  if (n >= N) return;
  float sum = 0.0f;
  for (int64_t r = r0; r < R && r < r0 + ACT_ROWS; ++r) {
    const float d = to_f32(dy[r * N + n]) * (pre != nullptr ? act_slope(pre[r * N + n], act) : 1.0f);
    if (out != nullptr) out[r * N + n] = from_f32<T>(d);
    sum += d;
  }
  if (part != nullptr) part[block * N + n] = sum;
}
__global__ __launch_bounds__(256) void col_sum_kernel(const float* part, int64_t blocks, int64_t N, float* db) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= N) return;
  double s = 0.0;
  for (int64_t b = 0; b < blocks; ++b) s += part[b * N + n];
  db[n] = (float)s;
}

}  // namespace

int64_t linear_row_blocks(int64_t R) { return (R + ACT_ROWS - 1) / ACT_ROWS; }

// Parts of the K axis, so that about 512 work-groups run where the outputs alone give
// fewer; a part has at least 256 terms.
int64_t linear_splits(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64);
  int64_t s = tiles > 0 ? 512 / tiles : 1;
  if (s > K / 256) s = K / 256;
  return s < 1 ? 1 : s > 64 ? 64 : s;
}

template <typename T>
hipError_t launch_gemm(const GemmArgs& a, hipStream_t st) {
  const int64_t tiles = ((a.M + 63) / 64) * ((a.N + 63) / 64);
  gemm_any_kernel<T><<<dim3((unsigned)tiles, (unsigned)a.splits), 256, 0, st>>>(a);
  if (a.splits > 1) gemm_join_kernel<T><<<dim3((unsigned)((a.M * a.N + 255) / 256)), 256, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_act_bwd(const void* dy, const float* pre, int act, void* out, float* part, float* db, int64_t R,
                          int64_t N, hipStream_t st) {
  const int64_t blocks = linear_row_blocks(R);
  if (blocks > 0)
    act_bwd_kernel<T><<<dim3((unsigned)((N + 255) / 256 * blocks)), 256, 0, st>>>(
        (const T*)dy, pre, act, (T*)out, part, R, N);
  if (db != nullptr) col_sum_kernel<<<dim3((unsigned)((N + 255) / 256)), 256, 0, st>>>(part, blocks, N, db);
  return hipGetLastError();
}

#define RES_LINEAR(T)                                                                                        \
  template hipError_t launch_gemm<T>(const GemmArgs&, hipStream_t);                                          \
  template hipError_t launch_act_bwd<T>(const void*, const float*, int, void*, float*, float*, int64_t, int64_t, hipStream_t);
RES_LINEAR(float)
RES_LINEAR(bf16_t)

}  // namespace res
