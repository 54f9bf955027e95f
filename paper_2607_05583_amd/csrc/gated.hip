// Gated scan: a diagonal recurrence whose damping depends on the data, per channel
//   s = gamma sigmoid(r_t), a = exp(-s), beta = sqrt(1 - a^2), q = sigmoid(i_t)
//   h_t = a h_{t-1} + beta q x_t,   y_t = h_t
// and its gradients.  With g_t the gradient of h_t (g_t = dy_t + a_{t+1} g_{t+1}),
//   dx = g beta q,   di = g beta q (1 - q) x,   w = g (a^2 / beta q x - a h_{t-1}),
//   dr = w s (1 - sigmoid(r)),   dgamma = sum w sigmoid(r),   dh0 = a_0 g_0.
// Where s = 0 (beta = 0) the derivative of beta is taken as zero.
//
// Both directions are scans of affine maps: steps t0..t1 take h to A h + H with A the
// product of their a, and the adjoint c_t = a_t g_t to A c + C with the same A.  A
// thread owns S consecutive steps of VEC channels in registers, composes their map,
// and gets the state before its first step from the maps of the threads before it
// (LDS); then it runs its steps again from that state.
#include "layer.h"

namespace res {
namespace {

// 1 - exp(-2 s), without the cancellation of 1 - a a for small s: the series of
// 1 - exp(-t) up to t^7 below t = 0.3 (relative error 6e-9 there).
__device__ __forceinline__ float one_minus_a2(float s, float a) {
  const float t = 2.0f * s;
  float p = fmaf(t, -1.0f / 7.0f, 1.0f);
  p = fmaf(t * (-1.0f / 6.0f), p, 1.0f);
  p = fmaf(t * (-1.0f / 5.0f), p, 1.0f);
  p = fmaf(t * (-1.0f / 4.0f), p, 1.0f);
  p = fmaf(t * (-1.0f / 3.0f), p, 1.0f);
  p = fmaf(t * (-1.0f / 2.0f), p, 1.0f);
  return t < 0.3f ? t * p : fmaf(-a, a, 1.0f);
}

// a and 1 / beta (0 where beta is 0) and beta of a step
struct Gate {
  float s, sr, a, beta, rbeta;
};
__device__ __forceinline__ Gate gate(float r, float gamma) {
  Gate g;
  g.sr = sigmoid_fast(r);
  g.s = gamma * g.sr;
  g.a = exp2_fast(-LOG2E * g.s);
  const float e = one_minus_a2(g.s, g.a);
  const bool some = !(e <= 1e-36f);  // NaN stays NaN
  g.rbeta = some ? __builtin_amdgcn_rsqf(e) : 0.0f;
  g.beta = e * g.rbeta;
  return g;
}

template <typename T, int VEC> struct __align__(sizeof(T) * VEC) Vec { T v[VEC]; };

// VEC channels from channel c of a row; channels from D on are zero
template <typename T, int VEC, bool VIO>
__device__ __forceinline__ Vec<T, VEC> load_row(const T* p, int c, int D) {
  Vec<T, VEC> o;
  if constexpr (VIO) {
    if (c < D) return *reinterpret_cast<const Vec<T, VEC>*>(p + c);
#pragma unroll
    for (int v = 0; v < VEC; ++v) o.v[v] = T(0);
  } else {
#pragma unroll
    for (int v = 0; v < VEC; ++v) o.v[v] = c + v < D ? p[c + v] : T(0);
  }
  return o;
}
template <typename T, int VEC, bool VIO>
__device__ __forceinline__ void store_row(T* p, int c, int D, const Vec<T, VEC>& o) {
  if constexpr (VIO) {
    if (c < D) *reinterpret_cast<Vec<T, VEC>*>(p + c) = o;
  } else {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (c + v < D) p[c + v] = o.v[v];
  }
}

__device__ __forceinline__ int row_len(const int* lengths, int64_t b, int64_t L) {
  if (lengths == nullptr) return (int)L;
  const int n = lengths[b];
  return n < 0 ? 0 : n < (int)L ? n : (int)L;
}

// One work-group a chain, tile after tile.
template <typename T, int VEC, int S, int NT, bool VIO>
__global__ __launch_bounds__(NT) void gated_fwd_kernel(GatedArgs A) {
  constexpr int CGL = GATED_CW / VEC, TG = NT / CGL, TILE = S * TG;
  __shared__ float2 agg[TG][GATED_CW];
  __shared__ float enter[GATED_CW];
  const int lane = threadIdx.x % CGL, tg = threadIdx.x / CGL;
  const int64_t b = blockIdx.x / A.NB;
  const int cl = lane * VEC, c = (int)(blockIdx.x % A.NB) * GATED_CW + cl;
  const int len = row_len(A.lengths, b, A.L);
  const int64_t NC = (A.L + GATED_CARRY - 1) / GATED_CARRY;
  float gam[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) gam[v] = c + v < A.D ? A.gamma[c + v] : 0.0f;
  if (tg == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v) enter[cl + v] = A.h0 != nullptr && c + v < A.D ? A.h0[b * A.D + c + v] : 0.0f;
  for (int64_t tile = 0; tile * TILE < A.L; ++tile) {
    const int64_t t0 = tile * TILE + tg * S;
    float a[S][VEC], u[S][VEC];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int64_t t = t0 + s;
      if (t < len) {
        const auto xv = load_row<T, VEC, VIO>((const T*)A.x.p + b * A.x.sb + t * A.x.st, c, A.D);
        const auto rv = load_row<T, VEC, VIO>((const T*)A.r.p + b * A.r.sb + t * A.r.st, c, A.D);
        const auto iv = load_row<T, VEC, VIO>((const T*)A.i.p + b * A.i.sb + t * A.i.st, c, A.D);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const Gate g = gate(to_f32(rv.v[v]), gam[v]);
          a[s][v] = g.a;
          u[s][v] = g.beta * sigmoid_fast(to_f32(iv.v[v])) * to_f32(xv.v[v]);
        }
      } else {
#pragma unroll
        for (int v = 0; v < VEC; ++v) a[s][v] = 1.0f, u[s][v] = 0.0f;
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float pa = 1.0f, ph = 0.0f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        pa *= a[s][v];
        ph = fmaf(a[s][v], ph, u[s][v]);
      }
      agg[tg][cl + v] = make_float2(pa, ph);
    }
    __syncthreads();
    float h[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) h[v] = enter[cl + v];
    for (int g = 0; g < tg; ++g)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float2 m = agg[g][cl + v];
        h[v] = fmaf(m.x, h[v], m.y);
      }
    if (A.carry != nullptr && t0 % GATED_CARRY == 0 && t0 < A.L) {
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (c + v < A.D) A.carry[(b * NC + t0 / GATED_CARRY) * A.D + c + v] = h[v];
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      Vec<T, VEC> o;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        h[v] = fmaf(a[s][v], h[v], u[s][v]);
        o.v[v] = from_f32<T>(t0 + s < len ? h[v] : 0.0f);
      }
      if (A.y != nullptr && t0 + s < A.L) store_row<T, VEC, VIO>((T*)A.y + (b * A.L + t0 + s) * A.D, c, A.D, o);
    }
    __syncthreads();
    if (tg == TG - 1)
#pragma unroll
      for (int v = 0; v < VEC; ++v) enter[cl + v] = h[v];
    __syncthreads();
  }
  if (A.h_out != nullptr && tg == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (c + v < A.D) A.h_out[b * A.D + c + v] = enter[cl + v];
}

// One work-group a chain, from the last tile to the first.  A tile starts at a
// kept state, so only the adjoint is carried from tile to tile.
template <typename T, int VEC, int S, int NT, bool VIO>
__global__ __launch_bounds__(NT) void gated_bwd_kernel(GatedArgs A) {
  constexpr int CGL = GATED_CW / VEC, TG = NT / CGL, TILE = S * TG;
  static_assert(TILE % GATED_CARRY == 0, "a tile starts at a kept state");
  __shared__ float4 agg[TG][GATED_CW];  // A, H, C
  __shared__ float enter[GATED_CW];
  __shared__ double gsum[TG][GATED_CW];
  const int lane = threadIdx.x % CGL, tg = threadIdx.x / CGL;
  const int64_t b = blockIdx.x / A.NB;
  const int cl = lane * VEC, c = (int)(blockIdx.x % A.NB) * GATED_CW + cl;
  const int len = row_len(A.lengths, b, A.L);
  const int64_t NC = (A.L + GATED_CARRY - 1) / GATED_CARRY, tiles = (A.L + TILE - 1) / TILE;
  float gam[VEC];
  double sum[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    gam[v] = c + v < A.D ? A.gamma[c + v] : 0.0f;
    sum[v] = 0.0;
  }
  if (tg == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v) enter[cl + v] = A.dh_out != nullptr && c + v < A.D ? A.dh_out[b * A.D + c + v] : 0.0f;
  for (int64_t tile = tiles - 1; tile >= 0; --tile) {
    const int64_t t0 = tile * TILE + tg * S;
    float x[S][VEC], q[S][VEC], d[S][VEC], hp[S][VEC];
    Gate gt[S][VEC];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int64_t t = t0 + s;
      if (t < len) {
        const auto xv = load_row<T, VEC, VIO>((const T*)A.x.p + b * A.x.sb + t * A.x.st, c, A.D);
        const auto rv = load_row<T, VEC, VIO>((const T*)A.r.p + b * A.r.sb + t * A.r.st, c, A.D);
        const auto iv = load_row<T, VEC, VIO>((const T*)A.i.p + b * A.i.sb + t * A.i.st, c, A.D);
        const auto dv = load_row<T, VEC, VIO>((const T*)A.dy.p + b * A.dy.sb + t * A.dy.st, c, A.D);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          gt[s][v] = gate(to_f32(rv.v[v]), gam[v]);
          x[s][v] = to_f32(xv.v[v]);
          q[s][v] = sigmoid_fast(to_f32(iv.v[v]));
          d[s][v] = to_f32(dv.v[v]);
        }
      } else {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          gt[s][v] = Gate{0.0f, 0.0f, 1.0f, 0.0f, 0.0f};
          x[s][v] = q[s][v] = d[s][v] = 0.0f;
        }
      }
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float pa = 1.0f, ph = 0.0f, pc = 0.0f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const Gate& g = gt[s][v];
        pa *= g.a;
        ph = fmaf(g.a, ph, g.beta * q[s][v] * x[s][v]);
      }
#pragma unroll
      for (int s = S - 1; s >= 0; --s) pc = gt[s][v].a * (d[s][v] + pc);
      agg[tg][cl + v] = make_float4(pa, ph, pc, 0.0f);
    }
    __syncthreads();
    float h[VEC], cc[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = c + v < A.D ? A.carry[(b * NC + tile * (TILE / GATED_CARRY)) * A.D + c + v] : 0.0f;
      cc[v] = enter[cl + v];
    }
    for (int g = 0; g < tg; ++g)
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = fmaf(agg[g][cl + v].x, h[v], agg[g][cl + v].y);
    for (int g = TG - 1; g > tg; --g)
#pragma unroll
      for (int v = 0; v < VEC; ++v) cc[v] = fmaf(agg[g][cl + v].x, cc[v], agg[g][cl + v].z);
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        hp[s][v] = h[v];
        h[v] = fmaf(gt[s][v].a, h[v], gt[s][v].beta * q[s][v] * x[s][v]);
      }
#pragma unroll
    for (int s = S - 1; s >= 0; --s) {
      Vec<T, VEC> ox, orr, oi;
      const bool in = t0 + s < len;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const Gate& k = gt[s][v];
        const float g = d[s][v] + cc[v];
        cc[v] = k.a * g;
        const float gb = g * k.beta * q[s][v];
        const float w = g * fmaf(k.a * k.a * k.rbeta * q[s][v], x[s][v], -k.a * hp[s][v]);
        ox.v[v] = from_f32<T>(in ? gb : 0.0f);
        oi.v[v] = from_f32<T>(in ? gb * (1.0f - q[s][v]) * x[s][v] : 0.0f);
        orr.v[v] = from_f32<T>(in ? w * k.s * (1.0f - k.sr) : 0.0f);
        sum[v] += in ? w * k.sr : 0.0f;
      }
      if (t0 + s < A.L) {
        const int64_t t = t0 + s;
        store_row<T, VEC, VIO>((T*)A.dx.p + b * A.dx.sb + t * A.dx.st, c, A.D, ox);
        store_row<T, VEC, VIO>((T*)A.dr.p + b * A.dr.sb + t * A.dr.st, c, A.D, orr);
        store_row<T, VEC, VIO>((T*)A.di.p + b * A.di.sb + t * A.di.st, c, A.D, oi);
      }
    }
    __syncthreads();
    if (tg == 0)
#pragma unroll
      for (int v = 0; v < VEC; ++v) enter[cl + v] = cc[v];
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) gsum[tg][cl + v] = sum[v];
  __syncthreads();
  if (tg == 0)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (A.dh0 != nullptr && c + v < A.D) A.dh0[b * A.D + c + v] = enter[cl + v];
      double s = 0.0;
      for (int g = 0; g < TG; ++g) s += gsum[g][cl + v];
      A.part[b * ((int64_t)A.NB * GATED_CW) + c + v] = (float)s;
    }
}

// dgamma[c] = sum of the rows of part [n][Dp], in order, in float64
__global__ __launch_bounds__(256) void gated_reduce_kernel(const float* part, int64_t n, int Dp, int D, float* dgamma) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= D) return;
  double s = 0.0;
  for (int64_t k = 0; k < n; ++k) s += part[k * Dp + c];
  dgamma[c] = (float)s;
}

template <typename T>
__global__ __launch_bounds__(256) void gated_step_kernel(Rows x, Rows r, Rows i, T* y, int64_t B, int64_t D,
                                                         const float* gamma, const float* h, float* h_out) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= B * D) return;
  const int64_t b = k / D, c = k - b * D;
  const Gate g = gate(to_f32(((const T*)r.p)[b * r.sb + c]), gamma[c]);
  const float u = g.beta * sigmoid_fast(to_f32(((const T*)i.p)[b * i.sb + c])) * to_f32(((const T*)x.p)[b * x.sb + c]);
  const float v = fmaf(g.a, h[k], u);
  h_out[k] = v;
  y[k] = from_f32<T>(v);
}

}  // namespace

template <typename T>
hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t st) {
  constexpr int VEC = 4, S = 8, NT = 256;
  const dim3 grid((unsigned)(a.B * a.NB));
  if (a.vec)
    gated_fwd_kernel<T, VEC, S, NT, true><<<grid, NT, 0, st>>>(a);
  else
    gated_fwd_kernel<T, VEC, S, NT, false><<<grid, NT, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_gated_bwd(const GatedArgs& a, float* dgamma, hipStream_t st) {
  constexpr int VEC = 4, S = 8, NT = 256;
  const dim3 grid((unsigned)(a.B * a.NB));
  if (a.vec)
    gated_bwd_kernel<T, VEC, S, NT, true><<<grid, NT, 0, st>>>(a);
  else
    gated_bwd_kernel<T, VEC, S, NT, false><<<grid, NT, 0, st>>>(a);
  gated_reduce_kernel<<<dim3((unsigned)((a.D + 255) / 256)), 256, 0, st>>>(a.part, a.B, a.NB * GATED_CW, a.D, dgamma);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_gated_step(const Rows& x, const Rows& r, const Rows& i, void* y, int64_t B, int64_t D,
                             const float* gamma, const float* h, float* h_out, hipStream_t st) {
  gated_step_kernel<T><<<dim3((unsigned)((B * D + 255) / 256)), 256, 0, st>>>(x, r, i, (T*)y, B, D, gamma, h, h_out);
  return hipGetLastError();
}

#define RES_GATED(T)                                                                                          \
  template hipError_t launch_gated_fwd<T>(const GatedArgs&, hipStream_t);                                     \
  template hipError_t launch_gated_bwd<T>(const GatedArgs&, float*, hipStream_t);                             \
  template hipError_t launch_gated_step<T>(const Rows&, const Rows&, const Rows&, void*, int64_t, int64_t,    \
                                           const float*, const float*, float*, hipStream_t);
RES_GATED(float)
RES_GATED(bf16_t)

}  // namespace res
