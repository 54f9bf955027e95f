// Short causal convolution, per channel d:
//   pre_t = sum_{k<K} w[d][k] x_{t-k} + bias[d],  y_t = act(pre_t),
// with x_{-1} .. x_{-(K-1)} the inputs before the call (its state, or zeros), and with
//   dpre_t = dy_t act'(pre_t),  dx_s = sum_k w[k] dpre_{s+k},
//   dw[k] = sum_t dpre_t x_{t-k},  dbias = sum_t dpre_t.
// The forward moves two elements a step and channel, the backward three, for 2 K and 8 K operations: memory bounds both.
// A thread owns a vector of channels over a tile of steps and keeps the last K inputs in registers, so that an input is read
// once and the K - 1 before its tile again.
#include <type_traits>

#include "select.h"

namespace res {
namespace {

// K taps: KX of them where `exact`, else any number up to KX.
template <int KX, bool EXACT> __device__ __forceinline__ bool tap(int k, int K) { return EXACT || k < K; }

template <typename T, int V>
__device__ __forceinline__ void widen(const T (&q)[V], float (&f)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) f[e] = to_f32(q[e]);
}

template <int KX, bool EXACT, int V>
__device__ __forceinline__ void load_taps(const ConvArgs& a, int64_t d, int nd, float (&w)[KX][V], float (&bias)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    bias[e] = a.bias != nullptr && e < nd ? a.bias[d + e] : 0.0f;
#pragma unroll
    for (int k = 0; k < KX; ++k) w[k][e] = e < nd && tap<KX, EXACT>(k, a.K) ? a.w[(d + e) * a.K + k] : 0.0f;
  }
}

template <int KX, bool EXACT, int V>
__device__ __forceinline__ float pre_of(const float (&w)[KX][V], const float* u, int step, int K, int e, float acc) {
  // u: the newest input's element, older ones `step` floats before it
#pragma unroll
  for (int k = 0; k < KX; ++k)
    if (tap<KX, EXACT>(k, K)) acc = fmaf(w[k][e], u[-k * step], acc);
  return acc;
}

// ACT: the activation, or -1 for that of the arguments.  WHOLE: D is a whole number of vectors.
template <int ACT> __device__ __forceinline__ int act_of(const ConvArgs& a) { return ACT < 0 ? a.act : ACT; }

// Rows of V elements, zeros where they are not wanted
template <typename T, int V, bool WHOLE>
__device__ __forceinline__ void load_row(bool wanted, const T* p, int nd, T (&q)[V]) {
  if (wanted)
    load_part<T, V>(p, WHOLE ? V : nd, q);
  else {
#pragma unroll
    for (int e = 0; e < V; ++e) q[e] = T(0);
  }
}

template <typename T, int KX, bool EXACT, int V, int ACT, bool WHOLE>
__global__ __launch_bounds__(CONV_THREADS) void conv_fwd_kernel(ConvArgs a, int64_t nb) {
  constexpr int U = 8, KB = KX - 1;  // steps loaded together, while those before them are computed
  const uint32_t id = blockIdx.x * CONV_THREADS + threadIdx.x, DV = (uint32_t)((a.D + V - 1) / V);
  const uint32_t tiles = (uint32_t)((a.L + a.tile - 1) >> a.shift) + (a.L == 0);
  const uint32_t cv = id % DV, rest = id / DV, tile = rest % tiles;
  if (rest / tiles >= (uint64_t)nb) return;
  const int64_t b = a.b0 + rest / tiles, d = (int64_t)cv * V, t0 = (int64_t)tile << a.shift;
  const int nd = (int)(a.D - d < V ? a.D - d : V), K = EXACT ? KX : a.K;
  int64_t n = a.L;
  if (a.lengths != nullptr) {
    n = a.lengths[b];
    n = n < 0 ? 0 : n > a.L ? a.L : n;
  }
  const T* x = static_cast<const T*>(a.x.p) + b * a.x.sb + d;
  const T* st = a.state != nullptr ? static_cast<const T*>(a.state) + b * (K - 1) * a.D + d : nullptr;
  auto input = [&](int64_t t, T(&q)[V]) {  // x_t, of the state where t < 0
    if (t >= 0)
      load_row<T, V, WHOLE>(true, x + t * a.x.st, nd, q);
    else
      load_row<T, V, WHOLE>(st != nullptr && t >= 1 - K, st + (t + K - 1) * a.D, nd, q);
  };
  const int in = (int)(n - t0 < 0 ? 0 : n - t0 < a.tile ? n - t0 : a.tile);         // the tile's steps
  const int end = (int)(a.L - t0 < a.tile ? a.L - t0 : a.tile);                     // its rows
  const T* xt = x + t0 * a.x.st;
  const uint32_t sx = (uint32_t)a.x.st, sy = (uint32_t)a.D;  // (within a tile offsets have 32 bits)
  T q[U][V];
#pragma unroll
  for (int s = 0; s < U; ++s) load_row<T, V, WHOLE>(s < in, xt + (uint32_t)s * sx, nd, q[s]);
  float f[KB + U][V];  // the inputs before the steps at hand, and theirs
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    T q[V] = {};
    if ((in > 0 || tile == 0) && tap<KX, EXACT>(KB - k, K)) input(t0 - KB + k, q);  // (the K - 1 before)
    widen<T, V>(q, f[k]);
  }
  // state_out may be the state: a thread has read its channels of it before it writes them, and then the first tile's threads alone
  // read it (a.tile >= K - 1).
  if (tile == 0 && a.state_out != nullptr) {
    T last[KB > 0 ? KB : 1][V];
#pragma unroll
    for (int j = 0; j < KB; ++j)
      if (tap<KX, EXACT>(j + 1, K)) input(n - (K - 1) + j, last[j]);
    T* so = static_cast<T*>(a.state_out) + b * (K - 1) * a.D + d;
#pragma unroll
    for (int j = 0; j < KB; ++j)
      if (tap<KX, EXACT>(j + 1, K)) store_part<T, V>(so + j * a.D, nd, last[j]);
  }
  float w[KX][V], bias[V];
  load_taps<KX, EXACT, V>(a, d, nd, w, bias);
  T* y = static_cast<T*>(a.y) + (b * a.L + t0) * a.D + d;
  for (int t = 0; t < end; t += U) {
#pragma unroll
    for (int s = 0; s < U; ++s) widen<T, V>(q[s], f[KB + s]);
    if (t + U < in)
#pragma unroll
      for (int s = 0; s < U; ++s) load_row<T, V, WHOLE>(t + U + s < in, xt + (uint32_t)(t + U + s) * sx, nd, q[s]);
#pragma unroll
    for (int s = 0; s < U; ++s) {
      T out[V];
#pragma unroll
      for (int e = 0; e < V; ++e)
        out[e] = t + s < in ? from_f32<T>(act_value(pre_of<KX, EXACT, V>(w, &f[KB + s][e], V, K, e, bias[e]), act_of<ACT>(a))) : T(0);
      if (t + s < end) store_part<T, V>(y + (uint32_t)(t + s) * sy, WHOLE ? V : nd, out);
    }
#pragma unroll
    for (int k = 0; k < KB; ++k)
#pragma unroll
      for (int e = 0; e < V; ++e) f[k][e] = f[k + U][e];
  }
}

// The backward's thread goes through its tile's steps and the K - 1 behind them: dpre of each (pre again from the inputs) enters
// a window, and dx of the step K - 1 before it leaves.  The first tile goes on with the state's gradients.
template <typename T, int KX, bool EXACT, int V, int ACT, bool WHOLE>
__global__ __launch_bounds__(CONV_THREADS) void conv_bwd_kernel(ConvArgs a, uint32_t blocks_d) {
  constexpr int U = 4, KB = KX - 1, CW = CONV_BWD_CHANNELS, LANES = CW / V, RB = CONV_THREADS / LANES;
  static_assert(RB * LANES == CONV_THREADS && RB <= CONV_BWD_ROWS && CONV_BWD_ROWS % RB == 0, "whole rows of threads");
  __shared__ float red[RB][CW];
  const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const uint32_t bd = blockIdx.x % blocks_d;
  const int64_t by = a.b0 + blockIdx.x / blocks_d;  // (b0: the launch's first block of rows)
  const int64_t tiles = ((a.L + a.tile - 1) >> a.shift) + (a.L == 0);
  const int64_t d = (int64_t)bd * CW + lane * V;
  const int nd = (int)(d >= a.D ? 0 : a.D - d < V ? a.D - d : V), K = EXACT ? KX : a.K;
  float w[KX][V], bias[V], dw[KX][V], db[V];
  load_taps<KX, EXACT, V>(a, d, nd, w, bias);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    db[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < KX; ++k) dw[k][e] = 0.0f;
  }
  for (int r = sub; r < CONV_BWD_ROWS; r += RB) {
    const int64_t row = by * CONV_BWD_ROWS + r, b = row / tiles, t0 = (row % tiles) << a.shift;
    if (nd == 0 || b >= a.B) continue;
    int64_t n = a.L;
    if (a.lengths != nullptr) {
      n = a.lengths[b];
      n = n < 0 ? 0 : n > a.L ? a.L : n;
    }
    // the tile's steps, its rows, and the steps that are there behind it
    const int in = (int)(n - t0 < 0 ? 0 : n - t0 < a.tile ? n - t0 : a.tile);
    const int held = (int)(a.L - t0 < a.tile ? a.L - t0 : a.tile);
    const int seen = (int)(n - t0 < 0 ? 0 : n - t0 < a.tile + K - 1 ? n - t0 : a.tile + K - 1);
    const T* x = static_cast<const T*>(a.x.p) + b * a.x.sb + t0 * a.x.st + d;
    const T* dy = static_cast<const T*>(a.dy.p) + b * a.dy.sb + t0 * a.dy.st + d;
    T* dx = static_cast<T*>(a.dx.p) + b * a.dx.sb + t0 * a.dx.st + d;
    const uint32_t sx = (uint32_t)a.x.st, sy = (uint32_t)a.dy.st, sd = (uint32_t)a.dx.st;
    const int64_t so = b * (K - 1) * a.D + d;
    const T* dso = a.dstate_out != nullptr ? static_cast<const T*>(a.dstate_out) + so : nullptr;
    const int64_t into = n - t0;                    // (step `into` of the tile is the row's end)
    const int first = t0 > 0 ? 0 : 1 - K;           // the first input whose gradient is made here
    T qx[U][V], qy[U][V];
    auto load = [&](int t) {
#pragma unroll
      for (int s = 0; s < U; ++s) {
        load_row<T, V, WHOLE>(t + s < seen, x + (uint32_t)(t + s) * sx, nd, qx[s]);
        load_row<T, V, WHOLE>(t + s < seen, dy + (uint32_t)(t + s) * sy, nd, qy[s]);
      }
    };
    load(0);
    float f[KB + U][V], g[KB + U][V];
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      T q[V] = {};
      const int64_t t = t0 - KB + k;
      if (t >= 0 && t < n)
        load_row<T, V, WHOLE>(true, x + (int64_t)(k - KB) * a.x.st, nd, q);
      else if (t < 0 && a.state != nullptr && t >= 1 - K)
        load_row<T, V, WHOLE>(true, static_cast<const T*>(a.state) + so + (t + K - 1) * a.D, nd, q);
      widen<T, V>(q, f[k]);
#pragma unroll
      for (int e = 0; e < V; ++e) g[k][e] = 0.0f;
    }
    for (int t = 0; t < in + K - 1; t += U) {
#pragma unroll
      for (int s = 0; s < U; ++s) {
        widen<T, V>(qx[s], f[KB + s]);
        widen<T, V>(qy[s], g[KB + s]);
      }
      if (t + U < in + K - 1) load(t + U);
#pragma unroll
      for (int s = 0; s < U; ++s) {
        const bool own = t + s < in;  // (later steps are another tile's)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float pre = pre_of<KX, EXACT, V>(w, &f[KB + s][e], V, K, e, bias[e]);
          const float dpre = t + s < seen ? g[KB + s][e] * act_slope(pre, act_of<ACT>(a)) : 0.0f;
          g[KB + s][e] = dpre;
          const float mine = own ? dpre : 0.0f;
          db[e] += mine;
          if (own)
#pragma unroll
            for (int k = 0; k < KX; ++k)
              if (tap<KX, EXACT>(k, K)) dw[k][e] = fmaf(mine, f[KB + s - k][e], dw[k][e]);
        }
        const int at = t + s - (K - 1);  // the input whose gradient is complete
        if (at >= first && at < in) {
          float du[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            du[e] = 0.0f;
            // g of step at + k is K - 1 - k places before the newest
            if constexpr (EXACT) {
#pragma unroll
              for (int k = 0; k < KX; ++k) du[e] = fmaf(w[k][e], g[s + k][e], du[e]);
            } else {
#pragma unroll
              for (int j = 0; j < KX; ++j)  // j = K - 1 - k
                if (j < K) {
                  float wk = 0.0f;
#pragma unroll
                  for (int k = 0; k < KX; ++k)
                    if (k == K - 1 - j) wk = w[k][e];
                  du[e] = fmaf(wk, g[KB + s - j][e], du[e]);
                }
            }
          }
          if (dso != nullptr && at + (K - 1) >= into) {  // its place in the state that the call leaves
            T q[V];
            load_row<T, V, WHOLE>(true, dso + (at + (K - 1) - into) * a.D, nd, q);
#pragma unroll
            for (int e = 0; e < V; ++e) du[e] += to_f32(q[e]);
          }
          T q[V];
#pragma unroll
          for (int e = 0; e < V; ++e) q[e] = from_f32<T>(du[e]);
          if (at >= 0)
            store_part<T, V>(dx + (uint32_t)at * sd, WHOLE ? V : nd, q);
          else if (a.dstate != nullptr)
            store_part<T, V>(static_cast<T*>(a.dstate) + so + (at + K - 1) * a.D, WHOLE ? V : nd, q);
        }
      }
#pragma unroll
      for (int k = 0; k < KB; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          f[k][e] = f[k + U][e];
          g[k][e] = g[k + U][e];
        }
    }
    T zero[V] = {};
    for (int t = in; t < held; ++t) store_part<T, V>(dx + (uint32_t)t * sd, WHOLE ? V : nd, zero);
  }
  // the block's sums, in the order of its rows
  for (int k = 0; k <= K; ++k) {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      v[e] = db[e];
#pragma unroll
      for (int j = 0; j < KX; ++j)
        if (j == k && tap<KX, EXACT>(j, K)) v[e] = dw[j][e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < V; ++e) red[sub][lane * V + e] = v[e];
    __syncthreads();
    if (threadIdx.x < CW && (int64_t)bd * CW + threadIdx.x < a.D) {
      float s = 0.0f;
#pragma unroll
      for (int r = 0; r < RB; ++r) s += red[r][threadIdx.x];
      a.part[(by * (K + 1) + k) * a.D + (int64_t)bd * CW + threadIdx.x] = s;
    }
  }
}

// dw [D][K] and dbias [D] from the blocks' sums: 16 channels of a tap a work-group, 16 threads a channel that take the blocks in turn.
__global__ __launch_bounds__(256) void conv_sum_kernel(const float* part, int64_t blocks, int64_t D, int K, float* dw, float* dbias,
                                                        uint32_t blocks_d) {
  __shared__ double red[16][17];
  const int c = threadIdx.x % 16, j = threadIdx.x / 16, k = (int)(blockIdx.x / blocks_d);
  const int64_t d = (int64_t)(blockIdx.x % blocks_d) * 16 + c;
  double s = 0.0;
  if (d < D)
    for (int64_t r = j; r < blocks; r += 16) s += (double)part[(r * (K + 1) + k) * D + d];
  red[j][c] = s;
  __syncthreads();
  if (j == 0 && d < D) {
    for (int i = 1; i < 16; ++i) s += red[i][c];
    if (k < K)
      dw[d * K + k] = (float)s;
    else if (dbias != nullptr)
      dbias[d] = (float)s;
  }
}

template <typename T, int KX, bool EXACT, int V>
__global__ __launch_bounds__(CONV_THREADS) void conv_step_kernel(ConvArgs a, int64_t nb) {
  constexpr int KB = KX - 1;
  const uint32_t id = blockIdx.x * CONV_THREADS + threadIdx.x, DV = (uint32_t)((a.D + V - 1) / V);
  if (id / DV >= (uint64_t)nb) return;
  const int64_t b = a.b0 + id / DV, d = (int64_t)(id % DV) * V;
  const int nd = (int)(a.D - d < V ? a.D - d : V), K = EXACT ? KX : a.K;
  const int64_t so = b * (K - 1) * a.D + d;
  T q[KX][V];  // q[k]: the input k steps back
  load_part<T, V>(static_cast<const T*>(a.x.p) + b * a.x.sb + d, nd, q[0]);
#pragma unroll
  for (int k = 1; k < KX; ++k)
    if (tap<KX, EXACT>(k, K)) load_part<T, V>(static_cast<const T*>(a.state) + so + (K - 1 - k) * a.D, nd, q[k]);
  float w[KX][V], bias[V];
  load_taps<KX, EXACT, V>(a, d, nd, w, bias);
  T y[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float s = bias[e];
#pragma unroll
    for (int k = 0; k < KX; ++k)
      if (tap<KX, EXACT>(k, K)) s = fmaf(w[k][e], to_f32(q[k][e]), s);
    y[e] = from_f32<T>(act_value(s, a.act));
  }
  store_part<T, V>(static_cast<T*>(a.y) + b * a.D + d, nd, y);
#pragma unroll
  for (int k = 0; k < KB; ++k)  // the state moves on by one: what was k back is k + 1 back
    if (tap<KX, EXACT>(k + 1, K)) store_part<T, V>(static_cast<T*>(a.state_out) + so + (K - 2 - k) * a.D, nd, q[k]);
}

// Launches of whole batch rows of `per` threads each, as many as 2^32 threads allow.
template <typename F>
hipError_t by_rows(int64_t B, int64_t per, F&& launch) {
  const int64_t most = (LAUNCH_THREADS - CONV_THREADS) / per;  // (1 at least: a row beyond one launch is refused before)
  for (int64_t b0 = 0; b0 < B; b0 += most) {
    const int64_t nb = B - b0 < most ? B - b0 : most;
    launch(b0, nb, (uint32_t)((nb * per + CONV_THREADS - 1) / CONV_THREADS));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// F with the number of taps as a constant up to four, which the windows of a model's convolutions have; any other at run time (65536
// steps of 640 channels, bf16: 137 us forward and 259 backward with 7 and with 16 taps, 46 and 53 with four).
template <typename F>
auto by_taps(int K, F&& f) {
  switch (K) {
    case 1: return f(std::integral_constant<int, 1>{}, std::true_type{});
    case 2: return f(std::integral_constant<int, 2>{}, std::true_type{});
    case 3: return f(std::integral_constant<int, 3>{}, std::true_type{});
    case 4: return f(std::integral_constant<int, 4>{}, std::true_type{});
    default: return f(std::integral_constant<int, CONV_TAPS>{}, std::false_type{});
  }
}

// Channels of a thread: two, so that a thread's windows leave room for many waves on a compute unit, whose loads cover each
// other's latency.  65536 steps of 640 channels, bf16: forward 50 us (3.4 TB/s; with four channels 55), backward 55 us
// (4.5 TB/s).
constexpr int CONV_VEC = 2;
// Steps of a thread: many read few inputs twice and make few partial sums; with too few threads for the chip a thread's chain of loads
// is the call's time.  5 x 2001 steps of 203 channels, float32: 32 forward and 64 backward 13 and 29 us, 8 and 8 take 8 and 11 us.

// F with the taps, whether the activation is silu, and whether D is whole vectors, as constants.
template <typename F>
hipError_t by_kind(const ConvArgs& a, F&& f) {
  return by_taps(a.K, [&](auto kx, auto exact) {
    if constexpr (exact) {
      if (a.act == ACT_SILU)
        return a.D % CONV_VEC == 0 ? f(kx, exact, std::integral_constant<int, ACT_SILU>{}, std::true_type{})
                            : f(kx, exact, std::integral_constant<int, ACT_SILU>{}, std::false_type{});
      return a.D % CONV_VEC == 0 ? f(kx, exact, std::integral_constant<int, -1>{}, std::true_type{})
                          : f(kx, exact, std::integral_constant<int, -1>{}, std::false_type{});
    } else {
      return f(kx, exact, std::integral_constant<int, -1>{}, std::false_type{});
    }
  });
}

}  // namespace

template <typename T>
hipError_t launch_conv_fwd(ConvArgs a, hipStream_t st) {
  const int64_t threads = a.B * ((a.D + CONV_VEC - 1) / CONV_VEC);
  const int least = a.state != nullptr && a.state_out == a.state ? conv_least(a.K) : CONV_LEAST;
  a.shift = conv_shift(CONV_SHIFT, least, a.L, [&](int64_t tiles) { return threads * tiles / CONV_THREADS; });
  a.tile = 1 << a.shift;
  return by_kind(a, [&](auto kx, auto exact, auto act, auto whole) {
    constexpr int V = CONV_VEC;
    const int64_t tiles = conv_tiles(a.L, a.shift);
    return by_rows(a.B, tiles * ((a.D + V - 1) / V), [&](int64_t b0, int64_t nb, uint32_t grid) {
      a.b0 = b0;
      conv_fwd_kernel<T, kx, exact, V, act, whole><<<grid, CONV_THREADS, 0, st>>>(a, nb);
    });
  });
}
template <typename T>
hipError_t launch_conv_step(ConvArgs a, hipStream_t st) {
  return by_taps(a.K, [&](auto kx, auto exact) {
    constexpr int V = CONV_VEC;
    return by_rows(a.B, (a.D + V - 1) / V, [&](int64_t b0, int64_t nb, uint32_t grid) {
      a.b0 = b0;
      conv_step_kernel<T, kx, exact, V><<<grid, CONV_THREADS, 0, st>>>(a, nb);
    });
  });
}
template <typename T>
hipError_t launch_conv_bwd(const ConvArgs& a, hipStream_t st) {
  const int shift = conv_bwd_shift(a.B, a.L, a.D);
  const int64_t rows = conv_row_blocks(a.B, a.L, shift);
  const uint32_t bd = (uint32_t)((a.D + CONV_BWD_CHANNELS - 1) / CONV_BWD_CHANNELS);
  const hipError_t e = by_kind(a, [&](auto kx, auto exact, auto act, auto whole) {
    const int64_t most = LAUNCH_THREADS / CONV_THREADS / bd;
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
      ConvArgs c = a;
      c.b0 = r0;
      c.shift = shift;
      c.tile = 1 << shift;
      const int64_t n = rows - r0 < most ? rows - r0 : most;
      conv_bwd_kernel<T, kx, exact, CONV_VEC, act, whole><<<(uint32_t)(n * bd), CONV_THREADS, 0, st>>>(c, bd);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
  if (e != hipSuccess) return e;
  const uint32_t sd = (uint32_t)((a.D + 15) / 16);
  conv_sum_kernel<<<sd * (uint32_t)(a.K + 1), 256, 0, st>>>(a.part, rows, a.D, a.K, a.dw, a.dbias, sd);
  return hipGetLastError();
}

template hipError_t launch_conv_fwd<float>(ConvArgs, hipStream_t);
template hipError_t launch_conv_fwd<bf16_t>(ConvArgs, hipStream_t);
template hipError_t launch_conv_bwd<float>(const ConvArgs&, hipStream_t);
template hipError_t launch_conv_bwd<bf16_t>(const ConvArgs&, hipStream_t);
template hipError_t launch_conv_step<float>(ConvArgs, hipStream_t);
template hipError_t launch_conv_step<bf16_t>(ConvArgs, hipStream_t);

}  // namespace res
