// Log probabilities of given tokens, the entropy, the likeliest tokens, and the logits' gradient.  Per row x of V logits,
// with z = scale x, m = max x and S = sum_j exp(scale (x_j - m)):
//   logp = scale (x_token - m) - log S,   H = log S - sum_j e_j d_j / S   (d_j = scale (x_j - m), e_j = exp d_j),
//   dx_j = scale [ dlogp (1{j = token} - p_j) - dH p_j (log p_j + H) ],   p_j = e_j / S.
// m and log S are kept apart: their sum loses what the difference z - m keeps, and overflows where z does.
// The forward reads V elements a row and the backward reads and writes them: memory bounds both.
#include "select.h"

namespace res {
namespace {

constexpr float LN2 = 0.693147180559945309417f;
constexpr float LOWEST = -3.402823466e38f;  // what the running maximum starts from: finite, so that it can be subtracted

// A float's place in the order of values: NaN above all, -0 and 0 the same.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return (b & 0x80000000u) != 0 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) != 0 ? o & 0x7fffffffu : ~o);  // (0xffffffff: a NaN)
}

// The running maximum, the sum of e^(scale (x - m)) and that of d e^d, with d in units of ln 2.
struct Stats {
  float m, s, w;
};
__device__ __forceinline__ void rescale(Stats& a, float m, float c) {  // to a maximum that is not smaller
  if (m > a.m) {
    const float by = (a.m - m) * c, f = exp2_fast(by);
    a.w = f == 0.0f || a.s == 0.0f ? 0.0f : f * fmaf(by, a.s, a.w);  // (by may be -inf)
    a.s *= f;
    a.m = m;
  }
}
__device__ __forceinline__ void join(Stats& a, Stats b, float c) {
  const float m = fmaxf(a.m, b.m);
  rescale(a, m, c);
  rescale(b, m, c);
  a.s += b.s;
  a.w += b.w;
}

constexpr int LIST = 2048;  // candidates kept in LDS: those not below the threshold that the first elements give

struct Shared {
  Stats part[16];
  float top[16];
  int count, finite;
  uint64_t best[16];
  uint32_t order[LIST];
  int at[LIST];
};

// The k-th largest of a wave's 64 values (k <= 64), as an order: bit after bit, how many are not below.
__device__ __forceinline__ uint32_t kth_of_wave(uint32_t o, int k) {
  uint32_t t = 0;
  for (int bit = 31; bit >= 0; --bit) {
    const uint32_t u = t | 1u << bit;
    if (__popcll(__ballot(o >= u)) >= k) t = u;
  }
  return t;
}

// One work-group a row.  Elements go through in one pass, 4 vectors a thread at a time: their maximum first, so that the sums
// are rescaled at most once for them.  For the alternatives the pass keeps those not below a threshold: the largest over the
// waves of the k-th largest of a wave's lanes' maxima over the first vectors, below which no alternative can be.  The list is
// ranked at the end.  Rows whose list overflows (many equal values, values that rise along the row) take one more pass for
// each alternative.
template <typename T, int NT, bool TOP>
__global__ __launch_bounds__(NT) void logprobs_fwd_kernel(LogprobsArgs a) {
  constexpr int V = 16 / (int)sizeof(T), U = 4, W = NT / 64;
  __shared__ Shared sh;
  const int64_t r = a.r0 + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* x = static_cast<const T*>(a.logits) + r * a.ld;
  const float c = a.scale * LOG2E;
  const int64_t N = a.V;
  Stats st{LOWEST, 0.0f, 0.0f};
  float threshold = -INFINITY;
  if (TOP && tid == 0) sh.count = sh.finite = 0;
  for (int64_t base = 0; base < N; base += (int64_t)NT * V * U) {
    T q[U][V];
    int n[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t j = base + ((int64_t)u * NT + tid) * V;
      n[u] = (int)(j >= N ? 0 : N - j < V ? N - j : V);
      load_part<T, V>(x + (n[u] > 0 ? j : 0), n[u], q[u]);
    }
    float v[U][V], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[u][e] = e < n[u] ? to_f32(q[u][e]) : -INFINITY;
        top = fmaxf(top, v[u][e]);
      }
    rescale(st, fmaxf(st.m, top), c);
    float s = 0.0f, w = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = (v[u][e] - st.m) * c, p = exp2_fast(d);
        s += p;
        w = fmaf(p, fmaxf(d, -1024.0f), w);  // (p is 0 there)
      }
    st.s += s;
    st.w += w;
    if constexpr (TOP) {
      if (base == 0) {
        const uint32_t k = kth_of_wave(order_of(top), a.top);
        if (lane == 0) sh.top[wave] = value_of(k);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i) threshold = fmaxf(threshold, sh.top[i]);  // (a NaN is left out)
      }
      // (a NaN is among what is not below; -inf is never listed)
      if (__any(!(top < threshold) || s != s)) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (e < n[u] && !(v[u][e] < threshold) && v[u][e] != -INFINITY) {
              const int k = atomicAdd(&sh.count, 1);
              if (k < LIST) {
                sh.order[k] = order_of(v[u][e]);
                sh.at[k] = (int)(base + ((int64_t)u * NT + tid) * V + e);
              }
            }
      }
    }
  }
  // the work-group's sums: every lane of the wave, then every wave, in a fixed order
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    Stats b{__shfl_xor(st.m, o), __shfl_xor(st.s, o), __shfl_xor(st.w, o)};
    join(st, b, c);
  }
  if (lane == 0) sh.part[wave] = st;
  __syncthreads();
  st = sh.part[0];
#pragma unroll
  for (int i = 1; i < W; ++i) join(st, sh.part[i], c);
  const bool empty = st.s == 0.0f;  // every logit is -inf: no token has a probability
  const float logs = empty ? 0.0f : logf(st.s), m = empty ? -INFINITY : st.m;
  if (tid == 0) {
    const int64_t tok = a.tokens[r];
    float lp = 0.0f;  // an ignored position
    if (tok >= N)
      lp = NAN;
    else if (tok >= 0)
      lp = empty ? -INFINITY : fmaf(a.scale, to_f32(x[tok]) - m, -logs);
    a.logp[r] = lp;
    if (a.stats != nullptr) {
      a.stats[2 * r] = m;
      a.stats[2 * r + 1] = logs;
    }
    if (a.entropy != nullptr) a.entropy[r] = empty ? 0.0f : fmaxf(fmaf(-LN2, st.w / st.s, logs), st.s != st.s ? NAN : 0.0f);
  }
  if constexpr (TOP) {
    int64_t* ids = a.top_ids + r * a.top;
    float* lps = a.top_logp + r * a.top;
    auto lp_of = [&](uint32_t o) { return empty ? -INFINITY : fmaf(a.scale, value_of(o) - m, -logs); };
    const int count = sh.count;
    if (count <= LIST) {
      // an entry's rank: how many are larger, or equal and at a lower place
      for (int i = tid; i < count; i += NT) {
        const uint32_t o = sh.order[i];
        const int at = sh.at[i];
        int rank = 0;
        for (int k = 0; k < count; ++k) rank += sh.order[k] > o || (sh.order[k] == o && sh.at[k] < at);
        if (rank < a.top) {
          ids[rank] = at;
          lps[rank] = lp_of(o);
        }
      }
      // fewer than asked for: then all but -inf are listed, and the lowest places of -inf follow
      if (count < a.top && wave == 0) {
        int have = count;
        for (int64_t j = 0; j < N && have < a.top; j += 64) {
          const bool is = j + lane < N && to_f32(x[j + lane]) == -INFINITY;
          const uint64_t who = __ballot(is);
          const int k = have + __popcll(who & ((1ull << lane) - 1));
          if (is && k < a.top) {
            ids[k] = j + lane;
            lps[k] = lp_of(order_of(-INFINITY));
          }
          have += __popcll(who);
        }
      }
    } else {
      // each time the largest (order, then lowest place) behind the last one found
      uint64_t last = ~0ull;
      for (int k = 0; k < a.top; ++k) {
        uint64_t best = 0;
        for (int64_t j = tid; j < N; j += NT) {
          const uint64_t e = (uint64_t)order_of(to_f32(x[j])) << 32 | (uint32_t)~(uint32_t)j;
          if ((k == 0 || e < last) && e > best) best = e;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const uint64_t b = (uint64_t)__shfl_xor((uint32_t)(best >> 32), o) << 32 | __shfl_xor((uint32_t)best, o);
          best = b > best ? b : best;
        }
        if (lane == 0) sh.best[wave] = best;
        __syncthreads();
        best = sh.best[0];
#pragma unroll
        for (int i = 1; i < W; ++i) best = sh.best[i] > best ? sh.best[i] : best;
        last = best;
        if (tid == 0) {
          ids[k] = (uint32_t)~(uint32_t)best;
          lps[k] = lp_of((uint32_t)(best >> 32));
        }
        __syncthreads();
      }
    }
  }
}

// Rows in pieces: a thread takes 4 vectors.  Reading and writing are the same elements, so that the gradient may take the
// logits' place.
constexpr int BWD_THREADS = 256, BWD_U = 4;

template <typename T>
__global__ __launch_bounds__(BWD_THREADS) void logprobs_bwd_kernel(LogprobsArgs a, uint32_t pieces) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t r = a.r0 + blockIdx.x / pieces;
  const int64_t j0 = (int64_t)(blockIdx.x % pieces) * (BWD_THREADS * V * BWD_U), N = a.V;
  const T* x = static_cast<const T*>(a.logits) + r * a.ld;
  T* out = static_cast<T*>(a.dlogits) + r * a.ldd;
  const int64_t tok = a.tokens[r];
  const float dl = a.dlogp != nullptr && tok >= 0 ? a.dlogp[r] : 0.0f, dh = a.dentropy != nullptr ? a.dentropy[r] : 0.0f;
  const float m = a.stats[2 * r], logs = a.stats[2 * r + 1];
  const bool bad = dl != 0.0f && tok >= N, none = (dl == 0.0f && dh == 0.0f) || m == -INFINITY;
  const float h = a.dentropy != nullptr ? a.entropy[r] : 0.0f;
  const float s = a.scale, sl = s * dl, sh = s * dh;
#pragma unroll
  for (int u = 0; u < BWD_U; ++u) {
    const int64_t j = j0 + ((int64_t)u * BWD_THREADS + threadIdx.x) * V;
    const int n = (int)(j >= N ? 0 : N - j < V ? N - j : V);
    if (n == 0) continue;
    T q[V];
    if (none && !bad) {
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = T(0);
    } else {
      load_part<T, V>(x + j, n, q);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float lp = fmaf(s, to_f32(q[e]) - m, -logs), p = exp2_fast(lp * LOG2E);
        float g = -p * fmaf(sh, fmaxf(lp + h, -1e4f), sl);  // (where lp is -inf, p is 0)
        if (j + e == tok) g += sl;
        q[e] = from_f32<T>(bad ? NAN : g);
      }
    }
    store_part<T, V>(out + j, n, q);
  }
}

template <typename T, int NT>
hipError_t fwd(LogprobsArgs a, hipStream_t st) {
  const int64_t most = LAUNCH_THREADS / NT, R = a.R;
  for (a.r0 = 0; a.r0 < R; a.r0 += most) {
    const uint32_t n = (uint32_t)(R - a.r0 < most ? R - a.r0 : most);
    if (a.top > 0)
      logprobs_fwd_kernel<T, NT, true><<<n, NT, 0, st>>>(a);
    else
      logprobs_fwd_kernel<T, NT, false><<<n, NT, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

template <typename T>
hipError_t launch_logprobs_fwd(LogprobsArgs a, hipStream_t st) {
  return a.V <= 8192 ? fwd<T, 256>(a, st) : fwd<T, 1024>(a, st);
}
template <typename T>
hipError_t launch_logprobs_bwd(LogprobsArgs a, hipStream_t st) {
  constexpr int64_t per = BWD_THREADS * (16 / sizeof(T)) * BWD_U;
  const uint32_t pieces = (uint32_t)((a.V + per - 1) / per);
  const int64_t most = LAUNCH_THREADS / BWD_THREADS / pieces, R = a.R;
  for (a.r0 = 0; a.r0 < R; a.r0 += most) {
    const int64_t n = R - a.r0 < most ? R - a.r0 : most;
    logprobs_bwd_kernel<T><<<(uint32_t)(n * pieces), BWD_THREADS, 0, st>>>(a, pieces);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template hipError_t launch_logprobs_fwd<float>(LogprobsArgs, hipStream_t);
template hipError_t launch_logprobs_fwd<bf16_t>(LogprobsArgs, hipStream_t);
template hipError_t launch_logprobs_bwd<float>(LogprobsArgs, hipStream_t);
template hipError_t launch_logprobs_bwd<bf16_t>(LogprobsArgs, hipStream_t);

}  // namespace res
