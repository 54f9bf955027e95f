// Log probabilities of given tokens, the entropy, the likeliest tokens, and the logits' gradient.  Per row x of V logits,
// with z = scale x, m = max x and S = sum_j exp(scale (x_j - m)):
//   logp = scale (x_token - m) - log S,   H = log S - sum_j e_j d_j / S   (d_j = scale (x_j - m), e_j = exp d_j),
//   dx_j = scale [ dlogp (1{j = token} - p_j) - dH p_j (log p_j + H) ],   p_j = e_j / S.
// m and log S are kept apart: their sum loses what the difference z - m keeps, and overflows where z does.
// The forward reads V elements a row and the backward reads and writes them: memory bounds both (8192 x 50304 bf16: 431 us for the two
// in turn, 5.7 TB/s; in traces 166 to 191 and 249 to 304 us from run to run).
#include <type_traits>

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

// The order of a bf16 value from its upper half: the lower one is zeros, below zero ones (and NaN's all ones).
__device__ __forceinline__ uint32_t whole_order(uint32_t o) { return (o & 0x80000000u) == 0 || o == 0xffff0000u ? o | 0xffffu : o; }

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

constexpr int LIST = 1536, EQUAL = 512;  // alternatives' candidates kept in LDS; those of them at the border itself

struct Shared {
  uint32_t kth[8], share[8], border;
  uint32_t tops[512];  // lanes' maxima not below the first border
  int lane[512];       // the lanes whose elements are looked at again
  int count, above, equal, lanes, again;
  uint64_t list[LIST];  // order << 32 | ~place: the larger one comes first
};

__device__ __forceinline__ uint64_t entry_of(float v, int64_t at) { return (uint64_t)order_of(v) << 32 | (uint32_t)~(uint32_t)at; }

// The k-th and the j-th largest of a wave's 64 orders (k, j <= 64), bit after bit: how many are not below.  (A loop: run once
// by each wave, unrolled it took 0.7 us more of 18 for 64 rows of 50304 with 1024 threads.)  HALF: the orders are of bf16 values.
template <bool HALF>
__device__ __forceinline__ void kth_of_wave(uint32_t o, int k, int j, uint32_t* kth, uint32_t* jth) {
  uint32_t t = 0, s = 0;
#pragma unroll 1
  for (int bit = 31; bit >= (HALF ? 16 : 0); --bit) {
    const uint32_t u = t | 1u << bit, v = s | 1u << bit;
    const int above = __popcll(__ballot(o >= u)), also = __popcll(__ballot(o >= v));
    t = above >= k ? u : t;
    s = also >= j ? v : s;
  }
  *kth = HALF ? whole_order(t) : t;
  *jth = HALF ? whole_order(s) : s;
}

// A row's elements, some vectors a thread at a time.
template <typename T, int NT, int UV> struct RowPiece {
  static constexpr int V = 16 / (int)sizeof(T), U = UV, STEP = NT * V * U;
  T q[U][V];
  __device__ __forceinline__ static int64_t at(int64_t base, int u) { return base + ((int64_t)u * NT + threadIdx.x) * V; }
  // -inf behind the row's end
  __device__ __forceinline__ void load(const T* x, int64_t base, int64_t N) {
    if (base + STEP <= N) {
#pragma unroll
      for (int u = 0; u < U; ++u) load_part<T, V>(x + at(base, u), V, q[u]);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t j = at(base, u);
#pragma unroll
        for (int e = 0; e < V; ++e) q[u][e] = from_f32<T>(-INFINITY);
        if (j + V <= N)
          load_part<T, V>(x + j, V, q[u]);
        else
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (j + e < N) q[u][e] = x[j + e];
      }
    }
  }
};

// One work-group a row, whose elements go through in one pass, the next ones loaded while these are added: their maximum first,
// so that the sums are rescaled at most once for them.
// Alternatives: no alternative is below the k-th largest of the lanes' maxima (the border), and only the lanes whose maximum is
// not below it, some k of them, have any, so that their elements alone are looked at again (k of 256 lanes: 8 % of the row for 20
// alternatives).  The lanes are few from the start: not below the largest of the waves' own k-th
// largest, nor below the least of their (k / waves)-th largest.  What is found is
// ranked in LDS.  Many elements at the border itself (a mask's value) are not all listed: those missing are its lowest places.
// Rows with NaN or infinity, or with more than LIST elements above the border, find the k-th largest by counting.
template <typename T, int NT, bool TOP, bool ENT>
__global__ __launch_bounds__(NT) void logprobs_fwd_kernel(LogprobsArgs a) {
  typedef RowPiece<T, NT, 4> Piece;
  constexpr int V = Piece::V, U = Piece::U, W = NT / 64;
  static_assert(NT <= 512 && W <= 8, "the shared arrays");
  __shared__ Stats part[W];
  extern __shared__ __align__(16) char raw[];
  Shared& sh = *reinterpret_cast<Shared*>(raw);  // (with alternatives only)
  const int64_t r = a.r0 + blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const T* x = static_cast<const T*>(a.logits) + r * a.ld;
  const float c = a.scale * LOG2E;
  const int64_t N = a.V;
  Stats st{LOWEST, 0.0f, 0.0f};
  float most = -INFINITY;
  if (TOP && tid == 0) sh.count = sh.above = sh.equal = sh.lanes = sh.again = 0;
  Piece next;
  next.load(x, 0, N);
  for (int64_t base = 0; base < N; base += Piece::STEP) {
    const Piece p = next;
    if (base + Piece::STEP < N) next.load(x, base + Piece::STEP, N);
    float v[U][V], top = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        v[u][e] = to_f32(p.q[u][e]);
        top = fmaxf(top, v[u][e]);
      }
    most = fmaxf(most, top);
    rescale(st, fmaxf(st.m, top), c);
    // d = c x - c m with one rounding of its own; that of c m is taken out of the sums at once, since it is the same for all.
    // (Where c m is next to float32's end, or is none, the difference is taken first.)
    const float cm = st.m * c;
    const bool far = !(fabsf(cm) < 1e30f);
    const float mc = far ? 0.0f : cm, fix = far ? 0.0f : fmaf(st.m, c, -mc);
    float s = 0.0f, w = 0.0f;
    auto add = [&](float d) {
      const float f = exp2_fast(d);
      s += f;
      if (ENT) w = fmaf(f, fmaxf(d, -1024.0f), w);  // (f is 0 there)
    };
    if (far) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) add((v[u][e] - st.m) * c);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < V; ++e) add(fmaf(v[u][e], c, -mc));
    }
    const float by = exp2_fast(-fix);
    s *= by;
    st.s += s;
    if (ENT) st.w += fmaf(-fix, s, w * by);
  }
  // the work-group's sums: every lane of the wave, then every wave, in a fixed order
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    Stats b{__shfl_xor(st.m, o), __shfl_xor(st.s, o), ENT ? __shfl_xor(st.w, o) : 0.0f};
    join(st, b, c);
  }
  if (lane == 0) part[wave] = st;
  __syncthreads();
  st = part[0];
#pragma unroll
  for (int i = 1; i < W; ++i) join(st, part[i], c);
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
    if (ENT) a.entropy[r] = empty ? 0.0f : fmaxf(fmaf(-LN2, st.w / st.s, logs), st.s != st.s ? NAN : 0.0f);
  }
  if constexpr (TOP) {
    int64_t* ids = a.top_ids + r * a.top;
    float* lps = a.top_logp + r * a.top;
    auto lp_of = [&](uint32_t o) { return empty ? -INFINITY : fmaf(a.scale, value_of(o) - m, -logs); };
    const uint32_t mine = order_of(most);
    uint32_t own, share;
    kth_of_wave<sizeof(T) == 2>(mine, a.top, (a.top + W - 1) / W, &own, &share);
    if (lane == 0) {
      sh.kth[wave] = own;
      sh.share[wave] = share;
    }
    __syncthreads();
    uint32_t first = 0, every = ~0u;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      first = sh.kth[i] > first ? sh.kth[i] : first;
      every = sh.share[i] < every ? sh.share[i] : every;
    }
    first = every > first ? every : first;
    if (mine >= first) sh.tops[atomicAdd(&sh.lanes, 1)] = mine;
    __syncthreads();
    if (mine >= first) {
      int more = 0, least = 0;  // lanes above this one's maximum, and not below it
      const int lanes = sh.lanes;
      for (int i = 0; i < lanes; i += 8)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t t = i + u < lanes ? sh.tops[i + u] : 0;
          more += t > mine;
          least += t >= mine;
        }
      if (more < a.top && a.top <= least) sh.border = mine;  // (all that write, write the same)
    }
    __syncthreads();
    uint32_t border = sh.border;
    if (mine >= border) sh.lane[atomicAdd(&sh.again, 1)] = tid;
    __syncthreads();
    const uint32_t again = (uint32_t)sh.again, each = (uint32_t)((N + NT * V - 1) / (NT * V));  // vectors of a lane
    for (uint32_t i = tid; i < again * each; i += NT) {
      const int64_t j = ((int64_t)(i % each) * NT + sh.lane[i / each]) * V;
      T q[V];
      const int n = (int)(j >= N ? 0 : N - j < V ? N - j : V);
      load_part<T, V>(x + (n > 0 ? j : 0), n, q);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float v = to_f32(q[e]);
        const uint32_t o = order_of(v);
        if (o < border || e >= n) continue;
        if (o == border ? atomicAdd(&sh.equal, 1) >= EQUAL : (atomicAdd(&sh.above, 1), false)) continue;
        const int k = atomicAdd(&sh.count, 1);
        if (k < LIST) sh.list[k] = entry_of(v, j + e);
      }
    }
    __syncthreads();
    int count = sh.count, above = sh.above, equal = sh.equal;
    if (count > LIST || st.s != st.s) {
      // the k-th largest, bit after bit, by counting what is not below; then what is above it and as many as fit at it
      uint32_t t = 0;
      for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 0); --bit) {
        const uint32_t u = t | 1u << bit;
        int n = 0;
        for (int64_t j = tid; j < N; j += NT) n += order_of(to_f32(x[j])) >= u;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
        __syncthreads();
        if (lane == 0) sh.kth[wave] = (uint32_t)n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) n += (int)sh.kth[i];
        if (n >= a.top) t = u;
      }
      border = sizeof(T) == 2 ? whole_order(t) : t;
      __syncthreads();
      if (tid == 0) sh.count = sh.above = sh.equal = 0;
      __syncthreads();
      for (int64_t j = tid; j < N; j += NT) {
        const float v = to_f32(x[j]);
        const uint32_t o = order_of(v);
        if (o < border) continue;
        if (o == border ? atomicAdd(&sh.equal, 1) >= EQUAL : (atomicAdd(&sh.above, 1), false)) continue;
        sh.list[atomicAdd(&sh.count, 1)] = entry_of(v, j);  // (fewer than k are above)
      }
      __syncthreads();
      count = sh.count;
      above = sh.above;
      equal = sh.equal;
    }
    const bool cut = equal > EQUAL;  // not all at the threshold are listed: only what is above it is ranked
    for (int i = tid; i < count; i += NT) {
      const uint64_t o = sh.list[i];
      if (cut && (uint32_t)(o >> 32) == border) continue;
      int rank = 0;
      for (int k = 0; k < count; k += 8)
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += (k + u < count ? sh.list[k + u] : 0) > o;
      if (rank < a.top) {
        ids[rank] = (uint32_t)~(uint32_t)o;
        lps[rank] = lp_of((uint32_t)(o >> 32));
      }
    }
    if (cut && above < a.top && wave == 0) {  // the lowest places of the threshold
      int have = above;
      for (int64_t j = 0; j < N && have < a.top; j += 64) {
        const bool is = j + lane < N && order_of(to_f32(x[j + lane])) == border;
        const uint64_t who = __ballot(is);
        const int k = have + __popcll(who & ((1ull << lane) - 1));
        if (is && k < a.top) {
          ids[k] = j + lane;
          lps[k] = lp_of(border);
        }
        have += __popcll(who);
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
  auto go = [&](auto top, auto ent) {
    for (a.r0 = 0; a.r0 < R; a.r0 += most) {
      const uint32_t n = (uint32_t)(R - a.r0 < most ? R - a.r0 : most);
      logprobs_fwd_kernel<T, NT, top, ent><<<n, NT, top ? sizeof(Shared) : 0, st>>>(a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  if (a.top > 0) return a.entropy != nullptr ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
  return a.entropy != nullptr ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}

}  // namespace

template <typename T>
hipError_t launch_logprobs_fwd(LogprobsArgs a, hipStream_t st) {
  // Threads of a row: more share its elements, but join their results and find the border over more lanes.  bf16 with the entropy and
  // 8 alternatives, 256, 512 and 1024 threads: 64 x 50304 13.9, 14.1 and 17.9 us, 512 x 50304 19.3, 22.2 and 37.3, 8 x 131072 19.9,
  // 17.4 and 19.7; with 20 of them 64 x 128000 25.7, 20.9 and 26.2.
  return a.V <= 65536 || a.R >= 512 ? fwd<T, 256>(a, st) : fwd<T, 512>(a, st);
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
