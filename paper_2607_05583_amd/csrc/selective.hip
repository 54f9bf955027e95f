// Selective scan, per head a state h [P, N]:
//   D_t = softplus(dt_t + dt_bias),  a_t = exp(-gamma D_t),
//   h_t = a_t h_{t-1} + D_t x_t b_t^T,  y_t = h_t c_t + skip x_t.
// In a chunk of Q = 64 steps with s_t = sum_{u<=t} gamma D_u, h the state before it and E[t,s] = exp(s_s - s_t) for s <= t:
//   y_t = exp(-s_t) h c_t + sum_{s<=t} (c_t.b_s) E[t,s] D_s x_s,
//   h' = exp(-s_Q) h + sum_s exp(s_s - s_Q) D_s x_s b_s^T,
// which are matrix products (MFMA).  The backward, with g the gradient of the state behind the chunk and K[t,s] = dy_t.x_s:
//   dc_t = sum_s E D_s K b_s + exp(-s_t) h^T dy_t,      db_s = D_s (sum_t E K c_t + exp(s_s - s_Q) g^T x_s),
//   du_s = sum_t E (c_t.b_s) dy_t + exp(s_s - s_Q) g b_s,  dx_s = D_s du_s + skip dy_s,
//   dl_t = <g, h'> + sum_{u>=t} (dy_u.y_u - D_u x_u.du_u)   (the gradient of log a_t; y without the skip),
//   dD_s = x_s.du_s - gamma dl_s,  dgamma = -sum D dl,  g' = exp(-s_Q) g + sum_t exp(-s_t) dy_t c_t^T.
// dy.y and x.du need no rounded products: their parts within the chunk are the row and column sums of Z = (c.b) E K in
// float32, those of the states are products of two-part operands.
//
// Rounding, bf16 inputs: products of two inputs are exact.  An operand that is computed (states, weighted b, c, x) goes in as
// two bf16 parts, hi + lo, 2^-16 relative, where float32 results depend on it (states, dl); the weights (c.b) E D and E K
// that only make bf16 outputs, and g in db, go in as one bf16 (2^-8 a term, as much as the output's own rounding).
// float32 inputs use float32 MFMA throughout.  Sums and states are float32.
#include "select.h"

namespace res {
namespace {

constexpr int Q = SEL_Q;
constexpr float NO_MORE = 512.0f;  // an exponent (base 2) behind which nothing is left; keeps the chunk's sums small

// ---------------------------------------------------------------------------
// Fragments: 8 elements of the K axis a lane (i = lane & 15 the row or column, q = lane >> 4).  Element j of lane group q is
// k = 16 (j >> 2) + 4 q + (j & 3): the 4 results of two products above each other in a lane (rows 4 q ..) are the fragment of
// a further product as they are.
// ---------------------------------------------------------------------------
template <typename T> struct Mx;
template <> struct Mx<bf16_t> {
  typedef bf8 Frag;
  struct Split { bf8 hi, lo; };
  struct Quad { uint32_t v[2]; } __attribute__((aligned(8)));
  static constexpr int PAD = 8;
  __device__ static __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  __device__ static __forceinline__ f4 mma(const Split& a, const Frag& b, f4 c) { return mma(a.hi, b, mma(a.lo, b, c)); }
  __device__ static __forceinline__ f4 mma(const Frag& a, const Split& b, f4 c) { return mma(a, b.hi, mma(a, b.lo, c)); }
  __device__ static __forceinline__ Frag one(const float (&v)[8]) {
    Frag f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (__bf16)v[j];
    return f;
  }
  __device__ static __forceinline__ Split split(const float (&v)[8]) {
    Split s;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s.hi[j] = (__bf16)v[j];
      s.lo[j] = (__bf16)(v[j] - (float)s.hi[j]);
    }
    return s;
  }
  __device__ static __forceinline__ float at(const Frag& f, int j) { return (float)f[j]; }
  // 4 consecutive elements at k, 4 at k + 16
  __device__ static __forceinline__ Frag row(const bf16_t* p) {
    const s4 lo = *reinterpret_cast<const s4*>(p), hi = *reinterpret_cast<const s4*>(p + 16);
    return __builtin_bit_cast(bf8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // the same of column i of rows at distance ld; p: the tile's first row and column (the transposing load: a group of 16 lanes
  // reads 4 rows of 16 columns, and lane i gets column i)
  __device__ static __forceinline__ Frag col(const bf16_t* p, int ld, int i, int q) {
    typedef __attribute__((address_space(3))) s4 lds_s4;
    const bf16_t* at = p + (4 * q + (i >> 2)) * ld + 4 * (i & 3);
    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)at);
    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(at + 16 * ld));
    return __builtin_bit_cast(bf8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};
template <> struct Mx<float> {
  struct Frag { f4 v[2]; };
  typedef Frag Split;
  static constexpr int PAD = 4;
  __device__ static __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) { return mma_f32(a.v[1], b.v[1], mma_f32(a.v[0], b.v[0], c)); }
  __device__ static __forceinline__ Frag one(const float (&v)[8]) { return Frag{{f4{v[0], v[1], v[2], v[3]}, f4{v[4], v[5], v[6], v[7]}}}; }
  __device__ static __forceinline__ Frag split(const float (&v)[8]) { return one(v); }
  __device__ static __forceinline__ float at(const Frag& f, int j) { return f.v[j >> 2][j & 3]; }
  __device__ static __forceinline__ Frag row(const float* p) { return Frag{{load_f4(p), load_f4(p + 16)}}; }
  __device__ static __forceinline__ Frag col(const float* p, int ld, int i, int q) {
    Frag f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j >> 2][j & 3] = p[(16 * (j >> 2) + 4 * q + (j & 3)) * ld + i];
    return f;
  }
};

// 4 consecutive elements
__device__ __forceinline__ f4 quad(const float* p) { return load_f4(p); }
__device__ __forceinline__ f4 quad(const bf16_t* p) {
  const s4 v = *reinterpret_cast<const s4*>(p);
  return f4{to_f32((bf16_t)v[0]), to_f32((bf16_t)v[1]), to_f32((bf16_t)v[2]), to_f32((bf16_t)v[3])};
}
__device__ __forceinline__ void put_quad(float* p, const f4& v) { *reinterpret_cast<f4*>(p) = v; }
__device__ __forceinline__ void put_quad(bf16_t* p, const f4& v) {
  typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf4*>(p) = __builtin_convertvector(v, bf4);
}
// 4 results to a row of memory, n of them
template <typename T>
__device__ __forceinline__ void store_quad(T* p, int n, const f4& v) {
  T q[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) q[r] = from_f32<T>(v[r]);
  store_part<T, 4>(p, n < 0 ? 0 : n, q);
}

// ---------------------------------------------------------------------------
// Tiles: Q rows of COLS elements from memory to registers (zeros outside) and on to LDS rows of COLS + PAD
// ---------------------------------------------------------------------------
template <typename T, int COLS> struct Tile {
  static constexpr int V = 16 / (int)sizeof(T), PR = COLS / V, RT = SEL_THREADS / PR, U = Q / RT, LD = COLS + Mx<T>::PAD;
  static constexpr int BYTES = Q * LD * (int)sizeof(T);
  T v[U][V];
  __device__ __forceinline__ void load(const T* p, int64_t st, int rows, int cols) {
    const int r0 = threadIdx.x / PR, c = threadIdx.x % PR * V;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * RT, n = r < rows ? cols - c : 0;
      if (n > 0)
        load_part<T, V>(p + r * st + c, n, v[u]);
      else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[u][e] = T(0);
      }
    }
  }
  __device__ __forceinline__ void put(T* lds) const {
    typedef T Vec __attribute__((ext_vector_type(V)));
    const int r0 = threadIdx.x / PR, c = threadIdx.x % PR * V;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Vec q;
#pragma unroll
      for (int e = 0; e < V; ++e) q[e] = v[u][e];
      *reinterpret_cast<Vec*>(lds + (r0 + u * RT) * LD + c) = q;
    }
  }
};

// A chunk's steps, one a lane (by one wave): D, s (inclusive sums of gamma D, base 2), what follows a step (exclusive), the total.
struct Steps {
  float d, s, after, total, slope;
};
template <typename T>
__device__ __forceinline__ Steps steps_of(const SelArgs& a, int64_t b, int64_t t, int64_t n, int h, int lane) {
  Steps o{0, 0, 0, 0, 0};
  float ld = 0.0f;
  if (t + lane < n) {
    const float v = to_f32(static_cast<const T*>(a.dt.p)[b * a.dt.sb + (t + lane) * a.dt.st + h]) + (a.dt_bias != nullptr ? a.dt_bias[h] : 0.0f);
    o.d = fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v)));
    if (v != v) o.d = v;
    o.slope = 1.0f / (1.0f + expf(-v));
    ld = o.d * a.gamma[h] * LOG2E;
    ld = ld > NO_MORE ? NO_MORE : ld;
  }
  o.s = ld;
  float back = ld;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const float up = __shfl_up(o.s, k), down = __shfl_down(back, k);
    if (lane >= k) o.s += up;
    if (lane + k < 64) back += down;
  }
  o.total = __shfl(o.s, 63);
  const float next = __shfl_down(back, 1);
  o.after = lane < 63 ? next : 0.0f;
  return o;
}

// Which rows a work-group has: its batch row, segment, group and row blocks hv0 .. hv0 + heads (of the batch row's HV).
struct Place {
  int64_t b, seg;
  int g, block, hv0, heads;
};
__device__ __forceinline__ Place place_of(const SelArgs& a, int per) {
  const int blocks = (a.p.HG + per - 1) / per;
  int64_t id = a.wg0 + blockIdx.x;
  Place o;
  o.block = (int)(id % blocks);
  id /= blocks;
  o.g = (int)(id % a.G);
  id /= a.G;
  o.seg = id % a.p.segs;
  o.b = id / a.p.segs;
  o.hv0 = o.g * a.p.HG + o.block * per;
  o.heads = a.p.HG - o.block * per < per ? a.p.HG - o.block * per : per;
  return o;
}
__device__ __forceinline__ int64_t length_of(const SelArgs& a, int64_t b) {
  if (a.lengths == nullptr) return a.L;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.L ? a.L : n;
}
__device__ __forceinline__ float sum_rows(float v) {  // over the 4 lanes of one column
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// A state [P][N] of a caller's tensor (or none: zeros) or a padded one of the workspace.
struct StateAt {
  const float* ext;
  const float* pad;
  int P, N, p0, NP;
  __device__ __forceinline__ float get(int p, int n) const {
    if (pad != nullptr) return pad[p * NP + n];
    return ext != nullptr && p0 + p < P && n < N ? ext[(int64_t)(p0 + p) * N + n] : 0.0f;
  }
};
__device__ __forceinline__ StateAt state_at(const SelArgs& a, const float* ext, const float* pad, int64_t b, int hv, int64_t seg) {
  const int h = hv / a.p.PB, NP = 16 * a.p.NT;
  StateAt s{ext, nullptr, a.P, a.N, hv % a.p.PB * SEL_P, NP};
  if (ext != nullptr) s.ext = ext + (b * a.H + h) * (int64_t)a.P * a.N;
  if (pad != nullptr) s.pad = pad + ((b * a.p.HV + hv) * a.p.segs + seg) * (int64_t)(SEL_P * NP);
  return s;
}

// ---------------------------------------------------------------------------
// Forward: a wave owns 16 of a row block's 64 rows.  Its states are in registers, transposed: lane (p, q) holds
// n = 16 v + 4 q .. + 3.  STATES: only the segment's end state from a zero start (and REV: the gradient that the segment
// gives to the state before it: dy, c and exp(-s_t) in the place of x, b and the weights, from the last chunk back).
// ---------------------------------------------------------------------------
template <typename T, int NT, int HF, bool STATES, bool REV>
__global__ __launch_bounds__(SEL_THREADS) void selective_fwd_kernel(SelArgs a) {
  typedef Mx<T> M;
  constexpr int NP = 16 * NT, KS = NT / 2;
  typedef Tile<T, NP> TB;
  typedef Tile<T, SEL_P> TX;
  __shared__ __align__(16) T bt[Q * TB::LD];
  __shared__ __align__(16) T ct[STATES ? 8 : Q * TB::LD];
  __shared__ __align__(16) T xt[2][Q * TX::LD];
  __shared__ __align__(16) T mt[STATES ? 1 : 2][STATES ? 8 : 6 * 64 * 8];
  __shared__ __align__(16) float ss[HF][Q], sd[HF][Q], sw[HF][Q], st[HF];  // s, D, D exp(what follows), the chunk's total
  const Place o = place_of(a, HF);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, li = lane & 15, lq = lane >> 4;
  const int64_t n = length_of(a, o.b);
  const int64_t c0 = o.seg * a.p.seg, c1 = c0 + a.p.seg < a.p.chunks ? c0 + a.p.seg : a.p.chunks;
  const Rows rx = REV ? a.dy : a.x, rb = REV ? a.c : a.b;
  const T* px = static_cast<const T*>(rx.p) + o.b * rx.sb;
  const T* pb = static_cast<const T*>(rb.p) + o.b * rb.sb + o.g * a.N;
  const T* pc = static_cast<const T*>(a.c.p) + o.b * a.c.sb + o.g * a.N;

  f4 h[HF][NT];
  float total[HF];
#pragma unroll
  for (int k = 0; k < HF; ++k) {
    total[k] = 0.0f;
#pragma unroll
    for (int v = 0; v < NT; ++v) h[k][v] = f4{0, 0, 0, 0};
    if (!STATES && k < o.heads) {
      const StateAt s = state_at(a, a.h0, a.p.segs > 1 ? a.enter : nullptr, o.b, o.hv0 + k, o.seg);
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) h[k][v][r] = s.get(16 * w + li, 16 * v + 4 * lq + r);
    }
  }
  if constexpr (!STATES) {
    // the tiles above the diagonal that share a fragment with one on it stay zero
    for (int i = tid; i < 2 * 6 * 64 * 8; i += SEL_THREADS) mt[0][i] = T(0);
  }
  for (int64_t ci = c0; ci < c1; ++ci) {
    const int64_t ch = REV ? c1 - 1 - (ci - c0) : ci, t0 = ch * Q;
    const int rows = (int)(n - t0 < 0 ? 0 : n - t0 < Q ? n - t0 : Q);
    const int held = (int)(a.L - t0 < Q ? a.L - t0 : Q);
    if (rows == 0) {  // behind the row's end: the state stays
      if constexpr (!STATES) {
        T* y = static_cast<T*>(a.y) + (o.b * a.L + t0) * a.H * a.P;
        for (int k = 0; k < o.heads; ++k) {
          const int hv = o.hv0 + k, p0 = hv % a.p.PB * SEL_P;
          const int cols = a.P - p0 < SEL_P ? a.P - p0 : SEL_P;
          for (int i = tid; i < held * SEL_P; i += SEL_THREADS)
            if (i % SEL_P < cols) y[(int64_t)(i / SEL_P) * a.H * a.P + hv / a.p.PB * a.P + p0 + i % SEL_P] = T(0);
        }
      }
      continue;
    }
    __syncthreads();  // the last chunk's readers are through
    {
      TB t;
      t.load(pb + t0 * rb.st, rb.st, rows, a.N);
      t.put(bt);
      if constexpr (!STATES) {
        t.load(pc + t0 * a.c.st, a.c.st, rows, a.N);
        t.put(ct);
      }
    }
    for (int k = w; k < o.heads; k += 4) {
      const Steps s = steps_of<T>(a, o.b, t0, n, (o.hv0 + k) / a.p.PB, lane);
      ss[k][lane] = s.s;
      sd[k][lane] = s.d;
      sw[k][lane] = REV ? exp2_fast(-s.s) : s.d * exp2_fast(-s.after);
      if (lane == 0) st[k] = s.total;
    }
    auto load_x = [&](int k) {
      const int hv = o.hv0 + k, p0 = hv % a.p.PB * SEL_P;
      TX t;
      t.load(px + t0 * rx.st + hv / a.p.PB * a.P + p0, rx.st, rows, a.P - p0);
      t.put(xt[k & 1]);
    };
    load_x(0);
    __syncthreads();
    // G^T [s][t] = b c^T: tile e of 10 (and this wave's are e = w, w + 4, w + 8) is t tile ti, s tile si <= ti
    f4 g[3];
    if constexpr (!STATES) {
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const int id = w + 4 * e, ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3, si = id - ti * (ti + 1) / 2;
        g[e] = f4{0, 0, 0, 0};
        if (id < 10)
#pragma unroll
          for (int k = 0; k < KS; ++k)
            g[e] = M::mma(M::row(bt + (16 * si + li) * TB::LD + 32 * k + 4 * lq), M::row(ct + (16 * ti + li) * TB::LD + 32 * k + 4 * lq), g[e]);
      }
    }
#pragma unroll
    for (int k = 0; k < HF; ++k) {
      if (k >= o.heads) break;
      const int hv = o.hv0 + k, hd = hv / a.p.PB, p0 = hv % a.p.PB * SEL_P;
      if constexpr (!STATES) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
          const int id = w + 4 * e, ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3, si = id - ti * (ti + 1) / 2;
          if (id < 10) {
            const float s_t = ss[k][16 * ti + li];
            const f4 s_s = load_f4(&ss[k][16 * si + 4 * lq]), d = load_f4(&sd[k][16 * si + 4 * lq]);
            f4 m;
#pragma unroll
            for (int r = 0; r < 4; ++r) m[r] = si < ti || 4 * lq + r <= li ? g[e][r] * (exp2_fast(s_s[r] - s_t) * d[r]) : 0.0f;
            // fragment (t tile, 32 steps s): 0, 1, 2 and 3, 4 and 5 of t tiles 0, 1, 2, 3
            const int f = ti < 2 ? ti : 2 * ti - 2 + (si >> 1);
            put_quad(&mt[k & 1][(f * 64 + lane) * 8 + (si & 1) * 4], m);
          }
        }
      }
      __syncthreads();
      if (k + 1 < o.heads) load_x(k + 1);  // (its buffer's readers were through before the barrier)
      const T* xk = xt[k & 1];
      typename M::Frag xf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) xf[j] = M::col(xk + 32 * j * TX::LD + 16 * w, TX::LD, li, lq);
      if constexpr (!STATES) {
        f4 y[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) y[t] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          float hf[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) hf[r] = h[k][2 * j + (r >> 2)][r & 3];
          const typename M::Split hp = M::split(hf);
#pragma unroll
          for (int t = 0; t < 4; ++t) y[t] = M::mma(hp, M::row(ct + (16 * t + li) * TB::LD + 32 * j + 4 * lq), y[t]);
        }
        const float skip = a.skip != nullptr ? a.skip[hd] : 0.0f;
        T* yp = static_cast<T*>(a.y) + (o.b * a.L + t0) * a.H * a.P + hd * a.P + p0 + 16 * w + 4 * lq;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float f = exp2_fast(-ss[k][16 * t + li]);
#pragma unroll
          for (int r = 0; r < 4; ++r) y[t][r] *= f;
#pragma unroll
          for (int j = 0; j <= t / 2; ++j) {
            const int fr = t < 2 ? t : 2 * t - 2 + j;
            const typename M::Frag mf = *reinterpret_cast<const typename M::Frag*>(&mt[k & 1][(fr * 64 + lane) * 8]);
            y[t] = M::mma(xf[j], mf, y[t]);
          }
          const int row = 16 * t + li;
          const f4 xr = quad(xk + row * TX::LD + 16 * w + 4 * lq);
#pragma unroll
          for (int r = 0; r < 4; ++r) y[t][r] = row < rows ? fmaf(skip, xr[r], y[t][r]) : 0.0f;
          if (row < held) store_quad(yp + (int64_t)row * a.H * a.P, a.P - p0 - 16 * w - 4 * lq, y[t]);
        }
      }
      const float keep = exp2_fast(-st[k]);
      total[k] += st[k];
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) h[k][v][r] *= keep;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f4 w0 = load_f4(&sw[k][32 * j + 4 * lq]), w1 = load_f4(&sw[k][32 * j + 16 + 4 * lq]);
        float xw[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) xw[r] = M::at(xf[j], r) * (r < 4 ? w0[r & 3] : w1[r & 3]);
        const typename M::Split xp = M::split(xw);
#pragma unroll
        for (int v = 0; v < NT; ++v) h[k][v] = M::mma(M::col(bt + 32 * j * TB::LD + 16 * v, TB::LD, li, lq), xp, h[k][v]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < HF; ++k) {
    if (k >= o.heads) break;
    const int hv = o.hv0 + k, p = 16 * w + li;
    if constexpr (STATES) {
      const int64_t at = (o.b * a.p.HV + hv) * a.p.segs + o.seg;
      float* s = (REV ? a.leave : a.enter) + (at * SEL_P + p) * NP + 4 * lq;
#pragma unroll
      for (int v = 0; v < NT; ++v) put_quad(s + 16 * v, h[k][v]);
      if (tid == 0) a.decay[at] = total[k];
    } else if (a.p.segs == 1 && a.h_out != nullptr) {
      const int p0 = hv % a.p.PB * SEL_P;
      float* s = a.h_out + ((o.b * a.H + hv / a.p.PB) * (int64_t)a.P + p0 + p) * a.N;
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (p0 + p < a.P && 16 * v + 4 * lq + r < a.N) s[16 * v + 4 * lq + r] = h[k][v][r];
    }
  }
}

// The segments' states one after the other: each segment's own end state makes way for the state that enters it.
template <bool REV>
__global__ __launch_bounds__(SEL_THREADS) void selective_join_kernel(SelArgs a) {
  const int NP = 16 * a.p.NT, per = SEL_P * NP / 4;
  const int64_t id = (int64_t)blockIdx.x * SEL_THREADS + threadIdx.x, bh = a.wg0 + id / per;
  if (bh >= a.B * a.p.HV) return;
  const int at = (int)(id % per) * 4, p = at / NP, n = at % NP, hv = (int)(bh % a.p.HV);
  const int64_t b = bh / a.p.HV;
  const StateAt s = state_at(a, REV ? a.dh_out : a.h0, nullptr, b, hv, 0);
  f4 e{s.get(p, n), s.get(p, n + 1), s.get(p, n + 2), s.get(p, n + 3)};
  float* buf = (REV ? a.leave : a.enter) + bh * a.p.segs * (int64_t)(SEL_P * NP) + at;
  const float* decay = a.decay + bh * a.p.segs;
  for (int64_t i = 0; i < a.p.segs; ++i) {
    const int64_t k = REV ? a.p.segs - 1 - i : i;
    float* q = buf + k * (int64_t)(SEL_P * NP);
    const f4 own = load_f4(q);
    const float keep = exp2_fast(-decay[k]);
    put_quad(q, e);
#pragma unroll
    for (int r = 0; r < 4; ++r) e[r] = fmaf(keep, e[r], own[r]);
  }
  float* out = REV ? a.dh0 : a.h_out;
  const int p1 = hv % a.p.PB * SEL_P + p;
  if (out != nullptr && p1 < a.P)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < a.N) out[((b * a.H + hv / a.p.PB) * (int64_t)a.P + p1) * a.N + n + r] = e[r];
}

// ---------------------------------------------------------------------------
// Backward: a work-group takes a segment of up to SEL_BWD_HEADS row blocks of a group, so that db and dc are summed over them
// in registers.  First the states before each chunk are made again (to hs); then the chunks from the last one back, head after
// head.  A wave owns the 16-state tiles w, w + 4: there states and their gradients are lanes (n, q) with p = 16 v + 4 q .. + 3,
// as their products with x and dy need them; du, which needs a row's states, takes them through LDS.
// ---------------------------------------------------------------------------
template <typename T, int NT> struct BwdLds {
  static constexpr int SL = NT < 4 ? NT : 4, NS = 16 * SL;  // state tiles of a slice, which goes through LDS at once
  typedef Tile<T, 16 * NT> TB;
  typedef Tile<T, SEL_P> TX;
  __align__(16) T bt[Q * TB::LD];
  __align__(16) T ct[Q * TB::LD];
  __align__(16) T xt[Q * TX::LD];
  __align__(16) T dt[Q * TX::LD];
  __align__(16) T ek[Q * TX::LD];              // row s: E[t,s] D_s K[t,s] over t
  __align__(16) T eg[Q * TX::LD];              // row s: E[t,s] (c_t.b_s)
  __align__(16) T gx[2][sizeof(T) == 2 ? NS * TX::LD : NS * TX::LD / 2];  // row n: g over p (two parts; float32: one)
  __align__(16) float s[Q], d[Q], suf[Q], pre[Q], slope[Q];  // s, D, exp(-what follows), exp(-s), dD/d dt
  float rowz[4][Q], colz[4][Q], ic[4][Q], ig[4][Q];  // by s tile, by t tile, by wave, by wave
  float lam[SEL_BWD_HEADS][4], sums[SEL_BWD_HEADS][3], skip[4], total;
};

template <typename T, int NT>
__global__ __launch_bounds__(SEL_THREADS) void selective_bwd_kernel(SelArgs a) {
  typedef Mx<T> M;
  typedef BwdLds<T, NT> Lds;
  typedef typename Lds::TB TB;
  typedef typename Lds::TX TX;
  constexpr int KS = NT / 2, NW = (NT + 3) / 4, SL = Lds::SL;
  extern __shared__ __align__(16) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  const Place o = place_of(a, a.p.HR);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, li = lane & 15, lq = lane >> 4;
  const int64_t n = length_of(a, o.b);
  const int64_t c0 = o.seg * a.p.seg, c1 = c0 + a.p.seg < a.p.chunks ? c0 + a.p.seg : a.p.chunks;
  const T* px = static_cast<const T*>(a.x.p) + o.b * a.x.sb;
  const T* pd = static_cast<const T*>(a.dy.p) + o.b * a.dy.sb;
  const T* pb = static_cast<const T*>(a.b.p) + o.b * a.b.sb + o.g * a.N;
  const T* pc = static_cast<const T*>(a.c.p) + o.b * a.c.sb + o.g * a.N;
  const bool mine = w < NT;  // the wave has state tiles
  // states of a work-group: [chunk (one more)][head][wave][own tile][p tile][lane]
  const int64_t wg = a.wg0 + blockIdx.x;
  f4* hs = a.hs + wg * (a.p.seg + 1) * a.p.HR * (4 * NW * 4 * 64) + w * (NW * 4 * 64) + lane;
  f4* gs = a.gs + wg * a.p.HR * (4 * NW * 4 * 64) + w * (NW * 4 * 64) + lane;
  auto hs_at = [&](int64_t c, int k) { return hs + (c * a.p.HR + k) * (4 * NW * 4 * 64); };
  auto gs_at = [&](int k) { return gs + k * (4 * NW * 4 * 64); };

  for (int i = tid; i < Q * TX::LD; i += SEL_THREADS) l.ek[i] = l.eg[i] = T(0);
  if (tid < 4) l.skip[tid] = 0.0f;
  // the states entering and the gradients behind the segment
  for (int k = 0; k < o.heads; ++k) {
    const StateAt s = state_at(a, a.h0, a.p.segs > 1 ? a.enter : nullptr, o.b, o.hv0 + k, o.seg);
    const StateAt e = state_at(a, a.dh_out, a.p.segs > 1 ? a.leave : nullptr, o.b, o.hv0 + k, o.seg);
    if (mine)
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          f4 hv, gv;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            hv[r] = s.get(16 * v + 4 * lq + r, 16 * (w + 4 * m) + li);
            gv[r] = e.get(16 * v + 4 * lq + r, 16 * (w + 4 * m) + li);
          }
          hs_at(0, k)[(m * 4 + v) * 64] = hv;
          gs_at(k)[(m * 4 + v) * 64] = gv;
        }
  }
  auto put_steps = [&](int64_t t0, int k) {  // by one wave
    const Steps s = steps_of<T>(a, o.b, t0, n, (o.hv0 + k) / a.p.PB, lane);
    l.s[lane] = s.s;
    l.d[lane] = s.d;
    l.suf[lane] = exp2_fast(-s.after);
    l.pre[lane] = exp2_fast(-s.s);
    l.slope[lane] = s.slope;
    if (lane == 0) l.total = s.total;
  };
  auto cols_of = [&](int k, int64_t* at) {  // a row block's columns within a step
    const int hv = o.hv0 + k, p0 = hv % a.p.PB * SEL_P;
    *at = hv / a.p.PB * a.P + p0;
    return a.P - p0;
  };

  // the states before each chunk, and behind the last
  for (int64_t ci = 0; ci < c1 - c0; ++ci) {
    const int64_t t0 = (c0 + ci) * Q;
    const int rows = (int)(n - t0 < 0 ? 0 : n - t0 < Q ? n - t0 : Q);
    __syncthreads();
    if (rows > 0) {
      TB t;
      t.load(pb + t0 * a.b.st, a.b.st, rows, a.N);
      t.put(l.bt);
    }
    for (int k = 0; k < o.heads; ++k) {
      __syncthreads();
      if (rows > 0) {
        int64_t at;
        const int cols = cols_of(k, &at);
        TX t;
        t.load(px + t0 * a.x.st + at, a.x.st, rows, cols);
        t.put(l.xt);
        if (w == 0) put_steps(t0, k);
      }
      __syncthreads();
      if (!mine) continue;
      f4 h[NW][4];
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) h[m][v] = hs_at(ci, k)[(m * 4 + v) * 64];
      if (rows > 0) {
        const float keep = exp2_fast(-l.total);
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) h[m][v][r] *= keep;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float ws[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int t = 32 * j + 16 * (r >> 2) + 4 * lq + (r & 3);
            ws[r] = l.d[t] * l.suf[t];
          }
          typename M::Split bs[NW];
#pragma unroll
          for (int m = 0; m < NW; ++m) {
            const typename M::Frag bf = M::col(l.bt + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
            float bw[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) bw[r] = M::at(bf, r) * ws[r];
            bs[m] = M::split(bw);
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const typename M::Frag xf = M::col(l.xt + 32 * j * TX::LD + 16 * v, TX::LD, li, lq);
#pragma unroll
            for (int m = 0; m < NW; ++m) h[m][v] = M::mma(xf, bs[m], h[m][v]);
          }
        }
      }
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) hs_at(ci + 1, k)[(m * 4 + v) * 64] = h[m][v];
    }
  }
  // <g, h> behind the segment
  for (int k = 0; k < o.heads; ++k) {
    float dot = 0.0f;
    if (mine)
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const f4 h = hs_at(c1 - c0, k)[(m * 4 + v) * 64], g = gs_at(k)[(m * 4 + v) * 64];
#pragma unroll
          for (int r = 0; r < 4; ++r) dot = fmaf(h[r], g[r], dot);
        }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) dot += __shfl_xor(dot, s);
    if (lane == 0) l.lam[k][w] = dot;
  }
  if (tid < SEL_BWD_HEADS * 3) l.sums[tid / 3][tid % 3] = 0.0f;

  for (int64_t ci = c1 - c0 - 1; ci >= 0; --ci) {
    const int64_t t0 = (c0 + ci) * Q;
    const int rows = (int)(n - t0 < 0 ? 0 : n - t0 < Q ? n - t0 : Q);
    const int held = (int)(a.L - t0 < Q ? a.L - t0 : Q);
    f4 db[NW][4], dc[NW][4], g0[3];
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int v = 0; v < 4; ++v) db[m][v] = dc[m][v] = f4{0, 0, 0, 0};
    __syncthreads();
    if (rows > 0) {
      TB t;
      t.load(pb + t0 * a.b.st, a.b.st, rows, a.N);
      t.put(l.bt);
      t.load(pc + t0 * a.c.st, a.c.st, rows, a.N);
      t.put(l.ct);
      __syncthreads();
      // (c.b)[t][s], by the tiles on and below the diagonal: tile e of 10 is t tile ti, s tile si
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const int id = w + 4 * e, ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3, si = id - ti * (ti + 1) / 2;
        g0[e] = f4{0, 0, 0, 0};
        if (id < 10)
#pragma unroll
          for (int k = 0; k < KS; ++k)
            g0[e] = M::mma(M::row(l.ct + (16 * ti + li) * TB::LD + 32 * k + 4 * lq), M::row(l.bt + (16 * si + li) * TB::LD + 32 * k + 4 * lq), g0[e]);
      }
    }
    float ddt = 0.0f;  // wave 0: a step's, over a head's row blocks
    for (int k = 0; k < o.heads; ++k) {
      const int hv = o.hv0 + k, hd = hv / a.p.PB;
      int64_t at;
      const int cols = cols_of(k, &at);
      T* pdx = static_cast<T*>(a.dx.p) + o.b * a.dx.sb + t0 * a.dx.st + at;
      T* pdd = static_cast<T*>(a.ddt.p) + o.b * a.ddt.sb + t0 * a.ddt.st + hd;
      if (rows == 0) {
        for (int i = tid; i < held * SEL_P; i += SEL_THREADS)
          if (i % SEL_P < cols) pdx[(int64_t)(i / SEL_P) * a.dx.st + i % SEL_P] = T(0);
        if (tid < held) pdd[tid * a.ddt.st] = T(0);
        continue;
      }
      const float skip = a.skip != nullptr ? a.skip[hd] : 0.0f;
      f4 g[NW][4], h[NW][4];
      if (mine)
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            g[m][v] = gs_at(k)[(m * 4 + v) * 64];
            h[m][v] = hs_at(ci, k)[(m * 4 + v) * 64];
          }
      __syncthreads();  // the last head's readers are through
      {
        TX t;
        t.load(px + t0 * a.x.st + at, a.x.st, rows, cols);
        t.put(l.xt);
        t.load(pd + t0 * a.dy.st + at, a.dy.st, rows, cols);
        t.put(l.dt);
      }
      if (w == 0) put_steps(t0, k);
      // du = exp(-what follows) g b, this wave's 16 rows p: g's slices through LDS
      f4 du[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) du[v] = f4{0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < NW; ++m) {
        if (m > 0) __syncthreads();
        if (mine)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            T* row = &l.gx[0][(16 * w + li) * TX::LD + 16 * v + 4 * lq];
            if constexpr (sizeof(T) == 2) {
              typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
              const bf4 hi = __builtin_convertvector(g[m][v], bf4);
              const f4 back = __builtin_convertvector(hi, f4);
              *reinterpret_cast<bf4*>(row) = hi;
              put_quad(&l.gx[1][(16 * w + li) * TX::LD + 16 * v + 4 * lq], g[m][v] - back);
            } else {
              put_quad(row, g[m][v]);
            }
          }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < SL / 2; ++j) {
          typename M::Split gf;
          if constexpr (sizeof(T) == 2) {
            gf.hi = M::col(&l.gx[0][32 * j * TX::LD + 16 * w], TX::LD, li, lq);
            gf.lo = M::col(&l.gx[1][32 * j * TX::LD + 16 * w], TX::LD, li, lq);
          } else {
            gf = M::col(&l.gx[0][32 * j * TX::LD + 16 * w], TX::LD, li, lq);
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) du[v] = M::mma(gf, M::row(l.bt + (16 * v + li) * TB::LD + 64 * m + 32 * j + 4 * lq), du[v]);
        }
      }
      {  // its part of x.du
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const f4 x = quad(l.xt + (16 * v + li) * TX::LD + 16 * w + 4 * lq);
          const float f = l.suf[16 * v + li];
          float dot = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            du[v][r] *= f;
            dot = fmaf(x[r], du[v][r], dot);
          }
          dot = sum_rows(dot);
          if (lq == 0) l.ig[w][16 * v + li] = dot;
        }
      }
      // K = dy.x; Z = (c.b) E K; the weights of the products within the chunk
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const int id = w + 4 * e, ti = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3, si = id - ti * (ti + 1) / 2;
        if (id >= 10) continue;
        f4 kk{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j)
          kk = M::mma(M::row(l.dt + (16 * ti + li) * TX::LD + 32 * j + 4 * lq), M::row(l.xt + (16 * si + li) * TX::LD + 32 * j + 4 * lq), kk);
        const float s_s = l.s[16 * si + li], d_s = l.d[16 * si + li];
        const f4 s_t = load_f4(&l.s[16 * ti + 4 * lq]);
        f4 ek, eg, z;
        float col = 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool in = si < ti || li <= 4 * lq + r;
          const float f = exp2_fast(s_s - s_t[r]);
          eg[r] = in ? f * g0[e][r] : 0.0f;
          const float kf = in ? f * kk[r] : 0.0f;
          ek[r] = kf * d_s;
          col = fmaf(eg[r], kk[r], col);
          z[r] = ek[r] * g0[e][r];
        }
        put_quad(l.ek + (16 * si + li) * TX::LD + 16 * ti + 4 * lq, ek);
        put_quad(l.eg + (16 * si + li) * TX::LD + 16 * ti + 4 * lq, eg);
        col = sum_rows(col);
        if (lq == 0) l.colz[ti][16 * si + li] = col;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int sft = 1; sft < 16; sft <<= 1) z[r] += __shfl_xor(z[r], sft);
        }
        if (li == 0) *reinterpret_cast<f4*>(&l.rowz[si][16 * ti + 4 * lq]) = z;
        if (si == ti) {  // the diagonal: dy_t.x_t
          float dg = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) dg += li == 4 * lq + r ? kk[r] : 0.0f;
#pragma unroll
          for (int sft = 1; sft < 64; sft <<= 1) dg += __shfl_xor(dg, sft);
          if (lane == 0) l.skip[ti] = dg;
        }
      }
      // dc's part from the states: exp(-s_t) h^T dy_t, and with c_t its part of dy.y
      if (mine) {
        float ic[4] = {0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          f4 acc[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[t] = f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float hf[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) hf[r] = h[m][2 * j + (r >> 2)][r & 3];
            const typename M::Split hp = M::split(hf);
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = M::mma(hp, M::row(l.dt + (16 * t + li) * TX::LD + 32 * j + 4 * lq), acc[t]);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float f = l.pre[16 * t + li];
            const f4 c = quad(l.ct + (16 * t + li) * TB::LD + 16 * (w + 4 * m) + 4 * lq);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = acc[t][r] * f;
              ic[t] = fmaf(c[r], v, ic[t]);
              dc[m][t][r] += v;
            }
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float v = sum_rows(ic[t]);
          if (lq == 0) l.ic[w][16 * t + li] = v;
        }
      } else if (lane < 16) {
#pragma unroll
        for (int t = 0; t < 4; ++t) l.ic[w][16 * t + lane] = 0.0f;
      }
      __syncthreads();
      if (w == 0) {  // dl, dD and the parameters' sums; one step a lane
        const int tile = lane >> 4;
        float ry = 0.0f, cu = 0.0f;
        for (int v = 0; v <= tile; ++v) ry += l.rowz[v][lane];
        for (int v = tile; v < 4; ++v) cu += l.colz[v][lane];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          ry += l.ic[v][lane];
          cu += l.ig[v][lane];
        }
        const float d = l.d[lane];
        float dl = ry - d * cu;
#pragma unroll
        for (int sft = 1; sft < 64; sft <<= 1) {
          const float v = __shfl_down(dl, sft);
          if (lane + sft < 64) dl += v;
        }
        dl += l.lam[k][0] + l.lam[k][1] + l.lam[k][2] + l.lam[k][3];
        const float v = (cu - a.gamma[hd] * dl) * l.slope[lane];
        float sg = -d * dl, sb = v;
#pragma unroll
        for (int sft = 1; sft < 64; sft <<= 1) {
          sg += __shfl_xor(sg, sft);
          sb += __shfl_xor(sb, sft);
        }
        if (lane == 0) {
          l.sums[k][0] += sg;
          l.sums[k][1] += sb;
          l.sums[k][2] += l.skip[0] + l.skip[1] + l.skip[2] + l.skip[3];
        }
        ddt = hv % a.p.PB == 0 ? v : ddt + v;
        if (hv % a.p.PB == a.p.PB - 1 && lane < held) pdd[lane * a.ddt.st] = from_f32<T>(lane < rows ? ddt : 0.0f);
      }
      // within the chunk: dc, db, du
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j <= t / 2; ++j)
          if (mine) {
            const typename M::Frag f = M::col(l.ek + 32 * j * TX::LD + 16 * t, TX::LD, li, lq);
#pragma unroll
            for (int m = 0; m < NW; ++m) dc[m][t] = M::mma(M::col(l.bt + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq), f, dc[m][t]);
          }
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int j = v / 2; j < 2; ++j) {
          if (mine) {
            const typename M::Frag f = M::row(l.ek + (16 * v + li) * TX::LD + 32 * j + 4 * lq);
#pragma unroll
            for (int m = 0; m < NW; ++m) db[m][v] = M::mma(M::col(l.ct + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq), f, db[m][v]);
          }
          du[v] = M::mma(M::col(l.dt + 32 * j * TX::LD + 16 * w, TX::LD, li, lq), M::row(l.eg + (16 * v + li) * TX::LD + 32 * j + 4 * lq), du[v]);
        }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int row = 16 * v + li;
        const float d = l.d[row];
        const f4 y = quad(l.dt + row * TX::LD + 16 * w + 4 * lq);
#pragma unroll
        for (int r = 0; r < 4; ++r) du[v][r] = row < rows ? fmaf(skip, y[r], d * du[v][r]) : 0.0f;
        if (row < held) store_quad(pdx + (int64_t)row * a.dx.st + 16 * w + 4 * lq, cols - 16 * w - 4 * lq, du[v]);
      }
      if (mine) {
        // db's part from the states' gradients
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          f4 acc[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[v] = f4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float gf[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) gf[r] = g[m][2 * j + (r >> 2)][r & 3];
            const typename M::Frag go = M::one(gf);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[v] = M::mma(go, M::row(l.xt + (16 * v + li) * TX::LD + 32 * j + 4 * lq), acc[v]);
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float f = l.d[16 * v + li] * l.suf[16 * v + li];
#pragma unroll
            for (int r = 0; r < 4; ++r) db[m][v][r] = fmaf(f, acc[v][r], db[m][v][r]);
          }
        }
        // g before the chunk, and its product with the state there
        const float keep = exp2_fast(-l.total);
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) g[m][v][r] *= keep;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f4 w0 = load_f4(&l.pre[32 * j + 4 * lq]), w1 = load_f4(&l.pre[32 * j + 16 + 4 * lq]);
          typename M::Split cs[NW];
#pragma unroll
          for (int m = 0; m < NW; ++m) {
            const typename M::Frag cf = M::col(l.ct + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
            float cw[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) cw[r] = M::at(cf, r) * (r < 4 ? w0[r & 3] : w1[r & 3]);
            cs[m] = M::split(cw);
          }
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const typename M::Frag yf = M::col(l.dt + 32 * j * TX::LD + 16 * v, TX::LD, li, lq);
#pragma unroll
            for (int m = 0; m < NW; ++m) g[m][v] = M::mma(yf, cs[m], g[m][v]);
          }
        }
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v) gs_at(k)[(m * 4 + v) * 64] = g[m][v];
      }
      float dot = 0.0f;
      if (mine)
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) dot = fmaf(g[m][v][r], h[m][v][r], dot);
#pragma unroll
      for (int sft = 1; sft < 64; sft <<= 1) dot += __shfl_xor(dot, sft);
      __syncthreads();  // (wave 0 has read the head's earlier value)
      if (lane == 0) l.lam[k][w] = dot;
    }
    if (mine) {
      const int64_t gn = (int64_t)a.G * a.N;
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int row = 16 * v + li, c = 16 * (w + 4 * m) + 4 * lq;
          if (row >= held) continue;
          if (row >= rows) db[m][v] = dc[m][v] = f4{0, 0, 0, 0};
          if (a.part != nullptr) {
            float* p = a.part + (((int64_t)o.block * 2 * a.B + o.b) * a.L + t0 + row) * gn + o.g * a.N + c;
            store_quad(p, a.N - c, db[m][v]);
            store_quad(p + a.B * a.L * gn, a.N - c, dc[m][v]);
          } else {
            store_quad(static_cast<T*>(a.db.p) + o.b * a.db.sb + (t0 + row) * a.db.st + o.g * a.N + c, a.N - c, db[m][v]);
            store_quad(static_cast<T*>(a.dc.p) + o.b * a.dc.sb + (t0 + row) * a.dc.st + o.g * a.N + c, a.N - c, dc[m][v]);
          }
        }
    }
  }
  for (int k = 0; k < o.heads; ++k) {
    if (mine && a.p.segs == 1 && a.dh0 != nullptr) {
      const int hv = o.hv0 + k, p0 = hv % a.p.PB * SEL_P;
      float* s = a.dh0 + ((o.b * a.H + hv / a.p.PB) * (int64_t)a.P + p0) * a.N;
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const f4 g = gs_at(k)[(m * 4 + v) * 64];
          const int c = 16 * (w + 4 * m) + li;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (c < a.N && p0 + 16 * v + 4 * lq + r < a.P) s[(int64_t)(16 * v + 4 * lq + r) * a.N + c] = g[r];
        }
    }
  }
  __syncthreads();
  if (tid < o.heads * 3) a.params[((o.b * a.p.segs + o.seg) * a.p.HV + o.hv0) * 3 + tid] = l.sums[tid / 3][tid % 3];
}

// db and dc of a group from its blocks of heads, in their order: 4 elements of a step a thread.
template <typename T>
__global__ __launch_bounds__(SEL_THREADS) void selective_bc_kernel(SelArgs a, int blocks) {
  const int64_t gn = (int64_t)a.G * a.N, per = (gn + 3) / 4, id = a.wg0 + (int64_t)blockIdx.x * SEL_THREADS + threadIdx.x;
  const int64_t row = id / per, c = id % per * 4, all = a.B * a.L * gn;
  if (row >= 2 * a.B * a.L) return;
  const bool second = row >= a.B * a.L;
  const int64_t at = second ? row - a.B * a.L : row, b = at / a.L, t = at % a.L;
  const int nc = (int)(gn - c < 4 ? gn - c : 4);
  f4 s{0, 0, 0, 0};
  for (int i = 0; i < blocks; ++i) {
    float q[4];
    load_part<float, 4>(a.part + ((int64_t)2 * i + second) * all + at * gn + c, nc, q);
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] += q[r];
  }
  const RowsOut& o = second ? a.dc : a.db;
  store_quad(static_cast<T*>(o.p) + b * o.sb + t * o.st + c, nc, s);
}

// dgamma, ddt_bias, dskip of a head: a work-group sums its row blocks' parts, each thread every 256th, in a fixed order.
__global__ __launch_bounds__(SEL_THREADS) void selective_params_kernel(SelArgs a) {
  __shared__ double red[3][SEL_THREADS];
  const int h = blockIdx.x, tid = threadIdx.x;
  const int64_t all = a.B * a.p.segs * a.p.PB;
  double v[3] = {0, 0, 0};
  for (int64_t i = tid; i < all; i += SEL_THREADS) {
    const float* p = a.params + (i / a.p.PB * a.p.HV + (int64_t)h * a.p.PB + i % a.p.PB) * 3;
    for (int j = 0; j < 3; ++j) v[j] += (double)p[j];
  }
  for (int j = 0; j < 3; ++j) red[j][tid] = v[j];
  __syncthreads();
  if (tid < 3) {
    double s = 0;
    for (int i = 0; i < SEL_THREADS; ++i) s += red[tid][i];
    float* out = tid == 0 ? a.dgamma : tid == 1 ? a.ddt_bias : a.dskip;
    if (out != nullptr) out[h] = (float)s;
  }
}

// ---------------------------------------------------------------------------
// One step: a group of LN lanes takes a row p of a state, 4 states a lane.  The states are read and written once; that bounds it.
// ---------------------------------------------------------------------------
template <typename T, int LN>
__global__ __launch_bounds__(SEL_THREADS) void selective_step_kernel(SelArgs a, const float* h, int64_t rows) {
  constexpr int RB = SEL_THREADS / LN;
  const int64_t row = a.wg0 + (int64_t)blockIdx.x * RB + threadIdx.x / LN;
  if (row >= rows) return;
  const int n = threadIdx.x % LN * 4, hp = a.H * a.P, j = (int)(row % hp), hd = j / a.P, g = hd / (a.H / a.G);
  const int64_t b = row / hp;
  const int nn = a.N - n;
  float v[4], bv[4], cv[4];
  if (nn > 0) load_part<float, 4>(h + row * a.N + n, nn, v);
  {
    T q[4];
    const int64_t at = (int64_t)g * a.N + n;
    if (nn > 0) load_part<T, 4>(static_cast<const T*>(a.b.p) + b * a.b.sb + at, nn, q);
#pragma unroll
    for (int r = 0; r < 4; ++r) bv[r] = nn > r ? to_f32(q[r]) : 0.0f;
    if (nn > 0) load_part<T, 4>(static_cast<const T*>(a.c.p) + b * a.c.sb + at, nn, q);
#pragma unroll
    for (int r = 0; r < 4; ++r) cv[r] = nn > r ? to_f32(q[r]) : 0.0f;
  }
  const float u = to_f32(static_cast<const T*>(a.dt.p)[b * a.dt.sb + hd]) + (a.dt_bias != nullptr ? a.dt_bias[hd] : 0.0f);
  const float x = to_f32(static_cast<const T*>(a.x.p)[b * a.x.sb + j]);
  const float d = u != u ? u : fmaxf(u, 0.0f) + log1pf(expf(-fabsf(u)));
  const float keep = expf(-d * a.gamma[hd]), dx = d * x;
  float y = 0.0f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    v[r] = nn > r ? fmaf(keep, v[r], dx * bv[r]) : 0.0f;
    y = nn > r ? fmaf(v[r], cv[r], y) : y;
  }
  if (nn > 0) store_part<float, 4>(a.h_out + row * a.N + n, nn, v);
#pragma unroll
  for (int o = LN / 2; o > 0; o >>= 1) y += __shfl_xor(y, o);
  if (n == 0) static_cast<T*>(a.y)[row] = from_f32<T>(a.skip != nullptr ? fmaf(a.skip[hd], x, y) : y);
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
// a kernel over `all` work-groups, as many launches as 2^32 threads each allow
template <typename F>
hipError_t over(SelArgs& a, int64_t all, F&& launch) {
  const int64_t most = LAUNCH_THREADS / SEL_THREADS;
  for (a.wg0 = 0; a.wg0 < all; a.wg0 += most) {
    launch((uint32_t)(all - a.wg0 < most ? all - a.wg0 : most));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename T, int NT, bool STATES, bool REV>
hipError_t forward(SelArgs a, hipStream_t st) {
  constexpr int HF = NT > 4 ? 2 : 4;
  const int64_t wgs = a.B * a.p.segs * a.G * ((a.p.HG + HF - 1) / HF);
  return over(a, wgs, [&](uint32_t grid) { selective_fwd_kernel<T, NT, HF, STATES, REV><<<grid, SEL_THREADS, 0, st>>>(a); });
}
template <bool REV>
hipError_t join(SelArgs a, hipStream_t st) {
  // (a launch begins with a whole row block)
  const int64_t per = SEL_P * 16 * a.p.NT / 4, all = a.B * a.p.HV, most = LAUNCH_THREADS / per;
  for (a.wg0 = 0; a.wg0 < all; a.wg0 += most) {
    const int64_t n = all - a.wg0 < most ? all - a.wg0 : most;
    selective_join_kernel<REV><<<(uint32_t)((n * per + SEL_THREADS - 1) / SEL_THREADS), SEL_THREADS, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <typename F>
hipError_t by_states(int NT, F&& f) {
  if (NT == 2) return f(std::integral_constant<int, 2>{});
  if (NT == 4) return f(std::integral_constant<int, 4>{});
  return f(std::integral_constant<int, 8>{});
}

}  // namespace

SelPlan sel_plan(bool bf16, int64_t B, int64_t L, int64_t H, int64_t P, int64_t G, int64_t N) {
  SelPlan p{};
  p.NT = N <= 32 ? 2 : N <= 64 ? 4 : 8;
  p.PB = (int)((P + SEL_P - 1) / SEL_P);
  p.HV = (int)(H * p.PB);
  p.HG = (int)(H / G * p.PB);
  p.HF = p.NT > 4 ? 2 : 4;
  p.HR = SEL_BWD_HEADS;
  p.chunks = (L + SEL_Q - 1) / SEL_Q;
  // segments: enough work-groups of the forward for the chip, each with two chunks at least
  const int64_t rows = B * G * ((p.HG + p.HF - 1) / p.HF);
  int64_t segs = (512 + rows - 1) / rows;
  segs = segs > p.chunks / 2 ? p.chunks / 2 : segs;
  segs = segs < 1 ? 1 : segs;
  p.seg = (p.chunks + segs - 1) / segs;
  p.seg = p.seg < 1 ? 1 : p.seg;
  p.segs = p.chunks > 0 ? (p.chunks + p.seg - 1) / p.seg : 1;
  return p;
}

template <typename T>
hipError_t launch_selective_fwd(const SelArgs& a, hipStream_t st) {
  return by_states(a.p.NT, [&](auto nt) {
    if (a.p.segs > 1) {
      hipError_t e = forward<T, nt, true, false>(a, st);
      if (e == hipSuccess) e = join<false>(a, st);
      if (e != hipSuccess) return e;
    }
    return a.y != nullptr || a.L == 0 ? forward<T, nt, false, false>(a, st) : hipSuccess;  // (no y: the states alone)
  });
}

template <typename T>
hipError_t launch_selective_bwd(const SelArgs& a, hipStream_t st) {
  const hipError_t e = by_states(a.p.NT, [&](auto nt) {
    if (a.p.segs > 1) {
      hipError_t e = forward<T, nt, true, true>(a, st);
      if (e == hipSuccess) e = join<true>(a, st);
      if (e != hipSuccess) return e;
    }
    constexpr int lds = (int)sizeof(BwdLds<T, nt>);
    static_assert(lds <= 163840, "a compute unit's LDS");
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(selective_bwd_kernel<T, nt>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
    SelArgs c = a;
    const int64_t wgs = a.B * a.p.segs * a.G * ((a.p.HG + a.p.HR - 1) / a.p.HR);
    return over(c, wgs, [&](uint32_t grid) { selective_bwd_kernel<T, nt><<<grid, SEL_THREADS, lds, st>>>(c); });
  });
  if (e != hipSuccess) return e;
  SelArgs c = a;
  if (a.part != nullptr) {
    const int blocks = (a.p.HG + a.p.HR - 1) / a.p.HR;
    const int64_t all = 2 * a.B * a.L * (((int64_t)a.G * a.N + 3) / 4);
    const int64_t most = LAUNCH_THREADS / SEL_THREADS * SEL_THREADS;
    for (c.wg0 = 0; c.wg0 < all; c.wg0 += most) {
      const int64_t n = all - c.wg0 < most ? all - c.wg0 : most;
      selective_bc_kernel<T><<<(uint32_t)((n + SEL_THREADS - 1) / SEL_THREADS), SEL_THREADS, 0, st>>>(c, blocks);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  }
  selective_params_kernel<<<a.H, SEL_THREADS, 0, st>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_selective_step(const SelArgs& a, const float* h, hipStream_t st) {
  SelArgs c = a;
  const int64_t rows = a.B * a.H * a.P;
  auto go = [&](auto ln) {
    constexpr int LN = ln, RB = SEL_THREADS / LN;
    const int64_t most = LAUNCH_THREADS / SEL_THREADS * RB;
    for (c.wg0 = 0; c.wg0 < rows; c.wg0 += most) {
      const int64_t n = rows - c.wg0 < most ? rows - c.wg0 : most;
      selective_step_kernel<T, LN><<<(uint32_t)((n + RB - 1) / RB), SEL_THREADS, 0, st>>>(c, h, rows);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  return a.N <= 16 ? go(std::integral_constant<int, 4>{}) : a.N <= 64 ? go(std::integral_constant<int, 16>{}) : go(std::integral_constant<int, 32>{});
}

template hipError_t launch_selective_fwd<float>(const SelArgs&, hipStream_t);
template hipError_t launch_selective_fwd<bf16_t>(const SelArgs&, hipStream_t);
template hipError_t launch_selective_bwd<float>(const SelArgs&, hipStream_t);
template hipError_t launch_selective_bwd<bf16_t>(const SelArgs&, hipStream_t);
template hipError_t launch_selective_step<float>(const SelArgs&, const float*, hipStream_t);
template hipError_t launch_selective_step<bf16_t>(const SelArgs&, const float*, hipStream_t);

}  // namespace res
