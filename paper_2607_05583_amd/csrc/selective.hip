// Selective scan, per head a state h [P, N]:
//   D_t = softplus(dt_t + dt_bias),  a_t = exp(-gamma D_t),
//   h_t = a_t h_{t-1} + D_t x_t b_t^T,  y_t = h_t c_t + skip x_t.
// In a chunk of Q = 64 steps with s_t = sum_{u<=t} gamma D_u, h the state before it and E[t,s] = exp(s_s - s_t) for s <= t:
//   y_t = exp(-s_t) h c_t + sum_{s<=t} (c_t.b_s) E[t,s] D_s x_s,
//   h' = exp(-s_Q) h + sum_s exp(s_s - s_Q) D_s x_s b_s^T,
// which are matrix products (MFMA).  The backward, with g the gradient of the state behind the chunk and K[t,s] = dy_t.x_s:
//   dc_t = sum_s E D_s K b_s + exp(-s_t) h^T dy_t,      db_s = D_s (sum_t E K c_t + exp(s_s - s_Q) g^T x_s),
//   du_s = sum_t E (c_t.b_s) dy_t + exp(s_s - s_Q) g b_s,  dx_s = D_s du_s + skip dy_s,
//   dl_t = exp(-s_Q) <g, h> + sum_{u>=t} exp(-s_u) dy_u.(h c_u) + sum_{s<t} (D_s exp(s_s - s_Q) x_s.(g b_s) + sum_{u>=t} Z[u,s])
//   (the gradient of log a_t; Z = (c.b) E D K),
//   dD_s = x_s.du_s - gamma dl_s,  dgamma = -sum D dl,  g' = exp(-s_Q) g + sum_t exp(-s_t) dy_t c_t^T.
// dl and x.du need no rounded products: their parts within the chunk are sums of Z in float32, those of the states are products
// of operands in three parts.
//
// Rounding, bf16 inputs: products of two inputs are exact.  An operand that is computed goes in as three bf16 parts (2^-24 of it is
// lost) where float32 results depend on it: the weighted x, b and c that make states and their gradients, and those in dl.
// States that are read for y go in as two parts (2^-16); the weights (c.b) E D and E D K that only make bf16 outputs, and g
// in du, as one (2^-8 a term, as much as the output's own rounding).
// float32 inputs use float32 MFMA throughout.  Sums and states are float32.
// The matrix unit's bf16 sums are low by some 2^-28 of their terms on average, whatever their sign (measured: 5 million products of
// normal values, each off by up to 2^-20 either way).  In dgamma, a sum over all steps, that stands out (5e-6 of it): every other
// chunk's states and gradients are held with the other sign in the backward, so that what is low there makes up for it.
#include <type_traits>

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
  struct Split { bf8 hi, lo; };       // two parts: 2^-16 of a value is lost
  struct Whole { bf8 hi, mid, lo; };  // three: 2^-24
  struct Quad { uint32_t v[2]; } __attribute__((aligned(8)));
  static constexpr int PAD = 8;
  __device__ static __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  __device__ static __forceinline__ f4 mma(const Split& a, const Frag& b, f4 c) { return mma(a.hi, b, mma(a.lo, b, c)); }
  __device__ static __forceinline__ f4 mma(const Whole& a, const Frag& b, f4 c) { return mma(a.hi, b, mma(a.mid, b, mma(a.lo, b, c))); }
  __device__ static __forceinline__ f4 mma(const Frag& a, const Whole& b, f4 c) { return mma(a, b.hi, mma(a, b.mid, mma(a, b.lo, c))); }
  __device__ static __forceinline__ Whole whole(const float (&v)[8]) {
    Whole s;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s.hi[j] = (__bf16)v[j];
      const float left = v[j] - (float)s.hi[j];
      s.mid[j] = (__bf16)left;
      s.lo[j] = (__bf16)(left - (float)s.mid[j]);
    }
    return s;
  }
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
  typedef Frag Split, Whole;
  static constexpr int PAD = 4;
  __device__ static __forceinline__ f4 mma(const Frag& a, const Frag& b, f4 c) { return mma_f32(a.v[1], b.v[1], mma_f32(a.v[0], b.v[0], c)); }
  __device__ static __forceinline__ Frag one(const float (&v)[8]) { return Frag{{f4{v[0], v[1], v[2], v[3]}, f4{v[4], v[5], v[6], v[7]}}}; }
  __device__ static __forceinline__ Frag split(const float (&v)[8]) { return one(v); }
  __device__ static __forceinline__ Frag whole(const float (&v)[8]) { return one(v); }
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
// 4 results to a row of memory, n of them (WHOLE: all or none)
template <bool WHOLE, typename T>
__device__ __forceinline__ void store_quad(T* p, int n, const f4& v) {
  if constexpr (WHOLE) {
    T q[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) q[r] = from_f32<T>(v[r]);
    if (n > 0) store_part<T, 4>(p, 4, q);
    return;
  }
  T q[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) q[r] = from_f32<T>(v[r]);
  store_part<T, 4>(p, n < 0 ? 0 : n, q);
}

// ---------------------------------------------------------------------------
// Tiles: Q rows of COLS elements from memory to registers (zeros outside) and on to LDS rows of COLS + PAD.  WHOLE: P and N are
// whole numbers of 16-byte vectors, so that no vector is cut.  (Both in one kernel, the paths of cut vectors were a third of its
// code, and their addresses spilled the scalar registers.)
// ---------------------------------------------------------------------------
template <typename T, int COLS, bool WHOLE> struct Tile {
  static constexpr int V = 16 / (int)sizeof(T), PR = COLS / V, RT = SEL_THREADS / PR, U = Q / RT, LD = COLS + Mx<T>::PAD;
  static constexpr int BYTES = Q * LD * (int)sizeof(T);
  T v[U][V];
  // rows at distance st (elements; below 2^21, so that a lane's offset has 32 bits) from p, which is the same in all lanes
  __device__ __forceinline__ void load(const T* p, uint32_t st, int rows, int cols, int tid) {
    const int r0 = tid / PR, c = tid % PR * V, n = cols - c;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* at = reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) + ((uint32_t)(r0 + u * RT) * st + (uint32_t)c) * (uint32_t)sizeof(T));
      if (r0 + u * RT < rows && n > 0)
        load_part<T, V>(at, WHOLE ? V : n, v[u]);
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

// Sums over lanes that stay in the vector unit.  (Through LDS, as a general shuffle goes, each step waits some 130 cycles.)
template <int CTRL>
__device__ __forceinline__ float lanes_add(float v) {  // v and that of another lane of the 16; 0 where there is none
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum_lanes(float v) {  // over the 16 lanes of a row
  v = lanes_add<0xB1>(v);         // neighbours
  v = lanes_add<0x4E>(v);         // pairs
  v = lanes_add<0x141>(v);        // halves of eight, mirrored
  return lanes_add<0x140>(v);     // halves of sixteen, mirrored
}
__device__ __forceinline__ float sum_rows(float v) {  // over the 4 lanes i, i + 16, i + 32, i + 48
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const unsigned a = __float_as_uint(v);
  const u2 p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const float s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  const unsigned b = __float_as_uint(s);
  const u2 q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
__device__ __forceinline__ float rows_behind(float v, int row) {  // over the lanes i + 16 r with r > row
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const unsigned a = __float_as_uint(v);
  const u2 p = __builtin_amdgcn_permlane16_swap(a, a, false, false);  // rows 0 0 2 2, rows 1 1 3 3
  const unsigned b = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
  const u2 q = __builtin_amdgcn_permlane32_swap(b, b, false, false);  // rows 0 + 1, rows 2 + 3
  return ((row & 1) == 0 ? __uint_as_float(p[1]) : 0.0f) + (row < 2 ? __uint_as_float(q[1]) : 0.0f);
}
__device__ __forceinline__ float sum_wave(float v) { return sum_rows(sum_lanes(v)); }
__device__ __forceinline__ float prefix_lanes(float v) {  // over the lanes of a row up to this one
  v = lanes_add<0x111>(v);
  v = lanes_add<0x112>(v);
  v = lanes_add<0x114>(v);
  return lanes_add<0x118>(v);
}
__device__ __forceinline__ float suffix_lanes(float v) {  // from this one on
  v = lanes_add<0x101>(v);
  v = lanes_add<0x102>(v);
  v = lanes_add<0x104>(v);
  return lanes_add<0x108>(v);
}
__device__ __forceinline__ float of_lane(float v, int lane) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// A chunk's steps, one a lane (by one wave).  Sums of gamma D (base 2): s up to and with a step, after behind it, and the same
// within its tile of 16 steps (in, behind): what decays between steps of two tiles is summed from these, since a difference of s
// loses what is small beside s (2^-24 of up to some hundred).  Between steps of one tile it is a difference of in, which has a
// second word for that (rest: what in lost to rounding).
struct Steps {
  float d, s, after, in, rest, behind, total, slope;
};
template <int CTRL>
__device__ __forceinline__ void lanes_add(float& v, float& rest) {  // with what each sum loses, exactly (the sum's error is a float)
  const float u = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
  rest = lanes_add<CTRL>(rest);
  const float s = v + u, of_u = s - v;
  rest += (v - (s - of_u)) + (u - of_u);
  v = s;
}
// the step's logit, loaded ahead of its use
template <typename T>
__device__ __forceinline__ float load_step(const SelArgs& a, int64_t b, int64_t t, int64_t n, int h, int lane) {
  return t + lane < n ? to_f32(static_cast<const T*>(a.dt.p)[b * a.dt.sb + (t + lane) * a.dt.st + h]) : 0.0f;
}
__device__ __forceinline__ Steps steps_of(const SelArgs& a, float v, bool inside, int h, int lane) {
  Steps o{0, 0, 0, 0, 0, 0, 0, 0};
  float ld = 0.0f;
  if (inside) {
    v += a.dt_bias != nullptr ? a.dt_bias[h] : 0.0f;
    o.d = fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v)));
    if (v != v) o.d = v;
    o.slope = 1.0f / (1.0f + expf(-v));
    ld = o.d * a.gamma[h] * LOG2E;
    ld = ld > NO_MORE ? NO_MORE : ld;
  }
  const float next = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, ld), 0x101, 0xF, 0xF, true));
  o.in = ld;
  lanes_add<0x111>(o.in, o.rest);
  lanes_add<0x112>(o.in, o.rest);
  lanes_add<0x114>(o.in, o.rest);
  lanes_add<0x118>(o.in, o.rest);
  o.behind = suffix_lanes(next);  // (the next lane's on; nothing behind the last)
  o.s = o.in;
  o.after = o.behind;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const float all = of_lane(o.in, 16 * t + 15);
    o.total += all;
    if (t < lane >> 4) o.s += all;
    if (t > lane >> 4) o.after += all;
  }
  return o;
}
// what a tile's steps decay, from s and in of its first step's lane on: sums of whole tiles between tiles si and ti
struct Between {
  float in[Q], rest[Q], behind[Q], tile[4];  // (behind: negative)
  __device__ __forceinline__ void put(const Steps& s, int lane) {
    in[lane] = s.in;
    rest[lane] = s.rest;
    behind[lane] = -s.behind;
    if ((lane & 15) == 15) tile[lane >> 4] = s.in;
  }
  // exponents of E over 4 steps t of a tile from step s (in its lane), or 4 steps s to step t: to[] + from
  __device__ __forceinline__ float gap(int si, int ti) const {  // whole tiles between
    return ti - si < 2 ? 0.0f : ti - si < 3 ? tile[si + 1] : tile[1] + tile[2];
  }
};

// The value again, as one that the compiler does not know: what is computed from it stays where it is used.  (Hoisted out of the
// loops, the backward's addresses took more registers than there are.)
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Which rows a work-group has: its batch row, segment, group and row blocks hv0 .. hv0 + heads (of the batch row's HV).
struct Place {
  int64_t b, seg;
  int g, block, hv0, heads;
};
__device__ __forceinline__ Place place_of(const SelArgs& a, int per, uint32_t* index) {
  const uint32_t blocks = (uint32_t)((a.p.HG + per - 1) / per), G = (uint32_t)a.G, segs = (uint32_t)a.p.segs;
  // Work-groups go to the eight dies in turn: die d takes the d-th eighth of the launch's, so that the blocks of a group, which
  // read the same b and c, run together on one die and share them in its cache.  (Fewer than 2^31 work-groups.)
  const uint32_t n = gridDim.x, d = blockIdx.x % 8, q = n / 8, r = n % 8;
  uint32_t id = (uint32_t)a.wg0 + d * q + (d < r ? d : r) + blockIdx.x / 8;
  *index = id;
  Place o;
  o.block = (int)(id % blocks);
  id /= blocks;
  o.g = (int)(id % G);
  id /= G;
  o.seg = id % segs;
  o.b = id / segs;
  o.hv0 = o.g * a.p.HG + o.block * per;
  o.heads = a.p.HG - o.block * per < per ? a.p.HG - o.block * per : per;
  return o;
}
__device__ __forceinline__ int64_t length_of(const SelArgs& a, int64_t b) {
  if (a.lengths == nullptr) return a.L;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.L ? a.L : n;
}

// A state of the workspace: tiles of 16 x 16, of 4 row tiles v for each state tile m, with lane (n, q) holding p = 4 q .. + 3 of it, as
// the backward's waves need them.
__device__ __forceinline__ int state_index(int p, int n) { return (((n >> 4) * 4 + (p >> 4)) * 64 + ((p >> 2) & 3) * 16 + (n & 15)) * 4 + (p & 3); }
__device__ __forceinline__ int64_t border(const SelArgs& a, int64_t b, int hv, int64_t seg) {
  return ((b * a.p.HV + hv) * a.p.segs + seg) * (int64_t)(SEL_P * 16 * a.p.NT);
}
// An element of a caller's state [B][H][P][N] (none: zero), of a row block
__device__ __forceinline__ float state_of(const SelArgs& a, const float* s, int64_t b, int hv, int p, int n) {
  p += (hv & a.p.PS) * SEL_P;
  return s != nullptr && p < a.P && n < a.N ? s[((b * a.H + (hv >> a.p.PS)) * a.P + p) * (int64_t)a.N + n] : 0.0f;
}

// The tiles on and below the diagonal: of the 10, wave w has w, w + 4 and w + 8, the last one again where there are no more.
struct TileId {
  int t, s;
};
__device__ __forceinline__ TileId tile_id(int w, int e) {
  const int id = w + 4 * e < 10 ? w + 4 * e : 9, t = id < 1 ? 0 : id < 3 ? 1 : id < 6 ? 2 : 3;
  return TileId{t, id - t * (t + 1) / 2};
}
// What is loaded before stays before, what is computed behind stays behind: loads of a product go together, and it waits once.
__device__ __forceinline__ void loads_first() { __builtin_amdgcn_sched_barrier(0); }

// ---------------------------------------------------------------------------
// Forward: a wave owns 16 of a row block's 64 rows.  Its states are in registers, transposed: lane (p, q) holds
// n = 16 v + 4 q .. + 3.  STATES: only the segment's end state from a zero start, the other way round (and REV: the gradient that the segment
// gives to the state before it: dy, c and exp(-s_t) in the place of x, b and the weights, from the last chunk back).
// The next head's x (the next chunk's b, c and steps) are loaded to registers while a head's products run.
// Some heads share a work-group's b, c and (c.b): four, or two where 128 states leave registers for no more.  Two passes over x and b
// instead of a wait for the segment before: 8 x 8192, 8 heads of 64 x 64, bf16: states 40 us, forward 95 (134 MB, a seventh of the
// matrix rate); 4 x 32768, 128 states: 90 and 224.  Vector instructions and their latency bound both: two waves a SIMD, whose
// registers are full, half of whose cycles they take; the matrix unit is busy for a fifth of the time.
// ---------------------------------------------------------------------------
template <typename T, int NT, int HF, bool WHOLE, bool STATES, bool REV>
__global__ __launch_bounds__(SEL_THREADS, sizeof(T) == 2 ? 2 : 1) void selective_fwd_kernel(SelArgs a) {
  typedef Mx<T> M;
  constexpr int NP = 16 * NT, KS = NT / 2;
  typedef Tile<T, NP, WHOLE> TB;
  typedef Tile<T, SEL_P, WHOLE> TX;
  __shared__ __align__(16) T bt[Q * TB::LD];
  __shared__ __align__(16) T ct[STATES ? 8 : Q * TB::LD];
  __shared__ __align__(16) T xt[2][Q * TX::LD];
  __shared__ __align__(16) T mt[STATES ? 1 : 2][STATES ? 8 : 6 * 64 * 8];
  __shared__ __align__(16) Between gap[STATES ? 1 : HF];
  __shared__ __align__(16) float sd[HF][Q], sw[HF][Q], sp[HF][Q], st[HF];  // D, D exp(what follows), exp(-s), the chunk's total
  uint32_t index;
  const Place o = place_of(a, HF, &index);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, lq = lane >> 4;
  const int64_t n = length_of(a, o.b);
  const int64_t c0 = o.seg * a.p.seg, c1 = c0 + a.p.seg < a.p.chunks ? c0 + a.p.seg : a.p.chunks;
  const int64_t some = (n + Q - 1) / Q - c0, active = some < 0 ? 0 : some < c1 - c0 ? some : c1 - c0;  // chunks with steps
  const Rows rx = REV ? a.dy : a.x, rb = REV ? a.c : a.b;
  const T* px = static_cast<const T*>(rx.p) + o.b * rx.sb;
  const T* pb = static_cast<const T*>(rb.p) + o.b * rb.sb + o.g * a.N;
  const T* pc = static_cast<const T*>(a.c.p) + o.b * a.c.sb + o.g * a.N;
  const int64_t hp = (int64_t)a.H * a.P;

  f4 h[HF][NT];
  float total[HF];
#pragma unroll
  for (int k = 0; k < HF; ++k) {
    total[k] = 0.0f;
#pragma unroll
    for (int v = 0; v < NT; ++v) h[k][v] = f4{0, 0, 0, 0};
    if (!STATES && k < o.heads) {
      const float* e = a.enter + border(a, o.b, o.hv0 + k, o.seg);
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int p = 16 * w + li, n = 16 * v + 4 * lq + r;
          h[k][v][r] = a.p.segs > 1 ? e[state_index(p, n)] : state_of(a, a.h0, o.b, o.hv0 + k, p, n);
        }
    }
  }
  if constexpr (!STATES) {
    // the tiles above the diagonal that share a fragment with one on it stay zero
    for (int i = tid; i < 2 * 6 * 64 * 8; i += SEL_THREADS) mt[0][i] = T(0);
  }
  auto start_of = [&](int64_t ci) { return (REV ? c0 + active - 1 - ci : c0 + ci) * Q; };
  auto rows_at = [&](int64_t t0) { return (int)(n - t0 < Q ? n - t0 : Q); };
  TB rb0, rc0;
  TX rx0;
  float step = 0.0f;
  auto load_chunk = [&](int64_t ci) {  // (a wave has at most one head)
    const int64_t t0 = start_of(ci);
    rb0.load(pb + t0 * rb.st, (uint32_t)rb.st, rows_at(t0), a.N, here(tid));
    if constexpr (!STATES) rc0.load(pc + t0 * a.c.st, (uint32_t)a.c.st, rows_at(t0), a.N, here(tid));
    if (w < o.heads) step = load_step<T>(a, o.b, t0, n, (o.hv0 + w) >> a.p.PS, lane);
  };
  auto load_x = [&](int64_t ci, int k) {
    const int64_t t0 = start_of(ci);
    const int hv = o.hv0 + k, p0 = (hv & a.p.PS) * SEL_P;
    rx0.load(px + t0 * rx.st + (hv >> a.p.PS) * a.P + p0, (uint32_t)rx.st, rows_at(t0), a.P - p0, here(tid));
  };
  if (active > 0) {
    load_chunk(0);
    load_x(0, 0);
  }
  int turn = 0;  // which of two buffers a head's x and weights are in
  for (int64_t ci = 0; ci < active; ++ci) {
    const int64_t t0 = start_of(ci);
    const int rows = rows_at(t0), held = (int)(a.L - t0 < Q ? a.L - t0 : Q);
    __syncthreads();  // the last chunk's readers are through
    rb0.put(bt);
    if constexpr (!STATES) rc0.put(ct);
    if (w < o.heads) {
      const Steps s = steps_of(a, step, lane < rows, (o.hv0 + w) >> a.p.PS, lane);
      sd[w][lane] = s.d;
      sp[w][lane] = exp2_fast(-s.s);
      sw[w][lane] = REV ? ((ci & 1) != 0 ? exp2_fast(-s.s) : -exp2_fast(-s.s)) : s.d * exp2_fast(-s.after);
      if constexpr (!STATES) gap[w].put(s, lane);
      if (lane == 0) st[w] = s.total;
    }
    if (ci + 1 < active) load_chunk(ci + 1);
    __syncthreads();
    // G^T [s][t] = b c^T: tile e of 10 (this wave's are w, w + 4, w + 8) is t tile ti, s tile si <= ti
    f4 g[3];
    if constexpr (!STATES) {
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const TileId id = tile_id(w, e);
        typename M::Frag fb[KS], fc[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          fb[k] = M::row(bt + (16 * id.s + li) * TB::LD + 32 * k + 4 * lq);
          fc[k] = M::row(ct + (16 * id.t + li) * TB::LD + 32 * k + 4 * lq);
        }
        loads_first();
        g[e] = f4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) g[e] = M::mma(fb[k], fc[k], g[e]);
      }
    }
#pragma unroll
    for (int k = 0; k < HF; ++k) {
      if (k >= o.heads) break;
      const int lane = here(tid & 63), li = lane & 15, lq = lane >> 4;
      const int hv = o.hv0 + k, hd = (hv >> a.p.PS), p0 = (hv & a.p.PS) * SEL_P;
      T* const xk = xt[turn];
      T* const mk = mt[STATES ? 0 : turn];
      turn ^= 1;
      rx0.put(xk);  // (its readers, two heads ago, were through before the last barrier)
      if (k + 1 < o.heads)
        load_x(ci, k + 1);
      else if (ci + 1 < active)
        load_x(ci + 1, 0);
      if constexpr (!STATES) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
          const TileId id = tile_id(w, e);
          const Between& b = gap[k];
          const float to = -(b.in[16 * id.t + li] + b.gap(id.s, id.t));
          // (rest: what it changes is below a bf16 y's rounding)
          constexpr bool REST = sizeof(T) == 4;
          const float to_rest = REST ? b.rest[16 * id.t + li] : 0.0f;
          const f4 rest = REST ? load_f4(&b.rest[16 * id.s + 4 * lq]) : f4{0, 0, 0, 0};
          const f4 from = load_f4((id.s == id.t ? b.in : b.behind) + 16 * id.s + 4 * lq), d = load_f4(&sd[k][16 * id.s + 4 * lq]);
          f4 m;
#pragma unroll
          for (int r = 0; r < 4; ++r) m[r] = id.s < id.t || 4 * lq + r <= li ? g[e][r] * (exp2_fast((from[r] + to) + (REST && id.s == id.t ? rest[r] - to_rest : 0.0f)) * d[r]) : 0.0f;
          // fragment (t tile, 32 steps s): 0, 1, 2 and 3, 4 and 5 of t tiles 0, 1, 2, 3
          const int f = id.t < 2 ? id.t : 2 * id.t - 2 + (id.s >> 1);
          put_quad(&mk[(f * 64 + lane) * 8 + (id.s & 1) * 4], m);
        }
      }
      __syncthreads();
      typename M::Frag xf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) xf[j] = M::col(xk + 32 * j * TX::LD + 16 * w, TX::LD, li, lq);
      if constexpr (!STATES) {
        f4 y[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) y[t] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          typename M::Frag cf[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) cf[t] = M::row(ct + (16 * t + li) * TB::LD + 32 * j + 4 * lq);
          float hf[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) hf[r] = h[k][2 * j + (r >> 2)][r & 3];
          const typename M::Split hp = M::split(hf);
          loads_first();
#pragma unroll
          for (int t = 0; t < 4; ++t) y[t] = M::mma(hp, cf[t], y[t]);
        }
        typename M::Frag mf[6];
        f4 xr[4];
        float f[4];
#pragma unroll
        for (int i = 0; i < 6; ++i) mf[i] = *reinterpret_cast<const typename M::Frag*>(&mk[(i * 64 + lane) * 8]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          f[t] = sp[k][16 * t + li];
          xr[t] = quad(xk + (16 * t + li) * TX::LD + 16 * w + 4 * lq);
        }
        loads_first();
        const float skip = a.skip != nullptr ? a.skip[hd] : 0.0f;
        T* yp = static_cast<T*>(a.y) + (o.b * a.L + t0) * hp + hd * a.P + p0 + 16 * w;
        const int cols = a.P - p0 - 16 * w - 4 * lq;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int r = 0; r < 4; ++r) y[t][r] *= f[t];
#pragma unroll
          for (int j = 0; j <= t / 2; ++j) y[t] = M::mma(xf[j], mf[t < 2 ? t : 2 * t - 2 + j], y[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int row = 16 * t + li;
#pragma unroll
          for (int r = 0; r < 4; ++r) y[t][r] = row < rows ? fmaf(skip, xr[t][r], y[t][r]) : 0.0f;
          if (row < held) store_quad<WHOLE>(yp + ((uint32_t)row * (uint32_t)hp + 4 * lq), cols, y[t]);
        }
      }
      const float keep = REV ? -exp2_fast(-st[k]) : exp2_fast(-st[k]);  // (a gradient's sign turns with each chunk)
      total[k] += st[k];
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) h[k][v][r] *= keep;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        typename M::Frag bf[NT];
#pragma unroll
        for (int v = 0; v < NT; ++v) bf[v] = M::col(bt + 32 * j * TB::LD + 16 * v, TB::LD, li, lq);
        const f4 w0 = load_f4(&sw[k][32 * j + 4 * lq]), w1 = load_f4(&sw[k][32 * j + 16 + 4 * lq]);
        float xw[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) xw[r] = M::at(xf[j], r) * (r < 4 ? w0[r & 3] : w1[r & 3]);
        const typename M::Whole xp = M::whole(xw);
        loads_first();
#pragma unroll
        for (int v = 0; v < NT; ++v) h[k][v] = STATES ? M::mma(xp, bf[v], h[k][v]) : M::mma(bf[v], xp, h[k][v]);
      }
    }
  }
  if constexpr (!STATES) {  // behind the row's end: the state stays
    for (int64_t ch = c0 + active; ch < c1; ++ch) {
      const int64_t t0 = ch * Q;
      const int held = (int)(a.L - t0 < Q ? a.L - t0 : Q);
      T* y = static_cast<T*>(a.y) + (o.b * a.L + t0) * hp;
      for (int k = 0; k < o.heads; ++k) {
        const int hv = o.hv0 + k, p0 = (hv & a.p.PS) * SEL_P;
        const int cols = a.P - p0 < SEL_P ? a.P - p0 : SEL_P;
        for (int i = tid; i < held * SEL_P; i += SEL_THREADS)
          if (i % SEL_P < cols) y[(i / SEL_P) * hp + (hv >> a.p.PS) * a.P + p0 + i % SEL_P] = T(0);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < HF; ++k) {
    if (k >= o.heads) break;
    const int hv = o.hv0 + k, p = 16 * w + li;
    if constexpr (STATES) {
      const int64_t at = (o.b * a.p.HV + hv) * a.p.segs + o.seg;
      f4* s = reinterpret_cast<f4*>((REV ? a.leave : a.enter) + at * (SEL_P * NP)) + w * 64 + lane;
#pragma unroll
      for (int v = 0; v < NT; ++v) s[v * 256] = REV && (active & 1) != 0 ? -h[k][v] : h[k][v];
      if (tid == 0) a.decay[at] = total[k];
    } else if (a.p.segs == 1 && a.h_out != nullptr) {
      const int p0 = (hv & a.p.PS) * SEL_P;
      float* s = a.h_out + ((o.b * a.H + (hv >> a.p.PS)) * (int64_t)a.P + p0 + p) * a.N;
#pragma unroll
      for (int v = 0; v < NT; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (p0 + p < a.P && 16 * v + 4 * lq + r < a.N) s[16 * v + 4 * lq + r] = h[k][v][r];
    }
  }
}

// The segments' states one after the other: each segment's own end state makes way for the state that enters it.  An element a
// thread, so that there are enough of them for the latency of the segments' loads, some of which go together.  64 rows of 64 x 64 states in
// 32 segments: 15 us (67 MB).
template <bool REV>
__global__ __launch_bounds__(SEL_THREADS) void selective_join_kernel(SelArgs a) {
  const int per = SEL_P * 16 * a.p.NT;
  const int64_t id = (int64_t)blockIdx.x * SEL_THREADS + threadIdx.x, bh = a.wg0 + id / per;
  if (bh >= a.B * a.p.HV) return;
  const int at = (int)(id % per), lane = (at >> 2) & 63, tile = at >> 8, hv = (int)(bh % a.p.HV);
  const int p = 16 * (tile & 3) + 4 * (lane >> 4) + (at & 3), n = 16 * (tile >> 2) + (lane & 15);
  const int64_t b = bh / a.p.HV;
  float e = state_of(a, REV ? a.dh_out : a.h0, b, hv, p, n);
  float* buf = (REV ? a.leave : a.enter) + bh * a.p.segs * (int64_t)per + at;
  const float* decay = a.decay + bh * a.p.segs;
  constexpr int U = 16;  // segments loaded together
  for (int64_t i = 0; i < a.p.segs; i += U) {
    float own[U], keep[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < a.p.segs) {
        const int64_t k = REV ? a.p.segs - 1 - i - u : i + u;
        own[u] = buf[k * per];
        keep[u] = decay[k];
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < a.p.segs) {
        const int64_t k = REV ? a.p.segs - 1 - i - u : i + u;
        buf[k * per] = e;
        e = fmaf(exp2_fast(-keep[u]), e, own[u]);
      }
  }
  float* out = REV ? a.dh0 : a.h_out;
  const int p1 = (hv & a.p.PS) * SEL_P + p;
  if (out != nullptr && n < a.N && p1 < a.P) out[((b * a.H + (hv >> a.p.PS)) * (int64_t)a.P + p1) * a.N + n] = e;
}

// ---------------------------------------------------------------------------
// Backward: a work-group takes a segment of up to SEL_BWD_HEADS row blocks of a group, so that db and dc are summed over them
// in registers.  First the states before each chunk are made again (to hs), a head after the other; then the chunks from the
// last one back, in each head after head.  A wave owns the 16-state tiles w, w + 4: there states and their gradients are
// lanes (n, q) with p = 16 v + 4 q .. + 3, as their products with x and dy need them; du, which needs a row's states, takes
// them through LDS.  What the next head needs is loaded to registers meanwhile.
// 8 x 8192, 8 heads of 64 x 64, bf16: 300 us, of which the states' second making some 45 and their way through memory 30.  Vector
// instructions take half of all cycles (some 2000 of a wave for a head's chunk; the matrix unit a tenth), at two waves a SIMD with 37
// registers spilled.  It writes 377 MB and reads 367 or more where inputs and outputs are 235: the rest are states, their gradients (a
// head's goes to memory and back at every chunk), and db and dc of the blocks of heads.
// ---------------------------------------------------------------------------
template <typename T, int NT, bool WHOLE> struct BwdLds {
  static constexpr int SL = NT < 4 ? NT : 4, NS = 16 * SL;  // state tiles of a slice, which goes through LDS at once
  typedef Tile<T, 16 * NT, WHOLE> TB;
  typedef Tile<T, SEL_P, WHOLE> TX;
  __align__(16) T bc[2][Q * TB::LD];  // b, c
  __align__(16) T xd[2][Q * TX::LD];  // x, dy
  __align__(16) T ek[Q * TX::LD];     // row s: E[t,s] D_s K[t,s] over t
  __align__(16) T eg[Q * TX::LD];     // row s: E[t,s] (c_t.b_s)
  __align__(16) T gx[NS * TX::LD];    // row n: g over p
  __align__(16) Between gap;
  __align__(16) float d[Q], suf[Q], pre[Q], slope[Q];  // D, exp(-what follows), exp(-s), dD / d dt
  __align__(16) float rowz[4][Q], colz[4][Q], ic[4][Q], ig[4][Q];  // by s tile, by t tile, by wave, by wave
  float zd[Q], lam[4], sums[SEL_BWD_HEADS][3], skip[4], total[2];  // Z's diagonal; <g, h> by wave
};

template <typename T, int NT, bool WHOLE>
__global__ __launch_bounds__(SEL_THREADS, sizeof(T) == 2 && NT <= 4 ? 2 : 1) void selective_bwd_kernel(SelArgs a) {
  typedef Mx<T> M;
  typedef BwdLds<T, NT, WHOLE> Lds;
  typedef typename Lds::TB TB;
  typedef typename Lds::TX TX;
  constexpr int KS = NT / 2, NW = (NT + 3) / 4, SL = Lds::SL, STATE = NT * 4 * 64;  // (f4 of a state, of the waves that have tiles)
  extern __shared__ __align__(16) char raw[];
  Lds& l = *reinterpret_cast<Lds*>(raw);
  T *const bt = l.bc[0], *const ct = l.bc[1], *const xt = l.xd[0], *const dt = l.xd[1];
  uint32_t index;
  const Place o = place_of(a, a.p.HR, &index);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, lq = lane >> 4;
  const int64_t n = length_of(a, o.b);
  const int64_t c0 = o.seg * a.p.seg;
  const int all = (int)(a.p.chunks - c0 < a.p.seg ? a.p.chunks - c0 : a.p.seg);  // chunks of the segment
  const int64_t some = (n + Q - 1) / Q - c0;
  const int active = (int)(some < 0 ? 0 : some < all ? some : all);              // those with steps
  // where the segment's rows begin, and the distance of their steps
  const uint32_t sx = (uint32_t)a.x.st, sy = (uint32_t)a.dy.st, sb = (uint32_t)a.b.st, sc = (uint32_t)a.c.st, sd = (uint32_t)a.dt.st;
  const T* px = static_cast<const T*>(a.x.p) + o.b * a.x.sb + c0 * Q * a.x.st;
  const T* pd = static_cast<const T*>(a.dy.p) + o.b * a.dy.sb + c0 * Q * a.dy.st;
  const T* pb = static_cast<const T*>(a.b.p) + o.b * a.b.sb + c0 * Q * a.b.st + o.g * a.N;
  const T* pc = static_cast<const T*>(a.c.p) + o.b * a.c.sb + c0 * Q * a.c.st + o.g * a.N;
  const T* pt = static_cast<const T*>(a.dt.p) + o.b * a.dt.sb + c0 * Q * a.dt.st;
  const int left = (int)(n - c0 * Q < (int64_t)active * Q ? n - c0 * Q : (int64_t)active * Q);  // steps of the segment (with active chunks)
  auto step_at = [&](int ci, int hd) { return ci * Q + lane < left ? to_f32(pt[(int64_t)(ci * Q) * sd + (uint32_t)lane * sd + hd]) : 0.0f; };
  const bool mine = w < NT;  // the wave has state tiles
  // states of a work-group before its chunks, and their gradients: [chunk][head][own tile][wave][p tile][lane].  Before the first
  // chunk and behind the last they are those at the segment's borders, or the caller's, which are put here first.
  f4* const hs = a.hs + (int64_t)index * a.p.seg * a.p.HR * STATE + w * 256;
  f4* const gs = a.gs + (int64_t)index * a.p.HR * STATE + w * 256;
  const bool several = a.p.segs > 1;
  const f4* const enter = reinterpret_cast<const f4*>(several ? a.enter + border(a, o.b, o.hv0, o.seg) : nullptr) + w * 256;
  const f4* const leave = reinterpret_cast<const f4*>(several ? a.leave + border(a, o.b, o.hv0, o.seg) : nullptr) + w * 256;
  const int64_t next = a.p.segs * (int64_t)(SEL_P * 16 * NT / 4);  // from a row block's to the next one's, in f4
  // (own tile m is the work-group's tile w + 4 m: four waves' tiles further in both layouts)
  auto hs_at = [&](int c, int k) { return c > 0 || !several ? hs + (int64_t)(c * a.p.HR + k) * STATE : const_cast<f4*>(enter) + k * next; };
  auto gs_at = [&](int k, bool last) { return last && several ? const_cast<f4*>(leave) + k * next : gs + k * STATE; };
  auto rows_at = [&](int ci) { return left - ci * Q < Q ? left - ci * Q : Q; };
  auto held_at = [&](int ci) { const int64_t h = a.L - (c0 + ci) * Q; return (int)(h < Q ? h : Q); };  // rows of the chunk at all
  auto at_of = [&](int k) { return ((o.hv0 + k) >> a.p.PS) * a.P + ((o.hv0 + k) & a.p.PS) * SEL_P; };  // a row block's columns
  auto cols_of = [&](int k) { return a.P - ((o.hv0 + k) & a.p.PS) * SEL_P; };

  for (int i = tid; i < Q * TX::LD; i += SEL_THREADS) l.ek[i] = l.eg[i] = T(0);
  if (tid < SEL_BWD_HEADS * 3) l.sums[tid / 3][tid % 3] = 0.0f;
  if (tid < 4) l.skip[tid] = 0.0f;

  // The states before each chunk: b's and x's tiles in two buffers each (bc, xd), the weights D exp(-what follows) in ic[0], ic[1].
  {
    TB rb;
    TX rx;
    float step = 0.0f;
    auto load = [&](int k, int ci) {
      rb.load(pb + (int64_t)(ci * Q) * sb, sb, rows_at(ci), a.N, here(tid));
      rx.load(px + (int64_t)(ci * Q) * sx + at_of(k), sx, rows_at(ci), cols_of(k), here(tid));
      if (w == (ci & 3)) step = step_at(ci, (o.hv0 + k) >> a.p.PS);
    };
    if (active > 1) load(0, 0);
    int turn = 0;
    for (int k = 0; k < o.heads; ++k) {
      f4 h[NW][4];
      if (mine) {
        if (!several)
#pragma unroll 1
          for (int i = 0; i < NW * 4; ++i) {
            f4 h, g;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int p = 16 * (i & 3) + 4 * lq + r, n = 16 * (w + (i & ~3)) + li;
              h[r] = state_of(a, a.h0, o.b, o.hv0 + k, p, n);
              g[r] = state_of(a, a.dh_out, o.b, o.hv0 + k, p, n);
            }
            hs_at(0, k)[((i & ~3) * 4 + (i & 3)) * 64 + lane] = h;
            gs_at(k, false)[((i & ~3) * 4 + (i & 3)) * 64 + lane] = g;
          }
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v) h[m][v] = hs_at(0, k)[(m * 16 + v) * 64 + lane];
      }
      for (int ci = 0; ci + 1 < active; ++ci) {
        const int lane = here(tid & 63), li = lane & 15, lq = lane >> 4;
        rb.put(l.bc[turn]);
        rx.put(l.xd[turn]);
        if (w == (ci & 3)) {
          const Steps p = steps_of(a, step, lane < rows_at(ci), (o.hv0 + k) >> a.p.PS, lane);
          l.ic[turn][lane] = ((ci & 1) != 0 ? p.d : -p.d) * exp2_fast(-p.after);
          if (lane == 0) l.total[turn] = p.total;
        }
        if (ci + 2 < active)
          load(k, ci + 1);
        else if (k + 1 < o.heads)
          load(k + 1, 0);
        __syncthreads();
        if (mine) {
          const T *b = l.bc[turn], *x = l.xd[turn];
          const float keep = -exp2_fast(-l.total[turn]);  // (the other sign)
#pragma unroll
          for (int m = 0; m < NW; ++m)
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
              for (int r = 0; r < 4; ++r) h[m][v][r] *= keep;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const f4 w0 = load_f4(&l.ic[turn][32 * j + 4 * lq]), w1 = load_f4(&l.ic[turn][32 * j + 16 + 4 * lq]);
            typename M::Frag xf[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) xf[v] = M::col(x + 32 * j * TX::LD + 16 * v, TX::LD, li, lq);
            typename M::Whole bs[NW];
#pragma unroll
            for (int m = 0; m < NW; ++m) {
              const typename M::Frag bf = M::col(b + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
              float bw[8];
#pragma unroll
              for (int r = 0; r < 8; ++r) bw[r] = M::at(bf, r) * (r < 4 ? w0[r & 3] : w1[r & 3]);
              bs[m] = M::whole(bw);
            }
            loads_first();
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
              for (int m = 0; m < NW; ++m) h[m][v] = M::mma(xf[v], bs[m], h[m][v]);
          }
#pragma unroll
          for (int m = 0; m < NW; ++m)
#pragma unroll
            for (int v = 0; v < 4; ++v) hs_at(ci + 1, k)[(m * 16 + v) * 64 + lane] = h[m][v];
        }
        turn ^= 1;
      }
    }
  }

  TB rb, rc;
  TX rx, rd;
  float step = 0.0f;
  f4 g[NW][4], h[NW][4], gn[NW][4];  // a head's, and the next one's
  auto load_g = [&](int ci, int k, int lane) {
    const f4* p = gs_at(k, ci == active - 1);
    if (mine)
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) gn[m][v] = p[(m * 16 + v) * 64 + lane];
  };
  // (a head alone has its gradient only when its chunk is through)
  const bool ahead = o.heads > 1;
  auto steps_wave = [&](int k) { return (k + 2) & 3; };  // which wave makes a head's steps
  auto load_chunk = [&](int ci) {
    rb.load(pb + (int64_t)(ci * Q) * sb, sb, rows_at(ci), a.N, here(tid));
    rc.load(pc + (int64_t)(ci * Q) * sc, sc, rows_at(ci), a.N, here(tid));
  };
  auto load_head = [&](int ci, int k) {
    rx.load(px + (int64_t)(ci * Q) * sx + at_of(k), sx, rows_at(ci), cols_of(k), here(tid));
    rd.load(pd + (int64_t)(ci * Q) * sy + at_of(k), sy, rows_at(ci), cols_of(k), here(tid));
    if (w == steps_wave(k)) step = step_at(ci, (o.hv0 + k) >> a.p.PS);
  };
  if (active > 0) {
    load_chunk(active - 1);
    load_head(active - 1, 0);
    if (ahead) load_g(active - 1, 0, lane);
  }
  for (int ci = active - 1; ci >= 0; --ci) {
    const int64_t t0 = (c0 + ci) * Q;
    const int rows = rows_at(ci), held = held_at(ci);
    // of g in registers and gs, of h there and in hs
    const float sign = ((active - 1 - ci) & 1) != 0 ? -1.0f : 1.0f, hsign = (ci & 1) != 0 ? -1.0f : 1.0f;
    f4 db[NW][4], dc[NW][4], g0[3];
#pragma unroll
    for (int m = 0; m < NW; ++m)
#pragma unroll
      for (int v = 0; v < 4; ++v) db[m][v] = dc[m][v] = f4{0, 0, 0, 0};
    __syncthreads();
    rb.put(bt);
    rc.put(ct);
    if (ci > 0) load_chunk(ci - 1);
    __syncthreads();
    // (c.b)[t][s], by the tiles on and below the diagonal
#pragma unroll
    for (int e = 0; e < 3; ++e) {
      const TileId id = tile_id(w, e);
      typename M::Frag fb[KS], fc[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        fb[k] = M::row(bt + (16 * id.s + li) * TB::LD + 32 * k + 4 * lq);
        fc[k] = M::row(ct + (16 * id.t + li) * TB::LD + 32 * k + 4 * lq);
      }
      loads_first();
      g0[e] = f4{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KS; ++k) g0[e] = M::mma(fc[k], fb[k], g0[e]);
    }
    float ddt = 0.0f;  // a step's, over a head's row blocks (of the wave that has the head)
    for (int k = 0; k < o.heads; ++k) {
      const int hv = o.hv0 + k, hd = (hv >> a.p.PS);
      const int lane = here(tid & 63), li = lane & 15, lq = lane >> 4;
      const int cols = cols_of(k);
      const float skip = a.skip != nullptr ? a.skip[hd] : 0.0f;
      if (!ahead) load_g(ci, k, lane);
#pragma unroll
      for (int m = 0; m < NW; ++m)
#pragma unroll
        for (int v = 0; v < 4; ++v) g[m][v] = gn[m][v];
      if (mine) {
        const f4* p = hs_at(ci, k);
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v) h[m][v] = p[(m * 16 + v) * 64 + lane];
      }
      __syncthreads();  // the last head's readers are through
      rx.put(xt);
      rd.put(dt);
      if (w == steps_wave(k)) {
        const Steps s = steps_of(a, step, lane < rows, hd, lane);
        l.gap.put(s, lane);
        l.d[lane] = s.d;
        l.suf[lane] = sign * exp2_fast(-s.after);
        l.pre[lane] = -sign * exp2_fast(-s.s);
        l.slope[lane] = s.slope;
        if (lane == 0) l.total[0] = s.total;
      }
      if (k + 1 < o.heads)
        load_head(ci, k + 1);
      else if (ci > 0)
        load_head(ci - 1, 0);
      // du = exp(-what follows) g b, this wave's 16 rows p: g's slices through LDS
      f4 du[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) du[v] = f4{0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < NW; ++m) {
        if (m > 0) __syncthreads();
        if (mine)
#pragma unroll
          for (int v = 0; v < 4; ++v) put_quad(&l.gx[(16 * w + li) * TX::LD + 16 * v + 4 * lq], g[m][v]);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < SL / 2; ++j) {
          typename M::Frag bf[4];
          const typename M::Frag gf = M::col(&l.gx[32 * j * TX::LD + 16 * w], TX::LD, li, lq);
#pragma unroll
          for (int v = 0; v < 4; ++v) bf[v] = M::row(bt + (16 * v + li) * TB::LD + 64 * m + 32 * j + 4 * lq);
          loads_first();
#pragma unroll
          for (int v = 0; v < 4; ++v) du[v] = M::mma(gf, bf[v], du[v]);
        }
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float f = l.suf[16 * v + li];
#pragma unroll
        for (int r = 0; r < 4; ++r) du[v][r] *= f;
      }
      // K = dy.x; Z = (c.b) E K; the weights of the products within the chunk
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        const TileId id = tile_id(w, e);
        typename M::Frag fy[2], fx[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          fy[j] = M::row(dt + (16 * id.t + li) * TX::LD + 32 * j + 4 * lq);
          fx[j] = M::row(xt + (16 * id.s + li) * TX::LD + 32 * j + 4 * lq);
        }
        const float from = (id.s == id.t ? l.gap.in : l.gap.behind)[16 * id.s + li] - l.gap.gap(id.s, id.t), d_s = l.d[16 * id.s + li];
        const float from_rest = l.gap.rest[16 * id.s + li];
        const f4 to = load_f4(&l.gap.in[16 * id.t + 4 * lq]), to_rest = load_f4(&l.gap.rest[16 * id.t + 4 * lq]);
        loads_first();
        f4 kk{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) kk = M::mma(fy[j], fx[j], kk);
        f4 ek, eg, z;
        float col = 0.0f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool in = id.s < id.t || li <= 4 * lq + r, below = id.s < id.t || li < 4 * lq + r;
          const float f = exp2_fast((from - to[r]) + (id.s == id.t ? from_rest - to_rest[r] : 0.0f));
          eg[r] = in ? f * g0[e][r] : 0.0f;
          ek[r] = in ? f * kk[r] * d_s : 0.0f;
          col += below ? eg[r] * kk[r] : 0.0f;
          z[r] = below ? ek[r] * g0[e][r] : 0.0f;
        }
        put_quad(l.ek + (16 * id.s + li) * TX::LD + 16 * id.t + 4 * lq, ek);
        put_quad(l.eg + (16 * id.s + li) * TX::LD + 16 * id.t + 4 * lq, eg);
        col = sum_rows(col);
        if (lq == 0) l.colz[id.t][16 * id.s + li] = col;
        if (id.s == id.t) {  // what passes step t within its tile: from s < t to the rows from t on
          z[2] += z[3];
          z[1] += z[2];
          z[0] += z[1];
          const float rows = rows_behind(z[0], lq);
#pragma unroll
          for (int r = 0; r < 4; ++r) z[r] = li < 4 * lq + r ? z[r] + rows : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) z[r] = sum_lanes(z[r]);
        if (li == 0) put_quad(&l.rowz[id.s][16 * id.t + 4 * lq], z);
        if (id.s == id.t) {  // the diagonal: (c.b) dy.x of a step, and dy.x
          float zd = 0.0f, dg = 0.0f;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            dg += li == 4 * lq + r ? kk[r] : 0.0f;
            zd += li == 4 * lq + r ? kk[r] * g0[e][r] : 0.0f;
          }
          zd = sum_rows(zd);
          dg = sum_wave(dg);
          if (lq == 0) l.zd[16 * id.t + li] = zd;
          if (lane == 0) l.skip[id.t] = dg;
        }
      }
      // dc's part from the states, exp(-s_t) h^T dy_t, and with c_t its part of dy.y; db's, D exp(-what follows) g^T x, and with b its part of
      // x.du; <g, h>
      if (mine) {
        auto inter = [&](const f4(&st)[NW][4], const T* act, const T* read, const float* by, float sign, const float* also, f4(&to)[NW][4], float* dots) {
          float dot[4] = {0, 0, 0, 0}, f[4], d[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            f[t] = sign * by[16 * t + li];
            d[t] = also != nullptr ? also[16 * t + li] : 1.0f;
          }
#pragma unroll
          for (int m = 0; m < NW; ++m) {
            f4 acc[4], c[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              acc[t] = f4{0, 0, 0, 0};
              c[t] = quad(read + (16 * t + li) * TB::LD + 16 * (w + 4 * m) + 4 * lq);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              typename M::Frag yf[4];
#pragma unroll
              for (int t = 0; t < 4; ++t) yf[t] = M::row(act + (16 * t + li) * TX::LD + 32 * j + 4 * lq);
              float hf[8];
#pragma unroll
              for (int r = 0; r < 8; ++r) hf[r] = st[m][2 * j + (r >> 2)][r & 3];
              const typename M::Whole hp = M::whole(hf);
              loads_first();
#pragma unroll
              for (int t = 0; t < 4; ++t) acc[t] = M::mma(hp, yf[t], acc[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float v = acc[t][r] * f[t];
                dot[t] = fmaf(c[t][r], v, dot[t]);
                to[m][t][r] = fmaf(d[t], v, to[m][t][r]);
              }
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) dot[t] = sum_rows(dot[t]);
          dots[lane] = lq == 0 ? dot[0] : lq == 1 ? dot[1] : lq == 2 ? dot[2] : dot[3];
        };
        inter(h, dt, ct, l.pre, -sign * hsign, nullptr, dc, l.ic[w]);
        inter(g, xt, bt, l.suf, 1.0f, l.d, db, l.ig[w]);
        float dot = 0.0f;
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) dot = fmaf(g[m][v][r], h[m][v][r], dot);
        dot = sum_wave(dot);
        if (lane == 0) l.lam[w] = dot;
      } else {
        l.ic[w][lane] = l.ig[w][lane] = 0.0f;
        if (lane == 0) l.lam[w] = 0.0f;
      }
      __syncthreads();
      if (ahead) {
        if (k + 1 < o.heads)
          load_g(ci, k + 1, lane);
        else if (ci > 0)
          load_g(ci - 1, 0, lane);
      }
      if (w == ((k >> a.p.PS) & 3)) {  // dl, dD and the parameters' sums; one step a lane
        const int tile = lane >> 4;
        float rz[4], cz[4], ic[4], ig[4], lam = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          rz[v] = l.rowz[v][lane];
          cz[v] = l.colz[v][lane];
          ic[v] = l.ic[v][lane];
          ig[v] = l.ig[v][lane];
          lam += l.lam[v];
        }
        const float d = l.d[lane], slope = l.slope[lane], zd = l.zd[lane], gamma = a.gamma[hd];
        lam *= sign * hsign * exp2_fast(-l.total[0]);
        loads_first();
        // What passes step t, from the steps before it and the state to those from it on and the gradient behind the chunk, as a sum of
        // only that: whole tiles beyond t's, rows and columns of its tile with those, and the tile's own.  (Sums of all that leaves and
        // all that arrives up to t are the same less what cancels; it left errors up to 2e-5 of dgamma and of dt_bias's gradient.)
        float after = 0.0f, before = 0.0f, row = 0.0f, col = 0.0f, own = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          after += ic[v];
          before += ig[v];
          row += v < tile ? rz[v] : 0.0f;
          col += v > tile ? cz[v] : 0.0f;
          own = v == tile ? rz[v] : own;
        }
        float cu = before + zd;
#pragma unroll
        for (int v = 0; v < 4; ++v) cu += v >= tile ? cz[v] : 0.0f;
        before *= d;
        const float arrive = suffix_lanes(after), leave = sum_lanes(before), z0 = sum_lanes(rz[0]), z1 = sum_lanes(rz[1]);
        const float sent = prefix_lanes(
            __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, fmaf(d, col, before)), 0x111, 0xF, 0xF, true)));
        float dl = lam + own + (arrive + suffix_lanes(row)) + sent;
        // (read in all lanes: in a branch the sums would be those of the branch's lanes)
        const float z20 = of_lane(z0, 32), z30 = of_lane(z0, 48), z31 = of_lane(z1, 48);
        dl += tile == 1 ? z20 + z30 : tile == 2 ? z30 + z31 : 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float a0 = of_lane(leave, 16 * v), a1 = of_lane(arrive, 16 * v);
          dl += v < tile ? a0 : v > tile ? a1 : 0.0f;
        }
        const float v = (cu - gamma * dl) * slope;
        const float sg = sum_wave(-d * dl), sb = sum_wave(v);
        if (lane == 0) {
          l.sums[k][0] += sg;
          l.sums[k][1] += sb;
          l.sums[k][2] += l.skip[0] + l.skip[1] + l.skip[2] + l.skip[3];
        }
        ddt = (hv & a.p.PS) == 0 ? v : ddt + v;
        if ((hv & a.p.PS) == a.p.PS && lane < held)
          static_cast<T*>(a.ddt.p)[o.b * a.ddt.sb + (t0 + lane) * a.ddt.st + hd] = from_f32<T>(lane < rows ? ddt : 0.0f);
      }
      // within the chunk: dc, db, du (6 fragments of 32 steps: of tiles 0, 1 one, of the others two; the other way round for s)
      if (mine) {
        typename M::Frag ef[6];
#pragma unroll
        for (int i = 0; i < 6; ++i) ef[i] = M::col(l.ek + 32 * (i < 2 ? 0 : i & 1) * TX::LD + 16 * (i < 2 ? i : (i + 2) / 2), TX::LD, li, lq);
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          typename M::Frag bf[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) bf[j] = M::col(bt + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
          loads_first();
#pragma unroll
          for (int i = 0; i < 6; ++i) dc[m][i < 2 ? i : (i + 2) / 2] = M::mma(bf[i < 2 ? 0 : i & 1], ef[i], dc[m][i < 2 ? i : (i + 2) / 2]);
        }
#pragma unroll
        for (int i = 0; i < 6; ++i) ef[i] = M::row(l.ek + (16 * (i < 4 ? i / 2 : i - 2) + li) * TX::LD + 32 * (i < 4 ? i & 1 : 1) + 4 * lq);
#pragma unroll
        for (int m = 0; m < NW; ++m) {
          typename M::Frag cf[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) cf[j] = M::col(ct + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
          loads_first();
#pragma unroll
          for (int i = 0; i < 6; ++i) db[m][i < 4 ? i / 2 : i - 2] = M::mma(cf[i < 4 ? i & 1 : 1], ef[i], db[m][i < 4 ? i / 2 : i - 2]);
        }
      }
      {
        typename M::Frag ef[6], yf[2];
#pragma unroll
        for (int i = 0; i < 6; ++i) ef[i] = M::row(l.eg + (16 * (i < 4 ? i / 2 : i - 2) + li) * TX::LD + 32 * (i < 4 ? i & 1 : 1) + 4 * lq);
#pragma unroll
        for (int j = 0; j < 2; ++j) yf[j] = M::col(dt + 32 * j * TX::LD + 16 * w, TX::LD, li, lq);
        f4 y[4];
        float d[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          y[v] = quad(dt + (16 * v + li) * TX::LD + 16 * w + 4 * lq);
          d[v] = l.d[16 * v + li];
        }
        loads_first();
#pragma unroll
        for (int i = 0; i < 6; ++i) du[i < 4 ? i / 2 : i - 2] = M::mma(yf[i < 4 ? i & 1 : 1], ef[i], du[i < 4 ? i / 2 : i - 2]);
        T* pdx = static_cast<T*>(a.dx.p) + o.b * a.dx.sb + t0 * a.dx.st + at_of(k) + 16 * w;
        const uint32_t sdx = (uint32_t)a.dx.st;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int row = 16 * v + li;
#pragma unroll
          for (int r = 0; r < 4; ++r) du[v][r] = row < rows ? fmaf(skip, y[v][r], d[v] * du[v][r]) : 0.0f;
          if (row < held) store_quad<WHOLE>(pdx + ((uint32_t)row * sdx + 4 * lq), cols - 16 * w - 4 * lq, du[v]);
        }
      }
      if (mine) {
        // g before the chunk, with the other sign
        const float keep = -exp2_fast(-l.total[0]);
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) g[m][v][r] *= keep;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f4 w0 = load_f4(&l.pre[32 * j + 4 * lq]), w1 = load_f4(&l.pre[32 * j + 16 + 4 * lq]);
          typename M::Frag yf[4];
#pragma unroll
          for (int v = 0; v < 4; ++v) yf[v] = M::col(dt + 32 * j * TX::LD + 16 * v, TX::LD, li, lq);
          typename M::Whole cs[NW];
#pragma unroll
          for (int m = 0; m < NW; ++m) {
            const typename M::Frag cf = M::col(ct + 32 * j * TB::LD + 16 * (w + 4 * m), TB::LD, li, lq);
            float cw[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) cw[r] = M::at(cf, r) * (r < 4 ? w0[r & 3] : w1[r & 3]);
            cs[m] = M::whole(cw);
          }
          loads_first();
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int m = 0; m < NW; ++m) g[m][v] = M::mma(yf[v], cs[m], g[m][v]);
        }
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (ci > 0)
              gs[k * STATE + (m * 16 + v) * 64 + lane] = g[m][v];
            else if (!several)
              gs[k * STATE + (m * 16 + v) * 64 + lane] = -sign * g[m][v];
      }
    }
    if (mine) {
      auto put = [&](auto* pb, auto* pc, uint32_t sb, uint32_t sc) {
#pragma unroll
        for (int m = 0; m < NW; ++m)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const int row = 16 * v + li, c = 16 * (w + 4 * m) + 4 * lq;
            if (row >= held) continue;
            if (row >= rows) db[m][v] = dc[m][v] = f4{0, 0, 0, 0};
            store_quad<WHOLE>(pb + ((uint32_t)row * sb + (uint32_t)c), a.N - c, db[m][v]);
            store_quad<WHOLE>(pc + ((uint32_t)row * sc + (uint32_t)c), a.N - c, dc[m][v]);
          }
      };
      if (a.part != nullptr) {
        const uint32_t gn = (uint32_t)(a.G * a.N);
        float* p = a.part + (((int64_t)o.block * 2 * a.B + o.b) * a.L + t0) * gn + o.g * a.N;
        put(p, p + a.B * a.L * gn, gn, gn);
      } else {
        put(static_cast<T*>(a.db.p) + o.b * a.db.sb + t0 * a.db.st + o.g * a.N, static_cast<T*>(a.dc.p) + o.b * a.dc.sb + t0 * a.dc.st + o.g * a.N,
            (uint32_t)a.db.st, (uint32_t)a.dc.st);
      }
    }
  }
  // behind the row's end
  for (int ci = active; ci < all; ++ci) {
    const int64_t t0 = (c0 + ci) * Q, gn = (int64_t)a.G * a.N;
    const int held = held_at(ci);
    for (int k = 0; k < o.heads; ++k) {
      const int cols = cols_of(k), hv = o.hv0 + k;
      T* pdx = static_cast<T*>(a.dx.p) + o.b * a.dx.sb + t0 * a.dx.st + at_of(k);
      for (int i = tid; i < held * SEL_P; i += SEL_THREADS)
        if (i % SEL_P < cols) pdx[(int64_t)(i / SEL_P) * a.dx.st + i % SEL_P] = T(0);
      if ((hv & a.p.PS) == 0 && tid < held) static_cast<T*>(a.ddt.p)[o.b * a.ddt.sb + (t0 + tid) * a.ddt.st + (hv >> a.p.PS)] = T(0);
    }
    for (int i = tid; i < held * a.N; i += SEL_THREADS) {
      const int64_t t = t0 + i / a.N, c = (int64_t)o.g * a.N + i % a.N;
      if (a.part != nullptr) {
        float* p = a.part + (((int64_t)o.block * 2 * a.B + o.b) * a.L + t) * gn + c;
        p[0] = p[a.B * a.L * gn] = 0.0f;
      } else {
        static_cast<T*>(a.db.p)[o.b * a.db.sb + t * a.db.st + c] = T(0);
        static_cast<T*>(a.dc.p)[o.b * a.dc.sb + t * a.dc.st + c] = T(0);
      }
    }
  }
  if (mine && !several && a.dh0 != nullptr)
    for (int k = 0; k < o.heads; ++k) {
      const int hv = o.hv0 + k, p0 = (hv & a.p.PS) * SEL_P;
      float* s = a.dh0 + ((o.b * a.H + (hv >> a.p.PS)) * (int64_t)a.P + p0) * a.N;
#pragma unroll 1
      for (int i = 0; i < NW * 4; ++i) {
        const f4 g = gs[k * STATE + ((i & ~3) * 4 + (i & 3)) * 64 + lane];
        const int c = 16 * (w + (i & ~3)) + li, p = 16 * (i & 3) + 4 * lq;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (c < a.N && p0 + p + r < a.P) s[(p + r) * a.N + c] = g[r];
      }
    }
  __syncthreads();
  if (tid < o.heads * 3) a.params[((o.b * a.p.segs + o.seg) * a.p.HV + o.hv0) * 3 + tid] = l.sums[tid / 3][tid % 3];
}

// db and dc of a group from its blocks of heads, in their order: 4 elements of a step a thread.  Two blocks of 65536 steps with 64
// states: 21 us (84 MB).
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
  store_quad<false>(static_cast<T*>(o.p) + b * o.sb + t * o.st + c, nc, s);
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
// One step: a group of LN lanes takes a row p of a state, 4 states a lane.  The states are read and written once; that bounds it
// (64 sequences of 8 heads of 64 x 64: 17 MB in 7.2 us, 2 of them a launch's).
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
template <typename T>
bool whole(const SelArgs& a) {
  constexpr int V = 16 / (int)sizeof(T);
  return a.P % V == 0 && a.N % V == 0;
}
template <typename T, int NT, bool STATES, bool REV>
hipError_t forward(SelArgs a, hipStream_t st) {
  constexpr int HF = NT > 4 ? 2 : 4;
  const int64_t wgs = a.B * a.p.segs * a.G * ((a.p.HG + HF - 1) / HF);
  return over(a, wgs, [&](uint32_t grid) {
    if (whole<T>(a))
      selective_fwd_kernel<T, NT, HF, true, STATES, REV><<<grid, SEL_THREADS, 0, st>>>(a);
    else
      selective_fwd_kernel<T, NT, HF, false, STATES, REV><<<grid, SEL_THREADS, 0, st>>>(a);
  });
}
template <typename T, int NT, bool WHOLE>
hipError_t backward(SelArgs a, hipStream_t st) {
  constexpr int lds = (int)sizeof(BwdLds<T, NT, WHOLE>);
  static_assert(lds <= 163840, "a compute unit's LDS");
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(selective_bwd_kernel<T, NT, WHOLE>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  const int64_t wgs = a.B * a.p.segs * a.G * ((a.p.HG + a.p.HR - 1) / a.p.HR);
  return over(a, wgs, [&](uint32_t grid) { selective_bwd_kernel<T, NT, WHOLE><<<grid, SEL_THREADS, lds, st>>>(a); });
}
template <bool REV>
hipError_t join(SelArgs a, hipStream_t st) {
  // (a launch begins with a whole row block)
  const int64_t per = SEL_P * 16 * a.p.NT, all = a.B * a.p.HV, most = LAUNCH_THREADS / per;
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
  p.PS = p.PB - 1;
  p.HV = (int)(H * p.PB);
  p.HG = (int)(H / G * p.PB);
  p.HF = p.NT > 4 ? 2 : 4;
  // (HF and HR are by one size, a large call's; fewer were not measured where work-groups are fewer than CUs.)
  // Row blocks of a group that a backward work-group has: more sum more of db and dc in registers and read b and c less often, fewer
  // keep more work-groups (8 x 8192, 8 heads of 64 x 64, bf16, a training step: 2, 4 and 8 took 521, 487 and 577 us).
  // The workspace counts the states of as many.
  p.HR = p.HG < SEL_BWD_HEADS ? p.HG : SEL_BWD_HEADS;
  p.chunks = (L + SEL_Q - 1) / SEL_Q;
  // segments: work-groups of the forward for two on each CU; a chunk at least.  (Half of that, it, twice that: the training step above
  // 656, 487 and 525 us, a forward of 4 x 32768 with 128 states 431, 295 and 330.  One row of 777 steps, 32 heads of 64 x 128: at
  // least one chunk 36 us, at least two 56.)
  const int64_t rows = B * G * ((p.HG + p.HF - 1) / p.HF);
  int64_t segs = (512 + rows - 1) / rows;
  segs = segs > p.chunks ? p.chunks : segs;
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
    return whole<T>(a) ? backward<T, nt, true>(a, st) : backward<T, nt, false>(a, st);
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
