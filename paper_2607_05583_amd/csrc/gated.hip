// Gated scan: a diagonal recurrence whose damping depends on the data, per channel
//   s = gamma sigmoid(r_t), a = exp(-s), beta = sqrt(1 - a^2), q = sigmoid(i_t)
//   h_t = a h_{t-1} + beta q x_t,   y_t = h_t
// and its gradients.  With g_t the gradient of h_t (g_t = dy_t + a_{t+1} g_{t+1}),
//   dx = g beta q,   di = g beta q (1 - q) x,   w = g (a^2 / beta q x - a h_{t-1}),
//   dr = w s (1 - sigmoid(r)),   dgamma = sum w sigmoid(r),   dh0 = a_0 g_0.
// Where s = 0 (beta = 0) the derivative of beta is taken as zero.
//
// Both directions are scans of affine maps: steps t0..t1 take h to A h + H with A the
// product of their a, and the adjoint c_t = a_t g_t to A c + C with the same A.
//
// A work-group takes a tile of a chain (one batch row, 64 channels: 128-byte rows of
// bf16) and holds it in registers: a thread has S consecutive steps of VEC channels and
// composes their map; the maps of the threads before it come from a scan over the wave
// and over the waves' totals (LDS).  Inputs are read once and outputs written once.
//
// The state before a tile comes from the tiles before it in one pass: a tile publishes
// its map as soon as it has it, and its end state as soon as it has that; a tile looks
// back over at most WINDOW tiles for the nearest end state and applies the maps from
// there on, one after the other.  That is the same sequence of operations wherever the
// search ends, so results do not depend on timing.  Tiles are taken in order from a
// ticket counter, so the tiles that one waits for are always at work (one work-group a
// tile: a loop over tiles took 60 registers more).  A published value is a 64-bit word with
// the call's number beside it: a word is its own flag, and nothing has to be cleared
// between calls.  A call of more than 2^32 threads is several launches of whole batch rows.
//
// A step of a channel is 8 bytes forward and 14 backward in bf16, and 36 and 94 vector
// instructions of a wave, six and ten of them transcendental.
//   forward   4 x 32768 x 256 bf16 in 75 us (3.6 TB/s): the bytes are 56 us of a large
//             copy's rate, the instructions 30; 8 x 8192 x 256 44 us (3.1 TB/s)
//   backward  8 x 8192 x 256 bf16 in 72 us (3.3 TB/s): 49 and 40
// The two overlap only in part: a tile loads before it computes, and the registers that it
// is held in leave two tiles of 512 threads on a unit to fill the gap.
#include "layer.h"

namespace res {
namespace {

// The gate's exponent is kept as z = s log2(e), so that a = 2^-z.
// 1 - a^2 = 1 - 4^-z without the cancellation for small z: the series up to z^5 below z = 0.108 (2 s = 0.15; relative
// error 1e-7 there, and 4e-7 above).
__device__ __forceinline__ float one_minus_a2(float z, float a) {
  constexpr double L = 2.0 * 0.69314718055994530942;  // ln 4
  float p = fmaf(z, (float)(L * L * L * L * L / 120), (float)(-L * L * L * L / 24));
  p = fmaf(z, p, (float)(L * L * L / 6));
  p = fmaf(z, p, (float)(-L * L / 2));
  p = fmaf(z, p, (float)L);
  return z < 0.108f ? z * p : fmaf(-a, a, 1.0f);
}
__device__ __forceinline__ float beta_of(float z, float a) { return __builtin_amdgcn_sqrtf(one_minus_a2(z, a)); }

template <typename T, int VEC> struct __align__(sizeof(T) * VEC) Vec { T v[VEC]; };

// Makes the compiler take the values for new ones.
template <typename T, int VEC, int S>
__device__ __forceinline__ void opaque(Vec<T, VEC> (&x)[S]) {
  typedef uint32_t u __attribute__((ext_vector_type(VEC * sizeof(T) > 4 ? VEC * sizeof(T) / 4 : 2)));
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if constexpr (VEC * sizeof(T) == 2) {
      asm volatile("" : "+v"(x[s].v[0]));
    } else if constexpr (VEC * sizeof(T) == 4) {
      uint32_t w = __builtin_bit_cast(uint32_t, x[s]);
      asm volatile("" : "+v"(w));
      x[s] = __builtin_bit_cast(Vec<T, VEC>, w);
    } else {
      u w = __builtin_bit_cast(u, x[s]);
      asm volatile("" : "+v"(w));
      x[s] = __builtin_bit_cast(Vec<T, VEC>, w);
    }
  }
}

// A thread's rows of a tile: the tile's first element (the same for all threads) and this thread's bytes from there.
struct Walk {
  const char* base;
  int64_t st;    // bytes of a step
  uint32_t off;  // this thread's first step, its channel
};
template <typename T>
__device__ __forceinline__ Walk walk(const void* p, int64_t sb, int64_t st, int64_t b, int64_t t0, int mine, int c) {
  return Walk{(const char*)((const T*)p + b * sb + t0 * st), st * (int64_t)sizeof(T), (uint32_t)((mine * st + c) * (int64_t)sizeof(T))};
}
// step s of this thread's, or (clamped) the step `most` of the tile where that comes first
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_row(const Walk& w, int s) {
  return *reinterpret_cast<const Vec<T, VEC>*>(w.base + s * w.st + w.off);
}
template <typename T, int VEC>
__device__ __forceinline__ Vec<T, VEC> load_row_clamped(const Walk& w, int s, int mine, int most) {
  const int back = mine + s > most ? mine + s - most : 0;  // steps past it
  return *reinterpret_cast<const Vec<T, VEC>*>(w.base + s * w.st + w.off - back * w.st);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_row(const Walk& w, int s, const Vec<T, VEC>& o) {
  typedef uint16_t u1 __attribute__((ext_vector_type(VEC * sizeof(T) / 2)));
  __builtin_nontemporal_store(__builtin_bit_cast(u1, o), reinterpret_cast<u1*>(const_cast<char*>(w.base) + s * w.st + w.off));
}

__device__ __forceinline__ int row_len(const int* lengths, int64_t b, int64_t L) {
  if (lengths == nullptr) return (int)L;
  const int n = lengths[b];
  return n < 0 ? 0 : n < (int)L ? n : (int)L;
}

// ---------------------------------------------------------------------------
// Tiles in order, and the look-back
// ---------------------------------------------------------------------------
// Tiles looked back over at a time.  More carry a state over long chains in fewer looks, fewer poll less: forward and backward
// of 1 x 32768 x 64 bf16 95 us with 8, 133 with 4; of 8 x 8192 x 256 123 with 8, 122 with 4, 139 with 16.
constexpr int WINDOW = 8;
constexpr int NONE = -2, END = -1;  // kinds of a published map, in the place of its A (which is never negative)

__device__ __forceinline__ uint64_t word(float v, uint32_t tag) { return (uint64_t)tag << 32 | __float_as_uint(v); }
__device__ __forceinline__ uint64_t load_word(const uint64_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_word(uint64_t* p, float v, uint32_t tag) {
  __hip_atomic_store(p, word(v, tag), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct LookShared {
  float2 map[WINDOW][GATED_CW];
  float enter[GATED_CW];
  int ticket, found;
};

// The value that enters tile `o` > 0 of a chain (in the order that they are taken; `words`: the chain's) into sh.enter, for
// the 64 channels.  Called by the whole work-group.
// What enters tile 0 is read by tile 0 alone and reaches the others in its end value: the chain's last tile stores its own
// end, which may go where the initial state came from (h_out = h0), and every tile waits for tile 0's end before it has one.
__device__ __forceinline__ void look_back(const uint64_t* words, int64_t o, uint32_t tag, uint32_t* status, LookShared& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = wave;  // this wave's tile, counted back
  for (int tries = 0;; ++tries) {
    if (g < WINDOW) {
      float2 m = make_float2(NONE, 0.0f);
      if (g < o) {
        const uint64_t* w = words + (o - 1 - g) * GATED_TILE_WORDS + lane;
        const uint64_t e = load_word(w + 128), a = load_word(w), h = load_word(w + 64);
        if ((uint32_t)(e >> 32) == tag)
          m = make_float2(END, __uint_as_float((uint32_t)e));
        else if ((uint32_t)(a >> 32) == tag && (uint32_t)(h >> 32) == tag)
          m = make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)h));
      }
      sh.map[g][lane] = m;
    }
    __syncthreads();
    if (wave == 0) {
      float v = 0.0f;
      bool have = false;
#pragma unroll
      for (int g = WINDOW - 1; g >= 0; --g) {
        const float2 m = sh.map[g][lane];
        if (m.x == END) {
          v = m.y;
          have = true;
        } else if (m.x == NONE) {
          have = false;
        } else {
          v = fmaf(m.x, v, m.y);
        }
      }
      if (tries > (1 << 20)) {  // (seconds: a work-group before it is gone; the result says so)
        if (lane == 0) *status = 1;
        v = __uint_as_float(0x7fc00000u);
        have = true;
      }
      sh.enter[lane] = v;
      if (lane == 0) sh.found = 0;
      if (__all(have) && lane == 0) sh.found = 1;
    }
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(sh.found)) return;
    __builtin_amdgcn_s_sleep(2);
  }
}

// This work-group's tile (whole work-group).
__device__ __forceinline__ uint32_t take_ticket(uint32_t* hdr, LookShared& sh) {
  if (threadIdx.x == 0) sh.ticket = (int)atomicAdd(hdr + 2, 1u);
  __syncthreads();
  const uint32_t t = (uint32_t)__builtin_amdgcn_readfirstlane(sh.ticket);
  __syncthreads();
  return t;
}
// The last work-group to end makes the counters ready for the next call.
__device__ __forceinline__ void leave(uint32_t* hdr, uint32_t tag) {
  if (threadIdx.x == 0 && atomicAdd(hdr + 3, 1u) == gridDim.x - 1) {
    hdr[2] = 0;
    hdr[3] = 0;
    hdr[1] = tag;
  }
}

// Maps of the threads of a wave that have the same channels (lane groups of CGL, in time order).
template <int CGL>
__device__ __forceinline__ void scan_up(float& A, float& H) {  // inclusive: all up to and with this one
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = CGL; d < 64; d <<= 1) {
    const float pa = __shfl_up(A, d, 64), ph = __shfl_up(H, d, 64);
    if (lane >= d) {
      H = fmaf(A, ph, H);
      A *= pa;
    }
  }
}
template <int CGL>
__device__ __forceinline__ void scan_down(float& A, float& C) {  // inclusive: this one and all after it
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = CGL; d < 64; d <<= 1) {
    const float pa = __shfl_down(A, d, 64), pc = __shfl_down(C, d, 64);
    if (lane + d < 64) {
      C = fmaf(A, pc, C);
      A *= pa;
    }
  }
}

template <typename T, int VEC, int S, int NT, bool LOOK>
__global__ __launch_bounds__(NT, 4) void gated_fwd_kernel(GatedArgs A) {
  constexpr int CGL = GATED_CW / VEC, TG = NT / CGL, TILE = S * TG, NW = NT / 64, WG = 64 / CGL;
  __shared__ float2 total[NW][GATED_CW];
  __shared__ LookShared sh;
  const int wl = threadIdx.x & 63, wave = threadIdx.x >> 6, lane = wl % CGL, tg = threadIdx.x / CGL, cl = lane * VEC;
  const int64_t tiles = gated_tiles(A.L, TILE), chains = A.B * A.NB, NC = (A.L + GATED_CARRY - 1) / GATED_CARRY;
  const uint32_t tag = LOOK ? A.hdr[1] + 1 : 0;
  int64_t o = 0, chain = blockIdx.x;
  if constexpr (LOOK) {
    const uint32_t t = take_ticket(A.hdr, sh);
    o = t / (uint32_t)chains;
    chain = t - (uint32_t)o * (uint32_t)chains;
  }
  const int64_t b = (uint32_t)chain / (uint32_t)A.NB;
  const int cb = (int)(chain - b * A.NB) * GATED_CW, c = cb + cl, cs = c < A.D ? c : 0;
  const int len = row_len(A.lengths, b, A.L);
  // steps of the tile: this thread's first, those before the row's end, those before the tensor's
  const int64_t tt = o * TILE;
  const int mine = tg * S, valid = (int)((len < tt ? 0 : len - tt) < TILE ? (len < tt ? 0 : len - tt) : TILE),
            there = (int)(A.L - tt < TILE ? A.L - tt : TILE);
  float a[S][VEC], u[S][VEC];
  {
    // All loads first and without branches: steps behind the row's end load its last one again, channels behind the
    // last one the first, and what they give is not used.
    Vec<T, VEC> x[S], r[S], i[S];
    const Walk wx = walk<T>(A.x.p, A.x.sb, A.x.st, b, tt, mine, cs), wr = walk<T>(A.r.p, A.r.sb, A.r.st, b, tt, mine, cs),
               wi = walk<T>(A.i.p, A.i.sb, A.i.st, b, tt, mine, cs);
    if (valid == TILE) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        r[s] = load_row<T, VEC>(wr, s);
        i[s] = load_row<T, VEC>(wi, s);
        x[s] = load_row<T, VEC>(wx, s);
      }
    } else if (there > 0) {
      const int most = valid > 0 ? valid - 1 : 0;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        r[s] = load_row_clamped<T, VEC>(wr, s, mine, most);
        i[s] = load_row_clamped<T, VEC>(wi, s, mine, most);
        x[s] = load_row_clamped<T, VEC>(wx, s, mine, most);
      }
    }
    float gam[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) gam[v] = LOG2E * A.gamma[cs + v];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float z = gam[v] * sigmoid_fast(to_f32(r[s].v[v]));
        a[s][v] = exp2_fast(-z);
        u[s][v] = beta_of(z, a[s][v]) * sigmoid_fast(to_f32(i[s].v[v])) * to_f32(x[s].v[v]);
      }
    if (valid < TILE) {  // behind the end the state is kept
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          a[s][v] = mine + s < valid ? a[s][v] : 1.0f;
          u[s][v] = mine + s < valid ? u[s][v] : 0.0f;
        }
    }
  }
  float ea[VEC], eh[VEC];  // the map of this wave's steps before this thread's
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    float pa = 1.0f, ph = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      pa *= a[s][v];
      ph = fmaf(a[s][v], ph, u[s][v]);
    }
    scan_up<CGL>(pa, ph);
    if (wl >= 64 - CGL) total[wave][cl + v] = make_float2(pa, ph);
    ea[v] = 1.0f;
    eh[v] = 0.0f;
    if constexpr (WG > 1) {
      const float xa = __shfl_up(pa, CGL, 64), xh = __shfl_up(ph, CGL, 64);
      if (wl >= CGL) ea[v] = xa, eh[v] = xh;
    }
  }
  __syncthreads();
  float ta = 1.0f, th = 0.0f;  // the tile's map (wave 0: a channel a lane)
  uint64_t* words = A.words + (size_t)chain * tiles * GATED_TILE_WORDS;
  const int cw = cb + wl;
  const float init = o == 0 && wave == 0 && A.h0 != nullptr && cw < A.D ? A.h0[b * A.D + cw] : 0.0f;
  if (wave == 0) {
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float2 m = total[w][wl];
      th = fmaf(m.x, th, m.y);
      ta *= m.x;
    }
    if (LOOK && o + 1 < tiles) {
      uint64_t* w = words + o * GATED_TILE_WORDS + wl;
      store_word(w, ta, tag);
      store_word(w + 64, th, tag);
    }
  }
  if (LOOK && o > 0) {
    look_back(words, o, tag, A.hdr, sh);
  } else {
    if (wave == 0) sh.enter[wl] = init;
    __syncthreads();
  }
  if (wave == 0) {
    const float end = fmaf(ta, sh.enter[wl], th);
    if (LOOK && o + 1 < tiles) store_word(words + o * GATED_TILE_WORDS + 128 + wl, end, tag);
    if (A.h_out != nullptr && o + 1 == tiles && cw < A.D) A.h_out[b * A.D + cw] = end;
  }
  float h[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = sh.enter[cl + v];
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float2 m = total[w][cl + v];
      h[v] = fmaf(m.x, h[v], m.y);
    }
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = fmaf(ea[v], h[v], eh[v]);
  if (A.carry != nullptr && mine % GATED_CARRY == 0 && mine < there && c < A.D) {
    float* to = A.carry + (b * NC + (tt + mine) / GATED_CARRY) * A.D + c;
#pragma unroll
    for (int v = 0; v < VEC; ++v) to[v] = h[v];
  }
  if (A.y != nullptr && c < A.D) {
    const Walk wy = walk<T>(A.y, A.L * A.D, A.D, b, tt, mine, c);
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = a[s][v] = fmaf(a[s][v], h[v], u[s][v]);
    if (valid < TILE) {
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int v = 0; v < VEC; ++v) a[s][v] = mine + s < valid ? a[s][v] : 0.0f;
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
      Vec<T, VEC> ov;
#pragma unroll
      for (int v = 0; v < VEC; ++v) ov.v[v] = from_f32<T>(a[s][v]);
      if (there == TILE || mine + s < there) store_row<T, VEC>(wy, s, ov);
    }
  }
  if constexpr (LOOK) leave(A.hdr, tag);
}

// Tiles from the last to the first; one starts at a kept state, so only the adjoint is looked back for.
template <typename T, int VEC, int S, int NT, bool LOOK>
__global__ __launch_bounds__(NT, sizeof(T) == 2 ? 4 : 2) void gated_bwd_kernel(GatedArgs A) {
  constexpr int CGL = GATED_CW / VEC, TG = NT / CGL, TILE = S * TG, NW = NT / 64, WG = 64 / CGL;
  static_assert(TILE % GATED_CARRY == 0, "a tile starts at a kept state");
  __shared__ float total[3][NW][GATED_CW];  // A, H, C of a wave's steps
  __shared__ float sums[NW][GATED_CW];
  __shared__ LookShared sh;
  const int wl = threadIdx.x & 63, wave = threadIdx.x >> 6, lane = wl % CGL, tg = threadIdx.x / CGL, cl = lane * VEC;
  const int64_t tiles = gated_tiles(A.L, TILE), chains = A.B * A.NB, NC = (A.L + GATED_CARRY - 1) / GATED_CARRY;
  const uint32_t tag = LOOK ? A.hdr[1] + 1 : 0;
  int64_t o = 0, chain = blockIdx.x;
  if constexpr (LOOK) {
    const uint32_t t = take_ticket(A.hdr, sh);
    o = t / (uint32_t)chains;
    chain = t - (uint32_t)o * (uint32_t)chains;
  }
  const int64_t tile = tiles - 1 - o, b = (uint32_t)chain / (uint32_t)A.NB;
  const int cb = (int)(chain - b * A.NB) * GATED_CW, c = cb + cl, cs = c < A.D ? c : 0;
  const int len = row_len(A.lengths, b, A.L);
  const int64_t tt = tile * TILE;
  const int mine = tg * S, valid = (int)((len < tt ? 0 : len - tt) < TILE ? (len < tt ? 0 : len - tt) : TILE),
            there = (int)(A.L - tt < TILE ? A.L - tt : TILE);
  float gam[VEC];
  Vec<T, VEC> x[S], d[S], i[S];
  float a[S][VEC], sr[S][VEC];
  float h[VEC];  // the state before the tile
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = 0.0f;
  {
    Vec<T, VEC> r[S];
    const Walk wx = walk<T>(A.x.p, A.x.sb, A.x.st, b, tt, mine, cs), wr = walk<T>(A.r.p, A.r.sb, A.r.st, b, tt, mine, cs),
               wi = walk<T>(A.i.p, A.i.sb, A.i.st, b, tt, mine, cs), wd = walk<T>(A.dy.p, A.dy.sb, A.dy.st, b, tt, mine, cs);
    if (valid == TILE) {
#pragma unroll
      for (int s = 0; s < S; ++s) {
        r[s] = load_row<T, VEC>(wr, s);
        i[s] = load_row<T, VEC>(wi, s);
        x[s] = load_row<T, VEC>(wx, s);
        d[s] = load_row<T, VEC>(wd, s);
      }
    } else if (there > 0) {
      const int most = valid > 0 ? valid - 1 : 0;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        r[s] = load_row_clamped<T, VEC>(wr, s, mine, most);
        i[s] = load_row_clamped<T, VEC>(wi, s, mine, most);
        x[s] = load_row_clamped<T, VEC>(wx, s, mine, most);
        d[s] = load_row_clamped<T, VEC>(wd, s, mine, most);
      }
    }
    if (there > 0) {
      const float* from = A.carry + (b * NC + tile * (TILE / GATED_CARRY)) * A.D + cs;
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = from[v];
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) gam[v] = LOG2E * A.gamma[cs + v];
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        sr[s][v] = sigmoid_fast(to_f32(r[s].v[v]));
        a[s][v] = exp2_fast(-gam[v] * sr[s][v]);
      }
    if (valid < TILE) {  // behind the end s = 0: a = 1 and nothing is added
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const bool in = mine + s < valid;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          a[s][v] = in ? a[s][v] : 1.0f;
          sr[s][v] = in ? sr[s][v] : 0.0f;
          i[s].v[v] = in ? i[s].v[v] : T(0);
          x[s].v[v] = in ? x[s].v[v] : T(0);
          d[s].v[v] = in ? d[s].v[v] : T(0);
        }
      }
    }
  }
  float hp[S][VEC];        // beta q x, then the state before the step
  float ea[VEC], eh[VEC];  // maps of this wave's steps before this thread's
  float fa[VEC], fc[VEC];  // and, for the adjoint, after them
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    float pa = 1.0f, ph = 0.0f, pc = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      hp[s][v] = beta_of(gam[v] * sr[s][v], a[s][v]) * sigmoid_fast(to_f32(i[s].v[v])) * to_f32(x[s].v[v]);
      pa *= a[s][v];
      ph = fmaf(a[s][v], ph, hp[s][v]);
    }
#pragma unroll
    for (int s = S - 1; s >= 0; --s) pc = a[s][v] * (to_f32(d[s].v[v]) + pc);
    float da = pa, dc = pc;
    scan_up<CGL>(pa, ph);
    scan_down<CGL>(da, dc);
    if (wl >= 64 - CGL) {
      total[0][wave][cl + v] = pa;
      total[1][wave][cl + v] = ph;
    }
    if (wl < CGL) total[2][wave][cl + v] = dc;
    ea[v] = fa[v] = 1.0f;
    eh[v] = fc[v] = 0.0f;
    if constexpr (WG > 1) {
      const float xa = __shfl_up(pa, CGL, 64), xh = __shfl_up(ph, CGL, 64);
      const float ya = __shfl_down(da, CGL, 64), yc = __shfl_down(dc, CGL, 64);
      if (wl >= CGL) ea[v] = xa, eh[v] = xh;
      if (wl < 64 - CGL) fa[v] = ya, fc[v] = yc;
    }
  }
  __syncthreads();
  float ta = 1.0f, tc = 0.0f;
  uint64_t* words = A.words + (size_t)chain * tiles * GATED_TILE_WORDS;
  const int cw = cb + wl;
  const float init = o == 0 && wave == 0 && A.dh_out != nullptr && cw < A.D ? A.dh_out[b * A.D + cw] : 0.0f;
  if (wave == 0) {
#pragma unroll
    for (int w = NW - 1; w >= 0; --w) {
      const float m = total[0][w][wl];
      tc = fmaf(m, tc, total[2][w][wl]);
      ta *= m;
    }
    if (LOOK && o + 1 < tiles) {
      uint64_t* w = words + o * GATED_TILE_WORDS + wl;
      store_word(w, ta, tag);
      store_word(w + 64, tc, tag);
    }
  }
  // the states before the steps (nothing of this waits for other tiles)
  for (int w = 0; w < wave; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) h[v] = fmaf(total[0][w][cl + v], h[v], total[1][w][cl + v]);
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    h[v] = fmaf(ea[v], h[v], eh[v]);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float before = h[v];
      h[v] = fmaf(a[s][v], h[v], hp[s][v]);
      hp[s][v] = before;
    }
  }
  if (LOOK && o > 0) {
    look_back(words, o, tag, A.hdr, sh);
  } else {
    if (wave == 0) sh.enter[wl] = init;
    __syncthreads();
  }
  if (wave == 0) {
    const float end = fmaf(ta, sh.enter[wl], tc);
    if (LOOK && o + 1 < tiles) store_word(words + o * GATED_TILE_WORDS + 128 + wl, end, tag);
    if (A.dh0 != nullptr && o + 1 == tiles && cw < A.D) A.dh0[b * A.D + cw] = end;
  }
  float cc[VEC], sum[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    cc[v] = sh.enter[cl + v];
    sum[v] = 0.0f;
  }
  for (int w = NW - 1; w > wave; --w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) cc[v] = fmaf(total[0][w][cl + v], cc[v], total[2][w][cl + v]);
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    cc[v] = fmaf(fa[v], cc[v], fc[v]);
    // a, beta and sigmoid(i) are computed again below: kept from above they would take half of the registers
#pragma unroll
    for (int s = 0; s < S; ++s) asm volatile("" : "+v"(sr[s][v]));
  }
  opaque(i);
  float dgam[VEC];  // gamma itself: dr = w s (1 - sr)
#pragma unroll
  for (int v = 0; v < VEC; ++v) dgam[v] = A.gamma[cs + v];
  const Walk ox = walk<T>(A.dx.p, A.dx.sb, A.dx.st, b, tt, mine, cs), orr = walk<T>(A.dr.p, A.dr.sb, A.dr.st, b, tt, mine, cs),
             oi = walk<T>(A.di.p, A.di.sb, A.di.st, b, tt, mine, cs);
#pragma unroll
  for (int s = S - 1; s >= 0; --s) {
    Vec<T, VEC> vx, vr, vi;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float z = gam[v] * sr[s][v], av = exp2_fast(-z), xv = to_f32(x[s].v[v]), qv = sigmoid_fast(to_f32(i[s].v[v]));
      const float e = one_minus_a2(z, av), rb = e <= 1e-36f ? 0.0f : __builtin_amdgcn_rsqf(e);  // 1 / beta
      const float g = to_f32(d[s].v[v]) + cc[v], ag = av * g, gb = g * (e * rb) * qv;
      cc[v] = ag;
      const float w = ag * fmaf(av * rb * qv, xv, -hp[s][v]);
      vx.v[v] = from_f32<T>(gb);
      vi.v[v] = from_f32<T>(gb * xv * (1.0f - qv));
      const float ws = w * sr[s][v];
      sum[v] += ws;
      vr.v[v] = from_f32<T>(ws * (1.0f - sr[s][v]) * dgam[v]);
    }
    if (valid < TILE && mine + s >= valid) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) vx.v[v] = vr.v[v] = vi.v[v] = T(0);
    }
    if (c < A.D && (there == TILE || mine + s < there)) {
      store_row<T, VEC>(ox, s, vx);
      store_row<T, VEC>(orr, s, vr);
      store_row<T, VEC>(oi, s, vi);
    }
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
#pragma unroll
    for (int k = CGL; k < 64; k <<= 1) sum[v] += __shfl_xor(sum[v], k, 64);
    if (wl < CGL) sums[wave][cl + v] = sum[v];
  }
  __syncthreads();
  if (wave == 0) {
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) t += sums[w][wl];
    // (a word like the others, so that what a later call finds here is never taken for one of its own)
    A.part[(b * tiles + tile) * ((int64_t)A.NB * GATED_CW) + cw] = word(t, tag);
  }
  if constexpr (LOOK) leave(A.hdr, tag);
}

// dgamma[c] = sum of the rows of part [n][Dp]: 16 channels of a work-group, its 64 rows of threads every 64th row, then
// their sums in order, in float64.  (512 rows of 256: 4.6 us, latency.)
__global__ __launch_bounds__(1024) void gated_reduce_kernel(const uint64_t* part, int64_t n, int Dp, int D, float* dgamma) {
  __shared__ double sums[64][16];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
  double s = 0.0;
  if (c < D)
    for (int64_t k = g; k < n; k += 64) s += __uint_as_float((uint32_t)part[k * Dp + c]);
  sums[g][l] = s;
  __syncthreads();
  if (g == 0 && c < D) {
    for (int k = 1; k < 64; ++k) s += sums[k][l];
    dgamma[c] = (float)s;
  }
}

// One step of every sequence: an element a thread (64 x 256 bf16 2.3 us, the latency of a launch and one round of loads).
template <typename T>
__global__ __launch_bounds__(256) void gated_step_kernel(Rows x, Rows r, Rows i, T* y, int64_t B, int64_t D,
                                                         const float* gamma, const float* h, float* h_out) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (k >= B * D) return;
  const int64_t b = k / D, c = k - b * D;
  const float z = LOG2E * gamma[c] * sigmoid_fast(to_f32(((const T*)r.p)[b * r.sb + c])), a = exp2_fast(-z);
  const float u = beta_of(z, a) * sigmoid_fast(to_f32(((const T*)i.p)[b * i.sb + c])) * to_f32(((const T*)x.p)[b * x.sb + c]);
  const float v = fmaf(a, h[k], u);
  h_out[k] = v;
  y[k] = from_f32<T>(v);
}

// A chain of one tile needs no look-back, no tickets and no words: the smallest tile that holds it (8 x 32 x 256 bf16 4.7 us
// with 64 threads, 8.8 with 512, 10.5 with the look-back; 512 x 128 x 256 with 256 threads 25, 42 and 62).
template <typename T, int VEC, int S>
void gated_fwd(const GatedArgs& a, hipStream_t st) {
  constexpr int STEPS = S * VEC;  // of a wave
  const dim3 chains((unsigned)(a.B * a.NB));
  if (a.L <= STEPS)
    gated_fwd_kernel<T, VEC, S, 64, false><<<chains, 64, 0, st>>>(a);
  else if (a.L <= 4 * STEPS)
    gated_fwd_kernel<T, VEC, S, 256, false><<<chains, 256, 0, st>>>(a);
  else if (a.L <= 8 * STEPS)
    gated_fwd_kernel<T, VEC, S, 512, false><<<chains, 512, 0, st>>>(a);
  else
    gated_fwd_kernel<T, VEC, S, 512, true><<<dim3((unsigned)(a.B * a.NB * gated_tiles(a.L, 8 * STEPS))), 512, 0, st>>>(a);
}
template <typename T, int VEC, int S>
void gated_bwd(const GatedArgs& a, hipStream_t st) {
  constexpr int STEPS = S * VEC;
  if (a.L <= 8 * STEPS)
    gated_bwd_kernel<T, VEC, S, 512, false><<<dim3((unsigned)(a.B * a.NB)), 512, 0, st>>>(a);
  else
    gated_bwd_kernel<T, VEC, S, 512, true><<<dim3((unsigned)(a.B * a.NB * gated_tiles(a.L, 8 * STEPS))), 512, 0, st>>>(a);
}

// The batch rows from b on, n of them.
template <typename T>
GatedArgs batch_rows(GatedArgs a, int64_t b, int64_t n) {
  const int64_t NC = (a.L + GATED_CARRY - 1) / GATED_CARRY;
  auto on = [](auto*& p, int64_t k) { if (p != nullptr) p += k; };
  for (Rows* v : {&a.x, &a.r, &a.i, &a.dy}) v->p = v->p != nullptr ? (const T*)v->p + b * v->sb : nullptr;
  for (RowsOut* v : {&a.dx, &a.dr, &a.di}) v->p = v->p != nullptr ? (T*)v->p + b * v->sb : nullptr;
  a.y = a.y != nullptr ? (T*)a.y + b * a.L * a.D : nullptr;
  on(a.h0, b * a.D);
  on(a.lengths, b);
  on(a.h_out, b * a.D);
  on(a.carry, b * NC * a.D);
  on(a.dh_out, b * a.D);
  on(a.dh0, b * a.D);
  on(a.part, b * gated_tiles(a.L, GATED_BWD_TILE) * a.NB * GATED_CW);
  a.B = n;
  return a;
}
// Calls f with as many batch rows at a time as one launch takes.
template <typename T, typename F>
void in_launches(const GatedArgs& a, int tile, F&& f) {
  const int64_t most = LAUNCH_THREADS / GATED_THREADS / (a.NB * gated_tiles(a.L, tile));
  for (int64_t b = 0; b < a.B; b += most) f(batch_rows<T>(a, b, a.B - b < most ? a.B - b : most));
}

}  // namespace

template <typename T>
hipError_t launch_gated_fwd(const GatedArgs& all, hipStream_t st) {
  in_launches<T>(all, GATED_FWD_TILE, [&](const GatedArgs& a) {
    if (a.vec)
      gated_fwd<T, 4, 8>(a, st);
    else
      gated_fwd<T, 1, 32>(a, st);  // a channel a lane: rows of any alignment read in one piece
  });
  return hipGetLastError();
}

template <typename T>
hipError_t launch_gated_bwd(const GatedArgs& a, float* dgamma, hipStream_t st) {
  in_launches<T>(a, GATED_BWD_TILE, [&](const GatedArgs& a) {
    if (a.vec)
      gated_bwd<T, sizeof(T) == 2 ? 2 : 4, sizeof(T) == 2 ? 8 : 4>(a, st);
    else
      gated_bwd<T, 1, 16>(a, st);
  });
  const int64_t rows = a.B * gated_tiles(a.L, GATED_BWD_TILE);
  gated_reduce_kernel<<<dim3((unsigned)((a.D + 15) / 16)), 1024, 0, st>>>(a.part, rows, a.NB * GATED_CW, a.D, dgamma);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_gated_step(const Rows& x, const Rows& r, const Rows& i, void* y, int64_t B, int64_t D,
                             const float* gamma, const float* h, float* h_out, hipStream_t st) {
  const int64_t most = (LAUNCH_THREADS - 255) / D;  // rows of a launch
  for (int64_t b = 0; b < B; b += most) {
    const int64_t n = B - b < most ? B - b : most;
    auto rows = [&](const Rows& v) { return Rows{(const T*)v.p + b * v.sb, v.sb, v.st}; };
    gated_step_kernel<T><<<dim3((unsigned)((n * D + 255) / 256)), 256, 0, st>>>(rows(x), rows(r), rows(i), (T*)y + b * D, n, D, gamma,
                                                                                h + b * D, h_out + b * D);
  }
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
