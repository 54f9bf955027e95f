// Linear product with bias, activation and residual, and its gradients:
//   pre = x W + b, y = act(pre) + residual;
//   dpre = dy act'(pre), dx = dpre W^T, dW = x^T dpre, db = sum over rows of dpre.
// All products are one tiled kernel over operands of either order; sums are float32 (MFMA).
// dpre is made by a product too where computing pre again costs less than keeping it.
// For bf16, dpre is rounded to bf16 before the products that give dx and dW, since the matrix unit takes operands of one
// type (two bf16 parts of it would double both products and the bytes of dpre): over all results of 65536 x 256 x 1024 with
// gelu the error is 2.4e-3 of their size, where the results' own rounding is 1.7e-3.  db sums dpre unrounded.
#include "layer.h"
#include "stream.h"

namespace res {
namespace {

template <typename T> struct __align__(4 * sizeof(T)) Quad { T v[4]; };
template <typename T>
__device__ __forceinline__ f4 wide(const Quad<T>& q) {
  f4 c;
#pragma unroll
  for (int r = 0; r < 4; ++r) c[r] = to_f32(q.v[r]);
  return c;
}
__device__ __forceinline__ Quad<float> round_quad(const f4& c, float) { return __builtin_bit_cast(Quad<float>, c); }
__device__ __forceinline__ Quad<bf16_t> round_quad(const f4& c, bf16_t) {
  typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(Quad<bf16_t>, __builtin_convertvector(c, bf4));
}
// N elements at the alignment of one: the unit takes vector accesses at any address.
template <typename T, int N> using Any = T __attribute__((ext_vector_type(N), aligned(sizeof(T))));
// Columns n .. n + 3 of a row of N; loose: no alignment, and columns from N on are the last one again.
template <typename T>
__device__ __forceinline__ Quad<T> load_quad(const T* row, int n, int64_t N, bool loose) {
  if (!loose) return *reinterpret_cast<const Quad<T>*>(row + n);
  if (n + 4 <= N) return __builtin_bit_cast(Quad<T>, *reinterpret_cast<const Any<T, 4>*>(row + n));
  Quad<T> q;
#pragma unroll
  for (int r = 0; r < 4; ++r) q.v[r] = row[n + r < N ? n + r : N - 1];
  return q;
}

// ---------------------------------------------------------------------------
// Tiles of BM x BN outputs; operands are 16-byte aligned with rows of whole 16-byte
// pieces (others are copied into such a form first).  A wave owns WM x WN of
// them in registers; 64 bytes of the K axis at a time (KB elements, the depth of one
// fragment) go straight to LDS (16 bytes a lane, no registers), the next ones while
// these are multiplied.
//
// An operand whose K axis is consecutive in memory lies in LDS as rows of 64
// bytes, 16-byte piece s of row r in slot s ^ (r >> 2 & 3): the lanes that read one
// piece of eight rows meet different banks.  One whose other axis is consecutive (X bytes a row)
// lies as it is in memory, one row for each k, and is transposed by the read: bf16 by
// the transposing LDS load (a group of 16 lanes reads 4 k of 16 columns, and lane i
// gets the 4 k of column i), float by single words.  There the 16 columns of a fragment
// are one granule (32 or 64 bytes), and granule c of row k is in slot c ^ f(k) with an f
// that tells apart the rows that are read at once.
// The loads go to LDS in order, so the swizzles are applied to the source addresses.
//
// The product is taken as C^T (the column operand first), so that a lane's four
// results are four columns of one row: 8-byte stores for bf16.
// ---------------------------------------------------------------------------
__device__ __align__(16) const uint32_t zero_piece[4] = {};  // what lies behind the K axis

template <typename T> struct Gemm {
  static constexpr int ES = sizeof(T), KB = 64 / ES, EP = 16 / ES;  // K elements of a step; elements of a piece
  typedef typename Path<T>::XOp Frag;
};

// a value that is the same in all lanes, in scalar registers
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const char*)((uint64_t)hi << 32 | lo);
}

// The lane again, as a value that the compiler does not know: what is computed from it stays where it is used.  (Hoisted out
// of the loop over items, the addresses of its rarer parts took 60 registers.)
__device__ __forceinline__ int lane_here(int lane) {
  asm volatile("" : "+v"(lane));
  return lane;
}

// Loads an operand's tile: rows x0.. of X and KB elements of the K axis.  KC: element (x, k) at p[x ld + k], else at
// p[k ld + x].  A lane's byte offsets from the tile's start do not change along K (only the scalar base does), and
// rows past the end are the last ones again: what they give is not stored.
template <typename T, int BX, int NW, bool KC> struct TileLoad {
  static constexpr int ES = sizeof(T), EP = 16 / ES, RB = KC ? 64 : BX * ES, PR = RB / 16, RU = 1024 / RB;
  static constexpr int UNITS = BX / 16 / NW;
  static_assert(BX % (16 * NW) == 0 && RB <= 1024, "whole units of a kilobyte for each wave");
  uint32_t off[UNITS];
  const char* base;  // the next step's first element (the same in all lanes)
  int64_t step;      // bytes of a step

  __device__ static __forceinline__ int row_of(int u, int wave, int lane) { return (wave * UNITS + u) * RU + lane / PR; }
  __device__ static __forceinline__ int piece_of(int row, int lane) {
    const int slot = lane % PR;
    if constexpr (KC) return slot ^ ((row >> 2) & 3);
    if constexpr (ES == 2 && RB >= 256) return slot ^ (((row & 3) | ((row >> 1) & 4)) << 1);
    if constexpr (ES == 2) return slot ^ ((((row >> 1) & 1) | ((row >> 2) & 2)) << 1);  // (four granules a row)
    return slot ^ (((row >> 2) & 3) << 2);
  }
  __device__ __forceinline__ void open(const T* p, int64_t ld, int64_t x0, int64_t X, int64_t k0, int wave, int lane) {
    base = uniform((const char*)(p + x0 * (KC ? ld : 1) + k0 * (KC ? 1 : ld)));
    step = (KC ? 1 : ld) * ES * Gemm<T>::KB;
    const int64_t left = X - x0;
    lane = lane_here(lane);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int row = row_of(u, wave, lane), piece = piece_of(row, lane);
      if constexpr (KC)
        off[u] = (uint32_t)((row < left ? row : left - 1) * ld * ES + piece * 16);
      else
        off[u] = (uint32_t)(row * ld * ES + (piece * EP < left ? piece * EP : left - EP) * ES);
    }
  }
  // the next step's elements
  __device__ __forceinline__ void load(char* lds, int wave) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) lds_dma16(base, off[u], lds + (wave * UNITS + u) * 1024);
    base = uniform(base + step);
  }
  // the same where only `left` elements of the K axis are left: zeros behind them
  __device__ __forceinline__ void load_last(int left, char* lds, int wave, int lane) {
    lane = lane_here(lane);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int row = row_of(u, wave, lane), piece = piece_of(row, lane);
      const void* src = (KC ? piece * EP : row) < left ? (const void*)(base + off[u]) : (const void*)zero_piece;
      lds_dma16_lane(src, lds + (wave * UNITS + u) * 1024);
    }
  }
};

// The fragment of columns (or rows) c .. c + 15.
template <typename T, int BX, bool KC>
__device__ __forceinline__ typename Gemm<T>::Frag fragment(const char* lds, int c, int li, int lq) {
  if constexpr (KC) {
    return *reinterpret_cast<const typename Gemm<T>::Frag*>(lds + (c + li) * 64 + ((lq ^ (li >> 2)) << 4));
  } else if constexpr (sizeof(T) == 2) {
    constexpr int RB = BX * 2;
    typedef __attribute__((address_space(3))) s4 lds_s4;
    const int row = 8 * lq + (li >> 2), f = RB >= 256 ? (li >> 2) | ((lq & 1) << 2) : (li >> 3) | ((lq & 1) << 1);
    const char* p = lds + row * RB + (((c >> 4) ^ f) << 5) + (li & 3) * 8;
    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)p);
    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(p + 4 * RB));
    return __builtin_bit_cast(bf8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    constexpr int RB = BX * 4;
    const char* p = lds + 4 * lq * RB + (((c >> 4) ^ lq) << 6) + li * 4;
    f4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float*>(p + j * RB);
    return v;
  }
}

// Tile of a work-group: work-groups go to the eight dies in turn, so die d takes the
// d-th eighth of the tiles; there, blocks of eight rows of tiles, column after column,
// so that the work-groups that run together share operands in the die's cache.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, int64_t* m, int64_t* n) {
  const uint32_t all = tm * tn, q = all / 8, r = all % 8, d = id % 8;
  id = d * q + (d < r ? d : r) + id / 8;
  const uint32_t g = id / (8 * tn), first = g * 8, rows = tm - first < 8 ? tm - first : 8, in = id - g * 8 * tn;
  *m = __builtin_amdgcn_readfirstlane(first + in % rows);
  *n = __builtin_amdgcn_readfirstlane(in / rows);
}

// LDS of a wave's outputs on their way out: rows of one fragment
template <typename T, int WN> constexpr int out_lds() { return 16 * WN * (int)sizeof(T); }

// What an item reads beside its operands (the residual, or dy) comes through the buffers too, behind its last step: SR
// rows of each wave's outputs at a time, every wave its own.  Reading it where it is needed exposed a memory latency and
// took 32-byte pieces.
template <typename T, int WM, int WN> struct SideLoad {
  static constexpr int ES = sizeof(T), EP = 16 / ES, RB = WN * ES, PR = RB / 16, SR = 64 / ES, STEPS = WM / SR, SW = PR < 8 ? PR - 1 : 7;
  static constexpr int BYTES = SR * RB, UNITS = BYTES / 1024, RU = 1024 / RB;
  static_assert(WM % SR == 0 && BYTES % 1024 == 0, "whole units");
  // rows m0 + SR s .. of the wave's, columns n0 ..; those past the end are the last ones again
  __device__ static __forceinline__ void load(const T* side, int64_t m0, int64_t n0, int64_t M, int64_t N, int s, char* lds, int lane) {
    const char* base = uniform((const char*)side);
    lane = lane_here(lane);
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int r = u * RU + lane / PR;
      int64_t m = m0 + s * SR + r, n = n0 + (((lane % PR) ^ (r & SW)) * EP);
      m = m < M ? m : M - 1;
      n = n < N ? n : N - EP;
      lds_dma16_lane(base + (m * N + n) * ES, lds + u * 1024);
    }
  }
  // columns 16 j + 4 lq .. of row r of a step
  __device__ static __forceinline__ Quad<T> read(const char* lds, int r, int j, int lq) {
    const int byte = (j * 16 + lq * 4) * ES;
    return *reinterpret_cast<const Quad<T>*>(lds + r * RB + (((byte >> 4) ^ (r & SW)) << 4) + (byte & 15));
  }
};

// A wave's outputs through its own part of the LDS, 16 rows at a time (16-byte piece p of row m in slot p ^ (m & 7)), so
// that they are stored as whole rows of the wave's: 128 bytes (the 128 x 256 tile, and float32) or, in bf16, 64 (the other
// tiles, whose waves are 32 columns wide); the results' own layout gives 32-byte pieces.  The stores are non-temporal
// (131072 x 256 x 1024 bf16: 139 to 123 us); of 64 bytes, half a line, they cost more than their bytes (the product that makes
// dpre of 65536 x 256 x 1024: 154 thousand KiB for 135).  Rows and columns past the end are computed from the
// last ones' operands and not stored.
// ANY: takes outputs of any alignment (g.loose): whole pieces all the same, the last of a row by elements (11573 x 32 x 1964
// bf16, gelu, with gradients: 201 to 147 us).  SLOPE: the results are pre, and what is stored is dy act'(pre); its
// columns' sums go to g.colpart.  stage(s): this wave's step s of the side input in the LDS, null where it is not there.
template <typename T, int ACT, bool SLOPE, bool ANY, int WM, int WN, typename Stage>
__device__ __forceinline__ void tile_out(const GemmArgs& g, int64_t m0, int64_t n0, const f4 (&acc)[WM / 16][WN / 16],
                                         char* mine, int lane, Stage&& stage) {
  constexpr int ES = sizeof(T), RB = WN * ES, PR = RB / 16, EP = 16 / ES, SW = PR < 8 ? PR - 1 : 7, FN = WN / 16;
  constexpr int RS = 64 / PR;  // rows of a store
  typedef SideLoad<T, WM, WN> Side;
  constexpr int SF = Side::SR / 16;  // fragments of rows in a side step
  lane = lane_here(lane);
  const int li = lane & 15, lq = lane >> 4;
  const bool loose = ANY && g.loose;
  const int rows = (int)(g.M - m0 < WM ? (g.M > m0 ? g.M - m0 : 0) : WM);  // of this wave's that there are
  int n[FN];
  f4 bias[FN], sum[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    n[j] = (int)n0 + j * 16 + lq * 4;
    n[j] = n[j] < (int)g.N ? n[j] : ((int)g.N - 1) & ~3;
    bias[j] = g.bias != nullptr ? wide(load_quad(g.bias, n[j], g.N, loose)) : f4{};
    sum[j] = f4{};
  }
  const T* side = (const T*)(SLOPE ? g.dy : g.res);
  const char* staged = nullptr;
  // stores: this lane's row of a fragment's first RS, and on from there
  T* to = (T*)g.out + (m0 + lane / PR) * g.N + n0;
  const int64_t next = RS * g.N;
#pragma unroll
  for (int i = 0; i < WM / 16; ++i) {
    const int row = i * 16 + li;
    f4 q[FN];
    if (side != nullptr) {
      if (i % SF == 0) staged = stage(i / SF);
      if (!loose) {
#pragma unroll
        for (int j = 0; j < FN; ++j) q[j] = wide(Side::read(staged, i % SF * 16 + li, j, lq));
      } else {
        const T* from = side + (m0 + row < g.M ? m0 + row : g.M - 1) * g.N;
#pragma unroll
        for (int j = 0; j < FN; ++j) q[j] = wide(load_quad(from, n[j], g.N, true));
      }
    }
    f4 c[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) c[j] = acc[i][j] + bias[j];
    if constexpr (SLOPE) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          c[j][r] = q[j][r] * act_slope(c[j][r], ACT);
          sum[j][r] += row < rows ? c[j][r] : 0.0f;
        }
    } else {
      if (g.pre != nullptr && row < rows) {
        float* pre = g.pre + (m0 + row) * g.N;
#pragma unroll
        for (int j = 0; j < FN; ++j)
          if ((int)n0 + j * 16 + lq * 4 < (int)g.N) {
            if (!loose || n[j] + 4 <= (int)g.N) {
              *reinterpret_cast<Any<float, 4>*>(pre + n[j]) = c[j];
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (n[j] + r < (int)g.N) pre[n[j] + r] = c[j][r];
            }
          }
      }
      if constexpr (ACT != ACT_NONE) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) c[j][r] = act_value(c[j][r], ACT);
      }
      if (side != nullptr) {
#pragma unroll
        for (int j = 0; j < FN; ++j) c[j] += q[j];
      }
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int byte = (j * 16 + lq * 4) * ES;
      *reinterpret_cast<Quad<T>*>(mine + li * RB + (((byte >> 4) ^ (li & SW)) << 4) + (byte & 15)) = round_quad(c[j], T());
    }
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    typedef uint32_t u4_any __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
    for (int u = 0; u < 16 / RS; ++u) {
      const int r = u * RS + lane / PR, slot = lane % PR, col = (slot ^ (r & SW)) * EP;
      const u4 v = *reinterpret_cast<const u4*>(mine + r * RB + slot * 16);
      const int there = (int)(g.N - n0) - col;  // columns of the piece that there are, or more
      if (i * 16 + r < rows && there > 0) {
        if (!loose) {
          __builtin_nontemporal_store(v, reinterpret_cast<u4*>(to + col));
        } else if (there >= EP) {
          __builtin_nontemporal_store((u4_any)v, reinterpret_cast<u4_any*>(to + col));
        } else {
          const Any<T, EP> e = __builtin_bit_cast(Any<T, EP>, v);
#pragma unroll
          for (int k = 0; k < EP - 1; ++k)
            if (k < there) to[col + k] = e[k];
        }
      }
      to += next;
    }
  }
  if constexpr (SLOPE) {
    if (g.colpart != nullptr && m0 < g.M) {
      float* part = g.colpart + m0 / WM * g.N;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float v = sum[j][r];
#pragma unroll
          for (int k = 1; k < 16; k <<= 1) v += __shfl_xor(v, k, 64);
          const int64_t col = n0 + j * 16 + lq * 4 + r;
          if (li == 0 && col < g.N) part[col] = v;
        }
    }
  }
}

// Work-groups stay: each takes every gridDim-th item (a tile and a part of the K axis), and the loads run NB - 1 steps
// ahead of the products over the borders of the items, so that neither an item's first loads nor its stores are waited
// for.  NB buffers of a step and the LDS of each wave's outputs.
//
// bf16 8192 x 4096 x 4096 (R x K x N) with a residual 243 us (1130 TFLOP/s, where a library product without one reaches
// 1313): bound by the cache's bytes into LDS.  With a short sum the epilogue bounds it, 14 vector instructions an output
// with gelu: 131072 x 256 x 1024 111 us (3.0 TB/s); with gelu's slope 36, 65536 x 256 x 1024 127 us; without either 53
// (data gradient).  float32 8192 x 2048 x 2048 590 us (116 TFLOP/s; the library 128).
template <typename T, int BM, int BN, int WM, int WN, int NB, bool ANY, bool AK, bool BK, int ACT, bool SLOPE>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN), (BM / WM) * (BN / WN) / 2) void gemm_tile_kernel(GemmArgs g) {
  constexpr int NW = (BM / WM) * (BN / WN), KB = Gemm<T>::KB, FM = WM / 16, FN = WN / 16, STEP = (BM + BN) * 64;
  __shared__ __align__(1024) char lds[NB * STEP + NW * out_lds<T, WN>()];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lq = lane >> 4;
  const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
  const uint32_t mt = (uint32_t)((g.M + BM - 1) / BM), nt = (uint32_t)((g.N + BN - 1) / BN), tiles = mt * nt, items = tiles * g.splits;
  const int64_t per = ((g.K + g.splits - 1) / g.splits + KB - 1) / KB * KB;  // (no part is empty: see linear_plan)
  typedef TileLoad<T, BM, NW, AK> LoadA;
  typedef TileLoad<T, BN, NW, BK> LoadB;
  typedef SideLoad<T, WM, WN> Side;
  static_assert(NW * Side::BYTES <= STEP, "a side step fits into a buffer");
  constexpr int UNITS = LoadA::UNITS + LoadB::UNITS;  // loads of a step by one wave
  constexpr int FEWER = Side::UNITS < UNITS ? Side::UNITS : UNITS;
  const T* side = (const T*)(SLOPE ? g.dy : g.res);
  const bool staged = side != nullptr && g.splits == 1 && !(ANY && g.loose);

  // Steps of an item's part of the K axis, and the elements of its last one.
  auto steps_of = [&](uint32_t part, int* last) {
    const int64_t k0 = part * per, n = k0 + per < g.K ? per : g.K - k0;
    const int steps = (int)((n + KB - 1) / KB);
    *last = __builtin_amdgcn_readfirstlane((int)(n - (int64_t)(steps - 1) * KB));
    return __builtin_amdgcn_readfirstlane(steps);
  };

  // the loads: the item they are at, and the steps left of it (the side input's are counted below zero)
  LoadA load_a;
  LoadB load_b;
  uint32_t next = blockIdx.x;
  int64_t pm = 0, pn = 0;
  int left = 0, last = 0, beside = 0;
  int ahead = 0;  // steps loaded or on their way that are not used yet
  auto prefetch = [&](int at) {
    if (left == 0 && beside == 0) {
      if (next >= items) return;
      int64_t tm, tn;
      const uint32_t part = next / tiles;
      tile_of(next - part * tiles, mt, nt, &tm, &tn);
      left = steps_of(part, &last);
      load_a.open((const T*)g.A, g.lda, tm * BM, g.xa, part * per, wave, lane);
      load_b.open((const T*)g.B, g.ldb, tn * BN, g.xb, part * per, wave, lane);
      pm = tm * BM + wm;
      pn = tn * BN + wn;
      if (staged) beside = Side::STEPS;
      next += gridDim.x;
    }
    ++ahead;
    if (left > 0) {
      --left;
      if (left > 0 || last == KB) {
        load_a.load(lds + at, wave);
        load_b.load(lds + at + BM * 64, wave);
      } else {
        load_a.load_last(last, lds + at, wave, lane);
        load_b.load_last(last, lds + at + BM * 64, wave, lane);
      }
    } else {
      Side::load(side, pm, pn, g.M, g.N, Side::STEPS - beside, lds + at + wave * Side::BYTES, lane);
      --beside;
    }
  };
  // Of the steps on their way all but NB - 2 have come: a wave's loads come in order, and none of the steps behind the one
  // that is waited for has fewer than UNITS (or, with side steps among them, FEWER).
  auto arrived = [&] {
    if (ahead < NB - 1) wait_vm<0>();
    else if (staged) wait_vm<(NB - 2) * FEWER>();
    else wait_vm<(NB - 2) * UNITS>();
  };
#pragma unroll
  for (int b = 0; b < NB - 1; ++b) prefetch(b * STEP);

  int at = 0, to = (NB - 1) * STEP;  // buffers of the step that is used and of the one that is loaded meanwhile
  auto advance = [&] {
    --ahead;
    to = at;
    at = at == (NB - 1) * STEP ? 0 : at + STEP;
  };
  bool waited = false;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    int64_t tm, tn;
    const uint32_t part = item / tiles;
    tile_of(item - part * tiles, mt, nt, &tm, &tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    f4 acc[FM][FN] = {};
    int unused;
    for (int s = steps_of(part, &unused); s > 0; --s) {
      // this wave's pieces of the step are there, and past the barrier everyone's; the buffer of the step before has been
      // read by all
      if (!waited) arrived();
      waited = false;
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const char* la = lds + at;
      const char* lb = la + BM * 64;
      // all fragments first, so that the products run through (left to itself the compiler reads them two at a time
      // and waits for each pair)
      typename Gemm<T>::Frag fb[FN], fa[FM];
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = fragment<T, BN, BK>(lb, wn + j * 16, li, lq);
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = fragment<T, BM, AK>(la, wm + i * 16, li, lq);
      prefetch(to);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          if constexpr (sizeof(T) == 2)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
          else
            acc[i][j] = mma_f32(fb[j], fa[i], acc[i][j]);
        }
      }
      advance();
    }
    if (g.splits > 1) {
      arrived();  // as below
      waited = true;
      float* o = g.part + part * g.M * g.N;
      const int l = lane_here(lane);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + wm + i * 16 + (l & 15);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int64_t n = n0 + wn + j * 16 + (l >> 4) * 4;
          if (m >= g.M) continue;
          if (g.N % 4 == 0) {
            if (n < g.N) *reinterpret_cast<f4*>(o + m * g.N + n) = acc[i][j];
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (n + r < g.N) o[m * g.N + n + r] = acc[i][j][r];
          }
        }
      }
      continue;
    }
    if (!staged) {
      // the next step's loads are waited for before the stores are issued, so that no step waits for the stores
      arrived();
      waited = true;
    }
    tile_out<T, ACT, SLOPE, ANY, WM, WN>(g, m0 + wm, n0 + wn, acc, lds + NB * STEP + wave * out_lds<T, WN>(), lane, [&](int) -> const char* {
      if (!staged) return nullptr;
      arrived();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      prefetch(to);
      const char* here = lds + at + wave * Side::BYTES;
      advance();
      return here;
    });
  }
}

// Few outputs: a work-group has one 64 x 64 tile, and each of its eight waves all of the tile for an eighth of the K axis,
// loaded and multiplied without a barrier; then the eight sums are added in order through the LDS and the epilogue follows.
// One launch instead of a split product's two and its partial sums in memory: 64 x 1024 x 4096 (R x K x N) bf16 8.4 us in a
// graph, where the 8 MB of the weights are 1.8 us of memory and the rest is the latency of a launch and of two to four
// loads one behind the other.
template <typename T, bool AK, bool BK>
__global__ __launch_bounds__(512, 2) void gemm_deep_kernel(GemmArgs g) {
  constexpr int NW = 8, NB = 2, KB = Gemm<T>::KB, STEP = 128 * 64;
  __shared__ __align__(1024) char lds[NW * NB * STEP];
  static_assert(NB * STEP == 64 * 64 * 4, "a wave's buffers hold its sums");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lq = lane >> 4;
  const uint32_t nt = (uint32_t)((g.N + 63) / 64);
  const int64_t m0 = (int64_t)(blockIdx.x / nt) * 64, n0 = (int64_t)(blockIdx.x % nt) * 64;
  char* mine = lds + wave * (NB * STEP);
  typedef TileLoad<T, 64, 1, AK> LoadA;
  typedef TileLoad<T, 64, 1, BK> LoadB;
  const int steps = (int)((g.K + KB - 1) / KB), last = (int)(g.K - (int64_t)(steps - 1) * KB);
  const int begin = wave * steps / NW, end = (wave + 1) * steps / NW;
  LoadA load_a;
  LoadB load_b;
  load_a.open((const T*)g.A, g.lda, m0, g.xa, (int64_t)begin * KB, 0, lane);
  load_b.open((const T*)g.B, g.ldb, n0, g.xb, (int64_t)begin * KB, 0, lane);
  int next = begin;
  auto prefetch = [&] {
    if (next >= end) return;
    char* to = mine + (next - begin) % NB * STEP;
    if (next + 1 < steps || last == KB) {
      load_a.load(to, 0);
      load_b.load(to + 64 * 64, 0);
    } else {
      load_a.load_last(last, to, 0, lane);
      load_b.load_last(last, to + 64 * 64, 0, lane);
    }
    ++next;
  };
#pragma unroll
  for (int b = 0; b < NB; ++b) prefetch();
  f4 acc[4][4] = {};
  for (int s = begin; s < end; ++s) {
    if (next - s < NB) wait_vm<0>();
    else wait_vm<(NB - 1) * (LoadA::UNITS + LoadB::UNITS)>();
    asm volatile("" ::: "memory");
    const char* la = mine + (s - begin) % NB * STEP;
    const char* lb = la + 64 * 64;
    typename Gemm<T>::Frag fa[4], fb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) fb[j] = fragment<T, 64, BK>(lb, j * 16, li, lq);
#pragma unroll
    for (int i = 0; i < 4; ++i) fa[i] = fragment<T, 64, AK>(la, i * 16, li, lq);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read, before the buffer is loaded again
    prefetch();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
        else
          acc[i][j] = mma_f32(fb[j], fa[i], acc[i][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<f4*>(mine + ((i * 4 + j) * 64 + lane) * 16) = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int at = k * 512 + threadIdx.x, l = at & 63, f = at >> 6;
    f4 c = *reinterpret_cast<const f4*>(lds + at * 16);
#pragma unroll
    for (int w = 1; w < NW; ++w) c += *reinterpret_cast<const f4*>(lds + w * (NB * STEP) + at * 16);
    const int64_t m = m0 + f / 4 * 16 + (l & 15);
    const int n = (int)n0 + f % 4 * 16 + (l >> 4) * 4;
    if (m >= g.M || n >= (int)g.N) continue;
    if (g.bias != nullptr) c += wide(load_quad(g.bias, n, g.N, g.loose));
    const int there = g.loose && g.N - n < 4 ? (int)(g.N - n) : 4;
    if (g.pre != nullptr)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r < there) g.pre[m * g.N + n + r] = c[r];
#pragma unroll
    for (int r = 0; r < 4; ++r) c[r] = act_value(c[r], g.act);
    if (g.res != nullptr) c += wide(load_quad((const T*)g.res + m * g.N, n, g.N, g.loose));
    const Quad<T> q = round_quad(c, T());
    T* o = (T*)g.out + m * g.N + n;
    if (!g.loose) {
      *reinterpret_cast<Quad<T>*>(o) = q;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r < there) o[r] = q.v[r];
    }
  }
}

// The parts of a split sum (none: zeros), in order, then the epilogue.  Eight parts are loaded together: 32 parts of 256 x
// 1024 in 7.5 us (4.5 TB/s, mostly out of the last cache), one after the other 11.
template <typename T, int V>
__global__ __launch_bounds__(256) void gemm_join_kernel(GemmArgs g) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * V, all = g.M * g.N;
  if (at >= all) return;
  const int64_t n = at % g.N;
  constexpr int AT = 8;  // parts loaded at a time
  float c[V] = {};
  for (int s0 = 0; s0 < g.splits; s0 += AT) {
    f4 p[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {  // (past the last: that one again, not used)
      const float* from = g.part + (s0 + i < g.splits ? s0 + i : g.splits - 1) * all + at;
      if constexpr (V == 4) p[i] = *reinterpret_cast<const f4*>(from);
      else p[i][0] = *from;
    }
#pragma unroll
    for (int i = 0; i < AT; ++i)
#pragma unroll
      for (int r = 0; r < V; ++r) c[r] += s0 + i < g.splits ? p[i][r] : 0.0f;
  }
#pragma unroll
  for (int r = 0; r < V; ++r) {
    if (g.bias != nullptr) c[r] += g.bias[n + r];
    if (g.pre != nullptr) g.pre[at + r] = c[r];
    c[r] = act_value(c[r], g.act);
    if (g.res != nullptr) c[r] += to_f32(((const T*)g.res)[at + r]);
    ((T*)g.out)[at + r] = from_f32<T>(c[r]);
  }
}

// An operand [rows][cols] with any start and ld as rows of `to` elements (whole 16-byte pieces), zeros behind cols.  (The
// product's loads take 16 bytes; 200 x 777 float32 takes 2 us, a launch.)
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* src, int64_t ld, int64_t rows, int64_t cols, T* dst, int64_t to) {
  constexpr int EP = 16 / sizeof(T);
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = to / EP;
  if (id >= rows * per) return;
  const int64_t row = id / per, c = (id - row * per) * EP;
  const T* from = src + row * ld + c;
  T __attribute__((ext_vector_type(EP))) o;
  if (c + EP <= cols) {
    o = *reinterpret_cast<const Any<T, EP>*>(from);
  } else {
#pragma unroll
    for (int e = 0; e < EP; ++e) o[e] = c + e < cols ? from[e] : T(0);
  }
  *reinterpret_cast<decltype(o)*>(dst + row * to + c) = o;
}

// dpre from a kept pre, and the sums of its columns over ACT_ROWS rows: a work-group takes 256 columns (four a lane, or
// one where V is 1), its four waves every fourth row.  The rows of out are `to` elements apart, with zeros from column N on,
// so that it is an operand as it is (2331 x 777 float32: 14 us and a copy of 4 to 8 us).
constexpr int ACT_ROWS = 64;
template <typename T, int V>
__global__ __launch_bounds__(256) void act_bwd_kernel(const T* dy, const float* pre, int act, T* out, int64_t to, float* part,
                                                      int64_t R, int64_t N) {
  constexpr int AT = 8 / V > 2 ? 8 : 4;  // rows loaded at a time
  __shared__ float sums[4][64 * V];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t cols = (to + 64 * V - 1) / (64 * V), block = blockIdx.x / cols;
  const int64_t n = (blockIdx.x % cols) * (64 * V) + lane * V, r0 = block * ACT_ROWS + wave;
  float sum[V] = {};
  for (int k = 0; k < ACT_ROWS / 4 && n < to; k += AT) {
    f4 d[AT], p[AT];
#pragma unroll
    for (int i = 0; i < AT; ++i) {  // (rows and columns past the end: the last ones again, not used)
      const int64_t r = r0 + (k + i) * 4, row = (r < R ? r : R - 1) * N, c = n < N ? n : N - V;
      if constexpr (V == 4) {
        d[i] = wide(load_quad(dy + row, (int)c, N, false));
        if (pre != nullptr) p[i] = *reinterpret_cast<const f4*>(pre + row + c);
      } else {
        d[i][0] = to_f32(dy[row + c]);
        if (pre != nullptr) p[i][0] = pre[row + c];
      }
    }
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      const int64_t r = r0 + (k + i) * 4;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (pre != nullptr) d[i][e] *= act_slope(p[i][e], act);
        d[i][e] = r < R && n < N ? d[i][e] : 0.0f;
        sum[e] += d[i][e];
      }
      if (out != nullptr && r < R) {
        if constexpr (V == 4)
          *reinterpret_cast<Quad<T>*>(out + r * to + n) = round_quad(d[i], T());
        else
          out[r * to + n] = from_f32<T>(d[i][0]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) sums[wave][lane * V + e] = sum[e];
  __syncthreads();
  if (part != nullptr && wave == 0 && n < N)
#pragma unroll
    for (int e = 0; e < V; ++e)
      part[block * N + n + e] = (sums[0][lane * V + e] + sums[1][lane * V + e]) + (sums[2][lane * V + e] + sums[3][lane * V + e]);
}

// db = sums of the columns of part [blocks][N]: 16 columns of a work-group, its 64 rows of threads every 64th block, then
// their sums in order, in float64.  (1024 blocks of 1024 columns 7 us: the latency of sixteen loads.)
__global__ __launch_bounds__(1024) void col_sum_kernel(const float* part, int64_t blocks, int64_t N, float* db) {
  __shared__ double sums[64][16];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int64_t n = (int64_t)blockIdx.x * 16 + c;
  double s = 0.0;
  if (n < N)
    for (int64_t b = g; b < blocks; b += 64) s += part[b * N + n];
  sums[g][c] = s;
  __syncthreads();
  if (g == 0 && n < N) {
    for (int k = 1; k < 64; ++k) s += sums[k][c];
    db[n] = (float)s;
  }
}

template <typename T, int BM, int BN, int WM, int WN, int NB, bool ANY>
void launch_tiles(const GemmArgs& a, hipStream_t st) {
  const int64_t items = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.splits;
  const dim3 grid((unsigned)(items < 512 ? items : 512));  // (two work-groups on each of 256 compute units)
  constexpr int NT = 64 * (BM / WM) * (BN / WN);
#define RES_TILES(AK, BK, ACT, SLOPE) gemm_tile_kernel<T, BM, BN, WM, WN, NB, ANY, AK, BK, ACT, SLOPE><<<grid, NT, 0, st>>>(a)
  const int act = a.splits > 1 ? ACT_NONE : a.act;  // (a split product's is applied where its parts are joined)
  if (!a.ak)
    RES_TILES(false, false, ACT_NONE, false);
  else if (a.bk)
    RES_TILES(true, true, ACT_NONE, false);
  else if (a.dy != nullptr) {
    if constexpr (ANY) {  // (the widest tile would keep its sums of columns in memory)
      if (act == ACT_RELU) RES_TILES(true, false, ACT_RELU, true);
      else if (act == ACT_SILU) RES_TILES(true, false, ACT_SILU, true);
      else RES_TILES(true, false, ACT_GELU_TANH, true);
    }
  } else if (act == ACT_RELU)
    RES_TILES(true, false, ACT_RELU, false);
  else if (act == ACT_SILU)
    RES_TILES(true, false, ACT_SILU, false);
  else if (act == ACT_GELU_TANH)
    RES_TILES(true, false, ACT_GELU_TANH, false);
  else
    RES_TILES(true, false, ACT_NONE, false);
#undef RES_TILES
}

}  // namespace

int64_t linear_row_blocks(int64_t R) { return (R + ACT_ROWS - 1) / ACT_ROWS; }

// Tiles of a product, and the parts its K axis is cut into where the tiles are fewer than the work-groups that the card
// runs: as many as fill it, a part having at least 256 terms (128 with the small tile).
// The widest tile reads least (24 KB for 512 matrix cycles of a unit's SIMD; 128 x 128 needs 16 KB for 256, as much as a
// unit gets from the cache), but takes many outputs: the others are for products that would leave units idle.
// Nor is one taken whose edges hold more than a third of outputs that there are not, against the next smaller one's (a
// training step of 25024 x 1792 x 55 float32 234 us with the small tile, 333 with 128 x 128; 30000 x 512 x 128 bf16 74 with
// 128 x 128, 83 with 128 x 256).
// A small product whose K axis would be cut is summed in one work-group a tile instead where the axis is short: bf16 (M x K x
// N) 64 x 256 x 1024 5.1 for 7.5 us, 64 x 1024 x 4096 8.4 for 14.1, 64 x 2048 x 2048 12.5 for 15.8, the weight gradient 256 x
// 2048 x 1024 8.4 for 12.9, but 64 x 4096 x 1024 20.4 for 19.2; float32, whose products take eight times the matrix cycles,
// 64 x 256 x 1024 9.1 for 9.8, but 16 x 512 x 2048 12.4 for 10.6.
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, size_t es, bool whole, bool wide) {
  LinearPlan p{};
  auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  auto parts = [&](int64_t least) { return whole || K < 2 * least ? 1 : K / least < 64 ? K / least : 64; };
  int64_t t, want, most = parts(256);
  if (es == 2 && wide && !whole && M > 64 && tiles(128, 256) * most >= 256 && 3 * tiles(128, 256) <= 2 * tiles(128, 128)) {
    p.tile = TILE_WIDE;
    t = tiles(128, 256);
    want = 256;
  } else if (M > 64 && tiles(128, 128) * most >= 256 && 3 * tiles(128, 128) <= tiles(64, 64)) {
    p.tile = TILE_SQUARE;
    t = tiles(128, 128);
    want = 256;
  } else {
    p.tile = TILE_SMALL;
    t = tiles(64, 64);
    want = 512;
    most = parts(128);
  }
  int64_t s = t > 0 ? want / t : 1;
  s = s < 1 ? 1 : s > most ? most : s;
  const int64_t kb = 64 / es, per = ((K + s - 1) / s + kb - 1) / kb * kb;  // whole steps, and no part without any
  p.splits = K > 0 ? (int)((K + per - 1) / per) : 0;
  if (p.tile == TILE_SMALL && p.splits > 1 && K * (int64_t)es <= (es == 2 ? 4096 : 1024)) {
    p.tile = TILE_DEEP;
    p.splits = 1;
  }
  return p;
}
int64_t linear_col_blocks(int tile, int64_t M) {
  const int64_t w = tile == TILE_WIDE ? 128 : tile == TILE_SQUARE ? 64 : 32;
  return (M + w - 1) / w;
}

template <typename T>
hipError_t launch_gemm(const GemmArgs& a, hipStream_t st) {
  if (a.splits > 0) {
    if (a.tile == TILE_WIDE) {
      if constexpr (sizeof(T) == 2) launch_tiles<T, 128, 256, 128, 64, 3, false>(a, st);
    } else if (a.tile == TILE_DEEP) {
      const dim3 grid((unsigned)(((a.M + 63) / 64) * ((a.N + 63) / 64)));
      if (!a.ak) gemm_deep_kernel<T, false, false><<<grid, 512, 0, st>>>(a);
      else if (a.bk) gemm_deep_kernel<T, true, true><<<grid, 512, 0, st>>>(a);
      else gemm_deep_kernel<T, true, false><<<grid, 512, 0, st>>>(a);
    } else if (a.tile == TILE_SQUARE) {
      launch_tiles<T, 128, 128, 64, 32, 4, true>(a, st);
    } else {
      launch_tiles<T, 64, 64, 32, 32, 6, true>(a, st);
    }
  }
  if (a.splits != 1) {
    // (a cut sum has fewer than 2^24 outputs; the zeros of an empty one may be more than a launch takes)
    const int64_t most = (LAUNCH_THREADS - 255) / a.N;
    for (int64_t m = 0; m < a.M; m += most) {
      GemmArgs b = a;
      b.M = a.M - m < most ? a.M - m : most;
      b.out = (T*)a.out + m * a.N;
      const int64_t n = b.M * a.N;
      if (!a.loose && a.N % 4 == 0)
        gemm_join_kernel<T, 4><<<dim3((unsigned)((n / 4 + 255) / 256)), 256, 0, st>>>(b);
      else
        gemm_join_kernel<T, 1><<<dim3((unsigned)((n + 255) / 256)), 256, 0, st>>>(b);
    }
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_pack(const void* src, int64_t ld, int64_t rows, int64_t cols, void* dst, int64_t to, hipStream_t st) {
  const int64_t per = to / (16 / (int64_t)sizeof(T)), most = (LAUNCH_THREADS - 255) / per;  // threads of a row, rows of a launch
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = rows - r < most ? rows - r : most;
    pack_kernel<T><<<dim3((unsigned)((n * per + 255) / 256)), 256, 0, st>>>((const T*)src + r * ld, ld, n, cols, (T*)dst + r * to, to);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_act_bwd(const void* dy, const float* pre, int act, void* out, int64_t to, float* part, int64_t R, int64_t N,
                          bool loose, hipStream_t st) {
  const bool four = !loose && N % 4 == 0;
  const int64_t cols = four ? (to + 255) / 256 : (to + 63) / 64, most = LAUNCH_THREADS / 256 / cols * ACT_ROWS;  // rows of a launch
  for (int64_t r = 0; r < R; r += most) {
    const int64_t n = R - r < most ? R - r : most;
    const dim3 grid((unsigned)(cols * linear_row_blocks(n)));
    const T* d = (const T*)dy + r * N;
    const float* p = pre != nullptr ? pre + r * N : nullptr;
    T* o = out != nullptr ? (T*)out + r * to : nullptr;
    float* s = part != nullptr ? part + r / ACT_ROWS * N : nullptr;
    if (four)
      act_bwd_kernel<T, 4><<<grid, 256, 0, st>>>(d, p, act, o, to, s, n, N);
    else
      act_bwd_kernel<T, 1><<<grid, 256, 0, st>>>(d, p, act, o, to, s, n, N);
  }
  return hipGetLastError();
}

hipError_t launch_col_sum(const float* part, int64_t blocks, int64_t N, float* db, hipStream_t st) {
  col_sum_kernel<<<dim3((unsigned)((N + 15) / 16)), 1024, 0, st>>>(part, blocks, N, db);
  return hipGetLastError();
}

#define RES_LINEAR(T)                                                                                                 \
  template hipError_t launch_gemm<T>(const GemmArgs&, hipStream_t);                                                   \
  template hipError_t launch_pack<T>(const void*, int64_t, int64_t, int64_t, void*, int64_t, hipStream_t);            \
  template hipError_t launch_act_bwd<T>(const void*, const float*, int, void*, int64_t, float*, int64_t, int64_t, bool, hipStream_t);
RES_LINEAR(float)
RES_LINEAR(bf16_t)

}  // namespace res
