// Linear product with bias, activation and residual, and its gradients:
//   pre = x W + b, y = act(pre) + residual;
//   dpre = dy act'(pre), dx = dpre W^T, dW = x^T dpre, db = sum over rows of dpre.
// All three products are one kernel over strided operands; sums are float32 (MFMA).
#include "layer.h"
#include "stream.h"

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

template <typename T> struct __align__(4 * sizeof(T)) Quad { T v[4]; };
__device__ __forceinline__ Quad<float> round_quad(const f4& c, float) { return __builtin_bit_cast(Quad<float>, c); }
__device__ __forceinline__ Quad<bf16_t> round_quad(const f4& c, bf16_t) {
  typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(Quad<bf16_t>, __builtin_convertvector(c, bf4));
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


// ---------------------------------------------------------------------------
// Tiles of BM x BN outputs for 16-byte aligned operands.  A wave owns WM x WN of
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

// Loads an operand's tile: rows x0.. of X and KB elements of the K axis.  KC: element (x, k) at p[x ld + k], else at
// p[k ld + x].  A lane's byte offsets from the tile's start do not change along K (only the scalar base does), and
// rows past the end are the last ones again: what they give is not stored.
template <typename T, int BX, int NW, bool KC> struct TileLoad {
  static constexpr int ES = sizeof(T), EP = 16 / ES, RB = KC ? 64 : BX * ES, PR = RB / 16, RU = 1024 / RB;
  static constexpr int UNITS = BX / 16 / NW;
  static_assert(BX % (16 * NW) == 0 && RB <= 1024, "whole units of a kilobyte for each wave");
  uint32_t off[UNITS];
  const char* start;  // the tile's first element at k = 0
  int64_t step;       // bytes of an element along K

  __device__ static __forceinline__ int row_of(int u, int wave, int lane) { return (wave * UNITS + u) * RU + lane / PR; }
  __device__ static __forceinline__ int piece_of(int row, int lane) {
    const int slot = lane % PR;
    if constexpr (KC) return slot ^ ((row >> 2) & 3);
    if constexpr (ES == 2) return slot ^ (((row & 3) | ((row >> 1) & 4)) << 1);
    return slot ^ (((row >> 2) & 3) << 2);
  }
  __device__ __forceinline__ void open(const T* p, int64_t ld, int64_t x0, int64_t X, int wave, int lane) {
    start = (const char*)(p + x0 * (KC ? ld : 1));
    step = (KC ? 1 : ld) * ES;
    const int64_t left = X - x0;
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int row = row_of(u, wave, lane), piece = piece_of(row, lane);
      if constexpr (KC)
        off[u] = (uint32_t)((row < left ? row : left - 1) * ld * ES + piece * 16);
      else
        off[u] = (uint32_t)(row * ld * ES + (piece * EP < left ? piece * EP : left - EP) * ES);
    }
  }
  // K elements k .. k + KB - 1, those from kend on as zeros
  __device__ __forceinline__ void operator()(int64_t k, int64_t kend, char* lds, int wave, int lane) const {
    const char* base = uniform(start + k * step);
    if (k + Gemm<T>::KB <= kend) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) lds_dma16(base, off[u], lds + (wave * UNITS + u) * 1024);
    } else {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int row = row_of(u, wave, lane), piece = piece_of(row, lane);
        const void* src = k + (KC ? piece * EP : row) < kend ? (const void*)(base + off[u]) : (const void*)zero_piece;
        lds_dma16_lane(src, lds + (wave * UNITS + u) * 1024);
      }
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
    const int row = 8 * lq + (li >> 2), f = (li >> 2) | ((lq & 1) << 2);
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

// A wave's outputs through its own part of the LDS, 16 rows at a time (16-byte piece p of row m in slot p ^ (m & 7)), so that they are stored as whole rows of 128 (bf16) or 256 bytes: the results' own layout
// gives 32-byte pieces.  Rows and columns past the end are computed from the last ones' operands and not stored.
template <typename T, int ACT, int WM, int WN>
__device__ __forceinline__ void tile_out(const GemmArgs& g, int64_t m0, int64_t n0, const f4 (&acc)[WM / 16][WN / 16],
                                         char* mine, int lane) {
  constexpr int ES = sizeof(T), RB = WN * ES, PR = RB / 16, EP = 16 / ES, SW = PR < 8 ? PR - 1 : 7, FN = WN / 16;
  const int li = lane & 15, lq = lane >> 4;
  int64_t n[FN];
  f4 bias[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    n[j] = n0 + j * 16 + lq * 4;
    n[j] = n[j] < g.N ? n[j] : g.N - 4;
    bias[j] = g.bias != nullptr ? *reinterpret_cast<const f4*>(g.bias + n[j]) : f4{};
  }
#pragma unroll
  for (int i = 0; i < WM / 16; ++i) {
    int64_t m = m0 + i * 16 + li;
    const bool in = m < g.M;
    m = in ? m : g.M - 1;
    f4 c[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) c[j] = acc[i][j] + bias[j];
    if (g.pre != nullptr && in) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
        if (n0 + j * 16 + lq * 4 < g.N) *reinterpret_cast<f4*>(g.pre + m * g.N + n[j]) = c[j];
    }
    if constexpr (ACT != ACT_NONE) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) c[j][r] = act_value(c[j][r], ACT);
    }
    if (g.res != nullptr) {
      Quad<T> q[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) q[j] = *reinterpret_cast<const Quad<T>*>((const T*)g.res + m * g.N + n[j]);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) c[j][r] += to_f32(q[j].v[r]);
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int byte = (j * 16 + lq * 4) * ES;
      *reinterpret_cast<Quad<T>*>(mine + li * RB + (((byte >> 4) ^ (li & SW)) << 4) + (byte & 15)) = round_quad(c[j], T());
    }
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int u = 0; u < 16 * PR / 64; ++u) {
      const int row = u * (64 / PR) + lane / PR, slot = lane % PR;
      const int64_t m = m0 + i * 16 + row, col = n0 + ((slot ^ (row & SW)) * EP);
      const u4 v = *reinterpret_cast<const u4*>(mine + row * RB + slot * 16);
      if (m < g.M && col < g.N) __builtin_nontemporal_store(v, reinterpret_cast<u4*>((T*)g.out + m * g.N + col));
    }
  }
}

// Work-groups stay: each takes every gridDim-th item (a tile and a part of the K axis), and the loads run NB - 1 steps
// ahead of the products over the borders of the items, so that neither an item's first loads nor its stores are waited
// for.  NB buffers of a step and the LDS of each wave's outputs.
template <typename T, int BM, int BN, int WM, int WN, int NB, int OCC, bool AK, bool BK>
__global__ __launch_bounds__(64 * (BM / WM) * (BN / WN), OCC) void gemm_tile_kernel(GemmArgs g) {
  constexpr int NW = (BM / WM) * (BN / WN), KB = Gemm<T>::KB, FM = WM / 16, FN = WN / 16, STEP = (BM + BN) * 64;
  __shared__ __align__(1024) char lds[NB * STEP + NW * out_lds<T, WN>()];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, lq = lane >> 4;
  const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;
  const uint32_t mt = (uint32_t)((g.M + BM - 1) / BM), nt = (uint32_t)((g.N + BN - 1) / BN), tiles = mt * nt, items = tiles * g.splits;
  const int64_t per = ((g.K + g.splits - 1) / g.splits + KB - 1) / KB * KB;  // (no part is empty: see linear_plan)
  typedef TileLoad<T, BM, NW, AK> LoadA;
  typedef TileLoad<T, BN, NW, BK> LoadB;
  constexpr int UNITS = LoadA::UNITS + LoadB::UNITS;  // loads of a step by one wave

  // the next step to load: item, and where in its part of the K axis
  LoadA load_a;
  LoadB load_b;
  uint32_t next = blockIdx.x;
  int64_t nk = 0, nk1 = 0;
  auto open = [&] {
    int64_t tm, tn;
    const uint32_t part = next / tiles;
    tile_of(next - part * tiles, mt, nt, &tm, &tn);
    nk = part * per;
    nk1 = nk + per < g.K ? nk + per : g.K;
    load_a.open((const T*)g.A, AK ? g.sam : g.sak, tm * BM, g.M, wave, lane);
    load_b.open((const T*)g.B, BK ? g.sbn : g.sbk, tn * BN, g.N, wave, lane);
  };
  int ahead = 0;  // steps loaded or on their way that are not multiplied yet
  auto prefetch = [&](int buf) {
    if (next >= items) return;
    load_a(nk, nk1, lds + buf * STEP, wave, lane);
    load_b(nk, nk1, lds + buf * STEP + BM * 64, wave, lane);
    ++ahead;
    nk += KB;
    if (nk >= nk1) {
      next += gridDim.x;
      if (next < items) open();
    }
  };
  open();
#pragma unroll
  for (int b = 0; b < NB - 1; ++b) prefetch(b);

  int buf = 0;
  bool waited = false;
  for (uint32_t item = blockIdx.x; item < items; item += gridDim.x) {
    int64_t tm, tn;
    const uint32_t part = item / tiles;
    tile_of(item - part * tiles, mt, nt, &tm, &tn);
    const int64_t m0 = tm * BM, n0 = tn * BN, k0 = part * per, k1 = k0 + per < g.K ? k0 + per : g.K;
    f4 acc[FM][FN] = {};
    for (int64_t k = k0; k < k1; k += KB) {
      // this wave's pieces of the step are there (loads arrive in order), and past the barrier everyone's; the buffer of
      // the step before has been read by all
      if (!waited) {
        if (ahead >= NB - 1) wait_vm<(NB - 2) * UNITS>(); else wait_vm<0>();
      }
      waited = false;
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      prefetch(buf == 0 ? NB - 1 : buf - 1);
      const char* la = lds + buf * STEP;
      const char* lb = la + BM * 64;
      typename Gemm<T>::Frag fb[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = fragment<T, BN, BK>(lb, wn + j * 16, li, lq);
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const auto fa = fragment<T, BM, AK>(la, wm + i * 16, li, lq);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          if constexpr (sizeof(T) == 2)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa, acc[i][j], 0, 0, 0);
          else
            acc[i][j] = mma_f32(fb[j], fa, acc[i][j]);
        }
      }
      --ahead;
      buf = buf == NB - 1 ? 0 : buf + 1;
    }
    // the next step's loads are waited for before the stores are issued, so that no step waits for the stores
    if (ahead >= NB - 1) wait_vm<(NB - 2) * UNITS>(); else wait_vm<0>();
    waited = true;
    if (g.splits > 1) {
      float* o = g.part + part * g.M * g.N;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + wm + i * 16 + li;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const int64_t n = n0 + wn + j * 16 + lq * 4;
          if (m < g.M && n < g.N) *reinterpret_cast<f4*>(o + m * g.N + n) = acc[i][j];
        }
      }
      continue;
    }
    char* mine = lds + NB * STEP + wave * out_lds<T, WN>();
    switch (g.act) {
      case ACT_RELU: tile_out<T, ACT_RELU, WM, WN>(g, m0 + wm, n0 + wn, acc, mine, lane); break;
      case ACT_SILU: tile_out<T, ACT_SILU, WM, WN>(g, m0 + wm, n0 + wn, acc, mine, lane); break;
      case ACT_GELU_TANH: tile_out<T, ACT_GELU_TANH, WM, WN>(g, m0 + wm, n0 + wn, acc, mine, lane); break;
      default: tile_out<T, ACT_NONE, WM, WN>(g, m0 + wm, n0 + wn, acc, mine, lane);
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

// Tiles of a product, and the parts its K axis is cut into where they are fewer than
// the compute units: as many as fill them, a part having at least 256 terms.
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, size_t es, bool fast) {
  LinearPlan p{};
  auto tiles = [&](int b) { return ((M + b - 1) / b) * ((N + b - 1) / b); };
  p.tile = !fast ? 64 : es == 2 && tiles(256) >= 256 ? 256 : 128;
  const int64_t t = tiles(p.tile), want = fast ? 256 : 512;
  int64_t s = t > 0 ? want / t : 1;
  if (s > K / 256) s = K / 256;
  s = s < 1 ? 1 : s > 64 ? 64 : s;
  const int64_t kb = 64 / es, per = ((K + s - 1) / s + kb - 1) / kb * kb;  // whole steps, and no part without any
  p.splits = per > 0 ? (int)((K + per - 1) / per) : 1;
  return p;
}

namespace {
template <typename T, int BM, int BN, int WM, int WN, int NB, int OCC>
void launch_tiles(const GemmArgs& a, hipStream_t st) {
  const int64_t items = ((a.M + BM - 1) / BM) * ((a.N + BN - 1) / BN) * a.splits;
  const dim3 grid((unsigned)(items < 512 ? items : 512));  // (two work-groups on each of 256 compute units)
  constexpr int NT = 64 * (BM / WM) * (BN / WN);
  if (a.sak == 1 && a.sbk == 1)
    gemm_tile_kernel<T, BM, BN, WM, WN, NB, OCC, true, true><<<grid, NT, 0, st>>>(a);
  else if (a.sak == 1)
    gemm_tile_kernel<T, BM, BN, WM, WN, NB, OCC, true, false><<<grid, NT, 0, st>>>(a);
  else
    gemm_tile_kernel<T, BM, BN, WM, WN, NB, OCC, false, false><<<grid, NT, 0, st>>>(a);
}
}  // namespace

template <typename T>
hipError_t launch_gemm(const GemmArgs& a, hipStream_t st) {
  if (a.tile == 256) {
    if constexpr (sizeof(T) == 2) launch_tiles<T, 128, 256, 128, 64, 3, 2>(a, st);
  } else if (a.tile == 128) {
    launch_tiles<T, 128, 128, 64, 64, 4, 2>(a, st);
  } else {
    const int64_t tiles = ((a.M + 63) / 64) * ((a.N + 63) / 64);
    gemm_any_kernel<T><<<dim3((unsigned)tiles, (unsigned)a.splits), 256, 0, st>>>(a);
  }
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
