// AdamW over many tensors in one launch:
//   g' = scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps).
// States are float32, or 8 bits in blocks of 256 elements: with S the block's largest
// |value|, m = sgn(c) (c / 127)^2 S for c in -127..127 and v = (c / 255)^4 S for c in
// 0..255 (a power law spends the codes on small sizes; a v that is not zero never gets
// code 0, since the step divides by its root).  The step itself uses the unrounded m and v.
//
// A wave takes one block of 256 elements, four consecutive ones a lane, so that a block's largest value is one reduction
// over the wave and every access 4 to 16 bytes a lane.  Memory bounds it: bfloat16 with float32 copies and states moves
// 28 bytes an element, 201 M of them in 994 to 1035 us on different cards (5.7 to 5.4 TB/s); float32 with float32 states 28
// bytes, 4.7 M in 22 us (out of the last cache); float32 with states of 8 bits 16 bytes, 80 M in 258 us (5.0 TB/s; 324 vector
// instructions a wave).
// Two blocks a wave and element 64 j + lane took 1026, 36 and 345 us.
#include "layer.h"

namespace res {
namespace {

constexpr int TABLE = 64;      // tensors of one launch (their table is a kernel argument)
constexpr int CHUNK_BLOCKS = 4;  // blocks of a work-group: one a wave (two: 1032 for 994 us with float32 copies)
constexpr int64_t CHUNK_ELEMS = (int64_t)CHUNK_BLOCKS * RES_ADAMW_BLOCK;
constexpr int64_t LAUNCH_CHUNKS = LAUNCH_THREADS / 256;
constexpr float TINY = 1e-30f;  // a smaller scale counts as zero (its reciprocal would leave float32)

struct Table {
  const void* p[TABLE];
  const void* g[TABLE];
  void* o[TABLE];
  int64_t n[TABLE];
  int64_t state[TABLE];
  uint32_t end[TABLE];  // chunks up to and with a tensor's last
  int count;
};

// The largest |value| of a wave's lanes; NaN is larger than infinity.
__device__ __forceinline__ float wave_absmax(const float (&f)[4]) {
  auto bits = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
  uint32_t x = max(max(bits(f[0]), bits(f[1])), max(bits(f[2]), bits(f[3])));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));   // lane ^ 1
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));   // lane ^ 2
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));  // 7 - lane of eight
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false));  // 15 - lane of sixteen
  uint32_t y = 0;
#pragma unroll
  for (int k = 0; k < 64; k += 16) y = max(y, (uint32_t)__builtin_amdgcn_readlane((int)x, k));
  return __uint_as_float(y);
}

__device__ __forceinline__ float value_m(int c, float s) {
#pragma clang fp contract(off)
  const float f = (float)c * (float)(1.0 / 127.0), f2 = f * f;
  return (f < 0.0f ? -f2 : f2) * s;
}
__device__ __forceinline__ float value_v(int c, float s) {
#pragma clang fp contract(off)
  const float f = (float)c * (float)(1.0 / 255.0), f2 = f * f;
  return (f2 * f2) * s;
}

// Codes are decided by correctly rounded operations (square roots, the reciprocal, no contraction), so that they do not
// depend on how a kernel is compiled.  The unit's own square root is within one unit in the last place; the two ways differ
// by less than 2^-13 before the rounding to 0..255.  Where that leaves no doubt to which whole number is rounded (all but
// one of two thousand), the correctly rounded ones, of four times the instructions, are not computed: 80 M elements 290 to 257 us.
__device__ __forceinline__ bool doubtful(float f) { return !(fabsf(fabsf(f - rintf(f)) - 0.5f) > 0x1p-12f); }
__device__ __forceinline__ void codes(float m, float v, float im, float iv, int* cm, int* cv) {
#pragma clang fp contract(off)
  const float xm = fabsf(m) * im, xv = v * iv;
  float fm = __builtin_amdgcn_sqrtf(xm) * 127.0f, fv = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(xv)) * 255.0f;
  if (__builtin_amdgcn_ballot_w64(doubtful(fm) || doubtful(fv)) != 0) {  // (a wave's branch: else both would be computed)
    fm = sqrtf(xm) * 127.0f;
    fv = sqrtf(sqrtf(xv)) * 255.0f;
  }
  *cm = (int)rintf(fm);
  *cv = (int)rintf(fv);
  if (m < 0.0f) *cm = -*cm;
  if (v > 0.0f && iv > 0.0f && *cv < 1) *cv = 1;
}

// The root of a second moment.  The unit's takes what is below 2^-126 for zero, by which a step with eps = 0 is divided.
__device__ __forceinline__ float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
  return small ? r * 0x1p-32f : r;
}

// A lane's four elements, one behind the other at the alignment of one: all of them (WHOLE), or the first `left`.
template <typename T> using Vec = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));
template <bool WHOLE, typename T>
__device__ __forceinline__ Vec<T> load_four(const T* from, int left) {
  Vec<T> r = {};
  if constexpr (WHOLE) {
    r = *reinterpret_cast<const Vec<T>*>(from);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) r[j] = from[j];
  }
  return r;
}
// (Stored past the caches, since what follows a step reads more than they hold: 54 tensors of together 4.7 M float32: 31 to 22 us.)
template <bool WHOLE, typename T>
__device__ __forceinline__ void store_four(T* to, Vec<T> v, int left) {
  if constexpr (WHOLE) {
    __builtin_nontemporal_store(v, reinterpret_cast<Vec<T>*>(to));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) to[j] = v[j];
  }
}

// One block: p, g and o are at this lane's elements, s is their place in the states.
template <bool WHOLE, typename TP, typename TG, int BITS, bool MASTER>
__device__ __forceinline__ void adamw_block(const AdamWArgs& a, float gs, const TP* p, const TG* g, TP* o, int64_t s, int left, int lane) {
  const int64_t sb = s / RES_ADAMW_BLOCK;
  const Vec<TG> gv = load_four<WHOLE>(g, left);
  float m[4], v[4], w[4];
  if constexpr (BITS == 8) {
    const Vec<int8_t> cm = load_four<WHOLE>((const int8_t*)a.m + s, left);
    const Vec<uint8_t> cv = load_four<WHOLE>((const uint8_t*)a.v + s, left);
    const float sm = a.sm[sb], sv = a.sv[sb];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = value_m(cm[j], sm);
      v[j] = value_v(cv[j], sv);
    }
  } else {
    const Vec<float> mv = load_four<WHOLE>((const float*)a.m + s, left), vv = load_four<WHOLE>((const float*)a.v + s, left);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = mv[j];
      v[j] = vv[j];
    }
  }
  if constexpr (MASTER) {
    const Vec<float> wv = load_four<WHOLE>(a.master + s, left);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = wv[j];
  } else {
    const Vec<TP> wv = load_four<WHOLE>(p, left);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = to_f32((TP)wv[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma clang fp contract(off)
    const float gr = to_f32((TG)gv[j]) * gs;
    m[j] = m[j] * a.b1 + gr * a.b1c;
    v[j] = v[j] * a.b2 + (gr * gr) * a.b2c;
    if (!WHOLE && j >= left) m[j] = v[j] = 0.0f;
  }
  float im = 0.0f, iv = 0.0f;
  if constexpr (BITS == 8) {
    const float sm = wave_absmax(m), sv = wave_absmax(v);
    im = sm >= TINY ? 1.0f / sm : 0.0f;
    iv = sv >= TINY ? 1.0f / sv : 0.0f;
    if (lane == 0) {
      a.sm_out[sb] = sm;
      a.sv_out[sb] = sv;
    }
  }
  Vec<TP> po;
  Vec<float> q;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float den = fmaf(root_of(v[j]), a.root, a.eps);
    // (a reciprocal within one unit in the last place: 2^-23 of the step, which is small beside the parameter)
    q[j] = fmaf(w[j], a.decay, -(a.step * m[j]) * __builtin_amdgcn_rcpf(den));
    po[j] = from_f32<TP>(q[j]);
  }
  store_four<WHOLE>(o, po, left);
  if constexpr (MASTER) store_four<WHOLE>(a.master_out + s, q, left);
  if constexpr (BITS == 8) {
    Vec<int8_t> cm;
    Vec<uint8_t> cv;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int c, d;
      codes(m[j], v[j], im, iv, &c, &d);
      cm[j] = (int8_t)c;
      cv[j] = (uint8_t)d;
    }
    store_four<WHOLE>((int8_t*)a.m_out + s, cm, left);
    store_four<WHOLE>((uint8_t*)a.v_out + s, cv, left);
  } else {
    store_four<WHOLE>((float*)a.m_out + s, Vec<float>{m[0], m[1], m[2], m[3]}, left);
    store_four<WHOLE>((float*)a.v_out + s, Vec<float>{v[0], v[1], v[2], v[3]}, left);
  }
}

template <typename TP, typename TG, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWArgs a, Table tab) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int k = 0;
  for (int hi = tab.count - 1; k < hi;) {  // the tensor of this chunk
    const int mid = (k + hi) >> 1;
    if (blockIdx.x < tab.end[mid]) hi = mid; else k = mid + 1;
  }
  const int64_t chunk = blockIdx.x - (k > 0 ? tab.end[k - 1] : 0u), n = tab.n[k];
  const TP* p = (const TP*)tab.p[k];
  const TG* g = (const TG*)tab.g[k];
  TP* o = (TP*)tab.o[k];
  const float gs = a.grad_scale != nullptr ? a.grad_scale[0] : 1.0f;
  const int64_t e0 = chunk * CHUNK_ELEMS + wave * RES_ADAMW_BLOCK, e = e0 + lane * 4, s = tab.state[k] + e;
  if (e0 + RES_ADAMW_BLOCK <= n)
    adamw_block<true, TP, TG, BITS, MASTER>(a, gs, p + e, g + e, o + e, s, 4, lane);
  else if (e0 < n)
    adamw_block<false, TP, TG, BITS, MASTER>(a, gs, p + e, g + e, o + e, s, (int)(e < n ? (n - e < 4 ? n - e : 4) : 0), lane);
}

// The values of codes, four a thread: 10 bytes an element, 80 M in 119 us (6.7 TB/s).
__global__ __launch_bounds__(256) void adamw_values_kernel(const int8_t* m, const uint8_t* v, const float* sm,
                                                           const float* sv, int64_t n, float* mo, float* vo) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e >= n) return;
  const int64_t b = e / RES_ADAMW_BLOCK;
  const char4 cm = *reinterpret_cast<const char4*>(m + e);
  const uchar4 cv = *reinterpret_cast<const uchar4*>(v + e);
  const float a = sm[b], c = sv[b];
  *reinterpret_cast<float4*>(mo + e) = make_float4(value_m(cm.x, a), value_m(cm.y, a), value_m(cm.z, a), value_m(cm.w, a));
  *reinterpret_cast<float4*>(vo + e) = make_float4(value_v(cv.x, c), value_v(cv.y, c), value_v(cv.z, c), value_v(cv.w, c));
}

template <typename TP, typename TG, int BITS, bool MASTER>
hipError_t launch_tables(const AdamWArgs& a, const res_adamw_tensor_t* t, int64_t count, hipStream_t st) {
  Table tab;
  tab.count = 0;
  uint64_t chunks = 0;
  auto flush = [&] {
    if (tab.count > 0) adamw_kernel<TP, TG, BITS, MASTER><<<dim3((unsigned)chunks), 256, 0, st>>>(a, tab);
    tab.count = 0;
    chunks = 0;
  };
  for (int64_t k = 0; k < count; ++k) {
    // a tensor of more chunks than a launch counts is taken in pieces
    for (int64_t at = 0; at < t[k].n;) {
      const int64_t most = (LAUNCH_CHUNKS - (int64_t)chunks) * CHUNK_ELEMS;
      const int64_t n = t[k].n - at < most ? t[k].n - at : most;
      const int c = tab.count++;
      tab.p[c] = (const TP*)t[k].p + at;
      tab.g[c] = (const TG*)t[k].g + at;
      tab.o[c] = (TP*)t[k].p_out + at;
      tab.n[c] = n;
      tab.state[c] = t[k].state + at;
      chunks += (n + CHUNK_ELEMS - 1) / CHUNK_ELEMS;
      tab.end[c] = (uint32_t)chunks;
      at += n;
      if (tab.count == TABLE || chunks >= (uint64_t)LAUNCH_CHUNKS) flush();
    }
  }
  flush();
  return hipGetLastError();
}

template <typename TP, typename TG>
hipError_t launch_bits(const AdamWArgs& a, const res_adamw_tensor_t* t, int64_t count, int bits, hipStream_t st) {
  if constexpr (sizeof(TP) == 2) {
    if (a.master != nullptr)
      return bits == 8 ? launch_tables<TP, TG, 8, true>(a, t, count, st) : launch_tables<TP, TG, 32, true>(a, t, count, st);
  }
  return bits == 8 ? launch_tables<TP, TG, 8, false>(a, t, count, st) : launch_tables<TP, TG, 32, false>(a, t, count, st);
}

}  // namespace

hipError_t launch_adamw(const AdamWArgs& a, const res_adamw_tensor_t* tensors, int64_t count, bool p_bf16, bool g_bf16,
                        int bits, hipStream_t st) {
  if (p_bf16)
    return g_bf16 ? launch_bits<bf16_t, bf16_t>(a, tensors, count, bits, st) : launch_bits<bf16_t, float>(a, tensors, count, bits, st);
  return g_bf16 ? launch_bits<float, bf16_t>(a, tensors, count, bits, st) : launch_bits<float, float>(a, tensors, count, bits, st);
}

hipError_t launch_adamw_values(const void* m, const void* v, const float* sm, const float* sv, int64_t n, float* mo,
                               float* vo, hipStream_t st) {
  const int64_t per = LAUNCH_CHUNKS * 1024;  // elements of a launch, four a thread
  for (int64_t at = 0; at < n; at += per) {
    const int64_t c = n - at < per ? n - at : per;
    adamw_values_kernel<<<dim3((unsigned)((c + 1023) / 1024)), 256, 0, st>>>(
        (const int8_t*)m + at, (const uint8_t*)v + at, sm + at / RES_ADAMW_BLOCK, sv + at / RES_ADAMW_BLOCK, c, mo + at, vo + at);
  }
  return hipGetLastError();
}

}  // namespace res
