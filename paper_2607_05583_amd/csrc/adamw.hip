// AdamW over many tensors in one launch:
//   g' = scale g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps).
// States are float32, or 8 bits in blocks of 256 elements: with S the block's largest
// |value|, m = sgn(c) (c / 127)^2 S for c in -127..127 and v = (c / 255)^4 S for c in
// 0..255 (a power law spends the codes on small sizes; a v that is not zero never gets
// code 0, since the step divides by its root).  The step itself uses the unrounded m and v.
//
// A wave takes blocks of 256 elements, four a lane, so that a block's largest value is
// one reduction over the wave.
#include "layer.h"

namespace res {
namespace {

constexpr int TABLE = 64;      // tensors of one launch (their table is a kernel argument)
constexpr int CHUNK_BLOCKS = 8;  // blocks of a work-group: two a wave
constexpr int64_t CHUNK_ELEMS = (int64_t)CHUNK_BLOCKS * RES_ADAMW_BLOCK;
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
__device__ __forceinline__ float wave_absmax(float a, float b, float c, float d) {
  auto bits = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
  uint32_t x = max(max(bits(a), bits(b)), max(bits(c), bits(d)));
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) x = max(x, (uint32_t)__shfl_xor((int)x, k, 64));
  return __uint_as_float(x);
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

// Codes are decided by correctly rounded operations (square roots, the reciprocal, no
// contraction), so that they do not depend on how a kernel is compiled.
__device__ __forceinline__ int code_m(float m, float inv) {
#pragma clang fp contract(off)
  const int c = (int)rintf(sqrtf(fabsf(m) * inv) * 127.0f);
  return m < 0.0f ? -c : c;
}
__device__ __forceinline__ int code_v(float v, float inv) {
#pragma clang fp contract(off)
  const int c = (int)rintf(sqrtf(sqrtf(v * inv)) * 255.0f);
  return v > 0.0f && inv > 0.0f && c < 1 ? 1 : c;
}

template <typename TP, typename TG, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWArgs a, Table tab) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
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
  for (int blk = wave; blk < CHUNK_BLOCKS; blk += 4) {
    const int64_t e0 = chunk * CHUNK_ELEMS + blk * RES_ADAMW_BLOCK, s0 = tab.state[k] + e0;
    if (e0 >= n) break;
    const int64_t sb = s0 / RES_ADAMW_BLOCK;
    float m[4], v[4], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t e = e0 + j * 64 + lane, s = s0 + j * 64 + lane;
      m[j] = v[j] = w[j] = 0.0f;
      if (e < n) {
#pragma clang fp contract(off)
        const float gr = to_f32(g[e]) * gs;
        float mo, vo;
        if constexpr (BITS == 8) {
          mo = value_m(((const int8_t*)a.m)[s], a.sm[sb]);
          vo = value_v(((const uint8_t*)a.v)[s], a.sv[sb]);
        } else {
          mo = ((const float*)a.m)[s];
          vo = ((const float*)a.v)[s];
        }
        m[j] = mo * a.b1 + gr * a.b1c;
        v[j] = vo * a.b2 + (gr * gr) * a.b2c;
        w[j] = MASTER ? a.master[s] : to_f32(p[e]);
      }
    }
    float im = 0.0f, iv = 0.0f;
    if constexpr (BITS == 8) {
      const float sm = wave_absmax(m[0], m[1], m[2], m[3]), sv = wave_absmax(v[0], v[1], v[2], v[3]);
      im = sm >= TINY ? 1.0f / sm : 0.0f;
      iv = sv >= TINY ? 1.0f / sv : 0.0f;
      if (lane == 0) {
        a.sm_out[sb] = sm;
        a.sv_out[sb] = sv;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t e = e0 + j * 64 + lane, s = s0 + j * 64 + lane;
      if (e >= n) continue;
      const float den = fmaf(__builtin_amdgcn_sqrtf(v[j]), a.root, a.eps);
      const float q = fmaf(w[j], a.decay, -(a.step * m[j]) / den);
      if constexpr (MASTER) a.master_out[s] = q;
      o[e] = from_f32<TP>(q);
      if constexpr (BITS == 8) {
        ((int8_t*)a.m_out)[s] = (int8_t)code_m(m[j], im);
        ((uint8_t*)a.v_out)[s] = (uint8_t)code_v(v[j], iv);
      } else {
        ((float*)a.m_out)[s] = m[j];
        ((float*)a.v_out)[s] = v[j];
      }
    }
  }
}

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
      const int64_t most = ((1LL << 30) - (int64_t)chunks) * CHUNK_ELEMS;
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
      if (tab.count == TABLE || chunks >= (1ULL << 30)) flush();
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
  const int64_t per = 1LL << 40;  // (n / 1024 work-groups)
  for (int64_t at = 0; at < n; at += per) {
    const int64_t c = n - at < per ? n - at : per;
    adamw_values_kernel<<<dim3((unsigned)((c + 1023) / 1024)), 256, 0, st>>>(
        (const int8_t*)m + at, (const uint8_t*)v + at, sm + at / RES_ADAMW_BLOCK, sv + at / RES_ADAMW_BLOCK, c, mo + at, vo + at);
  }
  return hipGetLastError();
}

}  // namespace res
