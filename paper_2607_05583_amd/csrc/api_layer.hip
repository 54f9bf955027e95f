// C ABI of the gated recurrent layer's operators: argument checks and dispatch.
// Declared in include/resonator.h.
#include <algorithm>
#include <cstdint>

#include "../../include/resonator.h"
#include "layer.h"

using namespace res;

namespace {

size_t elt(res_dtype_t t) { return t == RES_BF16 ? 2 : 4; }
bool known(int t) { return t == RES_F32 || t == RES_BF16; }
bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? RES_OK : api_error(RES_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// The bytes that rows [B][L] of D elements of `es` bytes reach over, and whether two such sets share any.
struct Span {
  uintptr_t lo, hi;     // [lo, hi)
  int64_t sb, st, row;  // strides and row length in bytes
  int64_t B, L;
};
Span span(const void* p, int64_t sb, int64_t st, int64_t B, int64_t L, int64_t D, size_t es) {
  Span s{(uintptr_t)p, (uintptr_t)p, sb * (int64_t)es, st * (int64_t)es, D * (int64_t)es, B, L};
  if (p != nullptr && B > 0 && L > 0) s.hi += (B - 1) * s.sb + (L - 1) * s.st + s.row;
  return s;
}
Span flat(const void* p, size_t bytes) {
  return Span{(uintptr_t)p, (uintptr_t)p + (p != nullptr ? bytes : 0), (int64_t)bytes, (int64_t)bytes, (int64_t)bytes, 1, 1};
}
bool touch(const Span& a, const Span& b) {
  if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
  // columns of one wider tensor: the same strides, and columns that do not meet within a step
  if (a.st == b.st && a.st > 0 && (a.sb == b.sb || (a.B == 1 && b.B == 1)) && (a.B == 1 || a.sb % a.st == 0)) {
    const int64_t d = (((int64_t)(b.lo - a.lo)) % a.st + a.st) % a.st;  // b's first column after a's
    if (d >= a.row && d + b.row <= a.st) return false;
  }
  return true;
}
// whether the rows of an output lie apart from each other
bool rows_apart(int64_t sb, int64_t st, int64_t B, int64_t L, int64_t D) {
  if (B <= 1 && L <= 1) return true;
  if (B <= 1) return st >= D;
  if (L <= 1) return sb >= D;
  return (st >= D && sb >= (L - 1) * st + D) || (sb >= D && st >= (B - 1) * sb + D);
}

int check_rows(const char* name, const void* p, int64_t sb, int64_t st, size_t es) {
  if (p == nullptr) return api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name);
  if (!aligned(p, es)) return api_error(RES_ERR_MISALIGNED, "%s must be aligned to its element", name);
  if (sb < 0 || st < 0 || sb > (1LL << 40) || st > (1LL << 40))
    return api_error(RES_ERR_INVALID_ARG, "%s: strides must be in [0, 2^40] elements", name);
  return RES_OK;
}

int check_scan(int64_t B, int64_t L, int64_t D, res_dtype_t dt) {
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (B < 1 || D < 1 || L < 0)
    return api_error(RES_ERR_INVALID_ARG, "B and D must be >= 1 and L >= 0 (got B=%lld L=%lld D=%lld)", (long long)B,
                     (long long)L, (long long)D);
  const int64_t NB = (D + GATED_CW - 1) / GATED_CW;
  if (D > (1 << 24) || L >= (1LL << 31) - 65536 || B > (1LL << 31) || B * NB >= (1LL << 31))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (B=%lld L=%lld D=%lld)", (long long)B,
                     (long long)L, (long long)D);
  return RES_OK;
}
int check_f32(const char* name, const float* p, bool needed) {
  if (p == nullptr) return needed ? api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name) : RES_OK;
  return aligned(p, 4) ? RES_OK : api_error(RES_ERR_MISALIGNED, "%s must be 4-byte aligned", name);
}

constexpr int GATED_VEC = 4;
bool vec_rows(const void* p, int64_t sb, int64_t st, int64_t B, int64_t L, size_t es) {
  return aligned(p, GATED_VEC * es) && (B <= 1 || sb % GATED_VEC == 0) && (L <= 1 || st % GATED_VEC == 0);
}

}  // namespace

extern "C" {

size_t resonator_gated_scan_workspace_bytes(res_dtype_t dt, int64_t B, int64_t L, int64_t D) {
  if (check_scan(B, L, D, dt)) return 0;
  const int64_t NB = (D + GATED_CW - 1) / GATED_CW;
  return 256 + (size_t)B * NB * GATED_CW * 8;
}

int resonator_gated_scan_fwd(res_rows_t x, res_rows_t r, res_rows_t i, res_dtype_t dt, void* y, int64_t B, int64_t L,
                             int64_t D, const float* gamma, const float* h0, const int32_t* lengths, float* h_out,
                             float* carry, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_scan(B, L, D, dt);
  if (rc) return rc;
  const size_t es = elt(dt);
  if (L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, es)) || (rc = check_rows("r", r.p, r.sb, r.st, es)) ||
                (rc = check_rows("i", i.p, i.sb, i.st, es))))
    return rc;
  if ((rc = check_f32("gamma", gamma, true)) || (rc = check_f32("h0", h0, false)) ||
      (rc = check_f32("h_out", h_out, false)) || (rc = check_f32("carry", carry, false)))
    return rc;
  if (y == nullptr && h_out == nullptr && carry == nullptr)
    return api_error(RES_ERR_INVALID_ARG, "one of y, h_out and carry must be non-null");
  if (!aligned(y, es) || !aligned(lengths, 4))
    return api_error(RES_ERR_MISALIGNED, "y must be aligned to its element, lengths to 4 bytes");
  const size_t need = resonator_gated_scan_workspace_bytes(dt, B, L, D);
  if (ws == nullptr || ws_bytes < need)
    return api_error(RES_ERR_WORKSPACE, "workspace null or too small (%zu bytes, %zu needed)", ws_bytes, need);
  if (!aligned(ws, 256)) return api_error(RES_ERR_MISALIGNED, "the workspace must be 256-byte aligned");
  const int64_t NC = (L + GATED_CARRY - 1) / GATED_CARRY;
  const Span in[] = {span(x.p, x.sb, x.st, B, L, D, es), span(r.p, r.sb, r.st, B, L, D, es),
                     span(i.p, i.sb, i.st, B, L, D, es), flat(gamma, 4 * D), flat(lengths, 4 * B), flat(h0, 4 * B * D)};
  const Span out[] = {flat(y, es * B * L * D), flat(carry, 4 * B * NC * D), flat(ws, need), flat(h_out, 4 * B * D)};
  for (int o = 0; o < 4; ++o) {
    for (int k = 0; k < 6; ++k)
      if (touch(out[o], in[k]) && !(o == 3 && k == 5 && h_out == h0))
        return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs (h_out may be h0 itself)");
    for (int k = 0; k < o; ++k)
      if (touch(out[o], out[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  }
  GatedArgs a{};
  a.x = Rows{x.p, x.sb, x.st};
  a.r = Rows{r.p, r.sb, r.st};
  a.i = Rows{i.p, i.sb, i.st};
  a.y = y;
  a.B = B;
  a.L = L;
  a.D = (int)D;
  a.NB = (int)((D + GATED_CW - 1) / GATED_CW);
  a.vec = D % GATED_VEC == 0 && vec_rows(x.p, x.sb, x.st, B, L, es) && vec_rows(r.p, r.sb, r.st, B, L, es) &&
          vec_rows(i.p, i.sb, i.st, B, L, es) && vec_rows(y, 0, 0, 1, 1, es);
  a.gamma = gamma;
  a.h0 = h0;
  a.lengths = lengths;
  a.h_out = h_out;
  a.carry = carry;
  return launched(dt == RES_BF16 ? launch_gated_fwd<bf16_t>(a, (hipStream_t)stream) : launch_gated_fwd<float>(a, (hipStream_t)stream),
                  "gated scan launch");
}

int resonator_gated_scan_bwd(res_rows_t x, res_rows_t r, res_rows_t i, res_rows_t dy, res_dtype_t dt,
                             res_rows_out_t dx, res_rows_out_t dr, res_rows_out_t di, int64_t B, int64_t L, int64_t D,
                             const float* gamma, const float* carry, const int32_t* lengths, const float* dh_out,
                             float* dgamma, float* dh0, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_scan(B, L, D, dt);
  if (rc) return rc;
  const size_t es = elt(dt);
  if (L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, es)) || (rc = check_rows("r", r.p, r.sb, r.st, es)) ||
                (rc = check_rows("i", i.p, i.sb, i.st, es)) || (rc = check_rows("dy", dy.p, dy.sb, dy.st, es)) ||
                (rc = check_rows("dx", dx.p, dx.sb, dx.st, es)) || (rc = check_rows("dr", dr.p, dr.sb, dr.st, es)) ||
                (rc = check_rows("di", di.p, di.sb, di.st, es))))
    return rc;
  if ((rc = check_f32("gamma", gamma, true)) || (rc = check_f32("carry", carry, L > 0)) ||
      (rc = check_f32("dh_out", dh_out, false)) || (rc = check_f32("dgamma", dgamma, true)) ||
      (rc = check_f32("dh0", dh0, false)))
    return rc;
  if (!aligned(lengths, 4)) return api_error(RES_ERR_MISALIGNED, "lengths must be 4-byte aligned");
  const size_t need = resonator_gated_scan_workspace_bytes(dt, B, L, D);
  if (ws == nullptr || ws_bytes < need)
    return api_error(RES_ERR_WORKSPACE, "workspace null or too small (%zu bytes, %zu needed)", ws_bytes, need);
  if (!aligned(ws, 256)) return api_error(RES_ERR_MISALIGNED, "the workspace must be 256-byte aligned");
  const int64_t NC = (L + GATED_CARRY - 1) / GATED_CARRY;
  const Span in[] = {span(x.p, x.sb, x.st, B, L, D, es),    span(r.p, r.sb, r.st, B, L, D, es),
                     span(i.p, i.sb, i.st, B, L, D, es),    span(dy.p, dy.sb, dy.st, B, L, D, es),
                     flat(gamma, 4 * D),                    flat(lengths, 4 * B),
                     flat(carry, 4 * B * NC * D),           flat(dh_out, 4 * B * D)};
  const Span out[] = {span(dx.p, dx.sb, dx.st, B, L, D, es), span(dr.p, dr.sb, dr.st, B, L, D, es),
                      span(di.p, di.sb, di.st, B, L, D, es), flat(ws, need), flat(dgamma, 4 * D), flat(dh0, 4 * B * D)};
  for (int o = 0; o < 6; ++o) {
    for (const Span& s : in)
      if (touch(out[o], s)) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs");
    for (int k = 0; k < o; ++k)
      if (touch(out[o], out[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  }
  if (L > 0 && !(rows_apart(dx.sb, dx.st, B, L, D) && rows_apart(dr.sb, dr.st, B, L, D) && rows_apart(di.sb, di.st, B, L, D)))
    return api_error(RES_ERR_INVALID_ARG, "the rows of dx, dr and di must not overlap");
  GatedArgs a{};
  a.x = Rows{x.p, x.sb, x.st};
  a.r = Rows{r.p, r.sb, r.st};
  a.i = Rows{i.p, i.sb, i.st};
  a.dy = Rows{dy.p, dy.sb, dy.st};
  a.dx = RowsOut{dx.p, dx.sb, dx.st};
  a.dr = RowsOut{dr.p, dr.sb, dr.st};
  a.di = RowsOut{di.p, di.sb, di.st};
  a.B = B;
  a.L = L;
  a.D = (int)D;
  a.NB = (int)((D + GATED_CW - 1) / GATED_CW);
  a.vec = D % GATED_VEC == 0;
  for (const Rows& v : {a.x, a.r, a.i, a.dy}) a.vec = a.vec && vec_rows(v.p, v.sb, v.st, B, L, es);
  for (const RowsOut& v : {a.dx, a.dr, a.di}) a.vec = a.vec && vec_rows(v.p, v.sb, v.st, B, L, es);
  a.gamma = gamma;
  a.lengths = lengths;
  a.carry = const_cast<float*>(carry);
  a.dh_out = dh_out;
  a.dh0 = dh0;
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + 256);
  return launched(dt == RES_BF16 ? launch_gated_bwd<bf16_t>(a, dgamma, (hipStream_t)stream)
                                 : launch_gated_bwd<float>(a, dgamma, (hipStream_t)stream),
                  "gated scan backward launch");
}

int resonator_gated_scan_step(res_rows_t x, res_rows_t r, res_rows_t i, res_dtype_t dt, void* y, int64_t B, int64_t D,
                              const float* gamma, const float* h, float* h_out, void* stream) {
  int rc = check_scan(B, 1, D, dt);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((rc = check_rows("x", x.p, x.sb, x.st, es)) || (rc = check_rows("r", r.p, r.sb, r.st, es)) ||
      (rc = check_rows("i", i.p, i.sb, i.st, es)) || (rc = check_f32("gamma", gamma, true)) ||
      (rc = check_f32("h", h, true)) || (rc = check_f32("h_out", h_out, true)))
    return rc;
  if (y == nullptr) return api_error(RES_ERR_INVALID_ARG, "y must be non-null");
  if (!aligned(y, es)) return api_error(RES_ERR_MISALIGNED, "y must be aligned to its element");
  const Span in[] = {span(x.p, x.sb, 0, B, 1, D, es), span(r.p, r.sb, 0, B, 1, D, es), span(i.p, i.sb, 0, B, 1, D, es),
                     flat(gamma, 4 * D), flat(h, 4 * B * D)};
  const Span oy = flat(y, es * B * D), oh = flat(h_out, 4 * B * D);
  for (int k = 0; k < 5; ++k)
    if (touch(oy, in[k]) || (touch(oh, in[k]) && !(k == 4 && h == h_out)))
      return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs (h_out may be h itself)");
  if (touch(oy, oh)) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  const Rows rx{x.p, x.sb, 0}, rr{r.p, r.sb, 0}, ri{i.p, i.sb, 0};
  return launched(dt == RES_BF16 ? launch_gated_step<bf16_t>(rx, rr, ri, y, B, D, gamma, h, h_out, (hipStream_t)stream)
                                 : launch_gated_step<float>(rx, rr, ri, y, B, D, gamma, h, h_out, (hipStream_t)stream),
                  "gated scan step launch");
}

}  // extern "C"
