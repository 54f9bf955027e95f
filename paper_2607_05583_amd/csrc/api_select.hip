// C ABI of the selective layer's operators and of the token probabilities: argument checks and dispatch.
// Declared in include/resonator.h.
#include <cstdint>

#include "../../include/resonator.h"
#include "api_check.h"
#include "select.h"

using namespace res;

namespace {

Rows rows_of(const res_rows_t& r, int64_t L) { return Rows{r.p, r.sb, L > 1 ? r.st : 0}; }
RowsOut rows_of(const res_rows_out_t& r, int64_t L) { return RowsOut{r.p, r.sb, L > 1 ? r.st : 0}; }
Span span(const res_rows_t& r, int64_t B, int64_t L, int64_t D, size_t es) { return res::span(r.p, r.sb, r.st, B, L, D, es); }
Span span(const res_rows_out_t& r, int64_t B, int64_t L, int64_t D, size_t es) { return res::span(r.p, r.sb, r.st, B, L, D, es); }

// Whether an output meets an input or another output; `same`: an output that may be the input itself.
struct Same {
  int out, in;
};
template <int NI, int NO>
int check_apart(const Span (&in)[NI], const Span (&out)[NO], Same same, const char* named) {
  for (int o = 0; o < NO; ++o) {
    for (int k = 0; k < NI; ++k) {
      const bool it = o == same.out && k == same.in && in[k].lo == out[o].lo && in[k].hi == out[o].hi;
      if (!it && touch(out[o], in[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs%s", named);
    }
    for (int k = 0; k < o; ++k)
      if (touch(out[o], out[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  }
  return RES_OK;
}
int check_elt(const char* name, const void* p, bool needed, size_t es) {
  if (p == nullptr) return needed ? api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name) : RES_OK;
  return aligned(p, es) ? RES_OK : api_error(RES_ERR_MISALIGNED, "%s must be aligned to its element", name);
}
int check_ws(const void* ws, size_t have, size_t need) {
  if (need > 0 && (ws == nullptr || have < need))
    return api_error(RES_ERR_WORKSPACE, "workspace null or too small (%zu bytes, %zu needed)", have, need);
  return need == 0 || aligned(ws, 256) ? RES_OK : api_error(RES_ERR_MISALIGNED, "the workspace must be 256-byte aligned");
}
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

// ---------------------------------------------------------------------------
// Short causal convolution
// ---------------------------------------------------------------------------
int check_conv(int64_t B, int64_t L, int64_t D, int64_t K, res_dtype_t dt, int act) {
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (act < RES_ACT_NONE || act > RES_ACT_GELU_TANH) return api_error(RES_ERR_INVALID_ARG, "unknown activation code %d", act);
  if (B < 1 || D < 1 || L < 0 || K < 1)
    return api_error(RES_ERR_INVALID_ARG, "B, D and K must be >= 1 and L >= 0 (got B=%lld L=%lld D=%lld K=%lld)", (long long)B,
                     (long long)L, (long long)D, (long long)K);
  // (A row's threads fit one launch, here counted with tiles of the most steps.  A call takes shorter ones only while its work-groups are
  // fewer than CONV_ENOUGH, so that it has no more than twice as many.)
  if (K > CONV_TAPS || D > (1 << 21) || B > (1LL << 31) || L >= (1LL << 31) - 65536 || (L / (1 << CONV_SHIFT) + 1) * ((D + 1) / 2) >= (1LL << 31) ||
      B * (L / (1 << CONV_BWD_SHIFT) + 1) >= (1LL << 40))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (B=%lld L=%lld D=%lld K=%lld)", (long long)B,
                     (long long)L, (long long)D, (long long)K);
  return RES_OK;
}

}  // namespace

extern "C" {

int resonator_short_conv_fwd(res_rows_t x, res_dtype_t dt, const float* w, const float* bias, int act, int64_t K,
                             const void* state, const int32_t* lengths, void* y, void* state_out, int64_t B, int64_t L,
                             int64_t D, void* stream) {
  int rc = check_conv(B, L, D, K, dt, act);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((L > 0 && (rc = check_rows("x", x.p, x.sb, x.st, L, es))) || (rc = check_f32("w", w, true)) ||
      (rc = check_f32("bias", bias, false)) || (rc = check_elt("state", state, false, es)) ||
      (rc = check_elt("lengths", lengths, false, 4)) || (rc = check_elt("y", y, L > 0, es)) ||
      (rc = check_elt("state_out", state_out, false, es)))
    return rc;
  const size_t sb = es * B * (K - 1) * D;
  const Span in[] = {span(x, B, L, D, es), flat(w, 4 * D * K), flat(bias, 4 * D), flat(lengths, 4 * B), flat(state, sb)};
  const Span out[] = {flat(y, es * B * L * D), flat(state_out, sb)};
  if ((rc = check_apart(in, out, Same{1, 4}, " (state_out may be state itself)"))) return rc;
  ConvArgs a{};
  a.x = rows_of(x, L);
  a.w = w;
  a.bias = bias;
  a.state = state;
  a.lengths = lengths;
  a.y = y;
  a.state_out = K > 1 ? state_out : nullptr;
  a.B = B;
  a.L = L;
  a.D = D;
  a.K = (int)K;
  a.act = act;
  return launched(dt == RES_BF16 ? launch_conv_fwd<bf16_t>(a, (hipStream_t)stream) : launch_conv_fwd<float>(a, (hipStream_t)stream),
                  "short convolution launch");
}

size_t resonator_short_conv_workspace_bytes(int64_t B, int64_t L, int64_t D, int64_t K) {
  if (check_conv(B, L, D, K, RES_F32, RES_ACT_NONE)) return 0;
  return up256((size_t)conv_part_floats(B, L, D, K) * 4);
}

int resonator_short_conv_bwd(res_rows_t x, res_rows_t dy, res_dtype_t dt, const float* w, const float* bias, int act,
                             int64_t K, const void* state, const int32_t* lengths, const void* dstate_out,
                             res_rows_out_t dx, float* dw, float* dbias, void* dstate, int64_t B, int64_t L, int64_t D,
                             void* ws, size_t ws_bytes, void* stream) {
  int rc = check_conv(B, L, D, K, dt, act);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, L, es)) || (rc = check_rows("dy", dy.p, dy.sb, dy.st, L, es)) ||
                 (rc = check_rows("dx", dx.p, dx.sb, dx.st, L, es)))) ||
      (rc = check_f32("w", w, true)) || (rc = check_f32("bias", bias, false)) || (rc = check_elt("state", state, false, es)) ||
      (rc = check_elt("lengths", lengths, false, 4)) || (rc = check_elt("dstate_out", dstate_out, false, es)) ||
      (rc = check_f32("dw", dw, true)) || (rc = check_f32("dbias", dbias, false)) || (rc = check_elt("dstate", dstate, false, es)))
    return rc;
  const size_t need = resonator_short_conv_workspace_bytes(B, L, D, K);
  if ((rc = check_ws(ws, ws_bytes, need))) return rc;
  const size_t sb = es * B * (K - 1) * D;
  const Span in[] = {span(x, B, L, D, es),  span(dy, B, L, D, es), flat(w, 4 * D * K),   flat(bias, 4 * D),
                     flat(lengths, 4 * B), flat(state, sb),       flat(dstate_out, sb)};
  const Span out[] = {span(dx, B, L, D, es), flat(dw, 4 * D * K), flat(dbias, 4 * D), flat(dstate, sb), flat(ws, need)};
  if ((rc = check_apart(in, out, Same{-1, -1}, ""))) return rc;
  if (L > 0 && !rows_apart(dx.sb, dx.st, B, L, D)) return api_error(RES_ERR_INVALID_ARG, "the rows of dx must not overlap");
  ConvArgs a{};
  a.x = rows_of(x, L);
  a.dy = rows_of(dy, L);
  a.dx = rows_of(dx, L);
  a.w = w;
  a.bias = bias;
  a.state = state;
  a.lengths = lengths;
  a.dstate_out = K > 1 ? dstate_out : nullptr;
  a.dstate = K > 1 ? dstate : nullptr;
  a.part = static_cast<float*>(ws);
  a.dw = dw;
  a.dbias = dbias;
  a.B = B;
  a.L = L;
  a.D = D;
  a.K = (int)K;
  a.act = act;
  return launched(dt == RES_BF16 ? launch_conv_bwd<bf16_t>(a, (hipStream_t)stream) : launch_conv_bwd<float>(a, (hipStream_t)stream),
                  "short convolution backward launch");
}

int resonator_short_conv_step(res_rows_t x, res_dtype_t dt, const float* w, const float* bias, int act, int64_t K,
                              const void* state, void* y, void* state_out, int64_t B, int64_t D, void* stream) {
  int rc = check_conv(B, 1, D, K, dt, act);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((rc = check_rows("x", x.p, x.sb, 0, 1, es)) || (rc = check_f32("w", w, true)) || (rc = check_f32("bias", bias, false)) ||
      (rc = check_elt("state", state, K > 1, es)) || (rc = check_elt("y", y, true, es)) ||
      (rc = check_elt("state_out", state_out, K > 1, es)))
    return rc;
  const size_t sb = es * B * (K - 1) * D;
  const Span in[] = {span(x, B, 1, D, es), flat(w, 4 * D * K), flat(bias, 4 * D), flat(state, sb)};
  const Span out[] = {flat(y, es * B * D), flat(state_out, sb)};
  if ((rc = check_apart(in, out, Same{1, 3}, " (state_out may be state itself)"))) return rc;
  ConvArgs a{};
  a.x = rows_of(x, 1);
  a.w = w;
  a.bias = bias;
  a.state = state;
  a.y = y;
  a.state_out = state_out;
  a.B = B;
  a.L = 1;
  a.D = D;
  a.K = (int)K;
  a.act = act;
  return launched(dt == RES_BF16 ? launch_conv_step<bf16_t>(a, (hipStream_t)stream) : launch_conv_step<float>(a, (hipStream_t)stream),
                  "short convolution step launch");
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Selective scan
// ---------------------------------------------------------------------------
namespace {

struct Sizes {
  int64_t B, L, H, P, G, N;
};
int check_selective(const Sizes& z, res_dtype_t dt) {
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (z.B < 1 || z.L < 0 || z.H < 1 || z.P < 1 || z.G < 1 || z.N < 1 || z.H % z.G != 0)
    return api_error(RES_ERR_INVALID_ARG, "B, H, P, G and N must be >= 1, L >= 0 and G divide H (got B=%lld L=%lld H=%lld P=%lld G=%lld N=%lld)",
                     (long long)z.B, (long long)z.L, (long long)z.H, (long long)z.P, (long long)z.G, (long long)z.N);
  // (work-groups are 32-bit counts)
  if (z.P > SEL_MAX || z.N > SEL_MAX || z.H > (1 << 16) || z.H * z.P > (1 << 21) || z.G * z.N > (1 << 21) || z.B > (1LL << 31) ||
      z.L >= (1LL << 31) - 65536 || z.B * z.H >= (1LL << 29) || z.B * z.H * (z.L / SEL_Q + 1) >= (1LL << 40))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (B=%lld L=%lld H=%lld P=%lld G=%lld N=%lld)", (long long)z.B,
                     (long long)z.L, (long long)z.H, (long long)z.P, (long long)z.G, (long long)z.N);
  return RES_OK;
}
SelPlan plan_of(const Sizes& z, res_dtype_t dt) { return sel_plan(dt == RES_BF16, z.B, z.L, z.H, z.P, z.G, z.N); }
// floats of the states at the segments' borders
size_t border_floats(const Sizes& z, const SelPlan& p) { return p.segs > 1 ? (size_t)(z.B * p.HV * p.segs) * SEL_P * 16 * p.NT : 0; }

// The workspace's pieces; with a null base it only counts.
size_t lay_out(const Sizes& z, bool backward, bool carry, char* base, SelArgs* a) {
  const SelPlan& p = a->p;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* q = base != nullptr && bytes > 0 ? base + off : nullptr;
    off += up256(bytes);
    return q;
  };
  a->decay = (float*)take(p.segs > 1 ? (size_t)(z.B * p.HV * p.segs) * 4 : 0);
  float* border = (float*)take(backward || !carry ? border_floats(z, p) * 4 : 0);
  if (!backward) {
    if (border != nullptr) a->enter = border;
    return off;
  }
  a->leave = border;
  const size_t wgs = (size_t)(z.B * p.segs * z.G * ((p.HG + p.HR - 1) / p.HR)), state = (size_t)p.HR * SEL_P * 16 * p.NT * 4;
  a->hs = (f4*)take(wgs * (size_t)p.seg * state);
  a->gs = (f4*)take(wgs * state);
  const int64_t blocks = (p.HG + p.HR - 1) / p.HR;
  a->part = (float*)take(blocks > 1 ? (size_t)(blocks * 2 * z.B * z.L * z.G * z.N) * 4 : 0);
  a->params = (float*)take((size_t)(z.B * p.segs * p.HV) * 3 * 4);
  return off;
}
void fill(SelArgs* a, const Sizes& z, const float* gamma, const float* dt_bias, const float* skip) {
  a->gamma = gamma;
  a->dt_bias = dt_bias;
  a->skip = skip;
  a->B = z.B;
  a->L = z.L;
  a->H = (int)z.H;
  a->P = (int)z.P;
  a->G = (int)z.G;
  a->N = (int)z.N;
}
int check_inputs(const Sizes& z, const res_rows_t& x, const res_rows_t& dt, const res_rows_t& b, const res_rows_t& c, size_t es,
                 const float* gamma, const float* dt_bias, const float* skip) {
  int rc;
  if (z.L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, z.L, es)) || (rc = check_rows("dt", dt.p, dt.sb, dt.st, z.L, es)) ||
                  (rc = check_rows("b", b.p, b.sb, b.st, z.L, es)) || (rc = check_rows("c", c.p, c.sb, c.st, z.L, es))))
    return rc;
  if ((rc = check_f32("gamma", gamma, true)) || (rc = check_f32("dt_bias", dt_bias, false)) || (rc = check_f32("skip", skip, false)))
    return rc;
  return RES_OK;
}

}  // namespace

extern "C" {

size_t resonator_selective_scan_workspace_bytes(int backward, res_dtype_t act_dt, int64_t B, int64_t L, int64_t H, int64_t P,
                                                int64_t G, int64_t N) {
  const Sizes z{B, L, H, P, G, N};
  if (check_selective(z, act_dt)) return 0;
  SelArgs a{};
  a.p = plan_of(z, act_dt);
  return lay_out(z, backward != 0, false, nullptr, &a);
}

int64_t resonator_selective_scan_carry_floats(res_dtype_t act_dt, int64_t B, int64_t L, int64_t H, int64_t P, int64_t G,
                                              int64_t N) {
  const Sizes z{B, L, H, P, G, N};
  if (check_selective(z, act_dt)) return -1;
  return (int64_t)border_floats(z, plan_of(z, act_dt));
}

int resonator_selective_scan_fwd(res_rows_t x, res_rows_t dt, res_rows_t b, res_rows_t c, res_dtype_t act_dt,
                                 const float* gamma, const float* dt_bias, const float* skip, const float* h0,
                                 const int32_t* lengths, void* y, float* h_out, float* carry, int64_t B, int64_t L,
                                 int64_t H, int64_t P, int64_t G, int64_t N, void* ws, size_t ws_bytes, void* stream) {
  const Sizes z{B, L, H, P, G, N};
  int rc = check_selective(z, act_dt);
  if (rc) return rc;
  const size_t es = elt(act_dt);
  if ((rc = check_inputs(z, x, dt, b, c, es, gamma, dt_bias, skip)) || (rc = check_f32("h0", h0, false)) ||
      (rc = check_elt("lengths", lengths, false, 4)) || (rc = check_elt("y", y, L > 0 && (h_out != nullptr || carry == nullptr), es)) ||
      (rc = check_f32("h_out", h_out, false)) || (rc = check_elt("carry", carry, false, 16)))
    return rc;
  SelArgs a{};
  a.p = plan_of(z, act_dt);
  const size_t need = lay_out(z, false, carry != nullptr, nullptr, &a);
  if ((rc = check_ws(ws, ws_bytes, need))) return rc;
  const size_t state = (size_t)(B * H * P * N) * 4;
  const Span in[] = {span(x, B, L, H * P, es), span(dt, B, L, H, es), span(b, B, L, G * N, es), span(c, B, L, G * N, es),
                     flat(gamma, 4 * H),       flat(dt_bias, 4 * H),  flat(skip, 4 * H),        flat(lengths, 4 * B),
                     flat(h0, state)};
  const Span out[] = {flat(y, es * B * L * H * P), flat(h_out, state), flat(carry, border_floats(z, a.p) * 4), flat(ws, need)};
  if ((rc = check_apart(in, out, Same{1, 8}, " (h_out may be h0 itself)"))) return rc;
  a.enter = carry;
  lay_out(z, false, carry != nullptr, static_cast<char*>(ws), &a);
  fill(&a, z, gamma, dt_bias, skip);
  a.x = rows_of(x, L);
  a.dt = rows_of(dt, L);
  a.b = rows_of(b, L);
  a.c = rows_of(c, L);
  a.h0 = h0;
  a.lengths = lengths;
  a.y = y;
  a.h_out = h_out;
  return launched(act_dt == RES_BF16 ? launch_selective_fwd<bf16_t>(a, (hipStream_t)stream) : launch_selective_fwd<float>(a, (hipStream_t)stream),
                  "selective scan launch");
}

int resonator_selective_scan_bwd(res_rows_t x, res_rows_t dt, res_rows_t b, res_rows_t c, res_rows_t dy, res_dtype_t act_dt,
                                 const float* gamma, const float* dt_bias, const float* skip, const float* h0,
                                 const int32_t* lengths, const float* carry, const float* dh_out, res_rows_out_t dx,
                                 res_rows_out_t ddt, res_rows_out_t db, res_rows_out_t dc, float* dgamma, float* ddt_bias,
                                 float* dskip, float* dh0, int64_t B, int64_t L, int64_t H, int64_t P, int64_t G, int64_t N,
                                 void* ws, size_t ws_bytes, void* stream) {
  const Sizes z{B, L, H, P, G, N};
  int rc = check_selective(z, act_dt);
  if (rc) return rc;
  const size_t es = elt(act_dt);
  if ((rc = check_inputs(z, x, dt, b, c, es, gamma, dt_bias, skip)) ||
      (L > 0 && ((rc = check_rows("dy", dy.p, dy.sb, dy.st, L, es)) || (rc = check_rows("dx", dx.p, dx.sb, dx.st, L, es)) ||
                 (rc = check_rows("ddt", ddt.p, ddt.sb, ddt.st, L, es)) || (rc = check_rows("db", db.p, db.sb, db.st, L, es)) ||
                 (rc = check_rows("dc", dc.p, dc.sb, dc.st, L, es)))))
    return rc;
  SelArgs a{};
  a.p = plan_of(z, act_dt);
  if ((rc = check_f32("h0", h0, false)) || (rc = check_elt("lengths", lengths, false, 4)) ||
      (rc = check_elt("carry", carry, a.p.segs > 1, 16)) || (rc = check_f32("dh_out", dh_out, false)) ||
      (rc = check_f32("dgamma", dgamma, true)) || (rc = check_f32("ddt_bias", ddt_bias, false)) ||
      (rc = check_f32("dskip", dskip, false)) || (rc = check_f32("dh0", dh0, false)))
    return rc;
  const size_t need = lay_out(z, true, true, nullptr, &a);
  if ((rc = check_ws(ws, ws_bytes, need))) return rc;
  const size_t state = (size_t)(B * H * P * N) * 4;
  const Span in[] = {span(x, B, L, H * P, es),  span(dt, B, L, H, es), span(b, B, L, G * N, es), span(c, B, L, G * N, es),
                     span(dy, B, L, H * P, es), flat(gamma, 4 * H),    flat(dt_bias, 4 * H),     flat(skip, 4 * H),
                     flat(lengths, 4 * B),      flat(h0, state),       flat(dh_out, state),      flat(carry, border_floats(z, a.p) * 4)};
  const Span out[] = {span(dx, B, L, H * P, es), span(ddt, B, L, H, es), span(db, B, L, G * N, es), span(dc, B, L, G * N, es),
                      flat(dgamma, 4 * H),       flat(ddt_bias, 4 * H),  flat(dskip, 4 * H),        flat(dh0, state),
                      flat(ws, need)};
  if ((rc = check_apart(in, out, Same{-1, -1}, ""))) return rc;
  if (L > 0 && !(rows_apart(dx.sb, dx.st, B, L, H * P) && rows_apart(ddt.sb, ddt.st, B, L, H) && rows_apart(db.sb, db.st, B, L, G * N) &&
                 rows_apart(dc.sb, dc.st, B, L, G * N)))
    return api_error(RES_ERR_INVALID_ARG, "the rows of dx, ddt, db and dc must not overlap");
  lay_out(z, true, true, static_cast<char*>(ws), &a);
  fill(&a, z, gamma, dt_bias, skip);
  a.x = rows_of(x, L);
  a.dt = rows_of(dt, L);
  a.b = rows_of(b, L);
  a.c = rows_of(c, L);
  a.dy = rows_of(dy, L);
  a.dx = rows_of(dx, L);
  a.ddt = rows_of(ddt, L);
  a.db = rows_of(db, L);
  a.dc = rows_of(dc, L);
  a.h0 = h0;
  a.lengths = lengths;
  a.enter = const_cast<float*>(carry);
  a.dh_out = dh_out;
  a.dgamma = dgamma;
  a.ddt_bias = ddt_bias;
  a.dskip = dskip;
  a.dh0 = dh0;
  return launched(act_dt == RES_BF16 ? launch_selective_bwd<bf16_t>(a, (hipStream_t)stream) : launch_selective_bwd<float>(a, (hipStream_t)stream),
                  "selective scan backward launch");
}

int resonator_selective_scan_step(res_rows_t x, res_rows_t dt, res_rows_t b, res_rows_t c, res_dtype_t act_dt,
                                  const float* gamma, const float* dt_bias, const float* skip, const float* h, void* y,
                                  float* h_out, int64_t B, int64_t H, int64_t P, int64_t G, int64_t N, void* stream) {
  const Sizes z{B, 1, H, P, G, N};
  int rc = check_selective(z, act_dt);
  if (rc) return rc;
  const size_t es = elt(act_dt);
  if ((rc = check_inputs(z, x, dt, b, c, es, gamma, dt_bias, skip)) || (rc = check_f32("h", h, true)) ||
      (rc = check_f32("h_out", h_out, true)) || (rc = check_elt("y", y, true, es)))
    return rc;
  const size_t state = (size_t)(B * H * P * N) * 4;
  const Span in[] = {span(x, B, 1, H * P, es), span(dt, B, 1, H, es), span(b, B, 1, G * N, es), span(c, B, 1, G * N, es),
                     flat(gamma, 4 * H),       flat(dt_bias, 4 * H),  flat(skip, 4 * H),        flat(h, state)};
  const Span out[] = {flat(y, es * B * H * P), flat(h_out, state)};
  if ((rc = check_apart(in, out, Same{1, 7}, " (h_out may be h itself)"))) return rc;
  SelArgs a{};
  fill(&a, z, gamma, dt_bias, skip);
  a.x = rows_of(x, 1);
  a.dt = rows_of(dt, 1);
  a.b = rows_of(b, 1);
  a.c = rows_of(c, 1);
  a.y = y;
  a.h_out = h_out;
  return launched(act_dt == RES_BF16 ? launch_selective_step<bf16_t>(a, h, (hipStream_t)stream)
                                     : launch_selective_step<float>(a, h, (hipStream_t)stream),
                  "selective scan step launch");
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Token log probabilities
// ---------------------------------------------------------------------------
namespace {

int check_logprobs(const void* logits, int64_t ld, res_dtype_t dt, const int64_t* tokens, int64_t R, int64_t V, float scale) {
  int rc;
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (R < 0 || V < 1 || ld < V)
    return api_error(RES_ERR_INVALID_ARG, "R must be >= 0, V >= 1 and ld >= V (got R=%lld V=%lld ld=%lld)", (long long)R, (long long)V,
                     (long long)ld);
  // (the kernels take it times log2 e: the largest logit's difference from itself times an infinite one would be none)
  if (!(scale > 0.0f) || !(scale <= 0x1p127f)) return api_error(RES_ERR_INVALID_ARG, "scale must be positive and at most 2^127 (got %g)", (double)scale);
  if (V > (1LL << 30) || ld > (1LL << 40) || R > (1LL << 31))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (R=%lld V=%lld ld=%lld)", (long long)R, (long long)V, (long long)ld);
  if ((rc = check_elt("logits", logits, R > 0, elt(dt))) || (rc = check_elt("tokens", tokens, R > 0, 8))) return rc;
  return RES_OK;
}

}  // namespace

extern "C" {

int resonator_token_logprobs_fwd(const void* logits, int64_t ld, res_dtype_t dt, const int64_t* tokens, int64_t R, int64_t V,
                                 float scale, float* logp, float* stats, float* entropy, int64_t top, int64_t* top_ids,
                                 float* top_logp, void* stream) {
  int rc = check_logprobs(logits, ld, dt, tokens, R, V, scale);
  if (rc) return rc;
  if (top < 0 || top > LOGPROBS_TOP || top > V)
    return api_error(RES_ERR_INVALID_ARG, "top must be in [0, min(V, %d)] (got %lld)", LOGPROBS_TOP, (long long)top);
  if ((rc = check_f32("logp", logp, R > 0)) || (rc = check_f32("stats", stats, false)) || (rc = check_f32("entropy", entropy, false)) ||
      (rc = check_elt("top_ids", top_ids, R > 0 && top > 0, 8)) || (rc = check_f32("top_logp", top_logp, R > 0 && top > 0)))
    return rc;
  if (R == 0) return RES_OK;
  const Span in[] = {res::span(logits, ld, 0, R, 1, V, elt(dt)), flat(tokens, 8 * R)};
  const Span out[] = {flat(logp, 4 * R), flat(stats, 8 * R), flat(entropy, 4 * R), flat(top > 0 ? top_ids : nullptr, 8 * R * top),
                      flat(top > 0 ? top_logp : nullptr, 4 * R * top)};
  if ((rc = check_apart(in, out, Same{-1, -1}, ""))) return rc;
  LogprobsArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.tokens = tokens;
  a.R = R;
  a.V = V;
  a.scale = scale;
  a.logp = logp;
  a.stats = stats;
  a.entropy = entropy;
  a.top = (int)top;
  a.top_ids = top_ids;
  a.top_logp = top_logp;
  return launched(dt == RES_BF16 ? launch_logprobs_fwd<bf16_t>(a, (hipStream_t)stream) : launch_logprobs_fwd<float>(a, (hipStream_t)stream),
                  "token log probabilities launch");
}

int resonator_token_logprobs_bwd(const void* logits, int64_t ld, res_dtype_t dt, const int64_t* tokens, int64_t R, int64_t V,
                                 float scale, const float* stats, const float* entropy, const float* dlogp,
                                 const float* dentropy, void* dlogits, int64_t ldd, void* stream) {
  int rc = check_logprobs(logits, ld, dt, tokens, R, V, scale);
  if (rc) return rc;
  if (ldd < V || ldd > (1LL << 40)) return api_error(RES_ERR_INVALID_ARG, "ldd must be in [V, 2^40] (got %lld)", (long long)ldd);
  if ((rc = check_f32("stats", stats, R > 0)) || (rc = check_f32("entropy", entropy, R > 0 && dentropy != nullptr)) ||
      (rc = check_f32("dlogp", dlogp, false)) || (rc = check_f32("dentropy", dentropy, false)) ||
      (rc = check_elt("dlogits", dlogits, R > 0, elt(dt))))
    return rc;
  if (R == 0) return RES_OK;
  const Span in[] = {res::span(logits, ld, 0, R, 1, V, elt(dt)), flat(tokens, 8 * R), flat(stats, 8 * R), flat(entropy, 4 * R),
                     flat(dlogp, 4 * R),                         flat(dentropy, 4 * R)};
  const Span out[] = {res::span(dlogits, ldd, 0, R, 1, V, elt(dt))};
  if ((rc = check_apart(in, out, Same{ld == ldd || R == 1 ? 0 : -1, 0}, " (dlogits may be the logits themselves)"))) return rc;
  LogprobsArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.ldd = ldd;
  a.tokens = tokens;
  a.R = R;
  a.V = V;
  a.scale = scale;
  a.stats = const_cast<float*>(stats);
  a.entropy = const_cast<float*>(entropy);
  a.dlogp = dlogp;
  a.dentropy = dentropy;
  a.dlogits = dlogits;
  return launched(dt == RES_BF16 ? launch_logprobs_bwd<bf16_t>(a, (hipStream_t)stream) : launch_logprobs_bwd<float>(a, (hipStream_t)stream),
                  "token log probabilities backward launch");
}

}  // extern "C"
