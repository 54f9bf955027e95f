// C ABI of the gated recurrent layer's operators: argument checks and dispatch.
// Declared in include/resonator.h.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <utility>
#include <vector>

#include "../../include/resonator.h"
#include "api_check.h"
#include "layer.h"

using namespace res;

namespace {

int check_scan(int64_t B, int64_t L, int64_t D, res_dtype_t dt) {
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (B < 1 || D < 1 || L < 0)
    return api_error(RES_ERR_INVALID_ARG, "B and D must be >= 1 and L >= 0 (got B=%lld L=%lld D=%lld)", (long long)B,
                     (long long)L, (long long)D);
  const int64_t NB = (D + GATED_CW - 1) / GATED_CW;
  // (tiles of a call are 32-bit counts)
  if (D > (1 << 21) || L >= (1LL << 31) - 65536 || B > (1LL << 31) || B * NB >= (1LL << 30) ||
      B * NB * (L / GATED_BWD_TILE + 1) >= (1LL << 31))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (B=%lld L=%lld D=%lld)", (long long)B,
                     (long long)L, (long long)D);
  return RES_OK;
}
// A launch takes whole batch rows.
int check_launch(int64_t L, int64_t D, int tile) {
  if ((D + GATED_CW - 1) / GATED_CW * gated_tiles(L, tile) <= LAUNCH_THREADS / GATED_THREADS) return RES_OK;
  return api_error(RES_ERR_UNSUPPORTED, "a row beyond one launch (L=%lld D=%lld)", (long long)L, (long long)D);
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
  // the forward's or the backward's published words, and behind the backward's its partial sums
  const int64_t f = gated_tiles(L, GATED_FWD_TILE), b = gated_tiles(L, GATED_BWD_TILE);
  return 256 + (size_t)(B * NB) * (size_t)std::max(f * GATED_TILE_WORDS, b * (GATED_TILE_WORDS + GATED_CW)) * 8;
}

int resonator_gated_scan_fwd(res_rows_t x, res_rows_t r, res_rows_t i, res_dtype_t dt, void* y, int64_t B, int64_t L,
                             int64_t D, const float* gamma, const float* h0, const int32_t* lengths, float* h_out,
                             float* carry, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_scan(B, L, D, dt);
  if (rc || (rc = check_launch(L, D, GATED_FWD_TILE))) return rc;
  const size_t es = elt(dt);
  if (L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, L, es)) || (rc = check_rows("r", r.p, r.sb, r.st, L, es)) ||
                (rc = check_rows("i", i.p, i.sb, i.st, L, es))))
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
  a.x = Rows{x.p, x.sb, L > 1 ? x.st : 0};
  a.r = Rows{r.p, r.sb, L > 1 ? r.st : 0};
  a.i = Rows{i.p, i.sb, L > 1 ? i.st : 0};
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
  a.hdr = static_cast<uint32_t*>(ws);
  a.words = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + 256);
  return launched(dt == RES_BF16 ? launch_gated_fwd<bf16_t>(a, (hipStream_t)stream) : launch_gated_fwd<float>(a, (hipStream_t)stream),
                  "gated scan launch");
}

int resonator_gated_scan_bwd(res_rows_t x, res_rows_t r, res_rows_t i, res_rows_t dy, res_dtype_t dt,
                             res_rows_out_t dx, res_rows_out_t dr, res_rows_out_t di, int64_t B, int64_t L, int64_t D,
                             const float* gamma, const float* carry, const int32_t* lengths, const float* dh_out,
                             float* dgamma, float* dh0, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_scan(B, L, D, dt);
  if (rc || (rc = check_launch(L, D, GATED_BWD_TILE))) return rc;
  const size_t es = elt(dt);
  if (L > 0 && ((rc = check_rows("x", x.p, x.sb, x.st, L, es)) || (rc = check_rows("r", r.p, r.sb, r.st, L, es)) ||
                (rc = check_rows("i", i.p, i.sb, i.st, L, es)) || (rc = check_rows("dy", dy.p, dy.sb, dy.st, L, es)) ||
                (rc = check_rows("dx", dx.p, dx.sb, dx.st, L, es)) || (rc = check_rows("dr", dr.p, dr.sb, dr.st, L, es)) ||
                (rc = check_rows("di", di.p, di.sb, di.st, L, es))))
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
  a.x = Rows{x.p, x.sb, L > 1 ? x.st : 0};
  a.r = Rows{r.p, r.sb, L > 1 ? r.st : 0};
  a.i = Rows{i.p, i.sb, L > 1 ? i.st : 0};
  a.dy = Rows{dy.p, dy.sb, L > 1 ? dy.st : 0};
  a.dx = RowsOut{dx.p, dx.sb, L > 1 ? dx.st : 0};
  a.dr = RowsOut{dr.p, dr.sb, L > 1 ? dr.st : 0};
  a.di = RowsOut{di.p, di.sb, L > 1 ? di.st : 0};
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
  a.hdr = static_cast<uint32_t*>(ws);
  a.words = reinterpret_cast<uint64_t*>(static_cast<char*>(ws) + 256);
  a.part = a.words + B * a.NB * gated_tiles(L, GATED_BWD_TILE) * GATED_TILE_WORDS;
  return launched(dt == RES_BF16 ? launch_gated_bwd<bf16_t>(a, dgamma, (hipStream_t)stream)
                                 : launch_gated_bwd<float>(a, dgamma, (hipStream_t)stream),
                  "gated scan backward launch");
}

int resonator_gated_scan_step(res_rows_t x, res_rows_t r, res_rows_t i, res_dtype_t dt, void* y, int64_t B, int64_t D,
                              const float* gamma, const float* h, float* h_out, void* stream) {
  int rc = check_scan(B, 1, D, dt);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((rc = check_rows("x", x.p, x.sb, x.st, 1, es)) || (rc = check_rows("r", r.p, r.sb, r.st, 1, es)) ||
      (rc = check_rows("i", i.p, i.sb, i.st, 1, es)) || (rc = check_f32("gamma", gamma, true)) ||
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

// ---------------------------------------------------------------------------
// Linear product
// ---------------------------------------------------------------------------
namespace {

int check_linear(int64_t R, int64_t K, int64_t N, res_dtype_t dt, int act) {
  if (!known(dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (act < RES_ACT_NONE || act > RES_ACT_GELU_TANH) return api_error(RES_ERR_INVALID_ARG, "unknown activation code %d", act);
  if (R < 0 || K < 1 || N < 1)
    return api_error(RES_ERR_INVALID_ARG, "K and N must be >= 1 and R >= 0 (got R=%lld K=%lld N=%lld)", (long long)R,
                     (long long)K, (long long)N);
  // (tiles of 64 x 64 are 32-bit counts)
  if (R > (1LL << 31) || K > (1 << 20) || N > (1 << 20) || R * std::max(K, N) > (1LL << 38))
    return api_error(RES_ERR_UNSUPPORTED, "sizes beyond the supported range (R=%lld K=%lld N=%lld)", (long long)R,
                     (long long)K, (long long)N);
  return RES_OK;
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// Whether pre is computed again in the backward rather than kept: the product costs 2 R K N operations, keeping pre 8 R N
// bytes written and read.  A training step (R x K x N, bf16, gelu) computing it and keeping it: 65536 x 256 x 1024 340 and
// 361 us, 2048 x 256 x 1024 43 and 49, 32768 x 512 x 2048 430 and 428 (and 268 MB less), 32768 x 768 x 2048 569 and 523.
// A float32 product costs eight times as much: 16384 x 64 x 1024 159 and 155, 16384 x 256 x 1024 338 and 282.
bool computes_pre(res_dtype_t dt, int act, int64_t K) { return act != RES_ACT_NONE && dt == RES_BF16 && K <= 512; }

// The workspace, a piece at a time; with a null base it only counts.
struct Pieces {
  char* base;
  size_t off;
  void* take(size_t bytes) {
    void* p = base != nullptr ? base + off : nullptr;
    off += up256(bytes);
    return p;
  }
};

// An operand of a product: [rows][cols] at distance ld.  `k`: its K axis is the consecutive one.
struct Operand {
  const void* p;
  int64_t ld, rows, cols;
};
bool whole(const Operand& o, size_t es) {
  const int64_t ep = 16 / (int64_t)es;
  return aligned(o.p, 16) && o.ld % ep == 0 && o.cols % ep == 0 && o.ld < RES_LINEAR_FAR;  // (32-bit offsets within a tile)
}
// The operand as the kernels take it, copied where it is not.
hipError_t pack(Operand* o, res_dtype_t dt, bool loose, Pieces* ws, bool count, hipStream_t st) {
  const size_t es = elt(dt);
  if (!loose || (!count && (o->rows == 0 || whole(*o, es)))) return hipSuccess;  // (no rows: nothing reads it)
  const int64_t to = up(o->cols, 16 / (int64_t)es);
  void* dst = ws->take((size_t)(o->rows * to) * es);
  if (count) return hipSuccess;
  const hipError_t e = dt == RES_BF16 ? launch_pack<bf16_t>(o->p, o->ld, o->rows, o->cols, dst, to, st)
                                      : launch_pack<float>(o->p, o->ld, o->rows, o->cols, dst, to, st);
  o->p = dst;
  o->ld = to;
  return e;
}

// C [M][N] from A and B whose K axis is consecutive (ak, bk) or not; `count` only counts the workspace.
hipError_t gemm(res_dtype_t dt, GemmArgs& g, const Operand& A, const Operand& B, bool ak, bool bk, bool loose, Pieces ws,
                size_t* need, hipStream_t st) {
  const size_t es = elt(dt);
  const int64_t ep = 16 / (int64_t)es;
  g.ak = ak;
  g.bk = bk;
  g.A = A.p;
  g.B = B.p;
  g.lda = A.ld;
  g.ldb = B.ld;
  g.xa = ak ? A.rows : up(A.cols, ep);
  g.xb = bk ? B.rows : up(B.cols, ep);
  g.loose = g.N % ep != 0 || !(aligned(g.out, 16) && aligned(g.res, 16) && aligned(g.bias, 16) && aligned(g.pre, 16) && aligned(g.dy, 16));
  if (need != nullptr) {  // (the outputs' alignment is not known yet)
    for (bool wide : {false, true}) {
      const int64_t s = linear_plan(g.M, g.N, g.K, es, g.dy != nullptr, wide).splits;
      *need = std::max(*need, ws.off + (s > 1 ? up256((size_t)(s * g.M * g.N) * 4) : 0));
    }
    return hipSuccess;
  }
  const LinearPlan p = linear_plan(g.M, g.N, g.K, es, g.dy != nullptr, !g.loose);
  g.tile = p.tile;
  g.splits = p.splits;
  g.part = static_cast<float*>(ws.take(p.splits > 1 ? (size_t)(p.splits * g.M * g.N) * 4 : 0));
  return dt == RES_BF16 ? launch_gemm<bf16_t>(g, st) : launch_gemm<float>(g, st);
}

struct LinearCall {
  const void *x, *W;
  int64_t ldx;
  res_dtype_t dt;
  int act;
  int64_t R, K, N;
  bool loose;  // operands that may have to be copied
};

// The forward's launches; `need` counts the workspace instead.
hipError_t linear_fwd(const LinearCall& c, const float* bias, const void* residual, void* y, float* pre, Pieces ws, size_t* need,
                      hipStream_t st) {
  Operand x{c.x, c.ldx, c.R, c.K}, W{c.W, c.N, c.K, c.N};
  hipError_t e = pack(&x, c.dt, c.loose, &ws, need != nullptr, st);
  if (e == hipSuccess) e = pack(&W, c.dt, c.loose, &ws, need != nullptr, st);
  if (e != hipSuccess) return e;
  GemmArgs g{};
  g.M = c.R;
  g.N = c.N;
  g.K = c.K;
  g.bias = bias;
  g.res = residual;
  g.pre = pre;
  g.out = y;
  g.act = c.act;
  return gemm(c.dt, g, x, W, true, false, c.loose, ws, need, st);
}

// The backward's launches; `need` counts the workspace instead (then pre and dx, dW, db only say what is asked for).
hipError_t linear_bwd(const LinearCall& c, const float* bias, const void* dy, const float* pre, const void* residual, void* dx,
                      void* dW, float* db, Pieces ws, size_t* need, hipStream_t st) {
  const bool count = need != nullptr, again = c.act != RES_ACT_NONE && pre == nullptr && c.R > 0;
  const size_t es = elt(c.dt);
  Operand x{c.x, c.ldx, c.R, c.K}, W{c.W, c.N, c.K, c.N}, d{dy, c.N, c.R, c.N};
  hipError_t e = hipSuccess;
  if (dW != nullptr || again) e = pack(&x, c.dt, c.loose, &ws, count, st);
  if (e == hipSuccess && (dx != nullptr || again)) e = pack(&W, c.dt, c.loose, &ws, count, st);
  if (e != hipSuccess) return e;
  int64_t blocks = 0;
  float* part = nullptr;
  bool ready = false;
  if (c.act != RES_ACT_NONE || db != nullptr) {
    // (room for the most rows of sums: which tile is taken depends on the alignments too)
    blocks = again ? linear_col_blocks(TILE_SMALL, c.R) : linear_row_blocks(c.R);
    if (db != nullptr) part = static_cast<float*>(ws.take((size_t)(blocks * c.N) * 4));
    const int64_t to = up(c.N, 16 / (int64_t)es);
    void* out = c.act != RES_ACT_NONE ? ws.take((size_t)(c.R * to) * es) : nullptr;
    if (again) {
      GemmArgs g{};
      g.M = c.R;
      g.N = c.N;
      g.K = c.K;
      g.bias = bias;
      g.out = out;
      g.act = c.act;
      g.dy = count ? &g : dy;
      g.colpart = part;
      e = gemm(c.dt, g, x, W, true, false, c.loose, ws, need, st);
      blocks = linear_col_blocks(g.tile, c.R);
    } else if (!count && c.R > 0) {
      const bool loose = c.N % 4 != 0 || !(aligned(dy, 16) && aligned(pre, 16));
      e = c.dt == RES_BF16 ? launch_act_bwd<bf16_t>(dy, pre, c.act, out, to, part, c.R, c.N, loose, st)
                           : launch_act_bwd<float>(dy, pre, c.act, out, to, part, c.R, c.N, loose, st);
    }
    if (e == hipSuccess && !count && db != nullptr) e = launch_col_sum(part, blocks, c.N, db, st);
    if (out != nullptr || count) d.p = out;
    if (out != nullptr || (count && c.act != RES_ACT_NONE)) {
      if (!again) d.ld = d.cols = to;  // (with zeros from column N on)
      ready = !again;
    }
  }
  if (e == hipSuccess && !ready && (dx != nullptr || dW != nullptr)) e = pack(&d, c.dt, c.loose, &ws, count, st);
  if (e == hipSuccess && dx != nullptr && c.R > 0) {
    GemmArgs g{};
    g.M = c.R;
    g.N = c.K;
    g.K = c.N;
    g.res = residual;
    g.out = dx;
    e = gemm(c.dt, g, d, W, true, true, c.loose, ws, need, st);
  }
  if (e == hipSuccess && dW != nullptr) {
    GemmArgs g{};
    g.M = c.K;
    g.N = c.N;
    g.K = c.R;
    g.out = dW;
    e = gemm(c.dt, g, x, d, false, false, c.loose, ws, need, st);
  }
  if (count) *need = std::max(*need, ws.off);
  return e;
}

size_t linear_bytes(bool backward, const LinearCall& c) {
  size_t need = 0;
  char* any = reinterpret_cast<char*>(256);  // stands for what a call asks for; nothing is read
  if (!backward) {
    (void)linear_fwd(c, nullptr, nullptr, nullptr, nullptr, Pieces{nullptr, 0}, &need, nullptr);
  } else {
    for (const float* pre : {static_cast<const float*>(nullptr), reinterpret_cast<const float*>(any)})
      (void)linear_bwd(c, nullptr, any, pre, nullptr, any, any, reinterpret_cast<float*>(any), Pieces{nullptr, 0}, &need, nullptr);
  }
  return need;
}
// whether some operand, as given, is not whole pieces
bool loose_call(const LinearCall& c, const void* dy) {
  const size_t es = elt(c.dt);
  return !((c.x == nullptr || whole(Operand{c.x, c.ldx, c.R, c.K}, es)) && (c.W == nullptr || whole(Operand{c.W, c.N, c.K, c.N}, es)) &&
           (dy == nullptr || whole(Operand{dy, c.N, c.R, c.N}, es)) && c.K % (16 / (int64_t)es) == 0 && c.N % (16 / (int64_t)es) == 0);
}
int check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return RES_OK;
  if (ws == nullptr || have < need)
    return api_error(RES_ERR_WORKSPACE, "workspace null or too small (%zu bytes, %zu needed)", have, need);
  return aligned(ws, 256) ? RES_OK : api_error(RES_ERR_MISALIGNED, "the workspace must be 256-byte aligned");
}
int check_mat(const char* name, const void* p, size_t es, bool needed) {
  if (p == nullptr) return needed ? api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name) : RES_OK;
  return aligned(p, es) ? RES_OK : api_error(RES_ERR_MISALIGNED, "%s must be aligned to its element", name);
}

}  // namespace

extern "C" {

size_t resonator_linear_workspace_bytes(int backward, res_dtype_t dt, int act, int64_t R, int64_t K, int64_t N, int loose) {
  if (check_linear(R, K, N, dt, act)) return 0;
  return linear_bytes(backward != 0, LinearCall{nullptr, nullptr, K, dt, act, R, K, N, loose != 0});
}

int resonator_linear_keeps_pre(res_dtype_t dt, int act, int64_t K) { return act != RES_ACT_NONE && !computes_pre(dt, act, K); }

int resonator_linear_fwd(const void* x, int64_t ldx, const void* W, res_dtype_t dt, const float* bias, int act,
                         const void* residual, void* y, float* pre, int64_t R, int64_t K, int64_t N, void* ws,
                         size_t ws_bytes, void* stream) {
  int rc = check_linear(R, K, N, dt, act);
  if (rc) return rc;
  const size_t es = elt(dt);
  if ((rc = check_mat("W", W, es, true)) || (rc = check_f32("bias", bias, false))) return rc;
  if (R == 0) return RES_OK;
  if (ldx < K || ldx > (1LL << 40)) return api_error(RES_ERR_INVALID_ARG, "ldx must be in [K, 2^40]");
  if ((rc = check_mat("x", x, es, true)) || (rc = check_mat("y", y, es, true)) || (rc = check_f32("pre", pre, false)) ||
      (rc = check_mat("residual", residual, es, false)))
    return rc;
  LinearCall c{x, W, ldx, dt, act, R, K, N, false};
  c.loose = loose_call(c, nullptr);
  const size_t need = linear_bytes(false, c);
  if ((rc = check_ws(ws, ws_bytes, need))) return rc;
  const Span in[] = {span(x, 0, ldx, 1, R, K, es), flat(W, es * K * N), flat(bias, 4 * N), flat(residual, es * R * N)};
  const Span out[] = {flat(y, es * R * N), flat(pre, 4 * R * N), flat(need ? ws : nullptr, need)};
  for (int o = 0; o < 3; ++o) {
    for (int k = 0; k < 4; ++k)
      if (touch(out[o], in[k]) && !(o == 0 && k == 3 && y == residual))
        return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs (y may be the residual itself)");
    for (int k = 0; k < o; ++k)
      if (touch(out[o], out[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  }
  return launched(linear_fwd(c, bias, residual, y, pre, Pieces{static_cast<char*>(ws), 0}, nullptr, (hipStream_t)stream), "linear launch");
}

int resonator_linear_bwd(const void* x, int64_t ldx, const void* W, res_dtype_t dt, const float* bias, const void* dy,
                         const float* pre, int act, const void* residual, void* dx, void* dW, float* db, int64_t R, int64_t K,
                         int64_t N, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_linear(R, K, N, dt, act);
  if (rc) return rc;
  const size_t es = elt(dt);
  if (dx == nullptr && dW == nullptr && db == nullptr)
    return api_error(RES_ERR_INVALID_ARG, "one of dx, dW and db must be non-null");
  const bool again = act != RES_ACT_NONE && pre == nullptr;
  if (R > 0 && ((rc = check_mat("dy", dy, es, true)) || (rc = check_f32("pre", pre, false)) || (rc = check_f32("bias", bias, false)) ||
                (rc = check_mat("x", x, es, dW != nullptr || again)) || (rc = check_mat("W", W, es, dx != nullptr || again))))
    return rc;
  if ((rc = check_mat("residual", residual, es, false)) || (rc = check_mat("dx", dx, es, false)) ||
      (rc = check_mat("dW", dW, es, false)) || (rc = check_f32("db", db, false)))
    return rc;
  if (R > 0 && (dW != nullptr || again) && (ldx < K || ldx > (1LL << 40)))
    return api_error(RES_ERR_INVALID_ARG, "ldx must be in [K, 2^40]");
  LinearCall c{dW != nullptr || again ? x : nullptr, dx != nullptr || again ? W : nullptr, ldx, dt, act, R, K, N, false};
  c.loose = loose_call(c, dy);
  size_t need = 0;
  {
    char* any = reinterpret_cast<char*>(256);
    (void)linear_bwd(c, nullptr, any, pre != nullptr ? reinterpret_cast<const float*>(any) : nullptr, nullptr, dx, dW, db,
               Pieces{nullptr, 0}, &need, nullptr);
  }
  if ((rc = check_ws(ws, ws_bytes, need))) return rc;
  const Span in[] = {span(c.x, 0, ldx, 1, R, K, es), flat(c.W, es * K * N), flat(dy, es * R * N), flat(pre, 4 * R * N),
                     flat(residual, es * R * K), flat(bias, 4 * N)};
  const Span out[] = {flat(dx, es * R * K), flat(dW, es * K * N), flat(db, 4 * N), flat(need ? ws : nullptr, need)};
  for (int o = 0; o < 4; ++o) {
    for (int k = 0; k < 6; ++k)
      if (touch(out[o], in[k]) && !(o == 0 && k == 4 && dx == residual))
        return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap inputs (dx may be the residual itself)");
    for (int k = 0; k < o; ++k)
      if (touch(out[o], out[k])) return api_error(RES_ERR_INVALID_ARG, "outputs must not overlap each other");
  }
  return launched(linear_bwd(c, bias, dy, pre, residual, dx, dW, db, Pieces{static_cast<char*>(ws), 0}, nullptr, (hipStream_t)stream),
                  "linear backward launch");
}

}  // extern "C"

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
namespace {

// Whether what a step writes overlaps what else it reads or writes: tensors are stepped side by side.  (54 of them in any order: 1 us.)
bool adamw_overlaps(const res_adamw_tensor_t* t, int64_t count, size_t pe, size_t ge, const res_adamw_state_t& in,
                    const res_adamw_state_t& out, const float* scale) {
  typedef std::pair<uintptr_t, uintptr_t> Range;
  auto range = [](const void* p, int64_t from, int64_t to, size_t es) {
    return Range{(uintptr_t)p + (uintptr_t)from * es, (uintptr_t)p + (uintptr_t)to * es};
  };
  // the tensors' places in the states
  std::vector<Range> w;
  w.reserve((size_t)count + 5);
  for (int64_t k = 0; k < count; ++k)
    if (t[k].n > 0) w.push_back(range(nullptr, t[k].state, t[k].state + t[k].n, 1));
  auto meet = [&w] {
    if (!std::is_sorted(w.begin(), w.end())) std::sort(w.begin(), w.end());
    for (size_t k = 1; k < w.size(); ++k)
      if (w[k].first < w[k - 1].second) return true;
    return false;
  };
  if (meet()) return true;
  const int64_t s0 = (int64_t)w.front().first, s1 = (int64_t)w.back().second;
  const int64_t b0 = s0 / RES_ADAMW_BLOCK, b1 = (s1 + RES_ADAMW_BLOCK - 1) / RES_ADAMW_BLOCK;
  const size_t es = in.bits == 8 ? 1 : 4;
  const bool eight = in.bits == 8;
  struct Buffer {
    const void *from, *to;
    int64_t lo, hi;
    size_t es;
  };
  const Buffer buffers[] = {{in.m, out.m, s0, s1, es},
                            {in.v, out.v, s0, s1, es},
                            {eight ? in.scale_m : nullptr, eight ? out.scale_m : nullptr, b0, b1, 4},
                            {eight ? in.scale_v : nullptr, eight ? out.scale_v : nullptr, b0, b1, 4},
                            {in.master, out.master, s0, s1, 4}};
  // what is written
  w.clear();
  for (int64_t k = 0; k < count; ++k)
    if (t[k].n > 0) w.push_back(range(t[k].p_out, 0, t[k].n, pe));
  for (const Buffer& b : buffers)
    if (b.to != nullptr) w.push_back(range(b.to, b.lo, b.hi, b.es));
  if (meet()) return true;
  // what is read, but for what is written in its own place
  auto written = [&w](const Range& r) {
    auto it = std::lower_bound(w.begin(), w.end(), Range{r.second, 0});  // the first that begins behind r
    return it != w.begin() && (it - 1)->second > r.first;
  };
  for (int64_t k = 0; k < count; ++k)
    if (t[k].n > 0 && (written(range(t[k].g, 0, t[k].n, ge)) || (t[k].p != t[k].p_out && written(range(t[k].p, 0, t[k].n, pe)))))
      return true;
  for (const Buffer& b : buffers)
    if (b.from != nullptr && b.from != b.to && written(range(b.from, b.lo, b.hi, b.es))) return true;
  return scale != nullptr && written(range(scale, 0, 1, 4));
}

}  // namespace

extern "C" {

int resonator_adamw_step(const res_adamw_tensor_t* tensors, int64_t count, res_dtype_t p_dt, res_dtype_t g_dt,
                         const res_adamw_state_t* state, const res_adamw_state_t* state_out, double lr, double beta1,
                         double beta2, double eps, double weight_decay, int64_t step, const float* grad_scale,
                         void* stream) {
  if (!known(p_dt) || !known(g_dt)) return api_error(RES_ERR_INVALID_ARG, "unknown dtype code");
  if (count < 0 || (count > 0 && tensors == nullptr) || state == nullptr || state_out == nullptr)
    return api_error(RES_ERR_INVALID_ARG, "tensors, state and state_out must be non-null");
  if (state->bits != state_out->bits || (state->bits != 8 && state->bits != 32))
    return api_error(RES_ERR_INVALID_ARG, "states must be of 8 or of 32 bits, both of the same");
  if (!(lr >= 0) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(eps >= 0) || !(weight_decay >= 0) || step < 1)
    return api_error(RES_ERR_INVALID_ARG, "lr, eps and weight_decay must be >= 0, betas in [0, 1), step >= 1");
  const bool master = state->master != nullptr;
  if (master != (state_out->master != nullptr))
    return api_error(RES_ERR_INVALID_ARG, "master must be given in both states or in none");
  if (master && p_dt != RES_BF16)
    return api_error(RES_ERR_INVALID_ARG, "float32 parameters need no master copy");
  int64_t total = 0;
  for (int64_t k = 0; k < count; ++k) {
    const res_adamw_tensor_t& t = tensors[k];
    if (t.n < 0 || t.n > (1LL << 40) || t.state < 0 || t.state % RES_ADAMW_BLOCK || t.state > (1LL << 40))
      return api_error(RES_ERR_INVALID_ARG, "tensor %lld: n must be >= 0 and its state start at a multiple of %d",
                       (long long)k, RES_ADAMW_BLOCK);
    if (t.n == 0) continue;
    if (t.p == nullptr || t.g == nullptr || t.p_out == nullptr)
      return api_error(RES_ERR_INVALID_ARG, "tensor %lld: p, g and p_out must be non-null", (long long)k);
    if (!aligned(t.p, elt(p_dt)) || !aligned(t.p_out, elt(p_dt)) || !aligned(t.g, elt(g_dt)))
      return api_error(RES_ERR_MISALIGNED, "tensor %lld: pointers must be aligned to their element", (long long)k);
    total += t.n;
  }
  if (total == 0) return RES_OK;
  for (const res_adamw_state_t* s : {state, state_out}) {
    if (s->m == nullptr || s->v == nullptr || (s->bits == 8 && (s->scale_m == nullptr || s->scale_v == nullptr)))
      return api_error(RES_ERR_INVALID_ARG, "the states' tensors must be non-null");
    if (!aligned(s->m, 16) || !aligned(s->v, 16) || !aligned(s->scale_m, 4) || !aligned(s->scale_v, 4) || !aligned(s->master, 16))
      return api_error(RES_ERR_MISALIGNED, "m, v and master must be 16-byte aligned, scales 4-byte");
  }
  if (!aligned(grad_scale, 4)) return api_error(RES_ERR_MISALIGNED, "grad_scale must be 4-byte aligned");
  try {
    if (adamw_overlaps(tensors, count, elt(p_dt), elt(g_dt), *state, *state_out, grad_scale))
      return api_error(RES_ERR_INVALID_ARG, "what the step writes must not overlap what else it reads or writes (a new value may be "
                                            "in its old one's place; tensors and their states must not meet)");
  } catch (const std::bad_alloc&) {
    return api_error(RES_ERR_UNSUPPORTED, "no host memory for a table of %lld tensors", (long long)count);
  }
  AdamWArgs a{};
  a.m = state->m;
  a.v = state->v;
  a.sm = state->scale_m;
  a.sv = state->scale_v;
  a.master = state->master;
  a.m_out = state_out->m;
  a.v_out = state_out->v;
  a.sm_out = state_out->scale_m;
  a.sv_out = state_out->scale_v;
  a.master_out = state_out->master;
  a.grad_scale = grad_scale;
  a.b1 = (float)beta1;
  a.b1c = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.b2c = (float)(1.0 - beta2);
  a.eps = (float)eps;
  a.decay = (float)(1.0 - lr * weight_decay);
  a.step = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  return launched(launch_adamw(a, tensors, count, p_dt == RES_BF16, g_dt == RES_BF16, state->bits, (hipStream_t)stream),
                  "AdamW launch");
}

int resonator_adamw_values(const res_adamw_state_t* state, int64_t n, float* m, float* v, void* stream) {
  if (state == nullptr || state->bits != 8) return api_error(RES_ERR_INVALID_ARG, "state must be of 8 bits");
  if (n < 0 || n % RES_ADAMW_BLOCK || n > (1LL << 40))
    return api_error(RES_ERR_INVALID_ARG, "n must be a multiple of %d", RES_ADAMW_BLOCK);
  if (n == 0) return RES_OK;
  if (state->m == nullptr || state->v == nullptr || state->scale_m == nullptr || state->scale_v == nullptr ||
      m == nullptr || v == nullptr)
    return api_error(RES_ERR_INVALID_ARG, "the state's tensors, m and v must be non-null");
  if (!aligned(state->m, 16) || !aligned(state->v, 16) || !aligned(m, 16) || !aligned(v, 16) || !aligned(state->scale_m, 4) ||
      !aligned(state->scale_v, 4))
    return api_error(RES_ERR_MISALIGNED, "the codes, m and v must be 16-byte aligned, scales 4-byte");
  const size_t scales = n / RES_ADAMW_BLOCK * 4;
  for (float* o : {m, v})
    if (touch(flat(o, 4 * n), flat(state->m, n)) || touch(flat(o, 4 * n), flat(state->v, n)) ||
        touch(flat(o, 4 * n), flat(state->scale_m, scales)) || touch(flat(o, 4 * n), flat(state->scale_v, scales)))
      return api_error(RES_ERR_INVALID_ARG, "m and v must not overlap the codes or their scales");
  if (touch(flat(m, 4 * n), flat(v, 4 * n))) return api_error(RES_ERR_INVALID_ARG, "m and v must not overlap each other");
  return launched(launch_adamw_values(state->m, state->v, state->scale_m, state->scale_v, n, m, v, (hipStream_t)stream),
                  "AdamW values launch");
}

}  // extern "C"
