// Argument checks that the C entry points of the layers' operators share.
#pragma once

#include <cstdint>

#include "../../include/resonator.h"
#include "layer.h"

namespace res {

inline size_t elt(res_dtype_t t) { return t == RES_BF16 ? 2 : 4; }
inline bool known(int t) { return t == RES_F32 || t == RES_BF16; }
inline bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

inline int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? RES_OK : api_error(RES_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// The bytes that rows [B][L] of D elements of `es` bytes reach over, and whether two such sets share any.
struct Span {
  uintptr_t lo, hi;     // [lo, hi)
  int64_t sb, st, row;  // strides and row length in bytes
  int64_t B, L;
};
inline Span span(const void* p, int64_t sb, int64_t st, int64_t B, int64_t L, int64_t D, size_t es) {
  Span s{(uintptr_t)p, (uintptr_t)p, sb * (int64_t)es, st * (int64_t)es, D * (int64_t)es, B, L};
  if (p != nullptr && B > 0 && L > 0) s.hi += (B - 1) * s.sb + (L - 1) * s.st + s.row;
  return s;
}
inline Span flat(const void* p, size_t bytes) {
  return Span{(uintptr_t)p, (uintptr_t)p + (p != nullptr ? bytes : 0), (int64_t)bytes, (int64_t)bytes, (int64_t)bytes, 1, 1};
}
inline bool touch(const Span& a, const Span& b) {
  if (a.lo == a.hi || b.lo == b.hi || a.hi <= b.lo || b.hi <= a.lo) return false;
  // columns of one wider tensor, whichever axis is outermost: every distance between rows is a multiple of the least, and
  // within that the columns do not meet
  const int64_t by[4] = {a.B > 1 ? a.sb : 0, a.L > 1 ? a.st : 0, b.B > 1 ? b.sb : 0, b.L > 1 ? b.st : 0};
  int64_t least = 0;
  for (int64_t s : by)
    if (s > 0 && (least == 0 || s < least)) least = s;
  if (least == 0) return true;
  for (int64_t s : by)
    if (s % least != 0) return true;
  const int64_t d = (((int64_t)(b.lo - a.lo)) % least + least) % least;  // b's first column after a's
  return !(d >= a.row && d + b.row <= least);
}
// whether the rows of an output lie apart from each other
inline bool rows_apart(int64_t sb, int64_t st, int64_t B, int64_t L, int64_t D) {
  if (B <= 1 && L <= 1) return true;
  if (B <= 1) return st >= D;
  if (L <= 1) return sb >= D;
  return (st >= D && sb >= (L - 1) * st + D) || (sb >= D && st >= (B - 1) * sb + D);
}

inline int check_rows(const char* name, const void* p, int64_t sb, int64_t st, int64_t L, size_t es) {
  if (p == nullptr) return api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name);
  if (!aligned(p, es)) return api_error(RES_ERR_MISALIGNED, "%s must be aligned to its element", name);
  // (a tile's bytes have 32-bit offsets; one step has no distance to a next one)
  if (sb < 0 || sb > (1LL << 40) || (L > 1 && (st < 0 || st > (1LL << 21))))
    return api_error(RES_ERR_UNSUPPORTED, "%s: strides must be in [0, 2^40] (rows) and [0, 2^21] (steps) elements", name);
  return RES_OK;
}

inline int check_f32(const char* name, const float* p, bool needed) {
  if (p == nullptr) return needed ? api_error(RES_ERR_INVALID_ARG, "%s must be non-null", name) : RES_OK;
  return aligned(p, 4) ? RES_OK : api_error(RES_ERR_MISALIGNED, "%s must be 4-byte aligned", name);
}

}  // namespace res
