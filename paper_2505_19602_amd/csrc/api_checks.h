// Argument checks of the C ABI that its translation units share.  Host code; a failing check leaves its message for
// scalekv_last_error().
#pragma once
#include <math.h>

#include "../../include/scalekv.h"
#include "common.h"

namespace scalekv {

// records the message and returns st
scalekv_status fail(scalekv_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

inline scalekv_status hip_fail(hipError_t e, const char* what) {
  return fail(SCALEKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int elem_bytes(const scalekv_shape* s) { return s->dtype == SCALEKV_F32 ? 4 : 2; }

inline float resolve_scale(const scalekv_shape* s) {
  return s->sm_scale > 0.f ? s->sm_scale : 1.0f / sqrtf((float)s->head_dim);
}

inline scalekv_status check_shape(const scalekv_shape* s) {
  if (!s) return fail(SCALEKV_ERR_INVALID_ARG, "shape is NULL");
  if (s->n_seq <= 0 || s->n_head <= 0)
    return fail(SCALEKV_ERR_INVALID_ARG, "n_seq and n_head must be positive (got %d, %d)",
                s->n_seq, s->n_head);
  if ((long long)s->n_seq * s->n_head > 65535)
    return fail(SCALEKV_ERR_UNSUPPORTED, "n_seq * n_head = %lld exceeds 65535",
                (long long)s->n_seq * s->n_head);
  if (s->dtype != SCALEKV_F32 && s->dtype != SCALEKV_BF16)
    return fail(SCALEKV_ERR_UNSUPPORTED, "dtype %d is neither SCALEKV_F32 nor SCALEKV_BF16",
                s->dtype);
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail(SCALEKV_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", s->head_dim);
  if (!(s->sm_scale == s->sm_scale))
    return fail(SCALEKV_ERR_INVALID_ARG, "sm_scale is NaN");
  return SCALEKV_OK;
}

// rows * head_dim must fit int32 (kernels index a unit with 32-bit offsets in places)
inline scalekv_status check_rows(const scalekv_shape* s, long long rows, const char* name) {
  if (rows < 0) return fail(SCALEKV_ERR_INVALID_ARG, "%s is negative (%lld)", name, rows);
  if (rows * s->head_dim > 0x7fffffffLL)
    return fail(SCALEKV_ERR_UNSUPPORTED, "%s = %lld rows is too large", name, rows);
  return SCALEKV_OK;
}

inline scalekv_status check_kv(const scalekv_shape* s, const scalekv_kv* kv, int rows_needed,
                        const char* name) {
  if (!kv) return fail(SCALEKV_ERR_INVALID_ARG, "%s is NULL", name);
  if (!kv->ptr) return fail(SCALEKV_ERR_INVALID_ARG, "%s.ptr is NULL", name);
  if (!aligned16(kv->ptr)) return fail(SCALEKV_ERR_INVALID_ARG, "%s.ptr is not 16-byte aligned", name);
  if (kv->capacity < 0) return fail(SCALEKV_ERR_INVALID_ARG, "%s.capacity is negative", name);
  if (rows_needed > kv->capacity)
    return fail(SCALEKV_ERR_INVALID_ARG, "%s: %d rows needed but capacity is %d", name,
                rows_needed, kv->capacity);
  const long long unit = (long long)kv->capacity * s->head_dim;
  const int epv = 16 / elem_bytes(s);
  if (kv->head_stride < unit || kv->head_stride % epv)
    return fail(SCALEKV_ERR_INVALID_ARG,
                "%s.head_stride %lld must be >= capacity*head_dim (%lld) and a multiple of %d",
                name, (long long)kv->head_stride, unit, epv);
  if (kv->seq_stride < kv->head_stride * s->n_head || kv->seq_stride % epv)
    return fail(SCALEKV_ERR_INVALID_ARG,
                "%s.seq_stride %lld must be >= n_head*head_stride and a multiple of %d", name,
                (long long)kv->seq_stride, epv);
  return SCALEKV_OK;
}

inline scalekv_status check_dense(const void* p, bool required, const char* name) {
  if (!p) return required ? fail(SCALEKV_ERR_INVALID_ARG, "%s is NULL", name) : SCALEKV_OK;
  if (!aligned16(p)) return fail(SCALEKV_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return SCALEKV_OK;
}

// byte range [lo, hi) spanned by a cache
inline void kv_span(const scalekv_shape* s, const scalekv_kv* kv, uintptr_t* lo, uintptr_t* hi) {
  const long long e = elem_bytes(s);
  *lo = reinterpret_cast<uintptr_t>(kv->ptr);
  *hi = *lo + (uintptr_t)(((long long)(s->n_seq - 1) * kv->seq_stride +
                           (long long)(s->n_head - 1) * kv->head_stride +
                           (long long)kv->capacity * s->head_dim) * e);
}

#define SCALEKV_TRY(expr)                       \
  do {                                          \
    scalekv_status _st = (expr);                \
    if (_st != SCALEKV_OK) return _st;          \
  } while (0)

#define SCALEKV_HIP(expr, what)                 \
  do {                                          \
    hipError_t _e = (expr);                     \
    if (_e != hipSuccess) return hip_fail(_e, what); \
  } while (0)

}  // namespace scalekv
