// Argument checks and small host helpers shared by the entry points.
#pragma once

#include <math.h>
#include <stdint.h>

#include "../../include/mea.h"
#include "kernels.hpp"

namespace mea_host {

constexpr int64_t kMaxSeq = (int64_t)1 << 31;  // n_q, n_k must stay below 2^31

inline bool mul_ok(int64_t a, int64_t b, int64_t* out) {
  if (a < 0 || b < 0) return false;
  if (a != 0 && b > INT64_MAX / a) return false;
  *out = a * b;
  return true;
}

// Head dimension of v and o (d_v = 0 means d).
inline int64_t dv_of(const mea_problem* p) { return p->d_v ? p->d_v : p->d; }

// Shape, dtype and scale checks shared by every entry point.
inline mea_status check_problem(const mea_problem* p) {
  if (!p) return MEA_ERR_INVALID_ARG;
  if (p->batch < 1 || p->heads < 1 || p->n_q < 1 || p->n_k < 1 || p->d < 1)
    return MEA_ERR_INVALID_ARG;
  if (p->n_q >= kMaxSeq || p->n_k >= kMaxSeq) return MEA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return MEA_ERR_INVALID_ARG;
  if (p->out_f32 != 0 && p->out_f32 != 1) return MEA_ERR_INVALID_ARG;
  if (!(p->scale > 0.0f) || !isfinite(p->scale)) return MEA_ERR_INVALID_ARG;
  if (p->kv_len && ((uintptr_t)p->kv_len & 3u)) return MEA_ERR_INVALID_ARG;
  if (p->d_v < 0) return MEA_ERR_INVALID_ARG;
  const int64_t dmax = p->d > dv_of(p) ? p->d : dv_of(p);
  int64_t bh, nq_d, nk_d, tot;
  if (!mul_ok(p->batch, p->heads, &bh) || bh >= kMaxSeq) return MEA_ERR_INVALID_ARG;
  if (!mul_ok(p->n_q, dmax, &nq_d) || !mul_ok(p->n_k, dmax, &nk_d)) return MEA_ERR_INVALID_ARG;
  if (!mul_ok(bh, nq_d, &tot) || !mul_ok(bh, nk_d, &tot)) return MEA_ERR_INVALID_ARG;
  if (!mul_ok(bh, p->n_q * 4, &tot)) return MEA_ERR_INVALID_ARG;
  if (p->d != 64 && p->d != 128) return MEA_ERR_UNSUPPORTED;
  if (dv_of(p) != 64 && dv_of(p) != 128) return MEA_ERR_UNSUPPORTED;
  if (p->dtype != MEA_F32 && p->dtype != MEA_F16 && p->dtype != MEA_BF16) return MEA_ERR_UNSUPPORTED;
  return MEA_OK;
}

// Strides of a tensor of n rows of w features: given, or contiguous [B, heads, n, w].
inline mea::TensorStrides strides_of(const mea_tensor_strides* given, int64_t heads, int64_t n, int64_t w) {
  if (given) return {given->batch, given->head, given->row};
  return {heads * n * w, n * w, w};
}

// Validation of one tensor's strides (see mea.h); w = features per row.
inline bool strides_ok(int64_t batch, int64_t heads, const mea::TensorStrides& s, int64_t n, bool output, size_t elem,
                int64_t w) {
  const int64_t align = 16 / (int64_t)elem;
  if (s.b < 0 || s.h < 0 || s.r < w || s.r >= ((int64_t)1 << 24)) return false;
  if (output && (s.b == 0 || s.h == 0)) return false;
  if (s.b % align || s.h % align || s.r % align) return false;
  int64_t a, b, c, tot;
  if (!mul_ok(batch - 1, s.b, &a) || !mul_ok(heads - 1, s.h, &b) || !mul_ok(n - 1, s.r, &c)) return false;
  if (__builtin_add_overflow(a, b, &tot) || __builtin_add_overflow(tot, c, &tot) ||
      __builtin_add_overflow(tot, w, &tot))
    return false;
  return true;
}

inline size_t elem_size(int32_t dtype) { return dtype == MEA_F32 ? 4 : 2; }

inline bool aligned16(const void* ptr) { return ((uintptr_t)ptr & 15u) == 0; }
inline bool dev_ptr_ok(const void* ptr) { return ptr != nullptr && aligned16(ptr); }

inline float* align256(void* base, size_t off) {
  uintptr_t a = (uintptr_t)base + off;
  a = (a + 255u) & ~(uintptr_t)255u;
  return reinterpret_cast<float*>(a);
}

constexpr float kLog2e = 1.4426950408889634f;

}  // namespace mea_host
