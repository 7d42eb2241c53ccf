// Host-side pieces shared by the C entry points: the last CUDA error of the thread, checks of
// AdamW hyper-parameters, pointers and ranges.
#pragma once
#include <cuda_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "abs_device.cuh"

namespace absnt {

// Remembers `e` for abs_last_cuda_error and returns ABS_ERR_CUDA.
int cuda_fail(cudaError_t e);

inline bool finite_nonneg(float x) { return std::isfinite(x) && x >= 0.f; }

inline int check_hparams(const abs_adamw_hparams* h, int64_t step) {
  if (!h) return ABS_ERR_NULL;
  if (step < 1) return ABS_ERR_RANGE;
  if (!finite_nonneg(h->lr) || !finite_nonneg(h->eps) || !finite_nonneg(h->weight_decay))
    return ABS_ERR_RANGE;
  if (!(h->beta1 >= 0.f && h->beta1 < 1.f) || !(h->beta2 >= 0.f && h->beta2 < 1.f))
    return ABS_ERR_RANGE;
  return ABS_OK;
}

inline AdamScalars make_adam(const abs_adamw_hparams* h, int64_t step) {
  AdamScalars a;
  const double b1 = h->beta1, b2 = h->beta2;
  a.beta1 = h->beta1;
  a.omb1 = static_cast<float>(1.0 - b1);
  a.beta2 = h->beta2;
  a.omb2 = static_cast<float>(1.0 - b2);
  a.step_size = static_cast<float>(static_cast<double>(h->lr) /
                                   (1.0 - std::pow(b1, static_cast<double>(step))));
  a.inv_bc2 = static_cast<float>(1.0 / (1.0 - std::pow(b2, static_cast<double>(step))));
  a.eps = h->eps;
  a.decay =
      static_cast<float>(1.0 - static_cast<double>(h->lr) * static_cast<double>(h->weight_decay));
  return a;
}

inline bool misaligned(const void* p, size_t a) {
  return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0;
}

// [a, a+na) and [b, b+nb) share a byte
inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + nb && b0 < a0 + na;
}

}  // namespace absnt
