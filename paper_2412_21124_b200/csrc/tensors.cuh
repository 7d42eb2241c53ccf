// Kernels over a list of tensors: the global norm (and the norm of each tensor), scaling by the
// clipping factor that follows from it, and AdamW on the clipped gradients.
//
// A list is cut into units: runs of `unit` consecutive elements of one tensor (the last one of a
// tensor is short).  The table of tensors and the tensor of each unit lie in device memory, written
// there once by the upload of the plan.
#pragma once
#include <cuda_fp16.h>

#include "abs_device.cuh"

namespace absnt {

constexpr int kTensorThreads = 256;
constexpr int kTensorWarps = kTensorThreads / 32;
constexpr int kMaxGroups = ABS_MAX_GROUPS;

// One tensor of the list.  A view with rows has `row` elements in each row, `stride` elements from
// one row to the next and `col` from one column to the next; element i lies at
// (i / row) * stride + (i % row) * col, and the quotient is (i * magic) >> (31 + shift) for every i
// below 2^31.
struct TensorEntry {
  const void* g;
  void* out;
  float *p, *m, *v;
  uint16_t* p16;
  int64_t numel;
  int64_t g_stride, g_col, out_stride, out_col;
  uint32_t g_row, g_magic, out_row, out_magic;
  int32_t first_unit, n_units;
  uint8_t g_shift, out_shift, g_dtype, out_dtype;
  uint8_t head;   // elements before the first one that lies on a vector boundary in every array
  uint8_t flags;  // kEntry* bits
  uint16_t group;
};
enum {
  kEntryRowsG = 1,     // the gradient has rows (else it is one run of elements)
  kEntryRowsOut = 2,   // so has the clipped output
  kEntryVecG = 4,      // from `head` on, 16-byte loads of the gradient are aligned
  kEntryVecClip = 8,   // from `head` on, 8 elements of gradient and output are
  kEntryVecAdam = 16,  // from `head` on, 8 elements of gradient, state and bf16 copy are
};

enum { kNormMax = ABS_NORM_MAX, kNorm1 = ABS_NORM_1, kNorm2 = ABS_NORM_2 };

struct TensorsParams {
  const TensorEntry* entries;
  const int32_t* unit_tensor;
  double* header;       // ABS_GRAD_* slots
  unsigned int* tickets;  // [0]: finished tensors, [1 + t]: finished units of tensor t
  double* tensor_sum;   // n
  double* unit_sum;     // n_units
  float* norms_out;     // 2 + n
  int n, n_units, n_nonempty, unit;
  int norm_type;
  double scale, max_norm;
  const double* sum_in;  // null: header[ABS_GRAD_SUM]
  int in_place;
};
struct GroupScalars {
  AdamScalars a[kMaxGroups];
};

// ---- element types -------------------------------------------------------------------
struct TF32 {
  using scalar = float;
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float to_float(float x) { return x; }
  static __device__ __forceinline__ float from_float(float x) { return x; }
  // the 16 bytes of a vector as floats, in ascending order
  static __device__ __forceinline__ void unpack(const uint4& r, float* x) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y);
    x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  }
};
struct TBF16 {
  using scalar = uint16_t;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float to_float(uint16_t x) {
    return __uint_as_float(static_cast<uint32_t>(x) << 16);
  }
  static __device__ __forceinline__ uint16_t from_float(float x) { return to_bf16(x); }
  static __device__ __forceinline__ void unpack(const uint4& r, float* x) {
    x[0] = bf16_lo(r.x), x[1] = bf16_hi(r.x), x[2] = bf16_lo(r.y), x[3] = bf16_hi(r.y);
    x[4] = bf16_lo(r.z), x[5] = bf16_hi(r.z), x[6] = bf16_lo(r.w), x[7] = bf16_hi(r.w);
  }
};
struct TF16 {
  using scalar = uint16_t;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float to_float(uint16_t x) {
    return __half2float(__ushort_as_half(x));
  }
  static __device__ __forceinline__ uint16_t from_float(float x) {
    return __half_as_ushort(__float2half_rn(x));
  }
  static __device__ __forceinline__ void unpack(const uint4& r, float* x) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = to_float(static_cast<uint16_t>(w[i] & 0xffffu));
      x[2 * i + 1] = to_float(static_cast<uint16_t>(w[i] >> 16));
    }
  }
};

// Calls f(type) with the element type of a dtype code.
template <typename F>
__device__ __forceinline__ void with_type(int dtype, F&& f) {
  if (dtype == ABS_BF16)
    f(TBF16{});
  else if (dtype == ABS_F32)
    f(TF32{});
  else
    f(TF16{});
}

// Where the elements of one unit lie in one array: offset of the unit's element i.
struct Span {
  int64_t base, stride, col_stride;
  uint32_t col, row, magic;
  int shift;
  bool rows;
  __device__ __forceinline__ int64_t at(uint32_t i) const {
    if (!rows) return base + i;
    const uint32_t idx = col + i;  // below 2^30 + 2^30
    const uint32_t q = static_cast<uint32_t>((static_cast<uint64_t>(idx) * magic) >> (31 + shift));
    return base + static_cast<int64_t>(q) * stride + static_cast<int64_t>(idx - q * row) * col_stride;
  }
};
__device__ __forceinline__ Span make_span(int64_t start, bool rows, uint32_t row, uint32_t magic,
                                          int shift, int64_t stride, int64_t col_stride) {
  if (!rows) return Span{start, 0, 0, 0, 0, 0, 0, false};
  const int64_t r0 = start / row;
  return Span{r0 * stride, stride, col_stride, static_cast<uint32_t>(start - r0 * row), row, magic,
              shift, true};
}
__device__ __forceinline__ Span grad_span(const TensorEntry& e, int64_t start) {
  return make_span(start, e.flags & kEntryRowsG, e.g_row, e.g_magic, e.g_shift, e.g_stride,
                   e.g_col);
}
__device__ __forceinline__ Span out_span(const TensorEntry& e, int64_t start) {
  return make_span(start, e.flags & kEntryRowsOut, e.out_row, e.out_magic, e.out_shift,
                   e.out_stride, e.out_col);
}

// The elements [start, start + n) of a unit; unit 0 also holds the head.
struct UnitRange {
  int64_t start;
  uint32_t n, head;
};
__device__ __forceinline__ UnitRange unit_range(const TensorEntry& e, int u, int unit) {
  const int k = u - e.first_unit;
  UnitRange r;
  r.start = k ? e.head + static_cast<int64_t>(k) * unit : 0;
  int64_t end = e.head + static_cast<int64_t>(k + 1) * unit;
  if (end > e.numel) end = e.numel;
  r.n = static_cast<uint32_t>(end - r.start);
  r.head = k ? 0u : (e.head < r.n ? e.head : r.n);
  return r;
}

// ---- the norm ------------------------------------------------------------------------
// Largest magnitude so far; a NaN stays.
__device__ __forceinline__ float max_abs(float acc, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(acc), "f"(fabsf(x)));
  return r;
}

// Running sum of one thread: |x|, x^2 or max |x|.  The values of a 16-byte vector are added in
// fp32 (their products of 8-bit significands are exact there), the vectors in fp64.
template <int NORM>
struct NormAcc {
  double s = 0.0;
  float mx = 0.f;
  uint32_t bits = 0;  // any bit set: not every value is +0
  template <int N>
  __device__ __forceinline__ void add(const float* x) {
    if constexpr (NORM == kNormMax) {
#pragma unroll
      for (int i = 0; i < N; ++i) mx = max_abs(mx, x[i]);
    } else {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) t = NORM == kNorm2 ? fmaf(x[i], x[i], t) : t + fabsf(x[i]);
      s += static_cast<double>(t);
    }
  }
};

// max in fp64 that keeps a NaN
__device__ __forceinline__ double max_keep_nan(double a, double b) {
  return (a != a || b != b) ? __longlong_as_double(0x7ff8000000000000ll) : (a > b ? a : b);
}
template <int NORM>
__device__ __forceinline__ double norm_join(double a, double b) {
  return NORM == kNormMax ? max_keep_nan(a, b) : a + b;
}

// Joins one value per thread in a fixed order; the result is in every thread.
template <int NORM>
__device__ __forceinline__ double block_join(double x, double* sm) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
    x = norm_join<NORM>(x, __shfl_down_sync(0xffffffffu, x, off));
  if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = x;
  __syncthreads();
  double r = sm[0];
#pragma unroll
  for (int w = 1; w < kTensorWarps; ++w) r = norm_join<NORM>(r, sm[w]);
  __syncthreads();
  return r;
}

// One thread's share of a unit.
template <typename T, int NORM>
__device__ __forceinline__ NormAcc<NORM> unit_acc(const TensorEntry& e, const UnitRange& r) {
  using S = typename T::scalar;
  constexpr int kBatch = 8;
  NormAcc<NORM> acc;
  const S* g = static_cast<const S*>(e.g);
  const Span sp = grad_span(e, r.start);
  const uint32_t tid = threadIdx.x;
  auto one = [&](uint32_t i) {
    const S raw = g[sp.at(i)];
    const float x = T::to_float(raw);
    acc.bits |= __float_as_uint(x);
    acc.template add<1>(&x);
  };
  if (e.flags & kEntryVecG) {
    if (tid < r.head) one(tid);
    const uint32_t nv = (r.n - r.head) / T::kVec;
    for (uint32_t v0 = tid; v0 < nv; v0 += kBatch * kTensorThreads) {
      uint4 raw[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t v = v0 + j * kTensorThreads;
        raw[j] = v < nv ? ld_once_16(g + sp.at(r.head + v * T::kVec)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        float x[T::kVec];
        T::unpack(raw[j], x);
        acc.bits |= raw[j].x | raw[j].y | raw[j].z | raw[j].w;
        acc.template add<T::kVec>(x);
      }
    }
    const uint32_t i = r.head + nv * T::kVec + tid;
    if (i < r.n) one(i);
  } else {
    for (uint32_t i0 = tid; i0 < r.n; i0 += kBatch * kTensorThreads) {
      float x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t i = i0 + j * kTensorThreads;
        x[j] = i < r.n ? T::to_float(g[sp.at(i)]) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) acc.bits |= __float_as_uint(x[j]);
      acc.template add<kBatch>(x);
    }
  }
  return acc;
}

// The same sum with every product in fp64, for units whose fp32 products leave the range.
template <typename T, int NORM>
__device__ __noinline__ double unit_acc_wide(const TensorEntry& e, const UnitRange& r) {
  using S = typename T::scalar;
  const S* g = static_cast<const S*>(e.g);
  const Span sp = grad_span(e, r.start);
  double s = 0.0;
  for (uint32_t i = threadIdx.x; i < r.n; i += kTensorThreads) {
    const double x = T::to_float(g[sp.at(i)]);
    s += NORM == kNorm2 ? x * x : fabs(x);
  }
  return s;
}

// What a caller makes of the power sum: the norm, the clipping coefficient and the factor that
// gradients are multiplied by.  A norm that is not finite clips nothing and raises the flag.
struct Clip {
  double norm, coef;
  float factor;
  bool finite;
};
__device__ __forceinline__ Clip clip_of(double sum, int norm_type, double scale, double max_norm) {
  Clip c;
  c.norm = fabs(scale) * (norm_type == kNorm2 ? sqrt(sum) : sum);
  c.finite = isfinite(c.norm);
  c.coef = 1.0;
  if (max_norm > 0.0 && c.finite) {
    const double k = max_norm / (c.norm + 1e-6);
    if (k < 1.0) c.coef = k;
  }
  c.factor = static_cast<float>(scale * c.coef);
  return c;
}
__device__ __forceinline__ void write_clip(const TensorsParams& prm, double sum, const Clip& c) {
  prm.header[ABS_GRAD_SUM] = sum;
  prm.header[ABS_GRAD_NORM] = c.norm;
  prm.header[ABS_GRAD_COEF] = c.coef;
  prm.header[ABS_GRAD_FLAGS] = c.finite ? 0.0 : static_cast<double>(ABS_FLAG_NONFINITE);
  prm.norms_out[0] = static_cast<float>(c.norm);
  prm.norms_out[1] = static_cast<float>(c.coef);
}

// Closes the list: the sums of all tensors are joined in order (by the block of the last unit).
template <int NORM>
__device__ __forceinline__ void close_list(const TensorsParams& prm, double* sm) {
  double s = 0.0;
  for (int t = threadIdx.x; t < prm.n; t += kTensorThreads) {
    const double x = __ldcg(prm.tensor_sum + t);
    s = norm_join<NORM>(s, x);
    prm.norms_out[2 + t] =
        static_cast<float>(fabs(prm.scale) * (NORM == kNorm2 ? sqrt(x) : x));
  }
  s = block_join<NORM>(s, sm);
  if (threadIdx.x == 0) write_clip(prm, s, clip_of(s, NORM, prm.scale, prm.max_norm));
}

// One CTA per unit.  The last unit of a tensor to finish adds that tensor's units in order, the
// last tensor to finish adds the tensors: one launch, and no order of finishing shows in the sums.
template <int NORM>
__global__ void __launch_bounds__(kTensorThreads)
    tensors_norm_kernel(const __grid_constant__ TensorsParams prm) {
  __shared__ double sm[kTensorWarps];
  __shared__ unsigned int s_ticket;
  grid_dependency_wait();
  if (prm.n_units == 0) {  // only empty tensors, or none
    close_list<NORM>(prm, sm);
    return;
  }
  const int u = blockIdx.x;
  const int t = prm.unit_tensor[u];
  const TensorEntry& e = prm.entries[t];
  const UnitRange r = unit_range(e, u, prm.unit);
  double x = 0.0;
  with_type(e.g_dtype, [&](auto type) {
    using T = decltype(type);
    const NormAcc<NORM> acc = unit_acc<T, NORM>(e, r);
    x = block_join<NORM>(NORM == kNormMax ? static_cast<double>(acc.mx) : acc.s, sm);
    if constexpr (NORM != kNormMax) {
      // fp32 squares overflow above 1.8e19 and lose bits below 1e-19; sums of |x| overflow
      // near the largest float.  A unit whose sum says so is taken again in fp64.
      const bool wide = !(x < 0x1p120) || (NORM == kNorm2 && x < 0x1p-90);
      if (wide && __syncthreads_or(acc.bits != 0))
        x = block_join<NORM>(unit_acc_wide<T, NORM>(e, r), sm);
    }
  });
  grid_launch_dependents();
  if (e.n_units > 1) {
    if (threadIdx.x == 0) {
      prm.unit_sum[u] = x;
      __threadfence();
      s_ticket = atomicAdd(prm.tickets + 1 + t, 1u);
    }
    __syncthreads();
    if (s_ticket != static_cast<unsigned>(e.n_units - 1)) return;
    __threadfence();
    x = 0.0;
    for (int k = threadIdx.x; k < e.n_units; k += kTensorThreads)
      x = norm_join<NORM>(x, __ldcg(prm.unit_sum + e.first_unit + k));
    x = block_join<NORM>(x, sm);
    if (threadIdx.x == 0) prm.tickets[1 + t] = 0;  // ready for the next call
  }
  if (threadIdx.x == 0) {
    prm.tensor_sum[t] = x;
    __threadfence();
    s_ticket = atomicAdd(prm.tickets, 1u);
  }
  __syncthreads();
  if (s_ticket != static_cast<unsigned>(prm.n_nonempty - 1)) return;
  __threadfence();
  if (threadIdx.x == 0) prm.tickets[0] = 0;
  close_list<NORM>(prm, sm);
}

// ---- scaling -------------------------------------------------------------------------
// The factor that this call's gradients are multiplied by, the same in every thread.
__device__ __forceinline__ Clip block_clip(const TensorsParams& prm, Clip* sm) {
  if (threadIdx.x == 0) {
    const double sum = __ldcg(prm.sum_in ? prm.sum_in : prm.header + ABS_GRAD_SUM);
    *sm = clip_of(sum, prm.norm_type, prm.scale, prm.max_norm);
    // a sum from elsewhere (added up over ranks): norm and coefficient follow it
    if (prm.sum_in && blockIdx.x == 0) write_clip(prm, sum, *sm);
  }
  __syncthreads();
  return *sm;
}

// Eight consecutive values, 16- or 32-byte aligned.
template <typename T>
struct Vec8 {
  uint4 r[8 / T::kVec];
};
template <typename T>
__device__ __forceinline__ Vec8<T> load8(const typename T::scalar* p) {
  Vec8<T> x;
#pragma unroll
  for (int i = 0; i < 8 / T::kVec; ++i) x.r[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  return x;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Vec8<T>& v, float* x) {
#pragma unroll
  for (int i = 0; i < 8 / T::kVec; ++i) T::unpack(v.r[i], x + i * T::kVec);
}
template <typename T>
__device__ __forceinline__ void store8(typename T::scalar* p, const float* x) {
  if constexpr (T::kVec == 4) {
    st_stream_32(p, make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = static_cast<uint32_t>(T::from_float(x[2 * i])) |
             (static_cast<uint32_t>(T::from_float(x[2 * i + 1])) << 16);
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
  }
}

template <typename TI, typename TO>
__device__ __forceinline__ void unit_scale(const TensorEntry& e, const UnitRange& r, float factor,
                                           const void* in, void* out, const Span& si,
                                           const Span& so, bool vec) {
  const typename TI::scalar* g = static_cast<const typename TI::scalar*>(in);
  typename TO::scalar* y = static_cast<typename TO::scalar*>(out);
  const uint32_t tid = threadIdx.x;
  auto one = [&](uint32_t i) {
    y[so.at(i)] = TO::from_float(factor * TI::to_float(g[si.at(i)]));
  };
  if (vec) {
    constexpr int kBatch = 4;
    if (tid < r.head) one(tid);
    const uint32_t nv = (r.n - r.head) / 8;
    for (uint32_t v0 = tid; v0 < nv; v0 += kBatch * kTensorThreads) {
      Vec8<TI> raw[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t v = v0 + j * kTensorThreads;
        if (v < nv) raw[j] = load8<TI>(g + si.at(r.head + v * 8));
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t v = v0 + j * kTensorThreads;
        if (v < nv) {
          float x[8];
          unpack8<TI>(raw[j], x);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= factor;
          store8<TO>(y + so.at(r.head + v * 8), x);
        }
      }
    }
    const uint32_t i = r.head + nv * 8 + tid;
    if (i < r.n) one(i);
  } else {
    constexpr int kBatch = 8;
    for (uint32_t i0 = tid; i0 < r.n; i0 += kBatch * kTensorThreads) {
      float x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t i = i0 + j * kTensorThreads;
        x[j] = i < r.n ? TI::to_float(g[si.at(i)]) : 0.f;
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t i = i0 + j * kTensorThreads;
        if (i < r.n) y[so.at(i)] = TO::from_float(factor * x[j]);
      }
    }
  }
}

__global__ void __launch_bounds__(kTensorThreads)
    tensors_scale_kernel(const __grid_constant__ TensorsParams prm) {
  __shared__ Clip s_clip;
  grid_dependency_wait();
  const Clip clip = block_clip(prm, &s_clip);
  if (prm.n_units == 0) return;
  if (prm.in_place && clip.factor == 1.f) return;  // x * 1 is x
  const int u = prm.n_units - 1 - blockIdx.x;  // last read, first scaled: it may still be in L2
  const TensorEntry& e = prm.entries[prm.unit_tensor[u]];
  const UnitRange r = unit_range(e, u, prm.unit);
  with_type(e.g_dtype, [&](auto ti) {
    using TI = decltype(ti);
    if (prm.in_place) {
      const Span sp = grad_span(e, r.start);
      // one array only: 8 elements are aligned wherever 16-byte loads are, for 16-bit types; fp32
      // vectors of 8 want 32 bytes
      const bool vec = e.flags & kEntryVecClip;
      unit_scale<TI, TI>(e, r, clip.factor, e.g, const_cast<void*>(e.g), sp, sp, vec);
    } else {
      with_type(e.out_dtype, [&](auto to) {
        using TO = decltype(to);
        unit_scale<TI, TO>(e, r, clip.factor, e.g, e.out, grad_span(e, r.start),
                           out_span(e, r.start), e.flags & kEntryVecClip);
      });
    }
  });
}

// ---- AdamW ---------------------------------------------------------------------------
// Four neighbouring coordinates.
__device__ __forceinline__ void adamw_quad(const AdamScalars& a, float2 g0, float2 g1, float4& w,
                                           float4& m, float4& v) {
  float2 w0 = make_float2(w.x, w.y), w1 = make_float2(w.z, w.w);
  float2 m0 = make_float2(m.x, m.y), m1 = make_float2(m.z, m.w);
  float2 v0 = make_float2(v.x, v.y), v1 = make_float2(v.z, v.w);
  adamw_pair(a, a.omb1, a.omb2, g0, w0, m0, v0);
  adamw_pair(a, a.omb1, a.omb2, g1, w1, m1, v1);
  w = make_float4(w0.x, w0.y, w1.x, w1.y);
  m = make_float4(m0.x, m0.y, m1.x, m1.y);
  v = make_float4(v0.x, v0.y, v1.x, v1.y);
}

__global__ void __launch_bounds__(kTensorThreads)
    tensors_adamw_kernel(const __grid_constant__ TensorsParams prm,
                         const __grid_constant__ GroupScalars groups, int clipped) {
  __shared__ Clip s_clip;
  grid_dependency_wait();
  float factor = static_cast<float>(prm.scale);
  if (clipped) {
    const Clip clip = block_clip(prm, &s_clip);
    if (!clip.finite) return;  // no update from a gradient that is not finite
    factor = clip.factor;
  }
  if (prm.n_units == 0) return;
  const int u = prm.n_units - 1 - blockIdx.x;
  const TensorEntry& e = prm.entries[prm.unit_tensor[u]];
  const UnitRange r = unit_range(e, u, prm.unit);
  const AdamScalars& a = groups.a[e.group];
  const Span sp = grad_span(e, r.start);
  float *p = e.p + r.start, *m = e.m + r.start, *v = e.v + r.start;
  uint16_t* p16 = e.p16 ? e.p16 + r.start : nullptr;
  const uint32_t tid = threadIdx.x;
  with_type(e.g_dtype, [&](auto type) {
    using T = decltype(type);
    const typename T::scalar* g = static_cast<const typename T::scalar*>(e.g);
    auto one = [&](uint32_t i) {
      float w = p[i], mi = m[i], vi = v[i];
      adamw_elem(a, a.omb1, a.omb2, factor * T::to_float(g[sp.at(i)]), w, mi, vi);
      p[i] = w, m[i] = mi, v[i] = vi;
      if (p16) p16[i] = to_bf16(w);
    };
    if (e.flags & kEntryVecAdam) {
      if (tid < r.head) one(tid);
      const uint32_t nv = (r.n - r.head) / 8;
      for (uint32_t q = tid; q < nv; q += kTensorThreads) {
        const uint32_t i = r.head + q * 8;
        const Vec8<T> raw = load8<T>(g + sp.at(i));
        Float8 w = ld_state_32(p + i), mm = ld_state_32(m + i), vv = ld_state_32(v + i);
        float x[8];
        unpack8<T>(raw, x);
        const float2 g0 = make_float2(factor * x[0], factor * x[1]);
        const float2 g1 = make_float2(factor * x[2], factor * x[3]);
        const float2 g2 = make_float2(factor * x[4], factor * x[5]);
        const float2 g3 = make_float2(factor * x[6], factor * x[7]);
        adamw_quad(a, g0, g1, w.lo, mm.lo, vv.lo);
        adamw_quad(a, g2, g3, w.hi, mm.hi, vv.hi);
        st_stream_32(p + i, w.lo, w.hi);
        st_stream_32(m + i, mm.lo, mm.hi);
        st_stream_32(v + i, vv.lo, vv.hi);
        if (p16) st_bf16x8(p16 + i, w.lo, w.hi);
      }
      const uint32_t i = r.head + nv * 8 + tid;
      if (i < r.n) one(i);
    } else {
      for (uint32_t i = tid; i < r.n; i += kTensorThreads) one(i);
    }
  });
}

}  // namespace absnt
