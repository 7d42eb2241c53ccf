// Kernels over a list of tensors: the global norm (and the norm of each tensor), scaling by the
// clipping factor that follows from it, and AdamW on the clipped gradients.
//
// A list is cut in two ways.  For the norm every warp of a fixed number of warps gets an equal share
// of the list's bytes, a run of whole 512-byte rows that is cut into segments where a tensor ends.
// For scaling and AdamW, which join nothing, it is cut into units: runs of `unit` consecutive
// elements of one tensor, one CTA each.  The tables lie in device memory, written there once by the
// upload of the plan.
#pragma once
#include <cuda_fp16.h>

#include "abs_device.cuh"

namespace absnt {

constexpr int kTensorThreads = 256;
constexpr int kMaxGroups = ABS_MAX_GROUPS;

// One tensor of the list.  A view with rows has `row` elements in each row, `stride` elements from
// one row to the next and `col` from one column to the next; element i lies at
// (i / row) * stride + (i % row) * col.
struct TensorEntry {
  const void* g;
  void* out;
  float *p, *m, *v;
  uint16_t* p16;
  int64_t numel;
  int64_t g_stride, g_col, out_stride, out_col;
  uint32_t g_row, out_row;
  int32_t first_unit, n_units;
  int32_t first_seg, n_segs;
  uint8_t g_dtype, out_dtype;
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

// A run of elements of one tensor, the work of one warp: [start, start + n), `head` of them before
// the first 16-byte boundary.
struct Segment {
  const void* g;  // of element `start`, for a gradient without rows
  int64_t start;
  uint32_t n;
  int32_t tensor;
  uint8_t dtype, vec, rows, head;
  int32_t pad;
};
constexpr int kNormThreads = 1024;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kNormCtas = 148;  // one for each SM

// A tensor whose segments lie in several blocks, first..last.
struct Spanning {
  int32_t tensor, first, last, pad;
};

enum { kNormMax = ABS_NORM_MAX, kNorm1 = ABS_NORM_1, kNorm2 = ABS_NORM_2 };

struct TensorsParams {
  const TensorEntry* entries;
  const int32_t* unit_tensor;
  const Segment* segments;
  const int32_t* warp_first;  // first segment of each warp, and the number of segments
  const Spanning* spanning;
  const int32_t* empty;  // tensors without elements
  double* header;         // ABS_GRAD_* slots
  unsigned int* ticket;   // blocks that have finished
  double* block_sum;      // kNormCtas
  double* edge_sum;       // 2 kNormCtas: each block's part of its first and of its last tensor
  float* norms_out;       // 2 + n
  int n, n_units, unit, n_segments, n_warps, n_spanning, n_empty;
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

// Walks the elements start + i0, start + i0 + step, ... of a view: `offset()` of the current one,
// `next()` to the one `step` further.  One division at the beginning, none on the way.
struct Walk {
  int64_t off, step_off, wrap_off;
  uint32_t col, step_col, row;
  __device__ __forceinline__ int64_t offset() const { return off; }
  __device__ __forceinline__ void next() {
    off += step_off;
    col += step_col;
    if (col >= row) {
      col -= row;
      off += wrap_off;
    }
  }
};
__device__ __forceinline__ Walk make_walk(int64_t first, uint32_t step, bool rows, uint32_t row,
                                          int64_t stride, int64_t col_stride) {
  if (!rows) return Walk{first, step, 0, 0, 0, 1};
  const int64_t r = first / row;
  const uint32_t c = static_cast<uint32_t>(first - r * row);
  const uint32_t dr = step / row, dc = step - dr * row;
  return Walk{r * stride + c * col_stride, dr * stride + dc * col_stride,
              stride - static_cast<int64_t>(row) * col_stride, c, dc, row};
}
__device__ __forceinline__ Walk grad_walk(const TensorEntry& e, int64_t first, uint32_t step) {
  return make_walk(first, step, e.flags & kEntryRowsG, e.g_row, e.g_stride, e.g_col);
}
__device__ __forceinline__ Walk out_walk(const TensorEntry& e, int64_t first, uint32_t step) {
  return make_walk(first, step, e.flags & kEntryRowsOut, e.out_row, e.out_stride, e.out_col);
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

template <int NORM>
__device__ __forceinline__ double warp_join(double x) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
    x = norm_join<NORM>(x, __shfl_xor_sync(0xffffffffu, x, off));
  return x;
}

// One lane's share of a segment.
template <typename T, int NORM>
__device__ __forceinline__ NormAcc<NORM> segment_acc(const TensorsParams& prm, const Segment& s,
                                                     uint32_t lane) {
  using S = typename T::scalar;
  constexpr int kBatch = 8;
  NormAcc<NORM> acc;
  auto one = [&](S raw) {
    const float x = T::to_float(raw);
    acc.bits |= __float_as_uint(x);
    acc.template add<1>(&x);
  };
  if (s.vec) {
    const S* g = static_cast<const S*>(s.g);
    if (lane < s.head) one(g[lane]);
    const uint32_t nv = (s.n - s.head) / T::kVec;
    const S* gv = g + s.head;
    for (uint32_t v0 = lane; v0 < nv; v0 += kBatch * 32) {
      uint4 raw[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t v = v0 + j * 32;
        raw[j] = v < nv ? ld_once_16(gv + static_cast<size_t>(v) * T::kVec) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        float x[T::kVec];
        T::unpack(raw[j], x);
        acc.bits |= raw[j].x | raw[j].y | raw[j].z | raw[j].w;
        acc.template add<T::kVec>(x);
      }
    }
    const uint32_t i = s.head + nv * T::kVec + lane;
    if (i < s.n) one(g[i]);
  } else {
    const TensorEntry& e = prm.entries[s.tensor];
    const S* g = static_cast<const S*>(e.g);
    Walk w = grad_walk(e, s.start + lane, 32);
    for (uint32_t i0 = lane; i0 < s.n; i0 += kBatch * 32) {
      float x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        x[j] = i0 + j * 32 < s.n ? T::to_float(g[w.offset()]) : 0.f;
        w.next();
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) acc.bits |= __float_as_uint(x[j]);
      acc.template add<kBatch>(x);
    }
  }
  return acc;
}

// The same sum with every product in fp64, for segments whose fp32 products leave the range.
template <typename T, int NORM>
__device__ __noinline__ double segment_acc_wide(const TensorsParams& prm, const Segment& s,
                                                uint32_t lane) {
  const TensorEntry& e = prm.entries[s.tensor];
  const typename T::scalar* g = static_cast<const typename T::scalar*>(e.g);
  Walk w = grad_walk(e, s.start + lane, 32);
  double sum = 0.0;
  for (uint32_t i = lane; i < s.n; i += 32, w.next()) {
    const double x = T::to_float(g[w.offset()]);
    sum += NORM == kNorm2 ? x * x : fabs(x);
  }
  return sum;
}

// The sum of a segment, in every lane of its warp.
template <int NORM>
__device__ __forceinline__ double segment_sum(const TensorsParams& prm, const Segment& s,
                                              uint32_t lane) {
  double x = 0.0;
  with_type(s.dtype, [&](auto type) {
    using T = decltype(type);
    const NormAcc<NORM> acc = segment_acc<T, NORM>(prm, s, lane);
    x = warp_join<NORM>(NORM == kNormMax ? static_cast<double>(acc.mx) : acc.s);
    if constexpr (NORM != kNormMax) {
      // fp32 squares overflow above 1.8e19 and lose bits below 1e-19; sums of |x| overflow
      // near the largest float.  A segment whose sum says so is taken again in fp64.
      const bool wide = !(x < 0x1p120) || (NORM == kNorm2 && x < 0x1p-90);
      if (wide && __any_sync(0xffffffffu, acc.bits != 0))
        x = warp_join<NORM>(segment_acc_wide<T, NORM>(prm, s, lane));
    }
  });
  return x;
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

template <int NORM>
__device__ __forceinline__ void write_norm(const TensorsParams& prm, int t, double x) {
  prm.norms_out[2 + t] = static_cast<float>(fabs(prm.scale) * (NORM == kNorm2 ? sqrt(x) : x));
}

// The sums of one block.  Segments are dealt out in order, so a tensor that is neither the first
// nor the last of a warp lies in that warp whole, and one that is neither the first nor the last
// of a block in that block: its norm is written where it is known.  What remains of a warp, its
// parts of its first and its last tensor, is joined through shared memory; what remains of a block
// goes to edge_sum.
struct WarpParts {
  double first[kNormWarps], last[kNormWarps];
  int first_tensor[kNormWarps];  // -1: the warp does not begin inside a tensor
  int last_tensor[kNormWarps];   // -1: the warp has no work
};
template <int NORM>
__device__ __forceinline__ double block_sums(const TensorsParams& prm, WarpParts& parts,
                                             double* sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int w = blockIdx.x * kNormWarps + warp;
  int first_tensor = -1, tensor = -1;
  double first = 0.0, x = 0.0, sum = 0.0;
  if (w < prm.n_warps) {
    const int begin = prm.warp_first[w], end = prm.warp_first[w + 1];
    bool closed = false;  // a tensor has ended in this warp
    for (int i = begin; i < end; ++i) {
      const Segment s = prm.segments[i];
      if (tensor >= 0 && s.tensor != tensor) {
        if (!closed && prm.entries[tensor].first_seg < begin) {
          first_tensor = tensor;
          first = x;
        } else if (lane == 0) {
          write_norm<NORM>(prm, tensor, x);
        }
        closed = true;
        x = 0.0;
      }
      tensor = s.tensor;
      const double y = segment_sum<NORM>(prm, s, lane);
      x = norm_join<NORM>(x, y);
      sum = norm_join<NORM>(sum, y);
    }
    if (!closed && prm.entries[tensor].first_seg < begin) {
      first_tensor = tensor;
      first = x;
    }
  }
  if (lane == 0) {
    parts.first[warp] = first;
    parts.last[warp] = x;
    parts.first_tensor[warp] = first_tensor;
    parts.last_tensor[warp] = tensor;
    sm[warp] = sum;
  }
  __syncthreads();
  // each warp: the tensor that it ends with, unless that one began in an earlier warp of the block
  if (tensor >= 0 && !(warp > 0 && first_tensor == tensor)) {
    double y = lane == warp ? x
               : lane > warp && parts.first_tensor[lane] == tensor ? parts.first[lane]
                                                                   : 0.0;
    y = warp_join<NORM>(y);
    const int seg = prm.entries[tensor].first_seg, n_seg = prm.entries[tensor].n_segs;
    const int w0 = blockIdx.x * kNormWarps, w1 = min(w0 + kNormWarps, prm.n_warps);
    const bool from = seg >= prm.warp_first[w0], to = seg + n_seg <= prm.warp_first[w1];
    if (lane == 0) {
      if (from && to) write_norm<NORM>(prm, tensor, y);
      if (!from) prm.edge_sum[2 * blockIdx.x] = y;
      if (!to) prm.edge_sum[2 * blockIdx.x + 1] = y;
    }
  }
  if (threadIdx.x == 0 && first_tensor >= 0 && first_tensor != tensor)
    prm.edge_sum[2 * blockIdx.x] = first;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < prm.n_empty; i += kNormThreads)
      write_norm<NORM>(prm, prm.empty[i], 0.0);
  return warp_join<NORM>(sm[lane]);
}

// The norm of a tensor that lies in several blocks, by one warp.
template <int NORM>
__device__ __forceinline__ void join_spanning(const TensorsParams& prm, int i) {
  const int lane = threadIdx.x & 31;
  const Spanning s = prm.spanning[i];
  double x = 0.0;
  for (int b = s.first + lane; b <= s.last; b += 32)
    x = norm_join<NORM>(x, __ldcg(prm.edge_sum + 2 * b + (b == s.first ? 1 : 0)));
  x = warp_join<NORM>(x);
  if (lane == 0) write_norm<NORM>(prm, s.tensor, x);
}

// The power sum of the list from the sums of the blocks, in every lane.
template <int NORM>
__device__ __forceinline__ double join_blocks(const TensorsParams& prm) {
  double x = 0.0;
  for (int b = threadIdx.x & 31; b < static_cast<int>(gridDim.x); b += 32)
    x = norm_join<NORM>(x, __ldcg(prm.block_sum + b));
  return warp_join<NORM>(x);
}

// Every warp sums its segments, every block its warps, the block that finishes last the blocks: one
// launch, and no order of finishing shows in a sum.
template <int NORM>
__global__ void __launch_bounds__(kNormThreads, 1)
    tensors_norm_kernel(const __grid_constant__ TensorsParams prm) {
  __shared__ WarpParts parts;
  __shared__ double sm[kNormWarps];
  __shared__ unsigned int s_ticket;
  grid_dependency_wait();
  const double sum = block_sums<NORM>(prm, parts, sm);
  grid_launch_dependents();
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    prm.block_sum[blockIdx.x] = sum;
    __threadfence();
    s_ticket = atomicAdd(prm.ticket, 1u);
  }
  __syncthreads();
  if (s_ticket != gridDim.x - 1) return;
  __threadfence();
  const int warp = threadIdx.x >> 5;
  if (warp == 0) {
    const double total = join_blocks<NORM>(prm);
    if (threadIdx.x == 0) {
      write_clip(prm, total, clip_of(total, NORM, prm.scale, prm.max_norm));
      *prm.ticket = 0;  // ready for the next call
    }
  }
  for (int i = (warp + kNormWarps - 1) % kNormWarps; i < prm.n_spanning; i += kNormWarps)
    join_spanning<NORM>(prm, i);
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
                                           const void* in, void* out, bool in_place, bool vec) {
  const typename TI::scalar* g = static_cast<const typename TI::scalar*>(in);
  typename TO::scalar* y = static_cast<typename TO::scalar*>(out);
  const uint32_t tid = threadIdx.x;
  if (vec) {
    // rows are whole vectors here, and there is no head then: the walk goes by vectors
    constexpr int kBatch = 4;
    auto one = [&](uint32_t i) {
      y[r.start + i] = TO::from_float(factor * TI::to_float(g[r.start + i]));
    };
    if (tid < r.head) one(tid);
    const uint32_t nv = (r.n - r.head) / 8;
    const int64_t first = r.start + r.head + tid * 8;
    Walk wi = grad_walk(e, first, 8 * kTensorThreads);
    Walk wo = in_place ? wi : out_walk(e, first, 8 * kTensorThreads);
    for (uint32_t v0 = tid; v0 < nv; v0 += kBatch * kTensorThreads) {
      Vec8<TI> raw[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (v0 + j * kTensorThreads < nv) raw[j] = load8<TI>(g + wi.offset());
        wi.next();
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (v0 + j * kTensorThreads < nv) {
          float x[8];
          unpack8<TI>(raw[j], x);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= factor;
          store8<TO>(y + wo.offset(), x);
        }
        wo.next();
      }
    }
    const uint32_t i = r.head + nv * 8 + tid;
    if (i < r.n) one(i);  // only without rows: the elements of a view with rows are whole vectors
  } else {
    constexpr int kBatch = 16;
    Walk wi = grad_walk(e, r.start + tid, kTensorThreads);
    Walk wo = in_place ? wi : out_walk(e, r.start + tid, kTensorThreads);
    for (uint32_t i0 = tid; i0 < r.n; i0 += kBatch * kTensorThreads) {
      typename TI::scalar x[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (i0 + j * kTensorThreads < r.n) x[j] = g[wi.offset()];
        wi.next();
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (i0 + j * kTensorThreads < r.n)
          y[wo.offset()] = TO::from_float(factor * TI::to_float(x[j]));
        wo.next();
      }
    }
  }
}

__global__ void __launch_bounds__(kTensorThreads, 3)
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
      unit_scale<TI, TI>(e, r, clip.factor, e.g, const_cast<void*>(e.g), true,
                         e.flags & kEntryVecClip);
    } else {
      with_type(e.out_dtype, [&](auto to) {
        using TO = decltype(to);
        unit_scale<TI, TO>(e, r, clip.factor, e.g, e.out, false, e.flags & kEntryVecClip);
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
  float *p = e.p + r.start, *m = e.m + r.start, *v = e.v + r.start;
  uint16_t* p16 = e.p16 ? e.p16 + r.start : nullptr;
  const uint32_t tid = threadIdx.x;
  with_type(e.g_dtype, [&](auto type) {
    using T = decltype(type);
    const typename T::scalar* g = static_cast<const typename T::scalar*>(e.g);
    auto one = [&](uint32_t i, int64_t at) {
      float w = p[i], mi = m[i], vi = v[i];
      adamw_elem(a, a.omb1, a.omb2, factor * T::to_float(g[at]), w, mi, vi);
      p[i] = w, m[i] = mi, v[i] = vi;
      if (p16) p16[i] = to_bf16(w);
    };
    if (e.flags & kEntryVecAdam) {
      if (tid < r.head) one(tid, r.start + tid);
      const uint32_t nv = (r.n - r.head) / 8;
      Walk wg = grad_walk(e, r.start + r.head + tid * 8, 8 * kTensorThreads);
      for (uint32_t q = tid; q < nv; q += kTensorThreads, wg.next()) {
        const uint32_t i = r.head + q * 8;
        const Vec8<T> raw = load8<T>(g + wg.offset());
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
      if (i < r.n) one(i, r.start + i);
    } else {
      Walk wg = grad_walk(e, r.start + tid, kTensorThreads);
      for (uint32_t i = tid; i < r.n; i += kTensorThreads, wg.next()) one(i, wg.offset());
    }
  });
}

}  // namespace absnt
