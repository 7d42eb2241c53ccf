// Kernels over a list of tensors: the global norm (and the norm of each tensor), scaling by the
// clipping factor that follows from it, and AdamW on the clipped gradients.
//
// A list is cut in two ways.  For the norm its bytes are dealt out to warps in rows of 512 bytes (32
// lanes of 16): every warp of every block gets the same number of rows, and where a tensor ends
// inside a warp's rows they are cut into segments.  For scaling and AdamW, which join nothing, it is
// cut into units: runs of consecutive elements of one tensor, one CTA each.
// The tables lie in device memory, written there once by the upload of the plan.
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "abs_device.cuh"
#include "normtest_bulk.cuh"

namespace absnt {

constexpr int kTensorThreads = 256;
constexpr int kMaxGroups = ABS_MAX_GROUPS;
constexpr int kListBlocks = 148;     // blocks of the norm kernel, one for each SM
constexpr int kClusterBlocks = 16;   // blocks of the one-cluster kernel
constexpr int kClusterRows = 16;     // most rows that one of its warps takes
constexpr int kListWarps = 16;       // warps of a block of either
constexpr int kAdamwUnit = 4096;     // elements of a unit of AdamW

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
  int32_t first_scale, first_adamw;  // its first unit for scaling and for AdamW
  uint8_t g_dtype, out_dtype;
  // elements before the first one on a boundary of 16 bytes of the gradient, of 8 elements of what
  // scaling writes, of 8 elements of the parameters; 0 for a view with rows
  uint8_t g_head, scale_head, adamw_head;
  uint8_t flags;  // kEntry* bits
  uint16_t group;
};
enum {
  kEntryRowsG = 1,      // the gradient has rows (else it is one run of elements)
  kEntryRowsOut = 2,    // so has the clipped output
  kEntryFar = 4,        // a unit of the gradient's view spans 2^31 elements or more
  kEntryStateVec = 8,   // state and bf16 copy reach a boundary together, after adamw_head
  kEntryVecScale = 16,  // 16 bytes of the gradient (after g_head) meet an aligned place in the output
  kEntryVecAdamw = 32,  // and in state and bf16 copy
  kEntryRuns = 64,      // the gradient's rows are runs of 16 elements or more, none of them far
};

// A run of elements of one tensor, the work of one warp: [start, start + n), `head` of them before
// the first 16-byte boundary.  The segments that open a warp's rows lie in one table, by warp;
// `more` others follow in another one from `next` on.
struct alignas(16) Segment {
  const void* g;  // of element `start`, for a gradient without rows
  int64_t start;
  uint32_t n;
  int32_t tensor;               // -1: no work
  uint8_t dtype, head, flags, pos;  // flags: the entry's; pos: kSeg* bits
  int32_t more, next, pad;
};
enum { kSegBegins = 1, kSegEnds = 2 };  // the first / last segment of its tensor

// A tensor whose segments lie in several blocks, first..last.
struct Spanning {
  int32_t tensor, first, last, pad;
};
// The tensors that a block shares with the blocks before and after it: places in the table of
// those, -1: none.
struct Shared2 {
  int32_t before, after;
};

enum { kNormMax = ABS_NORM_MAX, kNorm1 = ABS_NORM_1, kNorm2 = ABS_NORM_2 };

struct TensorsParams {
  const TensorEntry* entries;
  const int32_t* scale_tensor;  // the tensor of each unit
  const int32_t* adamw_tensor;
  const Segment* opening;   // blocks * warps
  const Segment* further;
  const Spanning* spanning;
  const Shared2* shared;    // blocks
  const int32_t* empty;     // tensors without elements
  double* header;           // ABS_GRAD_* slots
  float* factor;            // what gradients are multiplied by; NaN: the norm is not finite
  unsigned int* tickets;    // [0]: finished blocks, [1 + i]: those of spanning tensor i
  double* block_sum;        // blocks
  double* edge_sum;         // 2 * blocks: a block's parts of the tensors it shares
  float* norms_out;         // 2 + n
  int n_scale, n_adamw, n_spanning, n_empty;
  int scale_unit;  // elements of a unit for scaling
  int norm_type;
  double scale, max_norm;
  const double* sum_in;
  int in_place;
  int after_norm;  // the kernel before this one in the stream is this call's norm kernel
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

// Walks the elements first, first + step, ... of a view: `at` is the offset of the current one from
// `base`, next() goes `step` further.  One division at the beginning, none on the way; in 32 bits
// (I) where what is walked spans less than 2^31 elements.
template <typename I>
struct Walk {
  int64_t base;
  I at, step_at, wrap_at;
  uint32_t col, step_col, row;
  __device__ __forceinline__ void next() {
    at += step_at;
    col += step_col;
    if (col >= row) {
      col -= row;
      at += wrap_at;
    }
  }
};
template <typename I>
__device__ __forceinline__ Walk<I> make_walk(int64_t first, uint32_t step, bool rows, uint32_t row,
                                             int64_t stride, int64_t col_stride) {
  if (!rows) return Walk<I>{first, 0, static_cast<I>(step), 0, 0, 0, 1};
  const int64_t r = first / row;
  const uint32_t c = static_cast<uint32_t>(first - r * row);
  const uint32_t dr = step / row, dc = step - dr * row;
  return Walk<I>{r * stride + c * col_stride,
                 0,
                 static_cast<I>(dr * stride + dc * col_stride),
                 static_cast<I>(stride - static_cast<int64_t>(row) * col_stride),
                 c,
                 dc,
                 row};
}
template <typename I>
__device__ __forceinline__ Walk<I> grad_walk(const TensorEntry& e, int64_t first, uint32_t step) {
  return make_walk<I>(first, step, e.flags & kEntryRowsG, e.g_row, e.g_stride, e.g_col);
}
__device__ __forceinline__ Walk<int64_t> out_walk(const TensorEntry& e, int64_t first, uint32_t step) {
  return make_walk<int64_t>(first, step, e.flags & kEntryRowsOut, e.out_row, e.out_stride, e.out_col);
}

// The elements [start, start + n) of unit k of a tensor; unit 0 also holds the head.
struct UnitRange {
  int64_t start;
  uint32_t n;
};
__device__ __forceinline__ UnitRange unit_range(const TensorEntry& e, int k, int unit, int head) {
  UnitRange r;
  r.start = k ? head + static_cast<int64_t>(k) * unit : 0;
  int64_t end = head + static_cast<int64_t>(k + 1) * unit;
  if (end > e.numel) end = e.numel;
  r.n = static_cast<uint32_t>(end - r.start);
  return r;
}

// ---- the norm ------------------------------------------------------------------------
// Largest magnitude so far; a NaN stays.
__device__ __forceinline__ float max_abs(float acc, float x) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(acc), "f"(fabsf(x)));
  return r;
}

// Running sum of one thread: |x|, x^2 or max |x|.  The values of a 16-byte vector, or eight of a view
// with rows, are added in fp32 (products of 8-bit significands are exact there), the rest in fp64.
template <int NORM>
struct NormAcc {
  double s = 0.0;
  float mx = 0.f;
  uint32_t bits = 0;  // all values or-ed
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

// 16 bytes of a gradient.  Not the read-only path: a kernel may scale its gradients in place.
__device__ __forceinline__ uint4 ld_grad_16(const void* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p)
               : "memory");
  return r;
}

// One lane's share of a segment.  KEEP: its rows are also left in shared memory, at `keep` (this
// lane's place in row 0), one after the other.  SMALL: fewer loads at once, for lists of a few rows a
// warp, where fetching the instructions of a larger body is what shows (60k elements: 0.1 us of 3.5).
template <typename T, int NORM, bool KEEP, bool SMALL>
__device__ __forceinline__ NormAcc<NORM> segment_acc(const TensorsParams& prm, const Segment& s,
                                                     uint32_t lane, uint4* keep) {
  using S = typename T::scalar;
  constexpr int kBatch = SMALL ? 4 : 8;
  NormAcc<NORM> acc;
  auto one = [&](S raw) {
    const float x = T::to_float(raw);
    acc.bits |= __float_as_uint(x);
    acc.template add<1>(&x);
  };
  auto vec = [&](const uint4& raw) {
    float x[T::kVec];
    T::unpack(raw, x);
    acc.bits |= raw.x | raw.y | raw.z | raw.w;
    acc.template add<T::kVec>(x);
  };
  if (!(s.flags & kEntryRowsG)) {
    const S* g = static_cast<const S*>(s.g);
    if (lane < s.head) one(g[lane]);
    const uint32_t nv = (s.n - s.head) / T::kVec;
    const S* gv = g + s.head;
    for (uint32_t v0 = lane; v0 < nv; v0 += kBatch * 32) {
      uint4 raw[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint32_t v = v0 + j * 32;
        raw[j] = v < nv ? ld_grad_16(gv + static_cast<size_t>(v) * T::kVec) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        vec(raw[j]);
        if (KEEP && v0 + j * 32 < nv) keep[v0 - lane + j * 32] = raw[j];
      }
    }
    const uint32_t i = s.head + nv * T::kVec + lane;
    if (i < s.n) one(g[i]);
  } else {
    // a view with rows
    const TensorEntry& e = prm.entries[s.tensor];
    const S* g = static_cast<const S*>(e.g);
    S* kept = reinterpret_cast<S*>(keep - lane);
    if (e.flags & kEntryFar) {
      Walk<int64_t> w = grad_walk<int64_t>(e, s.start + lane, 32);
      for (uint32_t i = lane; i < s.n; i += 32, w.next()) {
        const S raw = g[w.base + w.at];
        one(raw);
        if (KEEP) kept[i] = raw;
      }
      return acc;
    }
    // 24 at once: few bytes are under way with single elements (30M fp16 in column slices, from
    // memory: 16, 24, 32 at once 32.4, 29.9, 30.3 us; dense 15.7).  The registers are those of the whole
    // kernel, 128 instead of 96 for 16 at once.  What that does to dense lists (us, 16 / 24): norm of 1.5M
    // bf16 5.7 / 5.8, 4M 5.8 / 5.8, 50M fp16 17.3 / 17.2, 300M bf16 89.1 / 89.2; with scaling 8.9 / 8.6,
    // 9.8 / 9.8, 48.5 / 48.3, 279.6 / 279.7, and 16M fp16 15.8 / 16.1
    constexpr int kWalk = SMALL ? 8 : 24;
    Walk<int32_t> w = grad_walk<int32_t>(e, s.start + lane, 32);
    g += w.base;
    const auto batch = [&](uint32_t i0, auto whole) {
      S raw[kWalk];
#pragma unroll
      for (int j = 0; j < kWalk; ++j) {
        raw[j] = decltype(whole)::value || i0 + j * 32 < s.n ? g[w.at] : S(0);
        w.next();
      }
#pragma unroll
      for (int j = 0; j < kWalk; j += 8) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] = T::to_float(raw[j + k]);
          acc.bits |= __float_as_uint(x[k]);
          if (KEEP && (decltype(whole)::value || i0 + (j + k) * 32 < s.n))
            kept[i0 + (j + k) * 32] = raw[j + k];
        }
        acc.template add<8>(x);
      }
    };
    uint32_t i0 = lane;
    for (; i0 - lane + kWalk * 32 <= s.n; i0 += kWalk * 32) batch(i0, std::true_type{});
    if (i0 < s.n) batch(i0, std::false_type{});
  }
  return acc;
}

// The same sum with every product in fp64, for segments whose fp32 products leave the range.
template <typename T, int NORM>
__device__ __forceinline__ double segment_acc_wide(const TensorsParams& prm, const Segment& s,
                                                   uint32_t lane) {
  const TensorEntry& e = prm.entries[s.tensor];
  const typename T::scalar* g = static_cast<const typename T::scalar*>(e.g);
  Walk<int64_t> w = grad_walk<int64_t>(e, s.start + lane, 32);
  double sum = 0.0;
#pragma unroll 1
  for (uint32_t i = lane; i < s.n; i += 32, w.next()) {
    const double x = T::to_float(g[w.base + w.at]);
    sum += NORM == kNorm2 ? x * x : fabs(x);
  }
  return sum;
}

// The sum of a segment, in every lane of its warp.
template <int NORM, bool KEEP, bool SMALL>
__device__ __forceinline__ double segment_sum(const TensorsParams& prm, const Segment& s,
                                              uint32_t lane, uint4* keep) {
  double x = 0.0;
  with_type(s.dtype, [&](auto type) {
    using T = decltype(type);
    const NormAcc<NORM> acc = segment_acc<T, NORM, KEEP, SMALL>(prm, s, lane, keep);
    x = warp_join<NORM>(NORM == kNormMax ? static_cast<double>(acc.mx) : acc.s);
    if constexpr (NORM != kNormMax) {
      // fp32 squares overflow above 1.8e19 and lose bits below 1e-19; sums of |x| overflow
      // near the largest float.  A segment whose sum says so is taken again in fp64.
      // (below 2^-100 a sum of 2^24 squares may be off by 2^-24 of itself: each loses up to 2^-150)
      const bool wide = !(x < 0x1p120) || (NORM == kNorm2 && x < 0x1p-100);
      constexpr uint32_t kSigns = T::kVec == 8 ? 0x80008000u : 0x80000000u;  // zeros have either
      if (wide && __any_sync(0xffffffffu, (acc.bits & ~kSigns) != 0))
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
  *prm.factor = c.finite ? c.factor : __int_as_float(0x7fc00000);
}

template <int NORM>
__device__ __forceinline__ void write_norm(const TensorsParams& prm, int t, double x) {
  prm.norms_out[2 + t] = static_cast<float>(fabs(prm.scale) * (NORM == kNorm2 ? sqrt(x) : x));
}

// What a warp's rows leave to be joined.  A tensor that begins and ends in them is done
// with there.  There may be one at the front that began before them (kHead: and ends in them), and
// one at the back that goes on after them (kTail: and begins in them; kThrough: began before them).
enum { kHead = 1, kTail = 2, kThrough = 4 };
struct BlockParts {
  double head[kListWarps], open[kListWarps], sum[kListWarps];
  int tensor[kListWarps], state[kListWarps];
};

// Rows of 512 bytes that a segment leaves in shared memory: all vectors of one run of elements
// (head and rest are not kept), all elements of a view with rows.
__device__ __forceinline__ uint32_t kept_rows(const Segment& s) {
  const uint32_t n = (s.flags & kEntryRowsG) ? s.n : s.n - s.head;
  const uint32_t per_row = s.dtype == ABS_F32 ? 128 : 256, per = per_row / 32;
  return (s.flags & kEntryRowsG) ? (n + per_row - 1) / per_row : (n / per + 31) / 32;
}

// One warp's rows; returns their sum.
template <int NORM, bool KEEP, bool SMALL>
__device__ __forceinline__ double warp_sum(const TensorsParams& prm, const Segment& opening,
                                           BlockParts& parts, uint4* keep) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double sum = 0.0, x = 0.0, head = 0.0;
  int state = 0, tensor = -1;
  bool begun = false, open = false;
  Segment s = opening;
  if (s.tensor >= 0) {
    for (int k = 0;; ++k) {
      Segment next = s;
      if (k < opening.more) next = prm.further[opening.next + k];
      const double y = segment_sum<NORM, KEEP, SMALL>(prm, s, lane, keep);
      if (KEEP) keep += kept_rows(s) * 32;
      sum = norm_join<NORM>(sum, y);
      x = norm_join<NORM>(x, y);
      begun |= (s.pos & kSegBegins) != 0;
      open = !(s.pos & kSegEnds);
      tensor = s.tensor;
      if (!open) {
        if (begun) {
          if (lane == 0) write_norm<NORM>(prm, tensor, x);
        } else {
          head = x;
          state = kHead;
        }
        x = 0.0;
        begun = false;
      }
      if (k == opening.more) break;
      s = next;
    }
    if (open) state |= begun ? kTail : kThrough;
  }
  if (lane == 0) {
    parts.head[warp] = head;
    parts.open[warp] = x;
    parts.tensor[warp] = tensor;
    parts.state[warp] = state;
  }
  return sum;
}

// Joins the parts of a block's warps, each tensor by the warp in which it begins (by warp 0, if it
// began before the block); edge(0, x) and edge(1, x), called by a whole warp, receive the parts of a
// tensor that the block shares with the one before and the one after it.  After a __syncthreads.
// Returns the tensor whose sum is now known to this warp (in `x`; to be written by the caller), or -1.
template <int NORM, typename F>
__device__ __forceinline__ int join_parts(const TensorsParams& prm, const BlockParts& parts, F&& edge,
                                          double& x) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int state = lane < kListWarps ? parts.state[lane] : 0;
  const uint32_t heads = __ballot_sync(0xffffffffu, state & kHead);
  const uint32_t throughs = __ballot_sync(0xffffffffu, state & kThrough);
  const int mine = parts.state[warp];
  if (warp == 0 && (mine & kHead)) edge(0, parts.head[0]);
  if (!((mine & kTail) || (warp == 0 && (mine & kThrough)))) return -1;
  const uint32_t stop = ~throughs & ~((2u << warp) - 1u);  // warps after this one that end it
  const uint32_t u = stop ? static_cast<uint32_t>(__ffs(stop)) - 1u : 32u;
  const bool ends = u < 32 && ((heads >> u) & 1u);
  x = lane == warp || (lane > warp && lane < u && lane < kListWarps) ? parts.open[lane]
      : lane == u && ends                                       ? parts.head[lane]
                                                                : 0.0;
  x = warp_join<NORM>(x);
  if (!(mine & kTail)) edge(0, x);
  if (!ends) edge(1, x);
  return (mine & kTail) && ends ? parts.tensor[warp] : -1;
}

// The sum of a block from those of its warps, in every lane.  After a __syncthreads.
template <int NORM>
__device__ __forceinline__ double join_warps(const double* sums) {
  const uint32_t lane = threadIdx.x & 31;
  return warp_join<NORM>(lane < kListWarps ? sums[lane] : 0.0);
}

// The norm of a tensor that several blocks share, by one warp.  edge(b, i): edge i of block b.
template <int NORM, typename F>
__device__ __forceinline__ void join_spanning(const TensorsParams& prm, const Spanning& s, F&& edge) {
  double x = 0.0;
  for (int b = s.first + (threadIdx.x & 31); b <= s.last; b += 32)
    x = norm_join<NORM>(x, edge(b, b == s.first ? 1 : 0));
  x = warp_join<NORM>(x);
  if ((threadIdx.x & 31) == 0) write_norm<NORM>(prm, s.tensor, x);
}

// Counts this block off; true in the whole warp if it was the last of `of` blocks.  Its sums are
// visible to the warp that gets true, and the counter is back at zero for the next call.
__device__ __forceinline__ bool last_of(unsigned int* ticket, unsigned int of) {
  unsigned int before = 0;
  if ((threadIdx.x & 31) == 0) {
    __threadfence();
    before = atomicAdd(ticket, 1u);
    if (before == of - 1) *ticket = 0;
    __threadfence();
  }
  before = __shfl_sync(0xffffffffu, before, 0);
  __syncwarp();  // a shuffle orders no memory: what lane 0 may see, the others may from here on
  return before == of - 1;
}

// sum |x|^p (or max |x|) of each tensor and of the list.  Every warp sums its rows, every block its
// warps; the block that finishes last joins the blocks, and of the blocks that share a tensor the last
// one joins that tensor: one launch, and no order of finishing shows in a sum.
//
// Bound by reading the gradients once.  Each warp reads one run of the list, eight 16-byte loads per
// lane at a time, and meets another warp only at the end, so that the tensors' boundaries cost
// nothing on the way: 1.24G bf16 (2.47 GB) 355 us = 7.0 TB/s, 124M fp32 (498 MB) 76 us = 6.5 TB/s, against
// 405 and 79.5 us with one CTA per 32768 elements of a tensor and a ticket each.  16 warps a block:
// 32 of half the registers take 358 and 78.4 us.  Below 50 MB what shows is the chain launch, table,
// data, join, ticket, join: 4.9 us for an empty list.
template <int NORM>
__global__ void __launch_bounds__(kListWarps * 32, 1)
    tensors_norm_kernel(const __grid_constant__ TensorsParams prm) {
  __shared__ BlockParts parts;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // the tables were there before any kernel of the stream
  const Segment opening = prm.opening[blockIdx.x * kListWarps + warp];
  Shared2 shared{-1, -1};
  if (warp == 1 || warp == 2) shared = prm.shared[blockIdx.x];
  grid_dependency_wait();
  grid_launch_dependents();  // see tensors_scale_kernel
  double sum = warp_sum<NORM, false, false>(prm, opening, parts, nullptr);
  if (lane == 0) parts.sum[warp] = sum;
  __syncthreads();
  double x;
  const auto edge = [&](int k, double part) {
    if (lane == 0) prm.edge_sum[2 * blockIdx.x + k] = part;
  };
  const int known = join_parts<NORM>(prm, parts, edge, x);
  if (known >= 0 && lane == 0) write_norm<NORM>(prm, known, x);
  if (warp == 0) {
    sum = join_warps<NORM>(parts.sum);
    if (lane == 0) prm.block_sum[blockIdx.x] = sum;
  }
  const int i = warp == 1 ? shared.before : warp == 2 ? shared.after : -1;
  Spanning span;
  if (i >= 0) span = prm.spanning[i];
  __syncthreads();  // all edges are written
  if (warp == 0 && last_of(prm.tickets, gridDim.x)) {
    double total = 0.0;
    for (int b = lane; b < static_cast<int>(gridDim.x); b += 32)
      total = norm_join<NORM>(total, __ldcg(prm.block_sum + b));
    total = warp_join<NORM>(total);
    if (lane == 0) write_clip(prm, total, clip_of(total, NORM, prm.scale, prm.max_norm));
  }
  if (i >= 0 && last_of(prm.tickets + 1 + i, span.last - span.first + 1))
    join_spanning<NORM>(prm, span, [&](int b, int k) { return __ldcg(prm.edge_sum + 2 * b + k); });
  if (blockIdx.x == 0)
    for (int k = threadIdx.x; k < prm.n_empty; k += kListWarps * 32)
      write_norm<NORM>(prm, prm.empty[k], 0.0);
}

// Norm and factor from a power sum that comes from elsewhere (added up over ranks).
__global__ void tensors_clip_kernel(const __grid_constant__ TensorsParams prm) {
  grid_dependency_wait();
  const double sum = __ldcg(prm.sum_in);
  if (threadIdx.x == 0) write_clip(prm, sum, clip_of(sum, prm.norm_type, prm.scale, prm.max_norm));
}

// ---- scaling -------------------------------------------------------------------------
// Values of a type known at run time: where there are few of them, or any pair of types may meet.
__device__ __forceinline__ float load_any(const void* p, int64_t i, int dtype) {
  if (dtype == ABS_F32) return static_cast<const float*>(p)[i];
  const uint16_t x = static_cast<const uint16_t*>(p)[i];
  return dtype == ABS_BF16 ? TBF16::to_float(x) : TF16::to_float(x);
}
__device__ __forceinline__ void store_any(void* p, int64_t i, int dtype, float x) {
  if (dtype == ABS_F32)
    static_cast<float*>(p)[i] = x;
  else
    static_cast<uint16_t*>(p)[i] = dtype == ABS_BF16 ? TBF16::from_float(x) : TF16::from_float(x);
}
// The 4 (fp32) or 8 values of 16 bytes of input, scaled, to an output that is aligned for 16-byte stores
// (8-byte ones from fp32 to 16 bits).
__device__ __forceinline__ void store_scaled(const uint4& raw, int in, void* p, int64_t i, int out,
                                             float factor) {
  float x[8] = {};
  if (in == ABS_F32)
    TF32::unpack(raw, x);
  else if (in == ABS_BF16)
    TBF16::unpack(raw, x);
  else
    TF16::unpack(raw, x);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] *= factor;
  if (out == ABS_F32) {
    float* y = static_cast<float*>(p) + i;
    st_stream_16(y, make_float4(x[0], x[1], x[2], x[3]));
    if (in != ABS_F32) st_stream_16(y + 4, make_float4(x[4], x[5], x[6], x[7]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      w[k] = out == ABS_BF16
                 ? pack_bf16x2(x[2 * k], x[2 * k + 1])
                 : static_cast<uint32_t>(TF16::from_float(x[2 * k])) |
                       (static_cast<uint32_t>(TF16::from_float(x[2 * k + 1])) << 16);
    uint16_t* y = static_cast<uint16_t*>(p) + i;
    if (in == ABS_F32)
      __stcs(reinterpret_cast<uint2*>(y), make_uint2(w[0], w[1]));
    else
      __stcs(reinterpret_cast<uint4*>(y), make_uint4(w[0], w[1], w[2], w[3]));
  }
}
// n elements from `first` on, every step-th of them by this thread, from and to any view.
__device__ __forceinline__ void scale_walk(const TensorEntry& e, int64_t first, uint32_t i0,
                                           uint32_t n, uint32_t step, float factor, bool in_place) {
  constexpr int kBatch = 8;
  Walk<int64_t> wi = grad_walk<int64_t>(e, first + i0, step);
  Walk<int64_t> wo = in_place ? wi : out_walk(e, first + i0, step);
  void* y = in_place ? const_cast<void*>(e.g) : e.out;
  const int in = e.g_dtype, out = in_place ? e.g_dtype : e.out_dtype;
  for (; i0 < n; i0 += kBatch * step) {
    float x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (i0 + j * step < n) x[j] = load_any(e.g, wi.base + wi.at, in);
      wi.next();
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (i0 + j * step < n) store_any(y, wo.base + wo.at, out, factor * x[j]);
      wo.next();
    }
  }
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

// Eight consecutive values that begin `o` bytes after a 16-byte boundary (o > 0): the 16-byte pieces
// that hold them, and the values out of those.
template <typename T>
struct Shifted8 {
  uint4 r[8 / T::kVec + 1];
};
template <typename T>
__device__ __forceinline__ Shifted8<T> load_shifted8(const typename T::scalar* p, uint32_t o) {
  const uint4* c = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - o);
  Shifted8<T> x;
#pragma unroll
  for (int i = 0; i < 8 / T::kVec + 1; ++i) x.r[i] = c[i];  // a neighbour reads them too: L1
  return x;
}
template <typename T>
__device__ __forceinline__ void unpack_shifted8(const Shifted8<T>& v, uint32_t o, float* x) {
  constexpr int kWords = 4 * (8 / T::kVec) + 4;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < 8 / T::kVec + 1; ++i)
    w[4 * i] = v.r[i].x, w[4 * i + 1] = v.r[i].y, w[4 * i + 2] = v.r[i].z, w[4 * i + 3] = v.r[i].w;
  if (o & 8) {
#pragma unroll
    for (int i = 0; i + 2 < kWords; ++i) w[i] = w[i + 2];
  }
  if (o & 4) {
#pragma unroll
    for (int i = 0; i + 1 < kWords; ++i) w[i] = w[i + 1];
  }
  if (T::kVec == 8 && (o & 2)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  Vec8<T> y;
#pragma unroll
  for (int i = 0; i < 8 / T::kVec; ++i)
    y.r[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  unpack8<T>(y, x);
}

// A run of n elements at g whose vectors of 8 begin at `head`: how far those lie behind a 16-byte
// boundary, with the head and the number of vectors such that no piece reaches out of [lo, hi).
struct Run {
  uint32_t head, nv, o;
};
template <typename S>
__device__ __forceinline__ Run make_run(const S* g, uint32_t n, uint32_t head, const S* lo,
                                        const S* hi) {
  Run r{head, 0, static_cast<uint32_t>(reinterpret_cast<uintptr_t>(g + head)) & 15u};
  if (r.o && reinterpret_cast<const char*>(g + head) - r.o < reinterpret_cast<const char*>(lo))
    r.head = min(head + 8, n);
  r.nv = (n - r.head) / 8;
  if (r.o && r.nv &&
      reinterpret_cast<const char*>(g + r.head + 8 * r.nv) + (16 - r.o) >
          reinterpret_cast<const char*>(hi))
    --r.nv;
  return r;
}

// `factor()` gives the factor, waiting for it the first time; a NaN: nothing is to be written.
template <typename TI, typename TO, typename F>
__device__ __forceinline__ void unit_scale(const TensorEntry& e, const UnitRange& r, F&& factor,
                                           void* out, bool in_place) {
  using SI = typename TI::scalar;
  using SO = typename TO::scalar;
  const SI* g = static_cast<const SI*>(e.g);
  SO* y = static_cast<SO*>(out);
  const uint32_t tid = threadIdx.x;
  if (!(e.flags & (in_place ? kEntryRowsG : kEntryRowsG | kEntryRowsOut))) {
    const SI *lo = g, *hi = g + e.numel;
    g += r.start;
    y += r.start;
    const Run run = make_run(g, r.n, r.start ? 0u : min(uint32_t{e.scale_head}, r.n), lo, hi);
    const auto store = [&](uint32_t v, float* x, float f) {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] *= f;
      store8<TO>(y + run.head + v * 8, x);
    };
    if (run.o == 0) {
      constexpr int kBatch = TI::kVec == 8 ? 8 : 4;  // 128 bytes in flight per thread
      for (uint32_t v0 = tid; v0 < run.nv; v0 += kBatch * kTensorThreads) {
        Vec8<TI> raw[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (v0 + j * kTensorThreads < run.nv)
            raw[j] = load8<TI>(g + run.head + (v0 + j * kTensorThreads) * 8);
        const float f = factor();
        if (f != f) return;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (v0 + j * kTensorThreads < run.nv) {
            float x[8];
            unpack8<TI>(raw[j], x);
            store(v0 + j * kTensorThreads, x, f);
          }
      }
    } else {
      constexpr int kBatch = 2;
      for (uint32_t v0 = tid; v0 < run.nv; v0 += kBatch * kTensorThreads) {
        Shifted8<TI> raw[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (v0 + j * kTensorThreads < run.nv)
            raw[j] = load_shifted8<TI>(g + run.head + (v0 + j * kTensorThreads) * 8, run.o);
        const float f = factor();
        if (f != f) return;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (v0 + j * kTensorThreads < run.nv) {
            float x[8];
            unpack_shifted8<TI>(raw[j], run.o, x);
            store(v0 + j * kTensorThreads, x, f);
          }
      }
    }
    // head and rest, at most 15 elements each
    const uint32_t rest = run.head + run.nv * 8 + tid;
    if (tid < run.head || rest < r.n) {
      const float f = factor();
      if (f != f) return;
      if (tid < run.head) y[tid] = TO::from_float(f * TI::to_float(g[tid]));
      if (rest < r.n) y[rest] = TO::from_float(f * TI::to_float(g[rest]));
    }
    return;
  }
  const float f = factor();
  if (f != f) return;
  if (!(e.flags & kEntryFar) && (in_place || !(e.flags & kEntryRowsOut))) {
    // rows into one run, or in place: one walk
    constexpr int kBatch = 16;
    Walk<int32_t> w = grad_walk<int32_t>(e, r.start + tid, kTensorThreads);
    g += w.base;
    y += in_place ? w.base : r.start + tid;
    const auto batch = [&](uint32_t i0, auto whole) {
      SI x[kBatch];
      Walk<int32_t> again = w;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (decltype(whole)::value || i0 + j * kTensorThreads < r.n) x[j] = g[w.at];
        w.next();
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (decltype(whole)::value || i0 + j * kTensorThreads < r.n)
          y[in_place ? again.at : j * kTensorThreads] = TO::from_float(f * TI::to_float(x[j]));
        if (in_place) again.next();
      }
      if (!in_place) y += kBatch * kTensorThreads;
    };
    uint32_t i0 = tid;
    for (; i0 - tid + kBatch * kTensorThreads <= r.n; i0 += kBatch * kTensorThreads)
      batch(i0, std::true_type{});
    if (i0 < r.n) batch(i0, std::false_type{});
  } else {
    scale_walk(e, r.start, tid, r.n, kTensorThreads, f, in_place);
  }
}

// y = factor * x in fp32, rounded to y's type.  Bound by reading x again and writing y: a list that is
// larger than what stays on chip is read twice, since the factor needs the whole norm.  One CTA per
// unit, the last unit of the list first.  After this call's norm kernel the first loads are made before
// the factor is waited for: that kernel lets this one start only after its own wait, so whatever wrote
// the tensors before is done.  Four CTAs of 64 registers to an SM (a thread spills 56
// bytes), against three of 80, norm and scaling (us): 4M bf16 9.7 / 10.6, 16M fp16 16 / 18, 50M fp16
// 48.1 / 49.0, 300M bf16 279.5 / 279.0, 1.24G fp32 into bf16 1832 / 1818.  The norm kernel's blocks of sums
// (128 registers x 512 threads, all of an SM) leave no room beside them, so what runs early are the CTAs on
// SMs whose block has ended; beside its blocks of maxima (101 registers) one fits neither.
// Norm and scaling of 124M bf16 into bf16: 121 us = 6.2 TB/s of the 747 MB that they move; 1.24G fp32
// into bf16: 1.84 ms = 6.7 TB/s of 12.4 GB.  Measured and dropped: one cooperative kernel in which each
// warp scales what it read itself, with its last rows kept in shared memory (167 us and 2.5 ms: the
// reads and writes of thousands of warps lie too far apart).
__global__ void __launch_bounds__(kTensorThreads, 4)
    tensors_scale_kernel(const __grid_constant__ TensorsParams prm) {
  const int u = prm.n_scale - 1 - blockIdx.x;
  const TensorEntry& e = prm.entries[prm.scale_tensor[u]];
  const UnitRange r = unit_range(e, u - e.first_scale, prm.scale_unit, e.scale_head);
  bool have = false;
  if (!prm.after_norm) grid_dependency_wait();
  float value = 0.f;
  const auto factor = [&]() {
    if (!have) {
      if (prm.after_norm) grid_dependency_wait();
      value = __ldcg(prm.factor);
      if (value != value) value = static_cast<float>(prm.scale);  // not finite: not clipped
      if (prm.in_place && value == 1.f) value = __int_as_float(0x7fc00000);  // x * 1 is x
      have = true;
    }
    return value;
  };
  with_type(e.g_dtype, [&](auto ti) {
    using TI = decltype(ti);
    if (prm.in_place)
      unit_scale<TI, TI>(e, r, factor, const_cast<void*>(e.g), true);
    else
      with_type(e.out_dtype, [&](auto to) {
        unit_scale<TI, decltype(to)>(e, r, factor, e.out, false);
      });
  });
}

// Eight values of a view whose rows are runs, from the place of a walk by vectors of 8: the aligned
// 16-byte pieces that hold them, or one by one where they reach into the next row or a piece would
// reach out of the view, [lo, hi).  (A piece may hold what lies between two rows.)
template <typename T>
struct Gathered8 {
  Shifted8<T> v;
  uint32_t o;  // as for Shifted8, or 0
};
template <typename T>
__device__ __forceinline__ Gathered8<T> gather8(const typename T::scalar* p, uint32_t col, uint32_t row,
                                                int32_t gap, const typename T::scalar* lo,
                                                const typename T::scalar* hi) {
  using S = typename T::scalar;
  constexpr int kPieces = 8 / T::kVec;
  Gathered8<T> x;
  x.o = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
  const S* c = p - x.o / sizeof(S);
  if (col + 8 <= row && c >= lo && c + T::kVec * (kPieces + 1) <= hi) {
#pragma unroll
    for (int i = 0; i < kPieces + 1; ++i) x.v.r[i] = reinterpret_cast<const uint4*>(c)[i];
  } else {
    x.o = 0;
    uint32_t w[4 * kPieces];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const S b = p[k + (col + k >= row ? gap : 0)];
      if constexpr (T::kVec == 4)
        w[k] = __float_as_uint(b);
      else
        w[k / 2] = k % 2 ? w[k / 2] | static_cast<uint32_t>(b) << 16 : b;
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      x.v.r[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    x.v.r[kPieces] = make_uint4(0, 0, 0, 0);
  }
  return x;
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


// One coordinate: element `at` of the gradient, element i of the other arrays.
struct StateArrays {
  float *p, *m, *v;
  uint16_t* p16;
};
__device__ __forceinline__ void adamw_one(const AdamScalars& a, const StateArrays& s, int64_t i,
                                          float g) {
  float w = s.p[i], m = s.m[i], v = s.v[i];
  adamw_elem(a, a.omb1, a.omb2, g, w, m, v);
  s.p[i] = w, s.m[i] = m, s.v[i] = v;
  if (s.p16) s.p16[i] = to_bf16(w);
}
// n elements from `first` on, every step-th of them by this thread.
template <typename T>
__device__ __forceinline__ void adamw_walk(const AdamScalars& a, const StateArrays& s,
                                           const TensorEntry& e, int64_t first, uint32_t i0,
                                           uint32_t n, uint32_t step, float factor) {
  constexpr int kBatch = 4;
  const typename T::scalar* g = static_cast<const typename T::scalar*>(e.g);
  Walk<int64_t> wg = grad_walk<int64_t>(e, first + i0, step);
  g += wg.base;
  for (; i0 < n; i0 += kBatch * step) {
    typename T::scalar x[kBatch];
    float w[kBatch], m[kBatch], v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int64_t i = first + i0 + j * step;
      if (i0 + j * step < n) x[j] = g[wg.at], w[j] = s.p[i], m[j] = s.m[i], v[j] = s.v[i];
      wg.next();
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int64_t i = first + i0 + j * step;
      if (i0 + j * step < n) {
        adamw_elem(a, a.omb1, a.omb2, factor * T::to_float(x[j]), w[j], m[j], v[j]);
        s.p[i] = w[j], s.m[i] = m[j], s.v[i] = v[j];
        if (s.p16) s.p16[i] = to_bf16(w[j]);
      }
    }
  }
}

// AdamW on factor * g (adamw_elem), the gradient read and never written.  Bound by its traffic: g once,
// p, m and v read and written, the bf16 copy.  Units and early loads as in the scaling kernel; units of
// 4096 elements (two vectors of 8 per thread) so that CTAs of 115 KB each fill the last wave: 1.24G bf16
// gradients with the copy 5.48 ms after the norm = 6.8 TB/s of the 37.1 GB that both move (2048: 5.53,
// 8192: 5.52, 32768: 5.68 ms); 124M 564 us; 1200 adapters of 24M fp32 together 124 us.
// Gradients that are views take vectors of 8 of the state as well, if their rows are runs of 16 or more
// (24M fp16 in rows of 333, norm and update: 131 us element by element, 120 so; fp32 137 and 130; rows
// of 16, in the order of the tested alignments, fp16 146 / 133 and 139 / 122, fp32 157 / 144 and
// 163 / 137; rows of 8 hardly ever hold a whole vector).
__global__ void __launch_bounds__(kTensorThreads, 4)
    tensors_adamw_kernel(const __grid_constant__ TensorsParams prm,
                         const __grid_constant__ GroupScalars groups, int clipped) {
  const bool after_norm = prm.after_norm;
  if (!after_norm) grid_dependency_wait();
  const int u = prm.n_adamw - 1 - blockIdx.x;
  const TensorEntry& e = prm.entries[prm.adamw_tensor[u]];
  const UnitRange r = unit_range(e, u - e.first_adamw, kAdamwUnit, e.adamw_head);
  const AdamScalars& a = groups.a[e.group];
  const StateArrays state{e.p, e.m, e.v, e.p16};
  const uint32_t tid = threadIdx.x;
  float factor = static_cast<float>(prm.scale);
  with_type(e.g_dtype, [&](auto type) {
    using T = decltype(type);
    using S = typename T::scalar;
    bool have = false;
    const auto skip = [&]() {  // gets the factor; true: no update, the gradient is not finite
      if (!have) {
        if (after_norm) grid_dependency_wait();
        if (clipped) factor = __ldcg(prm.factor);
        have = true;
      }
      return factor != factor;
    };
    const bool runs = e.flags & kEntryRuns;
    if (((e.flags & kEntryRowsG) && !runs) || !(e.flags & kEntryStateVec)) {
      if (!skip()) adamw_walk<T>(a, state, e, r.start, tid, r.n, kTensorThreads, factor);
      return;
    }
    const S *lo = static_cast<const S*>(e.g), *hi = lo + e.numel, *g = lo + r.start;
    float *p = e.p + r.start, *m = e.m + r.start, *v = e.v + r.start;
    const uint32_t head = r.start ? 0u : min(uint32_t{e.adamw_head}, r.n);
    const Run run = runs ? Run{head, (r.n - head) / 8, 0} : make_run(g, r.n, head, lo, hi);
    const auto update = [&](uint32_t i, const float* x, Float8& w, Float8& mm, Float8& vv) {
      const float2 g0 = make_float2(factor * x[0], factor * x[1]);
      const float2 g1 = make_float2(factor * x[2], factor * x[3]);
      const float2 g2 = make_float2(factor * x[4], factor * x[5]);
      const float2 g3 = make_float2(factor * x[6], factor * x[7]);
      adamw_quad(a, g0, g1, w.lo, mm.lo, vv.lo);
      adamw_quad(a, g2, g3, w.hi, mm.hi, vv.hi);
      st_stream_32(p + i, w.lo, w.hi);
      st_stream_32(m + i, mm.lo, mm.hi);
      st_stream_32(v + i, vv.lo, vv.hi);
      if (e.p16) st_bf16x8(e.p16 + r.start + i, w.lo, w.hi);
    };
    if (runs) {
      const S* end = lo + (e.numel / e.g_row - 1) * e.g_stride + e.g_row;
      const int32_t gap = static_cast<int32_t>(e.g_stride - e.g_row);
      Walk<int32_t> wg = grad_walk<int32_t>(e, r.start + head + tid * 8, 8 * kTensorThreads);
      const S* from = lo + wg.base;
      for (uint32_t q = tid; q < run.nv; q += kTensorThreads, wg.next()) {
        const uint32_t i = run.head + q * 8;
        const Gathered8<T> raw = gather8<T>(from + wg.at, wg.col, wg.row, gap, lo, end);
        Float8 w = ld_state_32(p + i), mm = ld_state_32(m + i), vv = ld_state_32(v + i);
        if (skip()) return;
        float x[8];
        unpack_shifted8<T>(raw.v, raw.o, x);
        update(i, x, w, mm, vv);
      }
    } else if (run.o == 0) {
      for (uint32_t q = tid; q < run.nv; q += kTensorThreads) {
        const uint32_t i = run.head + q * 8;
        const Vec8<T> raw = load8<T>(g + i);
        Float8 w = ld_state_32(p + i), mm = ld_state_32(m + i), vv = ld_state_32(v + i);
        if (skip()) return;
        float x[8];
        unpack8<T>(raw, x);
        update(i, x, w, mm, vv);
      }
    } else {
      for (uint32_t q = tid; q < run.nv; q += kTensorThreads) {
        const uint32_t i = run.head + q * 8;
        const Shifted8<T> raw = load_shifted8<T>(g + i, run.o);
        Float8 w = ld_state_32(p + i), mm = ld_state_32(m + i), vv = ld_state_32(v + i);
        if (skip()) return;
        float x[8];
        unpack_shifted8<T>(raw, run.o, x);
        update(i, x, w, mm, vv);
      }
    }
    // head and rest, at most 15 elements each
    const uint32_t rest = run.head + run.nv * 8 + tid;
    if (tid < run.head || rest < r.n) {
      if (skip()) return;
      const auto one = [&](uint32_t k) {
        const S* at = runs ? lo + grad_walk<int64_t>(e, r.start + k, 1).base : g + k;
        adamw_one(a, state, r.start + k, factor * T::to_float(*at));
      };
      if (tid < run.head) one(tid);
      if (rest < r.n) one(rest);
    }
  });
}

// ---- small lists: everything in one cluster -------------------------------------------------
// Norm and second pass in one launch.  Up to kClusterBlocks blocks, launched as one cluster, hold
// the whole list in shared memory, and every block writes its sums into the shared memory of all before
// the cluster's barrier: no ticket, no round trip to L2, and no wait that could run out in one block and
// not in another (asynchronous stores counted on an mbarrier took 0.08 us less and had that).
enum { kOpNone = 0, kOpScale = 1, kOpAdamw = 2 };

// What a block has for the others: its sum, and its parts of the tensors that it shares.
struct BlockSums {
  double sum, edge[2];
};

// Writes x into the shared memory of block `rank`, to the place where `p` points in this one's.
__device__ __forceinline__ void send_double(const double* p, int rank, double x) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(a), "d"(x) : "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The bits of a value of a type known at run time, and the value.
__device__ __forceinline__ uint32_t load_bits(const char* p, bool wide) {
  return wide ? *reinterpret_cast<const uint32_t*>(p) : *reinterpret_cast<const uint16_t*>(p);
}
__device__ __forceinline__ float value_of(uint32_t bits, int dtype) {
  return dtype == ABS_F32    ? __uint_as_float(bits)
         : dtype == ABS_BF16 ? __uint_as_float(bits << 16)
                             : TF16::to_float(static_cast<uint16_t>(bits));
}

// AdamW on n elements, this lane's i0, i0 + 32, ...; bits(i) are those of element i's gradient.
template <typename F>
__device__ __forceinline__ void adamw_elements(const AdamScalars& a, const StateArrays& s,
                                               uint32_t i0, uint32_t n, float factor, int dtype,
                                               F&& bits) {
  constexpr int kBatch = 4;
#pragma unroll 1
  for (; i0 < n; i0 += kBatch * 32) {
    uint32_t x[kBatch];
    float p[kBatch], m[kBatch], v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const uint32_t i = i0 + j * 32;
      if (i < n) p[j] = s.p[i], m[j] = s.m[i], v[j] = s.v[i], x[j] = bits(i);
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const uint32_t i = i0 + j * 32;
      if (i < n) {
        adamw_elem(a, a.omb1, a.omb2, factor * value_of(x[j], dtype), p[j], m[j], v[j]);
        s.p[i] = p[j], s.m[i] = m[j], s.v[i] = v[j];
        if (s.p16) s.p16[i] = to_bf16(p[j]);
      }
    }
  }
}

// Where the second pass of a segment goes, out of its tensor's entry.
struct Target {
  const void* g;
  void* out;
  StateArrays state;
  int out_dtype, group;
};
__device__ __forceinline__ Target target_of(const TensorEntry& e) {
  return Target{e.g, e.out, {e.p, e.m, e.v, e.p16}, e.out_dtype, e.group};
}

template <int OP>
__device__ __forceinline__ void segment_apply(const TensorsParams& prm, const GroupScalars& groups,
                                              const Target& e, const Segment& s, uint32_t lane,
                                              float factor, const uint4* keep) {
  const int in = s.dtype;
  const bool rows = s.flags & kEntryRowsG, wide = in == ABS_F32;
  const uint32_t per = wide ? 4 : 8, esz = wide ? 4 : 2;
  // what lies in shared memory: the body of one run (head and rest, at most 7 elements each, are in
  // global memory), or a view with rows whole
  const uint32_t head = rows ? 0 : s.head, nv = rows ? 0 : (s.n - s.head) / per;
  const uint32_t body = rows ? s.n : nv * per;
  const int64_t first = s.start + head;
  const char* kept = reinterpret_cast<const char*>(keep - lane);
  const auto bits = [&](uint32_t i) {
    const char* p = i - head < body ? kept + (i - head) * esz
                                    : static_cast<const char*>(s.g) + static_cast<size_t>(i) * esz;
    return load_bits(p, wide);
  };
  if constexpr (OP == kOpScale) {
    const int out = prm.in_place ? in : e.out_dtype;
    void* y = prm.in_place ? const_cast<void*>(e.g) : e.out;
    if (prm.in_place ? rows : (s.flags & kEntryRowsOut) != 0) {
      const TensorEntry& full = prm.entries[s.tensor];
      Walk<int64_t> w = prm.in_place ? grad_walk<int64_t>(full, s.start + lane, 32)
                                     : out_walk(full, s.start + lane, 32);
#pragma unroll 4
      for (uint32_t i = lane; i < s.n; i += 32, w.next())
        store_any(y, w.base + w.at, out, factor * value_of(bits(i), in));
      return;
    }
    uint32_t i0 = lane, end = s.n;  // what is taken element by element
    if (s.flags & kEntryVecScale) {
      for (uint32_t v = lane; v < nv; v += 32)
        store_scaled(keep[v - lane], in, y, first + static_cast<int64_t>(v) * per, out, factor);
      i0 = lane < 8 ? (lane < s.head ? lane : s.n) : s.head + body + lane - 8;
      end = i0 < s.n && lane < 16 ? i0 + 1 : i0;
    }
    with_type(in, [&](auto type) {
      using T = decltype(type);
      using S = typename T::scalar;
      const S *g = static_cast<const S*>(s.g), *k = reinterpret_cast<const S*>(kept) - head;
#pragma unroll 4
      for (; i0 < end; i0 += 32) {
        const S* p = (i0 - head < body ? k : g) + i0;
        store_any(y, s.start + i0, out, factor * T::to_float(*p));
      }
    });
  } else {
    const AdamScalars& a = groups.a[e.group];
    const StateArrays at{e.state.p + s.start, e.state.m + s.start, e.state.v + s.start,
                         e.state.p16 ? e.state.p16 + s.start : nullptr};
    uint32_t i0 = lane, end = s.n;
    if (s.flags & kEntryVecAdamw) {
#pragma unroll 1
      for (uint32_t v = lane; v < nv; v += 32) {
        const uint32_t i = s.head + v * per;
        const uint4 raw = keep[v - lane];
        float4 w = ld_state_16(at.p + i), m = ld_state_16(at.m + i), q = ld_state_16(at.v + i);
        float4 w1, m1, q1;
        if (!wide)
          w1 = ld_state_16(at.p + i + 4), m1 = ld_state_16(at.m + i + 4), q1 = ld_state_16(at.v + i + 4);
        float x[8] = {};
        if (wide)
          TF32::unpack(raw, x);
        else if (in == ABS_BF16)
          TBF16::unpack(raw, x);
        else
          TF16::unpack(raw, x);
        const auto store = [&](uint32_t k, const float4& p, const float4& mm, const float4& vv) {
          st_stream_16(at.p + k, p);
          st_stream_16(at.m + k, mm);
          st_stream_16(at.v + k, vv);
          if (at.p16) st_bf16x4(at.p16 + k, p);
        };
        adamw_quad(a, make_float2(factor * x[0], factor * x[1]),
                   make_float2(factor * x[2], factor * x[3]), w, m, q);
        store(i, w, m, q);
        if (!wide) {
          adamw_quad(a, make_float2(factor * x[4], factor * x[5]),
                     make_float2(factor * x[6], factor * x[7]), w1, m1, q1);
          store(i + 4, w1, m1, q1);
        }
      }
      // head and rest in one go: lanes 0..7 and 8..15
      i0 = lane < 8 ? (lane < s.head ? lane : s.n) : s.head + body + lane - 8;
      end = i0 < s.n && lane < 16 ? i0 + 1 : i0;
    }
    adamw_elements(a, at, i0, end, factor, in, bits);
  }
}

// Bound by a chain of latencies: launch, table (read before the predecessor's
// end is waited for), rows, join, one store into the other blocks and their barrier, the factor, the
// second pass out of shared memory.  20 tensors of 60k fp32 together: norm 3.6 us, clip 5.1, AdamW 6.6;
// with the kernels above 5.0, 7.6 and 7.8.
template <int NORM, int OP>
__global__ void __launch_bounds__(kListWarps * 32, 1)
    tensors_cluster_kernel(const __grid_constant__ TensorsParams prm,
                           const __grid_constant__ GroupScalars groups, int rows) {
  extern __shared__ uint4 kept[];  // `rows` rows for each warp
  __shared__ BlockParts parts;
  __shared__ BlockSums all[kClusterBlocks];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int blocks = gridDim.x;
  // the others' shared memory may be written once all blocks have come here
  cluster_arrive();
  // the tables were there before any kernel of the stream
  const Segment opening = prm.opening[blockIdx.x * kListWarps + warp];
  Target target{};
  if (OP != kOpNone && opening.tensor >= 0) target = target_of(prm.entries[opening.tensor]);
  // tensors that several blocks share (at most blocks - 1), dealt out to the warps of the cluster
  const int w = blockIdx.x + blocks * warp;
  Spanning span{-1, 0, 0, 0};
  if (w < prm.n_spanning) span = prm.spanning[w];
  uint4* keep = kept + warp * rows * 32 + lane;
  cluster_wait();
  grid_dependency_wait();
  double sum = warp_sum<NORM, OP != kOpNone, true>(prm, opening, parts, keep);
  if (lane == 0) parts.sum[warp] = sum;
  __syncthreads();
  double x;
  const auto edge = [&](int k, double part) {
    if (lane < blocks) send_double(&all[blockIdx.x].edge[k], lane, part);
  };
  const int known = join_parts<NORM>(prm, parts, edge, x);
  if (warp == 0) {
    sum = join_warps<NORM>(parts.sum);
    if (lane < blocks) send_double(&all[blockIdx.x].sum, lane, sum);
  }
  cluster_arrive();
  if (known >= 0 && lane == 0) write_norm<NORM>(prm, known, x);
  cluster_wait();  // all sums are here, and nothing more is written into this block's shared memory
  grid_launch_dependents();
  const double total = warp_join<NORM>(lane < blocks ? all[lane].sum : 0.0);
  const Clip clip = clip_of(total, NORM, prm.scale, prm.max_norm);
  const bool skip = OP == kOpNone || (OP == kOpAdamw && !clip.finite) ||
                    (OP == kOpScale && prm.in_place && clip.factor == 1.f);
  if (!skip && opening.tensor >= 0) {
    if constexpr (OP != kOpNone) {
      Segment s = opening;
#pragma unroll 1
      for (int k = 0;; ++k) {
        segment_apply<OP>(prm, groups, target, s, lane, clip.factor, keep);
        if (k == opening.more) break;
        keep += kept_rows(s) * 32;
        s = prm.further[opening.next + k];
        target = target_of(prm.entries[s.tensor]);
      }
    }
  }
  if (span.tensor >= 0)
    join_spanning<NORM>(prm, span, [&](int b, int k) { return all[b].edge[k]; });
  if (blockIdx.x == 0) {
    if (threadIdx.x == 0) write_clip(prm, total, clip);
    for (int i = threadIdx.x; i < prm.n_empty; i += kListWarps * 32)
      write_norm<NORM>(prm, prm.empty[i], 0.0);
  }
}

}  // namespace absnt
