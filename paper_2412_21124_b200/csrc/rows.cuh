// Device-side pieces shared by the kernels that work on rows of a matrix: pieces of a row as a warp
// loads and stores them, for every element type, and sums and maxima over the lanes of a row.
//
// A warp (or L of its lanes) takes a piece of L*E consecutive columns at a time, E values a lane:
//   VEC 8  columns 8l .. 8l+7 of lane l: one 128-bit access of 16-bit values, one 256-bit access of floats
//   VEC 4  columns 4l .. 4l+3: rows that start on multiples of four values only (heads of 100)
//   VEC 1  columns l, l+32, l+64, l+96: any alignment, any width
// The columns of a piece are consecutive in each case, so that a scale for 32, 64 or 128 columns never
// needs more than one warp.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "abs_device.cuh"

namespace absnt {

// rows of a matrix as a kernel sees them; strides in bytes
struct RowsArg {
  unsigned char* p;
  int64_t s0, s1;
};
__device__ __forceinline__ unsigned char* row_of(const RowsArg& a, uint32_t i, uint32_t j) {
  return a.p + static_cast<int64_t>(i) * a.s0 + static_cast<int64_t>(j) * a.s1;
}

template <int DT>
__host__ __device__ constexpr int elem_bytes() {
  return DT == ABS_F32 ? 4 : (DT == ABS_BF16 || DT == ABS_F16) ? 2 : 1;
}
template <int VEC>
__host__ __device__ constexpr int lane_values() {
  return VEC == 8 ? 8 : 4;
}
// the column of value j of lane l in a piece that begins at column `first`
template <int VEC>
__device__ __forceinline__ int col_of(int first, int l, int j) {
  return VEC == 1 ? first + l + 32 * j : first + l * VEC + j;
}

template <int DT>
__device__ __forceinline__ float from_half_word(uint32_t w) {  // 16 bits in the low half
  if constexpr (DT == ABS_BF16) return __uint_as_float(w << 16);
  return __half2float(__ushort_as_half(static_cast<unsigned short>(w)));
}

// The values of one lane in one piece, as loaded.  Rows are read once: their loads leave no copy in L1.
// They do not go through the read-only path either, since an output may lie where an input does.
template <int DT, int VEC>
struct Piece {
  static constexpr int E = lane_values<VEC>();
  static constexpr int WORDS = DT == ABS_F32 ? E : (VEC == 1 ? E : E / 2);
  uint32_t w[WORDS];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w[k] = 0u;
  }
  __device__ __forceinline__ void load(const unsigned char* row, int first, int l, int h) {
    if constexpr (VEC == 1) {
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const int c = first + l + 32 * j;
        w[j] = 0u;
        if (c < h) {
          if constexpr (DT == ABS_F32) {
            asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];" : "=r"(w[j]) : "l"(row + 4 * static_cast<int64_t>(c)));
          } else {
            unsigned short x;
            asm volatile("ld.global.L1::no_allocate.b16 %0, [%1];" : "=h"(x) : "l"(row + 2 * static_cast<int64_t>(c)));
            w[j] = x;
          }
        }
      }
    } else {
      const int c = first + l * VEC;
      zero();
      if (c < h) {
        const unsigned char* p = row + static_cast<int64_t>(c) * elem_bytes<DT>();
        if constexpr (WORDS == 8) {
          asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                       : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]),
                         "=r"(w[7])
                       : "l"(p));
        } else if constexpr (WORDS == 4) {
          asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                       : "l"(p));
        } else {
          asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
        }
      }
    }
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (DT == ABS_F32) return __uint_as_float(w[j]);
    if constexpr (VEC == 1) return from_half_word<DT>(w[j]);
    const uint32_t x = w[j >> 1];
    if constexpr (DT == ABS_BF16) return __uint_as_float((j & 1) ? (x & 0xffff0000u) : (x << 16));
    return from_half_word<DT>((j & 1) ? (x >> 16) : (x & 0xffffu));
  }
};

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int DT>
__device__ __forceinline__ uint32_t pack_16x2(float lo, float hi) {
  if constexpr (DT == ABS_BF16) return pack_bf16x2(lo, hi);
  return pack_f16x2(lo, hi);
}

// E values of a lane rounded once (to nearest, ties to even) to type DT and written.  8-bit types
// take values that their scale has brought into range; NaN stays NaN.
template <int DT, int VEC>
__device__ __forceinline__ void store_piece(unsigned char* row, int first, int l, int h, const float* v) {
  constexpr int E = lane_values<VEC>();
  if constexpr (VEC == 1) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int c = first + l + 32 * j;
      if (c >= h) continue;
      if constexpr (DT == ABS_F32) reinterpret_cast<float*>(row)[c] = v[j];
      else if constexpr (DT == ABS_BF16) reinterpret_cast<__nv_bfloat16*>(row)[c] = __float2bfloat16_rn(v[j]);
      else if constexpr (DT == ABS_F16) reinterpret_cast<__half*>(row)[c] = __float2half_rn(v[j]);
      else row[c] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, DT == ABS_E4M3 ? __NV_E4M3 : __NV_E5M2);
    }
  } else {
    const int c = first + l * VEC;
    if (c >= h) return;
    unsigned char* p = row + static_cast<int64_t>(c) * elem_bytes<DT>();
    if constexpr (DT == ABS_F32) {
      if constexpr (VEC == 8)
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]),
                     "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                     : "memory");
      else
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else if constexpr (DT == ABS_BF16 || DT == ABS_F16) {
      uint32_t w[E / 2];
#pragma unroll
      for (int k = 0; k < E / 2; ++k) w[k] = pack_16x2<DT>(v[2 * k], v[2 * k + 1]);
      if constexpr (VEC == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
      uint32_t w[E / 4];
#pragma unroll
      for (int k = 0; k < E / 4; ++k) {
        const __nv_fp8_interpretation_t as = DT == ABS_E4M3 ? __NV_E4M3 : __NV_E5M2;
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * k], v[4 * k + 1]), __NV_SATFINITE, as);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * k + 2], v[4 * k + 3]), __NV_SATFINITE, as);
        w[k] = lo | (hi << 16);
      }
      if constexpr (VEC == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(p) = w[0];
    }
  }
}

// the same for a type known when the kernel runs (the same for all threads)
template <int VEC>
__device__ __forceinline__ void store_piece_as(int dt, unsigned char* row, int first, int l, int h, const float* v) {
  if (dt == ABS_BF16) store_piece<ABS_BF16, VEC>(row, first, l, h, v);
  else if (dt == ABS_F32) store_piece<ABS_F32, VEC>(row, first, l, h, v);
  else if (dt == ABS_F16) store_piece<ABS_F16, VEC>(row, first, l, h, v);
  else if (dt == ABS_E4M3) store_piece<ABS_E4M3, VEC>(row, first, l, h, v);
  else store_piece<ABS_E5M2, VEC>(row, first, l, h, v);
}

// E values of a contiguous vector (a weight) of a type known when the kernel runs; ones if there is none
template <int VEC>
__device__ __forceinline__ void load_weight(float* v, const unsigned char* w, int dt, int first, int l, int h) {
  constexpr int E = lane_values<VEC>();
  if (!w) {
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = 1.f;
    return;
  }
  auto take = [&](auto piece) {
    piece.load(w, first, l, h);
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = piece.get(j);
  };
  if (dt == ABS_BF16) take(Piece<ABS_BF16, VEC>());
  else if (dt == ABS_F32) take(Piece<ABS_F32, VEC>());
  else take(Piece<ABS_F16, VEC>());
}

// sums and maxima over the aligned group of L lanes that a thread belongs to, in a fixed order
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int d = L / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t x, int lanes) {
  for (int d = lanes / 2; d > 0; d >>= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, d));
  return x;
}

}  // namespace absnt
