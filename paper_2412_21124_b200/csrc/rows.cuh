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

#include <type_traits>

#include "abs_device.cuh"

namespace absnt {

// Rows of a matrix as a kernel sees them; strides in bytes, and in units of `unit` bytes (the size of a thread's access)
// where rows are read in vectors: one multiplication of 32 bits finds a row that lies up to 2^32 units away.
struct RowsArg {
  unsigned char* p;
  int64_t s0, s1;
  uint32_t u0, u1, unit;
};
__device__ __forceinline__ unsigned char* row_of(const RowsArg& a, uint32_t i, uint32_t j) {
  return a.p + static_cast<int64_t>(i) * a.s0 + static_cast<int64_t>(j) * a.s1;
}
template <int VEC>
__device__ __forceinline__ unsigned char* row_of(const RowsArg& a, uint32_t i, uint32_t j) {
  if constexpr (VEC == 1) return row_of(a, i, j);
  return a.p + static_cast<uint64_t>(i * a.u0 + j * a.u1) * a.unit;
}

// n / d for n < 2^31 as a product with m = ceil(2^(31 + s) / d), s = ceil(log2 d): m d exceeds 2^(31 + s) by less than d <=
// 2^s, so n m / 2^(31 + s) exceeds n / d by less than n / (2^31 d) < 1 / d, which never reaches the next whole number.
struct Divisor {
  uint32_t d, m, shift;  // shift: s - 1
};
inline Divisor divisor(uint32_t d) {
  Divisor r = {d, 0, 0};
  if (d < 2) return r;
  uint32_t s = 1;
  while ((uint64_t{1} << s) < d) ++s;
  r.m = static_cast<uint32_t>(((uint64_t{1} << (31 + s)) + d - 1) / d);
  r.shift = s - 1;
  return r;
}
__device__ __forceinline__ void split_row(uint32_t row, const Divisor& by, uint32_t& i, uint32_t& j) {
  i = by.d == 1 ? row : __umulhi(row, by.m) >> by.shift;
  j = by.d == 1 ? 0u : row - i * by.d;
}

// ---- two floats in one instruction slot
__device__ __forceinline__ uint64_t pair_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 pair_as(uint64_t x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ uint64_t pair_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t pair_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
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

template <int DT>
__device__ __forceinline__ float load_value(const unsigned char* row, int i) {
  if constexpr (DT == ABS_F32) return reinterpret_cast<const float*>(row)[i];
  return from_half_word<DT>(reinterpret_cast<const unsigned short*>(row)[i]);
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
      const unsigned char* const at = row + static_cast<int64_t>(first + l) * elem_bytes<DT>();
      auto one = [&](int j) {
        if constexpr (DT == ABS_F32) {
          asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];" : "=r"(w[j]) : "l"(at + 128 * j));
        } else {
          asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=r"(w[j]) : "l"(at + 64 * j));
        }
      };
      if (first + 128 <= h) {  // all of the warp's pieces but the row's last
#pragma unroll
        for (int j = 0; j < E; ++j) one(j);
      } else {
#pragma unroll
        for (int j = 0; j < E; ++j) {
          w[j] = 0u;
          if (first + l + 32 * j < h) one(j);
        }
      }
    } else {
      const int c = first + l * VEC;
      zero();
      if (c < h) {
        const unsigned char* p = row + static_cast<uint32_t>(c) * elem_bytes<DT>();
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
  // what follows unpacks the words again instead of keeping the values in twice the registers until then
  __device__ __forceinline__ void keep_packed() {
    if constexpr (DT != ABS_F32) {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) asm volatile("" : "+r"(w[k]));
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
    unsigned char* const at = row + static_cast<int64_t>(first + l) * elem_bytes<DT>();
    auto one = [&](int j) {
      if constexpr (DT == ABS_F32) reinterpret_cast<float*>(at)[32 * j] = v[j];
      else if constexpr (DT == ABS_BF16) reinterpret_cast<__nv_bfloat16*>(at)[32 * j] = __float2bfloat16_rn(v[j]);
      else if constexpr (DT == ABS_F16) reinterpret_cast<__half*>(at)[32 * j] = __float2half_rn(v[j]);
      else at[32 * j] = __nv_cvt_float_to_fp8(v[j], __NV_SATFINITE, DT == ABS_E4M3 ? __NV_E4M3 : __NV_E5M2);
    };
    if (first + 128 <= h) {
#pragma unroll
      for (int j = 0; j < E; ++j) one(j);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (first + l + 32 * j < h) one(j);
    }
  } else {
    const int c = first + l * VEC;
    if (c >= h) return;
    unsigned char* p = row + static_cast<uint32_t>(c) * elem_bytes<DT>();
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

// f(the type) for one of the three types of 16 and 32 bits that is known when the kernel runs, the same for all threads
template <typename F>
__device__ __forceinline__ void with_type(int dt, F f) {
  if (dt == ABS_BF16) f(std::integral_constant<int, ABS_BF16>());
  else if (dt == ABS_F32) f(std::integral_constant<int, ABS_F32>());
  else f(std::integral_constant<int, ABS_F16>());
}

// E values of a contiguous vector (a weight); ones if there is none.  Every row wants the same few lines: they are
// left in L1.  From L2 alone, where all SMs ask for them at once, 50000 rows of 385 took 112 us instead of the 50 with
// a weight of twice the size, in twice the lines.
template <int DT, int VEC>
__device__ __forceinline__ void load_weight_of(float* v, const unsigned char* w, int first, int l, int h) {
  constexpr int E = lane_values<VEC>();
#pragma unroll
  for (int j = 0; j < E; ++j) v[j] = 1.f;
  if (!w) return;
  if constexpr (VEC == 1) {
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (first + l + 32 * j < h) v[j] = load_value<DT>(w, first + l + 32 * j);
  } else {
    const int c = first + l * VEC;
    if (c >= h) return;
    Piece<DT, VEC> piece;
    const unsigned char* const at = w + static_cast<uint32_t>(c) * elem_bytes<DT>();
    if constexpr (piece.WORDS == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(at);
      piece.w[0] = x.x;
      piece.w[1] = x.y;
    } else {
#pragma unroll
      for (int k = 0; k < piece.WORDS / 4; ++k) {
        const uint4 x = reinterpret_cast<const uint4*>(at)[k];
        piece.w[4 * k] = x.x;
        piece.w[4 * k + 1] = x.y;
        piece.w[4 * k + 2] = x.z;
        piece.w[4 * k + 3] = x.w;
      }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = piece.get(j);
  }
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
