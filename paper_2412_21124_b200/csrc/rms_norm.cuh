// Root-mean-square norm of rows, with the residual's addition before it and an output in 16 or 32 bits or
// in 8 bits with scales:
//
//   s = x + residual,   rstd = (sum_c s_c^2 / h + eps)^(-1/2),   y_c = s_c rstd w_c
//
// One pass: a row is loaded once into registers (8 to 32 values a thread), its squares are summed over the threads
// that hold it, and y, the rounded s and the scales are written from the same registers.  s is not rounded before
// it is normalised.
//
// Bounds: HBM where the output has 16 or 32 bits, 16384 x 2048 with an fp32 residual stream 61 us, 6.6 TB/s;
// 524288 heads of 64 23 us, 5.7 TB/s.  In 8 bits with a scale for 32 values (8192 x 8192 92 us, 5.1 TB/s) it is latency: issue
// is 50% busy and DRAM 55%, with 15 warps an SM of 88 registers.  Two values in one instruction slot brought nothing: what they save goes into moving registers side by side.
#pragma once
#include "rows.cuh"

namespace absnt {

struct NormParams {
  RowsArg x, r, sum, out;
  unsigned char* scales;           // NULL unless the output has 8 bits
  int64_t scale_s0, scale_s1, scale_s2;  // in elements
  const unsigned char* w;          // may be NULL
  uint32_t rows;
  Divisor n1;
  int h, group, group_shift;       // columns of a scale, their log2; the row's width: one scale a row
  int w_dtype, sum_dtype, out_dtype, scale_dtype;
  float inv_h, eps;
};

// Above this a sum of squares over all threads of a row might not be finite although the row is; such
// rows (and those that hold an infinity or a NaN, which stay what they are) are summed again scaled.
constexpr float kSquaresLimit = 1e36f;
constexpr float kDown = 0x1p-80f;
// eps beside squares of scaled values: the factor's square alone is no float
__device__ __forceinline__ float down_squared(float eps) { return eps * kDown * kDown; }

// The scale of a group whose largest |y| has the bits `a`, as it is stored (a float's bits, or the byte), and its
// reciprocal.  Not finite: NaN, which makes all values of the group NaN.
__device__ __forceinline__ uint32_t scale_of(uint32_t a, int out_dtype, int scale_dtype, float& inv) {
  const bool wild = a >= 0x7f800000u, zero = a == 0u;
  uint32_t stored;
  if (scale_dtype == ABS_F32) {
    const float scale = fmaxf(__uint_as_float(a) / (out_dtype == ABS_E4M3 ? 448.f : 57344.f), 0x1p-126f);
    inv = zero ? 1.f : 1.f / scale;
    stored = zero ? 0x3f800000u : __float_as_uint(scale);
    if (wild) stored = 0x7fffffffu;
  } else {
    // the smallest 2^e with a <= M 2^e, where M = 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2); at least 2^-127: a's exponent,
    // one more if its fraction is above .75, less 8 or 15
    const int byte = max(static_cast<int>((a + 0x1fffffu) >> 23) - (out_dtype == ABS_E4M3 ? 8 : 15), 0);
    stored = wild ? 255u : zero ? 127u : static_cast<uint32_t>(byte);
    inv = __uint_as_float((254u - stored) << 23);
  }
  if (wild) inv = __uint_as_float(0x7fffffffu);
  return stored;
}
__device__ __forceinline__ void store_scale(unsigned char* scales, int64_t at, int scale_dtype, uint32_t stored) {
  if (scale_dtype == ABS_F32) reinterpret_cast<uint32_t*>(scales)[at] = stored;
  else scales[at] = static_cast<unsigned char>(stored);
}

// v^(-1/2) with one step of Newton's method behind the approximation, whose 2 units in the last place would decide more often
// than the other roundings on which side of a power of two, or of a tie of 8-bit values, a result falls
__device__ __forceinline__ float inverse_root(float v) {
  const float r = rsqrtf(v), t = v * r;
  const float e = fmaf(-fmaf(v, r, -t), r, fmaf(-t, r, 1.f));
  return fabsf(e) < 1.f ? fmaf(0.5f * r, e, r) : r;  // as it is for an infinity and a NaN
}

// max(a, |b|), NaN if one is: a's sign is clear
__device__ __forceinline__ float larger(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
  return r;
}
template <int NI, int E>
__device__ __forceinline__ float squares(const float (&s)[NI][E]) {
  float t[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < E; ++j) t[j & 1] = fmaf(s[i][j], s[i][j], t[j & 1]);
  return t[0] + t[1];
}
// BLOCK: a row a block, in NI pieces a thread.  Otherwise L lanes hold a row in NI pieces, NR rows of a group of
// lanes at once; blockDim.y warps a block.
template <int XT, int RT, int VEC, int L, int NI, int NR, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? (NI * lane_values<VEC>() > 16 ? 512 : 1024) : 256, BLOCK ? 1 : NI > 2 ? 3 : 4)
    rms_norm_kernel(const NormParams p) {
  constexpr int E = lane_values<VEC>();
  constexpr bool HAS_R = RT >= 0;
  constexpr int kGroups = 32 / L;
  __shared__ float part[BLOCK ? 32 : 1];
  __shared__ float part_again[BLOCK ? 32 : 1];
  __shared__ uint32_t part_max[BLOCK ? 32 : 1];

  const int lane = threadIdx.x & 31, l = lane % L;
  const int warps = BLOCK ? static_cast<int>(blockDim.x) >> 5 : 1;       // of a row
  const int warp = BLOCK ? static_cast<int>(threadIdx.x) >> 5 : 0;       // in the row
  const uint32_t slot = BLOCK ? blockIdx.x : (blockIdx.x * blockDim.y + threadIdx.y) * (kGroups * NR) + lane / L;
  uint32_t row[NR], ri[NR], rj[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    row[k] = slot + k * kGroups;
    split_row(row[k], p.n1, ri[k], rj[k]);
  }
  grid_dependency_wait();

  float s[NR][NI][E];
  {
    Piece<XT, VEC> x[NR][NI];
    Piece<HAS_R ? RT : XT, VEC> r[HAS_R ? NR : 1][HAS_R ? NI : 1];
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const int h = row[k] < p.rows ? p.h : 0;  // nothing is loaded for rows behind the last
      const unsigned char* px = row_of<VEC>(p.x, ri[k], rj[k]);
      const unsigned char* pr = HAS_R ? row_of<VEC>(p.r, ri[k], rj[k]) : nullptr;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        x[k][i].load(px, (i * warps + warp) * (L * E), l, h);
        if constexpr (HAS_R) r[k][i].load(pr, (i * warps + warp) * (L * E), l, h);
      }
    }
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          s[k][i][j] = x[k][i].get(j);
          if constexpr (HAS_R) s[k][i][j] += r[k][i].get(j);
        }
  }

  float ss[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    ss[k] = lanes_sum<L>(squares(s[k]));
  }

  // the rounded sum goes out while the row's warps wait for one another
  if constexpr (HAS_R) {
    if (p.sum.p) {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (row[k] < p.rows) {
          unsigned char* ps = row_of<VEC>(p.sum, ri[k], rj[k]);
#pragma unroll
          for (int i = 0; i < NI; ++i) store_piece<RT, VEC>(ps, (i * warps + warp) * (L * E), l, p.h, s[k][i]);
        }
    }
  }

  bool again;  // some row of the block (the warp) needs its squares summed again, scaled
  if constexpr (BLOCK) {
    if (lane == 0) part[warp] = ss[0];
    __syncthreads();
    const float t = lane < warps ? part[lane] : 0.f;
    again = __any_sync(0xffffffffu, !(t <= kSquaresLimit));
    ss[0] = lanes_sum<32>(t);
  } else {
    bool over = false;
#pragma unroll
    for (int k = 0; k < NR; ++k) over |= !(ss[k] <= kSquaresLimit);
    again = __any_sync(0xffffffffu, over);
  }
  float rstd[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) rstd[k] = inverse_root(fmaf(ss[k], p.inv_h, p.eps));
  if (again) {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const bool down = !(ss[k] <= kSquaresLimit);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) s[k][i][j] *= down ? kDown : 1.f;
      float t = lanes_sum<L>(squares(s[k]));
      if constexpr (BLOCK) {
        if (lane == 0) part_again[warp] = t;
        __syncthreads();
        t = lanes_sum<32>(lane < warps ? part_again[lane] : 0.f);
      }
      if (down) rstd[k] = inverse_root(fmaf(t, p.inv_h, down_squared(p.eps)));
    }
  }

  // y, piece by piece; the branches on the types are taken once for all of a thread's pieces.
  // For 8 bits rstd is 2^e f with f in [1, 2), and y / f is formed: s 2^e w, mostly without a rounding for 16-bit tensors (s rstd w
  // falls to the other side of a tie a third more often), and a float wherever y is one (s w need not be).  So is f times
  // the scale's reciprocal, which is at most 2^127.  An rstd of 0 has f = 1, a NaN an infinite power.
  float frac[NR];
  auto split_rstd = [&]() {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const uint32_t bits = __float_as_uint(rstd[k]);
      frac[k] = __uint_as_float((bits & 0x007fffffu) | 0x3f800000u);
      rstd[k] = __uint_as_float(bits & 0x7f800000u);
    }
  };
  auto normalise = [&]() {
    with_type(p.w_dtype, [&](auto wt) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float w[E];
        load_weight_of<decltype(wt)::value, VEC>(w, p.w, (i * warps + warp) * (L * E), l, p.h);
#pragma unroll
        for (int k = 0; k < NR; ++k)
#pragma unroll
          for (int j = 0; j < E; ++j) s[k][i][j] = s[k][i][j] * rstd[k] * w[j];
      }
    });
  };
  // before the branch on the output for rows of lanes (524288 heads of 64: 23.0 us, in either branch 23.7), in either branch for
  // rows of blocks (8192 x 8192 into 8 bits: 92.6 us, before it 94.2)
  if constexpr (!BLOCK) {
    if (p.scales) split_rstd();
    normalise();
  }
  if (!p.scales) {
    if constexpr (BLOCK) normalise();
    with_type(p.out_dtype, [&](auto ot) {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (row[k] < p.rows) {
          unsigned char* const po = row_of<VEC>(p.out, ri[k], rj[k]);
#pragma unroll
          for (int i = 0; i < NI; ++i) store_piece<decltype(ot)::value, VEC>(po, (i * warps + warp) * (L * E), l, p.h, s[k][i]);
        }
    });
    return;
  }

  // 8 bits: the largest |y| of each group
  if constexpr (BLOCK) {
    split_rstd();
    normalise();
  }
  uint32_t a_row[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) a_row[k] = 0u;
  const bool of_row = p.group >= p.h;
  if (of_row) {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) a = larger(a, s[k][i][j]);
      a_row[k] = lanes_max(__float_as_uint(a), L);
      if constexpr (BLOCK) {
        if (lane == 0) part_max[warp] = a_row[k];
        __syncthreads();
        a_row[k] = lanes_max(lane < warps ? part_max[lane] : 0u, 32);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const bool live = row[k] < p.rows;
    unsigned char* const po = row_of<VEC>(p.out, ri[k], rj[k]);
    auto scale_from = [&](uint32_t a, bool writer, int group) {
      float inv;
      const uint32_t stored = scale_of(__float_as_uint(__uint_as_float(a) * frac[k]) & 0x7fffffffu, p.out_dtype, p.scale_dtype, inv);
      if (writer && live)
        store_scale(p.scales, ri[k] * p.scale_s0 + rj[k] * p.scale_s1 + group * p.scale_s2, p.scale_dtype, stored);
      return inv * frac[k];
    };
    if (of_row) {
      const float inv = scale_from(a_row[k], l == 0 && warp == 0, 0);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) s[k][i][j] *= inv;
    } else if constexpr (VEC == 1) {
      // a group is 1, 2 or 4 of the four values of every lane; the scale of value v's group is worked out by lane v
      static_assert(NI * E <= 32, "a lane for every value");
      uint32_t a = 0u;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(s[k][i][j]) & 0x7fffffffu);
          if (lane == i * E + j) a = top;
        }
      if (p.group >= 64) a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
      if (p.group >= 128) a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
      const int c = ((lane / E) * warps + warp) * (L * E) + 32 * (lane % E);
      const float inv = scale_from(a, lane < NI * E && c < p.h && (c & (p.group - 1)) == 0, c >> p.group_shift);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) s[k][i][j] *= __shfl_sync(0xffffffffu, inv, i * E + j);
    } else {
      uint32_t a[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) top = larger(top, s[k][i][j]);
        // the lanes of a group: 32 / VEC, twice or four times as many
        a[i] = __float_as_uint(top);
#pragma unroll
        for (int d = 1; d < 32 / VEC; d <<= 1) a[i] = max(a[i], __shfl_xor_sync(0xffffffffu, a[i], d));
        if (p.group >= 64) a[i] = max(a[i], __shfl_xor_sync(0xffffffffu, a[i], 32 / VEC));
        if (p.group >= 128) a[i] = max(a[i], __shfl_xor_sync(0xffffffffu, a[i], 64 / VEC));
      }
      // of four lanes, which are always of one group, each works out the scale of another piece
      static_assert(NI <= 4 && 32 / VEC >= 4, "a lane for every piece");
      const int i_mine = NI > 1 ? l & 3 : 0;
      uint32_t a_mine = a[0];
#pragma unroll
      for (int i = 1; i < NI; ++i)
        if (i_mine == i) a_mine = a[i];
      const int c = (i_mine * warps + warp) * (L * E) + (l - i_mine) * VEC;
      const float inv_mine = scale_from(a_mine, i_mine < NI && c < p.h && (c & (p.group - 1)) == 0, c >> p.group_shift);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const float inv = NI > 1 ? __shfl_sync(0xffffffffu, inv_mine, (lane & ~3) | i) : inv_mine;
#pragma unroll
        for (int j = 0; j < E; ++j) s[k][i][j] *= inv;
      }
    }
    if (live) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int first = (i * warps + warp) * (L * E);
        if (p.out_dtype == ABS_E4M3) store_piece<ABS_E4M3, VEC>(po, first, l, p.h, s[k][i]);
        else store_piece<ABS_E5M2, VEC>(po, first, l, p.h, s[k][i]);
      }
    }
  }
}

}  // namespace absnt
