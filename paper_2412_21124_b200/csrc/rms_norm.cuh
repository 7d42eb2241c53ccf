// Root-mean-square norm of rows, with the residual's addition before it and an output in 16 or 32 bits or
// in 8 bits with scales:
//
//   s = x + residual,   rstd = (sum_c s_c^2 / h + eps)^(-1/2),   y_c = s_c rstd w_c
//
// One pass: a row is loaded once into registers (at most 32 values a thread), its squares are summed over
// the threads that hold it, and y, the rounded s and the scales are written from the same registers.  s is
// not rounded before it is normalised.  Bound by HBM: 2 to 12 bytes a value and about ten instructions.
#pragma once
#include "rows.cuh"

namespace absnt {

struct NormParams {
  RowsArg x, r, sum, out;
  unsigned char* scales;           // NULL unless the output has 8 bits
  int64_t scale_s0, scale_s1, scale_s2;  // in elements
  const unsigned char* w;          // may be NULL
  uint32_t rows, n1;
  int h, group;                    // columns of a scale; the row's width: one scale a row
  int w_dtype, sum_dtype, out_dtype, scale_dtype;
  float inv_h, eps;
};

// Above this a sum of squares over all threads of a row might not be finite although the row is; such
// rows (and those that hold an infinity or a NaN, which stay what they are) are summed again scaled.
constexpr float kSquaresLimit = 1e36f;
constexpr float kDown = 0x1p-80f;

// The scale of a group whose largest |y| has the bits `a`, and its reciprocal.  Not finite: NaN, which
// makes all values of the group NaN.
__device__ __forceinline__ void scale_of(uint32_t a, int out_dtype, int scale_dtype, float& scale, float& inv) {
  if (a >= 0x7f800000u) {
    scale = inv = __uint_as_float(0x7fffffffu);
  } else if (a == 0u) {
    scale = inv = 1.f;
  } else if (scale_dtype == ABS_F32) {
    scale = fmaxf(__uint_as_float(a) / (out_dtype == ABS_E4M3 ? 448.f : 57344.f), 0x1p-126f);
    inv = 1.f / scale;
  } else {
    // the smallest 2^e with a <= M 2^e, where M = 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2); at least 2^-127
    int e = static_cast<int>(a >> 23) - 127 - (out_dtype == ABS_E4M3 ? 8 : 15) + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = max(e, -127);
    scale = __uint_as_float(static_cast<uint32_t>(e + 127));  // the byte; see store_scale
    inv = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  }
}
__device__ __forceinline__ void store_scale(unsigned char* scales, int64_t at, int scale_dtype, uint32_t a, float scale) {
  if (scale_dtype == ABS_F32) {
    reinterpret_cast<float*>(scales)[at] = scale;
  } else {
    scales[at] = a >= 0x7f800000u ? 255 : a == 0u ? 127 : static_cast<unsigned char>(__float_as_uint(scale));
  }
}

// L lanes (a whole warp if BLOCK: blockDim.x / 32 of them) hold one row in NI pieces; without BLOCK a group
// of lanes takes NR rows at once.  blockDim.y rows (warps) a block.
template <int XT, int RT, int VEC, int L, int NI, int NR, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? (NI * lane_values<VEC>() > 16 ? 512 : 1024) : 256)
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
  const int mine = BLOCK ? static_cast<int>(threadIdx.y) * warps : 0;    // first of the row's slots in part[]
  const uint32_t slot = BLOCK ? blockIdx.x * blockDim.y + threadIdx.y
                              : (blockIdx.x * blockDim.y + threadIdx.y) * (kGroups * NR) + lane / L;
  uint32_t row[NR], ri[NR], rj[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    row[k] = slot + k * kGroups;
    ri[k] = p.n1 == 1 ? row[k] : row[k] / p.n1;
    rj[k] = p.n1 == 1 ? 0 : row[k] - ri[k] * p.n1;
  }
  grid_dependency_wait();

  float s[NR][NI][E];
  {
    Piece<XT, VEC> x[NR][NI];
    Piece<HAS_R ? RT : XT, VEC> r[HAS_R ? NR : 1][HAS_R ? NI : 1];
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const int h = row[k] < p.rows ? p.h : 0;  // nothing is loaded for rows behind the last
      const unsigned char* px = row_of(p.x, ri[k], rj[k]);
      const unsigned char* pr = HAS_R ? row_of(p.r, ri[k], rj[k]) : nullptr;
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
    ss[k] = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < E; ++j) ss[k] = fmaf(s[k][i][j], s[k][i][j], ss[k]);
    ss[k] = lanes_sum<L>(ss[k]);
  }

  // the rounded sum goes out while the row's warps wait for one another
  if constexpr (HAS_R) {
    if (p.sum.p) {
#pragma unroll
      for (int k = 0; k < NR; ++k)
        if (row[k] < p.rows) {
          unsigned char* ps = row_of(p.sum, ri[k], rj[k]);
#pragma unroll
          for (int i = 0; i < NI; ++i)
            store_piece<RT, VEC>(ps, (i * warps + warp) * (L * E), l, p.h, s[k][i]);
        }
    }
  }

  bool again;  // some row of the block (the warp) needs its squares summed again, scaled
  if constexpr (BLOCK) {
    if (lane == 0) part[mine + warp] = ss[0];
    __syncthreads();
    const int all = warps * static_cast<int>(blockDim.y);
    again = __any_sync(0xffffffffu, lane < all && !(part[lane < all ? lane : 0] <= kSquaresLimit));
    ss[0] = lanes_sum<32>(lane < warps ? part[mine + lane] : 0.f);
  } else {
    bool over = false;
#pragma unroll
    for (int k = 0; k < NR; ++k) over |= !(ss[k] <= kSquaresLimit);
    again = __any_sync(0xffffffffu, over);
  }
  float rstd[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) rstd[k] = rsqrtf(fmaf(ss[k], p.inv_h, p.eps));
  if (again) {
#pragma unroll
    for (int k = 0; k < NR; ++k) {
      const bool down = !(ss[k] <= kSquaresLimit);
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          if (down) s[k][i][j] *= kDown;
          t = fmaf(s[k][i][j], s[k][i][j], t);
        }
      t = lanes_sum<L>(t);
      if constexpr (BLOCK) {
        if (lane == 0) part_again[mine + warp] = t;
        __syncthreads();
        t = lanes_sum<32>(lane < warps ? part_again[mine + lane] : 0.f);
      }
      if (down) rstd[k] = rsqrtf(t * p.inv_h);
    }
  }

#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int first = (i * warps + warp) * (L * E);
    float w[E];
    load_weight<VEC>(w, p.w, p.w_dtype, first, l, p.h);
#pragma unroll
    for (int k = 0; k < NR; ++k)
#pragma unroll
      for (int j = 0; j < E; ++j) s[k][i][j] = s[k][i][j] * rstd[k] * w[j];
  }

  if (p.scales) {
    if (p.group >= p.h) {  // one scale a row
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        uint32_t a = 0u;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) a = max(a, __float_as_uint(s[k][i][j]) & 0x7fffffffu);
        a = lanes_max(a, L);
        if constexpr (BLOCK) {
          if (lane == 0) part_max[mine + warp] = a;
          __syncthreads();
          a = lanes_max(lane < warps ? part_max[mine + lane] : 0u, 32);
        }
        float scale, inv;
        scale_of(a, p.out_dtype, p.scale_dtype, scale, inv);
        if (l == 0 && warp == 0 && row[k] < p.rows)
          store_scale(p.scales, ri[k] * p.scale_s0 + rj[k] * p.scale_s1, p.scale_dtype, a, scale);
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) s[k][i][j] *= inv;
      }
    } else {
#pragma unroll
      for (int k = 0; k < NR; ++k)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int first = (i * warps + warp) * (L * E);
          const int64_t at = ri[k] * p.scale_s0 + rj[k] * p.scale_s1;
          if constexpr (VEC == 1) {  // a group is 1, 2 or 4 of the four values of every lane
            uint32_t a[E];
#pragma unroll
            for (int j = 0; j < E; ++j) a[j] = lanes_max(__float_as_uint(s[k][i][j]) & 0x7fffffffu, 32);
            if (p.group >= 64) {
              a[0] = a[1] = max(a[0], a[1]);
              a[2] = a[3] = max(a[2], a[3]);
            }
            if (p.group >= 128) a[0] = a[1] = a[2] = a[3] = max(a[0], a[2]);
#pragma unroll
            for (int j = 0; j < E; ++j) {
              float scale, inv;
              scale_of(a[j], p.out_dtype, p.scale_dtype, scale, inv);
              const int c = first + 32 * j;
              if (l == 0 && c < p.h && c % p.group == 0 && row[k] < p.rows)
                store_scale(p.scales, at + c / p.group * p.scale_s2, p.scale_dtype, a[j], scale);
              s[k][i][j] *= inv;
            }
          } else {
            uint32_t a = 0u;
#pragma unroll
            for (int j = 0; j < E; ++j) a = max(a, __float_as_uint(s[k][i][j]) & 0x7fffffffu);
            a = lanes_max(a, min(p.group / VEC, L));
            float scale, inv;
            scale_of(a, p.out_dtype, p.scale_dtype, scale, inv);
            const int c = first + l * VEC;
            if (c < p.h && c % p.group == 0 && row[k] < p.rows)
              store_scale(p.scales, at + c / p.group * p.scale_s2, p.scale_dtype, a, scale);
#pragma unroll
            for (int j = 0; j < E; ++j) s[k][i][j] *= inv;
          }
        }
    }
  }

#pragma unroll
  for (int k = 0; k < NR; ++k)
    if (row[k] < p.rows) {
      unsigned char* po = row_of(p.out, ri[k], rj[k]);
#pragma unroll
      for (int i = 0; i < NI; ++i)
        store_piece_as<VEC>(p.out_dtype, po, (i * warps + warp) * (L * E), l, p.h, s[k][i]);
    }
}

}  // namespace absnt
