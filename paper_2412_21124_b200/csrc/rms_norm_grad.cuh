// Backward pass of the root-mean-square norm, with the weight's gradient of every sample of a packed batch:
//
//   rstd = (sum_c s_c^2 / h + eps)^(-1/2),  u_c = s_c rstd,  g_c = dy_c w_c,  a = sum_c g_c u_c / h
//   dx_c = rstd (g_c - u_c a) + dresidual_c
//   dw_c of sample b = sum over the rows of b of dy_c u_c
//
// rstd is formed again from s, which the pass reads anyway: one sum more in a row's reduction instead of a
// saved vector that has to fit its rows.  Here it is the approximate root as it comes, two units in the last place of fp32:
// no result of 8 bits hangs on it, as in the forward pass.
//
// Every block takes an equal run of consecutive rows, so that the sums over rows stay in registers while it
// walks them; it writes them once for each sample that it meets (a piece) and once for the whole run (a
// total).  A second kernel adds the pieces of each sample and the totals, in order: results do not depend
// on scheduling and no atomics are needed.  Piece (block c, sample b) lies at c + b: along the rows one of
// the two grows at every step, so that no two pieces share a place and a table is not needed.
//
// Bounds: HBM for rows that are read in vectors, 16384 x 2048 with an fp32 stream, the residual's gradient and eight samples
// 82 us, 5.7 TB/s, of which the records' sums are 5; 524288 heads of 64 46 us, 4.3 TB/s.  Rows on odd boundaries are read a
// value at a time, and issue bounds them: 9001 x 1537 in 16 bits 46 us, 2.4 TB/s (shifted 16-byte windows were slower: what
// they save in loads goes into the shifts).
#pragma once
#include "rms_norm.cuh"

namespace absnt {

struct NormGradParams {
  RowsArg dy, s, add, dx;          // add.p may be NULL
  const unsigned char* w;          // may be NULL
  const int32_t* offsets;          // NULL: all rows, one sample
  float *totals, *pieces;          // may be NULL
  int64_t pitch;                   // floats between two records
  uint32_t rows;
  Divisor n1;
  int n_samples;
  int h, w_dtype, dx_dtype;
  float inv_h, eps;
};

// The rows that the table covers, clamped to those there are.  A table that decreases somewhere gives
// wrong sums but no access out of range.
__device__ __forceinline__ uint32_t table_at(const int32_t* offsets, int b, uint32_t n1, uint32_t low, uint32_t rows) {
  const int64_t x = static_cast<int64_t>(offsets[b]) * n1;
  return x < low ? low : x > rows ? rows : static_cast<uint32_t>(x);
}
struct Span {
  uint32_t first, total;  // rows [first, first + total)
  uint32_t blocks;        // blocks that take part
  uint32_t each, more;    // rows of a block, and how many of the first blocks have one more
  __device__ uint32_t start(uint32_t c) const { return first + c * each + min(c, more); }
  // the block that holds row `first + y`
  __device__ uint32_t block_of(uint32_t y) const {
    const uint32_t big = more * (each + 1);
    return y < big ? y / (each + 1) : more + (y - big) / each;
  }
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, int n_samples, uint32_t n1, uint32_t rows, uint32_t blocks) {
  Span s;
  s.first = offsets ? table_at(offsets, 0, n1, 0, rows) : 0;
  s.total = (offsets ? table_at(offsets, n_samples, n1, s.first, rows) : rows) - s.first;
  s.blocks = min(blocks, s.total);
  s.each = s.blocks ? s.total / s.blocks : 0;
  s.more = s.total - s.each * s.blocks;
  return s;
}

// values that a thread keeps of one row: 16
template <int VEC>
__host__ __device__ constexpr int grad_pieces() {
  return VEC == 8 ? 2 : 4;
}

// Blocks of 256 threads on an SM: three of 80 registers; two of up to 128 where a block's threads have sixteen single
// values (a register each) instead of vectors.  With eight values a thread (`half`) four.
__host__ __device__ constexpr int grad_blocks_per_sm(bool block, int vec, bool half) {
  return block && half ? 4 : !block || vec > 1 ? 3 : 2;
}

// BLOCK: a row by blockDim.x / 32 warps, blockDim.y rows at once, the weight as floats in dynamic shared memory (its 16
// registers are the difference between three blocks on an SM and spills).  Otherwise a row by L lanes, NR rows
// of a group of lanes at once, the weight in registers.
template <int GT, int ST, bool ADD, int VEC, int L, int NI, int NR, bool BLOCK, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? grad_blocks_per_sm(BLOCK, VEC, NI < grad_pieces<VEC>()) : 1)
    rms_norm_grad_kernel(const NormGradParams p) {
  constexpr int E = lane_values<VEC>();
  constexpr int kGroups = 32 / L;
  constexpr bool JOIN = THREADS == 256;  // several groups of threads hold rows: their sums are added
  __shared__ float part[2][BLOCK ? 64 : 1];
  __shared__ float part_again[2][BLOCK ? 64 : 1];
  __shared__ float joined[JOIN ? 8 * 32 * NI * E : 1];
  extern __shared__ __align__(16) float weight_smem[];

  const int lane = threadIdx.x & 31, l = lane % L;
  const int warps = BLOCK ? static_cast<int>(blockDim.x) >> 5 : 1;
  const int warp = BLOCK ? static_cast<int>(threadIdx.x) >> 5 : 0;
  const int mine = BLOCK ? static_cast<int>(threadIdx.y) * warps : 0;
  const int apart = static_cast<int>(blockDim.y) * (BLOCK ? 1 : kGroups);  // rows between two of a thread's
  const int together = apart * NR;                                         // rows at once
  const int place = BLOCK ? static_cast<int>(threadIdx.y) : static_cast<int>(threadIdx.y) * kGroups + lane / L;
  const int cols = warps * (NI * L * E);
  grid_dependency_wait();

  const Span span = span_of(p.offsets, p.n_samples, p.n1.d, p.rows, gridDim.x);
  const uint32_t c = blockIdx.x;
  if (c >= span.blocks) return;
  uint32_t row0 = span.start(c);
  const uint32_t end = span.start(c + 1);
  int b = 0;
  if (p.offsets) {  // the last sample that begins at or before the first row
    int low = 0, high = p.n_samples - 1;
    while (low < high) {
      const int mid = (low + high + 1) >> 1;
      if (table_at(p.offsets, mid, p.n1.d, 0, p.rows) <= row0) low = mid;
      else high = mid - 1;
    }
    b = low;
  }

  float w[BLOCK ? 1 : NI][E], acc[NI][E];
  // four values of a thread side by side, so that a warp reads 512 bytes in a row
  auto weight_at = [&](int i, int q) { return weight_smem + ((i * (E / 4) + q) * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 4; };
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    float* const wi = w[BLOCK ? 0 : i];
    with_type(p.w_dtype, [&](auto t) { load_weight_of<decltype(t)::value, VEC>(wi, p.w, (i * warps + warp) * (L * E), l, p.h); });
    if (BLOCK && threadIdx.y == 0)
#pragma unroll
      for (int q = 0; q < E / 4; ++q)
        *reinterpret_cast<float4*>(weight_at(i, q)) = make_float4(wi[4 * q], wi[4 * q + 1], wi[4 * q + 2], wi[4 * q + 3]);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[i][j] = 0.f;
  }
  if (BLOCK) __syncthreads();
  auto take_weight = [&](int i, float (&to)[E]) {
    if constexpr (BLOCK) {
#pragma unroll
      for (int q = 0; q < E / 4; ++q) {
        const float4 x = *reinterpret_cast<const float4*>(weight_at(i, q));
        to[4 * q] = x.x;
        to[4 * q + 1] = x.y;
        to[4 * q + 2] = x.z;
        to[4 * q + 3] = x.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) to[j] = w[i][j];
    }
  };

  int parity = 0;
  bool first_of_run = true;
  while (row0 < end) {
    uint32_t stop = end;
    if (p.offsets) {
      while (b + 1 < p.n_samples && table_at(p.offsets, b + 1, p.n1.d, 0, p.rows) <= row0) ++b;
      if (b + 1 < p.n_samples) {
        stop = min(table_at(p.offsets, b + 1, p.n1.d, 0, p.rows), end);
      }
    }
    for (uint32_t at = row0; at < stop; at += together) {  // below 2^31 + 2^8
      uint32_t ri[NR], rj[NR];
      bool live[NR];
      Piece<ST, VEC> s[NR][NI], add[ADD ? NR : 1][ADD ? NI : 1];
      Piece<GT, VEC> dy[NR][NI];
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        const uint32_t row = at + place + k * apart;
        live[k] = row < stop;
        split_row(row, p.n1, ri[k], rj[k]);
        const int h = live[k] ? p.h : 0;
        const unsigned char *ps = row_of<VEC>(p.s, ri[k], rj[k]), *pg = row_of<VEC>(p.dy, ri[k], rj[k]);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          s[k][i].load(ps, (i * warps + warp) * (L * E), l, h);
          dy[k][i].load(pg, (i * warps + warp) * (L * E), l, h);
        }
        if constexpr (ADD) {
          const unsigned char* pa = row_of<VEC>(p.add, ri[k], rj[k]);
#pragma unroll
          for (int i = 0; i < NI; ++i) add[k][i].load(pa, (i * warps + warp) * (L * E), l, h);
        }
      }

      // sum s^2 and sum g s over the row's lanes, of s times `by`
      auto sums_of = [&](const Piece<ST, VEC> (&s)[NI], const Piece<GT, VEC> (&dy)[NI], float by, float& to_ss, float& to_sg) {
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          float wi[E];
          take_weight(i, wi);
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float x = by == 1.f ? s[i].get(j) : s[i].get(j) * by;
            a = fmaf(x, x, a);
            b = fmaf(dy[i].get(j) * wi[j], x, b);
          }
        }
        to_ss = lanes_sum<L>(a);
        to_sg = lanes_sum<L>(b);
      };
      float ss[NR], sg[NR];
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        sums_of(s[k], dy[k], 1.f, ss[k], sg[k]);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          s[k][i].keep_packed();
          dy[k][i].keep_packed();
        }
      }
      bool again;
      if constexpr (BLOCK) {
        static_assert(NR == 1, "one row of a block's group at a time");
        if (lane == 0) {
          part[parity][mine + warp] = ss[0];
          part[parity][32 + mine + warp] = sg[0];
        }
        __syncthreads();
        const int all = warps * static_cast<int>(blockDim.y);
        again = __any_sync(0xffffffffu, lane < all && !(part[parity][lane < all ? lane : 0] <= kSquaresLimit));
        ss[0] = lanes_sum<32>(lane < warps ? part[parity][mine + lane] : 0.f);
        sg[0] = lanes_sum<32>(lane < warps ? part[parity][32 + mine + lane] : 0.f);
      } else {
        bool over = false;
#pragma unroll
        for (int k = 0; k < NR; ++k) over |= !(ss[k] <= kSquaresLimit);
        again = __any_sync(0xffffffffu, over);
      }
      float rstd[NR], scale[NR];
#pragma unroll
      for (int k = 0; k < NR; ++k) {
        rstd[k] = rsqrtf(fmaf(ss[k], p.inv_h, p.eps));
        scale[k] = 1.f;
      }
      if (again) {  // see kSquaresLimit
#pragma unroll
        for (int k = 0; k < NR; ++k) {
          if (!(ss[k] <= kSquaresLimit)) scale[k] = kDown;
          float ts, tg;
          sums_of(s[k], dy[k], scale[k], ts, tg);
          if constexpr (BLOCK) {
            if (lane == 0) {
              part_again[parity][mine + warp] = ts;
              part_again[parity][32 + mine + warp] = tg;
            }
            __syncthreads();
            ts = lanes_sum<32>(lane < warps ? part_again[parity][mine + lane] : 0.f);
            tg = lanes_sum<32>(lane < warps ? part_again[parity][32 + mine + lane] : 0.f);
          }
          if (scale[k] != 1.f) {
            rstd[k] = rsqrtf(fmaf(ts, p.inv_h, down_squared(p.eps)));
            sg[k] = tg;
          }
        }
      }
      parity ^= 1;

#pragma unroll
      for (int k = 0; k < NR; ++k) {
        const float unit = scale[k] * rstd[k];  // of the row as it is: down to 2^-128, where it still has 21 bits
        const float a = sg[k] * rstd[k] * p.inv_h;
        if (live[k]) {
          unsigned char* const px = row_of<VEC>(p.dx, ri[k], rj[k]);
          with_type(p.dx_dtype, [&](auto xt) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
              float v[E], wi[E];
              take_weight(i, wi);
#pragma unroll
              for (int j = 0; j < E; ++j) {
                const float g = dy[k][i].get(j), u = s[k][i].get(j) * unit;
                acc[i][j] = fmaf(g, u, acc[i][j]);
                const float x = fmaf(-u, a, g * wi[j]);
                if constexpr (ADD) v[j] = fmaf(unit, x, add[k][i].get(j));
                else v[j] = unit * x;
              }
              store_piece<decltype(xt)::value, VEC>(px, (i * warps + warp) * (L * E), l, p.h, v);
            }
          });
        }
      }
    }

    // the sums of this sample's rows in this block
    if (p.totals || p.pieces) {
      if constexpr (!BLOCK && kGroups > 1) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j)
#pragma unroll
            for (int d = L; d < 32; d <<= 1) acc[i][j] += __shfl_xor_sync(0xffffffffu, acc[i][j], d);
      }
      bool writer = BLOCK || lane < L;
      if (JOIN && blockDim.y > 1) {
        if (writer)
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j)
              joined[threadIdx.y * cols + col_of<VEC>((i * warps + warp) * (L * E), l, j)] = acc[i][j];
        __syncthreads();
        writer = writer && threadIdx.y == 0;
        if (writer)
          for (int y = 1; y < static_cast<int>(blockDim.y); ++y)
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
              for (int j = 0; j < E; ++j)
                acc[i][j] += joined[y * cols + col_of<VEC>((i * warps + warp) * (L * E), l, j)];
        __syncthreads();
      }
      if (writer) {
        if (p.pieces) {
          unsigned char* to = reinterpret_cast<unsigned char*>(p.pieces + static_cast<int64_t>(c + b) * p.pitch);
#pragma unroll
          for (int i = 0; i < NI; ++i)
            store_piece<ABS_F32, VEC>(to, (i * warps + warp) * (L * E), l, p.h, acc[i]);
        }
        if (p.totals) {
          unsigned char* to = reinterpret_cast<unsigned char*>(p.totals + c * p.pitch);
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const int first = (i * warps + warp) * (L * E);
            if (!first_of_run) {
              Piece<ABS_F32, VEC> old;
              old.load(to, first, l, p.h);
#pragma unroll
              for (int j = 0; j < E; ++j) acc[i][j] += old.get(j);
            }
            store_piece<ABS_F32, VEC>(to, first, l, p.h, acc[i]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) acc[i][j] = 0.f;
    }
    first_of_run = false;
    row0 = stop;
  }
}

// Adds the records, a block of 256 threads for 8 columns by 128 slices of the totals, 32 by 32 of a sample's pieces, or
// 128 by 8 where a sample has fewer than 128 blocks.  The first blocks take the pieces, those behind them the totals.
// A thread has four columns, so that eight blocks fit an SM: what a block does is a chain of latencies (table, records,
// slices), and the others' hide it.  1024 threads of one column: 11 us instead of 7 (2048 x 2048 with 8 samples); totals by
// 32 columns: 8.7 us instead of 6 without samples.
constexpr int kMergeThreads = 256, kTotalsBits = 3;
struct NormMergeParams {
  const float *totals, *pieces;
  int64_t pitch;
  const int32_t* offsets;
  float *dw, *dw_samples;  // may be NULL
  int64_t ld;
  uint32_t rows, n1;
  int n_samples, h, blocks;
  int n_out;               // samples that are written: n_samples or 0
  int col_bits;            // of the samples' blocks: 5 or 7
  int sample_blocks;       // of a sample
  float scale;             // of dw_samples
};

#ifndef ABS_INST_XT  // no template: compiled where it is launched
__global__ void __launch_bounds__(kMergeThreads) rms_norm_merge_kernel(const NormMergeParams p) {
  __shared__ float4 sums[kMergeThreads];
  const int of_samples = p.n_out * p.sample_blocks;
  const bool sample = static_cast<int>(blockIdx.x) < of_samples;
  const int bits = sample ? p.col_bits : kTotalsBits;
  const int b = sample ? static_cast<int>(blockIdx.x) / p.sample_blocks : p.n_out;
  const int first = (sample ? static_cast<int>(blockIdx.x) - b * p.sample_blocks : static_cast<int>(blockIdx.x) - of_samples) << bits;
  const int fours = 1 << (bits - 2);
  const int col = first + 4 * (threadIdx.x & (fours - 1)), slice = threadIdx.x >> (bits - 2), slices = kMergeThreads >> (bits - 2);
  grid_dependency_wait();
  const Span span = span_of(p.offsets, p.n_samples, p.n1, p.rows, p.blocks);
  const float* from = p.totals;
  int lo = 0, hi = static_cast<int>(span.blocks);  // records [lo, hi)
  if (sample) {
    const uint32_t a = table_at(p.offsets, b, p.n1, span.first, span.first + span.total) - span.first;
    const uint32_t e = table_at(p.offsets, b + 1, p.n1, span.first, span.first + span.total) - span.first;
    from = p.pieces;
    lo = hi = 0;
    if (e > a) {
      lo = static_cast<int>(span.block_of(a)) + b;
      hi = static_cast<int>(span.block_of(e - 1)) + b + 1;
    }
  }
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  auto plus = [&](const float4& y) { x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); };
  if (col < p.h)  // and so are the four within the pitch
#pragma unroll 8
    for (int k = lo + slice; k < hi; k += slices) plus(*reinterpret_cast<const float4*>(from + k * p.pitch + col));
  for (int d = fours; d < 32; d <<= 1)  // the slices of a warp
    plus(make_float4(__shfl_xor_sync(0xffffffffu, x.x, d), __shfl_xor_sync(0xffffffffu, x.y, d),
                     __shfl_xor_sync(0xffffffffu, x.z, d), __shfl_xor_sync(0xffffffffu, x.w, d)));
  sums[threadIdx.x] = x;
  __syncthreads();
  if (slice == 0 && col < p.h) {
#pragma unroll
    for (int k = 1; k < kMergeThreads / 32; ++k) plus(sums[32 * k + threadIdx.x]);
    const float by = sample ? p.scale : 1.f;
    float* const to = sample ? p.dw_samples + b * p.ld : p.dw;
    const float v[4] = {x.x * by, x.y * by, x.z * by, x.w * by};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (col + j < p.h) to[col + j] = v[j];
  }
}
#endif

}  // namespace absnt
