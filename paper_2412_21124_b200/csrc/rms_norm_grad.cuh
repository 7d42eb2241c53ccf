// Backward pass of the root-mean-square norm, with the weight's gradient of every sample of a packed batch:
//
//   rstd = (sum_c s_c^2 / h + eps)^(-1/2),  u_c = s_c rstd,  g_c = dy_c w_c,  a = sum_c g_c u_c / h
//   dx_c = rstd (g_c - u_c a) + dresidual_c
//   dw_c of sample b = sum over the rows of b of dy_c u_c
//
// rstd is formed again from s, which the pass reads anyway: one sum more in a row's reduction instead of a
// saved vector that has to fit its rows.
//
// Every block takes an equal run of consecutive rows, so that the sums over rows stay in registers while it
// walks them; it writes them once for each sample that it meets (a piece) and once for the whole run (a
// total).  A second kernel adds the pieces of each sample and the totals, in order: results do not depend
// on scheduling and no atomics are needed.  Piece (block c, sample b) lies at c + b: along the rows one of
// the two grows at every step, so that no two pieces share a place and a table is not needed.
#pragma once
#include "rms_norm.cuh"

namespace absnt {

struct NormGradParams {
  RowsArg dy, s, add, dx;          // add.p may be NULL
  const unsigned char* w;          // may be NULL
  const int32_t* offsets;          // NULL: all rows, one sample
  float *totals, *pieces;          // may be NULL
  int64_t pitch;                   // floats between two records
  uint32_t rows, n1;
  int n_samples;
  int h, w_dtype, dx_dtype;
  float inv_h, eps;
};

// The rows that the table covers, clamped to those there are.  A table that decreases somewhere gives
// wrong sums but no access out of range.
__device__ __forceinline__ int64_t table_at(const int32_t* offsets, int b, uint32_t n1, int64_t low, int64_t rows) {
  const int64_t x = static_cast<int64_t>(offsets[b]) * n1;
  return x < low ? low : x > rows ? rows : x;
}
struct Span {
  int64_t first, total;  // rows [first, first + total)
  int64_t blocks;        // blocks that take part
  __device__ int64_t start(int64_t c) const { return first + c * total / blocks; }
  // the block that holds row `first + y`
  __device__ int64_t block_of(int64_t y) const { return ((y + 1) * blocks - 1) / total; }
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, int n_samples, uint32_t n1, uint32_t rows, int64_t blocks) {
  Span s;
  s.first = offsets ? table_at(offsets, 0, n1, 0, rows) : 0;
  s.total = (offsets ? table_at(offsets, n_samples, n1, s.first, rows) : rows) - s.first;
  s.blocks = blocks < s.total ? blocks : s.total;
  return s;
}

// values that a thread keeps of one row: 16
template <int VEC>
__host__ __device__ constexpr int grad_pieces() {
  return VEC == 8 ? 2 : 4;
}

template <int GT, int ST, int VEC, int L, int NI, bool BLOCK, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 1) rms_norm_grad_kernel(const NormGradParams p) {
  constexpr int E = lane_values<VEC>();
  constexpr int kGroups = 32 / L;
  constexpr bool JOIN = THREADS == 256;  // several groups of threads hold rows: their sums are added
  __shared__ float part[2][BLOCK ? 64 : 1];
  __shared__ float part_again[2][BLOCK ? 64 : 1];
  __shared__ float joined[JOIN ? 8 * 32 * NI * E : 1];

  const int lane = threadIdx.x & 31, l = lane % L;
  const int warps = BLOCK ? static_cast<int>(blockDim.x) >> 5 : 1;
  const int warp = BLOCK ? static_cast<int>(threadIdx.x) >> 5 : 0;
  const int mine = BLOCK ? static_cast<int>(threadIdx.y) * warps : 0;
  const int together = static_cast<int>(blockDim.y) * (BLOCK ? 1 : kGroups);  // rows at once
  const int place = BLOCK ? static_cast<int>(threadIdx.y) : static_cast<int>(threadIdx.y) * kGroups + lane / L;
  const int cols = warps * (NI * L * E);
  grid_dependency_wait();

  const Span span = span_of(p.offsets, p.n_samples, p.n1, p.rows, gridDim.x);
  const int64_t c = blockIdx.x;
  if (c >= span.blocks) return;
  int64_t row0 = span.start(c);
  const int64_t end = span.start(c + 1);
  int b = 0;
  if (p.offsets) {  // the last sample that begins at or before the first row
    int low = 0, high = p.n_samples - 1;
    while (low < high) {
      const int mid = (low + high + 1) >> 1;
      if (table_at(p.offsets, mid, p.n1, 0, p.rows) <= row0) low = mid;
      else high = mid - 1;
    }
    b = low;
  }

  float w[NI][E], acc[NI][E];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    load_weight<VEC>(w[i], p.w, p.w_dtype, (i * warps + warp) * (L * E), l, p.h);
#pragma unroll
    for (int j = 0; j < E; ++j) acc[i][j] = 0.f;
  }

  int parity = 0;
  bool first_of_run = true;
  while (row0 < end) {
    int64_t stop = end;
    if (p.offsets) {
      while (b + 1 < p.n_samples && table_at(p.offsets, b + 1, p.n1, 0, p.rows) <= row0) ++b;
      if (b + 1 < p.n_samples) {
        const int64_t next = table_at(p.offsets, b + 1, p.n1, 0, p.rows);
        stop = next < end ? next : end;
      }
    }
    for (int64_t at = row0; at < stop; at += together) {
      const uint32_t row = static_cast<uint32_t>(at) + place;
      const bool live = row < stop;
      const int h = live ? p.h : 0;
      const uint32_t ri = p.n1 == 1 ? row : row / p.n1;
      const uint32_t rj = p.n1 == 1 ? 0 : row - ri * p.n1;
      Piece<ST, VEC> s[NI], add[NI];
      Piece<GT, VEC> dy[NI];
      const unsigned char *ps = row_of(p.s, ri, rj), *pg = row_of(p.dy, ri, rj);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        s[i].load(ps, (i * warps + warp) * (L * E), l, h);
        dy[i].load(pg, (i * warps + warp) * (L * E), l, h);
      }
      if (p.add.p) {
        const unsigned char* pa = row_of(p.add, ri, rj);
#pragma unroll
        for (int i = 0; i < NI; ++i) add[i].load(pa, (i * warps + warp) * (L * E), l, h);
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) add[i].zero();
      }

      float ss = 0.f, sg = 0.f;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < E; ++j) {
          const float x = s[i].get(j);
          ss = fmaf(x, x, ss);
          sg = fmaf(dy[i].get(j) * w[i][j], x, sg);
        }
      ss = lanes_sum<L>(ss);
      sg = lanes_sum<L>(sg);
      bool again;
      if constexpr (BLOCK) {
        if (lane == 0) {
          part[parity][mine + warp] = ss;
          part[parity][32 + mine + warp] = sg;
        }
        __syncthreads();
        const int all = warps * static_cast<int>(blockDim.y);
        again = __any_sync(0xffffffffu, lane < all && !(part[parity][lane < all ? lane : 0] <= kSquaresLimit));
        ss = lanes_sum<32>(lane < warps ? part[parity][mine + lane] : 0.f);
        sg = lanes_sum<32>(lane < warps ? part[parity][32 + mine + lane] : 0.f);
      } else {
        again = __any_sync(0xffffffffu, !(ss <= kSquaresLimit));
      }
      float rstd = rsqrtf(fmaf(ss, p.inv_h, p.eps)), scale = 1.f;
      if (again) {  // see kSquaresLimit
        if (!(ss <= kSquaresLimit)) scale = kDown;
        float ts = 0.f, tg = 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float x = s[i].get(j) * scale;
            ts = fmaf(x, x, ts);
            tg = fmaf(dy[i].get(j) * w[i][j], x, tg);
          }
        ts = lanes_sum<L>(ts);
        tg = lanes_sum<L>(tg);
        if constexpr (BLOCK) {
          if (lane == 0) {
            part_again[parity][mine + warp] = ts;
            part_again[parity][32 + mine + warp] = tg;
          }
          __syncthreads();
          ts = lanes_sum<32>(lane < warps ? part_again[parity][mine + lane] : 0.f);
          tg = lanes_sum<32>(lane < warps ? part_again[parity][32 + mine + lane] : 0.f);
        }
        if (scale != 1.f) {
          rstd = rsqrtf(ts * p.inv_h);
          sg = tg;
        }
      }
      parity ^= 1;

      const float unit = scale * rstd;            // u = s scale rstd: one product where nothing was scaled
      const float a = sg * rstd * p.inv_h;
      if (live) {
        unsigned char* px = row_of(p.dx, ri, rj);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          float v[E];
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float g = dy[i].get(j);
            const float u = scale == 1.f ? s[i].get(j) * rstd : s[i].get(j) * scale * rstd;
            acc[i][j] = fmaf(g, u, acc[i][j]);
            v[j] = fmaf(unit, fmaf(-u, a, g * w[i][j]), add[i].get(j));
          }
          store_piece_as<VEC>(p.dx_dtype, px, (i * warps + warp) * (L * E), l, p.h, v);
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
          unsigned char* to = reinterpret_cast<unsigned char*>(p.pieces + (c + b) * p.pitch);
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

// Adds the records: blocks of 32 columns x kMergeSlices.  Block row b < n_out: the pieces of sample b, behind
// them the totals.
constexpr int kMergeSlices = 16;
struct NormMergeParams {
  const float *totals, *pieces;
  int64_t pitch;
  const int32_t* offsets;
  float *dw, *dw_samples;  // may be NULL
  int64_t ld;
  uint32_t rows, n1;
  int n_samples, h, blocks, col_blocks;
  int n_out;               // samples that are written: n_samples or 0
  float scale;             // of dw_samples
};

#ifndef ABS_INST_XT  // no template: compiled where it is launched
__global__ void __launch_bounds__(32 * kMergeSlices) rms_norm_merge_kernel(const NormMergeParams p) {
  __shared__ float sums[kMergeSlices][32];
  const int b = blockIdx.x / p.col_blocks;
  const int col = (blockIdx.x - b * p.col_blocks) * 32 + threadIdx.x;
  grid_dependency_wait();
  const Span span = span_of(p.offsets, p.n_samples, p.n1, p.rows, p.blocks);
  const float* from = p.totals;
  int64_t lo = 0, hi = span.blocks;  // records [lo, hi)
  if (b < p.n_out) {
    const int64_t a = table_at(p.offsets, b, p.n1, span.first, span.first + span.total) - span.first;
    const int64_t e = table_at(p.offsets, b + 1, p.n1, span.first, span.first + span.total) - span.first;
    from = p.pieces;
    lo = hi = 0;
    if (e > a) {
      lo = span.block_of(a) + b;
      hi = span.block_of(e - 1) + b + 1;
    }
  }
  float x = 0.f;
  if (col < p.h)
#pragma unroll 4
    for (int64_t k = lo + threadIdx.y; k < hi; k += kMergeSlices) x += from[k * p.pitch + col];
  sums[threadIdx.y][threadIdx.x] = x;
  __syncthreads();
  if (threadIdx.y == 0 && col < p.h) {
    x = 0.f;
#pragma unroll
    for (int k = 0; k < kMergeSlices; ++k) x += sums[k][threadIdx.x];
    if (b < p.n_out) p.dw_samples[b * p.ld + col] = x * p.scale;
    else p.dw[col] = x;
  }
}
#endif

}  // namespace absnt
