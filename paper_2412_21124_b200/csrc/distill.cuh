// Distillation from a teacher's top logits: the loss of every token and, in the same call, its gradient on
// the student's logits.  With z the student's logits of a row, tau the temperature, t the teacher's logits at the
// k indices it names, c = log2(e) / tau:
//
//   q_i = 2^((z_i - m) c) / S,  S = sum_i 2^((z_i - m) c)      the student's probabilities; m any reference
//   p_j = 2^((t_j - m') c) / S'                                 the teacher's, over its top or with its own log-sum-exp
//   p_r = max(0, 1 - sum p_j)  (0 without the log-sum-exp)      the teacher's mass outside of its top
//   loss = tau^2 (sum_j p_j ln(p_j / q_j) + p_r ln(p_r / q_r))  q_r = sum of q over what is not in the top
//   dz_i = w tau (q_i - p_i)   in the top,   w tau q_i (1 - p_r / q_r)   elsewhere
//
// The top is kept apart from the rest throughout: R = sum over the rest of e_i = 2^((z_i - m) c) is a sum of its
// own (S minus the top would lose it where the student is sure), and with it q_i (1 - p_r / q_r) is
// e_i (1 / S - p_r / R), which neither overflows nor cancels to nothing when q_r is tiny.
#pragma once
#include "rows.cuh"

namespace absnt {

struct DistillParams {
  RowsArg z, dz, t;        // dz.p may be NULL
  const unsigned char* ids;
  int64_t ids_stride;      // bytes
  const float *lse, *weights;    // may be NULL
  const int32_t* offsets;        // may be NULL
  float* losses;
  uint32_t rows;
  int n_samples;
  int vocab, top, t_dtype, id_bytes;
  int empty_polls;         // of the ring's feeder at a stage that has not been given back: kBulkWaitLimit but for its self-test
  double inv_tau;
  float c;                 // log2(e) / tau
  float tau;
  float loss_scale;        // tau^2 ln 2: of logarithms to base 2
  float grad_scale;        // tau grad_scale
};

constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A sum of 2^((z - m) c): the reference m is some z of the sum (or the lowest float) and S at most 2^60 times
// what it would be with the largest.
struct ExpSum {
  float m, s;
};
__device__ __forceinline__ ExpSum join(const ExpSum& a, const ExpSum& b, float c) {
  const float m = fmaxf(a.m, b.m);
  return {m, a.s * exp2_fast((a.m - m) * c) + b.s * exp2_fast((b.m - m) * c)};
}

// What a row is to the call: left alone (behind the last sample), counted with no weight, or worked on.
__device__ __forceinline__ bool row_has_sample(const DistillParams& p, uint32_t row) {
  return !p.offsets || (static_cast<int64_t>(row) >= p.offsets[0] && static_cast<int64_t>(row) < p.offsets[p.n_samples]);
}
__device__ __forceinline__ int load_id(const DistillParams& p, uint32_t row, int j) {  // -1: none
  const unsigned char* at = p.ids + static_cast<int64_t>(row) * p.ids_stride;
  const int64_t id = p.id_bytes == 8 ? reinterpret_cast<const int64_t*>(at)[j] : reinterpret_cast<const int32_t*>(at)[j];
  return id >= 0 && id < p.vocab ? static_cast<int>(id) : -1;
}
__device__ __forceinline__ float load_teacher(const DistillParams& p, uint32_t row, int j) {
  const unsigned char* at = row_of(p.t, row, 0);
  if (p.t_dtype == ABS_F32) return reinterpret_cast<const float*>(at)[j];
  const uint32_t w = reinterpret_cast<const unsigned short*>(at)[j];
  return p.t_dtype == ABS_BF16 ? from_half_word<ABS_BF16>(w) : from_half_word<ABS_F16>(w);
}
template <int DT>
__device__ __forceinline__ void store_one(unsigned char* row, int i, float v) {
  if constexpr (DT == ABS_F32) reinterpret_cast<float*>(row)[i] = v;
  else if constexpr (DT == ABS_BF16) reinterpret_cast<__nv_bfloat16*>(row)[i] = __float2bfloat16_rn(v);
  else reinterpret_cast<__half*>(row)[i] = __float2half_rn(v);
}

// log2 of exp(t / tau - lse): the two are often large and close, so their difference is taken in 64 bits
__device__ __forceinline__ float log_of_share(const DistillParams& p, float t, float lse) {
  return static_cast<float>(static_cast<double>(t) * p.inv_tau - static_cast<double>(lse)) * 1.44269504f;
}

// joins of a block of 16 warps, in a fixed order; `room` is not used again before the next barrier
constexpr int kDistillThreads = 512;
constexpr int kDistillWarps = kDistillThreads / 32;
__device__ __forceinline__ ExpSum block_join(ExpSum x, float c, ExpSum* room) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    x = join(x, {__shfl_xor_sync(0xffffffffu, x.m, d), __shfl_xor_sync(0xffffffffu, x.s, d)}, c);
  const int lane = threadIdx.x & 31;
  if (lane == 0) room[threadIdx.x >> 5] = x;
  __syncthreads();
  x = lane < kDistillWarps ? room[lane] : ExpSum{kLowest, 0.f};
#pragma unroll
  for (int d = 16; d > 0; d >>= 1)
    x = join(x, {__shfl_xor_sync(0xffffffffu, x.m, d), __shfl_xor_sync(0xffffffffu, x.s, d)}, c);
  return x;
}
__device__ __forceinline__ float block_sum(float x, float* room) {
  x = lanes_sum<32>(x);
  const int lane = threadIdx.x & 31;
  if (lane == 0) room[threadIdx.x >> 5] = x;
  __syncthreads();
  return lanes_sum<32>(lane < kDistillWarps ? room[lane] : 0.f);
}

// Any vocabulary, any alignment: a block a row, which is read twice (the second time mostly from L2).  The top's
// places are bits in shared memory.  For rows that do not fit a cluster's shared memory, and gradients at another
// distance from 16-byte boundaries than the logits: where both kernels may be taken it needs 464 us against 220 (4096
// rows of 50257, bf16, gradient) and 316 against 127 (8192 rows of 32000, f16, loss alone).
template <int DT, int VEC>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams p) {
  constexpr int E = lane_values<VEC>();
  extern __shared__ uint32_t in_top[];  // a bit for each index
  __shared__ ExpSum room_t[kDistillWarps], room_top[kDistillWarps], room_rest[kDistillWarps];
  __shared__ float room_p[kDistillWarps], room_l[kDistillWarps];
  __shared__ int sh_id[kDistillThreads];
  __shared__ float sh_p[kDistillThreads];

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t row = blockIdx.x;
  grid_dependency_wait();
  if (!row_has_sample(p, row)) return;
  const float weight = p.weights ? p.weights[row] : 1.f;
  const unsigned char* z = row_of(p.z, row, 0);
  unsigned char* dz = p.dz.p ? row_of(p.dz, row, 0) : nullptr;
  if (weight == 0.f) {
    if (tid == 0) p.losses[row] = 0.f;
    if (dz) {
      const float none[E] = {};
      for (int first = warp * 32 * E; first < p.vocab; first += kDistillWarps * 32 * E)
        store_piece<DT, VEC>(dz, first, lane, p.vocab, none);
    }
    return;
  }

  // the teacher's entries, one a thread
  const int id = tid < p.top ? load_id(p, row, tid) : -1;
  const float t = id >= 0 ? load_teacher(p, row, tid) : -INFINITY;
  const float zt = id >= 0 ? load_value<DT>(z, id) : -INFINITY;
  for (int i = tid; i < (p.vocab + 31) / 32; i += kDistillThreads) in_top[i] = 0u;
  sh_id[tid] = id;
  const ExpSum own{fmaxf(t, kLowest), 0.f};  // a NaN stays in the sum, not in the reference
  const ExpSum st = block_join({own.m, id >= 0 ? exp2_fast((t - own.m) * p.c) : 0.f}, p.c, room_t);  // a barrier is passed
  bool again = false;
  if (id >= 0) again = atomicOr(&in_top[id >> 5], 1u << (id & 31)) & (1u << (id & 31));
  // in units of log2; an entry that has no probability takes no part
  const float log_p = p.lse ? log_of_share(p, t, p.lse[row]) : (t - st.m) * p.c - log2f(st.s);
  const bool some = id >= 0 && t != -INFINITY;
  const float pj = some ? exp2_fast(log_p) : 0.f;
  sh_p[tid] = pj;
  const bool repeated = __syncthreads_or(again);
  bool first = id >= 0;  // the first entry with its index stands for all of them
  float p_all = pj;
  if (repeated) {
    for (int j = 0; j < p.top; ++j)
      if (sh_id[j] == id && j != tid) {
        if (j < tid) first = false;
        p_all += sh_p[j];
      }
  }

  // the rest: chunks of E values against a reference that is moved when a chunk's largest is 2^60 above it
  ExpSum rest{kLowest, 0.f};
  const float limit = 60.f / p.c;
  for (int first_col = warp * 32 * E; first_col < p.vocab; first_col += kDistillWarps * 32 * E) {
    Piece<DT, VEC> x;
    x.load(z, first_col, lane, p.vocab);
    float v[E], top = kLowest;
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const int i = col_of<VEC>(first_col, lane, j);
      const bool out = i >= p.vocab || (in_top[i >> 5] >> (i & 31) & 1u);
      v[j] = out ? -INFINITY : x.get(j);
      top = fmaxf(top, v[j]);
    }
    if (top - rest.m > limit) {
      rest.s *= exp2_fast((rest.m - top) * p.c);
      rest.m = top;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) rest.s += exp2_fast((v[j] - rest.m) * p.c);
  }
  rest = block_join(rest, p.c, room_rest);
  const float mt = fmaxf(zt, kLowest);
  const ExpSum top = block_join({mt, first ? exp2_fast((zt - mt) * p.c) : 0.f}, p.c, room_top);
  const ExpSum all = join(rest, top, p.c);

  const float sum_p = block_sum(pj, room_p);
  float p_rest = p.lse ? fmaxf(1.f - sum_p, 0.f) : 0.f;
  if (p.lse && sum_p != sum_p) p_rest = sum_p;  // NaN
  if (rest.s == 0.f) p_rest = 0.f;              // nothing can be given to what is not in the top
  const float log_s = log2f(all.s);
  // p tau^2 ln(p / q), the distance of z from the reference without the factor c and times p first: a masking value might not
  // bear c or tau alone
  const float mine = some && pj != 0.f ? pj * p.loss_scale * (log_p + log_s) + pj * p.tau * (all.m - zt) : 0.f;
  float loss = block_sum(mine, room_l);
  if (tid == 0) {
    if (p_rest != 0.f)
      loss += p_rest * p.loss_scale * (log2f(p_rest) - log2f(rest.s) + log_s) + p_rest * p.tau * (all.m - rest.m);
    p.losses[row] = loss;
  }
  if (!dz) return;

  const bool any = p.lse || st.s != 0.f;  // a teacher that names nothing asks for nothing
  const float g = any ? weight * p.grad_scale : 0.f;
  const float factor = g * (exp2_fast((rest.m - all.m) * p.c) / all.s - (p_rest != 0.f ? p_rest / rest.s : 0.f));
  for (int first_col = warp * 32 * E; first_col < p.vocab; first_col += kDistillWarps * 32 * E) {
    Piece<DT, VEC> x;
    x.load(z, first_col, lane, p.vocab);
    float v[E];
#pragma unroll
    for (int j = 0; j < E; ++j) v[j] = factor * exp2_fast((x.get(j) - rest.m) * p.c);
    store_piece<DT, VEC>(dz, first_col, lane, p.vocab, v);
  }
  __syncthreads();
  if (first) store_one<DT>(dz, id, g * (exp2_fast((zt - all.m) * p.c) / all.s - p_all));
}

// sample_losses[b] = sum over the rows of sample b of weight * loss, in fp64: a block a sample
struct SampleLossParams {
  const float *losses, *weights;  // weights may be NULL
  const int32_t* offsets;         // NULL: one sample of all rows
  float* out;
  uint32_t rows;
};
#ifndef ABS_INST_XT  // no template: compiled where it is launched
constexpr int kSampleLossThreads = 512;
__global__ void __launch_bounds__(kSampleLossThreads) distill_samples_kernel(const SampleLossParams p) {
  __shared__ double room[kSampleLossThreads / 32];
  const int lane = threadIdx.x & 31;
  grid_dependency_wait();
  int64_t a = 0, e = p.rows;
  if (p.offsets) {
    a = max(0, p.offsets[blockIdx.x]);
    e = min(e, static_cast<int64_t>(p.offsets[blockIdx.x + 1]));
  }
  double x = 0.0;
#pragma unroll 4
  for (int64_t i = a + threadIdx.x; i < e; i += kSampleLossThreads) {
    const float w = p.weights ? p.weights[i] : 1.f;
    x += static_cast<double>(w) * p.losses[i];
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  if (lane == 0) room[threadIdx.x >> 5] = x;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kSampleLossThreads / 32; ++k) x += room[k];
    p.out[blockIdx.x] = static_cast<float>(x);
  }
}
#endif

}  // namespace absnt
