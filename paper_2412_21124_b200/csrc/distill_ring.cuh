// The distillation kernel of vocabularies whose rows fit the shared memory of a cluster: logits are read from
// HBM once, gradient and loss come from what is on the chip.
//
// A row is cut into 16-byte units from the boundary before its first value, and the units go in equal runs to the
// blocks of a cluster of 1 to 8.  The warps of a block have four parts:
//   feeder   runs ahead: brings the block's run of the next rows into a ring of stages by bulk copies; meanwhile
//            finds out where the top's entries lie in it and works out the teacher's probabilities
//   workers  pass 1 of a row: take the top's logits out of the stage (-inf stays in their place), sum 2^((z - m) c)
//            over the rest.  Pass 2, of the row before: the same exponentials once more times one factor are the
//            gradient, written 16 bytes at a time; the top's places follow behind the next barrier
//   topper   sums over the top's entries while the workers are at pass 1
//   joiner   joins the warps' sums, exchanges them with the other blocks by asynchronous stores into their shared
//            memory, and gives the workers the factor
// so that neither the loads nor the joins keep a worker waiting.  A special warp gets an eighth of its
// scheduler's slots beside the workers: what it does in a row decides the rate, hence three of them.  Earlier
// forms, rows of 128256: workers that joined among themselves and kept the exponentials in registers meanwhile spent
// 13,000 cycles on a row of which 4,600 were passes; one warp for teacher, top and joins 9,400.
// Rows need not begin on 16-byte boundaries: gradient and logits must only lie at the same distance from one.
//
// Bounds: HBM, 2 bytes a value read and 2 written (16 bits), where the exponentials, 16 a clock and SM, take 0.73 of the
// time, with and without the gradient; what is reached is 0.6 to 0.7 of the bandwidth, and the same without the loads or
// without the stores: issue slots are half taken, the exponential unit a little less, and the rest is the chain of a
// row (largest, sum, join, answer) that two rows under way do not cover.  bf16 with the gradient: 8192 rows of 128256,
// a fifth of them without weight, 842 us, 4096 of 50257 220 us; f16, loss alone: 8192 of 32000 127 us.
//
// Every wait is bounded (see normtest_bulk.cuh).  A part whose wait runs out says nothing further to any mbarrier: a phase that
// is still open must not be entered twice.  A feeder or a joiner stops there, so that the waits of those that it
// would have served run out as well; workers go on without waiting and make NaN of what they sum.  So the row whose
// data did not come, and the rows behind it in the cluster, are NaN.
#pragma once
#include "distill.cuh"
#include "normtest_bulk.cuh"

#include <type_traits>

namespace absnt {

constexpr int kRingMaxCluster = 8;
constexpr int kRingMaxStages = 4;

struct RingParams {
  DistillParams d;
  int blocks;        // of a cluster
  int units;         // of a block
  int stages;        // at least 2: pass 2 of a row comes after pass 1 of the next
  int stage_bytes;   // units and 16 bytes an entry of the top, a multiple of 16
  const unsigned char *z_begin, *z_end;  // the logits' first byte and the one behind their last
};

enum { kRowAlone = 0, kRowNoWeight = 1, kRowWork = 2 };

// what a block knows of a row after pass 1: the rest's sum, the top's, and of the block's entries of the top the sum
// of p (tau^2 ln p - tau (z - m)) with m the top's reference, and the sum of p.  Distances of logits are multiplied by a
// probability first: times tau alone that of a masking value may not be a float
struct RingSums {
  ExpSum rest, top;
  float cross, p;
  float unused[2];
};
// what the workers need of a row for pass 2
struct RingAnswer {
  float factor, m;        // of the rest: factor * 2^((z - m) c)
  float g, m_all, over_s; // of the top: g (2^((z - m_all) c) over_s - p)
};
// the top's entries of a row in its stage: place in the block's run (-1: elsewhere), logit, log2 p, p.  When the
// topper is done log_p holds p summed over the entries of the same index
struct RingTop {
  int* place;
  float *z, *log_p, *p;
};

// the largest of a warp's values, by their bits: as signed integers they are ordered like the floats once those of
// negative ones are turned round.  No value is a NaN.
__device__ __forceinline__ float warp_max(float x) {
  int b = __float_as_int(x);
  b ^= (b >> 31) & 0x7fffffff;
  b = __reduce_max_sync(0xffffffffu, b);
  return __int_as_float(b ^ ((b >> 31) & 0x7fffffff));
}
// joins over the warp's lanes
__device__ __forceinline__ ExpSum warp_join(ExpSum x, float c) {
  const float m = warp_max(x.m);
  return {m, lanes_sum<32>(x.s * exp2_fast((x.m - m) * c))};
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 32 bytes into the same place of another block's shared memory, counted on the barrier there
__device__ __forceinline__ void send_sums(const RingSums& x, RingSums* to, uint64_t* bar, uint32_t rank) {
  uint32_t a, b;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(to)), "r"(rank));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_addr(bar)), "r"(rank));
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1,%2,%3,%4}, [%5];" ::"r"(a),
               "f"(x.rest.m), "f"(x.rest.s), "f"(x.top.m), "f"(x.top.s), "r"(b)
               : "memory");
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1,%2,%3,%4}, [%5];" ::"r"(a + 16),
               "f"(x.cross), "f"(x.p), "f"(0.f), "f"(0.f), "r"(b)
               : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// Barriers between the parts of a block.  A warp that waits at one takes no issue slots, one that polls an mbarrier
// does (a failed look comes back after some thirty cycles); and as every warp comes to each of them
// whatever has become of the mbarriers, none of them waits for good.
template <int N>
__device__ __forceinline__ void workers_barrier() {
  asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory");
}
enum { kTopTaken = 2, kSummed = 4, kAnswered = 6 };  // and one more each: of rows by turns
template <int N>
__device__ __forceinline__ void part_sync(int id) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void part_arrive(int id) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(N) : "memory");
}

template <int DT>
__host__ __device__ constexpr int unit_values() {
  return 16 / elem_bytes<DT>();
}
template <int DT>
__device__ __forceinline__ float value_of(const uint32_t (&w)[4], int j) {
  if constexpr (DT == ABS_F32) return __uint_as_float(w[j]);
  if constexpr (DT == ABS_BF16) return __uint_as_float((j & 1) ? (w[j >> 1] & 0xffff0000u) : (w[j >> 1] << 16));
  return from_half_word<DT>((j & 1) ? (w[j >> 1] >> 16) : (w[j >> 1] & 0xffffu));
}

// 2^((z - m) c) as 2^(z c - r) with r the rounded m c: one fma and one exponential.  What the rounding of r costs is
// the same factor for all values, 2^(m c - r), and is taken back once, in `correction`.  From |m c| = 2^24 on (a masking
// value, say) the exponent m c - r could exceed 1/2, and where |m c| is larger still the range of a float: there the
// difference z - m is formed first, exactly where it counts.  An infinite m and a NaN among the values give NaN.
struct Exponentials {
  float m, c, minus_r, correction;
  bool far;
  __device__ __forceinline__ Exponentials(float m_, float c_) : m(m_), c(c_) {
    minus_r = -(m * c);
    far = !(fabsf(minus_r) < 0x1p24f);
    correction = far ? 1.f : exp2_fast(-fmaf(m, c, minus_r));
  }
  __device__ __forceinline__ uint64_t operator()(float a, float b) const {
    const float2 x = pair_as(pair_fma(pair_of(a, b), pair_of(c, c), pair_of(minus_r, minus_r)));
    return pair_of(exp2_fast(x.x), exp2_fast(x.y));
  }
  __device__ __forceinline__ uint64_t of_far(float a, float b) const {
    const float2 x = pair_as(pair_mul(pair_add(pair_of(a, b), pair_of(-m, -m)), pair_of(c, c)));
    return pair_of(exp2_fast(x.x), exp2_fast(x.y));
  }
};
// the larger of two words of values, place by place
template <int DT>
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (DT == ABS_F32) r = __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  else if constexpr (DT == ABS_BF16) asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int DT>
__device__ __forceinline__ float max_of_word(uint32_t w) {
  if constexpr (DT == ABS_F32) return __uint_as_float(w);
  return fmaxf(from_half_word<DT>(w & 0xffffu), from_half_word<DT>(w >> 16));
}

// A unit of a row's gradient; i0: the index of its first value.  The first and last of a row may reach out of it.
template <int DT>
__device__ __forceinline__ void write_unit(unsigned char* to, int i0, int vocab, const uint32_t (&out)[4]) {
  constexpr int U = unit_values<DT>();
  if (i0 >= 0 && i0 + U <= vocab) {
    *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
    return;
  }
#pragma unroll
  for (int j = 0; j < U; ++j)
    if (i0 + j >= 0 && i0 + j < vocab) {
      if constexpr (DT == ABS_F32) reinterpret_cast<uint32_t*>(to)[j] = out[j];
      else reinterpret_cast<unsigned short*>(to)[j] = static_cast<unsigned short>(out[j >> 1] >> (16 * (j & 1)));
    }
}

// Units `from` to `end` of a stage, 32 at a time by a warp: from + 32 warp, then STEP further.  f gets a lane's unit, its
// words and whether there is one; which of the loop's branches are taken is the same for all lanes.
template <int STEP, typename F>
__device__ __forceinline__ void for_units(int from, int end, const unsigned char* stage, uint32_t none, F f) {
  const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0), lane = threadIdx.x & 31;
  auto words = [&](int u, uint32_t (&w)[4]) {
    const uint4 v = *reinterpret_cast<const uint4*>(stage + u * 16);
    w[0] = v.x;
    w[1] = v.y;
    w[2] = v.z;
    w[3] = v.w;
  };
  int first = from + 32 * warp;
  for (; first + STEP + 32 <= end; first += 2 * STEP) {
    uint32_t a[4], b[4];
    words(first + lane, a);
    words(first + STEP + lane, b);
    f(first + lane, a, true);
    f(first + STEP + lane, b, true);
  }
#pragma unroll 1
  for (; first < end; first += STEP) {
    const bool mine = first + lane < end;
    uint32_t a[4] = {none, none, none, none};
    if (mine) words(first + lane, a);
    f(first + lane, a, mine);
  }
}

constexpr int ring_blocks_per_sm(int threads) { return 512 / threads; }

// THREADS workers and three special warps
template <int DT, int THREADS, bool GRAD>
__global__ void __launch_bounds__(THREADS + 96, ring_blocks_per_sm(THREADS))
    distill_ring_kernel(const __grid_constant__ RingParams r) {
  constexpr int U = unit_values<DT>();
  constexpr int ESZ = elem_bytes<DT>();
  constexpr int kWarps = THREADS / 32;
  const DistillParams& p = r.d;
  extern __shared__ __align__(16) unsigned char ring[];  // the stages, then a bit for each place of the block's run
  __shared__ __align__(8) uint64_t full[kRingMaxStages], empty[kRingMaxStages];
  __shared__ __align__(8) uint64_t sums_here[2];
  __shared__ int repeated_in[kRingMaxStages];  // an index of this block's run is named twice
  __shared__ int any_in[kRingMaxStages];       // the teacher names something
  __shared__ __align__(16) ExpSum from_warps[2][kWarps];
  __shared__ __align__(16) RingSums from_top[2], from_blocks[2][kRingMaxCluster];
  __shared__ RingAnswer answers[2];

  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int rank = r.blocks > 1 ? static_cast<int>(cluster_rank()) : 0;
  const uint32_t cluster = blockIdx.x / r.blocks, clusters = gridDim.x / r.blocks;
  uint32_t* const marks = reinterpret_cast<uint32_t*>(ring + r.stages * r.stage_bytes);
  const int first_unit = rank * r.units;
  bool dead = false;  // a wait of this thread ran out: it waits no more, and what it computes is NaN
  const float nan = __uint_as_float(0x7fffffffu);

  if (tid == 0) {
    for (int s = 0; s < r.stages; ++s) {
      mbar_init(&full[s], 2);        // the copy has been asked for; the top's entries are there
      mbar_init(&empty[s], kWarps);
    }
    mbar_init(&sums_here[0], 1);
    mbar_init(&sums_here[1], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < (r.units * U + 31) / 32; i += THREADS + 96) marks[i] = 0u;
  __syncthreads();
  if (r.blocks > 1) cluster_barrier();
  grid_dependency_wait();

  int64_t low = 0, high = p.rows;
  if (p.offsets) {
    low = p.offsets[0];
    high = p.offsets[p.n_samples];
  }
  // Rows of this cluster: cluster, cluster + clusters, ...  Only rows that are worked on take a stage; n counts them.
  // Every warp finds out for itself, from the call's arguments alone, which those are, and so which barriers it
  // passes; a lane a row, the weights of 32 rows at a time.
  float weights_ahead = 0.f;
  uint32_t seen = 0;
  auto kind_of = [&](uint32_t row, float& weight) {
    if ((seen & 31) == 0) {
      const int64_t mine = static_cast<int64_t>(row) + static_cast<int64_t>(lane) * clusters;
      weights_ahead = p.weights && mine < p.rows ? p.weights[mine] : 1.f;
    }
    weight = __shfl_sync(0xffffffffu, weights_ahead, seen & 31);
    ++seen;
    return row < low || row >= high ? kRowAlone : __any_sync(0xffffffffu, weight != 0.f) ? kRowWork : kRowNoWeight;
  };
  struct Place {  // of row n in the ring: n = turn * stages + s
    int s, turn, stages;
    __device__ __forceinline__ void next() {
      if (++s == stages) {
        s = 0;
        ++turn;
      }
    }
  };
  Place ring_n{0, 0, r.stages};
  auto stage_of = [&](const Place& x) { return ring + x.s * r.stage_bytes; };
  auto top_of = [&](unsigned char* stage) {
    int* const place = reinterpret_cast<int*>(stage + r.units * 16);
    float* const z = reinterpret_cast<float*>(place + p.top);
    return RingTop{place, z, z + p.top, z + 2 * p.top};
  };
  float weight;

  if (warp == kWarps + 2) {
    // ---- the feeder; the first 64 entries of a row are asked for while the row before is prepared (as words that
    // nothing is done with until then: a conversion would wait for them)
    constexpr int kAhead = 2;
    struct Ahead {
      int64_t row;
      uint32_t id[kAhead], id_high[kAhead], t[kAhead];
      float lse;
    };
    uint32_t next_row = cluster;
    auto look_ahead = [&]() {
      Ahead x;
      x.row = -1;
      for (; next_row < p.rows && x.row < 0; next_row += clusters)
        if (kind_of(next_row, weight) == kRowWork) x.row = next_row;
      if (x.row >= 0) {
        const uint32_t row = static_cast<uint32_t>(x.row);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int j = lane + 32 * k;
          x.id[k] = x.id_high[k] = x.t[k] = 0u;
          if (j < p.top) {
            const uint32_t* const id = reinterpret_cast<const uint32_t*>(p.ids + static_cast<int64_t>(row) * p.ids_stride);
            if (p.id_bytes == 8) {
              x.id[k] = id[2 * j];
              x.id_high[k] = id[2 * j + 1];
            } else {
              x.id[k] = id[j];
            }
            const unsigned char* const t = row_of(p.t, row, 0);
            x.t[k] = p.t_dtype == ABS_F32 ? reinterpret_cast<const uint32_t*>(t)[j] : reinterpret_cast<const unsigned short*>(t)[j];
          }
        }
        x.lse = p.lse ? p.lse[row] : 0.f;
      }
      return x;
    };
    uint32_t n = 0;
    Ahead now = look_ahead();
    while (now.row >= 0) {
      const Ahead next = look_ahead();
      const uint32_t row = static_cast<uint32_t>(now.row);
      const int s = ring_n.s;
      if (ring_n.turn > 0) {
        // given back by the workers; and its last copy has landed, also where they gave up on it
        const uint32_t before = (ring_n.turn - 1) & 1;
        const bool free = mbar_wait_bounded(&empty[s], before, p.empty_polls) && mbar_wait_bounded(&full[s], before);
        if (__any_sync(0xffffffffu, !free)) break;
      }
      unsigned char* const stage = stage_of(ring_n);
      // the units of this block; the first and last of the row may reach out of the tensor at its ends
      const unsigned char* z = row_of(p.z, row, 0);
      const int before = static_cast<int>(reinterpret_cast<uintptr_t>(z) & 15);
      const unsigned char* from = z - before;
      const int n_units = (before + p.vocab * ESZ + 15) / 16;
      int a = first_unit, e = min(first_unit + r.units, n_units);
      if (a == 0 && from < r.z_begin) a = 1;
      if (e == n_units && from + static_cast<int64_t>(e) * 16 > r.z_end) --e;
      if (lane == 0) {
        if (e > a) {
          const uint32_t bytes = static_cast<uint32_t>(e - a) * 16u;
          mbar_expect_tx(&full[s], bytes);
          bulk_load(stage + (a - first_unit) * 16, from + static_cast<int64_t>(a) * 16, bytes, &full[s]);
        } else {
          mbar_arrive(&full[s]);
        }
      }
      const RingTop top = top_of(stage);
      const int shift = before / ESZ - first_unit * U;
      float m = kLowest, sum = 0.f;
      bool twice = false;
      auto take = [&](int j, int id, float t) {
        if (id < 0) t = -INFINITY;
        const int at = id >= 0 && id + shift >= 0 && id + shift < r.units * U ? id + shift : -1;
        top.place[j] = at;
        top.log_p[j] = t;
        m = fmaxf(m, t);
        if (at >= 0) twice |= (atomicOr(&marks[at >> 5], 1u << (at & 31)) >> (at & 31)) & 1u;
      };
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (lane + 32 * k < p.top) {
          // an index of 8 bytes is one of the vocabulary's if its high word is 0 and its low word is
          const bool known = now.id_high[k] == 0u && now.id[k] < static_cast<uint32_t>(p.vocab);
          const float t = p.t_dtype == ABS_F32    ? __uint_as_float(now.t[k])
                          : p.t_dtype == ABS_BF16 ? from_half_word<ABS_BF16>(now.t[k])
                                                  : from_half_word<ABS_F16>(now.t[k]);
          take(lane + 32 * k, known ? static_cast<int>(now.id[k]) : -1, t);
        }
      for (int j = lane + 32 * kAhead; j < p.top; j += 32) {
        const float t = load_teacher(p, row, j);
        take(j, load_id(p, row, j), t);
      }
      if (!p.lse) {
        m = warp_max(m);
        for (int j = lane; j < p.top; j += 32) sum += exp2_fast((top.log_p[j] - m) * p.c);
        sum = lanes_sum<32>(sum);
      }
      const float log_sum = log2f(sum);
      twice = __any_sync(0xffffffffu, twice);
      __syncwarp();  // all marks are set
      for (int j = lane; j < p.top; j += 32) {
        const float t = top.log_p[j];
        const float l = t == -INFINITY ? t : p.lse ? log_of_share(p, t, now.lse) : (t - m) * p.c - log_sum;
        top.log_p[j] = l;
        top.p[j] = exp2_fast(l);
        const int at = top.place[j];
        if (at >= 0) marks[at >> 5] = 0u;
      }
      if (lane == 0) {
        repeated_in[s] = twice;
        any_in[s] = p.lse || sum != 0.f;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[s]);
      now = next;
      ring_n.next();
      ++n;
    }
    // no copy is under way when the block ends, even where a worker gave up on one
    for (uint32_t k = 0; k < static_cast<uint32_t>(r.stages) && k < n; ++k)
      mbar_wait_bounded(&full[k], (n - 1 - k) / r.stages & 1);
  } else if (warp == kWarps + 1) {
    // ---- the topper
    uint32_t n = 0;
    for (uint32_t row = cluster; row < p.rows; row += clusters) {
      if (kind_of(row, weight) != kRowWork) continue;
      const uint32_t half = n & 1;
      part_sync<64>(kTopTaken + half);
      const RingTop top = top_of(stage_of(ring_n));
      const bool repeated = repeated_in[ring_n.s];
      ring_n.next();
      float m = kLowest, sum = 0.f, sum_p = 0.f, cross = 0.f;
      for (int j = lane; j < p.top; j += 32)
        if (top.place[j] >= 0) m = fmaxf(m, top.z[j]);
      m = warp_max(m);
      for (int j = lane; j < p.top; j += 32)
        if (top.place[j] >= 0) {
          // Of the workers of one index named twice one at least has read its logit, others perhaps the -inf
          // already.  The first entry stands for all of them in the sums; all of them write the gradient, so the
          // probabilities are added in the same order for each.
          float z = top.z[j];
          const float pj = top.p[j];
          float p_all = repeated ? 0.f : pj;
          bool first = true;
          if (repeated)
            for (int k = 0; k < p.top; ++k)
              if (top.place[k] == top.place[j]) {
                if (k < j) first = false;
                p_all += top.p[k];
                if (top.z[k] != -INFINITY) z = top.z[k];
              }
          if (first) sum += exp2_fast((z - m) * p.c);
          sum_p += pj;
          if (pj != 0.f) cross += pj * p.loss_scale * top.log_p[j] - pj * p.tau * (z - m);
          top.z[j] = z;
          top.log_p[j] = p_all;
        }
      sum = lanes_sum<32>(sum);
      sum_p = lanes_sum<32>(sum_p);
      cross = lanes_sum<32>(cross);
      if (lane == 0)
        from_top[half] = {{kLowest, 0.f}, {m, sum}, cross, sum_p, {}};
      part_arrive<THREADS + 64>(kSummed + half);
      ++n;
    }
  } else if (warp == kWarps) {
    // ---- the joiner
    uint32_t n = 0;
    for (uint32_t row = cluster; row < p.rows; row += clusters) {
      const int kind = kind_of(row, weight);
      if (kind == kRowNoWeight && rank == 0 && lane == 0) p.losses[row] = 0.f;
      if (kind != kRowWork) continue;
      const uint32_t half = n & 1;
      part_sync<THREADS + 64>(kSummed + half);
      const float g = any_in[ring_n.s] ? weight * p.grad_scale : 0.f;  // a teacher that names nothing asks for nothing
      ring_n.next();
      RingSums x = from_top[half];
      x.rest = warp_join(lane < kWarps ? from_warps[half][lane] : ExpSum{kLowest, 0.f}, p.c);
      if (dead) x.rest.s = nan;
      if (r.blocks > 1) {
        if (!dead) {
          if (lane == 0) mbar_expect_tx(&sums_here[half], r.blocks * 32u);
          __syncwarp();
          if (lane < r.blocks) send_sums(x, &from_blocks[half][rank], &sums_here[half], lane);
          dead = !mbar_wait_bounded(&sums_here[half], (n >> 1) & 1);
          dead = __any_sync(0xffffffffu, dead);
        }
        x = lane < r.blocks ? from_blocks[half][lane] : RingSums{{kLowest, 0.f}, {kLowest, 0.f}, 0.f, 0.f, {}};
        const float m_rest = warp_max(x.rest.m), m_top = warp_max(x.top.m);
        x.rest.s *= exp2_fast((x.rest.m - m_rest) * p.c);
        if (x.p != 0.f) x.cross += x.p * p.tau * (m_top - x.top.m);
        x.top.s *= exp2_fast((x.top.m - m_top) * p.c);
        static_assert(kRingMaxCluster == 8, "sums over the first eight lanes");
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) {
          x.rest.s += __shfl_xor_sync(0xffffffffu, x.rest.s, d);
          x.top.s += __shfl_xor_sync(0xffffffffu, x.top.s, d);
          x.p += __shfl_xor_sync(0xffffffffu, x.p, d);
          x.cross += __shfl_xor_sync(0xffffffffu, x.cross, d);
        }
        x.rest.m = m_rest;
        x.top.m = m_top;
        if (dead) x.rest.s = nan;
      }
      // lanes 0 to 7 know the row
      const ExpSum all = join(x.rest, x.top, p.c);
      float p_rest = p.lse ? fmaxf(1.f - x.p, 0.f) : 0.f;
      if (p.lse && x.p != x.p) p_rest = x.p;
      if (x.rest.s == 0.f) p_rest = 0.f;
      if (GRAD && lane == 0) {
        const float over_s = 1.f / all.s;
        answers[half] = {g * (exp2_fast((x.rest.m - all.m) * p.c) * over_s - (p_rest != 0.f ? p_rest / x.rest.s : 0.f)),
                         x.rest.m, g, all.m, over_s};
      }
      part_arrive<THREADS + 32>(kAnswered + half);
      if (rank == 0 && lane == 0) {
        const float log_s = log2f(all.s);
        float loss = x.cross + p.loss_scale * log_s * x.p;
        if (x.p != 0.f) loss += x.p * p.tau * (all.m - x.top.m);
        if (p_rest != 0.f)
          loss += p_rest * p.loss_scale * (log2f(p_rest) - log2f(x.rest.s) + log_s) + p_rest * p.tau * (all.m - x.rest.m);
        p.losses[row] = loss;
      }
      __syncwarp();
      ++n;
    }
  } else {
    // ---- the workers
    uint32_t row = cluster;
    unsigned char* late_at = nullptr;  // a gradient of the top that waits for the next barrier
    float late = 0.f;
    auto write_late = [&]() {
      if (late_at) store_one<DT>(late_at, 0, late);
      late_at = nullptr;
    };
    // the row whose pass 2 is still to come
    uint32_t n = 0;
    Place ring_before = ring_n;
    unsigned char* dz_before = nullptr;  // of this block's first unit
    int mine_before = 0, i_before = 0;
    for (;;) {
      // the next row to work on; those that do not count on the way
      const unsigned char* z = nullptr;
      unsigned char* dz = nullptr;
      int before = 0, n_units = 0, mine = 0, i_first = 0;
      bool have = false;
      for (; row < p.rows && !have; row += clusters) {
        const int kind = kind_of(row, weight);
        if (kind == kRowAlone) continue;
        z = row_of(p.z, row, 0);
        before = static_cast<int>(reinterpret_cast<uintptr_t>(z) & 15);
        n_units = (before + p.vocab * ESZ + 15) / 16;
        mine = min(r.units, n_units - first_unit);   // units of this block; may be negative
        i_first = first_unit * U - before / ESZ;     // index of its first value in the row; may be negative
        if constexpr (GRAD) dz = row_of(p.dz, row, 0) - before + static_cast<int64_t>(first_unit) * 16;
        have = kind == kRowWork;
        if (GRAD && !have) {
          const uint32_t none[4] = {};
          for (int u = tid; u < mine; u += THREADS) write_unit<DT>(dz + u * 16, i_first + u * U, p.vocab, none);
        }
      }
      unsigned char* const stage = stage_of(ring_n);
      // Every piece of a copy that lands wakes whoever waits for the whole: only the warps that have something to do
      // before the barrier wait for it there (with all of them at it, polling took four of ten instructions); the
      // others look once behind the barrier, when it has landed.
      const bool early = warp * 32 < max(p.top, 2 * U);
      if (have) {
        if (early && !dead) dead = !mbar_wait_bounded(&full[ring_n.s], ring_n.turn & 1);
        // values of the row's first and last unit: outside of the row, or not brought by the copy
        if (tid < 2 * U) {
          const int unit = tid < U ? 0 : n_units - 1;
          const int j = tid % U;
          if (unit >= first_unit && unit < first_unit + mine && (tid < U || n_units > 1)) {
            const int i = i_first + (unit - first_unit) * U + j;  // index in the row
            const unsigned char* from = z - before + static_cast<int64_t>(unit) * 16;
            unsigned char* to = stage + (unit - first_unit) * 16;
            if (i < 0 || i >= p.vocab) {
              store_one<DT>(to, j, -INFINITY);
            } else if (from < r.z_begin || from + 16 > r.z_end) {
              if constexpr (DT == ABS_F32) reinterpret_cast<uint32_t*>(to)[j] = reinterpret_cast<const uint32_t*>(from)[j];
              else reinterpret_cast<unsigned short*>(to)[j] = reinterpret_cast<const unsigned short*>(from)[j];
            }
          }
        }
        const bool edges = (first_unit == 0 && z - before < r.z_begin) ||
                           (first_unit + mine == n_units && z - before + static_cast<int64_t>(n_units) * 16 > r.z_end);
        if (edges) workers_barrier<THREADS>();  // the top may lie among what has just been put there
        if (tid < p.top) {
          const RingTop top = top_of(stage);
          const int at = top.place[tid];
          if (static_cast<unsigned>(at) < static_cast<unsigned>(r.units * U)) {
            top.z[tid] = load_value<DT>(stage, at);
            store_one<DT>(stage, at, -INFINITY);
          }
        }
      }
      workers_barrier<THREADS>();
      if constexpr (GRAD) write_late();

      if (have) {  // pass 1
        if (!early && !dead) dead = !mbar_wait_bounded(&full[ring_n.s], ring_n.turn & 1);
        if (warp == 0) part_arrive<64>(kTopTaken + (n & 1));
        const uint32_t none = DT == ABS_F32 ? 0xff800000u : DT == ABS_BF16 ? 0xff80ff80u : 0xfc00fc00u;  // -inf
        uint32_t top = none;
        for_units<THREADS>(0, mine, stage, none, [&](int, const uint32_t (&w)[4], bool) {
          top = max_words<DT>(top, max_words<DT>(max_words<DT>(w[0], w[1]), max_words<DT>(w[2], w[3])));
        });
        const float m = warp_max(fmaxf(max_of_word<DT>(top), kLowest));
        const Exponentials ex(m, p.c);
        uint64_t pairs = pair_of(0.f, 0.f);
        auto sum_of = [&](auto exponentials) {
          for_units<THREADS>(0, mine, stage, none, [&](int, const uint32_t (&w)[4], bool) {
            uint64_t e[U / 2];
#pragma unroll
            for (int j = 0; j < U; j += 2) e[j / 2] = exponentials(value_of<DT>(w, j), value_of<DT>(w, j + 1));
#pragma unroll
            for (int d = U / 4; d > 0; d /= 2)
#pragma unroll
              for (int j = 0; j < d; ++j) e[j] = pair_add(e[j], e[j + d]);
            pairs = pair_add(pairs, e[0]);
          });
        };
        if (!ex.far) sum_of([&](float a, float b) { return ex(a, b); });
        else sum_of([&](float a, float b) { return ex.of_far(a, b); });
        float sum = (pair_as(pairs).x + pair_as(pairs).y) * ex.correction;
        sum = lanes_sum<32>(dead ? nan : sum);
        if (lane == 0) from_warps[n & 1][warp] = {m, sum};
        part_arrive<THREADS + 64>(kSummed + (n & 1));
      }

      if (n > 0) {  // pass 2 of the row before
        const uint32_t half = (n - 1) & 1;
        part_sync<THREADS + 32>(kAnswered + half);
        if constexpr (GRAD) {
          unsigned char* const stage_before = stage_of(ring_before);
          const RingAnswer answer = answers[half];
          if (tid < p.top) {
            const RingTop top = top_of(stage_before);
            const int at = top.place[tid];
            if (static_cast<unsigned>(at) < static_cast<unsigned>(r.units * U) &&
                static_cast<unsigned>(i_before + at) < static_cast<unsigned>(p.vocab)) {
              late_at = dz_before + at * ESZ;
              late = answer.g * (exp2_fast((top.z[tid] - answer.m_all) * p.c) * answer.over_s - top.log_p[tid]);
            }
          }
          const Exponentials ex(answer.m, p.c);
          const float f = dead ? nan : answer.factor * ex.correction;
          // the units that lie in the row whole, then its first and last by a thread each
          const int from = i_before < 0 ? 1 : 0;
          const int to = i_before + mine_before * U > p.vocab ? mine_before - 1 : mine_before;
          const uint64_t ff = pair_of(f, f);
          auto write = [&](auto exponentials) {
            auto unit = [&](const uint32_t (&w)[4], uint32_t (&out)[4]) {
#pragma unroll
              for (int j = 0; j < U; j += 2) {
                const float2 d = pair_as(pair_mul(exponentials(value_of<DT>(w, j), value_of<DT>(w, j + 1)), ff));
                if constexpr (DT == ABS_F32) {
                  out[j] = __float_as_uint(d.x);
                  out[j + 1] = __float_as_uint(d.y);
                } else {
                  out[j / 2] = pack_16x2<DT>(d.x, d.y);
                }
              }
            };
            for_units<THREADS>(from, to, stage_before, 0u, [&](int u, const uint32_t (&w)[4], bool there) {
              uint32_t out[4];
              unit(w, out);
              if (there) *reinterpret_cast<uint4*>(dz_before + u * 16) = make_uint4(out[0], out[1], out[2], out[3]);
            });
            const int u = tid == 0 && from > 0 ? 0 : to;
            if ((tid == 0 && from > 0 && mine_before > 0) || (tid == (from > 0 ? 32 : 0) && to >= from && to < mine_before)) {
              const uint4 v = *reinterpret_cast<const uint4*>(stage_before + u * 16);
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
              uint32_t out[4];
              unit(w, out);
              write_unit<DT>(dz_before + u * 16, i_before + u * U, p.vocab, out);
            }
          };
          if (!ex.far) write([&](float a, float b) { return ex(a, b); });
          else write([&](float a, float b) { return ex.of_far(a, b); });
        }
        // the stage has been read: the copy of a later row may overwrite it
        fence_generic_to_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[ring_before.s]);
      }
      if (!have) break;
      ring_before = ring_n;
      dz_before = dz;
      mine_before = mine;
      i_before = i_first;
      ring_n.next();
      ++n;
    }
    workers_barrier<THREADS>();
    if constexpr (GRAD) write_late();
  }
  // no block leaves while another may still send sums to it
  __syncthreads();
  if (r.blocks > 1) cluster_barrier();
}

}  // namespace absnt
