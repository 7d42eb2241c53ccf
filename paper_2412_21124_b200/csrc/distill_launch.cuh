// Which kernel a call of abs_distill_loss runs.  Instantiated once for each type of the logits in a translation
// unit of its own, distill_inst.cu.
#pragma once
#include "distill_ring.cuh"
#include "launch.cuh"

namespace absnt {

template <int DT, int VEC>
cudaError_t distill_by_block(const DistillParams& p, cudaStream_t st) {
  // the limit is raised once for each kernel, so at once to what the largest vocabulary takes
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(distill_kernel<DT, VEC>), ABS_MAX_VOCAB / 8);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.rows);
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(p.vocab + 31) / 32 * 4;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, distill_kernel<DT, VEC>, p);
}

// How many clusters of a kernel the device holds at once: a persistent grid of just these.  Asked once for each
// (kernel, shared memory, cluster, device); 0 if the cluster is refused.
int ring_clusters(const void* kernel, const cudaLaunchConfig_t& cfg);

// How a row is cut: see distill_ring.cuh.  blocks 0: the row does not fit.
struct RingShape {
  int blocks, threads, units, stages, stage_bytes;
  size_t smem;
};
constexpr int kRingUnits = 8;  // of a worker, at most: 64 values of 16 bits, 32 floats
constexpr int kRingSmemPerSM = 228 * 1024, kRingStatic = 3 * 1024;  // the latter with what a block takes anyway
constexpr int kRingSmemMost = 224 * 1024;                            // dynamic, of a block that has an SM to itself

inline RingShape ring_shape(const DistillParams& p, int esz) {
  RingShape s = {};
  const int64_t total = (16 - esz + static_cast<int64_t>(p.vocab) * esz + 15) / 16;  // with the worst alignment
  // as few blocks as hold a row with two blocks on an SM; with 512 workers and one block if that is too many
  int64_t blocks = (total + 256 * kRingUnits - 1) / (256 * kRingUnits);
  if (blocks > kRingMaxCluster) blocks = (total + 512 * kRingUnits - 1) / (512 * kRingUnits);
  if (blocks > kRingMaxCluster) return s;
  // few rows: every SM gets a part of one, down to 4 KB
  while (blocks * 2 <= kRingMaxCluster && p.rows * blocks * 2 <= kSMs && total / (blocks * 2) >= 256) blocks *= 2;
  s.units = static_cast<int>((total + blocks - 1) / blocks);
  s.threads = 128;
  while (s.threads * kRingUnits < s.units || s.threads < p.top) s.threads *= 2;
  s.stage_bytes = s.units * 16 + p.top * 16;
  const int marks = (s.units * (16 / esz) + 31) / 32 * 4;
  for (int per_sm = ring_blocks_per_sm(s.threads);; per_sm = (per_sm + 1) / 2) {
    const int room = kRingSmemPerSM / per_sm - kRingStatic;
    s.stages = ((room < kRingSmemMost ? room : kRingSmemMost) - marks) / s.stage_bytes;
    if (s.stages >= 3 || per_sm == 1) break;
  }
  if (s.stages < 2) return s;
  if (s.stages > kRingMaxStages) s.stages = kRingMaxStages;
  s.smem = static_cast<size_t>(s.stages) * s.stage_bytes + marks;
  s.blocks = static_cast<int>(blocks);
  return s;
}

template <int DT, int THREADS, bool GRAD>
cudaError_t distill_by_ring(const DistillParams& p, const RingShape& s, cudaStream_t st) {
  const auto kernel = distill_ring_kernel<DT, THREADS, GRAD>;
  cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), kRingSmemMost);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(s.blocks);
  cfg.blockDim = dim3(THREADS + 96);
  cfg.dynamicSmemBytes = s.smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = s.blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int64_t clusters = ring_clusters(reinterpret_cast<const void*>(kernel), cfg);
  if (clusters < 1) return distill_by_block<DT, 1>(p, st);  // a device that does not take the cluster
  if (clusters > p.rows) clusters = p.rows;
  cfg.gridDim = dim3(static_cast<unsigned>(clusters * s.blocks));
  cfg.numAttrs = 2;
  RingParams r = {};
  r.d = p;
  r.blocks = s.blocks;
  r.units = s.units;
  r.stages = s.stages;
  r.stage_bytes = s.stage_bytes;
  r.z_begin = p.z.p;
  r.z_end = p.z.p + static_cast<int64_t>(p.rows - 1) * p.z.s0 + static_cast<int64_t>(p.vocab) * elem_bytes<DT>();
  return cudaLaunchKernelEx(&cfg, kernel, r);
}
template <int DT, bool GRAD>
cudaError_t distill_by_ring_of(const DistillParams& p, const RingShape& s, cudaStream_t st) {
  if (s.threads == 128) return distill_by_ring<DT, 128, GRAD>(p, s, st);
  if (s.threads == 256) return distill_by_ring<DT, 256, GRAD>(p, s, st);
  return distill_by_ring<DT, 512, GRAD>(p, s, st);
}

// vec: 8 where all rows of logits and gradient begin on boundaries of eight values, else 1
template <int DT>
cudaError_t launch_distill(const DistillParams& p, int vec, cudaStream_t st) {
  // the gradient at the logits' distance from a 16-byte boundary, in every row
  const bool in_step = !p.dz.p || ((p.z.p - p.dz.p) % 16 == 0 && (p.z.s0 - p.dz.s0) % 16 == 0);
  const RingShape s = ring_shape(p, elem_bytes<DT>());
  if (in_step && s.blocks > 0) return p.dz.p ? distill_by_ring_of<DT, true>(p, s, st) : distill_by_ring_of<DT, false>(p, s, st);
  if (vec == 8) return distill_by_block<DT, 8>(p, st);
  return distill_by_block<DT, 1>(p, st);
}

#ifndef ABS_INST_XT
extern template cudaError_t launch_distill<ABS_F32>(const DistillParams&, int, cudaStream_t);
extern template cudaError_t launch_distill<ABS_BF16>(const DistillParams&, int, cudaStream_t);
extern template cudaError_t launch_distill<ABS_F16>(const DistillParams&, int, cudaStream_t);
#endif

}  // namespace absnt
