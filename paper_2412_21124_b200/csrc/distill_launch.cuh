// Which kernel a call of abs_distill_loss runs.  Instantiated once for each type of the logits in a translation
// unit of its own, distill_inst.cu.
#pragma once
#include "distill.cuh"
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
// vec: 8 where all rows of logits and gradient begin on boundaries of eight values, else 1
template <int DT>
cudaError_t launch_distill(const DistillParams& p, int vec, cudaStream_t st) {
  if (vec == 8) return distill_by_block<DT, 8>(p, st);
  return distill_by_block<DT, 1>(p, st);
}

#ifndef ABS_INST_XT
extern template cudaError_t launch_distill<ABS_F32>(const DistillParams&, int, cudaStream_t);
extern template cudaError_t launch_distill<ABS_BF16>(const DistillParams&, int, cudaStream_t);
extern template cudaError_t launch_distill<ABS_F16>(const DistillParams&, int, cudaStream_t);
#endif

}  // namespace absnt
