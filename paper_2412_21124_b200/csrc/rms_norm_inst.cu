// One instantiation of the norm's kernels per translation unit: compiled once for each type
// -DABS_INST_XT=... by build.py.
#include "rms_norm_launch.cuh"

namespace absnt {
template cudaError_t launch_norm<ABS_INST_XT>(const NormParams&, int, int, cudaStream_t);
template cudaError_t launch_norm_grad<ABS_INST_XT>(const NormGradParams&, int, int64_t, int, cudaStream_t);
}  // namespace absnt
