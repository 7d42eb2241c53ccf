// One instantiation of the distillation kernels per translation unit: compiled once for each type
// -DABS_INST_XT=... by build.py.
#include "distill_launch.cuh"

namespace absnt {
template cudaError_t launch_distill<ABS_INST_XT>(const DistillParams&, int, cudaStream_t);
}  // namespace absnt
