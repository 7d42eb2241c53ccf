// Which kernel a call of abs_rms_norm or abs_rms_norm_grad runs.  The functions are instantiated once for
// each type of x (dy) in a translation unit of its own, rms_norm_inst.cu.
#pragma once
#include "launch.cuh"
#include "rms_norm_grad.cuh"

namespace absnt {

// the widest row: 32 warps of 16 values a lane
constexpr int kMaxNormWidth = 32 * 32 * 16;

// ---- forward
template <int XT, int RT, int VEC, int L, int NI, int NR>
cudaError_t norm_by_lanes(const NormParams& p, cudaStream_t st) {
  const uint32_t per_block = 8 * (32 / L) * NR;
  return launch_pdl(rms_norm_kernel<XT, RT, VEC, L, NI, NR, false>, dim3((p.rows + per_block - 1) / per_block),
                    dim3(32, 8), st, p);
}
template <int XT, int RT, int VEC, int NI>
cudaError_t norm_by_block(const NormParams& p, cudaStream_t st) {
  constexpr int cols = 32 * lane_values<VEC>() * NI;  // of a warp
  return launch_pdl(rms_norm_kernel<XT, RT, VEC, 32, NI, 1, true>, dim3(p.rows), dim3(32 * ((p.h + cols - 1) / cols)), st, p);
}
// Rows of a warp or less go to its lanes, several rows of a lane at once: 100000 x 255 in 16 bits 32 us, by a block a row 54;
// 80000 x 512 39 and 58; 40000 x 1024 29 and 33 (fp32, 51 and 50: by blocks).  Heads of 64, 524288 of them: 24 us
// with four rows at once, 36 with one.  Wider ones take a block, whose threads hold eight or sixteen values: more threads
// a row cost more in their meeting than they bring in loads (8192 x 8192 into 8 bits 101 us with 8 values a thread, 94
// with 16; 20000 x 2048 36 and 30), and from 4096 on 32 of them (91).  In smaller pieces: 40000 x 1028 61 us with 4
// values a thread, 44 with 8 and with 16; 10000 x 4100 48 with 8, 41 with 16.
template <int XT, int RT>
cudaError_t norm_vec(const NormParams& p, int vec, cudaStream_t st) {
  const int h = p.h;
  if (vec == 8) {
    if (h <= 64) return norm_by_lanes<XT, RT, 8, 8, 1, 4>(p, st);
    if (h <= 128) return norm_by_lanes<XT, RT, 8, 16, 1, 4>(p, st);
    if (h <= 256) return norm_by_lanes<XT, RT, 8, 32, 1, 4>(p, st);
    if (h <= 512) return norm_by_lanes<XT, RT, 8, 32, 2, 2>(p, st);
    if constexpr (XT != ABS_F32) {
      if (h <= 768) return norm_by_lanes<XT, RT, 8, 32, 3, 1>(p, st);
      if (h <= 1024) return norm_by_lanes<XT, RT, 8, 32, 4, 1>(p, st);
    }
    if (h <= 4096) return norm_by_block<XT, RT, 8, 2>(p, st);
    return norm_by_block<XT, RT, 8, 4>(p, st);
  }
  if (vec == 4) {
    if (h <= 128) return norm_by_lanes<XT, RT, 4, 32, 1, 4>(p, st);
    if (h <= 256) return norm_by_lanes<XT, RT, 4, 32, 2, 4>(p, st);
    if (h <= 512) return norm_by_lanes<XT, RT, 4, 32, 4, 2>(p, st);
    if (h <= 1536) return norm_by_block<XT, RT, 4, 2>(p, st);
    return norm_by_block<XT, RT, 4, 4>(p, st);
  }
  if (h <= 128) return norm_by_lanes<XT, RT, 1, 32, 1, 4>(p, st);
  if (h <= 256) return norm_by_lanes<XT, RT, 1, 32, 2, 2>(p, st);
  if (h <= 512) return norm_by_lanes<XT, RT, 1, 32, 4, 1>(p, st);
  if (h <= 1536) return norm_by_block<XT, RT, 1, 2>(p, st);
  return norm_by_block<XT, RT, 1, 4>(p, st);
}
// r_dtype < 0: no residual
template <int XT>
cudaError_t launch_norm(const NormParams& p, int r_dtype, int vec, cudaStream_t st) {
  if (r_dtype < 0) return norm_vec<XT, -1>(p, vec, st);
  if (r_dtype == XT) return norm_vec<XT, XT>(p, vec, st);
  return norm_vec<XT, ABS_F32>(p, vec, st);
}

// ---- backward
// A row of at most this many values goes to the lanes of a warp, two or four rows at once; one of at most kGradHalf to
// threads of eight values, wider ones to threads of sixteen (9001 x 1537 f16: five us more with sixteen; bf16 with an fp32
// stream, the residual's gradient and 8 samples, 43662 x 1537 182 us, 206 with sixteen, 43690 x 1536 156 and 157, 32768 x 2048 147
// and 148).
constexpr int kGradHalf = 2048;
constexpr int grad_lane_values(int vec) { return vec == 8 ? 256 : 128; }
// Blocks of the kernel that sums over rows: as many as fit the SMs at once, but two rows a block at least, since every
// block leaves a record: 512 x 2048 with 8 samples 15 us by 512 blocks, 11 by 256, 13 by 128, and 512 x 768 8.9, 7.8, 8.8.
// Rows above 4096 take blocks of 512 or 1024 threads, one an SM: 8192 x 8192 164 us, 169 with two of 64 registers.  (13106 x
// 5120 takes 197 us, and 177 with two; 4096 x 16384, of 1024 threads, 186.)
inline int64_t grad_most_blocks(int64_t h, int vec) {
  return kSMs * (h <= 8 * 512 ? grad_blocks_per_sm(h > grad_lane_values(vec), vec, h <= kGradHalf) : 1);
}
inline int64_t grad_blocks(int64_t rows, int64_t h, int vec) {
  const int64_t most = grad_most_blocks(h, vec), pairs = (rows + 1) / 2;
  return pairs < most ? pairs : most;
}
inline int64_t record_pitch(int64_t h) { return (h + 7) / 8 * 8; }  // VEC 8 writes 32 bytes at once

template <int GT, int ST, bool ADD, int VEC, int L, int NI, int NR>
cudaError_t grad_by_lanes(const NormGradParams& p, int64_t blocks, cudaStream_t st) {
  return launch_pdl(rms_norm_grad_kernel<GT, ST, ADD, VEC, L, NI, NR, false, 256>, dim3(static_cast<unsigned>(blocks)),
                    dim3(32, 8), st, p);
}
template <int GT, int ST, bool ADD, int VEC, int THREADS, int NI = grad_pieces<VEC>()>
cudaError_t grad_by_block_of(const NormGradParams& p, int64_t blocks, int warps, cudaStream_t st) {
  const auto kernel = rms_norm_grad_kernel<GT, ST, ADD, VEC, 32, NI, 1, true, THREADS>;
  const int values = warps * 32 * lane_values<VEC>() * NI;  // of the weight, with what lies behind the row's end
  const cudaError_t e = allow_dynamic_smem(reinterpret_cast<const void*>(kernel), THREADS * NI * lane_values<VEC>() * sizeof(float));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(32 * warps, THREADS == 256 ? 8 / warps : 1);
  cfg.dynamicSmemBytes = values * sizeof(float);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}
template <int GT, int ST, bool ADD, int VEC>
cudaError_t grad_by_block(const NormGradParams& p, int64_t blocks, cudaStream_t st) {
  constexpr int cols = 32 * lane_values<VEC>() * grad_pieces<VEC>();
  static_assert(cols == 512, "grad_blocks counts on it");
  const int warps = (p.h + cols - 1) / cols;
  if (p.h <= kGradHalf) {
    constexpr int half = 32 * lane_values<VEC>() * (grad_pieces<VEC>() / 2);
    return grad_by_block_of<GT, ST, ADD, VEC, 256, grad_pieces<VEC>() / 2>(p, blocks, (p.h + half - 1) / half, st);
  }
  if (warps <= 8) return grad_by_block_of<GT, ST, ADD, VEC, 256>(p, blocks, warps, st);
  if (warps <= 16) return grad_by_block_of<GT, ST, ADD, VEC, 512>(p, blocks, warps, st);
  return grad_by_block_of<GT, ST, ADD, VEC, 1024>(p, blocks, warps, st);
}
template <int GT, int ST, bool ADD>
cudaError_t grad_vec(const NormGradParams& p, int64_t blocks, int vec, cudaStream_t st) {
  const int h = p.h;
  if (vec == 8) {
    if (h <= 64) return grad_by_lanes<GT, ST, ADD, 8, 8, 1, 2>(p, blocks, st);
    if (h <= 128) return grad_by_lanes<GT, ST, ADD, 8, 16, 1, 2>(p, blocks, st);
    if (h <= grad_lane_values(8)) return grad_by_lanes<GT, ST, ADD, 8, 32, 1, 2>(p, blocks, st);
    return grad_by_block<GT, ST, ADD, 8>(p, blocks, st);
  }
  if (vec == 4) {
    if (h <= grad_lane_values(4)) return grad_by_lanes<GT, ST, ADD, 4, 32, 1, 4>(p, blocks, st);
    return grad_by_block<GT, ST, ADD, 4>(p, blocks, st);
  }
  if (h <= grad_lane_values(1)) return grad_by_lanes<GT, ST, ADD, 1, 32, 1, 4>(p, blocks, st);
  return grad_by_block<GT, ST, ADD, 1>(p, blocks, st);
}
template <int GT>
cudaError_t launch_norm_grad(const NormGradParams& p, int s_dtype, int64_t blocks, int vec, cudaStream_t st) {
  if (s_dtype == GT)
    return p.add.p ? grad_vec<GT, GT, true>(p, blocks, vec, st) : grad_vec<GT, GT, false>(p, blocks, vec, st);
  return p.add.p ? grad_vec<GT, ABS_F32, true>(p, blocks, vec, st) : grad_vec<GT, ABS_F32, false>(p, blocks, vec, st);
}

#ifndef ABS_INST_XT
extern template cudaError_t launch_norm<ABS_F32>(const NormParams&, int, int, cudaStream_t);
extern template cudaError_t launch_norm<ABS_BF16>(const NormParams&, int, int, cudaStream_t);
extern template cudaError_t launch_norm<ABS_F16>(const NormParams&, int, int, cudaStream_t);
extern template cudaError_t launch_norm_grad<ABS_F32>(const NormGradParams&, int, int64_t, int, cudaStream_t);
extern template cudaError_t launch_norm_grad<ABS_BF16>(const NormGradParams&, int, int64_t, int, cudaStream_t);
extern template cudaError_t launch_norm_grad<ABS_F16>(const NormGradParams&, int, int64_t, int, cudaStream_t);
#endif

}  // namespace absnt
