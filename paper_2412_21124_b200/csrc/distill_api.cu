// C entry point of the distillation loss: checks and launches.
#include "distill_launch.cuh"
#include "rows_checks.cuh"

using namespace absnt;

namespace absnt {

int ring_clusters(const void* kernel, const cudaLaunchConfig_t& cfg) {
  struct Known {
    const void* kernel;
    size_t smem;
    unsigned blocks;
    int device, clusters;
  };
  static std::mutex mu;
  static Known known[64];
  static int n_known = 0, oldest = 0;
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return 0;
  const Known want = {kernel, cfg.dynamicSmemBytes, cfg.gridDim.x, device, 0};
  {
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < n_known; ++i)
      if (known[i].kernel == want.kernel && known[i].smem == want.smem && known[i].blocks == want.blocks &&
          known[i].device == want.device)
        return known[i].clusters;
  }
  int clusters = 0;
  if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess) {
    (void)cudaGetLastError();
    return 0;
  }
  std::lock_guard<std::mutex> lock(mu);
  Known& to = n_known < 64 ? known[n_known++] : known[oldest++ % 64];
  to = want;
  to.clusters = clusters;
  return clusters;
}

}  // namespace absnt

namespace {

int distill_loss(const abs_distill_args* a, int empty_polls, abs_stream_t stream) {
  if (!a) return ABS_ERR_NULL;
  const bool table = a->offsets != nullptr;
  if (a->rows < 0 || a->rows > INT32_MAX || a->vocab < 1 || a->top < 1 || a->top > ABS_MAX_TOP) return ABS_ERR_RANGE;
  if (a->vocab > ABS_MAX_VOCAB) return ABS_ERR_TOO_LARGE;
  if (!(a->temperature >= 1e-3 && a->temperature <= 1e3) || !(std::fabs(a->grad_scale) <= 1e30)) return ABS_ERR_RANGE;
  if (a->n_samples < 0 || a->n_samples > ABS_MAX_SAMPLES) return ABS_ERR_RANGE;
  if (table != (a->n_samples > 0)) return ABS_ERR_NULL;
  if (a->id_bytes != 4 && a->id_bytes != 8) return ABS_ERR_DTYPE;
  const bool empty = a->rows == 0;
  const int64_t rows = empty ? 1 : a->rows;
  int rc;
  Rows z, dz, t;
  if ((rc = take_rows(a->logits, rows, 1, a->vocab, z)) != ABS_OK) return rc;
  if ((rc = take_rows(a->dlogits, rows, 1, a->vocab, dz)) != ABS_OK) return rc;
  if ((rc = take_rows(a->top_logits, rows, 1, a->top, t)) != ABS_OK) return rc;
  // the indices as rows of another type: described by their size alone
  abs_rows ids_as = {const_cast<void*>(a->top_ids), a->ids_stride, 0, ABS_F32, 0};
  Rows ids;
  if ((rc = take_rows(ids_as, rows, 1, a->top, ids)) != ABS_OK) return rc;
  if (a->id_bytes == 8 && misaligned(a->top_ids, 8)) return ABS_ERR_ALIGN;
  ids.s0 = ids.s0 / 4 * a->id_bytes;
  ids.esz = a->id_bytes;
  if (!empty && (!z.given() || !t.given() || !ids.given() || !a->losses)) return ABS_ERR_NULL;
  if (!empty && (!wide_float(z.dtype) || !wide_float(t.dtype) || (dz.given() && dz.dtype != z.dtype))) return ABS_ERR_DTYPE;
  for (const void* f : {static_cast<const void*>(a->teacher_lse), static_cast<const void*>(a->weights),
                        static_cast<const void*>(a->offsets), static_cast<const void*>(a->losses),
                        static_cast<const void*>(a->sample_losses)})
    if (misaligned(f, 4)) return ABS_ERR_ALIGN;

  // dlogits may be the logits, element by element; nothing else may share a byte with an output
  const size_t n = static_cast<size_t>(a->rows) * 4;
  const size_t samples = static_cast<size_t>(table ? a->n_samples : 1);
  struct { const void* p; size_t n; } flat[] = {{a->losses, n},
                                                {a->sample_losses, samples * 4},
                                                {a->teacher_lse, n},
                                                {a->weights, n},
                                                {a->offsets, (samples + 1) * 4}};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i && j < 2; ++j)
      if (flat[i].p && flat[j].p && overlaps(flat[i].p, flat[i].n, flat[j].p, flat[j].n)) return ABS_ERR_ALIAS;
  if (!empty) {
    if (dz.given()) {
      if (!separate_rows(dz)) return ABS_ERR_ALIAS;
      if (!same_rows(dz, z) && rows_touch(dz, z)) return ABS_ERR_ALIAS;
      for (const Rows* in : {&t, &ids})
        if (overlaps(dz.p, dz.bytes(), in->p, in->bytes())) return ABS_ERR_ALIAS;
    }
    for (int i = 0; i < 5; ++i) {
      if (!flat[i].p) continue;
      if (dz.given() && overlaps(flat[i].p, flat[i].n, dz.p, dz.bytes())) return ABS_ERR_ALIAS;
      if (i < 2)
        for (const Rows* in : {&z, &t, &ids})
          if (overlaps(flat[i].p, flat[i].n, in->p, in->bytes())) return ABS_ERR_ALIAS;
    }
  }

  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!empty) {
    DistillParams p = {};
    p.z = z.arg();
    p.dz = dz.arg();
    p.t = t.arg();
    p.ids = static_cast<const unsigned char*>(a->top_ids);
    p.ids_stride = ids.s0;
    p.lse = a->teacher_lse;
    p.weights = a->weights;
    p.offsets = a->offsets;
    p.losses = a->losses;
    p.rows = static_cast<uint32_t>(rows);
    p.n_samples = static_cast<int>(a->n_samples);
    p.vocab = static_cast<int>(a->vocab);
    p.top = static_cast<int>(a->top);
    p.t_dtype = t.dtype;
    p.id_bytes = a->id_bytes;
    p.empty_polls = empty_polls;
    constexpr double kLog2e = 1.4426950408889634;
    p.c = static_cast<float>(kLog2e / a->temperature);
    p.inv_tau = 1.0 / a->temperature;
    p.tau = static_cast<float>(a->temperature);
    p.loss_scale = static_cast<float>(a->temperature * a->temperature / kLog2e);
    p.grad_scale = static_cast<float>(a->temperature * a->grad_scale);
    const int vec = a->vocab % 8 == 0 && rows_aligned(z, 8) && rows_aligned(dz, 8) ? 8 : 1;
    cudaError_t e;
    if (z.dtype == ABS_F32) e = launch_distill<ABS_F32>(p, vec, st);
    else if (z.dtype == ABS_BF16) e = launch_distill<ABS_BF16>(p, vec, st);
    else e = launch_distill<ABS_F16>(p, vec, st);
    if (e != cudaSuccess) return cuda_fail(e);
  }
  if (!a->sample_losses) return ABS_OK;
  SampleLossParams s = {a->losses, a->weights, a->offsets, a->sample_losses, static_cast<uint32_t>(a->rows)};
  const cudaError_t e = launch_pdl(distill_samples_kernel, dim3(static_cast<unsigned>(samples)), dim3(kSampleLossThreads), st, s);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

}  // namespace

extern "C" {

int abs_distill_loss(const abs_distill_args* a, abs_stream_t stream) { return distill_loss(a, kBulkWaitLimit, stream); }

int abs_selftest_distill_wait(const abs_distill_args* a, int polls, abs_stream_t stream) {
  if (polls < 0 || polls > kBulkWaitLimit) return ABS_ERR_RANGE;
  return distill_loss(a, polls, stream);
}

}  // extern "C"
