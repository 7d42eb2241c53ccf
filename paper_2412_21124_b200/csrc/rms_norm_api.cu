// C entry points of the root-mean-square norm and its backward pass: checks and launches.
#include <algorithm>

#include "rms_norm_launch.cuh"
#include "rows_checks.cuh"

using namespace absnt;

namespace {

// rows and width of a call; every count fits the kernels' 32 bits
int check_shape(int64_t n0, int64_t n1, int64_t h) {
  if (n0 < 0 || n1 < 0 || h < 1) return ABS_ERR_RANGE;
  if (n0 > INT32_MAX || n1 > INT32_MAX || n0 * n1 > INT32_MAX) return ABS_ERR_RANGE;
  if (h > kMaxNormWidth) return ABS_ERR_TOO_LARGE;
  return ABS_OK;
}

int check_weight(const void* w, int dtype) {
  if (!w) return ABS_OK;
  if (!wide_float(dtype)) return ABS_ERR_DTYPE;
  return misaligned(w, bytes_of(dtype)) ? ABS_ERR_ALIGN : ABS_OK;
}

bool good_eps(double eps) { return eps >= ABS_MIN_NORM_EPS && eps <= 1e30; }

// how many consecutive values a thread may load at once: see Piece
int vector_width(int64_t h, const void* w, int w_dtype, const Rows* const* all, int n) {
  for (int vec : {8, 4}) {
    bool fits = h % vec == 0 && (!w || !misaligned(w, static_cast<size_t>(vec) * bytes_of(w_dtype)));
    for (int k = 0; k < n; ++k) fits = fits && rows_aligned(*all[k], vec);
    if (fits) return vec;
  }
  return 1;
}

}  // namespace

extern "C" {

int abs_rms_norm(const abs_rms_norm_args* a, abs_stream_t stream) {
  if (!a) return ABS_ERR_NULL;
  int rc = check_shape(a->n0, a->n1, a->h);
  if (rc != ABS_OK) return rc;
  if (!good_eps(a->eps)) return ABS_ERR_RANGE;
  if (a->n0 == 0 || a->n1 == 0) return ABS_OK;
  Rows x, r, sum, out;
  if ((rc = take_rows(a->x, a->n0, a->n1, a->h, x)) != ABS_OK) return rc;
  if ((rc = take_rows(a->residual, a->n0, a->n1, a->h, r)) != ABS_OK) return rc;
  if ((rc = take_rows(a->sum, a->n0, a->n1, a->h, sum)) != ABS_OK) return rc;
  if ((rc = take_rows(a->out, a->n0, a->n1, a->h, out)) != ABS_OK) return rc;
  if (!x.given() || !out.given() || (sum.given() && !r.given())) return ABS_ERR_NULL;
  if (!wide_float(x.dtype) || (r.given() && r.dtype != x.dtype && r.dtype != ABS_F32) ||
      (sum.given() && sum.dtype != r.dtype) || out.dtype == ABS_E8M0)
    return ABS_ERR_DTYPE;
  if ((rc = check_weight(a->weight, a->weight_dtype)) != ABS_OK) return rc;

  const bool eight = out.dtype == ABS_E4M3 || out.dtype == ABS_E5M2;
  const int64_t group = a->group > 0 ? a->group : a->h;
  Rows scales{};
  if (eight) {
    if (a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128) return ABS_ERR_RANGE;
    if (!a->scales.data) return ABS_ERR_NULL;
    if (a->scales.dtype != ABS_F32 && a->scales.dtype != ABS_E8M0) return ABS_ERR_DTYPE;
    // a matrix of (n0 n1) x groups for the checks, its three strides kept apart for the kernel
    const int64_t groups = (a->h + group - 1) / group;
    const int64_t s2 = groups > 1 ? a->scale_stride2 : 0;
    if (s2 < 0 || s2 > kMostElements || static_cast<__int128>(groups - 1) * s2 > kMostElements) return ABS_ERR_RANGE;
    if ((rc = take_rows(a->scales, a->n0, a->n1, (groups - 1) * s2 + 1, scales)) != ABS_OK) return rc;
    if (groups > 1 && s2 == 0) return ABS_ERR_ALIAS;
  } else if (a->scales.data || a->group != 0) {
    return ABS_ERR_RANGE;
  }

  // outputs: rows apart from one another, from other outputs and the weight; from an input unless they are
  // that input, element by element
  const Rows* const outs[] = {&out, &sum, &scales};
  for (int i = 0; i < 3; ++i) {
    const Rows& o = *outs[i];
    if (!o.given()) continue;
    // (the scales of a row may lie apart, so that rows interleave: a transposed matrix of scales)
    if (i < 2 && !separate_rows(o)) return ABS_ERR_ALIAS;
    for (int j = 0; j < i; ++j)
      if (outs[j]->given() && rows_touch(o, *outs[j])) return ABS_ERR_ALIAS;
    if (a->weight && overlaps(o.p, o.bytes(), a->weight, a->h * bytes_of(a->weight_dtype))) return ABS_ERR_ALIAS;
    for (const Rows* in : {&x, &r})
      if (in->given() && !(i < 2 && same_rows(o, *in)) && rows_touch(o, *in)) return ABS_ERR_ALIAS;
  }
  if (eight) {  // no two scales at one place: the strides of the dimensions that have more than one, in order
    const int64_t groups = (a->h + group - 1) / group;
    int64_t n[3] = {a->n0, a->n1, groups};
    int64_t s[3] = {scales.s0, scales.s1, groups > 1 ? a->scale_stride2 * scales.esz : 0};
    int64_t reach = scales.esz;  // bytes that the dimensions so far span
    for (int round = 0; round < 3; ++round) {
      int k = -1;
      for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (k < 0 || s[i] < s[k])) k = i;
      if (k < 0) break;
      if (s[k] < reach) return ABS_ERR_ALIAS;
      reach += (n[k] - 1) * s[k];
      n[k] = 1;
    }
  }

  NormParams p = {};
  const Rows* const all[] = {&x, &r, &sum, &out};
  const int vec = vector_width(a->h, a->weight, a->weight_dtype, all, 4);
  p.x = x.arg(vec);
  p.r = r.arg(vec);
  p.sum = sum.arg(vec);
  p.out = out.arg(vec);
  if (eight) {
    p.scales = const_cast<unsigned char*>(scales.p);
    p.scale_s0 = scales.s0 / scales.esz;
    p.scale_s1 = scales.s1 / scales.esz;
    p.scale_s2 = a->scale_stride2;
  }
  p.w = static_cast<const unsigned char*>(a->weight);
  p.rows = static_cast<uint32_t>(a->n0 * a->n1);
  p.n1 = divisor(static_cast<uint32_t>(a->n1));
  for (int g = static_cast<int>(group); g > 1; g >>= 1) ++p.group_shift;
  p.h = static_cast<int>(a->h);
  p.group = static_cast<int>(group);
  p.w_dtype = a->weight_dtype;
  p.out_dtype = out.dtype;
  p.scale_dtype = scales.dtype;
  p.inv_h = static_cast<float>(1.0 / static_cast<double>(a->h));
  p.eps = static_cast<float>(a->eps);
  const int r_dtype = r.given() ? r.dtype : -1;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (x.dtype == ABS_F32) e = launch_norm<ABS_F32>(p, r_dtype, vec, st);
  else if (x.dtype == ABS_BF16) e = launch_norm<ABS_BF16>(p, r_dtype, vec, st);
  else e = launch_norm<ABS_F16>(p, r_dtype, vec, st);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

size_t abs_rms_norm_grad_bytes(int64_t n0, int64_t n1, int64_t h, int64_t n_samples) {
  if (check_shape(n0, n1, h) != ABS_OK || n_samples < 0 || n_samples > ABS_MAX_SAMPLES) return 0;
  int64_t blocks = 0;  // the most that a call may take: its tensors' alignment decides; at most one for each row
  for (int vec : {8, 4, 1}) blocks = std::max(blocks, std::min(n0 * n1, grad_most_blocks(h, vec)));
  // one record a block, and with a table one for each sample and one more for each block
  return static_cast<size_t>(blocks + (n_samples ? blocks + n_samples : 0) + 1) * record_pitch(h) * sizeof(float);
}

int abs_rms_norm_grad(const abs_rms_norm_grad_args* a, abs_stream_t stream) {
  if (!a) return ABS_ERR_NULL;
  int rc = check_shape(a->n0, a->n1, a->h);
  if (rc != ABS_OK) return rc;
  if (!good_eps(a->eps) || !(std::fabs(a->sample_scale) <= 1e30)) return ABS_ERR_RANGE;
  if (a->n_samples < 0 || a->n_samples > ABS_MAX_SAMPLES) return ABS_ERR_RANGE;
  if ((a->n_samples > 0) != (a->offsets != nullptr)) return ABS_ERR_NULL;
  if (a->dweight_samples && !a->offsets) return ABS_ERR_NULL;
  const bool sums = a->dweight || a->dweight_samples;
  const bool empty = a->n0 == 0 || a->n1 == 0;
  const int64_t n0 = empty ? 1 : a->n0, n1 = empty ? 1 : a->n1;
  Rows dy, s, add, dx;
  if ((rc = take_rows(a->dy, n0, n1, a->h, dy)) != ABS_OK) return rc;
  if ((rc = take_rows(a->s, n0, n1, a->h, s)) != ABS_OK) return rc;
  if ((rc = take_rows(a->dresidual, n0, n1, a->h, add)) != ABS_OK) return rc;
  if ((rc = take_rows(a->dx, n0, n1, a->h, dx)) != ABS_OK) return rc;
  if (!empty && (!dy.given() || !s.given() || !dx.given())) return ABS_ERR_NULL;
  if (!empty && (!wide_float(dy.dtype) || (s.dtype != dy.dtype && s.dtype != ABS_F32) ||
                 (add.given() && add.dtype != s.dtype) || !wide_float(dx.dtype)))
    return ABS_ERR_DTYPE;
  if ((rc = check_weight(a->weight, a->weight_dtype)) != ABS_OK) return rc;
  if (a->offsets && misaligned(a->offsets, 4)) return ABS_ERR_ALIGN;
  if (misaligned(a->dweight, 4) || misaligned(a->dweight_samples, 4)) return ABS_ERR_ALIGN;
  const size_t need = abs_rms_norm_grad_bytes(a->n0, a->n1, a->h, a->n_samples);
  if (sums && !empty) {
    if (!a->work) return ABS_ERR_NULL;
    if (misaligned(a->work, 32)) return ABS_ERR_ALIGN;
    if (a->work_bytes < 0 || static_cast<size_t>(a->work_bytes) < need) return ABS_ERR_TOO_LARGE;
  }
  if (a->dweight_samples && (a->n_samples > 1 ? a->samples_ld : a->h) < a->h) return ABS_ERR_RANGE;
  if (a->dweight_samples && a->samples_ld > kMostElements / (a->n_samples + 1)) return ABS_ERR_RANGE;

  // dx may be dy, s or dresidual, element by element; nothing else may share a byte with an output
  struct { const void* p; size_t n; } flat[] = {
      {a->dweight, static_cast<size_t>(a->h) * 4},
      {a->dweight_samples, static_cast<size_t>((a->n_samples - 1) * a->samples_ld + a->h) * 4},
      {sums && !empty ? a->work : nullptr, need},
      {a->weight, static_cast<size_t>(a->h) * bytes_of(a->weight_dtype)},
      {a->offsets, static_cast<size_t>(a->n_samples + 1) * 4}};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (j < 3 && flat[i].p && flat[j].p && overlaps(flat[i].p, flat[i].n, flat[j].p, flat[j].n)) return ABS_ERR_ALIAS;
  if (!empty) {
    if (!separate_rows(dx)) return ABS_ERR_ALIAS;
    for (const Rows* in : {&dy, &s, &add})
      if (in->given() && !same_rows(dx, *in) && rows_touch(dx, *in)) return ABS_ERR_ALIAS;
    for (int i = 0; i < 5; ++i) {
      if (!flat[i].p) continue;
      if (overlaps(flat[i].p, flat[i].n, dx.p, dx.bytes())) return ABS_ERR_ALIAS;
      if (i < 3)
        for (const Rows* in : {&dy, &s, &add})
          if (in->given() && overlaps(flat[i].p, flat[i].n, in->p, in->bytes())) return ABS_ERR_ALIAS;
    }
  }

  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  NormGradParams p = {};
  p.rows = empty ? 0 : static_cast<uint32_t>(n0 * n1);
  p.n1 = divisor(static_cast<uint32_t>(n1));
  p.h = static_cast<int>(a->h);
  p.offsets = a->offsets;
  p.n_samples = static_cast<int>(a->n_samples);
  p.pitch = record_pitch(a->h);
  int64_t blocks = 0;
  float* const work = static_cast<float*>(a->work);
  if (!empty) {
    const Rows* const all[] = {&dy, &s, &add, &dx};
    const int vec = vector_width(a->h, a->weight, a->weight_dtype, all, 4);
    blocks = grad_blocks(p.rows, a->h, vec);
    p.dy = dy.arg(vec);
    p.s = s.arg(vec);
    p.add = add.arg(vec);
    p.dx = dx.arg(vec);
    p.w = static_cast<const unsigned char*>(a->weight);
    p.w_dtype = a->weight_dtype;
    p.dx_dtype = dx.dtype;
    if (a->dweight) p.totals = work;
    if (a->dweight_samples) p.pieces = work + blocks * p.pitch;
    p.inv_h = static_cast<float>(1.0 / static_cast<double>(a->h));
    p.eps = static_cast<float>(a->eps);
    cudaError_t e;
    if (dy.dtype == ABS_F32) e = launch_norm_grad<ABS_F32>(p, s.dtype, blocks, vec, st);
    else if (dy.dtype == ABS_BF16) e = launch_norm_grad<ABS_BF16>(p, s.dtype, blocks, vec, st);
    else e = launch_norm_grad<ABS_F16>(p, s.dtype, blocks, vec, st);
    if (e != cudaSuccess) return cuda_fail(e);
  }
  if (!sums) return ABS_OK;
  NormMergeParams m = {};
  m.totals = p.totals;
  m.pieces = p.pieces;
  m.pitch = p.pitch;
  m.offsets = a->offsets;
  m.dw = a->dweight;
  m.dw_samples = a->dweight_samples;
  m.ld = a->samples_ld;
  m.rows = p.rows;
  m.n1 = p.n1.d;
  m.n_samples = p.n_samples;
  m.h = p.h;
  m.blocks = static_cast<int>(blocks);
  m.n_out = a->dweight_samples ? p.n_samples : 0;
  // 2048 x 2048 with 8 samples: 17.4 us with 128 columns, 18.3 with 32; 2048 x 4096 28.7 and 30.3
  m.col_bits = m.n_out > 0 && blocks / m.n_out < 128 ? 7 : 5;
  m.sample_blocks = ((p.h - 1) >> m.col_bits) + 1;
  m.scale = static_cast<float>(a->sample_scale);
  const int64_t grid = static_cast<int64_t>(m.n_out) * m.sample_blocks + (a->dweight ? ((p.h - 1) >> kTotalsBits) + 1 : 0);
  const cudaError_t e = launch_pdl(rms_norm_merge_kernel, dim3(static_cast<unsigned>(grid)), dim3(kMergeThreads), st, m);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

}  // extern "C"
