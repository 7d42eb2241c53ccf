// C ABI of the calls over a list of tensors: the plan of a list (host), its upload, and the norm,
// clipping and AdamW calls.
#include <algorithm>
#include <cstring>
#include <vector>

#include "host_checks.cuh"
#include "launch.cuh"
#include "tensors.cuh"

using namespace absnt;

namespace {

constexpr uint64_t kPlanMagic = 0x6e616c7054534241ull;  // "ABSTplan"
constexpr int64_t kMaxRow = int64_t{1} << 30;
constexpr int64_t kMaxElements = int64_t{1} << 46;
enum { kRoleOut = 1, kRoleAdam = 2, kRoleBf16 = 4, kGradsOverlap = 8 };

// Host image of a plan: this header, the table of tensors, the tensor of each unit.
struct PlanHeader {
  uint64_t magic;
  int32_t n, n_units, n_nonempty, unit, roles, n_groups;
};
TensorEntry* entries_of(void* plan) {
  return reinterpret_cast<TensorEntry*>(static_cast<char*>(plan) + sizeof(PlanHeader));
}
size_t image_bytes(int64_t n, int64_t n_units) {
  return static_cast<size_t>(n) * sizeof(TensorEntry) + static_cast<size_t>(n_units) * 4;
}

// Device work area: header, sums of tensors and units, tickets, then the image of the plan.
struct WorkLayout {
  size_t tensor_sum, unit_sum, tickets, image, bytes;
  WorkLayout(int64_t n, int64_t n_units) {
    tensor_sum = sizeof(double) * ABS_STATS_HEADER;
    unit_sum = tensor_sum + sizeof(double) * static_cast<size_t>(n);
    tickets = unit_sum + sizeof(double) * static_cast<size_t>(n_units);
    image = (tickets + 4 * (static_cast<size_t>(n) + 1) + 15) / 16 * 16;
    bytes = image + image_bytes(n, n_units);
  }
};

// Elements per unit: a power of two that gives about eight units to each of the 148 SMs, between
// 1024 (a quarter of a vector per thread, so that small lists spread over the SMs) and 32768.  A
// function of the element count alone, and with it the shape of every sum.
int unit_for(int64_t total) {
  int unit = 1024;
  while (unit < 32768 && total / unit > 8 * 148) unit *= 2;
  return unit;
}

size_t element_size(int dtype) { return dtype == ABS_F32 ? 4 : 2; }
bool known_dtype(int dtype) { return dtype == ABS_F32 || dtype == ABS_BF16 || dtype == ABS_F16; }

// A tensor with its rows normalised: contiguous tensors have row = stride = numel, col = 1.
struct View {
  const void* data;
  int64_t numel, row, stride, col;
  size_t esz;
  bool rows() const { return row != numel || col != 1; }
  size_t extent() const {  // bytes from the first element to the end of the last
    return numel ? (static_cast<size_t>(numel / row - 1) * stride +
                    static_cast<size_t>(row - 1) * col + 1) * esz
                 : 0;
  }
};

int view_of(const abs_tensor& t, View* v) {
  if (!known_dtype(t.dtype)) return ABS_ERR_DTYPE;
  if (t.numel < 0 || t.numel > kMaxElements) return ABS_ERR_RANGE;
  v->data = t.data;
  v->numel = v->row = v->stride = t.numel;
  v->col = 1;
  v->esz = element_size(t.dtype);
  if (t.numel == 0) return ABS_OK;
  if (!t.data) return ABS_ERR_NULL;
  if (misaligned(t.data, v->esz)) return ABS_ERR_ALIGN;
  if (!t.row_len) return ABS_OK;
  if (t.row_len < 1 || t.numel % t.row_len) return ABS_ERR_RANGE;
  const int64_t n_rows = t.numel / t.row_len;
  if (t.row_stride < 1 || t.col_stride < 1 || t.row_stride > kMaxElements / n_rows ||
      t.col_stride > kMaxElements / t.row_len)
    return ABS_ERR_RANGE;
  // one of the two strides steps over all that the other one reaches: no place is taken twice
  if (t.row_stride <= (t.row_len - 1) * t.col_stride && t.col_stride <= (n_rows - 1) * t.row_stride)
    return ABS_ERR_RANGE;
  if (t.col_stride == 1 && (t.row_stride == t.row_len || n_rows == 1)) return ABS_OK;  // no gap
  if (t.row_len > kMaxRow) return ABS_ERR_RANGE;
  v->row = t.row_len;
  v->stride = t.row_stride;
  v->col = t.col_stride;
  return ABS_OK;
}

// i / d = (i * magic) >> (31 + shift) for 0 <= i < 2^31, 1 <= d <= 2^30: with 2^shift >= d the
// excess of magic / 2^(31+shift) over 1/d is at most 2^-(31+shift), less than 1/(d i).
void divisor(uint32_t d, uint32_t* magic, uint8_t* shift) {
  int s = 0;
  while ((uint64_t{1} << s) < d) ++s;
  *magic = static_cast<uint32_t>(((uint64_t{1} << (31 + s)) + d - 1) / d);
  *shift = static_cast<uint8_t>(s);
}

// Whether elements [head, ...) of a view can be taken in groups of `vec`, each aligned.
bool vector_ok(const View& v, int head, int vec) {
  if (v.rows() && (head || v.col != 1 || v.row % vec || v.stride % vec)) return false;
  return (reinterpret_cast<uintptr_t>(v.data) + head * v.esz) % (vec * v.esz) == 0;
}

// Two views share an element.  Rows of the same stride that interleave do not.
bool views_overlap(const View& a, const View& b) {
  if (!overlaps(a.data, a.extent(), b.data, b.extent())) return false;
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.data), pb = reinterpret_cast<uintptr_t>(b.data);
  const View &lo = pa <= pb ? a : b, &hi = pa <= pb ? b : a;
  const size_t s = static_cast<size_t>(lo.stride) * lo.esz;
  if (lo.rows() && hi.rows() && lo.col == 1 && hi.col == 1 && s == static_cast<size_t>(hi.stride) * hi.esz) {
    const size_t phase = (pa <= pb ? pb - pa : pa - pb) % s;
    if (phase >= lo.row * lo.esz && phase + hi.row * hi.esz <= s) return false;
  }
  return true;
}

// Any pair of views of which at least one is written (`written`) that shares an element; pairs of
// read-only views may.  Sorted by address, so that only neighbours are compared.
bool any_conflict(std::vector<std::pair<View, bool>>& list) {
  std::sort(list.begin(), list.end(),
            [](const auto& a, const auto& b) { return a.first.data < b.first.data; });
  for (size_t i = 0; i < list.size(); ++i) {
    const View& a = list[i].first;
    const uintptr_t end = reinterpret_cast<uintptr_t>(a.data) + a.extent();
    for (size_t j = i + 1; j < list.size(); ++j) {
      if (reinterpret_cast<uintptr_t>(list[j].first.data) >= end) break;
      if ((list[i].second || list[j].second) && views_overlap(a, list[j].first)) return true;
    }
  }
  return false;
}

const PlanHeader* plan_of(const void* plan) {
  if (!plan || misaligned(plan, 8)) return nullptr;
  const PlanHeader* h = static_cast<const PlanHeader*>(plan);
  return h->magic == kPlanMagic ? h : nullptr;
}

int fill_params(const void* plan, void* work, int norm_type, double scale, double max_norm,
                const double* sum_in, float* norms_out, TensorsParams* prm) {
  if (!plan || !work) return ABS_ERR_NULL;
  const PlanHeader* h = plan_of(plan);
  if (!h) return ABS_ERR_RANGE;
  if (norm_type != ABS_NORM_2 && norm_type != ABS_NORM_1 && norm_type != ABS_NORM_MAX)
    return ABS_ERR_RANGE;
  if (!std::isfinite(scale) || scale == 0.0) return ABS_ERR_RANGE;
  if (!std::isfinite(max_norm) || max_norm < 0.0) return ABS_ERR_RANGE;
  if (misaligned(work, 16) || misaligned(norms_out, 4) || misaligned(sum_in, 8))
    return ABS_ERR_ALIGN;
  const WorkLayout L(h->n, h->n_units);
  char* w = static_cast<char*>(work);
  if (norms_out && overlaps(norms_out, 4 * (static_cast<size_t>(h->n) + 2), work, L.bytes)) return ABS_ERR_ALIAS;
  prm->header = reinterpret_cast<double*>(w);
  prm->tensor_sum = reinterpret_cast<double*>(w + L.tensor_sum);
  prm->unit_sum = reinterpret_cast<double*>(w + L.unit_sum);
  prm->tickets = reinterpret_cast<unsigned int*>(w + L.tickets);
  prm->entries = reinterpret_cast<const TensorEntry*>(w + L.image);
  prm->unit_tensor = reinterpret_cast<const int32_t*>(prm->entries + h->n);
  prm->norms_out = norms_out;
  prm->n = h->n;
  prm->n_units = h->n_units;
  prm->n_nonempty = h->n_nonempty;
  prm->unit = h->unit;
  prm->norm_type = norm_type;
  prm->scale = scale;
  prm->max_norm = max_norm;
  prm->sum_in = sum_in;
  prm->in_place = !(h->roles & kRoleOut);
  return ABS_OK;
}

dim3 unit_grid(const TensorsParams& prm) {
  return dim3(static_cast<unsigned>(prm.n_units > 0 ? prm.n_units : 1));
}

cudaError_t launch_norm(const TensorsParams& prm, cudaStream_t st) {
  const dim3 grid = unit_grid(prm), block(kTensorThreads);
  return prm.norm_type == ABS_NORM_2   ? launch_pdl(tensors_norm_kernel<kNorm2>, grid, block, st, prm)
         : prm.norm_type == ABS_NORM_1 ? launch_pdl(tensors_norm_kernel<kNorm1>, grid, block, st, prm)
                                       : launch_pdl(tensors_norm_kernel<kNormMax>, grid, block, st, prm);
}

// Everything of abs_tensors_plan that can run out of memory or throw.
int make_plan(const abs_tensor* grads, const abs_tensor* outs, const abs_tensor* params,
              const abs_tensor* m, const abs_tensor* v, const abs_tensor* params_bf16, int n,
              void* plan, size_t plan_bytes) {
  std::vector<std::pair<View, bool>> all;
  std::vector<std::pair<View, bool>> grads_written;
  PlanHeader h;
  std::memset(&h, 0, sizeof h);
  h.magic = kPlanMagic;
  h.n = n;
  h.roles = (outs ? kRoleOut : 0) | (params ? kRoleAdam : 0) | (params_bf16 ? kRoleBf16 : 0);
  int64_t total = 0;
  for (int t = 0; t < n; ++t) {
    View g;
    const int rc = view_of(grads[t], &g);
    if (rc != ABS_OK) return rc;
    if (grads[t].group < 0 || grads[t].group >= ABS_MAX_GROUPS) return ABS_ERR_RANGE;
    if (g.numel > kMaxElements - total) return ABS_ERR_RANGE;
    total += g.numel;
  }
  h.unit = unit_for(total);
  TensorEntry* entries = entries_of(plan);
  if (plan_bytes < sizeof(PlanHeader) + image_bytes(n, 0)) return ABS_ERR_TOO_LARGE;
  int64_t units = 0;
  for (int t = 0; t < n; ++t) {
    View g, out, state[3], b16;
    view_of(grads[t], &g);
    TensorEntry e;
    std::memset(&e, 0, sizeof e);
    e.g = g.data;
    e.numel = g.numel;
    e.g_dtype = static_cast<uint8_t>(grads[t].dtype);
    e.group = static_cast<uint16_t>(grads[t].group);
    if (grads[t].group + 1 > h.n_groups) h.n_groups = grads[t].group + 1;
    const bool rows_g = g.rows();
    if (rows_g) {
      e.flags |= kEntryRowsG;
      e.g_row = static_cast<uint32_t>(g.row);
      e.g_stride = g.stride;
      e.g_col = g.col;
      divisor(e.g_row, &e.g_magic, &e.g_shift);
    }
    if (outs) {
      const int rc = view_of(outs[t], &out);
      if (rc != ABS_OK) return rc;
      if (out.numel != g.numel) return ABS_ERR_RANGE;
      e.out = const_cast<void*>(out.data);
      e.out_dtype = static_cast<uint8_t>(outs[t].dtype);
      if (out.rows()) {
        e.flags |= kEntryRowsOut;
        e.out_row = static_cast<uint32_t>(out.row);
        e.out_stride = out.stride;
        e.out_col = out.col;
        divisor(e.out_row, &e.out_magic, &e.out_shift);
      }
      if (out.numel) all.push_back({out, true});
    }
    if (params) {
      const abs_tensor* roles[3] = {&params[t], &m[t], &v[t]};
      for (int i = 0; i < 3; ++i) {
        const int rc = view_of(*roles[i], &state[i]);
        if (rc != ABS_OK) return rc;
        if (roles[i]->dtype != ABS_F32) return ABS_ERR_DTYPE;
        if (state[i].numel != g.numel || state[i].rows()) return ABS_ERR_RANGE;
        if (g.numel) all.push_back({state[i], true});
      }
      e.p = static_cast<float*>(params[t].data);
      e.m = static_cast<float*>(m[t].data);
      e.v = static_cast<float*>(v[t].data);
      if (params_bf16) {
        const int rc = view_of(params_bf16[t], &b16);
        if (rc != ABS_OK) return rc;
        if (params_bf16[t].dtype != ABS_BF16) return ABS_ERR_DTYPE;
        if (b16.numel != g.numel || b16.rows()) return ABS_ERR_RANGE;
        if (g.numel) all.push_back({b16, true});
        e.p16 = static_cast<uint16_t*>(params_bf16[t].data);
      }
    }
    if (g.numel) {
      all.push_back({g, false});
      grads_written.push_back({g, true});
    }
    // the head that aligns most: the update's arrays before the output before the gradient alone
    int best = -1;
    for (int head = 0; head < 8; ++head) {
      int flags = 0;
      if (vector_ok(g, head, static_cast<int>(16 / g.esz))) flags |= kEntryVecG;
      const bool g8 = vector_ok(g, head, 8);
      if (g8 && (!outs || vector_ok(out, head, 8))) flags |= kEntryVecClip;
      if (params && g8 && vector_ok(state[0], head, 8) && vector_ok(state[1], head, 8) &&
          vector_ok(state[2], head, 8) && (!params_bf16 || vector_ok(b16, head, 8)))
        flags |= kEntryVecAdam;
      if (flags > best) {
        best = flags;
        e.head = static_cast<uint8_t>(flags ? head : 0);
      }
    }
    e.flags |= static_cast<uint8_t>(best);
    if (e.numel) {
      const int64_t body = e.numel > e.head ? e.numel - e.head : 1;
      const int64_t k = (body + h.unit - 1) / h.unit;
      if (units + k > (int64_t{1} << 30)) return ABS_ERR_RANGE;
      e.first_unit = static_cast<int32_t>(units);
      e.n_units = static_cast<int32_t>(k);
      units += k;
      ++h.n_nonempty;
    }
    entries[t] = e;
  }
  h.n_units = static_cast<int32_t>(units);
  if (plan_bytes < sizeof(PlanHeader) + image_bytes(n, units)) return ABS_ERR_TOO_LARGE;
  if (any_conflict(all)) return ABS_ERR_ALIAS;
  if (any_conflict(grads_written)) h.roles |= kGradsOverlap;
  int32_t* unit_tensor = reinterpret_cast<int32_t*>(entries + n);
  for (int t = 0; t < n; ++t)
    for (int k = 0; k < entries[t].n_units; ++k) unit_tensor[entries[t].first_unit + k] = t;
  std::memcpy(plan, &h, sizeof h);
  return ABS_OK;
}

}  // namespace

extern "C" {

size_t abs_tensors_plan_bytes(const abs_tensor* grads, int n) {
  if (n < 0 || (n > 0 && !grads)) return 0;
  int64_t total = 0, units = 0;
  for (int t = 0; t < n; ++t) {
    if (grads[t].numel < 0 || grads[t].numel > kMaxElements - total) return 0;
    total += grads[t].numel;
  }
  const int unit = unit_for(total);
  for (int t = 0; t < n; ++t) units += (grads[t].numel + unit - 1) / unit;
  return sizeof(PlanHeader) + image_bytes(n, units);
}

int abs_tensors_plan(const abs_tensor* grads, const abs_tensor* outs, const abs_tensor* params,
                     const abs_tensor* m, const abs_tensor* v, const abs_tensor* params_bf16, int n,
                     void* plan, size_t plan_bytes) {
  if (!plan) return ABS_ERR_NULL;
  if (n < 0 || n > ABS_MAX_TENSORS) return ABS_ERR_RANGE;
  if (n > 0 && !grads) return ABS_ERR_NULL;
  if (n > 0 && (params || m || v || params_bf16) && !(params && m && v)) return ABS_ERR_NULL;
  if (misaligned(plan, 8)) return ABS_ERR_ALIGN;
  if (plan_bytes >= sizeof(PlanHeader)) static_cast<PlanHeader*>(plan)->magic = 0;  // not yet one
  try {
    return make_plan(grads, outs, params, m, v, params_bf16, n, plan, plan_bytes);
  } catch (...) {  // the host is out of memory for the check of overlaps
    return ABS_ERR_TOO_LARGE;
  }
}

size_t abs_tensors_work_bytes(const void* plan) {
  const PlanHeader* h = plan_of(plan);
  return h ? WorkLayout(h->n, h->n_units).bytes : 0;
}

int abs_tensors_upload(const void* plan, void* work, abs_stream_t stream) {
  if (!plan || !work) return ABS_ERR_NULL;
  const PlanHeader* h = plan_of(plan);
  if (!h) return ABS_ERR_RANGE;
  if (misaligned(work, 16)) return ABS_ERR_ALIGN;
  const WorkLayout L(h->n, h->n_units);
  char* w = static_cast<char*>(work);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemsetAsync(w, 0, L.image, st);
  if (e == cudaSuccess && L.bytes > L.image)
    e = cudaMemcpyAsync(w + L.image, static_cast<const char*>(plan) + sizeof(PlanHeader),
                        L.bytes - L.image, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

int abs_grad_norm(const void* plan, void* work, int norm_type, double grad_scale, double max_norm,
                  float* norms_out, abs_stream_t stream) {
  TensorsParams prm;
  const int rc = fill_params(plan, work, norm_type, grad_scale, max_norm, nullptr, norms_out, &prm);
  if (rc != ABS_OK) return rc;
  if (!norms_out) return ABS_ERR_NULL;
  const cudaError_t e = launch_norm(prm, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

int abs_grad_clip(const void* plan, void* work, int norm_type, double grad_scale, double max_norm,
                  const double* sum_in, float* norms_out, abs_stream_t stream) {
  TensorsParams prm;
  const int rc = fill_params(plan, work, norm_type, grad_scale, max_norm, sum_in, norms_out, &prm);
  if (rc != ABS_OK) return rc;
  if (!norms_out) return ABS_ERR_NULL;
  if (!(max_norm > 0.0)) return ABS_ERR_RANGE;
  if (prm.in_place && (plan_of(plan)->roles & kGradsOverlap)) return ABS_ERR_ALIAS;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = sum_in ? cudaSuccess : launch_norm(prm, st);
  if (e == cudaSuccess && (prm.n_units > 0 || sum_in))
    e = launch_pdl(tensors_scale_kernel, unit_grid(prm), dim3(kTensorThreads), st, prm);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

int abs_grad_adamw(const void* plan, void* work, const abs_adamw_hparams* hparams, int n_groups,
                   int64_t step, int norm_type, double grad_scale, double max_norm,
                   const double* sum_in, float* norms_out, abs_stream_t stream) {
  TensorsParams prm;
  const int rc = fill_params(plan, work, norm_type, grad_scale, max_norm, sum_in, norms_out, &prm);
  if (rc != ABS_OK) return rc;
  const bool clipped = max_norm > 0.0;
  const PlanHeader* h = plan_of(plan);
  if (!(h->roles & kRoleAdam) && h->n > 0) return ABS_ERR_NULL;
  if (!hparams || (clipped && !norms_out)) return ABS_ERR_NULL;
  if (n_groups < 1 || n_groups > ABS_MAX_GROUPS || n_groups < h->n_groups) return ABS_ERR_RANGE;
  GroupScalars groups;
  std::memset(&groups, 0, sizeof groups);
  for (int i = 0; i < n_groups; ++i) {
    const int rch = check_hparams(hparams + i, step);
    if (rch != ABS_OK) return rch;
    groups.a[i] = make_adam(hparams + i, step);
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = clipped && !sum_in ? launch_norm(prm, st) : cudaSuccess;
  if (e == cudaSuccess && (prm.n_units > 0 || (clipped && sum_in)))
    e = launch_pdl(tensors_adamw_kernel, unit_grid(prm), dim3(kTensorThreads), st, prm, groups,
                   clipped ? 1 : 0);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

}  // extern "C"
