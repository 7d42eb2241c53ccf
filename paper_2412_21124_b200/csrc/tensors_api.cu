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
constexpr int64_t kMaxUnits = int64_t{1} << 30;
enum { kRoleOut = 1, kRoleAdam = 2, kRoleBf16 = 4, kGradsOverlap = 8 };

// Host image of a plan: this header, then the tables in the order of `Image`.
struct PlanHeader {
  uint64_t magic;
  int32_t n, n_units, n_segments, n_warps, n_spanning, n_empty, unit, roles, n_groups, pad;
};
// Offsets of the tables in the image (which the device holds as well).
struct Image {
  size_t segments, spanning, warp_first, unit_tensor, empty, bytes;
  explicit Image(const PlanHeader& h) {
    segments = static_cast<size_t>(h.n) * sizeof(TensorEntry);
    spanning = segments + static_cast<size_t>(h.n_segments) * sizeof(Segment);
    warp_first = spanning + static_cast<size_t>(h.n_spanning) * sizeof(Spanning);
    unit_tensor = warp_first + 4 * (static_cast<size_t>(h.n_warps) + 1);
    empty = unit_tensor + 4 * static_cast<size_t>(h.n_units);
    bytes = empty + 4 * static_cast<size_t>(h.n_empty);
  }
};
char* image_of(void* plan) { return static_cast<char*>(plan) + sizeof(PlanHeader); }

// Device work area: header, sums and edge sums of the blocks, the ticket, then the image of the plan.
struct WorkLayout {
  size_t block_sum, edge_sum, ticket, image, bytes;
  explicit WorkLayout(const PlanHeader& h) {
    block_sum = sizeof(double) * ABS_STATS_HEADER;
    edge_sum = block_sum + sizeof(double) * kNormCtas;
    ticket = edge_sum + sizeof(double) * 2 * kNormCtas;
    image = (ticket + 4 + 15) / 16 * 16;
    bytes = image + Image(h).bytes;
  }
};

// How the bytes of a list are shared out: `rows` rows of 512 bytes (32 lanes of 16 bytes) to each of
// `warps` warps, at most as many as fill the device.
constexpr int64_t kRowBytes = 512;
struct Share {
  int64_t rows;
  int64_t warps;
};
Share share_of(int64_t total_rows) {
  const int64_t most = static_cast<int64_t>(kNormCtas) * kNormWarps;
  Share s;
  s.rows = std::max<int64_t>(1, (total_rows + most - 1) / most);
  s.warps = (total_rows + s.rows - 1) / s.rows;
  return s;
}
// Rows of a tensor, the last one short.
int64_t rows_of(int64_t numel, size_t esz) {
  return (numel * static_cast<int64_t>(esz) + kRowBytes - 1) / kRowBytes;
}
// A segment is counted in 32 bits; longer runs of one warp are cut.
constexpr int64_t kMaxSegmentRows = int64_t{1} << 20;

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
  const WorkLayout L(*h);
  char* w = static_cast<char*>(work);
  if (norms_out && overlaps(norms_out, 4 * (static_cast<size_t>(h->n) + 2), work, L.bytes)) return ABS_ERR_ALIAS;
  prm->header = reinterpret_cast<double*>(w);
  prm->block_sum = reinterpret_cast<double*>(w + L.block_sum);
  prm->edge_sum = reinterpret_cast<double*>(w + L.edge_sum);
  prm->ticket = reinterpret_cast<unsigned int*>(w + L.ticket);
  const Image I(*h);
  w += L.image;
  prm->entries = reinterpret_cast<const TensorEntry*>(w);
  prm->segments = reinterpret_cast<const Segment*>(w + I.segments);
  prm->spanning = reinterpret_cast<const Spanning*>(w + I.spanning);
  prm->empty = reinterpret_cast<const int32_t*>(w + I.empty);
  prm->warp_first = reinterpret_cast<const int32_t*>(w + I.warp_first);
  prm->unit_tensor = reinterpret_cast<const int32_t*>(w + I.unit_tensor);
  prm->norms_out = norms_out;
  prm->n = h->n;
  prm->n_units = h->n_units;
  prm->unit = h->unit;
  prm->n_segments = h->n_segments;
  prm->n_warps = h->n_warps;
  prm->n_spanning = h->n_spanning;
  prm->n_empty = h->n_empty;
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
  const dim3 grid(std::max(1, (prm.n_warps + kNormWarps - 1) / kNormWarps)), block(kNormThreads);
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
  int64_t total = 0, total_rows = 0;
  for (int t = 0; t < n; ++t) {
    View g;
    const int rc = view_of(grads[t], &g);
    if (rc != ABS_OK) return rc;
    if (grads[t].group < 0 || grads[t].group >= ABS_MAX_GROUPS) return ABS_ERR_RANGE;
    if (g.numel > kMaxElements - total) return ABS_ERR_RANGE;
    total += g.numel;
    total_rows += rows_of(g.numel, g.esz);
  }
  h.unit = unit_for(total);
  std::vector<TensorEntry> entries(n);
  std::vector<int32_t> unit_tensor;
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
      if (k > kMaxUnits - static_cast<int64_t>(unit_tensor.size())) return ABS_ERR_RANGE;
      e.first_unit = static_cast<int32_t>(unit_tensor.size());
      e.n_units = static_cast<int32_t>(k);
      unit_tensor.insert(unit_tensor.end(), static_cast<size_t>(k), t);
    }
    entries[t] = e;
  }
  if (any_conflict(all)) return ABS_ERR_ALIAS;
  if (any_conflict(grads_written)) h.roles |= kGradsOverlap;

  // the segments: the rows of all tensors in order, dealt out to the warps
  const Share share = share_of(total_rows);
  std::vector<Segment> segments;
  std::vector<int32_t> warp_first;
  int64_t left = 0;  // rows that the current warp still takes
  for (int t = 0; t < n; ++t) {
    TensorEntry& e = entries[t];
    const size_t esz = element_size(e.g_dtype);
    const int64_t per_row = kRowBytes / static_cast<int64_t>(esz);
    const int head = (e.flags & kEntryVecG) ? e.head : 0;
    int64_t rows = rows_of(e.numel, esz), start = 0;
    e.first_seg = static_cast<int32_t>(segments.size());
    while (rows > 0) {
      if (left == 0) {
        warp_first.push_back(static_cast<int32_t>(segments.size()));
        left = share.rows;
      }
      const int64_t take = std::min(std::min(rows, left), kMaxSegmentRows);
      rows -= take;
      left -= take;
      // every segment but the last ends on a 16-byte boundary: `head` elements further
      const int64_t end = rows ? start + take * per_row + (start ? 0 : head) : e.numel;
      Segment s;
      std::memset(&s, 0, sizeof s);
      s.start = start;
      s.n = static_cast<uint32_t>(std::min(end, e.numel) - start);
      s.g = static_cast<const char*>(e.g) + (e.flags & kEntryRowsG ? 0 : start * esz);
      s.tensor = t;
      s.dtype = e.g_dtype;
      s.rows = (e.flags & kEntryRowsG) ? 1 : 0;
      s.vec = (e.flags & kEntryVecG) && !s.rows;
      s.head = static_cast<uint8_t>(start ? 0 : std::min<int64_t>(head, s.n));
      start += s.n;
      segments.push_back(s);
      if (start == e.numel) {  // the head has taken the last, short row
        left += rows;
        rows = 0;
      }
    }
    e.n_segs = static_cast<int32_t>(segments.size()) - e.first_seg;
  }
  // the tensors that blocks (kNormWarps warps each) share
  std::vector<Spanning> spanning;
  std::vector<int32_t> empty;
  const auto block_of = [&](int32_t segment) {  // the warps' first segments ascend
    const auto it = std::upper_bound(warp_first.begin(), warp_first.end(), segment);
    return static_cast<int32_t>((it - warp_first.begin() - 1) / kNormWarps);
  };
  for (int t = 0; t < n; ++t) {
    const TensorEntry& e = entries[t];
    if (!e.n_segs) {
      empty.push_back(t);
      continue;
    }
    const int32_t a = block_of(e.first_seg), b = block_of(e.first_seg + e.n_segs - 1);
    if (a != b) spanning.push_back({t, a, b, 0});
  }
  h.n_spanning = static_cast<int32_t>(spanning.size());
  h.n_empty = static_cast<int32_t>(empty.size());
  h.n_warps = static_cast<int32_t>(warp_first.size());
  h.n_segments = static_cast<int32_t>(segments.size());
  h.n_units = static_cast<int32_t>(unit_tensor.size());
  warp_first.push_back(h.n_segments);

  const Image I(h);
  if (plan_bytes < sizeof(PlanHeader) + I.bytes) return ABS_ERR_TOO_LARGE;
  char* image = image_of(plan);
  const auto put = [](char* to, const void* from, size_t bytes) {
    if (bytes) std::memcpy(to, from, bytes);
  };
  put(image, entries.data(), entries.size() * sizeof(TensorEntry));
  put(image + I.segments, segments.data(), segments.size() * sizeof(Segment));
  put(image + I.warp_first, warp_first.data(), warp_first.size() * 4);
  put(image + I.spanning, spanning.data(), spanning.size() * sizeof(Spanning));
  put(image + I.empty, empty.data(), empty.size() * 4);
  put(image + I.unit_tensor, unit_tensor.data(), unit_tensor.size() * 4);
  std::memcpy(plan, &h, sizeof h);
  return ABS_OK;
}

}  // namespace

extern "C" {

size_t abs_tensors_plan_bytes(const abs_tensor* grads, int n) {
  if (n < 0 || n > ABS_MAX_TENSORS || (n > 0 && !grads)) return 0;
  int64_t total = 0, rows = 0, units = 0, segments = 0;
  for (int t = 0; t < n; ++t) {
    if (grads[t].numel < 0 || grads[t].numel > kMaxElements - total) return 0;
    total += grads[t].numel;
    rows += rows_of(grads[t].numel, element_size(grads[t].dtype));
  }
  // upper bounds: a tensor has a segment of its own and one more for each warp that begins in it
  const int unit = unit_for(total);
  const Share share = share_of(rows);
  for (int t = 0; t < n; ++t) {
    const int64_t r = rows_of(grads[t].numel, element_size(grads[t].dtype));
    units += (grads[t].numel + unit - 1) / unit;
    segments += r ? 1 + r / share.rows + r / kMaxSegmentRows + 1 : 0;
  }
  if (units > kMaxUnits || segments > kMaxUnits) return 0;
  PlanHeader h;
  std::memset(&h, 0, sizeof h);
  h.n = h.n_empty = n;
  h.n_units = static_cast<int32_t>(units);
  h.n_segments = static_cast<int32_t>(segments);
  h.n_warps = static_cast<int32_t>(share.warps);
  h.n_spanning = std::min(n, kNormCtas);
  return sizeof h + Image(h).bytes;
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
  return h ? WorkLayout(*h).bytes : 0;
}

int abs_tensors_upload(const void* plan, void* work, abs_stream_t stream) {
  if (!plan || !work) return ABS_ERR_NULL;
  const PlanHeader* h = plan_of(plan);
  if (!h) return ABS_ERR_RANGE;
  if (misaligned(work, 16)) return ABS_ERR_ALIGN;
  const WorkLayout L(*h);
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
