// C ABI of the calls over a list of tensors: the plan of a list (host), its upload, and the norm,
// clipping and AdamW calls.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cstring>
#include <mutex>
#include <numeric>
#include <vector>

#include "host_checks.cuh"
#include "launch.cuh"
#include "tensors.cuh"

using namespace absnt;

namespace {

constexpr uint64_t kPlanMagic = 0x6e616c7054534241ull;  // "ABSTplan"
constexpr int64_t kMaxRow = int64_t{1} << 30;
// Most elements that AdamW takes in one cluster: above, the state's traffic wants all SMs (fp32, us,
// cluster against norm and AdamW kernel: 60k 6.6 / 7.8, 100k 7.5 / 7.5, 240k 14.1 / 8.3).
constexpr int64_t kClusterAdamw = 96 * 1024;
constexpr size_t kKeepBytes = size_t{kListWarps} * 512;  // one row of each warp of a block
constexpr int64_t kMaxElements = int64_t{1} << 46;
constexpr int64_t kMaxUnits = int64_t{1} << 30;
enum { kRoleOut = 1, kRoleAdam = 2, kRoleBf16 = 4, kGradsOverlap = 8 };

// Host image of a plan: this header, the tables in the order of `Image`, and the ranges of addresses that
// the list's tensors take up.
struct PlanHeader {
  uint64_t magic;
  int32_t n, n_scale, n_adamw, n_further, n_spanning, n_empty, scale_unit;
  int32_t blocks, rows, cluster;  // rows: of each warp; cluster: the blocks make up one
  int32_t roles, n_groups, n_taken;
  int64_t total;  // elements
};
// Offsets of the tables in the image (which the device holds as well).
struct Image {
  size_t opening, further, spanning, shared, scale_tensor, adamw_tensor, empty, bytes;
  explicit Image(const PlanHeader& h) {
    opening = (static_cast<size_t>(h.n) * sizeof(TensorEntry) + 15) / 16 * 16;
    further = opening + sizeof(Segment) * static_cast<size_t>(h.blocks) * kListWarps;
    spanning = further + sizeof(Segment) * static_cast<size_t>(h.n_further);
    shared = spanning + sizeof(Spanning) * static_cast<size_t>(h.n_spanning);
    scale_tensor = shared + sizeof(Shared2) * static_cast<size_t>(h.blocks);
    adamw_tensor = scale_tensor + 4 * static_cast<size_t>(h.n_scale);
    empty = adamw_tensor + 4 * static_cast<size_t>(h.n_adamw);
    bytes = empty + 4 * static_cast<size_t>(h.n_empty);
  }
};
char* image_of(void* plan) { return static_cast<char*>(plan) + sizeof(PlanHeader); }
const char* image_of(const void* plan) { return static_cast<const char*>(plan) + sizeof(PlanHeader); }

// A range of addresses, from the first to the last element of a tensor or of several that touch.
struct Taken {
  uintptr_t begin, end;
};
size_t taken_offset(const Image& image) { return sizeof(PlanHeader) + (image.bytes + 7) / 8 * 8; }

// Device work area: header, sums of the blocks, their edge sums, the factor, the tickets, the image
// of the plan.
struct WorkLayout {
  size_t block_sum, edge_sum, factor, tickets, image, bytes;
  explicit WorkLayout(const PlanHeader& h) {
    block_sum = sizeof(double) * ABS_STATS_HEADER;
    edge_sum = block_sum + sizeof(double) * static_cast<size_t>(h.blocks);
    factor = edge_sum + sizeof(double) * 2 * static_cast<size_t>(h.blocks);
    tickets = factor + sizeof(float);
    image = (tickets + 4 * (1 + static_cast<size_t>(h.n_spanning)) + 15) / 16 * 16;
    bytes = image + Image(h).bytes;
  }
};

// How the rows of a list are dealt out, a function of the list's sizes alone (and with it the shape of
// every sum).  Lists of up to 2 MiB and 384 tensors go to the warps of one cluster, others to the
// warps of all SMs.  Measured (fp32, us, cluster against all SMs): 60k elements in 20 tensors, norm
// 3.5 / 5.0, clip 5.0 / 7.6; 500k: 4.3 / 5.4 and 8.7 / 9.1; 400 tensors of 100 elements: 5.1 / 5.0 and
// 7.1 / 7.0; 1600 tensors: 10.5 / 5.6 and 18.1 / 11.7.
constexpr int kClusterTensors = 384;
constexpr int64_t kRowBytes = 512;
struct Deal {
  bool cluster;
  int blocks;
  int64_t rows;  // of each warp
};
Deal deal_of(int64_t rows, int tensors) {
  Deal d;
  d.cluster = rows <= int64_t{kClusterBlocks} * kListWarps * kClusterRows && tensors <= kClusterTensors;
  const int64_t most = static_cast<int64_t>(d.cluster ? kClusterBlocks : kListBlocks) * kListWarps;
  d.rows = std::max<int64_t>(1, (rows + most - 1) / most);
  const int64_t slots = std::max<int64_t>(1, (rows + d.rows - 1) / d.rows);
  d.blocks = static_cast<int>((slots + kListWarps - 1) / kListWarps);
  return d;
}
// Rows of a tensor, the last one short.
int64_t rows_of(int64_t numel, size_t esz) {
  return (numel * static_cast<int64_t>(esz) + kRowBytes - 1) / kRowBytes;
}

// Elements per unit of scaling: a power of two between 4096 and 32768, the smallest that leaves at most
// eight units to each of the 148 SMs.  Measured (us): 124M bf16, units of 8192 / 16384 / 32768: 134 / 127 /
// 125; 50M fp16, at most 8 / 16 / 32 / 64 units to an SM: 38.8 / 40.0 / 42.2 / 53.8.
int scale_unit_for(int64_t total) {
  int unit = 4096;
  while (unit < 32768 && total / unit > 8 * 148) unit *= 2;
  return unit;
}
int64_t units_of(int64_t numel, int head, int unit) {
  return numel > head ? (numel - head + unit - 1) / unit : 1;
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

// Elements of a contiguous view before the first one on a boundary of `bytes` bytes.
int head_of(const View& v, size_t bytes) {
  const size_t a = reinterpret_cast<uintptr_t>(v.data) % bytes;
  return v.rows() || !a ? 0 : static_cast<int>((bytes - a) / v.esz);
}
// Whether element `i` of a contiguous view lies on a boundary of `bytes` bytes.
bool aligned_at(const View& v, int i, size_t bytes) {
  return !v.rows() && (reinterpret_cast<uintptr_t>(v.data) + i * v.esz) % bytes == 0;
}
// Whether offsets within a run of `most` elements of a view may need more than 31 bits.
bool spans_far(const View& v, int64_t most) {
  const int64_t rows = std::min(v.numel / v.row, most / v.row + 2);
  return rows > (int64_t{1} << 30) / v.stride || v.row > (int64_t{1} << 30) / v.col;
}

// The bytes of a view: `n` groups, `step` apart, of `pieces` runs of `width` bytes, `piece_step` apart.
// Neither the groups nor the runs of a group reach into each other.
struct Places {
  uintptr_t at;
  int64_t n, step, pieces, piece_step, width;
  int64_t group() const { return (pieces - 1) * piece_step + width; }
  explicit Places(const View& v) : at(reinterpret_cast<uintptr_t>(v.data)) {
    const int64_t esz = static_cast<int64_t>(v.esz);
    n = v.numel / v.row, step = v.stride * esz, pieces = v.row, piece_step = v.col * esz, width = esz;
    if (step <= (pieces - 1) * piece_step) std::swap(n, pieces), std::swap(step, piece_step);
    if (piece_step == width) width *= pieces, pieces = 1;
    if (n == 1) n = pieces, step = piece_step, pieces = 1;
  }
};

// Items of `ea` bytes at a, a + sa, .. (na of them) against such at b: whether f(place in a, place in b)
// is true for two that share a byte.  No two of a meet, nor two of b, so those that share form one chain,
// which is walked from its beginning.  What lies where repeats after the common multiple of sa and sb.
template <typename F>
bool any_pair(int64_t a, int64_t na, int64_t sa, int64_t ea, int64_t b, int64_t nb, int64_t sb, int64_t eb,
              F&& f) {
  int64_t period_a = na, period_b = nb;  // in items
  if (na > 1 && nb > 1) {
    const int64_t g = std::gcd(sa, sb);
    period_a = std::min(na, sb / g);
    period_b = std::min(nb, sa / g);
  }
  int64_t i = 0, k = 0;
  while (true) {
    // the first items that end after the other one begins
    if (a + i * sa + ea <= b + k * sb) i = (b + k * sb - ea - a) / sa + 1;
    if (i >= na) return false;
    if (b + k * sb + eb <= a + i * sa) k = (a + i * sa - eb - b) / sb + 1;
    if (k >= nb || (i >= period_a && k >= period_b)) return false;
    const int64_t pa = a + i * sa, pb = b + k * sb;
    if (pa + ea <= pb) continue;
    if (f(pa, pb)) return true;
    if (pa + ea <= pb + eb)
      ++i;
    else
      ++k;
  }
}

// Two views share an element.
bool views_overlap(const View& a, const View& b) {
  if (!overlaps(a.data, a.extent(), b.data, b.extent())) return false;
  const Places p(a), q(b);
  const int64_t from = static_cast<int64_t>(q.at - p.at);
  return any_pair(0, p.n, p.step, p.group(), from, q.n, q.step, q.group(), [&](int64_t x, int64_t y) {
    return any_pair(x, p.pieces, p.piece_step, p.width, y, q.pieces, q.piece_step, q.width,
                    [](int64_t, int64_t) { return true; });
  });
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

// The ranges that the views of a list take up, in order, those that touch as one.  Sorted by address.
std::vector<Taken> taken_by(const std::vector<std::pair<View, bool>>& list) {
  std::vector<Taken> all;
  for (const auto& [v, written] : list) {
    const uintptr_t begin = reinterpret_cast<uintptr_t>(v.data), end = begin + v.extent();
    if (!all.empty() && begin <= all.back().end)
      all.back().end = std::max(all.back().end, end);
    else
      all.push_back({begin, end});
  }
  return all;
}

const PlanHeader* plan_of(const void* plan) {
  if (!plan || misaligned(plan, 8)) return nullptr;
  const PlanHeader* h = static_cast<const PlanHeader*>(plan);
  return h->magic == kPlanMagic ? h : nullptr;
}

// Whether `bytes` bytes at p hold an element of a tensor of the plan.  Outside of the ranges that the
// tensors take up that is one search; inside (it may still be a gap between rows) every tensor is asked.
bool over_tensors(const PlanHeader& h, const void* p, size_t bytes) {
  const char* image = image_of(&h);
  const Taken* taken = reinterpret_cast<const Taken*>(reinterpret_cast<const char*>(&h) + taken_offset(Image(h)));
  const uintptr_t begin = reinterpret_cast<uintptr_t>(p);
  const Taken* first = std::partition_point(taken, taken + h.n_taken, [&](const Taken& t) { return t.end <= begin; });
  if (first == taken + h.n_taken || first->begin >= begin + bytes) return false;
  const int64_t n = static_cast<int64_t>(bytes);
  const View here{p, n, n, n, 1, 1};
  const TensorEntry* entries = reinterpret_cast<const TensorEntry*>(image);
  for (int t = 0; t < h.n; ++t) {
    const TensorEntry& e = entries[t];
    if (!e.numel) continue;
    View g{e.g, e.numel, e.numel, e.numel, 1, element_size(e.g_dtype)};
    if (e.flags & kEntryRowsG) g.row = e.g_row, g.stride = e.g_stride, g.col = e.g_col;
    if (views_overlap(here, g)) return true;
    if (e.out) {
      View out{e.out, e.numel, e.numel, e.numel, 1, element_size(e.out_dtype)};
      if (e.flags & kEntryRowsOut) out.row = e.out_row, out.stride = e.out_stride, out.col = e.out_col;
      if (views_overlap(here, out)) return true;
    }
    const size_t numel = static_cast<size_t>(e.numel);
    for (const float* s : {e.p, e.m, e.v})
      if (s && overlaps(p, bytes, s, 4 * numel)) return true;
    if (e.p16 && overlaps(p, bytes, e.p16, 2 * numel)) return true;
  }
  return false;
}

int fill_params(const void* plan, void* work, int norm_type, double scale, double max_norm,
                const double* sum_in, float* norms_out, TensorsParams* prm) {
  if (!plan || !work) return ABS_ERR_NULL;
  const PlanHeader* h = plan_of(plan);
  if (!h) return ABS_ERR_RANGE;
  if (norm_type != ABS_NORM_2 && norm_type != ABS_NORM_1 && norm_type != ABS_NORM_MAX)
    return ABS_ERR_RANGE;
  if (!(std::fabs(scale) <= FLT_MAX) || static_cast<float>(scale) == 0.f) return ABS_ERR_RANGE;
  if (!std::isfinite(max_norm) || max_norm < 0.0) return ABS_ERR_RANGE;
  if (misaligned(work, 16) || misaligned(norms_out, 4) || misaligned(sum_in, 8))
    return ABS_ERR_ALIGN;
  const WorkLayout L(*h);
  char* w = static_cast<char*>(work);
  const size_t norms_bytes = 4 * (static_cast<size_t>(h->n) + 2);
  if (norms_out && overlaps(norms_out, norms_bytes, work, L.bytes)) return ABS_ERR_ALIAS;
  if ((norms_out && over_tensors(*h, norms_out, norms_bytes)) || over_tensors(*h, work, L.bytes))
    return ABS_ERR_ALIAS;
  prm->header = reinterpret_cast<double*>(w);
  prm->block_sum = reinterpret_cast<double*>(w + L.block_sum);
  prm->edge_sum = reinterpret_cast<double*>(w + L.edge_sum);
  prm->factor = reinterpret_cast<float*>(w + L.factor);
  prm->tickets = reinterpret_cast<unsigned int*>(w + L.tickets);
  const Image I(*h);
  w += L.image;
  prm->entries = reinterpret_cast<const TensorEntry*>(w);
  prm->opening = reinterpret_cast<const Segment*>(w + I.opening);
  prm->further = reinterpret_cast<const Segment*>(w + I.further);
  prm->spanning = reinterpret_cast<const Spanning*>(w + I.spanning);
  prm->shared = reinterpret_cast<const Shared2*>(w + I.shared);
  prm->scale_tensor = reinterpret_cast<const int32_t*>(w + I.scale_tensor);
  prm->adamw_tensor = reinterpret_cast<const int32_t*>(w + I.adamw_tensor);
  prm->empty = reinterpret_cast<const int32_t*>(w + I.empty);
  prm->norms_out = norms_out;
  prm->n_scale = h->n_scale;
  prm->n_adamw = h->n_adamw;
  prm->scale_unit = h->scale_unit;
  prm->n_spanning = h->n_spanning;
  prm->n_empty = h->n_empty;
  prm->norm_type = norm_type;
  prm->scale = scale;
  prm->max_norm = max_norm;
  prm->sum_in = sum_in;
  prm->in_place = !(h->roles & kRoleOut);
  prm->after_norm = 0;
  return ABS_OK;
}

// Whether the current device can run a cluster kernel with all its blocks.  Asked once per device,
// for the kernel with the largest need; sets what each kernel has to be allowed.
template <int NORM, int OP>
cudaError_t allow_cluster() {
  const auto kernel = tensors_cluster_kernel<NORM, OP>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess || OP == kOpNone) return e;
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(kKeepBytes * kClusterRows));
}
template <int OP>
cudaError_t allow_clusters() {
  cudaError_t e = allow_cluster<kNorm2, OP>();
  if (e == cudaSuccess) e = allow_cluster<kNorm1, OP>();
  return e == cudaSuccess ? allow_cluster<kNormMax, OP>() : e;
}
bool cluster_runs() {
  static std::mutex mu;
  static std::atomic<int> cached[64] = {};  // 0: not asked, 1: no, 2: yes
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (const int c = cached[dev].load(std::memory_order_acquire)) return c == 2;
  std::lock_guard<std::mutex> lock(mu);
  int clusters = 0;
  bool yes = allow_clusters<kOpNone>() == cudaSuccess && allow_clusters<kOpScale>() == cudaSuccess &&
             allow_clusters<kOpAdamw>() == cudaSuccess;
  if (yes) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kClusterBlocks);
    cfg.blockDim = dim3(kListWarps * 32);
    cfg.dynamicSmemBytes = kKeepBytes * kClusterRows;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kClusterBlocks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    yes = cudaOccupancyMaxActiveClusters(&clusters, tensors_cluster_kernel<kNorm2, kOpAdamw>, &cfg) ==
              cudaSuccess && clusters >= 1;
  }
  (void)cudaGetLastError();  // a refused query is an answer, not an error of the call
  cached[dev].store(yes ? 2 : 1, std::memory_order_release);
  return yes;
}

template <int OP>
cudaError_t launch_cluster(const PlanHeader& h, const TensorsParams& prm, const GroupScalars& groups,
                           cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(h.blocks);
  cfg.blockDim = dim3(kListWarps * 32);
  cfg.dynamicSmemBytes = OP == kOpNone ? 0 : kKeepBytes * h.rows;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = h.blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const int rows = h.rows;
  return prm.norm_type == ABS_NORM_2
             ? cudaLaunchKernelEx(&cfg, tensors_cluster_kernel<kNorm2, OP>, prm, groups, rows)
         : prm.norm_type == ABS_NORM_1
             ? cudaLaunchKernelEx(&cfg, tensors_cluster_kernel<kNorm1, OP>, prm, groups, rows)
             : cudaLaunchKernelEx(&cfg, tensors_cluster_kernel<kNormMax, OP>, prm, groups, rows);
}

cudaError_t launch_norm(const PlanHeader& h, const TensorsParams& prm, cudaStream_t st) {
  const dim3 grid(h.blocks), block(kListWarps * 32);
  return prm.norm_type == ABS_NORM_2   ? launch_pdl(tensors_norm_kernel<kNorm2>, grid, block, st, prm)
         : prm.norm_type == ABS_NORM_1 ? launch_pdl(tensors_norm_kernel<kNorm1>, grid, block, st, prm)
                                       : launch_pdl(tensors_norm_kernel<kNormMax>, grid, block, st, prm);
}

// The factor of a call: from the list's own norm, or from the sum that it is given.
cudaError_t launch_norm_or_clip(const PlanHeader& h, const TensorsParams& prm, cudaStream_t st) {
  return prm.sum_in ? launch_pdl(tensors_clip_kernel, dim3(1), dim3(32), st, prm)
                    : launch_norm(h, prm, st);
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
  int nonempty = 0;
  for (int t = 0; t < n; ++t) {
    View g;
    const int rc = view_of(grads[t], &g);
    if (rc != ABS_OK) return rc;
    if (grads[t].group < 0 || grads[t].group >= ABS_MAX_GROUPS) return ABS_ERR_RANGE;
    if (g.numel > kMaxElements - total) return ABS_ERR_RANGE;
    total += g.numel;
    total_rows += rows_of(g.numel, g.esz);
    nonempty += g.numel > 0;
  }
  h.total = total;
  h.scale_unit = scale_unit_for(total);
  const Deal deal = deal_of(total_rows, nonempty);
  h.blocks = deal.blocks;
  h.cluster = deal.cluster;
  h.rows = static_cast<int32_t>(deal.rows);
  std::vector<TensorEntry> entries(n);
  std::vector<int32_t> scale_tensor, adamw_tensor;
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
    const size_t per = 16 / g.esz;  // values in 16 bytes of the gradient
    e.g_head = static_cast<uint8_t>(head_of(g, 16));
    const int64_t longest = std::max<int64_t>(h.scale_unit, deal.rows * (kRowBytes / 2));
    if (rows_g && spans_far(g, longest)) e.flags |= kEntryFar;
    if (rows_g && g.col == 1 && g.row >= 16 && !(e.flags & kEntryFar)) e.flags |= kEntryRuns;
    const View& y = outs ? out : g;
    e.scale_head = static_cast<uint8_t>(head_of(y, 8 * y.esz));
    if (!rows_g && aligned_at(y, e.g_head, std::min<size_t>(16, per * y.esz)))
      e.flags |= kEntryVecScale;
    if (params) {
      e.adamw_head = static_cast<uint8_t>(head_of(state[0], 32));
      bool together = true, vec = !rows_g;
      for (int i = 0; i < 3; ++i) {
        together = together && aligned_at(state[i], e.adamw_head, 32);
        vec = vec && aligned_at(state[i], e.g_head, 16);
      }
      if (params_bf16) {
        together = together && aligned_at(b16, e.adamw_head, 16);
        vec = vec && aligned_at(b16, e.g_head, 8);
      }
      if (together) e.flags |= kEntryStateVec;
      if (vec) e.flags |= kEntryVecAdamw;
    }
    if (e.numel) {
      e.first_scale = static_cast<int32_t>(scale_tensor.size());
      e.first_adamw = static_cast<int32_t>(adamw_tensor.size());
      const int64_t k = units_of(e.numel, e.adamw_head, kAdamwUnit);
      if (k > kMaxUnits - static_cast<int64_t>(adamw_tensor.size())) return ABS_ERR_RANGE;
      scale_tensor.insert(scale_tensor.end(),
                          static_cast<size_t>(units_of(e.numel, e.scale_head, h.scale_unit)), t);
      if (params) adamw_tensor.insert(adamw_tensor.end(), static_cast<size_t>(k), t);
    }
    entries[t] = e;
  }
  if (any_conflict(all)) return ABS_ERR_ALIAS;
  if (any_conflict(grads_written)) h.roles |= kGradsOverlap;
  const std::vector<Taken> taken = taken_by(all);  // which any_conflict has sorted
  h.n_taken = static_cast<int32_t>(taken.size());

  // the segments: the rows of all tensors in order, dealt out warp by warp
  Segment idle;
  std::memset(&idle, 0, sizeof idle);
  idle.tensor = -1;
  std::vector<Segment> opening(static_cast<size_t>(deal.blocks) * kListWarps, idle), further;
  std::vector<Spanning> spanning;
  std::vector<int32_t> empty;
  int64_t slot = -1, left = 0;  // the warp that is dealt to, and the rows that it still takes
  for (int t = 0; t < n; ++t) {
    const TensorEntry& e = entries[t];
    if (!e.numel) {
      empty.push_back(t);
      continue;
    }
    const size_t esz = element_size(e.g_dtype);
    const int64_t per_row = kRowBytes / static_cast<int64_t>(esz);
    const int head = e.g_head;
    int64_t rows = rows_of(e.numel, esz), start = 0, first_block = 0;
    while (start < e.numel) {
      const bool opens = left == 0;
      if (opens) {
        ++slot;
        left = deal.rows;
      }
      const int64_t take = std::min(rows, left);
      rows -= take;
      left -= take;
      // every segment but the last ends on a 16-byte boundary: `head` elements further
      int64_t end = rows ? start + take * per_row + (start ? 0 : head) : e.numel;
      if (end >= e.numel) {  // perhaps the head has taken the last, short row
        end = e.numel;
        rows = 0;
      }
      Segment s;
      std::memset(&s, 0, sizeof s);
      s.g = static_cast<const char*>(e.g) + (e.flags & kEntryRowsG ? 0 : start * esz);
      s.start = start;
      s.n = static_cast<uint32_t>(end - start);
      s.tensor = t;
      s.dtype = e.g_dtype;
      s.head = static_cast<uint8_t>(start ? 0 : std::min<int64_t>(head, s.n));
      s.flags = e.flags;
      s.pos = (start ? 0 : kSegBegins) | (end == e.numel ? kSegEnds : 0);
      if (opens) {
        s.next = static_cast<int32_t>(further.size());
        opening[slot] = s;
      } else {
        ++opening[slot].more;
        further.push_back(s);
      }
      const int64_t block = slot / kListWarps;
      if (!start) first_block = block;
      if (end == e.numel && block != first_block)
        spanning.push_back({t, static_cast<int32_t>(first_block), static_cast<int32_t>(block), 0});
      start = end;
    }
  }
  std::vector<Shared2> shared(static_cast<size_t>(deal.blocks), Shared2{-1, -1});
  for (size_t i = 0; i < spanning.size(); ++i)
    for (int32_t b = spanning[i].first; b <= spanning[i].last; ++b) {
      // a tensor that fills a block whole is counted off once there, as one from before
      if (b > spanning[i].first) shared[b].before = static_cast<int32_t>(i);
      if (b == spanning[i].first) shared[b].after = static_cast<int32_t>(i);
    }
  h.n_spanning = static_cast<int32_t>(spanning.size());
  h.n_empty = static_cast<int32_t>(empty.size());
  h.n_further = static_cast<int32_t>(further.size());
  h.n_scale = static_cast<int32_t>(scale_tensor.size());
  h.n_adamw = static_cast<int32_t>(adamw_tensor.size());

  const Image I(h);
  if (plan_bytes < taken_offset(I) + taken.size() * sizeof(Taken)) return ABS_ERR_TOO_LARGE;
  char* image = image_of(plan);
  const auto put = [](char* to, const void* from, size_t bytes) {
    if (bytes) std::memcpy(to, from, bytes);
  };
  put(image, entries.data(), entries.size() * sizeof(TensorEntry));
  put(image + I.opening, opening.data(), opening.size() * sizeof(Segment));
  put(image + I.further, further.data(), further.size() * sizeof(Segment));
  put(image + I.spanning, spanning.data(), spanning.size() * sizeof(Spanning));
  put(image + I.shared, shared.data(), shared.size() * sizeof(Shared2));
  put(image + I.scale_tensor, scale_tensor.data(), scale_tensor.size() * 4);
  put(image + I.adamw_tensor, adamw_tensor.data(), adamw_tensor.size() * 4);
  put(image + I.empty, empty.data(), empty.size() * 4);
  put(static_cast<char*>(plan) + taken_offset(I), taken.data(), taken.size() * sizeof(Taken));
  std::memcpy(plan, &h, sizeof h);
  return ABS_OK;
}

}  // namespace

extern "C" {

size_t abs_tensors_plan_bytes(const abs_tensor* grads, int n) {
  if (n < 0 || n > ABS_MAX_TENSORS || (n > 0 && !grads)) return 0;
  int64_t total = 0, rows = 0, scale = 0, adamw = 0;
  int nonempty = 0;
  for (int t = 0; t < n; ++t) {
    if (grads[t].numel < 0 || grads[t].numel > kMaxElements - total) return 0;
    total += grads[t].numel;
    rows += rows_of(grads[t].numel, element_size(grads[t].dtype));
    nonempty += grads[t].numel > 0;
  }
  const int unit = scale_unit_for(total);
  for (int t = 0; t < n; ++t) {
    scale += (grads[t].numel + unit - 1) / unit;
    adamw += (grads[t].numel + kAdamwUnit - 1) / kAdamwUnit;
  }
  if (adamw > kMaxUnits) return 0;
  const Deal deal = deal_of(rows, nonempty);
  PlanHeader h;  // upper bounds
  std::memset(&h, 0, sizeof h);
  h.n = h.n_empty = h.n_further = n;
  h.n_scale = static_cast<int32_t>(scale);
  h.n_adamw = static_cast<int32_t>(adamw);
  h.blocks = deal.blocks;
  h.n_spanning = std::min(n, deal.blocks);
  return taken_offset(Image(h)) + 6 * static_cast<size_t>(n) * sizeof(Taken);  // six roles
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
  if (over_tensors(*h, work, L.bytes)) return ABS_ERR_ALIAS;
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
  const PlanHeader& h = *plan_of(plan);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = h.cluster && cluster_runs()
                            ? launch_cluster<kOpNone>(h, prm, GroupScalars{}, st)
                            : launch_norm(h, prm, st);
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

int abs_grad_clip(const void* plan, void* work, int norm_type, double grad_scale, double max_norm,
                  const double* sum_in, float* norms_out, abs_stream_t stream) {
  TensorsParams prm;
  const int rc = fill_params(plan, work, norm_type, grad_scale, max_norm, sum_in, norms_out, &prm);
  if (rc != ABS_OK) return rc;
  if (!norms_out) return ABS_ERR_NULL;
  if (!(max_norm > 0.0)) return ABS_ERR_RANGE;
  const PlanHeader& h = *plan_of(plan);
  if (prm.in_place && (h.roles & kGradsOverlap)) return ABS_ERR_ALIAS;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (!sum_in && h.cluster && cluster_runs()) {
    e = launch_cluster<kOpScale>(h, prm, GroupScalars{}, st);
  } else {
    e = launch_norm_or_clip(h, prm, st);
    prm.after_norm = !sum_in;
    if (e == cudaSuccess && prm.n_scale > 0)
      e = launch_pdl(tensors_scale_kernel, dim3(prm.n_scale), dim3(kTensorThreads), st, prm);
  }
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
  cudaError_t e;
  if (clipped && !sum_in && h->cluster && h->total <= kClusterAdamw && cluster_runs()) {
    e = launch_cluster<kOpAdamw>(*h, prm, groups, st);
  } else {
    e = clipped ? launch_norm_or_clip(*h, prm, st) : cudaSuccess;
    prm.after_norm = clipped && !sum_in;
    if (e == cudaSuccess && prm.n_adamw > 0)
      e = launch_pdl(tensors_adamw_kernel, dim3(prm.n_adamw), dim3(kTensorThreads), st, prm, groups,
                     clipped ? 1 : 0);
  }
  return e == cudaSuccess ? ABS_OK : cuda_fail(e);
}

}  // extern "C"
