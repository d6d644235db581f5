// Host side of the operators between a tower's products: the norm, 4-bit weights with group scales, and the norm of the
// gradients (include/emb_dense.h).  Checks arguments, lays out buffers and launches the kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>
#include <utility>
#include <vector>

#include "dense_checks.h"
#include "dense_internal.h"

using namespace embd;

namespace {

// A matrix whose byte offsets fit 63 bits, or one of 8-bit rows.
bool rows8_ok(const void* x, int64_t rows, int64_t cols, int64_t ld) {
  return x && ld >= cols && (double)rows * (double)ld <= 4.0 * kMaxBytes;
}

bool norm_dims_ok(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 1 && rows < kMaxDim && cols < kMaxDim; }

bool gain_ok(const void* gain, int32_t gain_type, int32_t type) {
  if (gain_type != EMB_TYPE_FP32 && gain_type != type) return false;
  return reinterpret_cast<uintptr_t>(gain) % type_bytes(gain_type) == 0;
}

// A matrix by its bytes: whether two of them share one, and whether they lie alike.
struct Span {
  const void* p;
  int64_t rows, width, stride;
};
Span span(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t bytes) { return {p, p ? rows : 0, cols * bytes, ld * bytes}; }
bool meet(const Span& a, const Span& b) { return share_elements(a.p, a.rows, a.width, a.stride, b.p, b.rows, b.width, b.stride, 1); }
bool alike(const Span& a, const Span& b) { return a.p == b.p && a.width == b.width && (a.stride == b.stride || a.rows == 1); }
// An output that may lie over an input, if exactly.
bool over_ok(const Span& out, const Span& in) { return alike(out, in) || !meet(out, in); }

int norm_forward(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const void* residual, int64_t ldr,
                 const void* gain, int32_t gain_type, float eps, void* sum, int64_t lds, void* y, int64_t ldy, float* inverse,
                 float* scales, bool bits8, void* stream) {
  if (!type_ok(type) || !norm_dims_ok(rows, cols) || !(eps >= 0x1p-126f) || !std::isfinite(eps)) return EMB_EINVAL;
  if (!gain_ok(gain, gain_type, type) || (sum && !residual)) return EMB_EINVAL;
  if (rows == 0) return EMB_OK;
  const int64_t b = type_bytes(type);
  if (!matrix_ok(x, type, rows, cols, ldx) || (residual && !matrix_ok(residual, type, rows, cols, ldr)) ||
      (sum && !matrix_ok(sum, type, rows, cols, lds)))
    return EMB_EINVAL;
  if (bits8 ? !rows8_ok(y, rows, cols, ldy) || !scales || reinterpret_cast<uintptr_t>(scales) % 4
            : !matrix_ok(y, type, rows, cols, ldy))
    return EMB_EINVAL;
  if (reinterpret_cast<uintptr_t>(inverse) % 4) return EMB_EINVAL;
  const Span sx = span(x, rows, cols, ldx, b), sr = span(residual, rows, cols, ldr, b), sh = span(sum, rows, cols, lds, b);
  const Span sy = span(y, rows, cols, ldy, bits8 ? 1 : b), sg = span(gain, 1, cols, cols, type_bytes(gain_type));
  const Span si = span(inverse, 1, rows, rows, 4), sc = span(scales, 1, rows, rows, 4);
  if (!over_ok(sh, sx) || !over_ok(sh, sr) || meet(sh, sy)) return EMB_EINVAL;
  if (bits8 ? meet(sy, sx) || meet(sy, sr) : !over_ok(sy, sx) || !over_ok(sy, sr)) return EMB_EINVAL;
  for (const Span& small : {si, sc})
    for (const Span& other : {sx, sr, sh, sy, sg})
      if (meet(small, other)) return EMB_EINVAL;
  if (meet(sg, sh) || meet(sg, sy) || meet(si, sc)) return EMB_EINVAL;
  const NormForward a = {{x, ldx}, {residual, ldr}, {sum, lds}, {y, ldy}, rows, cols, gain, inverse, scales, eps};
  return status(launch_norm(a, type, gain_type == EMB_TYPE_FP32, S(stream)));
}

bool group_ok(int32_t g) { return g == 32 || g == 64 || g == 128; }

// A W4 matrix of at most kMaxBytes.
bool w4_ok(int64_t rows, int64_t cols, int32_t group) {
  if (!group_ok(group) || rows < 0 || cols < 0 || rows >= kMaxDim || cols >= kMaxDim) return false;
  return (double)W4(nullptr, rows, cols, group).bytes() <= kMaxBytes;
}

// Bytes from begin to end; none of an absent buffer.
struct Range {
  uintptr_t begin = 0, end = 0;
  bool meets(const Range& o) const { return begin < o.end && o.begin < end; }
};
Range range(const void* p, size_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return p && bytes ? Range{at, at + bytes} : Range{};
}

// A W4 matrix and its plain form.
struct Plain {
  Range q, codes, scales, biases;
  Plain(const W4& w, const void* c, const void* s, const void* b)
      : q(range(w.base, (size_t)w.bytes())),
        codes(range(c, (size_t)(w.rows * ((w.cols + 1) / 2)))),
        scales(range(s, (size_t)(w.rows * ceil_div(w.cols, w.group) * 2))),
        biases(range(b, (size_t)(w.rows * ceil_div(w.cols, w.group) * 2))) {}
  bool over_matrix() const { return q.meets(codes) || q.meets(scales) || q.meets(biases); }
  bool over_each_other() const { return codes.meets(scales) || codes.meets(biases) || scales.meets(biases); }
};

}  // namespace

struct emb_clip {
  std::vector<int64_t> sizes, part0;   // part0[t]: first part of tensor t, part0[num_tensors] their number
  std::vector<int32_t> types;
  ClipDev dev;
  Range state;
};

namespace {

struct ClipPlan {
  std::vector<ClipTensor> tensors;
  std::vector<int64_t> part0;
  size_t o_tensors, o_parts, bytes;
};

// Elements for a workgroup: few enough that small models fill the device, many enough that the parts of a large one are
// soon joined.
constexpr int64_t kClipLeast = 2048, kClipParts = 2048;

int plan_clip(const emb_clip_config* c, ClipPlan* p) {
  if (!c || c->num_tensors < 1 || !c->sizes || (!c->types && !type_ok(c->type))) return EMB_EINVAL;
  int64_t total = 0;
  for (int t = 0; t < c->num_tensors; ++t) {
    const int64_t n = c->sizes[t];
    const int32_t type = c->types ? c->types[t] : c->type;
    if (n < 0 || n > ((int64_t)1 << 40) || !type_ok(type)) return EMB_EINVAL;
    p->tensors.push_back({n, type, 0});
    total += n;
    if (total > ((int64_t)1 << 40)) return EMB_EINVAL;
  }
  int64_t chunk = kClipLeast;
  while (total / chunk > kClipParts) chunk *= 2;
  int64_t parts = 0;
  for (ClipTensor& t : p->tensors) {
    p->part0.push_back(parts);
    t.parts = (uint32_t)ceil_div(t.size, chunk);
    parts += t.parts;
  }
  p->part0.push_back(parts);
  p->o_tensors = 0;
  p->o_parts = align_up(sizeof(ClipTensor) * p->tensors.size());
  p->bytes = align_up(p->o_parts + sizeof(AdamPart) * (size_t)parts);
  return EMB_OK;
}

size_t clip_workspace(int64_t parts) { return align_up(sizeof(double) * (size_t)parts); }

// Calls f(pointers, first tensor, first part, parts) for each launch.
template <class F>
hipError_t over_tensors(const emb_clip* h, const void* const* grads, F f) {
  const int T = (int)h->sizes.size();
  for (int first = 0; first < T; first += kClipTensors) {
    const int n = T - first < kClipTensors ? T - first : kClipTensors;
    const int64_t part0 = h->part0[first], parts = h->part0[first + n] - part0;
    if (!parts) continue;
    ClipPointers ptr;
    for (int k = 0; k < kClipTensors; ++k) ptr.g[k] = k < n ? const_cast<void*>(grads[first + k]) : nullptr;
    const hipError_t e = in_launches(parts, kClipThreads, [&](int64_t from, unsigned some) { return f(ptr, (uint32_t)first, part0 + from, some); });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

bool grads_ok(const emb_clip* h, const void* const* grads) {
  for (size_t t = 0; t < h->sizes.size(); ++t)
    if (h->sizes[t] && reinterpret_cast<uintptr_t>(grads[t]) % type_bytes(h->types[t])) return false;
  return true;
}

Range place(const emb_clip* h, const void* const* grads, size_t t) { return range(grads[t], (size_t)h->sizes[t] * type_bytes(h->types[t])); }

// Whether no gradient shares memory with one of `others`.
bool clear_of(const emb_clip* h, const void* const* grads, std::initializer_list<Range> others) {
  for (size_t t = 0; t < h->sizes.size(); ++t) {
    const Range p = place(h, grads, t);
    for (const Range& o : others)
      if (p.meets(o)) return false;
  }
  return true;
}

// Whether no two gradients share memory.  They mostly lie one behind the other already.
bool apart(const emb_clip* h, const void* const* grads) {
  uintptr_t end = 0;
  bool rising = true;
  size_t there = 0;
  for (size_t t = 0; t < h->sizes.size(); ++t) {
    const Range p = place(h, grads, t);
    if (!p.end) continue;
    rising = rising && p.begin >= end;
    end = p.end;
    ++there;
  }
  if (rising) return true;
  try {
    std::vector<std::pair<uintptr_t, uintptr_t>> places;
    places.reserve(there);
    for (size_t t = 0; t < h->sizes.size(); ++t) {
      const Range p = place(h, grads, t);
      if (p.end) places.emplace_back(p.begin, p.end);
    }
    std::sort(places.begin(), places.end());
    for (size_t i = 1; i < places.size(); ++i)
      if (places[i].first < places[i - 1].second) return false;
    return true;
  } catch (const std::bad_alloc&) {
    return false;
  }
}

// The checks of a call that takes a norm, and the parts' sums of squares into the workspace.  What is written (the parts'
// sums, which are read until the last launch, and the result) lies over nothing that is read, nor over the tables.
int squares(const emb_clip* h, const void* const* grads, double max_norm, float* result, void* workspace, size_t workspace_bytes,
            void* stream) {
  if (!h || !grads || !(max_norm > 0.0) || !result || reinterpret_cast<uintptr_t>(result) % 4 || !grads_ok(h, grads)) return EMB_EINVAL;
  const size_t need = clip_workspace(h->part0.back());
  if (need && (!workspace || !aligned(workspace))) return EMB_EINVAL;
  const Range r = range(result, 8), w = range(workspace, need);
  if (r.meets(w) || r.meets(h->state) || w.meets(h->state) || !clear_of(h, grads, {r, w})) return EMB_EINVAL;
  if (workspace_bytes < need) return EMB_ENOMEM;
  return status(over_tensors(h, grads, [&](const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned some) {
    return launch_clip_squares(h->dev, ptr, first, part0, some, static_cast<double*>(workspace), S(stream));
  }));
}

}  // namespace

extern "C" {

int emb_rmsnorm_forward(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const void* residual, int64_t ldr,
                        const void* gain, int32_t gain_type, float eps, void* sum, int64_t lds, void* y, int64_t ldy,
                        float* inverse, void* stream) {
  return norm_forward(x, type, rows, cols, ldx, residual, ldr, gain, gain_type, eps, sum, lds, y, ldy, inverse, nullptr, false, stream);
}

int emb_rmsnorm_forward8(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ldx, const void* residual, int64_t ldr,
                         const void* gain, int32_t gain_type, float eps, void* sum, int64_t lds, int8_t* codes, int64_t ldc,
                         float* scales, void* stream) {
  return norm_forward(x, type, rows, cols, ldx, residual, ldr, gain, gain_type, eps, sum, lds, codes, ldc, nullptr, scales, true, stream);
}

int emb_rows8_dequantize(const int8_t* codes, int64_t rows, int64_t cols, int64_t ldc, const float* scales, void* x, int32_t type,
                         int64_t ldx, void* stream) {
  if (!type_ok(type) || rows < 0 || cols < 0 || rows >= kMaxDim || cols >= kMaxDim) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!rows8_ok(codes, rows, cols, ldc) || !scales || reinterpret_cast<uintptr_t>(scales) % 4 || !matrix_ok(x, type, rows, cols, ldx))
    return EMB_EINVAL;
  const Span sx = span(x, rows, cols, ldx, type_bytes(type));
  if (meet(sx, span(codes, rows, cols, ldc, 1)) || meet(sx, span(scales, 1, rows, rows, 4))) return EMB_EINVAL;
  return status(launch_rows8_dequantize(codes, rows, cols, ldc, scales, x, type, ldx, S(stream)));
}

int emb_rmsnorm_backward_workspace(int32_t type, int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes || !type_ok(type) || !norm_dims_ok(rows, cols)) return EMB_EINVAL;
  const int64_t slabs = norm_slabs(rows, cols, type);
  *bytes = slabs > 1 || !norm_in_registers(cols, type) ? align_up((size_t)slabs * (size_t)cols * 4) : 0;
  return EMB_OK;
}

int emb_rmsnorm_backward(const void* dy, int32_t type, int64_t rows, int64_t cols, int64_t lddy, const void* h, int64_t ldh,
                         const float* inverse, const void* gain, int32_t gain_type, const void* dsum, int64_t ldds, void* dx,
                         int64_t lddx, void* dgain, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (emb_rmsnorm_backward_workspace(type, rows, cols, &need) != EMB_OK || !gain_ok(gain, gain_type, type) ||
      !gain_ok(dgain, gain_type, type))
    return EMB_EINVAL;
  if (!dgain) need = 0;
  if (need && (!workspace || !aligned(workspace))) return EMB_EINVAL;
  if (rows) {
    if (!matrix_ok(dy, type, rows, cols, lddy) || !matrix_ok(h, type, rows, cols, ldh) || !matrix_ok(dx, type, rows, cols, lddx) ||
        (dsum && !matrix_ok(dsum, type, rows, cols, ldds)) || !inverse || reinterpret_cast<uintptr_t>(inverse) % 4)
      return EMB_EINVAL;
    const int64_t b = type_bytes(type), g = type_bytes(gain_type);
    const Span sx = span(dx, rows, cols, lddx, b), sd = span(dgain, 1, cols, cols, g), sw = span(need ? workspace : nullptr, 1, (int64_t)need, (int64_t)need, 1);
    const Span ins[] = {span(dy, rows, cols, lddy, b), span(h, rows, cols, ldh, b), span(dsum, rows, cols, ldds, b),
                        span(inverse, 1, rows, rows, 4), span(gain, 1, cols, cols, g)};
    for (int i = 0; i < 5; ++i)
      if ((i < 3 ? !over_ok(sx, ins[i]) : meet(sx, ins[i])) || meet(sd, ins[i]) || meet(sw, ins[i])) return EMB_EINVAL;
    if (meet(sx, sd) || meet(sx, sw) || meet(sd, sw)) return EMB_EINVAL;
  }
  if (workspace_bytes < need) return EMB_ENOMEM;
  const NormBackward a = {{dy, lddy}, {h, ldh}, {dsum, ldds}, {dx, lddx}, rows, cols, inverse, gain, dgain, static_cast<float*>(workspace)};
  return status(launch_norm_backward(a, type, gain_type == EMB_TYPE_FP32, S(stream)));
}

int emb_w4_query_bytes(int64_t rows, int64_t cols, int32_t group, size_t* bytes) {
  if (!bytes || !w4_ok(rows, cols, group)) return EMB_EINVAL;
  *bytes = rows && cols ? (size_t)W4(nullptr, rows, cols, group).bytes() : 0;
  return EMB_OK;
}

int emb_w4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld, int32_t group, void* q, void* stream) {
  if (!type_ok(type) || !w4_ok(rows, cols, group)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!q || !aligned(q) || !matrix_ok(x, type, rows, cols, ld)) return EMB_EINVAL;
  const W4 w(q, rows, cols, group);
  if (meet(span(q, 1, w.bytes(), w.bytes(), 1), span(x, rows, cols, ld, type_bytes(type)))) return EMB_EINVAL;
  return status(launch_w4_quantize(x, type, ld, w, S(stream)));
}

int emb_w4_dequantize(const void* q, int64_t rows, int64_t cols, int32_t group, void* x, int32_t type, int64_t ld, void* stream) {
  if (!type_ok(type) || !w4_ok(rows, cols, group)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!q || !aligned(q) || !matrix_ok(x, type, rows, cols, ld)) return EMB_EINVAL;
  const W4 w(q, rows, cols, group);
  if (meet(span(q, 1, w.bytes(), w.bytes(), 1), span(x, rows, cols, ld, type_bytes(type)))) return EMB_EINVAL;
  return status(launch_w4_dequantize(w, x, type, ld, S(stream)));
}

int emb_w4_pack(const uint8_t* codes, const void* scales, const void* biases, int64_t rows, int64_t cols, int32_t group, void* q,
                void* stream) {
  if (!w4_ok(rows, cols, group)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!codes || !scales || !biases || !q || !aligned(q)) return EMB_EINVAL;
  if (reinterpret_cast<uintptr_t>(scales) % 2 || reinterpret_cast<uintptr_t>(biases) % 2) return EMB_EINVAL;
  const W4 w(q, rows, cols, group);
  if (Plain(w, codes, scales, biases).over_matrix()) return EMB_EINVAL;
  return status(launch_w4_pack(codes, static_cast<const uint16_t*>(scales), static_cast<const uint16_t*>(biases), w, S(stream)));
}

int emb_w4_unpack(const void* q, int64_t rows, int64_t cols, int32_t group, uint8_t* codes, void* scales, void* biases, void* stream) {
  if (!w4_ok(rows, cols, group)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!codes || !scales || !biases || !q || !aligned(q)) return EMB_EINVAL;
  if (reinterpret_cast<uintptr_t>(scales) % 2 || reinterpret_cast<uintptr_t>(biases) % 2) return EMB_EINVAL;
  const W4 w(q, rows, cols, group);
  const Plain p(w, codes, scales, biases);
  if (p.over_matrix() || p.over_each_other()) return EMB_EINVAL;
  return status(launch_w4_unpack(w, codes, static_cast<uint16_t*>(scales), static_cast<uint16_t*>(biases), S(stream)));
}

int emb_w4_linear_workspace(int32_t type, int64_t m, int64_t n, int64_t k, int32_t group, size_t* bytes) {
  if (!bytes || (!type_ok(type) && type != EMB_TYPE_INT8) || !w4_ok(n, k, group) || k > kMaxDepth || m < 0 || m >= kMaxDim)
    return EMB_EINVAL;
  *bytes = m && n && k ? w4_linear_workspace(type, m, n, k, group) : 0;
  return EMB_OK;
}

int emb_w4_linear(const void* x, int32_t type, const float* scales, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n,
                  int32_t group, const float* bias, int32_t relu, void* y, int32_t y_type, int64_t ldy, void* workspace,
                  size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (emb_w4_linear_workspace(type, m, n, k, group, &need) != EMB_OK || !type_ok(y_type)) return EMB_EINVAL;
  if (m == 0 || n == 0) return EMB_OK;
  const bool bits8 = type == EMB_TYPE_INT8;
  if (!matrix_ok(y, y_type, m, n, ldy) || reinterpret_cast<uintptr_t>(bias) % 4) return EMB_EINVAL;
  if (k && (!w || !aligned(w))) return EMB_EINVAL;
  if (k && (bits8 ? !rows8_ok(x, m, k, ldx) : !matrix_ok(x, type, m, k, ldx))) return EMB_EINVAL;
  if (bits8 ? !scales || reinterpret_cast<uintptr_t>(scales) % 4 : scales != nullptr) return EMB_EINVAL;
  if (need && (!workspace || !aligned(workspace))) return EMB_EINVAL;
  if (workspace_bytes < need) return EMB_ENOMEM;
  const W4 q(w, n, k, group);
  const Span sy = span(y, m, n, ldy, type_bytes(y_type)), sw = span(need ? workspace : nullptr, 1, (int64_t)need, (int64_t)need, 1);
  const Span ins[] = {span(k ? x : nullptr, m, k, ldx, bits8 ? 1 : type_bytes(type)), span(scales, 1, m, m, 4), span(bias, 1, n, n, 4),
                      span(k ? w : nullptr, 1, q.bytes(), q.bytes(), 1)};
  for (const Span& in : ins)
    if (meet(sy, in) || meet(sw, in)) return EMB_EINVAL;
  if (meet(sy, sw)) return EMB_EINVAL;
  const W4Linear a = {x, scales, m, ldx, bias, y, ldy, y_type, relu != 0};
  return status(launch_w4_linear(a, type, q, workspace, S(stream)));
}

int emb_clip_query_sizes(const emb_clip_config* cfg, emb_clip_sizes* out) {
  if (!out) return EMB_EINVAL;
  try {
    ClipPlan p;
    const int st = plan_clip(cfg, &p);
    if (st != EMB_OK) return st;
    *out = {p.bytes, clip_workspace(p.part0.back())};
    return EMB_OK;
  } catch (const std::bad_alloc&) {
    return EMB_EINVAL;
  }
}

int emb_clip_create(const emb_clip_config* cfg, void* state, size_t state_bytes, void* stream, emb_clip_t* out) {
  if (!out) return EMB_EINVAL;
  *out = nullptr;
  emb_clip* h = nullptr;
  try {
    ClipPlan p;
    const int st = plan_clip(cfg, &p);
    if (st != EMB_OK) return st;
    if (!state || !aligned(state)) return EMB_EINVAL;
    if (state_bytes < p.bytes) return EMB_ENOMEM;
    std::vector<AdamPart> parts;
    parts.reserve((size_t)p.part0.back());
    h = new emb_clip();
    for (int t = 0; t < cfg->num_tensors; ++t) {
      h->sizes.push_back(p.tensors[t].size);
      h->types.push_back(p.tensors[t].type);
      for (int64_t k = p.part0[t]; k < p.part0[t + 1]; ++k) parts.push_back({(uint32_t)t, (uint32_t)(k - p.part0[t])});
    }
    h->part0 = p.part0;
    uint8_t* b = static_cast<uint8_t*>(state);
    h->state = range(state, p.bytes);
    h->dev = {reinterpret_cast<const ClipTensor*>(b + p.o_tensors), reinterpret_cast<const AdamPart*>(b + p.o_parts)};
    hipError_t e = hipMemcpyAsync(b + p.o_tensors, p.tensors.data(), sizeof(ClipTensor) * p.tensors.size(), hipMemcpyHostToDevice, S(stream));
    if (e == hipSuccess && !parts.empty())
      e = hipMemcpyAsync(b + p.o_parts, parts.data(), sizeof(AdamPart) * parts.size(), hipMemcpyHostToDevice, S(stream));
    const hipError_t done = hipStreamSynchronize(S(stream));   // the host arrays go now
    if (e == hipSuccess) e = done;
    if (e != hipSuccess) {
      delete h;
      return EMB_EHIP;
    }
    *out = h;
    return EMB_OK;
  } catch (const std::bad_alloc&) {
    delete h;
    return EMB_EINVAL;
  }
}

int emb_clip_destroy(emb_clip_t h) {
  delete h;
  return EMB_OK;
}

int emb_clip_norm(emb_clip_t h, const void* const* grads, double max_norm, float* result, void* workspace, size_t workspace_bytes,
                  void* stream) {
  const int st = squares(h, grads, max_norm, result, workspace, workspace_bytes, stream);
  return st != EMB_OK ? st : status(launch_clip_join(static_cast<const double*>(workspace), h->part0.back(), max_norm, result, S(stream)));
}

int emb_clip_scale(emb_clip_t h, void* const* grads, const float* factor, void* stream) {
  if (!h || !grads || !factor || reinterpret_cast<uintptr_t>(factor) % 4 || !grads_ok(h, grads) || !apart(h, grads) ||
      !clear_of(h, grads, {range(factor, 4), h->state}))
    return EMB_EINVAL;
  return status(over_tensors(h, grads, [&](const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned some) {
    return launch_clip_scale(h->dev, ptr, first, part0, some, factor, S(stream));
  }));
}

int emb_clip_apply(emb_clip_t h, void* const* grads, double max_norm, float* result, void* workspace, size_t workspace_bytes,
                   void* stream) {
  if (!h || !grads || !grads_ok(h, grads) || !apart(h, grads) || !clear_of(h, grads, {h->state})) return EMB_EINVAL;
  const int64_t parts = h->part0.back();
  if (!parts) return emb_clip_norm(h, grads, max_norm, result, workspace, workspace_bytes, stream);
  if (h->sizes.size() > (size_t)kClipTensors) {   // of more than one launch: joined once (k_clip_join_scale)
    const int st = emb_clip_norm(h, grads, max_norm, result, workspace, workspace_bytes, stream);
    return st != EMB_OK ? st : emb_clip_scale(h, grads, result + 1, stream);
  }
  const int st = squares(h, grads, max_norm, result, workspace, workspace_bytes, stream);
  if (st != EMB_OK) return st;
  return status(over_tensors(h, grads, [&](const ClipPointers& ptr, uint32_t first, int64_t part0, unsigned some) {
    return launch_clip_join_scale(h->dev, ptr, first, part0, some, static_cast<const double*>(workspace), parts, max_norm, result, S(stream));
  }));
}

}  // extern "C"
