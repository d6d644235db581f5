// Host side of the dense operators: the C ABI of include/emb_dense.h.  Checks arguments,
// lays out buffers and launches the kernels; device memory is the caller's.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <vector>

#include "dense_checks.h"
#include "dense_internal.h"

using namespace embd;

namespace {

// Steps that a counter may be set to: the next one is above 0, and a negative number of a binding is none.
constexpr uint64_t kMaxStep = (uint64_t)INT64_MAX;

}  // namespace

struct emb_adamw {
  std::vector<int64_t> sizes, part0;  // part0[t]: first part of tensor t, part0[num_tensors] their number
  int32_t param_type, grad_type, state_bits, rounding;
  double beta1, beta2, eps;
  uint64_t seed, step = 0;
  AdamDev dev;
};

namespace {

struct AdamPlan {
  std::vector<AdamTensor> tensors;
  std::vector<AdamPart> parts;
  std::vector<int64_t> part0;
  int64_t elements = 0;
  size_t o_first, o_second, o_scale1, o_scale2, o_tensors, o_parts, bytes;
};

int plan_adamw(const emb_adamw_config* c, AdamPlan* p) {
  if (!c || c->num_tensors < 1 || !c->sizes) return EMB_EINVAL;
  if (c->param_type != EMB_TYPE_FP32 && c->param_type != EMB_TYPE_BF16) return EMB_EINVAL;
  if (!type_ok(c->grad_type) || !rounding_ok(c->rounding)) return EMB_EINVAL;
  if (c->state_bits != 32 && c->state_bits != 8) return EMB_EINVAL;
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0)) return EMB_EINVAL;
  if (!(c->eps >= 0.0) || !std::isfinite(c->eps)) return EMB_EINVAL;
  int64_t parts = 0;
  for (int t = 0; t < c->num_tensors; ++t) {
    const int64_t n = c->sizes[t];
    const double wd = c->weight_decays ? c->weight_decays[t] : c->weight_decay;
    if (n < 0 || n > ((int64_t)1 << 40) || !std::isfinite(wd)) return EMB_EINVAL;
    p->tensors.push_back({p->elements, n, wd});
    p->part0.push_back(parts);
    parts += (n + kAdamChunk - 1) / kAdamChunk;
    p->elements += (n + kBlock - 1) / kBlock * kBlock;
    if (p->elements > ((int64_t)1 << 40) || parts >= ((int64_t)1 << 31)) return EMB_EINVAL;
  }
  p->part0.push_back(parts);
  const size_t each = c->state_bits == 32 ? 4 : 1, n = (size_t)p->elements;
  const size_t scales = c->state_bits == 32 ? 0 : n / kBlock;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o = align_up(o + bytes);
    return at;
  };
  p->o_first = take(n * each);
  p->o_second = take(n * each);
  p->o_scale1 = take(scales);
  p->o_scale2 = take(scales);
  p->o_tensors = take(sizeof(AdamTensor) * (size_t)c->num_tensors);
  p->o_parts = take(sizeof(AdamPart) * (size_t)parts);
  p->bytes = o;
  return EMB_OK;
}

int quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld, void* by_rows, void* by_columns,
             int32_t rounding, uint64_t seed, uint32_t step, Mx4Stream draws, void* stream) {
  if (!type_ok(type) || !rounding_ok(rounding) || !dims_ok(rows, cols) || !dims_ok(cols, rows)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!matrix_ok(x, type, rows, cols, ld) || (!by_rows && !by_columns)) return EMB_EINVAL;
  if (!aligned(by_rows) || !aligned(by_columns)) return EMB_EINVAL;
  const uintptr_t r = reinterpret_cast<uintptr_t>(by_rows), c = reinterpret_cast<uintptr_t>(by_columns);
  if (r && c && r < c + (uintptr_t)Mx4(nullptr, cols, rows).bytes() && c < r + (uintptr_t)Mx4(nullptr, rows, cols).bytes())
    return EMB_EINVAL;   // one kernel writes both
  return status(launch_quantize(x, type, rows, cols, ld, by_rows, by_columns, rounding, seed, step, draws, S(stream)));
}

}  // namespace

extern "C" {

int emb_mx4_query_bytes(int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes || !dims_ok(rows, cols)) return EMB_EINVAL;
  *bytes = rows && cols ? (size_t)Mx4(nullptr, rows, cols).bytes() : 0;
  return EMB_OK;
}

int emb_mx4_quantize(const void* x, int32_t type, int64_t rows, int64_t cols, int64_t ld, void* by_rows,
                     void* by_columns, int32_t rounding, uint64_t seed, uint32_t step, void* stream) {
  return quantize(x, type, rows, cols, ld, by_rows, by_columns, rounding, seed, step, kStreamMatrix, stream);
}

int emb_mx4_dequantize(const void* q, int64_t rows, int64_t cols, void* x, int32_t type, int64_t ld, void* stream) {
  if (!type_ok(type) || !dims_ok(rows, cols)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!q || !aligned(q) || !matrix_ok(x, type, rows, cols, ld)) return EMB_EINVAL;
  return status(launch_dequantize(q, rows, cols, x, type, ld, S(stream)));
}

int emb_mx4_pack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* q, void* stream) {
  if (!dims_ok(rows, cols)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!codes || !scales || !q || !aligned(q)) return EMB_EINVAL;
  return status(launch_pack(codes, scales, rows, cols, q, S(stream)));
}

int emb_mx4_unpack(const void* q, int64_t rows, int64_t cols, uint8_t* codes, uint8_t* scales, void* stream) {
  if (!dims_ok(rows, cols)) return EMB_EINVAL;
  if (rows == 0 || cols == 0) return EMB_OK;
  if (!codes || !scales || !q || !aligned(q)) return EMB_EINVAL;
  return status(launch_unpack(q, rows, cols, codes, scales, S(stream)));
}

int emb_mx4_matmul(const void* a, const void* b, int64_t m, int64_t n, int64_t k, void* c, int32_t type, int64_t ldc,
                   void* stream) {
  if (!type_ok(type) || !product_ok(m, n, k)) return EMB_EINVAL;
  if (m == 0 || n == 0) return EMB_OK;
  if (!matrix_ok(c, type, m, n, ldc)) return EMB_EINVAL;
  if (k && (!a || !b || !aligned(a) || !aligned(b))) return EMB_EINVAL;
  return status(launch_matmul(a, b, m, n, k, c, type, ldc, S(stream)));
}

int emb_mx4_linear_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes || !product_ok(m, n, k)) return EMB_EINVAL;
  *bytes = m && n && k ? linear_workspace(m, n, k) : 0;
  return EMB_OK;
}

int emb_mx4_linear(const void* x, int32_t type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n, void* y,
                   int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  if (!type_ok(type) || !product_ok(m, n, k)) return EMB_EINVAL;
  if (m == 0 || n == 0) return EMB_OK;
  if (!matrix_ok(y, type, m, n, ldy)) return EMB_EINVAL;
  if (k && (!matrix_ok(x, type, m, k, ldx) || !w || !aligned(w))) return EMB_EINVAL;
  const size_t need = k ? linear_workspace(m, n, k) : 0;
  if (need && (!workspace || !aligned(workspace))) return EMB_EINVAL;
  if (workspace_bytes < need) return EMB_ENOMEM;
  if (k && !need && share_elements(x, m, k, ldx, y, m, n, ldy, type_bytes(type))) return EMB_EINVAL;
  return status(launch_linear(x, type, m, k, ldx, w, n, y, ldy, workspace, S(stream)));
}

int emb_mx4_linear_train_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes || !product_ok(m, n, k) || !dims_ok(k, m)) return EMB_EINVAL;
  *bytes = m && k ? (size_t)Mx4(nullptr, m, k).bytes() : 0;
  return EMB_OK;
}

int emb_mx4_linear_train(const void* x, int32_t type, int64_t m, int64_t k, int64_t ldx, const void* w, int64_t n,
                         void* y, int64_t ldy, void* saved, int32_t rounding, uint64_t seed, uint32_t step,
                         void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  if (emb_mx4_linear_train_workspace(m, n, k, &need) != EMB_OK) return EMB_EINVAL;
  if (need && (!workspace || !aligned(workspace) || !saved)) return EMB_EINVAL;
  if (m && n && (!type_ok(type) || !matrix_ok(y, type, m, n, ldy) || (k && (!w || !aligned(w))))) return EMB_EINVAL;
  if (workspace_bytes < need) return EMB_ENOMEM;
  const int st = quantize(x, type, m, k, ldx, workspace, saved, rounding, seed, step, kStreamTrainRows, stream);
  return st != EMB_OK ? st : emb_mx4_matmul(workspace, w, m, n, k, y, type, ldy, stream);
}

int emb_mx4_linear_grad_workspace(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes || !product_ok(m, k, n) || !product_ok(n, k, m)) return EMB_EINVAL;
  *bytes = m && n ? align_up((size_t)Mx4(nullptr, m, n).bytes()) + (size_t)Mx4(nullptr, n, m).bytes() : 0;
  return EMB_OK;
}

int emb_mx4_linear_grad(const void* dy, int32_t type, int64_t m, int64_t n, int64_t ldy, const void* w_columns, int64_t k,
                        const void* saved, void* dx, int64_t ldx, void* dw, int32_t dw_type, int64_t ldw,
                        int32_t rounding, uint64_t seed, uint32_t step, void* workspace, size_t workspace_bytes,
                        void* stream) {
  size_t need = 0;
  if (emb_mx4_linear_grad_workspace(m, n, k, &need) != EMB_OK || !type_ok(type) || !type_ok(dw_type)) return EMB_EINVAL;
  if (need && (!workspace || !aligned(workspace))) return EMB_EINVAL;
  if (m && k && (!matrix_ok(dx, type, m, k, ldx) || (n && (!w_columns || !aligned(w_columns))))) return EMB_EINVAL;
  if (n && k && (!matrix_ok(dw, dw_type, n, k, ldw) || (m && (!saved || !aligned(saved))))) return EMB_EINVAL;
  if (workspace_bytes < need) return EMB_ENOMEM;
  uint8_t* rows = static_cast<uint8_t*>(workspace);
  uint8_t* columns = need ? rows + align_up((size_t)Mx4(nullptr, m, n).bytes()) : nullptr;
  const int st = quantize(dy, type, m, n, ldy, rows, columns, rounding, seed, step, kStreamMatrix, stream);
  if (st != EMB_OK) return st;
  return status(launch_two_products(rows, w_columns, m, k, n, dx, type, ldx, columns, saved, n, k, m, dw, dw_type, ldw, S(stream)));
}

int emb_adamw_query_sizes(const emb_adamw_config* cfg, emb_adamw_sizes* out) {
  if (!out) return EMB_EINVAL;
  try {
    AdamPlan p;
    const int st = plan_adamw(cfg, &p);
    if (st != EMB_OK) return st;
    *out = {p.bytes, p.elements, p.o_first, p.o_second, p.o_scale1, p.o_scale2};
    return EMB_OK;
  } catch (const std::bad_alloc&) {
    return EMB_EINVAL;
  }
}

int emb_adamw_create(const emb_adamw_config* cfg, void* state, size_t state_bytes, void* stream, emb_adamw_t* out) {
  if (!out) return EMB_EINVAL;
  *out = nullptr;
  emb_adamw* h = nullptr;
  try {
    AdamPlan p;
    const int st = plan_adamw(cfg, &p);
    if (st != EMB_OK) return st;
    if (!state || !aligned(state)) return EMB_EINVAL;
    if (state_bytes < p.bytes) return EMB_ENOMEM;
    int64_t parts = p.part0.back();
    p.parts.reserve((size_t)parts);
    for (int t = 0; t < cfg->num_tensors; ++t)
      for (int64_t k = p.part0[t]; k < p.part0[t + 1]; ++k)
        p.parts.push_back({(uint32_t)t, (uint32_t)(k - p.part0[t])});
    h = new emb_adamw();
    h->sizes.assign(cfg->sizes, cfg->sizes + cfg->num_tensors);
    h->part0 = p.part0;
    h->param_type = cfg->param_type;
    h->grad_type = cfg->grad_type;
    h->state_bits = cfg->state_bits;
    h->rounding = cfg->rounding;
    h->beta1 = cfg->beta1;
    h->beta2 = cfg->beta2;
    h->eps = cfg->eps;
    h->seed = cfg->seed;
    uint8_t* b = static_cast<uint8_t*>(state);
    h->dev = {reinterpret_cast<const AdamTensor*>(b + p.o_tensors), reinterpret_cast<const AdamPart*>(b + p.o_parts),
              b + p.o_first, b + p.o_second, b + p.o_scale1, b + p.o_scale2};
    hipError_t e = hipMemsetAsync(b, 0, p.o_tensors, S(stream));
    if (e == hipSuccess)
      e = hipMemcpyAsync(b + p.o_tensors, p.tensors.data(), sizeof(AdamTensor) * p.tensors.size(),
                         hipMemcpyHostToDevice, S(stream));
    if (e == hipSuccess && !p.parts.empty())
      e = hipMemcpyAsync(b + p.o_parts, p.parts.data(), sizeof(AdamPart) * p.parts.size(), hipMemcpyHostToDevice,
                         S(stream));
    const hipError_t done = hipStreamSynchronize(S(stream));  // the host arrays go now
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

int emb_adamw_destroy(emb_adamw_t h) {
  delete h;
  return EMB_OK;
}

int emb_adamw_step(emb_adamw_t h, void* const* params, const void* const* grads, double lr, const float* grad_scale,
                   void* stream) {
  if (!h || !params || !grads || !std::isfinite(lr) || reinterpret_cast<uintptr_t>(grad_scale) % 4) return EMB_EINVAL;
  const int T = (int)h->sizes.size();
  const size_t pb = type_bytes(h->param_type), gb = type_bytes(h->grad_type);
  for (int t = 0; t < T; ++t) {
    if (!h->sizes[t] || !grads[t]) continue;
    if (!params[t] || reinterpret_cast<uintptr_t>(params[t]) % pb || reinterpret_cast<uintptr_t>(grads[t]) % gb)
      return EMB_EINVAL;
  }
  const double t = (double)(h->step + 1);
  AdamConst c;
  c.beta1 = (float)h->beta1;
  c.beta2 = (float)h->beta2;
  c.rest1 = (float)(1.0 - h->beta1);
  c.rest2 = (float)(1.0 - h->beta2);
  c.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
  c.eps = (float)h->eps;
  c.rate = (float)(lr / (1.0 - std::pow(h->beta1, t)));
  c.lr = lr;
  c.k0 = (uint32_t)h->seed;
  c.k1 = (uint32_t)(h->seed >> 32);
  c.t = (uint32_t)(h->step + 1);
  for (int first = 0; first < T; first += kAdamTensors) {
    const int n = T - first < kAdamTensors ? T - first : kAdamTensors;
    const int64_t part0 = h->part0[first], parts = h->part0[first + n] - part0;
    if (!parts) continue;
    AdamPointers ptr;
    for (int k = 0; k < kAdamTensors; ++k) {
      ptr.p[k] = k < n ? params[first + k] : nullptr;
      ptr.g[k] = k < n ? grads[first + k] : nullptr;
    }
    const hipError_t e = in_launches(parts, kAdamThreads, [&](int64_t from, unsigned some) {
      return launch_adamw(h->dev, ptr, (uint32_t)first, part0 + from, some, c, grad_scale, h->param_type, h->grad_type,
                          h->state_bits, h->rounding, S(stream));
    });
    if (e != hipSuccess) return EMB_EHIP;
  }
  h->step += 1;
  return EMB_OK;
}

int emb_adamw_get_step(emb_adamw_t h, uint64_t* step) {
  if (!h || !step) return EMB_EINVAL;
  *step = h->step;
  return EMB_OK;
}

int emb_adamw_set_step(emb_adamw_t h, uint64_t step) {
  if (!h || step > kMaxStep) return EMB_EINVAL;
  h->step = step;
  return EMB_OK;
}

}  // extern "C"
