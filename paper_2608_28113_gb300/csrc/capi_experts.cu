// capi_experts.cu -- the extern "C" boundary of the mixture-of-experts operators and of the gradients' norm.
//
// Every entry point validates its arguments on the host before enqueueing anything.  No exception crosses the ABI.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>

#include "../../include/hscale.h"
#include "experts.cuh"
#include "hscale_internal.h"

static_assert(HSCALE_ACT_SILU == hscale::kActSilu && HSCALE_ACT_GELU_TANH == hscale::kActGeluTanh, "activations");
static_assert(HSCALE_BF16 == hscale::kGradBF16 && HSCALE_F32 == hscale::kGradF32 && HSCALE_F16 == hscale::kGradF16, "types");

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int from_cuda(cudaError_t e) { return e == cudaSuccess ? HSCALE_OK : HSCALE_ERR_CUDA; }
inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

// tokens, experts and k of a routing
inline int check_routing(int64_t tokens, int64_t experts, int64_t k) {
  if (tokens < 0 || experts < 1 || experts > hscale::kRouteExperts || k < 1 || k > 32) return HSCALE_ERR_SHAPE;
  if (tokens > (int64_t)INT32_MAX / 32) return HSCALE_ERR_SHAPE;
  return HSCALE_OK;
}

inline int check_logits(const void* l, int32_t type, int64_t tokens, int64_t experts, int64_t ld) {
  if (type != HSCALE_BF16 && type != HSCALE_F32) return HSCALE_ERR_ARG;
  if (ld < experts || (tokens > 0 && ld > INT64_MAX / 4 / tokens)) return HSCALE_ERR_SHAPE;
  if (tokens == 0) return HSCALE_OK;
  if (l == nullptr) return HSCALE_ERR_NULL;
  return aligned(l, type == HSCALE_BF16 ? 2 : 4) ? HSCALE_OK : HSCALE_ERR_ALIGN;
}

// rows of bf16
inline int check_rows(const void* x, int64_t rows, int64_t cols, int64_t ld) {
  if (ld < cols || (rows > 0 && ld > INT64_MAX / 2 / rows)) return HSCALE_ERR_SHAPE;
  if (rows == 0 || cols == 0) return HSCALE_OK;
  if (x == nullptr) return HSCALE_ERR_NULL;
  return aligned(x, 16) && ld % 8 == 0 ? HSCALE_OK : HSCALE_ERR_ALIGN;
}

// Whether an int64 holds every product of these sizes and an int32 the number of tiles' blocks (128 x 128, four products of
// them at most); beyond it the operands are terabytes.
inline bool experts_fit(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  constexpr int64_t kMost = (int64_t)1 << 40;
  if (tokens > INT32_MAX / 32 || k > 32 || experts > hscale::kRouteExperts || n > INT32_MAX || inner > INT32_MAX / 2) return false;
  const int64_t slots = tokens * k, blocks = ((n + 127) / 128) * ((inner + 127) / 128);
  const int64_t chunks = hscale::plan_chunks(slots, experts, hscale::experts_width(slots, experts));
  return slots <= kMost / std::max(n, inner) && n <= (kMost << 10) / inner / experts && blocks <= INT32_MAX / 8 / chunks;
}

inline int check_experts(int64_t tokens, int64_t n, int64_t k, const int32_t* ids, const float* weights,
                         const hscale::Experts& w, int32_t activation) {
  if (activation != HSCALE_ACT_SILU && activation != HSCALE_ACT_GELU_TANH) return HSCALE_ERR_ARG;
  if (n < 0 || w.inner < 0 || n % 16 != 0 || w.inner % 16 != 0 || n > INT32_MAX || w.inner > INT32_MAX / 2) return HSCALE_ERR_SHAPE;
  if (tokens > 0 && n > 0 && w.inner > 0 && !experts_fit(tokens, k, n, w.inner, w.count)) return HSCALE_ERR_SHAPE;
  if (tokens == 0 || n == 0 || w.inner == 0) return HSCALE_OK;
  if (ids == nullptr || weights == nullptr) return HSCALE_ERR_NULL;
  if (!aligned(ids, 4) || !aligned(weights, 4)) return HSCALE_ERR_ALIGN;
  const hscale::ExpertMatrix* all[3] = {&w.gate, &w.up, &w.down};
  for (const hscale::ExpertMatrix* m : all)
    if (m->packed == nullptr || m->codes == nullptr || m->scale == nullptr) return HSCALE_ERR_NULL;
  for (const hscale::ExpertMatrix* m : all)
    if (!aligned(m->packed, 8) || !aligned(m->scale, 4)) return HSCALE_ERR_ALIGN;
  return HSCALE_OK;
}

inline cudaError_t zero_rows(void* x, int64_t rows, int64_t cols, int64_t ld, cudaStream_t stream) {
  return cudaMemset2DAsync(x, (size_t)ld * 2, 0, (size_t)cols * 2, (size_t)rows, stream);
}

// Whether no tensor that is written (out; nullptr: in) overlaps another one, written or read, and the norm none of them: out_i may
// be in_i itself.
// HSCALE_OK, HSCALE_ERR_ARG, or HSCALE_ERR_CUDA where the host has no memory for the list.
int written_apart(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int64_t count,
                  const float* norm) {
  struct Span {
    uintptr_t first, end;
    int64_t at;
  };
  const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[(size_t)std::max<int64_t>(count, 1)]);
  if (spans == nullptr) return HSCALE_ERR_CUDA;
  const auto span = [&](const void* p, int64_t i) {
    const uintptr_t first = reinterpret_cast<uintptr_t>(p);
    return Span{first, first + (uintptr_t)sizes[i] * (types[i] == HSCALE_F32 ? 4 : 2), i};
  };
  Span *const begin = spans.get(), *end = begin;
  bool ascending = true;  // as the parts of one buffer are
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    *end = span(out != nullptr ? out[i] : in[i], i);
    ascending = ascending && (end == begin || end[-1].first < end->first);
    ++end;
  }
  if (!ascending) std::sort(begin, end, [](const Span& a, const Span& b) { return a.first < b.first; });
  for (Span* s = begin; s + 1 < end; ++s)
    if (s->end > s[1].first) return HSCALE_ERR_ARG;
  // the first one written that ends behind an address
  const auto behind = [&](uintptr_t p) { return std::upper_bound(begin, end, p, [](uintptr_t p, const Span& v) { return p < v.end; }); };
  const uintptr_t norm_at = reinterpret_cast<uintptr_t>(norm);
  if (const Span* s = behind(norm_at); s != end && s->first < norm_at + 4) return HSCALE_ERR_ARG;
  if (out == nullptr) return HSCALE_OK;
  for (int64_t i = 0; i < count; ++i) {
    if (sizes[i] == 0) continue;
    const Span read = span(in[i], i);
    if (read.first < norm_at + 4 && norm_at < read.end) return HSCALE_ERR_ARG;
    // if the first one behind this one's beginning is its own place, the next one begins behind it
    const Span* s = behind(read.first);
    if (s != end && s->first < read.end && !(s->at == i && s->first == read.first)) return HSCALE_ERR_ARG;
  }
  return HSCALE_OK;
}

int grads(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int64_t count, bool clip,
          float max_norm, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  if (count < 0) return HSCALE_ERR_SHAPE;
  if (clip && !(max_norm >= 0.0f)) return HSCALE_ERR_ARG;
  if (norm == nullptr || (count > 0 && (in == nullptr || sizes == nullptr || types == nullptr))) return HSCALE_ERR_NULL;
  if (!aligned(norm, 4)) return HSCALE_ERR_ALIGN;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (types[i] != HSCALE_BF16 && types[i] != HSCALE_F32 && types[i] != HSCALE_F16) return HSCALE_ERR_ARG;
    if (sizes[i] < 0 || sizes[i] > ((int64_t)1 << 42) || (total += sizes[i]) > ((int64_t)1 << 50)) return HSCALE_ERR_SHAPE;
    if (sizes[i] == 0) continue;
    if (in[i] == nullptr || (out != nullptr && out[i] == nullptr)) return HSCALE_ERR_NULL;
    const uintptr_t size = types[i] == HSCALE_F32 ? 4 : 2;
    if (!aligned(in[i], size) || (out != nullptr && !aligned(out[i], size))) return HSCALE_ERR_ALIGN;
  }
  if (workspace == nullptr || workspace_bytes < hscale_grad_norm_workspace_bytes() || !aligned(workspace, 256)) return HSCALE_ERR_WORKSPACE;
  if (clip)
    if (const int st = written_apart(in, out, sizes, types, count, norm); st != HSCALE_OK) return st;
  return from_cuda(hscale::launch_grad_norm(in, out, sizes, types, count, clip, max_norm, norm, static_cast<double*>(workspace),
                                            as_stream(stream)));
}

}  // namespace

extern "C" {

int hscale_route(const void* logits, int32_t type, int64_t tokens, int64_t experts, int64_t ld_logits, int64_t k,
                 int32_t renormalize, int32_t* ids, float* weights, void* stream) {
  int st = check_routing(tokens, experts, k);
  if (st == HSCALE_OK) st = check_logits(logits, type, tokens, experts, ld_logits);
  if (st != HSCALE_OK || tokens == 0) return st;
  if (ids == nullptr || weights == nullptr) return HSCALE_ERR_NULL;
  if (!aligned(ids, 4) || !aligned(weights, 4)) return HSCALE_ERR_ALIGN;
  return from_cuda(hscale::launch_route(type == HSCALE_BF16, logits, tokens, experts, ld_logits, k, renormalize != 0, ids, weights,
                                        as_stream(stream)));
}

int hscale_route_backward(const void* logits, int32_t type, int64_t tokens, int64_t experts, int64_t ld_logits,
                          const int32_t* ids, const float* weights, const float* dweights, int64_t k, int32_t renormalize,
                          void* dlogits, int64_t ld_dlogits, void* stream) {
  int st = check_routing(tokens, experts, k);
  if (st == HSCALE_OK && renormalize == 0) st = check_logits(logits, type, tokens, experts, ld_logits);
  if (st == HSCALE_OK) st = check_logits(dlogits, type, tokens, experts, ld_dlogits);
  if (st != HSCALE_OK || tokens == 0) return st;
  if (ids == nullptr || weights == nullptr || dweights == nullptr) return HSCALE_ERR_NULL;
  if (!aligned(ids, 4) || !aligned(weights, 4) || !aligned(dweights, 4)) return HSCALE_ERR_ALIGN;
  return from_cuda(hscale::launch_route_backward(type == HSCALE_BF16, logits, tokens, experts, ld_logits, ids, weights, dweights,
                                                 k, renormalize != 0, dlogits, ld_dlogits, as_stream(stream)));
}

size_t hscale_experts_workspace_bytes(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  if (tokens <= 0 || k <= 0 || n <= 0 || inner <= 0 || experts <= 0) return 0;
  if (!experts_fit(tokens, k, n, inner, experts)) return SIZE_MAX;  // which no call takes
  return (size_t)hscale::experts_workspace(tokens, k, n, inner, experts);
}

int hscale_experts(const void* x_bf16, int64_t tokens, int64_t n, int64_t ld_x, const int32_t* ids, const float* weights,
                   int64_t k, const uint8_t* gate_packed, const uint8_t* gate_codes, const float* gate_scale,
                   const uint8_t* up_packed, const uint8_t* up_codes, const float* up_scale, const uint8_t* down_packed,
                   const uint8_t* down_codes, const float* down_scale, int64_t experts, int64_t inner, int32_t activation,
                   void* y_bf16, int64_t ld_y, void* workspace, size_t workspace_bytes, void* stream) {
  const hscale::Experts w = {{gate_packed, gate_codes, gate_scale}, {up_packed, up_codes, up_scale},
                             {down_packed, down_codes, down_scale}, n, inner, (int32_t)experts, activation};
  int st = check_routing(tokens, experts, k);
  if (st == HSCALE_OK) st = check_experts(tokens, n, k, ids, weights, w, activation);
  if (st == HSCALE_OK) st = check_rows(x_bf16, tokens, n, ld_x);
  if (st == HSCALE_OK) st = check_rows(y_bf16, tokens, n, ld_y);
  if (st != HSCALE_OK || tokens == 0 || n == 0) return st;
  if (inner == 0) return from_cuda(zero_rows(y_bf16, tokens, n, ld_y, as_stream(stream)));
  if (workspace == nullptr || workspace_bytes < hscale_experts_workspace_bytes(tokens, k, n, inner, experts) ||
      !aligned(workspace, 256))
    return HSCALE_ERR_WORKSPACE;
  const hscale::Routing r = {ids, weights, tokens, (int32_t)k};
  return from_cuda(hscale::launch_experts(x_bf16, ld_x, r, w, y_bf16, ld_y, workspace, as_stream(stream)));
}

size_t hscale_experts_backward_workspace_bytes(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  if (tokens <= 0 || k <= 0 || n <= 0 || inner <= 0 || experts <= 0) return 0;
  if (!experts_fit(tokens, k, n, inner, experts)) return SIZE_MAX;  // which no call takes
  return (size_t)hscale::experts_backward_workspace(tokens, k, n, inner, experts);
}

int hscale_experts_backward(const void* dy_bf16, int64_t tokens, int64_t n, int64_t ld_dy, const void* x_bf16, int64_t ld_x,
                            const int32_t* ids, const float* weights, int64_t k, const uint8_t* gate_packed,
                            const uint8_t* gate_codes, const float* gate_scale, const uint8_t* up_packed,
                            const uint8_t* up_codes, const float* up_scale, const uint8_t* down_packed,
                            const uint8_t* down_codes, const float* down_scale, int64_t experts, int64_t inner,
                            int32_t activation, void* dx_bf16, int64_t ld_dx, float* dweights, void* workspace,
                            size_t workspace_bytes, void* stream) {
  const hscale::Experts w = {{gate_packed, gate_codes, gate_scale}, {up_packed, up_codes, up_scale},
                             {down_packed, down_codes, down_scale}, n, inner, (int32_t)experts, activation};
  int st = check_routing(tokens, experts, k);
  if (st == HSCALE_OK) st = check_experts(tokens, n, k, ids, weights, w, activation);
  if (st == HSCALE_OK) st = check_rows(dy_bf16, tokens, n, ld_dy);
  if (st == HSCALE_OK) st = check_rows(x_bf16, tokens, n, ld_x);
  if (st == HSCALE_OK && dx_bf16 != nullptr) st = check_rows(dx_bf16, tokens, n, ld_dx);
  if (st != HSCALE_OK) return st;
  if (!aligned(dweights, 4)) return HSCALE_ERR_ALIGN;
  if (tokens == 0) return HSCALE_OK;
  if (n == 0 || inner == 0) {
    // empty sums: the outputs that exist are zero
    cudaError_t err = cudaSuccess;
    if (dx_bf16 != nullptr && n > 0) err = zero_rows(dx_bf16, tokens, n, ld_dx, as_stream(stream));
    if (err == cudaSuccess && dweights != nullptr) err = cudaMemsetAsync(dweights, 0, (size_t)(tokens * k) * 4, as_stream(stream));
    return from_cuda(err);
  }
  if (workspace == nullptr || workspace_bytes < hscale_experts_backward_workspace_bytes(tokens, k, n, inner, experts) ||
      !aligned(workspace, 256))
    return HSCALE_ERR_WORKSPACE;
  if (dx_bf16 == nullptr && dweights == nullptr) return HSCALE_OK;
  const hscale::Routing r = {ids, weights, tokens, (int32_t)k};
  return from_cuda(hscale::launch_experts_backward(dy_bf16, ld_dy, x_bf16, ld_x, r, w, dx_bf16, ld_dx, dweights, workspace,
                                                   as_stream(stream)));
}

size_t hscale_grad_norm_workspace_bytes(void) { return hscale::kGradParts * sizeof(double); }

int hscale_grad_norm(const void* const* tensors, const int64_t* sizes, const int32_t* types, int64_t count, float* norm,
                     void* workspace, size_t workspace_bytes, void* stream) {
  return grads(tensors, nullptr, sizes, types, count, false, 0.0f, norm, workspace, workspace_bytes, stream);
}

int hscale_grad_clip(const void* const* tensors, const int64_t* sizes, const int32_t* types, int64_t count, float max_norm,
                     float* norm, void* const* out, void* workspace, size_t workspace_bytes, void* stream) {
  return grads(tensors, out, sizes, types, count, true, max_norm, norm, workspace, workspace_bytes, stream);
}

}  // extern "C"
