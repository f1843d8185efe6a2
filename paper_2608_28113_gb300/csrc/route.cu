// route.cu -- the router of a mixture of experts, and its gradient.
//   p = softmax(l),  ids = the k largest l in descending order (ties: the lowest index first),
//   w_j = p_j, or p_j / sum of the chosen p (renormalized);
//   backward, over all experts:    dl_e = p_e ([e chosen] dw_e - sum_j w_j dw_j)
//             over the chosen ones: dl_j = w_j (dw_j - sum_i w_i dw_i), 0 elsewhere.
// -Inf and NaN are experts that are switched off: never chosen, p = 0.  +Inf counts as the type's largest finite number.
//
// One warp a token, its logits in registers (up to 1024).  A choice is two warp-wide integer reductions: the largest key
// (a float's bits, ordered as integers) and the lowest index that has it.  Up to 256 bf16 logits go another way: a
// logit's 16 bits and its index make one word, each lane sorts its eight, and a choice is one reduction over the
// lanes' first ones (16384 tokens of 256, k 8: 17.5 us before, 9.6 now).  Bound by these instructions, 439 a token: the ALU pipe is
// busy 81 % of the active cycles, the bytes are 9.4 MB, 1.4 us at the card's bandwidth.  In fp32 the same take 15.4 us.  From 257
// experts on there is one instance, of 32 logits a lane: 16384 tokens of 512 take 46 us (bf16) and 66 (fp32), of 1024 86 and
// 104; the gradient over all experts of 256, 512 and 1024 15, 69 and 120 us (bf16).  Sums and exponentials are fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cfloat>
#include <cstdint>

#include "hscale_internal.h"

namespace hscale {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr uint32_t kAll = 0xFFFFFFFFu;

template <typename T>
__device__ __forceinline__ float as_float(T v);
template <>
__device__ __forceinline__ float as_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A logit's key: larger floats have larger keys, -0 is 0, and 0 stands for an expert that is off.
template <typename T>
__device__ __forceinline__ uint32_t key_of(T logit) {
  const float v = as_float<T>(logit);
  if (!(v > -INFINITY)) return 0u;
  constexpr float kLargest = sizeof(T) == 2 ? 0x1.FEp127f : FLT_MAX;  // bf16's, fp32's
  const uint32_t b = __float_as_uint(fminf(v, kLargest) + 0.0f);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((key >> 31) ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

template <typename T, int kPer>
__device__ __forceinline__ void load_keys(const T* row, int experts, int lane, uint32_t (&key)[kPer]) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 32 * i;
    key[i] = e < experts ? key_of<T>(row[e]) : 0u;
  }
}

template <typename T, int kPer>
__global__ void __launch_bounds__(kThreads) route_kernel(const T* __restrict__ logits, int64_t tokens, int experts, int64_t ld,
                                                         int k, bool renormalize, int32_t* __restrict__ ids,
                                                         float* __restrict__ weights) {
  const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= tokens) return;
  uint32_t key[kPer];
  load_keys<T, kPer>(logits + t * ld, experts, lane, key);
  uint32_t mine = 0u;  // lane j: the j-th choice
  int mine_at = -1;
  float top = 0.0f, total = 0.0f;
  for (int j = 0; j < k; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) best = max(best, key[i]);
    best = __reduce_max_sync(kAll, best);
    if (j == 0) {
      top = value_of(best);
      if (!renormalize) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s += key[i] ? expf(value_of(key[i]) - top) : 0.0f;
        total = warp_sum(s);
      }
    }
    if (best == 0u) break;  // no expert is left
    uint32_t at = kAll;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i)
      if (key[i] == best) at = (uint32_t)(lane + 32 * i);
    at = __reduce_min_sync(kAll, at);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (at == (uint32_t)(lane + 32 * i)) key[i] = 0u;
    if (lane == j) mine = best, mine_at = (int)at;
  }
  const float p = mine ? expf(value_of(mine) - top) : 0.0f;
  if (renormalize) total = warp_sum(p);
  if (lane < k) {
    ids[t * k + lane] = mine_at;
    weights[t * k + lane] = mine ? p / total : 0.0f;
  }
}

// ---------------------------------------------------------------- up to 256 bf16 logits
// A logit and its index as one word: larger logits have larger words, of equal ones the lower index; 0: an expert that
// is off.
__device__ __forceinline__ uint32_t word_of(uint32_t bits, int e) {
  if (bits == 0x8000u) bits = 0u;                                      // -0
  if ((bits & 0x7FFFu) > 0x7F80u || bits == 0xFF80u) return 0u;        // NaN, -Inf
  const uint32_t key = (bits & 0x8000u) ? ~bits & 0xFFFFu : min(bits, 0x7F7Fu) | 0x8000u;
  return key << 16 | (uint32_t)(0xFFFF - e);
}
__device__ __forceinline__ float value_of_word(uint32_t w) {
  const uint32_t key = w >> 16;
  return __uint_as_float((key & 0x8000u ? key & 0x7FFFu : ~key & 0xFFFFu) << 16);
}
__device__ __forceinline__ void order(uint32_t& a, uint32_t& b) {  // the larger first
  const uint32_t hi = max(a, b), lo = min(a, b);
  a = hi, b = lo;
}
template <int kPer>
__device__ __forceinline__ void sort_words(uint32_t (&w)[kPer]) {
  if constexpr (kPer == 2) order(w[0], w[1]);
  if constexpr (kPer >= 4) {
#pragma unroll
    for (int o = 0; o < kPer; o += 4) {
      order(w[o], w[o + 1]), order(w[o + 2], w[o + 3]);
      order(w[o], w[o + 2]), order(w[o + 1], w[o + 3]);
      order(w[o + 1], w[o + 2]);
    }
  }
  if constexpr (kPer == 8) {  // two sorted fours merged (odd-even)
    order(w[0], w[4]), order(w[1], w[5]), order(w[2], w[6]), order(w[3], w[7]);
    order(w[2], w[4]), order(w[3], w[5]);
    order(w[1], w[2]), order(w[3], w[4]), order(w[5], w[6]);
  }
}

template <int kPer>
__global__ void __launch_bounds__(kThreads) route_words_kernel(const uint16_t* __restrict__ logits, int64_t tokens, int experts,
                                                               int64_t ld, int k, bool renormalize, int32_t* __restrict__ ids,
                                                               float* __restrict__ weights) {
  const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= tokens) return;
  const uint16_t* row = logits + t * ld;
  uint32_t w[kPer];
  const int e0 = lane * kPer;
  if (kPer == 8 && (reinterpret_cast<uintptr_t>(row) & 15) == 0 && e0 + 8 <= experts) {
    const uint4 v = *reinterpret_cast<const uint4*>(row + e0);
    const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < kPer; ++i) w[i] = word_of((q[i / 2] >> (16 * (i & 1))) & 0xFFFFu, e0 + i);
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) w[i] = e0 + i < experts ? word_of(row[e0 + i], e0 + i) : 0u;
  }
  sort_words<kPer>(w);
  uint32_t mine = 0u;  // lane j: the j-th choice
  float top = 0.0f, total = 0.0f;
  for (int j = 0; j < k; ++j) {
    const uint32_t best = __reduce_max_sync(kAll, w[0]);
    if (j == 0) {
      top = value_of_word(best);
      if (!renormalize) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) s += w[i] ? expf(value_of_word(w[i]) - top) : 0.0f;
        total = warp_sum(s);
      }
    }
    if (best == 0u) break;  // no expert is left
    if (lane == j) mine = best;
    const bool taken = w[0] == best;
#pragma unroll
    for (int i = 0; i + 1 < kPer; ++i) w[i] = taken ? w[i + 1] : w[i];
    w[kPer - 1] = taken ? 0u : w[kPer - 1];
  }
  const float p = mine ? expf(value_of_word(mine) - top) : 0.0f;
  if (renormalize) total = warp_sum(p);
  if (lane < k) {
    ids[t * k + lane] = mine ? 0xFFFF - (int)(mine & 0xFFFFu) : -1;
    weights[t * k + lane] = mine ? p / total : 0.0f;
  }
}

template <typename T, int kPer>
__global__ void __launch_bounds__(kThreads)
route_backward_kernel(const T* logits, int64_t tokens, int experts, int64_t ld, const int32_t* __restrict__ ids,
                      const float* __restrict__ weights, const float* __restrict__ dweights, int k, bool renormalize, T* dlogits,
                      int64_t ld_out) {
  __shared__ float row_of[kWarps][32 * kPer];
  const int64_t t = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= tokens) return;
  float* row = row_of[threadIdx.x >> 5];
#pragma unroll
  for (int i = 0; i < kPer; ++i) row[lane + 32 * i] = 0.0f;
  int id = lane < k ? ids[t * k + lane] : -1;
  if ((unsigned)id >= (unsigned)experts) id = -1;
  const float w = id >= 0 ? weights[t * k + lane] : 0.0f, dw = id >= 0 ? dweights[t * k + lane] : 0.0f;
  const float mean = warp_sum(id >= 0 ? w * dw : 0.0f);
  const float term = renormalize ? w * (dw - mean) : dw;
  __syncwarp();
  // an expert that a token has more than once gets the sum, in order
  const uint32_t alike = __match_any_sync(kAll, id);
  float sum = 0.0f;
  for (int j = 0; j < k; ++j) {
    const float v = __shfl_sync(kAll, term, j);
    if ((alike >> j) & 1u) sum += v;
  }
  if (id >= 0 && __ffs(alike) - 1 == lane) row[id] = sum;
  __syncwarp();
  T* out = dlogits + t * ld_out;
  if (renormalize) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (lane + 32 * i < experts) out[lane + 32 * i] = from_float<T>(row[lane + 32 * i]);
    return;
  }
  uint32_t key[kPer];
  load_keys<T, kPer>(logits + t * ld, experts, lane, key);
  uint32_t best = key[0];
#pragma unroll
  for (int i = 1; i < kPer; ++i) best = max(best, key[i]);
  const float top = value_of(__reduce_max_sync(kAll, best));
  float p[kPer], s = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    p[i] = key[i] ? expf(value_of(key[i]) - top) : 0.0f;
    s += p[i];
  }
  s = warp_sum(s);
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (lane + 32 * i < experts) out[lane + 32 * i] = from_float<T>(key[i] ? p[i] / s * (row[lane + 32 * i] - mean) : 0.0f);
}

template <typename T, int kPer>
cudaError_t launch(const void* logits, int64_t tokens, int64_t experts, int64_t ld, const int32_t* ids_in, const float* w_in,
                   const float* dweights, int64_t k, bool renormalize, int32_t* ids, float* weights, void* dlogits,
                   int64_t ld_out, cudaStream_t stream) {
  const unsigned grid = (unsigned)((tokens + kWarps - 1) / kWarps);
  if (dlogits != nullptr)
    route_backward_kernel<T, kPer><<<grid, kThreads, 0, stream>>>(static_cast<const T*>(logits), tokens, (int)experts, ld,
                                                                  ids_in, w_in, dweights, (int)k, renormalize,
                                                                  static_cast<T*>(dlogits), ld_out);
  else if constexpr (kPer <= 8 && sizeof(T) == 2)
    route_words_kernel<kPer><<<grid, kThreads, 0, stream>>>(static_cast<const uint16_t*>(logits), tokens, (int)experts, ld, (int)k,
                                                            renormalize, ids, weights);
  else
    route_kernel<T, kPer><<<grid, kThreads, 0, stream>>>(static_cast<const T*>(logits), tokens, (int)experts, ld, (int)k,
                                                         renormalize, ids, weights);
  return cudaGetLastError();
}

template <typename T, typename... Args>
cudaError_t by_size(const void* logits, int64_t tokens, int64_t experts, Args... args) {
  if (experts <= 32) return launch<T, 1>(logits, tokens, experts, args...);
  if (experts <= 64) return launch<T, 2>(logits, tokens, experts, args...);
  if (experts <= 128) return launch<T, 4>(logits, tokens, experts, args...);
  if (experts <= 256) return launch<T, 8>(logits, tokens, experts, args...);
  return launch<T, 32>(logits, tokens, experts, args...);
}

}  // namespace

cudaError_t launch_route(bool bf16, const void* logits, int64_t tokens, int64_t experts, int64_t ld, int64_t k,
                         bool renormalize, int32_t* ids, float* weights, cudaStream_t stream) {
  const int32_t* no_ids = nullptr;
  const float* none = nullptr;
  void* no_out = nullptr;
  return bf16 ? by_size<__nv_bfloat16>(logits, tokens, experts, ld, no_ids, none, none, k, renormalize, ids, weights, no_out,
                                       (int64_t)0, stream)
              : by_size<float>(logits, tokens, experts, ld, no_ids, none, none, k, renormalize, ids, weights, no_out, (int64_t)0,
                               stream);
}

cudaError_t launch_route_backward(bool bf16, const void* logits, int64_t tokens, int64_t experts, int64_t ld, const int32_t* ids,
                                  const float* weights, const float* dweights, int64_t k, bool renormalize, void* dlogits,
                                  int64_t ld_out, cudaStream_t stream) {
  int32_t* no_ids = nullptr;
  float* none = nullptr;
  return bf16 ? by_size<__nv_bfloat16>(logits, tokens, experts, ld, ids, weights, dweights, k, renormalize, no_ids, none, dlogits,
                                       ld_out, stream)
              : by_size<float>(logits, tokens, experts, ld, ids, weights, dweights, k, renormalize, no_ids, none, dlogits, ld_out,
                               stream);
}

}  // namespace hscale
