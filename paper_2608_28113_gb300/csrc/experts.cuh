// experts.cuh -- what the kernels of a mixture of experts share: its weights, the grouping of its tokens, its
// activations.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "hscale_device.cuh"
#include "nvfp4_weight.cuh"

namespace hscale {

// One NVFP4 matrix per expert: packed [experts, rows, cols / 2], codes [experts, rows, cols / 16], scale [experts].
struct ExpertMatrix {
  const uint8_t* packed;
  const uint8_t* codes;
  const float* scale;
};

// gate and up [inner, n], down [n, inner] of each expert.
struct Experts {
  ExpertMatrix gate, up, down;
  int64_t n, inner;
  int32_t count, activation;
};

// Slot t k + j is token t's j-th expert.  An id outside [0, experts) is none.
struct Routing {
  const int32_t* ids;
  const float* weights;
  int64_t tokens;
  int32_t k;
};

// The slots grouped by their experts (experts.cu): slot_of[pos], the experts one after another, slots ascending; chunks of
// at most `width` positions of one expert.
struct Chunk {
  int32_t expert, first, count, pad;
};
struct Plan {
  int32_t* header;  // chunks, positions
  Chunk* chunks;
  int32_t* slot_of;
};
inline __host__ __device__ int64_t plan_chunks(int64_t slots, int64_t experts, int64_t width) {
  return (slots < experts ? slots : experts) + slots / width;
}

constexpr int kActSilu = 0, kActGeluTanh = 1;

// act(g) = g s(q) with s the logistic function and q = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (the tanh form of
// gelu); approximate exponential and quotient (some 2^-20), for values that are rounded to 16 bits next.
__device__ __forceinline__ float activate_fast(int kind, float g) {
  const float q = kind == kActSilu ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
  return __fdividef(g, 1.0f + __expf(-q));
}
// act(g) and its derivative, in fp32 throughout.
__device__ __forceinline__ float2 activate(int kind, float g) {
  const float q = kind == kActSilu ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
  const float dq = kind == kActSilu ? 1.0f : 1.5957691216057308f * fmaf(0.134145f * g, g, 1.0f);
  const float e = expf(-fabsf(q)), part = 1.0f / (1.0f + e), other = e * part;
  const float s = q >= 0.0f ? part : other, rest = q >= 0.0f ? other : part;
  const float slope = rest > 0.0f ? g * dq * s * rest : 0.0f;  // rest or s may be 0 where dq is infinite
  return make_float2(g * s, s > 0.0f ? s + slope : 0.0f);
}

}  // namespace hscale
