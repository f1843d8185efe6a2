// adapter.cu -- the low-rank adapters' own products beside a projection (project.cu):
//   z  = alpha_a A_a x_t       dz = alpha_a B_a^T dy_t        for every token t of an adapter a
//   dA = sum_t dz_t x_t^T      dB = sum_t dy_t z_t^T          over the tokens of each adapter
// z and dz are fp32 [tokens, rank]; rows of tokens without an adapter are left as they are.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"

namespace hscale {
namespace {

// Rows of activations: bf16 (kFormat -1) or a checkpoint.
template <int kFormat>
struct Rows {
  const uint16_t* x;
  int64_t ld;
  Checkpoint ckpt;
  __device__ __forceinline__ float at(int64_t t, int64_t k) const {
    if constexpr (kFormat < 0) {
      return __uint_as_float((uint32_t)x[t * ld + k] << 16);
    } else {
      return ckpt_element<kFormat>(ckpt.codes[t * ckpt.ld_codes + k]) * ckpt_scale(ckpt.scales[t * ckpt.ld_scales + k / kCkptBlock]);
    }
  }
};

// One warp per token.  kDown: z = alpha A x over n; else dz = alpha B^T dy over m.
template <int kFormat, bool kDown>
__global__ void __launch_bounds__(128)
shrink_kernel(Rows<kFormat> rows, int64_t tokens, int64_t cols, Adapters ad, float* z) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= tokens) return;
  const int a = adapter_of(ad, t);
  if (a < 0) return;
  for (int r = 0; r < ad.rank; ++r) {
    float s = 0.0f;
    for (int64_t k = lane; k < cols; k += 32) {
      const int64_t w = kDown ? ((int64_t)a * ad.rank + r) * cols + k : ((int64_t)a * cols + k) * ad.rank + r;
      s = fmaf(rows.at(t, k), __bfloat162float((kDown ? ad.a : ad.b)[w]), s);
    }
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, off);
    if (lane == 0) z[t * ad.rank + r] = s * ad.alpha[a];
  }
}

// One thread per entry of dA (kRankMajor: [rank, cols]) or dB ([cols, rank]).
template <int kFormat, bool kRankMajor>
__global__ void __launch_bounds__(256)
grad_kernel(Rows<kFormat> rows, int64_t tokens, int64_t cols, Adapters ad, const float* z, __nv_bfloat16* out) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int r = blockIdx.y % ad.rank, a = blockIdx.y / ad.rank;
  if (col >= cols) return;
  float s = 0.0f;
  for (int64_t t = 0; t < tokens; ++t)
    if (adapter_of(ad, t) == a) s = fmaf(z[t * ad.rank + r], rows.at(t, col), s);
  out[kRankMajor ? ((int64_t)a * ad.rank + r) * cols + col : ((int64_t)a * cols + col) * ad.rank + r] = __float2bfloat16_rn(s);
}

}  // namespace

cudaError_t launch_adapter_down(const void* x, int64_t ld_x, const Checkpoint* ckpt, int format, int64_t tokens, int64_t n,
                                const Adapters& ad, float* z, cudaStream_t stream) {
  const unsigned grid = (unsigned)((tokens + 3) / 4);
  if (ckpt == nullptr) shrink_kernel<-1, true><<<grid, 128, 0, stream>>>({(const uint16_t*)x, ld_x, {}}, tokens, n, ad, z);
  else if (format == kCkptInt8) shrink_kernel<kCkptInt8, true><<<grid, 128, 0, stream>>>({nullptr, 0, *ckpt}, tokens, n, ad, z);
  else shrink_kernel<kCkptE4M3, true><<<grid, 128, 0, stream>>>({nullptr, 0, *ckpt}, tokens, n, ad, z);
  return cudaGetLastError();
}

cudaError_t launch_adapter_up_t(const void* dy, int64_t ld_dy, int64_t tokens, int64_t m, const Adapters& ad, float* dz,
                                cudaStream_t stream) {
  shrink_kernel<-1, false><<<(unsigned)((tokens + 3) / 4), 128, 0, stream>>>({(const uint16_t*)dy, ld_dy, {}}, tokens, m, ad, dz);
  return cudaGetLastError();
}

cudaError_t launch_adapter_grad_a(const Checkpoint& ckpt, int format, int64_t tokens, int64_t n, const Adapters& ad,
                                  const float* dz, void* da, cudaStream_t stream) {
  const dim3 grid((unsigned)((n + 255) / 256), (unsigned)(ad.count * ad.rank));
  if (format == kCkptInt8) grad_kernel<kCkptInt8, true><<<grid, 256, 0, stream>>>({nullptr, 0, ckpt}, tokens, n, ad, dz, (__nv_bfloat16*)da);
  else grad_kernel<kCkptE4M3, true><<<grid, 256, 0, stream>>>({nullptr, 0, ckpt}, tokens, n, ad, dz, (__nv_bfloat16*)da);
  return cudaGetLastError();
}

cudaError_t launch_adapter_grad_b(const void* dy, int64_t ld_dy, int64_t tokens, int64_t m, const Adapters& ad, const float* z,
                                  void* db, cudaStream_t stream) {
  const dim3 grid((unsigned)((m + 255) / 256), (unsigned)(ad.count * ad.rank));
  grad_kernel<-1, false><<<grid, 256, 0, stream>>>({(const uint16_t*)dy, ld_dy, {}}, tokens, m, ad, z, (__nv_bfloat16*)db);
  return cudaGetLastError();
}

}  // namespace hscale
