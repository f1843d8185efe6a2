// project.cu -- the product of activations with a packed NVFP4 weight, with each token's adapter added:
//   y_t  = W_hat x_t + B_a z_t        (forward;  z  = alpha_a A_a x_t,    adapter.cu)
//   dx_t = W_hat^T dy_t + A_a^T dz_t  (backward; dz = alpha_a B_a^T dy_t, adapter.cu)
// Accumulated in fp32 and rounded once, to bf16.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"

namespace hscale {
namespace {

// 64 tokens x 64 outputs a block, 16 of the summed axis a step, 4 x 4 outputs a thread.
// kForward: out[t, f] over k < n; else out[t, j] over f < m.
template <bool kForward>
__global__ void __launch_bounds__(256)
project_kernel(const uint16_t* __restrict__ v, int64_t tokens, int64_t ld_v, Nvfp4Weight w, Adapters ad, const float* z,
               __nv_bfloat16* out, int64_t ld_out) {
  __shared__ float sv[16][65], sw[16][65];
  const int64_t outs = kForward ? w.m : w.n, depth = kForward ? w.n : w.m;
  const int64_t t0 = (int64_t)blockIdx.y * 64, o0 = (int64_t)blockIdx.x * 64;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < depth; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int k = i & 15, t = i >> 4;
      sv[k][t] = t0 + t < tokens && k0 + k < depth ? __uint_as_float((uint32_t)v[(t0 + t) * ld_v + k0 + k] << 16) : 0.0f;
      const int kk = kForward ? k : i >> 6, oo = kForward ? t : i & 63;
      const int64_t f = kForward ? o0 + oo : k0 + kk, c = kForward ? k0 + kk : o0 + oo;
      float q = 0.0f;
      if (f < w.m && c < w.n) {
        const uint32_t nib = (w.packed[f * (w.n / 2) + c / 2] >> (4 * (c & 1))) & 15u;
        q = e4m3_mag(ladder_code(w.codes[f * (w.n / 16) + c / 16])) * e2m1_from_raw((nib & 7u) << 22);
        if (nib & 8u) q = -q;
      }
      sw[kk][oo] = q;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sv[k][ty + 16 * i], sw[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
  const float sg = *w.global_scale;
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + ty + 16 * i;
    if (t >= tokens) continue;
    const int a = adapter_of(ad, t);
    for (int j = 0; j < 4; ++j) {
      const int64_t o = o0 + tx + 16 * j;
      if (o >= outs) continue;
      float s = acc[i][j] * sg;
      if (a >= 0) {
        float low = 0.0f;
        for (int r = 0; r < ad.rank; ++r) {
          const int64_t e = kForward ? ((int64_t)a * w.m + o) * ad.rank + r : ((int64_t)a * ad.rank + r) * w.n + o;
          low = fmaf(z[t * ad.rank + r], __bfloat162float((kForward ? ad.b : ad.a)[e]), low);
        }
        s += low;
      }
      out[t * ld_out + o] = __float2bfloat16_rn(s);
    }
  }
}

}  // namespace

cudaError_t launch_project(bool forward, const void* v, int64_t tokens, int64_t ld_v, const Nvfp4Weight& w, const Adapters& ad,
                           const float* z, void* out, int64_t ld_out, cudaStream_t stream) {
  const dim3 grid((unsigned)(((forward ? w.m : w.n) + 63) / 64), (unsigned)((tokens + 63) / 64));
  if (forward)
    project_kernel<true><<<grid, 256, 0, stream>>>((const uint16_t*)v, tokens, ld_v, w, ad, z, (__nv_bfloat16*)out, ld_out);
  else
    project_kernel<false><<<grid, 256, 0, stream>>>((const uint16_t*)v, tokens, ld_v, w, ad, z, (__nv_bfloat16*)out, ld_out);
  return cudaGetLastError();
}

}  // namespace hscale
