// checkpoint.cu -- activations kept in 8 bits between the passes of a training step.
//
// A row is cut into blocks of 32 channels.  With amax = f 2^p the block's largest magnitude, 1 <= f < 2:
//   INT8   E = p - 6,                        q = clamp(RNE(x 2^-E), -127, 127)
//   E4M3   E = p - 8, + 1 where f > 1.75,    q = RNE_E4M3(x 2^-E)          (so nothing exceeds 448)
// with E >= -124, stored as the byte E + 127.  Scaling by a power of two is exact, so each element is
// rounded once (and in the topmost E4M3 blocks, E = 120, held to +-240: 256 2^120 is past bf16's range).
// Both formats' values (7 and 4 significant bits times 2^E, multiples of 2^-133) are
// exact in bf16: a load is exact, and kernels that read a checkpoint may feed it to bf16 tensor cores.
// A block that holds Inf or NaN gets the byte 255 and loads as NaN.
//
// Bound by HBM: 2 B in and 1 + 1/32 B out per element for a save, the reverse for a load.  Four lanes
// share a block, 16 bytes of x each.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"

namespace hscale {
namespace {

constexpr int kThreads = 256;

// (row, block) of a flat unit index; 32-bit arithmetic where it reaches
__device__ __forceinline__ void unit_of(int64_t u, int64_t units, int blocks, int64_t& row, int& blk) {
  row = units <= UINT32_MAX ? (int64_t)((uint32_t)u / (uint32_t)blocks) : u / blocks;
  blk = (int)(u - row * blocks);
}

// RNE to INT8 or E4M3 of v = x 2^-E
template <int kFormat>
__device__ __forceinline__ uint32_t encode(float v) {
  if (kFormat == kCkptInt8) return (uint32_t)(uint8_t)(int8_t)__float2int_rn(v);
  uint16_t r;  // satfinite: +-448 at most, which no v exceeds
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
  return r & 0xFFu;
}

// kVec: rows of x are 16-byte and rows of codes 8-byte aligned
template <int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads)
checkpoint_save_kernel(const uint16_t* __restrict__ x, int64_t tokens, int64_t n, int64_t ld_x, int blocks,
                       uint8_t* __restrict__ codes, int64_t ld_codes, uint8_t* __restrict__ scales,
                       int64_t ld_scales) {
  const int64_t units = tokens * blocks;
  const int64_t lanes = (units * 4 + 31) / 32 * 32;  // whole warps take part in the shuffles
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < lanes; i += (int64_t)gridDim.x * kThreads) {
    const int64_t u = i >> 2;
    const bool on = u < units;
    int64_t row = 0;
    int blk = 0;
    if (on) unit_of(u, units, blocks, row, blk);
    const int64_t col = (int64_t)blk * kCkptBlock + (i & 3) * 8;
    const int have = on ? (int)max((int64_t)0, min((int64_t)8, n - col)) : 0;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    const uint16_t* src = x + row * ld_x + col;
    if (kVec && have == 8) {
      const uint4 v = ld_stream_v4(src);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < have) w[j >> 1] |= (uint32_t)src[j] << (16 * (j & 1));
    }
    uint32_t amax = 0;  // bf16 bit patterns order as magnitudes; NaN above Inf
#pragma unroll
    for (int j = 0; j < 4; ++j) amax = max(amax, max(w[j] & 0x7FFFu, (w[j] >> 16) & 0x7FFFu));
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
    int e = (int)(amax >> 7) - 127 - (kFormat == kCkptInt8 ? 6 : 8);
    if (kFormat == kCkptE4M3 && (amax & 0x7Fu) > 0x60u) ++e;
    e = max(e, -124);
    const bool finite = amax < 0x7F80u;
    // INT8: |v 2^-E| <= 127.5, and 127.5 itself would round to the even 128
    const float top = kFormat == kCkptInt8 ? 127.0f : e == 120 ? 240.0f : 448.0f;
    const float inv = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.0f;
    uint32_t q[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = (j & 1) ? bf16_hi(w[j >> 1]) : bf16_lo(w[j >> 1]);
      const uint32_t c = finite ? encode<kFormat>(fmaxf(fminf(v * inv, top), -top)) : 0u;
      q[j >> 2] |= c << (8 * (j & 3));
    }
    uint8_t* dst = codes + row * ld_codes + col;
    if (kVec && have == 8) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(q[0], q[1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < have) dst[j] = (uint8_t)(q[j >> 2] >> (8 * (j & 3)));
    }
    if (on && (i & 3) == 0) scales[row * ld_scales + blk] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
  }
}

template <int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads)
checkpoint_load_kernel(const uint8_t* __restrict__ codes, int64_t ld_codes, const uint8_t* __restrict__ scales,
                       int64_t ld_scales, int64_t tokens, int64_t n, int blocks, uint16_t* __restrict__ x,
                       int64_t ld_x) {
  const int64_t units = tokens * blocks;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < units * 4; i += (int64_t)gridDim.x * kThreads) {
    int64_t row;
    int blk;
    unit_of(i >> 2, units, blocks, row, blk);
    const int64_t col = (int64_t)blk * kCkptBlock + (i & 3) * 8;
    const int have = (int)max((int64_t)0, min((int64_t)8, n - col));
    const uint8_t* src = codes + row * ld_codes + col;
    uint32_t q[2] = {0u, 0u};
    if (kVec && have == 8) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(src));
      q[0] = v.x, q[1] = v.y;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < have) q[j >> 2] |= (uint32_t)src[j] << (8 * (j & 3));
    }
    const uint32_t scale = ckpt_scale(scales[row * ld_scales + blk]);
    const uint32_t w[4] = {ckpt_values<kFormat, 0>(q[0], scale), ckpt_values<kFormat, 1>(q[0], scale),
                           ckpt_values<kFormat, 0>(q[1], scale), ckpt_values<kFormat, 1>(q[1], scale)};
    uint16_t* dst = x + row * ld_x + col;
    if (kVec && have == 8) {
      *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < have) dst[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  }
}

bool rows_aligned(const void* x, int64_t ld_x, const void* codes, int64_t ld_codes) {
  return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld_x % 8 == 0 && reinterpret_cast<uintptr_t>(codes) % 8 == 0 &&
         ld_codes % 8 == 0;
}

unsigned grid_of(int64_t tokens, int blocks, int sms) {
  const int64_t want = (tokens * blocks * 4 + kThreads - 1) / kThreads;
  return (unsigned)std::min<int64_t>(want, (int64_t)sms * 8);
}

}  // namespace

cudaError_t launch_checkpoint_save(const void* x, int64_t tokens, int64_t n, int64_t ld_x, int format, uint8_t* codes,
                                   int64_t ld_codes, uint8_t* scales, int64_t ld_scales, cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int blocks = (int)((n + kCkptBlock - 1) / kCkptBlock);
  const bool vec = rows_aligned(x, ld_x, codes, ld_codes);
  auto* kernel = format == kCkptInt8 ? (vec ? checkpoint_save_kernel<kCkptInt8, true> : checkpoint_save_kernel<kCkptInt8, false>)
                                     : (vec ? checkpoint_save_kernel<kCkptE4M3, true> : checkpoint_save_kernel<kCkptE4M3, false>);
  kernel<<<grid_of(tokens, blocks, info.sm_count), kThreads, 0, stream>>>(static_cast<const uint16_t*>(x), tokens, n, ld_x, blocks, codes,
                                                                    ld_codes, scales, ld_scales);
  return cudaGetLastError();
}

cudaError_t launch_checkpoint_load(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                   int64_t tokens, int64_t n, int format, void* x, int64_t ld_x, cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int blocks = (int)((n + kCkptBlock - 1) / kCkptBlock);
  const bool vec = rows_aligned(x, ld_x, codes, ld_codes);
  auto* kernel = format == kCkptInt8 ? (vec ? checkpoint_load_kernel<kCkptInt8, true> : checkpoint_load_kernel<kCkptInt8, false>)
                                     : (vec ? checkpoint_load_kernel<kCkptE4M3, true> : checkpoint_load_kernel<kCkptE4M3, false>);
  kernel<<<grid_of(tokens, blocks, info.sm_count), kThreads, 0, stream>>>(codes, ld_codes, scales, ld_scales, tokens, n, blocks,
                                                                    static_cast<uint16_t*>(x), ld_x);
  return cudaGetLastError();
}

}  // namespace hscale
