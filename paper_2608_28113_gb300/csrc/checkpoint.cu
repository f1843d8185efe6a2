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
// 2 B in and 1 + 1/32 B out per element for a save, the reverse for a load: one pass, 4.7 TB/s over both at 8192 x 4096.  A load
// is bound by HBM, a save by its integer instructions (64 % of their pipe's rate under a profiler, HBM at 42 %).  Two lanes
// share a block, 16 elements each, and a thread has kUnroll such pieces in flight.  Rows off 16 bytes (kVec false) go element
// by element: 8192 x 4104 with contiguous rows of codes 94 us saved and 178 loaded, 21 and 21 with rows of 4112.
#include <algorithm>
#include <type_traits>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"

namespace hscale {
namespace {

constexpr int kThreads = 256, kUnroll = 2;
constexpr int kPiece = 16;  // elements a lane

// (row, block) of a flat unit index; 32-bit arithmetic where it reaches
__device__ __forceinline__ void unit_of(int64_t u, int64_t units, int blocks, int64_t& row, int& blk) {
  row = units <= UINT32_MAX ? (int64_t)((uint32_t)u / (uint32_t)blocks) : u / blocks;
  blk = (int)(u - row * blocks);
}

// RNE of four values x 2^-E to bytes; within +-top where asked for: few blocks have a value that needs it (save and load of
// 8192 x 4096: 44.8 us with it in every block, 43.3).
template <int kFormat, bool kClamp>
__device__ __forceinline__ uint32_t encode4(const float (&v)[4], float inv, float top) {
  float c[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) c[j] = kClamp ? fmaxf(fminf(v[j] * inv, top), -top) : v[j] * inv;
  if (kFormat == kCkptInt8) {
    // added to 1.5 2^23, a number is rounded to a whole one whose low byte is the code (the products are exact)
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(kClamp ? c[j] + 12582912.0f : fmaf(v[j], inv, 12582912.0f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  }
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(c[1]), "f"(c[0]));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(c[3]), "f"(c[2]));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

// kVec: rows of x and of codes are 16-byte aligned
template <int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads)
checkpoint_save_kernel(const uint16_t* __restrict__ x, int64_t tokens, int64_t n, int64_t ld_x, int blocks,
                       uint8_t* __restrict__ codes, int64_t ld_codes, uint8_t* __restrict__ scales,
                       int64_t ld_scales) {
  const int64_t units = tokens * blocks;
  const int64_t lanes = (units * 2 + 31) / 32 * 32;  // whole warps take part in the shuffles
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; i0 < lanes; i0 += step * kUnroll) {
    uint32_t w[kUnroll][8];
    int64_t row[kUnroll];
    int blk[kUnroll], have[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * step;
      const bool on = (i >> 1) < units;
      row[u] = 0, blk[u] = 0;
      if (on) unit_of(i >> 1, units, blocks, row[u], blk[u]);
      const int64_t col = (int64_t)blk[u] * kCkptBlock + (i & 1) * kPiece;
      have[u] = on ? (int)max((int64_t)0, min((int64_t)kPiece, n - col)) : 0;
      const uint16_t* src = x + row[u] * ld_x + col;
#pragma unroll
      for (int j = 0; j < 8; ++j) w[u][j] = 0u;
      if (kVec) {
        ld_16_ahead(have[u] >= 8, src, w[u][0], w[u][1], w[u][2], w[u][3]);
        ld_16_ahead(have[u] == 16, src + 8, w[u][4], w[u][5], w[u][6], w[u][7]);
      }
      if (!kVec || (have[u] & 7) != 0) {
#pragma unroll
        for (int j = 0; j < kPiece; ++j)
          if (j < have[u] && (!kVec || j >= (have[u] & ~7))) w[u][j >> 1] |= (uint32_t)src[j] << (16 * (j & 1));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * step;
      uint32_t amax = 0;  // bf16 bit patterns order as magnitudes; NaN above Inf
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = __vmaxu2(amax, w[u][j] & 0x7FFF7FFFu);
      amax = max(amax & 0xFFFFu, amax >> 16);
      amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
      int e = (int)(amax >> 7) - 127 - (kFormat == kCkptInt8 ? 6 : 8);
      if (kFormat == kCkptE4M3 && (amax & 0x7Fu) > 0x60u) ++e;
      e = max(e, -124);
      const bool finite = amax < 0x7F80u;
      const float inv = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.0f;
      uint32_t q[4];
      const auto encode = [&](auto clamp, float top) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v[4] = {bf16_lo(w[u][2 * j]), bf16_hi(w[u][2 * j]), bf16_lo(w[u][2 * j + 1]), bf16_hi(w[u][2 * j + 1])};
          q[j] = finite ? encode4<kFormat, clamp.value>(v, inv, top) : 0u;
        }
      };
      // INT8: |v 2^-E| <= 127.5, and 127.5 itself, of the longest mantissa, would round to the even 128
      if (kFormat == kCkptInt8 ? (amax & 0x7Fu) == 0x7Fu : e == 120)
        encode(std::true_type{}, kFormat == kCkptInt8 ? 127.0f : 240.0f);
      else
        encode(std::false_type{}, 0.0f);
      uint8_t* dst = codes + row[u] * ld_codes + (int64_t)blk[u] * kCkptBlock + (i & 1) * kPiece;
      if (kVec && have[u] == kPiece) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(q[0], q[1], q[2], q[3]);
      } else {
#pragma unroll
        for (int j = 0; j < kPiece; ++j)
          if (j < have[u]) dst[j] = (uint8_t)(q[j >> 2] >> (8 * (j & 3)));
      }
      if ((i & 1) == 0 && (i >> 1) < units) scales[row[u] * ld_scales + blk[u]] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
    }
  }
}

template <int kFormat, bool kVec>
__global__ void __launch_bounds__(kThreads)
checkpoint_load_kernel(const uint8_t* __restrict__ codes, int64_t ld_codes, const uint8_t* __restrict__ scales,
                       int64_t ld_scales, int64_t tokens, int64_t n, int blocks, uint16_t* __restrict__ x,
                       int64_t ld_x) {
  const int64_t units = tokens * blocks, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; i0 < units * 2; i0 += step * kUnroll) {
    uint32_t q[kUnroll][4], byte[kUnroll];
    int64_t row[kUnroll], col[kUnroll];
    int have[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * step;
      const bool on = i < units * 2;
      int blk = 0;
      row[u] = 0;
      if (on) unit_of(i >> 1, units, blocks, row[u], blk);
      col[u] = (int64_t)blk * kCkptBlock + (i & 1) * kPiece;
      have[u] = on ? (int)max((int64_t)0, min((int64_t)kPiece, n - col[u])) : 0;
      const uint8_t* src = codes + row[u] * ld_codes + col[u];
      byte[u] = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) q[u][j] = 0u;
      ld_1_ahead(on, scales + row[u] * ld_scales + blk, byte[u]);
      if (kVec) ld_16_ahead(have[u] == kPiece, src, q[u][0], q[u][1], q[u][2], q[u][3]);
      if (!kVec || have[u] < kPiece) {
#pragma unroll
        for (int j = 0; j < kPiece; ++j)
          if (j < have[u]) q[u][j >> 2] |= (uint32_t)src[j] << (8 * (j & 3));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t scale = ckpt_scale(byte[u]);
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[2 * j] = ckpt_values<kFormat, 0>(q[u][j], scale);
        w[2 * j + 1] = ckpt_values<kFormat, 1>(q[u][j], scale);
      }
      uint16_t* dst = x + row[u] * ld_x + col[u];
      if (kVec && have[u] == kPiece) {
        reinterpret_cast<uint4*>(dst)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(dst)[1] = make_uint4(w[4], w[5], w[6], w[7]);
      } else {
#pragma unroll
        for (int j = 0; j < kPiece; ++j)
          if (j < have[u]) dst[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      }
    }
  }
}

bool rows_aligned(const void* x, int64_t ld_x, const void* codes, int64_t ld_codes) {
  return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld_x % 8 == 0 && reinterpret_cast<uintptr_t>(codes) % 16 == 0 &&
         ld_codes % 16 == 0;
}

unsigned grid_of(int64_t tokens, int blocks, int sms) {
  const int64_t want = (tokens * blocks * 2 + kThreads * kUnroll - 1) / (kThreads * kUnroll);
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(want, (int64_t)sms * 8));
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
