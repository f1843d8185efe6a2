// project_decode.cu -- the packed projection for a few tokens (a decoding batch): y_t = W_hat x_t + B_a z_t.
//
// Bound by the weight's bytes and by unpacking them (about 2.4 instructions a weight).  tcgen05 would take
// 128-row tiles of W through shared memory; here the unpacked weights are the A fragments of warp-level MMAs
// (m16n8k16) in the registers they were unpacked in.  A CTA takes 16 kMT outputs and its 8 warps split K in blocks
// of 128: a lane holds 32 consecutive nibbles of each of its rows (16 bytes, one load, the next block's ahead of the
// present one's products).  The order of K within a block is free, so a word's nibbles are paired as they are
// cheapest to unpack (0 with 4, 1 with 5, ...), and x is paired alike.  The warps' sums meet in
// shared memory, in order, where each thread adds its outputs' adapter terms in fp32 and rounds once.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"
#include "tma.cuh"
#include "warp_mma.cuh"

namespace hscale {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

struct DecodeArgs {
  Nvfp4Weight w;
  Adapters ad;
  const uint16_t* x;
  const float* z;
  __nv_bfloat16* y;
  int64_t ld_x, ld_y;
  int32_t tokens, chained;
  bool wide;  // rows of W are 16-byte and rows of codes 2-byte aligned, n % 32 == 0
};

// Eight nibbles times a scale (bf16x2, both halves): pairs (0, 4), (1, 5), (2, 6), (3, 7).  A nibble's magnitude bits
// at bf16's bits 8-6 read as E2M1 2^-126.
__device__ __forceinline__ void unpack_pairs(uint32_t w, uint32_t scale, uint32_t (&r)[4]) {
  constexpr uint32_t kSign = 0x80008000u, kMag = 0x01C001C0u;
  r[0] = mul_bf16x2(((w << 12) & kSign) | ((w << 6) & kMag), scale);
  r[1] = mul_bf16x2(((w << 8) & kSign) | ((w << 2) & kMag), scale);
  r[2] = mul_bf16x2(((w << 4) & kSign) | ((w >> 2) & kMag), scale);
  r[3] = mul_bf16x2((w & kSign) | ((w >> 6) & kMag), scale);
}

// A block's words of a lane's rows and their two codes each
template <int kMT>
struct Block {
  uint32_t w[2 * kMT][4], c[2 * kMT];
};

// Rows past the end of W and tokens past the end of x are read as the last ones, and their results dropped, so only
// the last block of a row needs bounds.
template <int kMT>
__device__ __forceinline__ void load_block(const uint8_t* const (&wp)[2 * kMT], const uint8_t* const (&cp)[2 * kMT], int64_t k,
                                           int64_t n, bool wide, Block<kMT>& b) {
  const int64_t wk = k >> 1, ck = k >> 4;
  if (wide) {
    const bool on = k < n;  // n % 32 == 0
#pragma unroll
    for (int i = 0; i < 2 * kMT; ++i) {
      ld_16_ahead(on, wp[i] + wk, b.w[i][0], b.w[i][1], b.w[i][2], b.w[i][3]);
      ld_2_ahead(on, cp[i] + ck, b.c[i]);
    }
  } else {
    const bool on = k < n, on1 = k + 16 < n;
#pragma unroll
    for (int i = 0; i < 2 * kMT; ++i) {
      uint32_t c0 = 0u, c1 = 0u;
      ld_8_ahead(on, wp[i] + wk, b.w[i][0], b.w[i][1]);
      ld_8_ahead(on1, wp[i] + wk + 8, b.w[i][2], b.w[i][3]);
      ld_1_ahead(on, cp[i] + ck, c0);
      ld_1_ahead(on1, cp[i] + ck + 1, c1);
      b.c[i] = c0 | c1 << 8;
    }
  }
}

template <int kMT, int kNT>
__global__ void __launch_bounds__(kThreads, 2) project_decode_kernel(const __grid_constant__ DecodeArgs p) {
  __shared__ float part[kWarps][8 * kNT][16 * kMT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int64_t n = p.w.n, f0 = (int64_t)blockIdx.x * (16 * kMT);
  constexpr int kOuts = 16 * kMT * 8 * kNT;
  float acc[kMT][kNT][4];
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;

  constexpr int64_t kStep = kWarps * 128;
  const uint8_t *wp[2 * kMT], *cp[2 * kMT];
#pragma unroll
  for (int i = 0; i < 2 * kMT; ++i) {
    const int64_t f = min(f0 + g + 8 * i, p.w.m - 1);
    wp[i] = p.w.packed + f * (n >> 1), cp[i] = p.w.codes + f * (n >> 4);
  }
  const uint16_t* xp[kNT];
#pragma unroll
  for (int j = 0; j < kNT; ++j) xp[j] = p.x + min(8 * j + g, p.tokens - 1) * p.ld_x;
  int64_t k = (int64_t)warp * 128 + 32 * q;  // this lane's 32 of the warp's block
  // what a block past the end leaves in the ring is multiplied by x's zeros there, and any word is a finite weight
  Block<kMT> ring[2];
#pragma unroll
  for (int i = 0; i < 2 * kMT; ++i) {
#pragma unroll
    for (int e = 0; e < 4; ++e) ring[0].w[i][e] = ring[1].w[i][e] = 0u;
    ring[0].c[i] = ring[1].c[i] = 0u;
  }
  load_block<kMT>(wp, cp, k, n, p.wide, ring[0]);
  for (int64_t kb = (int64_t)warp * 128; kb < n;) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (kb >= n) break;
      load_block<kMT>(wp, cp, k + kStep, n, p.wide, ring[u ^ 1]);
      Block<kMT>& b = ring[u];
      uint32_t scale[2 * kMT];
#pragma unroll
      for (int i = 0; i < 2 * kMT; ++i) scale[i] = unpack_codes(b.c[i]);
      const bool whole = kb + 128 <= n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t xb[kNT][4];
#pragma unroll
        for (int j = 0; j < kNT; ++j) {
          uint32_t v[4] = {0u, 0u, 0u, 0u};
          ld_16_ahead(whole || k + 8 * i < n, xp[j] + k + 8 * i, v[0], v[1], v[2], v[3]);
          xb[j][0] = __byte_perm(v[0], v[2], 0x5410), xb[j][1] = __byte_perm(v[0], v[2], 0x7632);
          xb[j][2] = __byte_perm(v[1], v[3], 0x5410), xb[j][3] = __byte_perm(v[1], v[3], 0x7632);
        }
#pragma unroll
        for (int t = 0; t < kMT; ++t) {
          uint32_t lo[4], hi[4];
          const uint32_t pick = i < 2 ? 0x1010u : 0x3232u;
          unpack_pairs(b.w[2 * t][i], __byte_perm(scale[2 * t], 0u, pick), lo);
          unpack_pairs(b.w[2 * t + 1][i], __byte_perm(scale[2 * t + 1], 0u, pick), hi);
          const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
          for (int j = 0; j < kNT; ++j) {
            mma_bf16(acc[t][j], a0, xb[j][0], xb[j][1]);
            mma_bf16(acc[t][j], a1, xb[j][2], xb[j][3]);
          }
        }
      }
      k += kStep, kb += kStep;
    }
  }
#pragma unroll
  for (int i = 0; i < kMT; ++i)
#pragma unroll
    for (int j = 0; j < kNT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[warp][8 * j + 2 * q + (e & 1)][16 * i + 8 * (e >> 1) + g] = acc[i][j][e];
  __syncthreads();
  const float unit = kWeightUnit * *p.w.global_scale;
  if (p.chained) pdl_wait_primary();  // z
  for (int i = threadIdx.x; i < kOuts; i += kThreads) {
    const int t = i / (16 * kMT), r = i % (16 * kMT);
    const int64_t f = f0 + r;
    if (t >= p.tokens || f >= p.w.m) continue;
    float s = part[0][t][r];
#pragma unroll
    for (int v = 1; v < kWarps; ++v) s += part[v][t][r];
    s *= unit;
    const int a = adapter_of(p.ad, t);
    if (a >= 0) {
      const int rank = p.ad.rank;
      const __nv_bfloat16* b = p.ad.b + ((int64_t)a * p.w.m + f) * rank;
      const float4* z = reinterpret_cast<const float4*>(p.z + (int64_t)t * rank);
      for (int r0 = 0; r0 < rank; r0 += 8) {
        const uint4 h = ld_nc_v4(b + r0);
        const float4 z0 = z[r0 / 4], z1 = z[r0 / 4 + 1];
        s = fmaf(z0.x, bf16_lo(h.x), s), s = fmaf(z0.y, bf16_hi(h.x), s), s = fmaf(z0.z, bf16_lo(h.y), s);
        s = fmaf(z0.w, bf16_hi(h.y), s), s = fmaf(z1.x, bf16_lo(h.z), s), s = fmaf(z1.y, bf16_hi(h.z), s);
        s = fmaf(z1.z, bf16_lo(h.w), s), s = fmaf(z1.w, bf16_hi(h.w), s);
      }
    }
    p.y[(int64_t)t * p.ld_y + f] = __float2bfloat16_rn(s);
  }
}

template <int kMT, int kNT>
cudaError_t launch(const DecodeArgs& p, bool early, cudaStream_t stream) {
  auto kernel = project_decode_kernel<kMT, kNT>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.w.m + 16 * kMT - 1) / (16 * kMT)), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = early ? 1 : 0;
  const cudaError_t err = cudaLaunchKernelEx(&cfg, kernel, p);
  return err != cudaSuccess ? err : cudaGetLastError();
}

}  // namespace

cudaError_t launch_project_decode(const void* x, int64_t tokens, int64_t ld_x, const Nvfp4Weight& w, const Adapters& ad,
                                  const float* z, void* y, int64_t ld_y, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  DecodeArgs p = {};
  p.w = w, p.ad = ad, p.x = static_cast<const uint16_t*>(x), p.z = z, p.y = static_cast<__nv_bfloat16*>(y);
  p.ld_x = ld_x, p.ld_y = ld_y, p.tokens = (int32_t)tokens, p.chained = ad.count > 0;
  p.wide = w.n % 32 == 0 && reinterpret_cast<uintptr_t>(w.packed) % 16 == 0 && reinterpret_cast<uintptr_t>(w.codes) % 2 == 0;
  // 32 outputs a CTA (x is read once for them) where that fills the SMs twice, else 16
  const bool two = (w.m + 31) / 32 >= 2 * info.sm_count;
  // Beside the kernel that makes z (chained launch) where x fits the L1 that that kernel's shared memory leaves: an SM
  // keeps its split while a CTA of it is resident.  In a graph, 16 adapters of rank 16, beside it and behind it: one token on
  // 4096 x 4096 7.6 and 11.0 us, 16 tokens on 28672 x 8192 92 and 67.  The bound lies below all that lose: 28672 x 8192
  // does from 3 tokens on (52.6 and 48.1), while 4096 x 4096 would still gain at 8 (11.7 and 12.6), 14336 x 4096 too
  // (20.4 and 24.2) and 4096 x 14336 at 4 (18.7 and 24.8).
  const bool early = p.chained && tokens * w.n <= 8192;
  if (tokens <= 8) return two ? launch<2, 1>(p, early, stream) : launch<1, 1>(p, early, stream);
  return two ? launch<2, 2>(p, early, stream) : launch<1, 2>(p, early, stream);
}

}  // namespace hscale
