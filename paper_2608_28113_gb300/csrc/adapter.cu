// adapter.cu -- the low-rank adapters' own products beside a projection (project.cu):
//   z  = alpha_a A_a x_t       dz = alpha_a B_a^T dy_t        for every token t of an adapter a
//   dA = sum_t dz_t x_t^T      dB = sum_t dy_t z_t^T          over the tokens of each adapter
// z and dz are fp32 [tokens, rank]; rows of tokens without an adapter are left as they are.
//
// All four read long rows of activations once and multiply them by something narrow (`rank` wide), so they
// are bound by HBM, and their tiles are too thin for tcgen05 (N = rank, or K = the tokens of one adapter): they
// run on warp-level MMAs (m16n8k16, bf16 operands, fp32 sums) whose fragments come straight from global
// memory.  The order of a contracted axis is free, so a lane takes 16 consecutive bytes of a row and calls
// its 8 elements whatever slots of K the fragment layout gives it, on both operands alike.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"
#include "tma.cuh"
#include "warp_mma.cuh"

namespace hscale {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(const float* p, uint32_t rank) {
  uint32_t a;
  float v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// ---------------------------------------------------------------- rows of activations
// bf16 (kFormat -1) or a checkpoint; `cols` elements a row.
template <int kFormat>
struct Rows {
  const uint16_t* x;
  int64_t ld;
  Checkpoint ckpt;
  int64_t cols;
  bool vec;  // whole groups of 8 elements may be loaded at once

  struct Raw {
    uint4 v;         // bf16: 8 elements; checkpoint: 8 codes in x, y
    uint32_t scale;  // checkpoint: the block's byte
  };
  // elements [k, k + 8) of row t, zeros past the end of the row; k % 8 == 0
  __device__ __forceinline__ Raw load(int64_t t, int64_t k) const {
    Raw r;
    r.v = make_uint4(0u, 0u, 0u, 0u);
    r.scale = 0u;
    if (k >= cols) return r;
    if constexpr (kFormat < 0) {
      const uint16_t* p = x + t * ld + k;
      if (k + 8 <= cols) {
        r.v = ld_nc_v4(p);
      } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < cols) w[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
        r.v = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      const uint8_t* p = ckpt.codes + t * ckpt.ld_codes + k;
      r.scale = ckpt.scales[t * ckpt.ld_scales + k / kCkptBlock];
      if (vec && k + 8 <= cols) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        r.v.x = q.x, r.v.y = q.y;
      } else {
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < cols) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
        r.v.x = w[0], r.v.y = w[1];
      }
    }
    return r;
  }
  // as 4 x bf16x2; a checkpoint's values are exact in bf16
  static __device__ __forceinline__ uint4 values(const Raw& r) {
    if constexpr (kFormat < 0) {
      return r.v;
    } else {
      const float s = ckpt_scale(r.scale);
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = ckpt_values<kFormat>((j < 2 ? r.v.x : r.v.y) >> (16 * (j & 1)), s);
      return make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
};

// ---------------------------------------------------------------- z and dz
// A CTA (of a cluster of csize that splits the contracted axis) takes 16 kMT tokens; its warps split the
// axis too, in blocks of 64.  For each adapter among the tokens (in order of their first token) the warps
// multiply all the tile's tokens by it and keep the rows of its own tokens: other rows' results are
// dropped, never added, so nothing passes from one request to another.  An adapter's factors are read once per
// tile; the tokens once per adapter of the tile, from L1 or L2 after the first time.  Warps and ranks are summed
// in order.
// kDown: A_a [rank, cols] (contracted axis contiguous); else B_a [cols, rank], whose 8 x 8 blocks are
// transposed in registers.  kNT: ranks / 8 of one pass.
template <int kFormat, bool kDown, int kMT, int kNT>
__device__ __forceinline__ void shrink_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, float* z,
                                            int64_t tile, int csize, int crank, float* part) {
  constexpr int kTok = 16 * kMT;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int64_t t0 = tile * kTok;
  const int rank = ad.rank;
  const int mine = lane < kTok && t0 + lane < tokens ? adapter_of(ad, t0 + lane) : -1;
  // rows past the end are read as the last one; their results have no adapter
  const __nv_bfloat16* factors = kDown ? ad.a : ad.b;
  int64_t trow[2 * kMT];
#pragma unroll
  for (int i = 0; i < 2 * kMT; ++i) trow[i] = min(t0 + 8 * i + g, tokens - 1);
  float* out = part + warp * kTok * rank;
  uint32_t left = __ballot_sync(0xFFFFFFFFu, mine >= 0);
  while (left) {
    const int a = __shfl_sync(0xFFFFFFFFu, mine, __ffs(left) - 1);
    const uint32_t sel = __ballot_sync(0xFFFFFFFFu, mine == a);
    left &= ~sel;
    for (int r0 = 0; r0 < rank; r0 += 8 * kNT) {
      float acc[kMT][kNT][4];
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
      const int64_t stride = (int64_t)kWarps * csize * 64;
      for (int64_t kb = ((int64_t)crank * kWarps + warp) * 64; kb < rows.cols; kb += stride) {
        typename Rows<kFormat>::Raw raw[2][2 * kMT];
        uint4 w[2][kNT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t k = kb + 32 * h + 8 * q;
#pragma unroll
          for (int i = 0; i < 2 * kMT; ++i) raw[h][i] = rows.load(trow[i], k);
          if (kDown) {
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              const int r = r0 + 8 * j + g;
              w[h][j] = make_uint4(0u, 0u, 0u, 0u);
              if (r < rank && k < rows.cols) w[h][j] = ld_nc_v4(factors + ((int64_t)a * rank + r) * rows.cols + k);
            }
          } else {
            // register u of the fragment: slots 2 q', 2 q' + 1 are elements 8 q' + 2 u, + 1
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              uint32_t v[4];
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const int64_t kk = kb + 32 * h + (g >> 1) * 8 + 2 * u + (g & 1);
                const int r = r0 + 8 * j + 2 * q;
                v[u] = 0u;
                if (kk < rows.cols && r < rank)
                  v[u] = __ldg(reinterpret_cast<const uint32_t*>(factors + ((int64_t)a * rows.cols + kk) * rank + r));
              }
              w[h][j] = make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!kDown) {
#pragma unroll
            for (int j = 0; j < kNT; ++j)
              w[h][j] = make_uint4(transpose_8x8(w[h][j].x), transpose_8x8(w[h][j].y), transpose_8x8(w[h][j].z),
                                   transpose_8x8(w[h][j].w));
          }
#pragma unroll
          for (int i = 0; i < kMT; ++i) {
            const uint4 lo = Rows<kFormat>::values(raw[h][2 * i]), hi = Rows<kFormat>::values(raw[h][2 * i + 1]);
            const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              mma_bf16(acc[i][j], a0, w[h][j].x, w[h][j].y);
              mma_bf16(acc[i][j], a1, w[h][j].z, w[h][j].w);
            }
          }
        }
      }
      // rows g, g + 8 of each 16; ranks 2 q, 2 q + 1 of each 8
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int t = 16 * i + 8 * e + g;
          if (!((sel >> t) & 1u)) continue;
#pragma unroll
          for (int j = 0; j < kNT; ++j) {
            const int r = r0 + 8 * j + 2 * q;
            if (r < rank) *reinterpret_cast<float2*>(out + t * rank + r) = make_float2(acc[i][j][2 * e], acc[i][j][2 * e + 1]);
          }
        }
    }
  }
  __syncthreads();
  // the warps' partials in order, into the first warp's; then the ranks' in order
  for (int i = threadIdx.x; i < kTok * rank; i += kThreads) {
    float s = part[i];
    for (int v = 1; v < kWarps; ++v) s += part[v * kTok * rank + i];
    part[i] = s;
  }
  if (csize > 1) cluster_sync(); else __syncthreads();
  const int share = (kTok * rank + csize - 1) / csize;
  for (int i = crank * share + threadIdx.x; i < min(kTok * rank, (crank + 1) * share); i += kThreads) {
    const int64_t t = t0 + i / rank;
    if (t >= tokens) continue;
    const int a = adapter_of(ad, t);
    if (a < 0) continue;
    float s = csize > 1 ? ld_cluster(part + i, 0) : part[i];
    for (int d = 1; d < csize; ++d) s += ld_cluster(part + i, (uint32_t)d);
    z[t0 * rank + i] = s * ad.alpha[a];
  }
  if (csize > 1) cluster_sync();  // the others' shared memory stays until it has been read
}

template <int kFormat, bool kDown, int kMT, int kNT>
__global__ void __launch_bounds__(kThreads, 2)
shrink_kernel(Rows<kFormat> rows, int64_t tokens, Adapters ad, float* z, int csize) {
  extern __shared__ __align__(16) float shrink_part[];
  pdl_launch_dependents();  // the projection's own product needs no z
  const int crank = csize > 1 ? (int)cluster_rank() : 0;
  shrink_tile<kFormat, kDown, kMT, kNT>(rows, tokens, ad, z, blockIdx.x / csize, csize, crank, shrink_part);
}

template <int kFormat, bool kDown, int kMT, int kNT>
cudaError_t launch_shrink_of(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, float* z, int csize,
                             cudaStream_t stream) {
  auto kernel = shrink_kernel<kFormat, kDown, kMT, kNT>;
  const int smem = kWarps * 16 * kMT * ad.rank * 4;
  cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), kWarps * 16 * kMT * 128 * 4);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((tokens + 16 * kMT - 1) / (16 * kMT) * csize), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  err = cudaLaunchKernelEx(&cfg, kernel, rows, tokens, ad, z, csize);
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <int kFormat, bool kDown>
cudaError_t launch_shrink(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, float* z, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  // 32 tokens a tile where that leaves a tile an SM, 16 below; the axis split until there are two CTAs an SM
  // or a warp has one block of it
  const int64_t tok = tokens > (int64_t)32 * info.sm_count ? 32 : 16;
  const int64_t tiles = (tokens + tok - 1) / tok;
  int csize = 1;
  while (csize < 8 && tiles * csize < 2 * info.sm_count && (int64_t)csize * kWarps * 64 < rows.cols) csize *= 2;
  if (tok == 32) {
    if (ad.rank <= 8) return launch_shrink_of<kFormat, kDown, 2, 1>(rows, tokens, ad, z, csize, stream);
    if (ad.rank <= 16) return launch_shrink_of<kFormat, kDown, 2, 2>(rows, tokens, ad, z, csize, stream);
    return launch_shrink_of<kFormat, kDown, 2, 4>(rows, tokens, ad, z, csize, stream);
  }
  if (ad.rank <= 8) return launch_shrink_of<kFormat, kDown, 1, 1>(rows, tokens, ad, z, csize, stream);
  if (ad.rank <= 16) return launch_shrink_of<kFormat, kDown, 1, 2>(rows, tokens, ad, z, csize, stream);
  return launch_shrink_of<kFormat, kDown, 1, 4>(rows, tokens, ad, z, csize, stream);
}

// ---------------------------------------------------------------- dA and dB
// A CTA (of a cluster of csize that splits the tokens) takes 64 columns of one adapter's gradient and all of
// the adapter's tokens, 16 at a time and warp.  As an MMA: M = ranks (z or dz transposed, as a pair hi + lo of
// bf16 numbers: 2^-17 of a value is lost), N = columns, K = tokens.  A lane loads 8 columns of four tokens and
// pairs the tokens' halves up into the fragments of 8 column tiles.  The adapter's tokens are found in windows of
// kWindow: the CTA scans their adapters and lists its own, in order, so an adapter without tokens gets
// zeros and the sums' order does not depend on anything but the tokens'.
constexpr int kWindow = 2048;

template <int kFormat, bool kRankMajor, int kRT>
__device__ __forceinline__ void grad_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, const float* z,
                                          __nv_bfloat16* out, int64_t col0, int a, int r0, int csize, int crank,
                                          float* part, int* list, int* counts) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int rank = ad.rank;
  const int64_t col = col0 + 8 * g;
  float acc[kRT][8][4];
#pragma unroll
  for (int i = 0; i < kRT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;

  for (int64_t w0 = 0; w0 < tokens; w0 += kWindow) {
    int have = (int)min((int64_t)kWindow, tokens - w0);
    if (ad.of_token != nullptr) {
      // warp w lists tokens [w kWindow / 8, ..) of the window behind the warps' before it
      constexpr int kSpan = kWindow / kWarps;
      __syncthreads();
      uint32_t own[kSpan / 32];
      int count = 0;
#pragma unroll
      for (int i = 0; i < kSpan / 32; ++i) {
        const int t = warp * kSpan + 32 * i + lane;
        own[i] = __ballot_sync(0xFFFFFFFFu, t < have && ad.of_token[w0 + t] == a);
        count += __popc(own[i]);
      }
      if (lane == 0) counts[warp] = count;
      __syncthreads();
      int at = 0;
      have = 0;
      for (int v = 0; v < kWarps; ++v) {
        if (v == warp) at = have;
        have += counts[v];
      }
#pragma unroll
      for (int i = 0; i < kSpan / 32; ++i) {
        if ((own[i] >> lane) & 1u) list[at + __popc(own[i] & ((1u << lane) - 1u))] = warp * kSpan + 32 * i + lane;
        at += __popc(own[i]);
      }
      __syncthreads();
    }
    const int units = (have + 15) >> 4;
    for (int u = crank * kWarps + warp; u < units; u += csize * kWarps) {
      typename Rows<kFormat>::Raw raw[4];
      int64_t tok[4];
      bool on[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = 16 * u + 2 * q + (i & 1) + 8 * (i >> 1);  // slots 2 q, 2 q + 1, 2 q + 8, 2 q + 9
        on[i] = e < have;
        tok[i] = w0 + (on[i] ? (ad.of_token != nullptr ? list[e] : e) : 0);
        raw[i] = on[i] ? rows.load(tok[i], col) : typename Rows<kFormat>::Raw{make_uint4(0u, 0u, 0u, 0u), 0u};
      }
      float zv[kRT][2][4];
#pragma unroll
      for (int i = 0; i < kRT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 4; ++s) {
            const int r = r0 + 16 * i + 8 * h + g;
            zv[i][h][s] = on[s] && r < rank ? z[tok[s] * rank + r] : 0.0f;
          }
      uint32_t v[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 x = Rows<kFormat>::values(raw[i]);
        v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
      }
#pragma unroll
      for (int i = 0; i < kRT; ++i) {
        // rows g | g + 8, slots (2 q, 2 q + 1) | (2 q + 8, 2 q + 9)
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const float z0 = zv[i][h][2 * s], z1 = zv[i][h][2 * s + 1];
            const uint32_t p = pack_bf16(z0, z1);
            hi[2 * s + h] = p;
            lo[2 * s + h] = pack_bf16(z0 - bf16_lo(p), z1 - bf16_hi(p));
          }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t pick = (j & 1) ? 0x7632u : 0x5410u;
          const uint32_t b0 = __byte_perm(v[0][j >> 1], v[1][j >> 1], pick);
          const uint32_t b1 = __byte_perm(v[2][j >> 1], v[3][j >> 1], pick);
          mma_bf16(acc[i][j], hi, b0, b1);
          mma_bf16(acc[i][j], lo, b0, b1);
        }
      }
    }
  }
  // acc[i][j]: ranks 16 i + g (e 0, 1) and + 8 (e 2, 3), N slots 2 q, 2 q + 1 of column tile j, which are
  // columns 8 (2 q) + j and 8 (2 q + 1) + j.  The warps' partials: [warp][rank][64].
  constexpr int kSize = 16 * kRT * 64;
#pragma unroll
  for (int i = 0; i < kRT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[warp * kSize + (16 * i + 8 * (e >> 1) + g) * 64 + 8 * (2 * q + (e & 1)) + j] = acc[i][j][e];
  __syncthreads();
  for (int i = threadIdx.x; i < kSize; i += kThreads) {
    float s = part[i];
#pragma unroll
    for (int v = 1; v < kWarps; ++v) s += part[v * kSize + i];
    part[i] = s;
  }
  if (csize > 1) cluster_sync(); else __syncthreads();
  const int share = kSize / csize;
  for (int i = crank * share + threadIdx.x; i < (crank + 1) * share; i += kThreads) {
    // dA's rows run along the columns, dB's along the ranks
    const int e = kRankMajor ? i : (i % (16 * kRT)) * 64 + i / (16 * kRT);
    const int r = r0 + (e >> 6);
    const int64_t c = col0 + (e & 63);
    if (r >= rank || c >= rows.cols) continue;
    float s = csize > 1 ? ld_cluster(part + e, 0) : part[e];
    for (int d = 1; d < csize; ++d) s += ld_cluster(part + e, (uint32_t)d);
    out[kRankMajor ? ((int64_t)a * rank + r) * rows.cols + c : ((int64_t)a * rows.cols + c) * rank + r] = __float2bfloat16_rn(s);
  }
  if (csize > 1) cluster_sync();
}

template <int kFormat, bool kRankMajor, int kRT>
__global__ void __launch_bounds__(kThreads, kRT == 1 ? 3 : 2)
grad_kernel(Rows<kFormat> rows, int64_t tokens, Adapters ad, const float* z, __nv_bfloat16* out, int csize) {
  extern __shared__ __align__(16) float grad_part[];
  __shared__ int list[kWindow];
  __shared__ int counts[kWarps];
  const int crank = csize > 1 ? (int)cluster_rank() : 0;
  grad_tile<kFormat, kRankMajor, kRT>(rows, tokens, ad, z, out, (int64_t)(blockIdx.x / csize) * 64, blockIdx.y,
                                      blockIdx.z * 16 * kRT, csize, crank, grad_part, list, counts);
}

template <int kFormat, bool kRankMajor, int kRT>
cudaError_t launch_grad_of(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, const float* z, void* out,
                           int csize, cudaStream_t stream) {
  auto kernel = grad_kernel<kFormat, kRankMajor, kRT>;
  constexpr int kSmem = kWarps * 16 * kRT * 64 * 4;
  cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmem);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((rows.cols + 63) / 64 * csize), (unsigned)ad.count, (unsigned)((ad.rank + 16 * kRT - 1) / (16 * kRT)));
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  err = cudaLaunchKernelEx(&cfg, kernel, rows, tokens, ad, z, static_cast<__nv_bfloat16*>(out), csize);
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <int kFormat, bool kRankMajor>
cudaError_t launch_grad(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, const float* z, void* out,
                        cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int64_t tiles = (rows.cols + 63) / 64 * ad.count;
  int csize = 1;
  while (csize < 8 && tiles * csize < 2 * info.sm_count && tokens / ad.count > (int64_t)csize * kWarps * 16) csize *= 2;
  if (ad.rank <= 16) return launch_grad_of<kFormat, kRankMajor, 1>(rows, tokens, ad, z, out, csize, stream);
  return launch_grad_of<kFormat, kRankMajor, 2>(rows, tokens, ad, z, out, csize, stream);
}

Rows<-1> bf16_rows(const void* x, int64_t ld, int64_t cols) { return {static_cast<const uint16_t*>(x), ld, {}, cols, true}; }

template <int kFormat>
Rows<kFormat> ckpt_rows(const Checkpoint& c, int64_t cols) {
  return {nullptr, 0, c, cols, reinterpret_cast<uintptr_t>(c.codes) % 8 == 0 && c.ld_codes % 8 == 0};
}

}  // namespace

cudaError_t launch_adapter_down(const void* x, int64_t ld_x, const Checkpoint* ckpt, int format, int64_t tokens, int64_t n,
                                const Adapters& ad, float* z, cudaStream_t stream) {
  if (ckpt == nullptr) return launch_shrink<-1, true>(bf16_rows(x, ld_x, n), tokens, ad, z, stream);
  if (format == kCkptInt8) return launch_shrink<kCkptInt8, true>(ckpt_rows<kCkptInt8>(*ckpt, n), tokens, ad, z, stream);
  return launch_shrink<kCkptE4M3, true>(ckpt_rows<kCkptE4M3>(*ckpt, n), tokens, ad, z, stream);
}

cudaError_t launch_adapter_up_t(const void* dy, int64_t ld_dy, int64_t tokens, int64_t m, const Adapters& ad, float* dz,
                                cudaStream_t stream) {
  return launch_shrink<-1, false>(bf16_rows(dy, ld_dy, m), tokens, ad, dz, stream);
}

cudaError_t launch_adapter_grad_a(const Checkpoint& ckpt, int format, int64_t tokens, int64_t n, const Adapters& ad,
                                  const float* dz, void* da, cudaStream_t stream) {
  if (format == kCkptInt8) return launch_grad<kCkptInt8, true>(ckpt_rows<kCkptInt8>(ckpt, n), tokens, ad, dz, da, stream);
  return launch_grad<kCkptE4M3, true>(ckpt_rows<kCkptE4M3>(ckpt, n), tokens, ad, dz, da, stream);
}

cudaError_t launch_adapter_grad_b(const void* dy, int64_t ld_dy, int64_t tokens, int64_t m, const Adapters& ad, const float* z,
                                  void* db, cudaStream_t stream) {
  return launch_grad<-1, false>(bf16_rows(dy, ld_dy, m), tokens, ad, z, db, stream);
}

}  // namespace hscale
