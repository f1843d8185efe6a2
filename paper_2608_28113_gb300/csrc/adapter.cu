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

// ---------------------------------------------------------------- asynchronous copies
// Each lane copies what it will itself read into a place of its own (a ring of 16-byte slots per lane), so a
// block's data need no registers while they are in flight and no barrier when they have come.  `bytes` of the 16, 8
// or 4 are read, the rest are zeros.
__device__ __forceinline__ void copy_16(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_16_l1(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_8(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_4(void* dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but this lane's `kLeft` latest groups have come.
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// ---------------------------------------------------------------- rows of activations
// bf16 (kFormat -1) or a checkpoint; `cols` elements a row.
template <int kFormat>
struct Rows {
  const uint16_t* x;
  int64_t ld;
  Checkpoint ckpt;
  int64_t cols;
  int vec;  // checkpoint: codes that may be copied at once (16, 8 or 1)

  // elements [k, k + 8) of row t to dst (16 bytes of bf16, 8 codes), zeros past the end of the row; k % 8 == 0
  __device__ __forceinline__ void copy(uint8_t* dst, int64_t t, int64_t k, bool on) const {
    on = on && k < cols;
    if constexpr (kFormat < 0) {
      copy_16(dst, on ? x + t * ld + k : x, on ? (int)min((int64_t)16, (cols - k) * 2) : 0);
    } else {
      const uint8_t* p = on ? ckpt.codes + t * ckpt.ld_codes + k : ckpt.codes;
      if (vec >= 8) {
        copy_8(dst, p, on ? 8 : 0);  // cols % 16 == 0
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) dst[j] = on ? __ldg(p + j) : (uint8_t)0;
      }
    }
  }
  __device__ __forceinline__ uint32_t scale(int64_t t, int64_t k, bool on) const {
    uint32_t r = 0u;
    if (kFormat >= 0) ld_1_ahead(on && k < cols, ckpt.scales + t * ckpt.ld_scales + k / kCkptBlock, r);
    return r;
  }
  // A lane's two groups of 8 of the block of 64 elements from kb, for q = 0 .. 3: where they begin
  static __device__ __forceinline__ int64_t group(int64_t kb, int q, int h) {
    return kFormat < 0 ? kb + 32 * h + 8 * q : kb + 16 * q + 8 * h;
  }
  // both groups: two slots of bf16, one of codes
  static constexpr int kSlots = kFormat < 0 ? 2 : 1;
  static constexpr int kSlotStep = 512;  // a lane's next slot
  __device__ __forceinline__ void copy_pair(uint8_t* dst, int64_t t, int64_t kb, int q) const {
    if constexpr (kFormat < 0) {
      copy(dst, t, group(kb, q, 0), true);
      copy(dst + kSlotStep, t, group(kb, q, 1), true);
    } else {
      const int64_t k = group(kb, q, 0);
      if (vec == 16) {
        copy_16(dst, k < cols ? ckpt.codes + t * ckpt.ld_codes + k : ckpt.codes, k < cols ? 16 : 0);
      } else {
        copy(dst, t, k, true);
        copy(dst + 8, t, k + 8, true);
      }
    }
  }
  // group h of a pair as 4 x bf16x2; a checkpoint's values are exact in bf16
  static __device__ __forceinline__ uint4 values_of(const uint8_t* src, int h, uint32_t byte) {
    if constexpr (kFormat < 0) {
      return *reinterpret_cast<const uint4*>(src + h * kSlotStep);
    } else {
      return values(*reinterpret_cast<const uint2*>(src + 8 * h), byte);
    }
  }
  static __device__ __forceinline__ uint4 values(uint2 v, uint32_t byte) {
    const float s = ckpt_scale(byte);
    return make_uint4(ckpt_values<kFormat>(v.x, s), ckpt_values<kFormat>(v.x >> 16, s), ckpt_values<kFormat>(v.y, s),
                      ckpt_values<kFormat>(v.y >> 16, s));
  }
};

// ---------------------------------------------------------------- z and dz
// A CTA takes kTG groups of 16 kMT tokens; the 8 / kTG warps of a group, and the CTAs of a cluster of csize, split
// the contracted axis in blocks of 64, kDepth blocks of tokens and factors in flight, each CTA and warp from another place on
// (all of them reading the same factors at once would queue at one slice of L2).  For each
// adapter among a group's tokens (in order of their first token) the warps multiply all the group's tokens by it and
// keep the rows of its own tokens: other rows' results are dropped, never added, so nothing passes from one request to
// another.  An adapter's factors are read from L2 once per CTA that has it (kTG groups share them through L1), so wide
// ranks take more tokens a CTA.  Where tokens are few, CTAs `turn` of `turns` share the adapters of the same
// tokens out.  Warps and ranks are summed in order.
// kDown: A_a [rank, cols] (contracted axis contiguous); else B_a [cols, rank], whose 8 x 8 blocks are
// transposed in registers.  kNT: ranks / 8 of one pass.
struct Split {
  int csize, crank, turns, turn;
};
constexpr int kDepth = 2;  // two CTAs an SM fit
template <int kMT, int kNT>
constexpr int ring_bytes() {  // of a warp: the slots of kDepth blocks
  return kDepth * (4 * kMT + 2 * kNT) * 512;
}
template <int kFormat, bool kDown, int kMT, int kTG, int kNT>
__device__ __forceinline__ void shrink_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, float* z,
                                            int64_t tile, const Split& sp, float* part, float* mark, uint8_t* rings) {
  constexpr int kGroup = 16 * kMT, kTok = kTG * kGroup, kSplits = kWarps / kTG;
  constexpr int kPair = Rows<kFormat>::kSlots * 512, kX = 2 * kMT * kPair, kBlock = kX + 2 * kNT * 512;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int tg = warp % kTG, split = warp / kTG;
  const int64_t t0 = tile * kTok, tw = t0 + tg * kGroup;
  const int rank = ad.rank;
  const int mine = lane < kGroup && tw + lane < tokens ? adapter_of(ad, tw + lane) : -1;
  const __nv_bfloat16* factors = kDown ? ad.a : ad.b;
  uint8_t* ring = rings + warp * ring_bytes<kMT, kNT>() + lane * 16;
  int64_t trow[2 * kMT];  // rows past the end are read as the last one; their results have no adapter
#pragma unroll
  for (int i = 0; i < 2 * kMT; ++i) trow[i] = min(tw + 8 * i + g, tokens - 1);
  // this warp's blocks of 64: first, first + ways, ...: `count` of them, taken from a place of its own on
  const int ways = kSplits * sp.csize, blocks = (int)((rows.cols + 63) / 64);
  const int first = (int)((sp.crank * kSplits + split + tile) % ways);
  const int count = first < blocks ? (blocks - first + ways - 1) / ways : 0;
  const int lead = count > 0 ? (int)((tile / ways) % count) : 0;
  float* out = part + (split * kTok + tg * kGroup) * rank;
  uint32_t left = __ballot_sync(0xFFFFFFFFu, mine >= 0);
  for (int nth = 0; left; ++nth) {
    const int a = __shfl_sync(0xFFFFFFFFu, mine, __ffs(left) - 1);
    const uint32_t sel = __ballot_sync(0xFFFFFFFFu, mine == a);
    left &= ~sel;
    if (nth % sp.turns != sp.turn) continue;
    for (int r0 = 0; r0 < rank; r0 += 8 * kNT) {
      float acc[kMT][kNT][4];
#pragma unroll
      for (int i = 0; i < kMT; ++i)
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
      const auto block_at = [&](int i) {
        const int at = i + lead;
        return (int64_t)(first + (at < count ? at : at - count) * ways) * 64;
      };
      uint32_t byte[2 * kMT];  // the next block's scales
      const auto fetch = [&](int i) {
        if (i < count) {
          const int64_t kb = block_at(i);
          uint8_t* dst = ring + i % kDepth * kBlock;
#pragma unroll
          for (int t = 0; t < 2 * kMT; ++t) rows.copy_pair(dst + t * kPair, trow[t], kb, q);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              uint8_t* slot = dst + kX + (h * kNT + j) * 512;
              if (kDown) {
                const int64_t k = Rows<kFormat>::group(kb, q, h);
                const int r = r0 + 8 * j + g;
                const bool on = r < rank && k < rows.cols;
                copy_16_l1(slot, on ? factors + ((int64_t)a * rank + r) * rows.cols + k : factors, on ? 16 : 0);
              } else {
                // register u of the fragment: slots 2 q', 2 q' + 1 are elements 8 q' + 2 u, + 1
                const int r = r0 + 8 * j + 2 * q;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const int64_t k = kb + 32 * h + (g >> 1) * 8 + 2 * u + (g & 1);
                  const bool on = r < rank && k < rows.cols;
                  copy_4(slot + 4 * u, on ? factors + ((int64_t)a * rows.cols + k) * rank + r : factors, on ? 4 : 0);
                }
              }
            }
        }
        copies_end();
      };
      const auto fetch_scales = [&](int i) {
#pragma unroll
        for (int t = 0; t < 2 * kMT; ++t)
          byte[t] = rows.scale(trow[t], Rows<kFormat>::group(i < count ? block_at(i) : 0, q, 0), i < count);
      };
#pragma unroll
      for (int i = 0; i < kDepth - 1; ++i) fetch(i);
      if (kFormat >= 0) fetch_scales(0);
      for (int it = 0; it < count; ++it) {
        fetch(it + kDepth - 1);
        uint32_t now[2 * kMT];
#pragma unroll
        for (int t = 0; t < 2 * kMT; ++t) now[t] = kFormat >= 0 ? byte[t] : 0u;
        if (kFormat >= 0) fetch_scales(it + 1);
        copies_wait<kDepth - 1>();
        const uint8_t* src = ring + it % kDepth * kBlock;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 w[kNT];
#pragma unroll
          for (int j = 0; j < kNT; ++j) {
            w[j] = *reinterpret_cast<const uint4*>(src + kX + (h * kNT + j) * 512);
            if (!kDown) w[j] = make_uint4(transpose_8x8(w[j].x), transpose_8x8(w[j].y), transpose_8x8(w[j].z), transpose_8x8(w[j].w));
          }
#pragma unroll
          for (int i = 0; i < kMT; ++i) {
            const uint4 lo = Rows<kFormat>::values_of(src + 2 * i * kPair, h, now[2 * i]);
            const uint4 hi = Rows<kFormat>::values_of(src + (2 * i + 1) * kPair, h, now[2 * i + 1]);
            const uint32_t a0[4] = {lo.x, hi.x, lo.y, hi.y}, a1[4] = {lo.z, hi.z, lo.w, hi.w};
#pragma unroll
            for (int j = 0; j < kNT; ++j) {
              mma_bf16(acc[i][j], a0, w[j].x, w[j].y);
              mma_bf16(acc[i][j], a1, w[j].z, w[j].w);
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
    if (sp.turns > 1) {  // this CTA's tokens
      if (split == 0 && lane < kGroup && ((sel >> lane) & 1u)) mark[tg * kGroup + lane] = 1.0f;
    }
  }
  __syncthreads();
  // the warps' partials in order, into the first warp's; then the ranks' in order
  for (int i = threadIdx.x; i < kTok * rank; i += kThreads) {
    float s = part[i];
#pragma unroll
    for (int v = 1; v < kSplits; ++v) s += part[v * kTok * rank + i];
    part[i] = s;
  }
  if (sp.csize > 1) cluster_sync(); else __syncthreads();
  const int share = (kTok * rank + sp.csize - 1) / sp.csize;
  for (int i = sp.crank * share + threadIdx.x; i < min(kTok * rank, (sp.crank + 1) * share); i += kThreads) {
    const int64_t t = t0 + i / rank;
    if (t >= tokens) continue;
    const int a = adapter_of(ad, t);
    if (a < 0 || (sp.turns > 1 && mark[i / rank] == 0.0f)) continue;
    float s = sp.csize > 1 ? ld_cluster(part + i, 0) : part[i];
    for (int d = 1; d < sp.csize; ++d) s += ld_cluster(part + i, (uint32_t)d);
    z[t0 * rank + i] = s * ad.alpha[a];
  }
  if (sp.csize > 1) cluster_sync();  // the others' shared memory stays until it has been read
}

// blockIdx.y: the turns of z (x's rows against A), then those of dz (dy's rows against B), whichever are wanted.
struct ShrinkArgs {
  Adapters ad;
  int64_t tokens;
  float *z, *dz;
  int csize, turns;
};
template <int kFormat, int kMT, int kTG, int kNT>
__global__ void __launch_bounds__(kThreads, 2) shrink_kernel(Rows<kFormat> x, Rows<-1> dy, ShrinkArgs p) {
  extern __shared__ __align__(16) uint8_t shrink_smem[];
  __shared__ float mark[16 * kMT * kTG];
  pdl_launch_dependents();  // the projection's own product needs no z
  const Split sp = {p.csize, p.csize > 1 ? (int)cluster_rank() : 0, p.turns, (int)blockIdx.y % p.turns};
  float* part = reinterpret_cast<float*>(shrink_smem + kWarps * ring_bytes<kMT, kNT>());
  if (p.turns > 1) {
    for (int i = threadIdx.x; i < 16 * kMT * kTG; i += kThreads) mark[i] = 0.0f;
    __syncthreads();
  }
  const int64_t tile = blockIdx.x / p.csize;
  if (p.z != nullptr && (int)blockIdx.y < p.turns)
    shrink_tile<kFormat, true, kMT, kTG, kNT>(x, p.tokens, p.ad, p.z, tile, sp, part, mark, shrink_smem);
  else if constexpr (kFormat >= 0)  // the forward pass has no dz
    shrink_tile<-1, false, kMT, kTG, kNT>(dy, p.tokens, p.ad, p.dz, tile, sp, part, mark, shrink_smem);
}

template <int kFormat, int kMT, int kTG, int kNT>
cudaError_t launch_shrink_of(const Rows<kFormat>& x, const Rows<-1>& dy, ShrinkArgs p, int parts, int sms, cudaStream_t stream) {
  auto kernel = shrink_kernel<kFormat, kMT, kTG, kNT>;
  constexpr int kTok = 16 * kMT * kTG;
  const auto smem_of = [](int rank) { return kWarps * ring_bytes<kMT, kNT>() + kWarps / kTG * kTok * rank * 4; };
  constexpr int kMostRanks = kNT < 4 ? 8 * kNT : kMT == 1 ? 128 : 64;
  static_assert(kWarps * ring_bytes<kMT, kNT>() + kWarps / kTG * kTok * kMostRanks * 4 <= 227 * 1024, "shared memory");
  cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem_of(kMostRanks));
  if (err != cudaSuccess) return err;
  // up to two CTAs an SM: first the contracted axis split (down to one block a warp), then the adapters
  const int64_t tiles = (p.tokens + kTok - 1) / kTok, cols = std::max(x.cols, dy.cols);
  p.csize = 1;
  while (p.csize < 8 && tiles * parts * p.csize * 2 <= 2 * sms && (int64_t)p.csize * (kWarps / kTG) * 64 < cols) p.csize *= 2;
  p.turns = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)p.ad.count, (int64_t)kTok, 2 * sms / (tiles * parts * p.csize)}));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.csize), (unsigned)(parts * p.turns), 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = (size_t)smem_of(p.ad.rank);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  err = cudaLaunchKernelEx(&cfg, kernel, x, dy, p);
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <int kFormat>
cudaError_t launch_shrink(const Rows<kFormat>& x, const Rows<-1>& dy, const ShrinkArgs& p, int parts, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int sms = info.sm_count;
  // tokens a CTA: as many as still give two CTAs an SM with the axis split eight ways, up to 32, or 128 for wide
  // ranks, whose factors weigh more than the tokens
  const auto fits = [&](int tok) { return p.tokens / tok * 8 * parts >= 2 * sms; };
  const int rank = p.ad.rank;
  if (rank > 64) return launch_shrink_of<kFormat, 1, 1, 4>(x, dy, p, parts, sms, stream);  // the partials' room
  if (rank > 16 && fits(128)) return launch_shrink_of<kFormat, 2, 4, 4>(x, dy, p, parts, sms, stream);
  if (rank > 16 && fits(64)) return launch_shrink_of<kFormat, 2, 2, 4>(x, dy, p, parts, sms, stream);
  if (fits(32)) {
    if (rank <= 8) return launch_shrink_of<kFormat, 2, 1, 1>(x, dy, p, parts, sms, stream);
    if (rank <= 16) return launch_shrink_of<kFormat, 2, 1, 2>(x, dy, p, parts, sms, stream);
    return launch_shrink_of<kFormat, 2, 1, 4>(x, dy, p, parts, sms, stream);
  }
  if (rank <= 8) return launch_shrink_of<kFormat, 1, 1, 1>(x, dy, p, parts, sms, stream);
  if (rank <= 16) return launch_shrink_of<kFormat, 1, 1, 2>(x, dy, p, parts, sms, stream);
  return launch_shrink_of<kFormat, 1, 1, 4>(x, dy, p, parts, sms, stream);
}

// ---------------------------------------------------------------- dA and dB
// A CTA (of a cluster of csize that splits the tokens) takes 64 columns of one adapter's gradient and all of
// the adapter's tokens, 16 at a time and warp, kUnits such units in flight.  As an MMA: M = ranks (z or dz transposed, as a
// pair hi + lo of bf16 numbers: 2^-17 of a value is lost), N = columns, K = tokens.  A lane loads 8 columns of four
// tokens and pairs the tokens' halves up into the fragments of 8 column tiles.  The adapter's tokens are found in windows
// of kWindow: the CTA scans their adapters and lists its own, in order, so an adapter without tokens gets
// zeros and the sums' order does not depend on anything but the tokens'.
constexpr int kUnits = 3;
constexpr int kWindow = 4096;
struct GradShared {
  uint16_t list[kWindow];
  int counts[kWarps];
};

template <int kRT>
constexpr int unit_bytes() { return 2048 + kRT * 1024; }

template <int kFormat, bool kRankMajor, int kRT>
__device__ __forceinline__ void grad_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, const float* z,
                                          __nv_bfloat16* out, int64_t col0, int a, int r0, int csize, int crank,
                                          float* part, uint8_t* rings, GradShared& sh) {
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

  // the warp's ring: a unit of 16 tokens is four slots of rows and 8 kRT words of z a lane
  constexpr int kRow = kFormat < 0 ? 512 : 256, kUnit = 4 * kRow + kRT * 1024;
  static_assert(kUnit <= unit_bytes<kRT>(), "a unit's place");
  uint8_t* ring = rings + warp * kUnits * unit_bytes<kRT>();
  uint8_t* ring_x = ring + lane * (kRow / 32);
  uint8_t* ring_z = ring + 4 * kRow + lane * 16;
  for (int64_t w0 = 0; w0 < tokens; w0 += kWindow) {
    int have = (int)min((int64_t)kWindow, tokens - w0);
    if (ad.of_token != nullptr) {
      // warp w lists tokens [w span, ..) of the window behind the warps' before it
      constexpr int kSpan = kWindow / kWarps;
      const int span = ((have + kWarps - 1) / kWarps + 31) & ~31;
      __syncthreads();
      uint32_t own[kSpan / 32];
      int count = 0;
#pragma unroll
      for (int i = 0; i < kSpan / 32; ++i) {
        const int s = 32 * i + lane, t = warp * span + s;
        own[i] = 0u;
        if (32 * i < span) own[i] = __ballot_sync(0xFFFFFFFFu, t < have && __ldg(ad.of_token + w0 + t) == a);
        count += __popc(own[i]);
      }
      if (lane == 0) sh.counts[warp] = count;
      __syncthreads();
      int at = 0;
      have = 0;
      for (int v = 0; v < kWarps; ++v) {
        if (v == warp) at = have;
        have += sh.counts[v];
      }
#pragma unroll
      for (int i = 0; i < kSpan / 32; ++i) {
        if ((own[i] >> lane) & 1u)
          sh.list[at + __popc(own[i] & ((1u << lane) - 1u))] = (uint16_t)(warp * span + 32 * i + lane);
        at += __popc(own[i]);
      }
      __syncthreads();
    }
    const int units = (have + 15) >> 4;
    const int first = crank * kWarps + warp, stride = csize * kWarps;
    const auto token = [&](int u, int i, bool& on) {  // slots 2 q, 2 q + 1, 2 q + 8, 2 q + 9
      const int e = 16 * u + 2 * q + (i & 1) + 8 * (i >> 1);
      on = e < have;
      return w0 + (on ? (ad.of_token != nullptr ? (int)sh.list[e] : e) : 0);
    };
    const auto fetch = [&](int u, int stage) {
      if (u < units) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bool on;
          const int64_t t = token(u, i, on);
          rows.copy(ring_x + stage * unit_bytes<kRT>() + i * kRow, t, col, on);
#pragma unroll
          for (int m = 0; m < kRT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int r = r0 + 16 * m + 8 * h + g;
              const bool have_z = on && r < rank;
              copy_4(ring_z + stage * unit_bytes<kRT>() + (m * 2 + h) * 512 + 4 * i, have_z ? z + t * rank + r : z, have_z ? 4 : 0);
            }
        }
      }
      copies_end();
    };
    uint32_t byte[4];  // the next unit's scales
    const auto fetch_scales = [&](int u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bool on = false;
        const int64_t t = u < units ? token(u, i, on) : 0;
        byte[i] = rows.scale(t, col, on);
      }
    };
#pragma unroll
    for (int i = 0; i < kUnits - 1; ++i) fetch(first + i * stride, i);
    if (kFormat >= 0) fetch_scales(first);
    int stage = 0;
    for (int u = first; u < units; u += stride) {
      fetch(u + (kUnits - 1) * stride, stage == 0 ? kUnits - 1 : stage - 1);
      uint32_t now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) now[i] = kFormat >= 0 ? byte[i] : 0u;
      if (kFormat >= 0) fetch_scales(u + stride);
      copies_wait<kUnits - 1>();
      uint32_t v[4][4], hi[kRT][4], lo[kRT][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 x;
        if constexpr (kFormat < 0)
          x = *reinterpret_cast<const uint4*>(ring_x + stage * unit_bytes<kRT>() + i * kRow);
        else
          x = Rows<kFormat>::values(*reinterpret_cast<const uint2*>(ring_x + stage * unit_bytes<kRT>() + i * kRow), now[i]);
        v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
      }
#pragma unroll
      for (int i = 0; i < kRT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 zq = *reinterpret_cast<const float4*>(ring_z + stage * unit_bytes<kRT>() + (i * 2 + h) * 512);
          const float zv[4] = {zq.x, zq.y, zq.z, zq.w};
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            // rows g | g + 8, slots (2 q, 2 q + 1) | (2 q + 8, 2 q + 9)
            const uint32_t p = pack_bf16(zv[2 * s], zv[2 * s + 1]);
            hi[i][2 * s + h] = p;
            lo[i][2 * s + h] = pack_bf16(zv[2 * s] - bf16_lo(p), zv[2 * s + 1] - bf16_hi(p));
          }
        }
      stage = stage + 1 == kUnits ? 0 : stage + 1;
#pragma unroll
      for (int i = 0; i < kRT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t pick = (j & 1) ? 0x7632u : 0x5410u;
          const uint32_t b0 = __byte_perm(v[0][j >> 1], v[1][j >> 1], pick);
          const uint32_t b1 = __byte_perm(v[2][j >> 1], v[3][j >> 1], pick);
          mma_bf16(acc[i][j], hi[i], b0, b1);
          mma_bf16(acc[i][j], lo[i], b0, b1);
        }
    }
  }
  // acc[i][j]: ranks 16 i + g (e 0, 1) and + 8 (e 2, 3), N slots 2 q, 2 q + 1 of column tile j, which are
  // columns 8 (2 q) + j and 8 (2 q + 1) + j.  The warps' partials: [warp][rank][64].
  constexpr int kSize = 16 * kRT * 64;
  copies_wait<0>();
  __syncthreads();  // the partials take the rings' place
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
  const int share = (kSize + csize - 1) / csize;
  for (int i = crank * share + threadIdx.x; i < min(kSize, (crank + 1) * share); i += kThreads) {
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

// blockIdx.x / csize: the column tiles of dA (tiles_a of them), then those of dB.
struct GradArgs {
  Adapters ad;
  int64_t tokens;
  const float *z, *dz;
  __nv_bfloat16 *da, *db;
  int csize, tiles_a;
};
template <int kFormat, int kRT>
__global__ void __launch_bounds__(kThreads, 2) grad_kernel(Rows<kFormat> x, Rows<-1> dy, GradArgs p) {
  extern __shared__ __align__(16) uint8_t grad_smem[];
  __shared__ GradShared sh;
  float* part = reinterpret_cast<float*>(grad_smem);  // after the rings
  const int crank = p.csize > 1 ? (int)cluster_rank() : 0, tile = blockIdx.x / p.csize, r0 = blockIdx.z * 16 * kRT;
  if (tile < p.tiles_a)
    grad_tile<kFormat, true, kRT>(x, p.tokens, p.ad, p.dz, p.da, (int64_t)tile * 64, blockIdx.y, r0, p.csize, crank, part,
                                  grad_smem, sh);
  else
    grad_tile<-1, false, kRT>(dy, p.tokens, p.ad, p.z, p.db, (int64_t)(tile - p.tiles_a) * 64, blockIdx.y, r0, p.csize, crank,
                              part, grad_smem, sh);
}

template <int kFormat, int kRT>
cudaError_t launch_grad_of(const Rows<kFormat>& x, const Rows<-1>& dy, GradArgs p, cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  auto kernel = grad_kernel<kFormat, kRT>;
  constexpr int kSmem = std::max(kWarps * 16 * kRT * 64 * 4, kWarps * kUnits * unit_bytes<kRT>());
  err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmem);
  if (err != cudaSuccess) return err;
  p.tiles_a = p.da != nullptr ? (int)((x.cols + 63) / 64) : 0;
  const int64_t tiles = p.tiles_a + (p.db != nullptr ? (dy.cols + 63) / 64 : 0);
  const int passes = (p.ad.rank + 16 * kRT - 1) / (16 * kRT);
  // the tokens split while two CTAs an SM hold all, and a warp of an adapter's share has 16 of them
  p.csize = 1;
  while (p.csize < 8 && tiles * p.ad.count * passes * (p.csize + 1) <= 2 * info.sm_count &&
         p.tokens / p.ad.count > (int64_t)p.csize * kWarps * 16)
    ++p.csize;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.csize), (unsigned)p.ad.count, (unsigned)passes);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  err = cudaLaunchKernelEx(&cfg, kernel, x, dy, p);
  return err != cudaSuccess ? err : cudaGetLastError();
}

Rows<-1> bf16_rows(const void* x, int64_t ld, int64_t cols) { return {static_cast<const uint16_t*>(x), ld, {}, cols, 1}; }

template <int kFormat>
Rows<kFormat> ckpt_rows(const Checkpoint& c, int64_t cols) {
  const uintptr_t base = reinterpret_cast<uintptr_t>(c.codes);
  const int vec = base % 16 == 0 && c.ld_codes % 16 == 0 ? 16 : base % 8 == 0 && c.ld_codes % 8 == 0 ? 8 : 1;
  return {nullptr, 0, c, cols, vec};
}

template <int kFormat>
cudaError_t backward_products(const Checkpoint& c, int64_t n, const Rows<-1>& dy, const ShrinkArgs& p, cudaStream_t stream) {
  const int parts = (p.z != nullptr) + (p.dz != nullptr);
  return launch_shrink<kFormat>(ckpt_rows<kFormat>(c, n), dy, p, parts, stream);
}
template <int kFormat>
cudaError_t gradients(const Checkpoint& c, int64_t n, const Rows<-1>& dy, const GradArgs& p, cudaStream_t stream) {
  const Rows<kFormat> x = ckpt_rows<kFormat>(c, n);
  return p.ad.rank <= 16 ? launch_grad_of<kFormat, 1>(x, dy, p, stream) : launch_grad_of<kFormat, 2>(x, dy, p, stream);
}

}  // namespace

cudaError_t launch_adapter_down(const void* x, int64_t ld_x, int64_t tokens, int64_t n, const Adapters& ad, float* z,
                                cudaStream_t stream) {
  const ShrinkArgs p = {ad, tokens, z, nullptr, 1, 1};
  return launch_shrink<-1>(bf16_rows(x, ld_x, n), bf16_rows(nullptr, 0, 0), p, 1, stream);
}

cudaError_t launch_adapter_backward(const Checkpoint& x, int format, int64_t n, const void* dy, int64_t ld_dy, int64_t m,
                                    int64_t tokens, const Adapters& ad, float* z, float* dz, cudaStream_t stream) {
  const ShrinkArgs p = {ad, tokens, z, dz, 1, 1};
  const Rows<-1> rows = bf16_rows(dy, ld_dy, m);
  return format == kCkptE4M3 ? backward_products<kCkptE4M3>(x, n, rows, p, stream)
                             : backward_products<kCkptInt8>(x, n, rows, p, stream);
}

cudaError_t launch_adapter_gradients(const Checkpoint& x, int format, int64_t n, const void* dy, int64_t ld_dy, int64_t m,
                                     int64_t tokens, const Adapters& ad, const float* z, const float* dz, void* da, void* db,
                                     cudaStream_t stream) {
  const GradArgs p = {ad, tokens, z, dz, static_cast<__nv_bfloat16*>(da), static_cast<__nv_bfloat16*>(db), 1, 0};
  const Rows<-1> rows = bf16_rows(dy, ld_dy, m);
  return format == kCkptE4M3 ? gradients<kCkptE4M3>(x, n, rows, p, stream) : gradients<kCkptInt8>(x, n, rows, p, stream);
}

}  // namespace hscale
