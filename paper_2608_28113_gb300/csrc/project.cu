// project.cu -- the product of activations with a packed NVFP4 weight on the tcgen05 tensor cores, with each
// token's adapter added as the result leaves tensor memory:
//   y_t  = W_hat x_t + B_a z_t        (forward;  z  = alpha_a A_a x_t,    adapter.cu)
//   dx_t = W_hat^T dy_t + A_a^T dz_t  (backward; dz = alpha_a B_a^T dy_t, adapter.cu)
// Accumulated in fp32 and rounded once, to bf16.
//
// The weight never exists in bf16 outside shared memory.  E2M1 times E4M3 has at most 6 significant bits, so
// each weight without s_g is exact in bf16 (2^-7 of it is what the tile holds, see unpack8); s_g is a
// factor of the accumulator.
//
// Tile: 128 outputs (M, the weight) x kN tokens (N), K in blocks of 64.  18 warps:
//   0      TMA loads of the tokens' tile, K-major, 128-byte swizzle
//   1      MMAs
//   2-5    epilogue: tensor memory -> s_g, adapter, bf16 -> out (lane = output, columns = tokens)
//   6-17   the weight's tile: three groups of four warps take the K blocks in turn, 32 packed bytes and 4 codes
//          a thread, kept kAhead of the group's blocks ahead in registers and unpacked into the swizzled tile (the
//          groups' waits and fences overlap; all warps on one block was slower).  Forward (K = n) the tile is K-major,
//          backward (K = m, outputs = n) the same packed rows make it MN-major, so W is read as it is stored.
// Each weight is unpacked once per kN tokens: about 2.7 instructions a weight against kN / 64 tensor-core
// cycles, so at kN = 256 the unpacking hides behind the MMAs.
//
// What bounds it.  Many tokens: the tensor cores, 0.78 of the measured bf16 rate (8192 tokens, 14336 x 4096: 650 us without
// adapters, 1.48 PFLOP/s); the rest is the ring's four stages, whose hand-over the unpacking warps' issue and shared-memory
// writes delay.  Few tokens: the K blocks' chain, 0.2-0.34 us each whatever the rate (launch_project's estimate).
//
// Where the tiles leave SMs idle, a cluster of csize CTAs splits K: each rank accumulates its share, hands the
// others the columns they own through distributed shared memory (all warps but two take part), and finishes its own
// columns, summing in rank order.  With csize 1 the grid is persistent and the epilogue of a tile runs beside the MMAs
// of the next (two accumulators in tensor memory).
//
// The adapters' terms.  An adapter with enough tokens in a tile takes its term on the tensor cores: after the
// weight's K blocks the epilogue's warps, idle by then, write its factors and its tokens' z (as a pair hi + lo of
// bf16 numbers, so 2^-17 of it is lost; zeros for the other tokens) as one more K block per 32 ranks or per two or
// four adapters of fewer ranks, fetched before the stage is free.  A block takes them 0.8 us (load, write, fence), so 16
// adapters in requests cost 8192 tokens 20-35 us, and 32 adapters in any order cost 2048 tokens 35 us.  An adapter
// with few tokens there ("loose": a decoding batch) is cheaper in the epilogue itself, a dot product of `rank` fp32
// numbers per result; these are bound by the four warps' instructions (64 tokens of 64 adapters, 14336 x 4096: 35.5 us
// in the kernel, 23.5 without adapters).  Zeros times factors are zeros only while the
// factors are finite: an output whose factors hold an Inf or NaN is left out of the K block, and the tokens
// of that adapter get NaN there; so nothing passes from one request's adapter to another's tokens.
// Which adapters a tile has is found by one warp, two tiles ahead (TileInfo).
//
// 576 threads leave 96 registers each: the large tiles' instances spill (bytes stored and loaded, by the compiler: 256 tokens
// backward 136 and 68, 128 backward 108 and 56, 256 forward 28 and 20, 128 forward 20 and 28), the others do not.
//
// Every wait is bounded; a CTA in which one ran out writes NaN for what it owed and sets the error flag.
#include <algorithm>

#include "hscale_internal.h"
#include "nvfp4_weight.cuh"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace hscale {
namespace {

constexpr int kBM = 128, kBK = 64;
constexpr int kThreads = 576;
constexpr int kUnpackWarp0 = 6, kUnpackGroups = 3, kGroupThreads = 128;
constexpr int kAhead = 2;  // blocks of its own that a group has in flight
constexpr uint32_t kTileABytes = kBM * kBK * 2;  // 16 KB
constexpr uint32_t kGroupBytes = 64 * kBK * 2;   // MN-major: 64 outputs x 64 rows of K
constexpr int kInfos = 4;                        // TileInfo of as many tiles
constexpr uint32_t kInfoBytes = 576;
constexpr uint32_t kBarBytes = 512;
constexpr uint32_t kTurnBytes = 4 * 2048;        // of the epilogue's warps: z, and results on their way out
constexpr int kGo = 16;                          // tiles whose place in the ring's order is kept: more than it has stages

template <int kN>
struct Tile {
  // a small batch's loose terms are made beside the MMAs and kept (14336 x 4096, 64 tokens of 64 adapters: 53 -> 49.5 us)
  static constexpr bool kStash = kN <= 64;
  static constexpr int kStages = kN == 256 ? 4 : kN == 128 ? 5 : 6;
  static constexpr uint32_t kBBytes = kN * kBK * 2;
  static constexpr uint32_t kStageBytes = kTileABytes + kBBytes;
  static constexpr uint32_t kSmemBytes = kStages * kStageBytes + 1024 /* alignment */ + kBarBytes + kTurnBytes +
                                         kInfos * kInfoBytes + 1024 /* bad */ + (kStash ? kN * kBM * 4 : 0);

  static constexpr uint32_t kTmemCols = 2 * kN;
};

__device__ uint32_t g_project_flags = 0;

struct ProjectArgs {
  Nvfp4Weight w;
  Adapters ad;
  const float* z;
  const uint32_t* z_split;
  __nv_bfloat16* out;
  int64_t tokens, ld_out;
  int32_t kb_total, tiles_t, tiles_o, csize, chained;
};

// ---------------------------------------------------------------- weights
// Eight nibbles times a scale (bf16x2, both halves): a nibble's magnitude bits at bf16's bits 8-6 read as
// E2M1 2^-126, so with scales E4M3 2^119 the products are the weights 2^-7, exact.
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t scale, uint32_t (&r)[4]) {
  constexpr uint32_t kSign = 0x80008000u, kMag = 0x01C001C0u;
  const uint32_t up = w << 4;
  // halves (nibble 0 | 2 at bits 4 | 12, nibble 1 | 3 likewise), and the same of nibbles 4-7
  const uint32_t a = __byte_perm(up, w, 0x5410), b = __byte_perm(up, w, 0x7632);
  r[0] = mul_bf16x2(((a << 8) & kSign) | ((a << 2) & kMag), scale);
  r[1] = mul_bf16x2((a & kSign) | ((a >> 6) & kMag), scale);
  r[2] = mul_bf16x2(((b << 8) & kSign) | ((b << 2) & kMag), scale);
  r[3] = mul_bf16x2((b & kSign) | ((b >> 6) & kMag), scale);
}

__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

__device__ __forceinline__ void tmem_ld_32x32b_x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

// ---------------------------------------------------------------- epilogue
// The 8 factors r0 .. r0 + 7 that adapter a has for output o, as 4 x bf16x2: B_a[o, r] (contiguous) or A_a[r, o].
template <bool kForward>
__device__ __forceinline__ uint4 factors8(const ProjectArgs& p, int a, int64_t o, int r0, bool on) {
  uint4 q = make_uint4(0u, 0u, 0u, 0u);
  if (!on) return q;
  if (kForward) return ld_nc_v4(p.ad.b + ((int64_t)a * p.w.m + o) * p.ad.rank + r0);
  uint32_t e[8];
  const uint16_t* src = reinterpret_cast<const uint16_t*>(p.ad.a) + ((int64_t)a * p.ad.rank + r0) * p.w.n + o;
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = __ldg(src + i * p.w.n);
  q.x = e[0] | e[1] << 16, q.y = e[2] | e[3] << 16, q.z = e[4] | e[5] << 16, q.w = e[6] | e[7] << 16;
  return q;
}
__device__ __forceinline__ float dot8(const float* z, const float (&f)[8], float s) {
  const float4 z0 = reinterpret_cast<const float4*>(z)[0], z1 = reinterpret_cast<const float4*>(z)[1];
  s = fmaf(z0.x, f[0], s), s = fmaf(z0.y, f[1], s), s = fmaf(z0.z, f[2], s), s = fmaf(z0.w, f[3], s);
  s = fmaf(z1.x, f[4], s), s = fmaf(z1.y, f[5], s), s = fmaf(z1.z, f[6], s), s = fmaf(z1.w, f[7], s);
  return s;
}
__device__ __forceinline__ void unpack_factors(const uint4& q, float (&f)[8]) {
  f[0] = bf16_lo(q.x), f[1] = bf16_hi(q.x), f[2] = bf16_lo(q.y), f[3] = bf16_hi(q.y);
  f[4] = bf16_lo(q.z), f[5] = bf16_hi(q.z), f[6] = bf16_lo(q.w), f[7] = bf16_hi(q.w);
}

// Tokens t0 .. t0 + W - 1 and this lane's output o: each loose token's adapter added to v.  loose: bit j where token
// t0 + j's term is added here.  zs: 2 KB of the warp's own.  Eight ranks a pass: each lane fetches its token's z into zs,
// from where every lane reads all of them; z and factors of the next pass are fetched before the present one's
// products.  Tokens on one adapter share a lane's 8 factors; otherwise the factors of 8 tokens are fetched at once.
// A token without an adapter keeps v as it is (no product by zero: the factors may be Inf or NaN).
template <bool kForward, int W>
__device__ __forceinline__ void add_loose(float (&v)[W], int64_t t0, int64_t o, int lane, const ProjectArgs& p, uint32_t loose,
                                       float* zs) {
  const bool on = o < (kForward ? p.w.m : p.w.n);
  int id = -1;
  if (lane < W && ((loose >> lane) & 1u)) id = adapter_of(p.ad, t0 + lane);
  const uint32_t with = __ballot_sync(0xFFFFFFFFu, id >= 0);
  if (with) {
    const int rank = p.ad.rank;
    const int a0 = __shfl_sync(0xFFFFFFFFu, id, __ffs(with) - 1);
    const bool one = __all_sync(0xFFFFFFFFu, id < 0 || id == a0);
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    const float4* zp = reinterpret_cast<const float4*>(p.z + (t0 + lane) * rank);
    float4 z0 = id >= 0 ? zp[0] : zero, z1 = id >= 0 ? zp[1] : zero;
    uint4 q = one ? factors8<kForward>(p, a0, o, 0, on) : make_uint4(0u, 0u, 0u, 0u);
    for (int r0 = 0; r0 < rank; r0 += 8) {
      __syncwarp();
      if (lane < W) {
        reinterpret_cast<float4*>(zs)[2 * lane] = z0;
        reinterpret_cast<float4*>(zs)[2 * lane + 1] = z1;
      }
      __syncwarp();
      float f[8];
      unpack_factors(q, f);
      if (r0 + 8 < rank) {
        zp += 2;
        if (id >= 0) z0 = zp[0], z1 = zp[1];
        if (one) q = factors8<kForward>(p, a0, o, r0 + 8, on);
      }
      if (one) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float s = dot8(zs + 8 * j, f, v[j]);
          v[j] = ((with >> j) & 1u) ? s : v[j];
        }
      } else {
#pragma unroll
        for (int j0 = 0; j0 < W; j0 += 8) {
          uint4 e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int a = __shfl_sync(0xFFFFFFFFu, id, j0 + j);
            e[j] = factors8<kForward>(p, a, o, r0, on && a >= 0);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            unpack_factors(e[j], f);
            const float s = dot8(zs + 8 * (j0 + j), f, v[j0 + j]);
            v[j0 + j] = ((with >> (j0 + j)) & 1u) ? s : v[j0 + j];
          }
        }
      }
    }
  }
}

// v rounded and stored.
template <bool kForward, int W>
__device__ __forceinline__ void store(const float (&v)[W], int64_t t0, int64_t o, int lane, const ProjectArgs& p, float* zs) {
  // Rounded, and turned in zs (pairs of tokens, an output a lane) so that a lane stores 8 outputs of a token at once:
  // stores of one output a lane kept the epilogue from the next tile's adapters (8192 x 14336 x 4096, rank 16: 806 us,
  // 727 now)
  uint32_t* turn = reinterpret_cast<uint32_t*>(zs);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < W / 2; ++j) turn[j * 32 + lane] = pack_bf16(v[2 * j], v[2 * j + 1]);
  __syncwarp();
  const int64_t outs = kForward ? p.w.m : p.w.n, first = o - lane;
#pragma unroll
  for (int i = lane; i < W * 2; i += 32) {
    const int pair = i >> 2, group = i & 3;
    const uint4 a = reinterpret_cast<const uint4*>(turn)[pair * 8 + group * 2];
    const uint4 b = reinterpret_cast<const uint4*>(turn)[pair * 8 + group * 2 + 1];
    const int64_t t = t0 + 2 * pair, at = first + 8 * group;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (t + e >= p.tokens) continue;
      const uint32_t pick = e ? 0x7632u : 0x5410u;
      const uint4 r = make_uint4(__byte_perm(a.x, a.y, pick), __byte_perm(a.z, a.w, pick), __byte_perm(b.x, b.y, pick),
                                 __byte_perm(b.z, b.w, pick));
      uint16_t* dst = reinterpret_cast<uint16_t*>(p.out) + (t + e) * p.ld_out + at;
      if (at + 8 <= outs) {
        *reinterpret_cast<uint4*>(dst) = r;
      } else {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (at + k < outs) dst[k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
      }
    }
  }
}

constexpr int kMaxListed = 32;  // adapters of a tile that may take their term on the tensor cores
// The adapters of a tile of kN <= 256 tokens.
struct TileInfo {
  int listed, blocks;            // adapters on the tensor cores, K blocks that they add
  uint32_t loose[8];             // tokens whose term the epilogue adds
  int adapter[kMaxListed];
  uint32_t sel[kMaxListed];      // bit b: the adapter has tokens among 16 b .. 16 b + 15
  uint8_t index[256];            // a token's place in the list, or 255
};
static_assert(sizeof(TileInfo) <= kInfoBytes, "TileInfo's place");
// A K block of the adapters: [factors | factors] times [hi | lo] of 8, 16 or 32 ranks, of as many adapters as fit in
// 64.
__device__ __forceinline__ int half_ranks(int rank) { return rank <= 8 ? 8 : rank <= 16 ? 16 : 32; }
__device__ __forceinline__ int adapters_a_block(int rank) { return rank <= 8 ? 4 : rank <= 16 ? 2 : 1; }
__device__ __forceinline__ int blocks_of(int listed, int rank) {
  const int per = adapters_a_block(rank);
  return (listed + per - 1) / per * ((rank + 31) >> 5);
}

// A K block costs the epilogue's warps about 1500 cycles; a loose token about 112 cycles per 8 ranks forward, where its
// factors are 16 bytes an output, and 450 backward, where they are 8 loads (eight tokens' factors fetched at once).  An
// adapter is listed where its tokens' share would cost more than its part of a K block.  None is where the
// accumulator's unit is so far from 1 that z in it may leave fp32's range (a global scale of 0 among them).
// One pass over the words of 32 tokens: each token's place among the tile's adapters, in order of their first tokens,
// then the choice (a pass over the tokens for each adapter took 32 adapters 11 us a tile).  seen: 2 KB of the warp's own.
template <bool kForward, int kN>
__device__ __forceinline__ void find_adapters(const ProjectArgs& p, int64_t t0, int lane, TileInfo& info, int* seen) {
  constexpr int kWords = kN / 32;
  int* held = seen + 256;  // of each adapter seen: its tokens << 16 | its bits of sel; then its place in the list
  int at[kWords];          // a token's place in seen, or none
  int id[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const int64_t t = t0 + 32 * i + lane;
    id[i] = t < p.tokens ? adapter_of(p.ad, t) : -1;
  }
  int count = 0;  // seen
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    at[i] = -1;
#pragma unroll 4
    for (int k = 0; k < count; ++k)
      if (seen[k] == id[i]) at[i] = k;  // none is negative
    const uint32_t alike = __match_any_sync(0xFFFFFFFFu, id[i]);
    const bool leads = id[i] >= 0 && __ffs(alike) - 1 == lane;
    const uint32_t fresh = __ballot_sync(0xFFFFFFFFu, leads && at[i] < 0);
    if (leads) {
      const int value = __popc(alike) << 16 | ((alike & 0xFFFFu ? 1 : 0) | (alike >> 16 ? 2 : 0)) << (2 * i);
      if (at[i] < 0) {
        at[i] = count + __popc(fresh & ((1u << lane) - 1u));
        seen[at[i]] = id[i], held[at[i]] = value;
      } else {
        held[at[i]] += value;  // another word's bits
      }
    }
    at[i] = __shfl_sync(0xFFFFFFFFu, at[i], __ffs(alike) - 1);
    count += __popc(fresh);
    __syncwarp();
  }
  const int block = 1500 * ((p.ad.rank + 31) / 32) / adapters_a_block(p.ad.rank), loose_token = (kForward ? 14 : 56) * p.ad.rank;
  const float unit = fabsf(*p.w.global_scale * kWeightUnit);  // read again: a register over the tile's loops costs more
  const bool in_range = unit >= 0x1p-64f && unit <= 0x1p64f;
  const int enough = in_range ? (block + loose_token - 1) / loose_token : INT32_MAX;
  int listed = 0;
  for (int k0 = 0; k0 < count; k0 += 32) {
    const int k = k0 + lane, value = k < count ? held[k] : 0;
    const uint32_t take = __ballot_sync(0xFFFFFFFFu, k < count && value >> 16 >= enough);
    const int place = listed + __popc(take & ((1u << lane) - 1u));
    const bool on = ((take >> lane) & 1u) && place < kMaxListed;
    if (on) info.adapter[place] = seen[k], info.sel[place] = (uint32_t)value & 0xFFFFu;
    if (k < count) held[k] = on ? place : 255;
    listed = min(listed + __popc(take), kMaxListed);
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const int place = at[i] >= 0 ? held[at[i]] : 255;
    info.index[32 * i + lane] = (uint8_t)place;
    const uint32_t loose = __ballot_sync(0xFFFFFFFFu, at[i] >= 0 && place == 255);
    if (lane == i) info.loose[i] = loose;
  }
  if (lane == 0) info.listed = listed, info.blocks = blocks_of(listed, p.ad.rank);
  __syncwarp();
}

// Bits of a register's bf16 halves that are Inf or NaN (0xFFFF each).
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return __vcmpeq2(w & 0x7F807F80u, 0x7F807F80u); }

// The K block of ranks r0 .. of the list's adapters from e on, by the epilogue's 128 threads: the factors (as the
// weight's tile) and the z of their tokens (as the tokens' tile; z_split: the accumulator is in units of 128 s_g), zeros
// for the other tokens.  Loaded before `acquire` waits for the stage.  bad[output] gets an adapter's bit
// where a factor is Inf or NaN.
template <bool kForward, int kN, typename Acquire>
__device__ __forceinline__ bool adapter_block(const ProjectArgs& p, const TileInfo& info, int e, int r0, int64_t t0, int64_t o0,
                                              int line, uint32_t* bad, uint8_t* tile_a, uint8_t* tile_b,
                                              Acquire acquire) {
  constexpr int kRows = (kN + 127) / 128;
  const int rank = p.ad.rank, half = half_ranks(rank), hc = half / 8, per = adapters_a_block(rank);
  const int hs = rank <= 8 ? 0 : rank <= 16 ? 1 : 2;  // hc = 2^hs
  // 16-byte piece i of the factors: forward ranks 8 (i % hc) .. of this output, of adapter e + i / hc; backward 8 outputs of
  // row (line + 128 i) / 16 of the block's 32 rows of factors
  const auto owner = [&](int i) { return kForward ? i >> hs : (line + i * 128) >> (7 + hs); };
  uint4 f[4], hi[kRows][4], lo[kRows][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = make_uint4(0u, 0u, 0u, 0u);
    const int sub = owner(i);
    if (e + sub >= info.listed) continue;
    const int64_t a = info.adapter[e + sub];
    if (kForward) {
      const int r = r0 + 8 * (i & (hc - 1));
      if (o0 + line < p.w.m && r < rank) f[i] = ld_nc_v4(p.ad.b + (a * p.w.m + o0 + line) * rank + r);
    } else {
      const int r = r0 + (((line + i * 128) >> 4) & (half - 1));
      const int64_t o = o0 + (line & 15) * 8;
      if (o < p.w.n && r < rank) f[i] = ld_nc_v4(p.ad.a + (a * rank + r) * p.w.n + o);
    }
  }
  int mine[kRows];  // the row's adapter among the block's, or none
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int t = line + 128 * k, index = info.index[t < kN ? t : 0];
    mine[k] = t < kN && index >= e && index < e + per ? index - e : -1;  // 255: none
    const uint4* src = reinterpret_cast<const uint4*>(p.z_split + (t0 + t) * rank + r0);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint4 v0 = make_uint4(0u, 0u, 0u, 0u), v1 = v0;
      if (mine[k] >= 0 && c < hc && r0 + 8 * c < rank) v0 = src[2 * c], v1 = src[2 * c + 1];
      hi[k][c] = make_uint4(__byte_perm(v0.x, v0.y, 0x5410), __byte_perm(v0.z, v0.w, 0x5410), __byte_perm(v1.x, v1.y, 0x5410),
                            __byte_perm(v1.z, v1.w, 0x5410));
      lo[k][c] = make_uint4(__byte_perm(v0.x, v0.y, 0x7632), __byte_perm(v0.z, v0.w, 0x7632), __byte_perm(v1.x, v1.y, 0x7632),
                            __byte_perm(v1.z, v1.w, 0x7632));
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!(not_finite(f[i].x) | not_finite(f[i].y) | not_finite(f[i].z) | not_finite(f[i].w))) continue;
    const uint32_t bit = 1u << (e + owner(i));
    uint32_t w[4] = {f[i].x, f[i].y, f[i].z, f[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t x = not_finite(w[j]);
      if (kForward) {
        if (x) atomicOr(&bad[line], bit);
      } else {
        if (x & 0xFFFFu) atomicOr(&bad[(line & 15) * 8 + 2 * j], bit);
        if (x >> 16) atomicOr(&bad[(line & 15) * 8 + 2 * j + 1], bit);
      }
      w[j] &= ~x;
    }
    f[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  int s;
  if (!acquire(s)) return false;
  uint8_t* ta = tile_a + s * kTileABytes;
  uint8_t* tb = tile_b + s * Tile<kN>::kBBytes;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int sub = owner(i);
    if (kForward) {
      const int c = sub * 2 * hc + (i & (hc - 1));
      *reinterpret_cast<uint4*>(ta + line * 128 + ((c ^ (line & 7)) << 4)) = f[i];
      *reinterpret_cast<uint4*>(ta + line * 128 + (((c + hc) ^ (line & 7)) << 4)) = f[i];
    } else {
      const int r = sub * 2 * half + (((line + i * 128) >> 4) & (half - 1)), c = line & 7;
      uint8_t* dst = ta + ((line >> 3) & 1) * kGroupBytes + r * 128 + ((c ^ (r & 7)) << 4);
      *reinterpret_cast<uint4*>(dst) = f[i];
      *reinterpret_cast<uint4*>(dst + half * 128) = f[i];
    }
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int t = line + 128 * k;
    if (t >= kN) continue;
    uint8_t* dst = tb + t * 128;
    const int at = mine[k] * 2 * hc;  // the row's first 16 bytes that are not zeros
    if (per > 1) {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (mine[k] < 0 || c < at || c >= at + 2 * hc) *reinterpret_cast<uint4*>(dst + ((c ^ (t & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
      if (mine[k] < 0) continue;
    }
    const int first = per > 1 ? at : 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (c >= hc) continue;
      *reinterpret_cast<uint4*>(dst + (((first + c) ^ (t & 7)) << 4)) = hi[k][c];
      *reinterpret_cast<uint4*>(dst + (((first + c + hc) ^ (t & 7)) << 4)) = lo[k][c];
    }
  }
  return true;
}

// Tile t of the persistent order: groups of 8 token tiles, the outputs' tiles along a group, so that the
// tiles in flight at once share token tiles and weights in L2.
__device__ __forceinline__ void raster(int t, const ProjectArgs& p, int& tt, int& to) {
  const int group = t / (8 * p.tiles_o) * 8;
  const int rows = min(8, p.tiles_t - group);
  const int within = t - group * p.tiles_o;
  tt = group + within % rows;
  to = within / rows;
}

// NaN where this output's factors of the token's adapter were left out of the K block.
template <int W>
__device__ __forceinline__ void spoil(uint32_t (&q)[W], uint32_t bad, const uint8_t* index) {
  if (!__any_sync(0xFFFFFFFFu, bad != 0u)) return;
#pragma unroll
  for (int j = 0; j < W; ++j)
    if (index[j] < kMaxListed && ((bad >> index[j]) & 1u)) q[j] = 0x7FC00000u;
}
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <bool kForward, int kN>
__global__ void __launch_bounds__(kThreads, 1)
project_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ ProjectArgs p) {
  using T = Tile<kN>;
  constexpr int kStages = T::kStages;
  extern __shared__ __align__(16) uint8_t dynamic_smem[];
  uint8_t* smem = dynamic_smem + ((1024u - (smem_addr(dynamic_smem) & 1023u)) & 1023u);
  uint8_t* tile_a = smem;
  uint8_t* tile_b = smem + kStages * kTileABytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + kStages * T::kStageBytes);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* info_full = acc_empty + 2;
  uint64_t* slot = info_full + kInfos;  // a stage is free for an adapter's block
  uint64_t* go_full = slot + kStages;   // a tile's place in the ring's order is known
  uint64_t* mma_done = go_full + kGo;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  uint32_t* failed = tmem_slot + 1;
  int* place = reinterpret_cast<int*>(failed + 1);  // [kGo]
  float* zs = reinterpret_cast<float*>(smem + kStages * T::kStageBytes + kBarBytes) + (threadIdx.x >> 5 & 3) * (kTurnBytes / 16);
  uint8_t* info_base = smem + kStages * T::kStageBytes + kBarBytes + kTurnBytes;
  uint32_t* bad = reinterpret_cast<uint32_t*>(info_base + kInfos * kInfoBytes);  // [2][128]
  float* stash = reinterpret_cast<float*>(bad + 256);                             // [kN][128]
  auto info_of = [&](int i) -> TileInfo& { return *reinterpret_cast<TileInfo*>(info_base + (i % kInfos) * kInfoBytes); };

  const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int csize = p.csize;
  const int crank = csize > 1 ? (int)cluster_rank() : 0;
  const int tiles = p.tiles_t * p.tiles_o;
  // csize 1: tiles blockIdx.x, + gridDim.x, ...; else one tile a cluster, K blocks [kb0, kb1) of it
  const int first = csize > 1 ? (int)blockIdx.x / csize : (int)blockIdx.x;
  const int step = (int)gridDim.x;
  const int ntiles = csize > 1 ? 1 : (tiles - first + step - 1) / step;
  const int kb0 = (int)((int64_t)p.kb_total * crank / csize), kb1 = (int)((int64_t)p.kb_total * (crank + 1) / csize);
  const int kbs = kb1 - kb0;
  const bool adapters = p.ad.count > 0, adds = adapters && crank == csize - 1;  // the last rank adds the K blocks

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1 + kGroupThreads / 32);  // the TMA load and the unpacking group's warps
      mbar_init(&empty[s], 1);
      mbar_init(&slot[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 128);
    }
    for (int i = 0; i < kInfos; ++i) mbar_init(&info_full[i], 1);
    for (int i = 0; i < kGo; ++i) mbar_init(&go_full[i], 1);
    mbar_init(mma_done, 1);
    *failed = 0u;
    mbar_fence_init();
    prefetch_tensormap(&vmap);
  }
  if (warp == 1) {
    tmem_alloc(smem_addr(tmem_slot), T::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem_d = warp_uniform(*tmem_slot);

  // the epilogue's thread: tensor-memory lane, output of a tile
  const uint32_t quarter = (uint32_t)(warp & 3);
  const uint32_t lane_base = (quarter * 32u) << 16;
  const int out_row = (int)quarter * 32 + lane;
  bool have = true;  // of the epilogue's warps: no wait has run out
  // the adapters of the CTA's tile i
  auto wait_info = [&](int i) { return mbar_wait_warp(&info_full[i % kInfos], (uint32_t)(i / kInfos) & 1u); };

  if (warp == 0) {
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    int extras = 0;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      int tt, to;
      raster(first + i * step, p, tt, to);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_warp(&empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(&full[s], T::kBBytes);
          tma_load_2d(tile_b + s * T::kBBytes, &vmap, kb * kBK, tt * kN, &full[s], policy);
        }
        __syncwarp();
        if (++s == kStages) {
          s = 0;
          parity ^= 1u;
        }
      }
      // the adapters' blocks are the epilogue warps' alone, which this warp tells when a stage is theirs (they come
      // from far behind in the ring's order, and the parity of `empty` only tells neighbouring turns apart)
      if (adds && go && !(go = wait_info(i)) && lane == 0) atomicOr(failed, 1u);
      const int extra = adds && go ? info_of(i).blocks : 0;
      for (int e = 0; e < extra; ++e) {
        if (!mbar_wait_warp(&empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive(&full[s]);
          mbar_arrive(&slot[s]);
        }
        __syncwarp();
        if (++s == kStages) {
          s = 0;
          parity ^= 1u;
        }
      }
      // the unpacking warps skip them: the next tile's place, told once this warp has come to it
      extras += extra;
      if (adds && go && lane == 0) {
        place[i % kGo] = (i + 1) * kbs + extras;
        mbar_arrive(&go_full[i % kGo]);
      }
    }
    // a full barrier also waits for the unpacking warps, whose waits are bounded like this one's
    ring_drain(full, kStages, s, parity);
  } else if (warp == 1) {
    constexpr uint32_t kMajor = kForward ? 0u : 1u << 15;
    constexpr uint32_t kIdesc = idesc_bf16_f32(kBM, kN) | kMajor;
    constexpr uint32_t kStepA = kForward ? 2 : 128;  // 16 of K further in the descriptor
    uint32_t s = 0, parity = 0;
    bool ok = true;
    for (int i = 0; i < ntiles && ok; ++i) {
      const uint32_t acc = (uint32_t)i & 1u;
      if (i >= 2 && !mbar_wait_warp(&acc_empty[acc], (uint32_t)((i >> 1) - 1) & 1u)) {
        ok = false;
        break;
      }
      tc_fence_after_sync();
      for (int kb = 0; kb < kbs; ++kb) {
        if (!mbar_wait_warp(&full[s], parity)) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        if (elect_one()) {
          const uint32_t a = smem_addr(tile_a + s * kTileABytes), b = smem_addr(tile_b + s * T::kBBytes);
          const uint64_t ad = kForward ? smem_desc_k_sw128(a) : smem_desc_mn_sw128(a, kGroupBytes);
          const uint64_t bd = smem_desc_k_sw128(b);
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk)
            umma_bf16(tmem_d + acc * kN, ad + kStepA * kk, bd + 2 * kk, kIdesc, (uint32_t)(kb > 0 || kk > 0));
          umma_commit(smem_addr(&empty[s]));
        }
        __syncwarp();
        if (++s == kStages) {
          s = 0;
          parity ^= 1u;
        }
      }
      if (adds && ok) ok = wait_info(i);
      if (adds && ok) {
        const TileInfo& info = info_of(i);
        const int per = adapters_a_block(p.ad.rank);
        for (int e = 0; e < info.listed && ok; e += per) {
          uint32_t sel = 0u;
          const int subs = min(per, info.listed - e);
          for (int k = 0; k < subs; ++k) sel |= info.sel[e + k];
          for (int r0 = 0; r0 < p.ad.rank && ok; r0 += 32) {
            if (!mbar_wait_warp(&full[s], parity)) {
              ok = false;
              break;
            }
            tc_fence_after_sync();
            const uint32_t a = smem_addr(tile_a + s * kTileABytes), b = smem_addr(tile_b + s * T::kBBytes);
            const uint64_t ad = kForward ? smem_desc_k_sw128(a) : smem_desc_mn_sw128(a, kGroupBytes);
            const uint64_t bd = smem_desc_k_sw128(b);
            const int steps = subs * half_ranks(p.ad.rank) / 8;
            if (elect_one()) {
              for (uint32_t runs = sel; runs;) {  // each run of neighbouring blocks
                const int b0 = __ffs(runs) - 1, len = __ffs(~(runs >> b0)) - 1;
                runs &= ~(((1u << len) - 1u) << b0);
                const uint32_t idesc = idesc_bf16_f32(kBM, 0) | kMajor | ((uint32_t)(2 * len) << 17);
                for (int kk = 0; kk < steps; ++kk)
                  umma_bf16(tmem_d + acc * kN + 16 * b0, ad + kStepA * kk, bd + 128 * b0 + 2 * kk, idesc, 1u);
              }
              umma_commit(smem_addr(&empty[s]));
            }
            __syncwarp();
            if (++s == kStages) {
              s = 0;
              parity ^= 1u;
            }
          }
        }
      }
      // fires once every MMA issued above has completed
      if (ok && elect_one()) umma_commit(smem_addr(&acc_full[acc]));
      __syncwarp();
    }
    if (!ok && lane == 0) atomicOr(failed, 1u);
    __syncwarp();
    umma_drain(mma_done);
  } else if (warp < kUnpackWarp0) {
    // columns at a time: the small tiles' loops need the registers that 32 would take
    constexpr int kWide = kN == 256 || (!kForward && kN == 128) ? 32 : 16;
    const float scale = *p.w.global_scale * 128.0f;
    const auto find = [&](int i) {
      if (!adapters || warp != 2 || i >= ntiles) return;
      int tt, to;
      raster(first + i * step, p, tt, to);
      find_adapters<kForward, kN>(p, (int64_t)tt * kN, lane, info_of(i), reinterpret_cast<int*>(zs));
      if (lane == 0) mbar_arrive(&info_full[i % kInfos]);
    };
    bad[out_row] = bad[128 + out_row] = 0u;
    find(0);
    find(1);
    epilogue_sync();
    if (p.chained) pdl_wait_primary();  // z
    int extras = 0;          // the adapters' blocks so far
    uint32_t slot_turn = 0;  // parity of each stage's next `slot`
    // a wait that ran out ends the waiting, not the tiles: every warp reaches every barrier
    for (int i = 0; i < ntiles; ++i) {
      int tt, to;
      raster(first + i * step, p, tt, to);
      const uint32_t acc = (uint32_t)i & 1u;
      const int64_t o = (int64_t)to * kBM + out_row;
      const TileInfo& info = info_of(i);
      uint32_t spoiled = 0u;
      if (adapters && have) have = wait_info(i);
      if (adds) {
        for (int e = 0; have && e < info.listed; e += adapters_a_block(p.ad.rank))
          for (int r0 = 0; r0 < p.ad.rank && have; r0 += 32, ++extras) {
            int s = 0;
            const auto acquire = [&](int& stage) {
              s = stage = ((i + 1) * kbs + extras) % kStages;
              const uint32_t parity = (slot_turn >> s) & 1u;
              slot_turn ^= 1u << s;
              return mbar_wait_warp(&slot[s], parity);
            };
            have = adapter_block<kForward, kN>(p, info, e, r0, (int64_t)tt * kN, (int64_t)to * kBM, out_row,
                                               bad + acc * 128, tile_a, tile_b, acquire);
            if (have) {
              fence_proxy_async_smem();
              __syncwarp();
              if (lane == 0) mbar_arrive(&full[s]);
            }
          }
        epilogue_sync();
        spoiled = bad[acc * 128 + out_row];
        bad[acc * 128 + out_row] = 0u;  // its next use is two tiles on, behind the next tile's barrier
      }
      if (T::kStash && adapters && have) {
        // this rank's columns; eight at a time, whose factors are fetched at once
        const int own = kN / csize;
#pragma unroll 1
        for (int c = crank * own; c < (crank + 1) * own; c += 8) {
          const uint32_t loose = info.loose[c >> 5] >> (c & 31) & 0xFFu;
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = 0.0f;
          if (loose) add_loose<kForward, 8>(v, (int64_t)tt * kN + c, o, lane, p, loose, zs);
#pragma unroll
          for (int j = 0; j < 8; ++j) stash[(c + j) * kBM + out_row] = v[j];
        }
      }
      if (have) have = __all_sync(0xFFFFFFFFu, mbar_wait_acc(&acc_full[acc], (uint32_t)(i >> 1) & 1u));
      if (!have) continue;
      tc_fence_after_sync();
      find(i + 2);  // every role is done with tile i - 2, whose place it takes
      if (csize > 1) {
        bad[out_row] = spoiled;
        break;
      }
#pragma unroll 1
      for (int c = 0; c < kN; c += kWide) {
        const int64_t t0 = (int64_t)tt * kN + c;
        uint32_t q[kWide];
        if constexpr (kWide == 32)
          tmem_ld_32x32b_x32(tmem_d + acc * kN + lane_base + (uint32_t)c, q);
        else
          tmem_ld_32x32b_x16(tmem_d + acc * kN + lane_base + (uint32_t)c, q);
        tmem_ld_wait();
        if (c + kWide == kN) {
          tc_fence_before_sync();
          mbar_arrive(&acc_empty[acc]);
        }
        if (t0 >= p.tokens) continue;
        if (adapters) spoil<kWide>(q, spoiled, info.index + c);
        float v[kWide];
#pragma unroll
        for (int j = 0; j < kWide; ++j)
          v[j] = T::kStash && adapters ? fmaf(__uint_as_float(q[j]), scale, stash[(c + j) * kBM + out_row]) : __uint_as_float(q[j]) * scale;
        if (!T::kStash && adapters) add_loose<kForward, kWide>(v, t0, o, lane, p, info.loose[c >> 5] >> (c & 31), zs);
        store<kForward, kWide>(v, t0, o, lane, p, zs);
      }
    }
    if (!have && lane == 0) atomicOr(failed, 1u);
  } else {
    // ---- the weight's tile.  Thread: one row of 64 nibbles, K-major an output's, MN-major 64 outputs of a K
    const int tid = (int)threadIdx.x - kUnpackWarp0 * 32;
    const int who = tid / kGroupThreads;              // takes blocks who, who + kUnpackGroups, ... of the CTA's
    const int line = tid % kGroupThreads;             // 128-byte line of the tile
    const int row = kForward ? line : line & 63;
    const int64_t m = p.w.m, n = p.w.n;
    const bool wide = (n & 63) == 0 && (reinterpret_cast<uintptr_t>(p.w.packed) & 31) == 0 &&
                      (reinterpret_cast<uintptr_t>(p.w.codes) & 3) == 0;
    // the next block to load: where its 32 bytes and 4 codes are, and K blocks left in its tile
    int li = -1, left = 0;
    int64_t f = 0, k0 = 0;
    // Blocks past W's edges are read inside it: outputs past the end are not stored, and past the end of K the tokens'
    // tile is zeros, which any weight, a finite number, leaves zeros.
    const uint8_t *wp = nullptr, *cp = nullptr, *last_w = nullptr, *last_c = nullptr;
    const int64_t w_step = kUnpackGroups * (kForward ? (int64_t)kBK / 2 : kBK * (n >> 1));
    const int64_t c_step = kUnpackGroups * (kForward ? (int64_t)kBK / 16 : kBK * (n >> 4));
    const int total = ntiles * kbs;
    auto advance = [&](int blocks) {
      left -= blocks;
      if (left > 0) {
        if (kForward) k0 += kUnpackGroups * kBK; else f += kUnpackGroups * kBK;
        wp += w_step, cp += c_step;
        if (!kForward && f >= m) wp = last_w, cp = last_c;
        return;
      }
      while (left <= 0 && ++li < ntiles) left += kbs;
      if (li >= ntiles) return;
      int tt, to;
      raster(first + li * step, p, tt, to);
      const int64_t kb = kb1 - left;
      f = kForward ? (int64_t)to * kBM + row : kb * kBK + row;
      k0 = kForward ? kb * kBK : (int64_t)to * kBM + (line >> 6) * 64;
      const int64_t fin = min(f, m - 1), kin = min(k0, (n - 1) & ~(int64_t)63);
      wp = p.w.packed + fin * (n >> 1) + (kin >> 1);
      cp = p.w.codes + fin * (n >> 4) + (kin >> 4);
      last_w = p.w.packed + (m - 1) * (n >> 1) + (kin >> 1), last_c = p.w.codes + (m - 1) * (n >> 4) + (kin >> 4);
    };
    uint32_t ring[kAhead][8], codes[kAhead][4] = {};  // codes: one word, or one byte a word
    auto load = [&](uint32_t (&q)[8], uint32_t (&c)[4]) {
      if (wide) {
        ld_32_ahead(wp, q);
        ld_4_ahead(true, cp, c[0]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = q[2 * i] = q[2 * i + 1] = 0u;
          ld_8_ahead(k0 + 16 * i < n, wp + 8 * i, q[2 * i], q[2 * i + 1]);
          ld_1_ahead(k0 + 16 * i < n, cp + i, c[i]);
        }
      }
      advance(kUnpackGroups);
    };
    advance(who);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (who + u * kUnpackGroups < total) load(ring[u], codes[u]);
    int tile_end = adds ? kbs : INT32_MAX;  // the first block behind the present tile
    uint32_t s = (uint32_t)who % kStages, parity = 1;
    bool go = true;
    for (int base = who; base < total && go; base += kAhead * kUnpackGroups) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int next = base + u * kUnpackGroups;
        if (next >= total || !go) break;
        if (next >= tile_end) {
          const int tile = next / kbs, before = tile - 1;
          tile_end = (tile + 1) * kbs;
          go = mbar_wait_warp(&go_full[before % kGo], (uint32_t)(before / kGo) & 1u);
          if (!go) break;
          const uint32_t pos = (uint32_t)(place[before % kGo] + next - tile * kbs);
          s = pos % kStages;
          parity = ((pos / kStages) & 1u) ^ 1u;
        }
        if (!mbar_wait_warp(&empty[s], parity)) {
          go = false;
          break;
        }
        uint8_t* dst = tile_a + s * kTileABytes + line * 128;
        const uint32_t code = wide ? codes[u][0] : codes[u][0] | codes[u][1] << 8 | codes[u][2] << 16 | codes[u][3] << 24;
        const uint32_t ca = unpack_codes(code & 0xFFFFu), cb = unpack_codes(code >> 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = i < 4 ? ca : cb;
          uint32_t r[4];
          unpack8(ring[u][i], __byte_perm(c, c, (i & 2) ? 0x3232 : 0x1010), r);
          *reinterpret_cast<uint4*>(dst + ((i ^ (row & 7)) << 4)) = make_uint4(r[0], r[1], r[2], r[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[s]);
        s += kUnpackGroups;
        if (s >= kStages) {
          s -= kStages;
          parity ^= 1u;
        }
        if (base + (u + kAhead) * kUnpackGroups < total) load(ring[u], codes[u]);
      }
    }
    if (!go && lane == 0) atomicOr(failed, 1u);
  }

  if (csize > 1) {
    // The ranks' partials: rank d owns columns [d own, (d + 1) own); the ring is free once every rank's MMAs
    // have completed, and its memory takes [source][column][output].  All warps but the first two take part, four to a
    // quarter of tensor memory, eight columns in turn (the epilogue's four alone took 20 us for 256 columns).
    const int own = kN / csize, share = (warp - 2) >> 2;
    float* inbox = reinterpret_cast<float*>(smem);
    float* turn = reinterpret_cast<float*>(smem + kN * kBM * 4) + (warp - 2) * (kTurnBytes / 16);
    static_assert(kN * kBM * 4 + (kThreads / 32 - 2) * (kTurnBytes / 4) <= kStages * T::kStageBytes, "the ring's room");
    tc_fence_before_sync();
    __syncthreads();
    const bool complete = *failed == 0u;
    cluster_sync();
    tc_fence_after_sync();
    int tt, to;
    raster(first, p, tt, to);
    if (warp >= 2) {
      for (int d = 0; d < csize; ++d) {
        if (d == crank) continue;
        const uint32_t base = mapa(smem_addr(inbox + (crank * own) * kBM + out_row), (uint32_t)d);
        for (int c = 8 * share; c < own; c += 32) {
          uint32_t q[8];
          tmem_ld_32x32b_x8(tmem_d + lane_base + (uint32_t)(d * own + c), q);
          tmem_ld_wait();
          if (adds) spoil<8>(q, bad[out_row], info_of(0).index + d * own + c);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(base + (uint32_t)((c + j) * kBM * 4)),
                         "r"(complete ? q[j] : 0x7FC00000u)
                         : "memory");
        }
      }
    }
    cluster_sync();
    if (warp >= 2) {
      const float scale = *p.w.global_scale * 128.0f;
      if (p.chained) pdl_wait_primary();  // z
      const int64_t o = (int64_t)to * kBM + out_row;
      for (int c = 8 * share; c < own; c += 32) {
        const int64_t t0 = (int64_t)tt * kN + crank * own + c;
        const int col = crank * own + c;
        uint32_t q[8];
        tmem_ld_32x32b_x8(tmem_d + lane_base + (uint32_t)col, q);
        tmem_ld_wait();
        if (t0 >= p.tokens) continue;
        if (adds) spoil<8>(q, bad[out_row], info_of(0).index + col);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.0f;
        for (int d = 0; d < csize; ++d) {
          const float* src = inbox + (d * own + c) * kBM + out_row;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            v[j] += d != crank ? src[j * kBM] : complete ? __uint_as_float(q[j]) : __int_as_float(0x7FC00000);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[j] = T::kStash && adapters && complete ? fmaf(v[j], scale, stash[(col + j) * kBM + out_row]) : v[j] * scale;
        if (!T::kStash && adapters && complete)
          add_loose<kForward, 8>(v, t0, o, lane, p, info_of(0).loose[col >> 5] >> (col & 31), turn);
        store<kForward, 8>(v, t0, o, lane, p, turn);
      }
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_d, T::kTmemCols);
  }
  if (*failed) {
    if (threadIdx.x == 0) atomicOr(&g_project_flags, kErrMbarTimeout);
    if (csize == 1 && warp >= 2 && warp < kUnpackWarp0) {
      for (int i = 0; i < ntiles; ++i) {
        int tt, to;
        raster(first + i * step, p, tt, to);
        const int64_t o = (int64_t)to * kBM + out_row;
        for (int64_t t = (int64_t)tt * kN; t < min(p.tokens, (int64_t)(tt + 1) * kN); ++t)
          if (o < (kForward ? p.w.m : p.w.n)) p.out[t * p.ld_out + o] = __ushort_as_bfloat16(0x7FC0);
      }
    }
  }
}

template <bool kForward, int kN>
cudaError_t launch(const void* v, int64_t ld_v, ProjectArgs p, int csize, int sms, cudaStream_t stream) {
  using T = Tile<kN>;
  EncodeTiledFn encode = nullptr;
  cudaError_t err = encode_tiled_fn(&encode);
  if (err != cudaSuccess) return err;
  CUtensorMap map;
  const int64_t depth = kForward ? p.w.n : p.w.m;
  const cuuint64_t dims[2] = {(cuuint64_t)depth, (cuuint64_t)p.tokens};
  const cuuint64_t strides[1] = {(cuuint64_t)ld_v * 2};
  const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)kN};
  const cuuint32_t estr[2] = {1, 1};
  if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(v), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  auto kernel = project_kernel<kForward, kN>;
  err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)T::kSmemBytes);
  if (err != cudaSuccess) return err;
  p.csize = csize;
  p.tiles_t = (int32_t)((p.tokens + kN - 1) / kN);
  const int64_t tiles = (int64_t)p.tiles_t * p.tiles_o;
  if (tiles * csize > INT32_MAX) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(csize > 1 ? tiles * csize : std::min<int64_t>(tiles, sms)), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = T::kSmemBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.chained ? 2 : 1;
  err = cudaLaunchKernelEx(&cfg, kernel, map, p);
  return err != cudaSuccess ? err : cudaGetLastError();
}

}  // namespace

cudaError_t launch_project(bool forward, const void* v, int64_t tokens, int64_t ld_v, const Nvfp4Weight& w, const Adapters& ad,
                           const float* z, const uint32_t* z_split, void* out, int64_t ld_out, cudaStream_t stream) {
  if (forward && tokens <= kDecodeTokens) return launch_project_decode(v, tokens, ld_v, w, ad, z, out, ld_out, stream);
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int sms = info.sm_count;
  ProjectArgs p = {};
  p.w = w, p.ad = ad, p.z = z, p.z_split = z_split, p.out = static_cast<__nv_bfloat16*>(out), p.tokens = tokens, p.ld_out = ld_out;
  p.kb_total = (int32_t)(((forward ? w.n : w.m) + kBK - 1) / kBK);
  p.tiles_o = (int32_t)(((forward ? w.m : w.n) + kBM - 1) / kBM);
  p.chained = ad.count > 0;
  // Tokens a tile and CTAs a tile by an estimate of the time: a wave's start and end, and its K blocks one after
  // another, as fitted to measurements (us, 64 tokens on 4096 x 4096 with 1, 2, 4 CTAs a tile: 22.1, 15.6, 12.0; 256:
  // 64 tokens a tile 22.6, 128 by two CTAs 18.2; 512 on 4096 x 14336: 83.0 with 128 a tile, 55.3 with 256 by two CTAs).
  // One CTA a tile is persistent and starts once.  Clusters of eight leave a sixth of the SMs out.  The adapters' K blocks are
  // not in it (which a tile has is known on the GPU only): 32 adapters in any order add 8 to the 16 of a 1024-row weight's dx.
  constexpr double kStart[4] = {9.0, 9.0, 11.0, 14.0}, kBlock[4] = {0.20, 0.21, 0.27, 0.34};  // 32, 64, 128, 256 tokens
  int best_n = 32, best_c = 1;
  double best = 1e300;
  for (int i = 0, kn = 32; kn <= 256; ++i, kn *= 2) {
    if (kn > 32 && kn / 2 >= tokens) break;
    const int64_t tiles = (tokens + kn - 1) / kn * p.tiles_o;
    for (int c = 1; c <= 8 && kn / c >= 8 && c <= p.kb_total; c *= 2) {
      const int64_t room = c == 8 ? sms * 5 / 6 : sms, waves = (tiles * c + room - 1) / room;
      const double blocks = (double)((p.kb_total + c - 1) / c);
      const double cost = (c == 1 ? kStart[i] : waves * kStart[i]) + waves * blocks * kBlock[i];
      if (cost < best) best = cost, best_n = kn, best_c = c;
    }
  }
  if (forward) {
    switch (best_n) {
      case 32: return launch<true, 32>(v, ld_v, p, best_c, sms, stream);
      case 64: return launch<true, 64>(v, ld_v, p, best_c, sms, stream);
      case 128: return launch<true, 128>(v, ld_v, p, best_c, sms, stream);
      default: return launch<true, 256>(v, ld_v, p, best_c, sms, stream);
    }
  }
  switch (best_n) {
    case 32: return launch<false, 32>(v, ld_v, p, best_c, sms, stream);
    case 64: return launch<false, 64>(v, ld_v, p, best_c, sms, stream);
    case 128: return launch<false, 128>(v, ld_v, p, best_c, sms, stream);
    default: return launch<false, 256>(v, ld_v, p, best_c, sms, stream);
  }
}

cudaError_t read_project_device_error(uint32_t* flags) {
  uint32_t v = 0;
  cudaError_t err = cudaMemcpyFromSymbol(&v, g_project_flags, sizeof v);
  if (err != cudaSuccess) return err;
  *flags = v;
  if (v) {
    const uint32_t zero = 0;
    err = cudaMemcpyToSymbol(g_project_flags, &zero, sizeof zero);
  }
  return err;
}

}  // namespace hscale
