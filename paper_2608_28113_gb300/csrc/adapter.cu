// adapter.cu -- the low-rank adapters' own products beside a projection (project.cu):
//   z  = alpha_a A_a x_t       dz = alpha_a B_a^T dy_t        for every token t of an adapter a
//   dA = sum_t dz_t x_t^T      dB = sum_t dy_t z_t^T          over the tokens of each adapter
// z and dz are fp32 [tokens, rank]; rows of tokens without an adapter are left as they are.
//
// All four multiply long rows of activations by something narrow (`rank` wide), grouped by the tokens' adapters: tiles
// too thin for tcgen05 (N = rank, or K = the tokens of one adapter).  They run on warp-level MMAs (m16n8k16,
// bf16 operands, fp32 sums); a warp's operands come through a ring of its own in shared memory by asynchronous copies, so
// warps wait for no one but themselves until their sums meet.  The order of a contracted axis is free, so a lane takes
// 16 consecutive bytes of a row and calls its 8 elements whatever slots of K the fragment layout gives it, on both
// operands alike.
//
// The bytes (each row once) would take a tenth of the time that they do: few ranks are bound by the latency of the copies
// and of each launch's start and end, many ranks by L2, from where a job's factors and the rows of each
// pass come again, and by the MMAs.  Under a profiler, one GB300: z and dz of 8192 tokens, 4096 x 4096, rank 16: 35 us, dA
// and dB 59; of 4096 tokens, 4096 x 14336, rank 64: 137 and 191.
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
  int vec;     // checkpoint: codes that may be copied at once (16, 8 or 1)
  bool words;  // checkpoint: the scales of 4 blocks may be copied at once

  static constexpr int kElement = kFormat < 0 ? 2 : 1;  // bytes
  __device__ __forceinline__ const uint8_t* row(int64_t t) const {
    return kFormat < 0 ? reinterpret_cast<const uint8_t*>(x + t * ld) : ckpt.codes + t * ckpt.ld_codes;
  }
  __device__ __forceinline__ const uint8_t* scale_row(int64_t t) const { return ckpt.scales + t * ckpt.ld_scales; }
  // elements [k, k + 8) of a row: how many bytes of them there are (0 where `on` is false)
  __device__ __forceinline__ int bytes(int64_t k, bool on) const {
    return on && k < cols ? (int)min((int64_t)8, cols - k) * kElement : 0;
  }
  // those elements to dst (16 bytes of bf16, 8 codes), zeros past the end; k % 8 == 0 and inside the row
  __device__ __forceinline__ void copy(uint8_t* dst, const uint8_t* row, int64_t k, int bytes) const {
    if constexpr (kFormat < 0) {
      copy_16(dst, row + k * 2, bytes);
    } else if (vec >= 8) {
      copy_8(dst, row + k, bytes);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) dst[j] = j < bytes ? __ldg(row + k + j) : (uint8_t)0;
    }
  }
  // the scale bytes of the two blocks from element k on (k % 64 == 0), in the word at dst as scale_of finds them
  __device__ __forceinline__ void copy_scales(uint8_t* dst, const uint8_t* scale_row, int64_t k, bool on) const {
    const int64_t block = k / kCkptBlock;
    if (words) {
      copy_4(dst, scale_row + (block & ~(int64_t)3), on ? 4 : 0);
    } else {
      uint32_t two = 0u;
      if (on) two = (uint32_t)__ldg(scale_row + block);
      if (on && k + kCkptBlock < cols) two |= (uint32_t)__ldg(scale_row + block + 1) << 8;
      *reinterpret_cast<uint32_t*>(dst) = two << (8 * (block & 3));
    }
  }
  static __device__ __forceinline__ uint32_t scale_of(uint32_t word, int64_t k) {
    return ckpt_scale((word >> (8 * ((uint32_t)(k / kCkptBlock) & 3u))) & 0xFFu);
  }
  // 8 codes as 4 x bf16x2; a checkpoint's values are exact in bf16
  static __device__ __forceinline__ uint4 values(uint2 v, uint32_t scale) {
    return make_uint4(ckpt_values<kFormat, 0>(v.x, scale), ckpt_values<kFormat, 1>(v.x, scale),
                      ckpt_values<kFormat, 0>(v.y, scale), ckpt_values<kFormat, 1>(v.y, scale));
  }
};

// ---------------------------------------------------------------- z and dz
// A tile is 256 tokens.  Its jobs: 32 tokens (or what is left) of one adapter, wherever in the tile they stand, in order of
// the adapters' first tokens; so a request's tokens and tokens in any order cost the same, each row is read once, and
// an adapter's factors once per job.  As an MMA: M = ranks, N = tokens (8 a group, as many groups as the job has),
// K = the contracted axis in blocks of 64.  CTAs `turn` of `turns` take a tile's jobs in turn; the warps, and the CTAs of a
// cluster of csize, split K, kDepth blocks in flight each, from different places on (all of them reading the same factors
// at once would queue at one slice of L2).  Partials are summed in order.
// kDown: A_a [rank, cols] (contracted axis contiguous); else B_a [cols, rank], whose 8 x 8 blocks are
// transposed in registers.  kNT: ranks / 8 of a pass.
constexpr int kTile = 256, kJob = 32;
constexpr int kDepth = 2;
struct Split {
  int csize, crank, turns, turn;
};
struct JobShared {
  int adapter;
  uint16_t token[kJob];  // in the tile
  const uint8_t* row[kJob];
  const uint8_t* scale_row[kJob];
};
template <int kFormat, int kNT>
constexpr int block_bytes() {  // of a warp's ring: the tokens' rows of 128 bytes (a checkpoint's 64 and a scale word), the factors
  return kJob * (kFormat < 0 ? 128 : 68) + 1024 * kNT;
}
template <int kNT>
constexpr int part_bytes() {
  return kWarps * kJob * 8 * kNT * 4;
}

// What the CTA's threads, one a token of the tile, tell each other of the tokens' adapters.
struct TileScratch {
  alignas(16) int2 seen[kTile];  // the adapters of warp w's tokens, in the order of their first ones, from 32 w on; their tokens
  int first_job[kTile];     // of those whose first token in the tile is this warp's
  int adapters[kWarps], jobs[kWarps];
};
static_assert(kTile == kThreads && sizeof(TileScratch) <= part_bytes<1>(), "a token a thread");

// (job, place in it) of this thread's token, whose adapter is id; (-1, 0) without one.  Jobs are numbered in the order of the
// adapters' first tokens.  Every thread of the CTA calls.  (Each warp going through the adapters for itself, with
// eight ballots each, took dx of 2048 tokens on 32 adapters 8 us longer.)
__device__ __forceinline__ int2 place_token(int id, int words, int warp, int lane, TileScratch& sh, int& jobs) {
  const uint32_t before = (1u << lane) - 1u;
  const uint32_t alike = __match_any_sync(0xFFFFFFFFu, id);
  const int leader = __ffs(alike) - 1;
  const bool leads = id >= 0 && leader == lane;
  const uint32_t leaders = __ballot_sync(0xFFFFFFFFu, leads);
  const int entry = 32 * warp + __popc(leaders & before);
  // behind a word's adapters, entries of none
  sh.seen[leads ? entry : 32 * warp + __popc(leaders) + __popc(~leaders & before)] = leads ? make_int2(id, __popc(alike)) : make_int2(-2, 0);
  if (lane == 0) sh.adapters[warp] = __popc(leaders);
  __syncthreads();
  int ahead = 0, total = 0, first = -1;  // the adapter's tokens in earlier warps, in all, and its first entry
  for (int w = 0; w < words; ++w) {
    const int end = 32 * w + sh.adapters[w];
    int hit = -1, held = 0;
    for (int k = 32 * w; k < end; k += 4) {
      const int4 e0 = *reinterpret_cast<const int4*>(&sh.seen[k]), e1 = *reinterpret_cast<const int4*>(&sh.seen[k + 2]);
      if (e0.x == id) hit = k, held = e0.y;
      if (e0.z == id) hit = k + 1, held = e0.w;
      if (e1.x == id) hit = k + 2, held = e1.y;
      if (e1.z == id) hit = k + 3, held = e1.w;
    }
    if (first < 0) first = hit;
    if (w < warp) ahead += held;
    total += held;
  }
  const bool opens = leads && first == entry;
  const int own = opens ? (total + kJob - 1) / kJob : 0;
  int sum = own;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int v = __shfl_up_sync(0xFFFFFFFFu, sum, d);
    if (lane >= d) sum += v;
  }
  if (lane == 31) sh.jobs[warp] = sum;
  __syncthreads();
  int base = 0;
  jobs = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w >= words) break;
    if (w == warp) base = jobs;
    jobs += sh.jobs[w];
  }
  if (opens) sh.first_job[entry] = base + sum - own;
  __syncthreads();
  if (id < 0) return make_int2(-1, 0);
  const int at = ahead + __popc(alike & before);
  return make_int2(sh.first_job[first] + at / kJob, at % kJob);
}

template <int kFormat, bool kDown, int kNT>
__device__ __forceinline__ void shrink_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, float* z,
                                            uint32_t* z_split, float unit, int64_t tile, const Split& sp, JobShared& job,
                                            uint8_t* smem) {
  constexpr int kMR = (kNT + 1) / 2, kPass = 8 * kNT;
  constexpr int kX = kJob * (kFormat < 0 ? 128 : 68), kBlock = block_bytes<kFormat, kNT>();
  constexpr int kOdd = kFormat < 0 ? 4 : 1;  // odd rows of A: pieces elsewhere than the even rows' of the same reads
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int64_t t0 = tile * kTile, cols = rows.cols;
  const int rank = ad.rank;
  uint8_t* ring = smem + warp * kDepth * kBlock;
  float* part = reinterpret_cast<float*>(smem);  // the warps' partials take the rings' place
  // this warp's blocks of 64: first, first + ways, ...: `count` of them, taken from a place of its own on
  const int ways = kWarps * sp.csize, blocks = (int)((cols + 63) / 64), shift = (int)(tile * sp.turns + sp.turn);
  const int first = (sp.crank * kWarps + warp + shift) % ways;
  const int count = first < blocks ? (blocks - first + ways - 1) / ways : 0;
  const int lead = count > 0 ? (shift / ways) % count : 0;
  const auto block_at = [&](int i) {
    const int at = i + lead;
    return (int64_t)(first + (at < count ? at : at - count) * ways) * 64;
  };
  // A thread's token: its job, and its place in it.
  const int words = (int)min((int64_t)kWarps, (tokens - t0 + 31) / 32);  // of 32 tokens
  const int64_t mine = t0 + threadIdx.x;
  const int id = mine < tokens ? adapter_of(ad, mine) : -1;
  int jobs;
  const int2 slot = place_token(id, words, warp, lane, reinterpret_cast<TileScratch&>(*part), jobs);
  for (int at = sp.turn; at < jobs; at += sp.turns) {
    if (slot.x == at) {
      job.token[slot.y] = (uint16_t)threadIdx.x;
      job.row[slot.y] = rows.row(mine), job.scale_row[slot.y] = rows.scale_row(mine);
      if (slot.y == 0) job.adapter = id;
    }
    const int have = __syncthreads_count(slot.x == at);
    if ((int)threadIdx.x >= have && threadIdx.x < kJob)  // places past the job's tokens copy nothing
      job.row[threadIdx.x] = rows.row(t0), job.scale_row[threadIdx.x] = rows.scale_row(t0);
    __syncthreads();
    const int a = job.adapter;
    const int groups = (have + 7) >> 3;
    for (int r0 = 0; r0 < rank; r0 += kPass) {
      float acc[kMR][4][4];
#pragma unroll
      for (int i = 0; i < kMR; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][c][e] = 0.0f;
      const __nv_bfloat16* factors = kDown ? ad.a + ((int64_t)a * rank + r0) * cols : ad.b + (int64_t)a * cols * rank + r0;
      // One block's copies, 16 bytes a lane, whole rows at a time: a row's 16-byte pieces stand in its 128 (64) bytes as the
      // reads below have them free of bank conflicts.
      const auto fetch = [&](int i) {
        if (i < count) {
          const int64_t kb = block_at(i);
          uint8_t* dst = ring + (i & (kDepth - 1)) * kBlock;
          if constexpr (kFormat < 0) {
            const int piece = lane & 7;
            const int64_t k = kb + 8 * piece, kin = min(k, cols - 1) & ~(int64_t)7;
            const int bytes = rows.bytes(k, true);
#pragma unroll
            for (int n = 0; n < 8; ++n) {
              if (n >= 2 * groups) continue;
              const int p = 4 * n + (lane >> 3);
              copy_16(dst + p * 128 + ((piece ^ ((p & 1) << 2)) << 4), job.row[p] + kin * 2, p < have ? bytes : 0);
            }
          } else {
            const int piece = lane & 3;
            const int64_t k = kb + 16 * piece, kin = min(k, cols - 1) & ~(int64_t)15;
            const int bytes = k < cols ? 16 : 0;  // cols % 16 == 0
#pragma unroll
            for (int n = 0; n < 4; ++n) {
              if (n >= groups) continue;
              const int p = 8 * n + (lane >> 2);
              uint8_t* slot = dst + p * 64 + (piece << 4);
              if (rows.vec == 16) {
                copy_16(slot, job.row[p] + kin, p < have ? bytes : 0);
              } else {
                rows.copy(slot, job.row[p], kin, p < have ? bytes / 2 : 0);
                rows.copy(slot + 8, job.row[p], kin + 8, p < have ? bytes / 2 : 0);
              }
            }
            // the two blocks of 32 of a token: one word
            rows.copy_scales(dst + kJob * 64 + 4 * lane, job.scale_row[lane], kb, lane < have);
          }
          if constexpr (kDown) {
            const int piece = lane & 7;
            const int64_t k = kb + 8 * piece;
#pragma unroll
            for (int n = 0; n < 2 * kNT; ++n) {  // cols % 16 == 0
              const int r = 4 * n + (lane >> 3);
              const bool on = r0 + r < rank && k < cols;
              copy_16_l1(dst + kX + r * 128 + ((piece ^ ((r & 1) * kOdd)) << 4), factors + (on ? (int64_t)r * cols + k : 0), on ? 16 : 0);
            }
          } else {
#pragma unroll
            for (int n = 0; n < 2 * kNT; ++n) {
              const int at = 32 * n + lane, kk = at / kNT, c = at % kNT, v = (kk >> 3) & 3;
              const bool on = kb + kk < cols && r0 + 8 * c < rank;
              const int swizzle = kNT == 4 ? v : kNT == 2 ? (v & 1) | (v & 2) << 1 : v << 1;
              copy_16_l1(dst + kX + ((at ^ swizzle) << 4), factors + (on ? (kb + kk) * rank + 8 * c : 0), on ? 16 : 0);
            }
          }
        }
        copies_end();
      };
#pragma unroll
      for (int i = 0; i < kDepth - 1; ++i) fetch(i);
      for (int it = 0; it < count; ++it) {
        __syncwarp();  // the stage's last reads
        fetch(it + kDepth - 1);
        copies_wait<kDepth - 1>();
        __syncwarp();  // every lane's copies
        const uint8_t* src = ring + (it & (kDepth - 1)) * kBlock;
        uint32_t scale[4];
        if constexpr (kFormat >= 0) {
          const int64_t kb = block_at(it);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const uint32_t word = *reinterpret_cast<const uint32_t*>(src + kJob * 64 + 4 * (8 * c + g));
            scale[c] = Rows<kFormat>::scale_of(word, kb + 16 * q);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint4 w[2 * kMR];
#pragma unroll
          for (int j = 0; j < 2 * kMR; ++j) {
            w[j] = make_uint4(0u, 0u, 0u, 0u);
            if (j >= kNT) continue;
            if constexpr (kDown) {
              // the tokens' groups of 8: bf16 from 32 h + 8 q on, a checkpoint's from 16 q + 8 h on
              const int piece = kFormat < 0 ? 4 * h + q : 2 * q + h;
              w[j] = *reinterpret_cast<const uint4*>(src + kX + (8 * j + g) * 128 + ((piece ^ ((g & 1) * kOdd)) << 4));
            } else {
              // register u: slots 2 q', 2 q' + 1 are elements 8 q' + 2 u, + 1 of the half
              const int u = lane >> 3, r = lane & 7, kk = 32 * h + (r >> 1) * 8 + 2 * u + (r & 1), v = (kk >> 3) & 3;
              const int swizzle = kNT == 4 ? v : kNT == 2 ? (v & 1) | (v & 2) << 1 : v << 1;
              w[j] = load_transposed_x4(smem_addr(src + kX + (((kk * kNT + j) ^ swizzle) << 4)));
            }
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (c >= groups) continue;
            const int p = 8 * c + g;
            uint4 x;
            if constexpr (kFormat < 0)
              x = *reinterpret_cast<const uint4*>(src + p * 128 + (((4 * h + q) ^ ((p & 1) << 2)) << 4));
            else
              x = Rows<kFormat>::values(*reinterpret_cast<const uint2*>(src + p * 64 + 16 * q + 8 * h), scale[c]);
#pragma unroll
            for (int i = 0; i < kMR; ++i) {
              const uint32_t a0[4] = {w[2 * i].x, w[2 * i + 1].x, w[2 * i].y, w[2 * i + 1].y};
              const uint32_t a1[4] = {w[2 * i].z, w[2 * i + 1].z, w[2 * i].w, w[2 * i + 1].w};
              mma_bf16(acc[i][c], a0, x.x, x.y);
              mma_bf16(acc[i][c], a1, x.z, x.w);
            }
          }
        }
      }
      copies_wait<0>();
      __syncthreads();
      // ranks 16 i + g (+ 8), tokens 8 c + 2 q (+ 1): the warps' partials [warp][token][rank of the pass]
      float* out = part + warp * kJob * kPass;
#pragma unroll
      for (int i = 0; i < kMR; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c < groups && 16 * i + 8 * (e >> 1) < kPass)
              out[(8 * c + 2 * q + (e & 1)) * kPass + 16 * i + 8 * (e >> 1) + g] = acc[i][c][e];
      __syncthreads();
      // the warps' partials in order, into the first ones'; then the ranks' in order
      constexpr int kAll = kJob * kPass;
      for (int i = threadIdx.x; i < kAll; i += kThreads) {
        float s = part[i];
#pragma unroll
        for (int v = 1; v < kWarps; ++v) s += part[v * kAll + i];
        part[i] = s;
      }
      if (sp.csize > 1) cluster_sync(); else __syncthreads();
      const int share = kAll / sp.csize;
      for (int i = sp.crank * share + threadIdx.x; i < (sp.crank + 1) * share; i += kThreads) {
        const int p = i / kPass, r = r0 + i % kPass;
        if (p >= have || r >= rank) continue;
        float s = sp.csize > 1 ? ld_cluster(part + i, 0) : part[i];
        for (int d = 1; d < sp.csize; ++d) s += ld_cluster(part + i, (uint32_t)d);
        s *= ad.alpha[a];
        const int64_t at = (t0 + job.token[p]) * rank + r;
        z[at] = s;
        if (z_split != nullptr) {
          const float v = s * unit;
          const uint32_t hi = pack_bf16(v, 0.0f);
          z_split[at] = hi | pack_bf16(0.0f, v - bf16_lo(hi));
        }
      }
      if (sp.csize > 1) cluster_sync(); else __syncthreads();  // the partials, and the others' shared memory, have been read
    }
  }
}

// blockIdx.y: the turns of z (x's rows against A), then those of dz (dy's rows against B), whichever are wanted.
struct ShrinkArgs {
  Adapters ad;
  int64_t tokens;
  const float* global_scale;
  float *z, *dz;
  uint32_t *z_split, *dz_split;
  int csize, turns_z, turns_dz;
};
constexpr int dz_ranks(int kNT) { return std::min(kNT, 2); }  // so that two CTAs fit an SM
template <int kFormat, int kNT>
constexpr int shrink_smem_bytes() {
  return std::max({kWarps * kDepth * block_bytes<kFormat, kNT>(), kFormat < 0 ? 0 : kWarps * kDepth * block_bytes<-1, dz_ranks(kNT)>(),
                   part_bytes<kNT>()});
}
template <int kFormat, int kNT>
__global__ void __launch_bounds__(kThreads, 2) shrink_kernel(Rows<kFormat> x, Rows<-1> dy, ShrinkArgs p) {
  extern __shared__ __align__(16) uint8_t shrink_smem[];
  __shared__ JobShared job;
  pdl_launch_dependents();  // the projection's own product needs no z
  const bool is_z = (int)blockIdx.y < p.turns_z;
  const Split sp = {p.csize, p.csize > 1 ? (int)cluster_rank() : 0, is_z ? p.turns_z : p.turns_dz,
                    (int)blockIdx.y - (is_z ? 0 : p.turns_z)};
  const int64_t tile = blockIdx.x / p.csize;
  const float unit = 1.0f / (kWeightUnit * *p.global_scale);
  if (is_z)
    shrink_tile<kFormat, true, kNT>(x, p.tokens, p.ad, p.z, p.z_split, unit, tile, sp, job, shrink_smem);
  else if constexpr (kFormat >= 0)  // the forward pass has no dz
    shrink_tile<-1, false, dz_ranks(kNT)>(dy, p.tokens, p.ad, p.dz, p.dz_split, unit, tile, sp, job, shrink_smem);
}

// Adapters that tokens may be on: the work is dealt out for these.
int64_t used_adapters(const Adapters& ad) { return ad.of_token == nullptr ? std::min(ad.count, 1) : ad.count; }

template <int kFormat, int kNT>
cudaError_t launch_shrink_of(const Rows<kFormat>& x, const Rows<-1>& dy, ShrinkArgs p, int jobs, int sms, cudaStream_t stream) {
  auto kernel = shrink_kernel<kFormat, kNT>;
  constexpr int kSmem = shrink_smem_bytes<kFormat, kNT>();
  constexpr int kCtas = kSmem <= 113 * 1024 ? 2 : 1;  // an SM holds
  cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmem);
  if (err != cudaSuccess) return err;
  // first a CTA for each job, z's and dz's by the length of their sums, then the contracted axis split (down to one block a
  // warp), while the SMs hold all
  const int64_t tiles = (p.tokens + kTile - 1) / kTile, cols = std::max(x.cols, dy.cols), room = (int64_t)kCtas * sms;
  const int64_t slots = std::max<int64_t>(1, room / tiles);
  p.turns_z = p.turns_dz = 0;
  if (p.z != nullptr && p.dz != nullptr) {
    p.turns_z = (int)std::max<int64_t>(1, std::min<int64_t>(jobs, slots * x.cols / (x.cols + dy.cols)));
    p.turns_dz = (int)std::max<int64_t>(1, std::min<int64_t>(jobs, slots - p.turns_z));
  } else {
    (p.z != nullptr ? p.turns_z : p.turns_dz) = (int)std::min<int64_t>(jobs, slots);
  }
  const int turns = p.turns_z + p.turns_dz;
  p.csize = 1;
  while (p.csize < 8 && tiles * turns * p.csize * 2 <= room && (int64_t)p.csize * kWarps * 64 < cols) p.csize *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.csize), (unsigned)turns, 1);
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

template <int kFormat>
cudaError_t launch_shrink(const Rows<kFormat>& x, const Rows<-1>& dy, const ShrinkArgs& p, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int sms = info.sm_count, rank = p.ad.rank;
  // jobs that a tile may have: its adapters are not known here
  const int64_t tok = std::min<int64_t>(p.tokens, kTile);
  const int jobs = (int)std::min<int64_t>(tok, (tok + kJob - 1) / kJob + std::min<int64_t>(used_adapters(p.ad), tok) - 1);
  if (rank <= 8) return launch_shrink_of<kFormat, 1>(x, dy, p, jobs, sms, stream);
  if (rank <= 16) return launch_shrink_of<kFormat, 2>(x, dy, p, jobs, sms, stream);
  // 32 ranks a pass of bf16 rows leave room for one CTA an SM, and gain all the same (4096 tokens x 14336, rank 64: 167 us
  // at 16 ranks a pass and two CTAs, 150); z of a checkpoint takes 32, two CTAs fit (z, dz, dA and dB of 4096 x (4096 x
  // 14336), rank 64: 311 us at 16 ranks, 258)
  return launch_shrink_of<kFormat, 4>(x, dy, p, jobs, sms, stream);
}

// ---------------------------------------------------------------- dA and dB
// A CTA takes 256 columns of one adapter's gradient and the adapter's tokens, in chunks of 128 that the CTAs of a
// cluster of csize take in turn; 64 columns a warp, kSub sets of four warps that take a chunk's units of 16 tokens in
// turn.  As an MMA: M = ranks (z or dz transposed, as a pair hi + lo of bf16 numbers: 2^-17 of a value is lost),
// N = columns, K = tokens.
//   * The rows: a lane copies 8 columns of four tokens of a unit into its own ring, kUnits units ahead, and pairs
//     the tokens' halves up into the fragments of 8 column tiles.
//   * z and a checkpoint's scales are the same for all warps: the CTA copies the next chunk's while it works on the
//     present one, and turns z into A fragments once, which the warps then read (copied and split by each warp for
//     itself they took a third of the kernel's time).
// The adapter's tokens are found in windows of kWindow: the CTA scans their adapters and lists its own, in order, so an
// adapter without tokens gets zeros and the sums' order does not depend on anything but the tokens'.
constexpr int kUnits = 3;
constexpr int kWindow = 4096, kChunk = 128;
constexpr int kColumns = 256, kPitch = kColumns + 2;
struct GradShared {
  uint16_t list[kWindow];
  int counts[16];
  alignas(16) uint8_t scales[2][kChunk][8];
};
// Sets of warps: four and one CTA an SM, or two and two CTAs (more than 32 ranks: two and one, whose registers they take).
// 17 to 32 ranks take all 128 registers and spill (36 bytes stored and 88 loaded with two sets, 4 and 8 with four).
constexpr int grad_ctas(int rt, int sets) { return rt == 4 ? 1 : 4 / sets; }  // an SM holds
constexpr int kUnitBytes = 2048;  // of rows, in a warp's ring
template <int kRT>
constexpr int frag_bytes() { return kChunk / 16 * kRT * 1024; }       // of a chunk: hi and lo, 16 bytes a lane each
template <int kRT>
constexpr int zrow_floats() { return 16 * kRT + 4; }                  // a token's z as copied
template <int kRT, int kSets>
constexpr int grad_smem_bytes() {
  return 4 * kSets * kUnits * kUnitBytes + 2 * frag_bytes<kRT>() + kChunk * zrow_floats<kRT>() * 4;
}

template <int kFormat, bool kRankMajor, int kRT, int kSub>
__device__ __forceinline__ void grad_tile(const Rows<kFormat>& rows, int64_t tokens, const Adapters& ad, const float* z,
                                          __nv_bfloat16* out, int64_t col0, int a, int r0, int csize, int crank,
                                          uint8_t* smem, GradShared& sh) {
  constexpr int kWarpsG = 4 * kSub, kThreadsG = 32 * kWarpsG;
  constexpr int kTurns = kChunk / 16 / kSub;  // a warp's units of a chunk
  constexpr int kZRow = zrow_floats<kRT>();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int sub = warp >> 2;
  const int rank = ad.rank;
  const int64_t cols = rows.cols;
  float acc[kRT][8][4];
#pragma unroll
  for (int i = 0; i < kRT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
  // the lane's 8 columns: bytes of them inside the rows, and a place inside
  const int64_t col = col0 + 64 * (warp & 3) + 8 * g;
  const int64_t colin = min(col, cols - 1) & ~(int64_t)7;
  const int colbytes = rows.bytes(col, true);
  const int block = (int)((colin - col0) / kCkptBlock) & 7;  // a column past the end may take any scale
  constexpr int kRow = kFormat < 0 ? 512 : 256;
  uint8_t* ring = smem + warp * kUnits * kUnitBytes + lane * (kRow / 32);
  uint8_t* frags = smem + kWarpsG * kUnits * kUnitBytes;
  float* zraw = reinterpret_cast<float*>(frags + 2 * frag_bytes<kRT>());
  bool any = false;  // tokens; alike in a cluster
  for (int64_t w0 = 0; w0 < tokens; w0 += kWindow) {
    __syncthreads();  // every warp has read the list and the scales of the window before
    int have = (int)min((int64_t)kWindow, tokens - w0);
    if (ad.of_token == nullptr) {
      if (a != 0) have = 0;  // all tokens are adapter 0's
    } else {
      // warp w lists tokens [w span, ..) of the window behind the warps' before it
      constexpr int kSpan = kWindow / kWarpsG;
      const int span = ((have + kWarpsG - 1) / kWarpsG + 31) & ~31;
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
      for (int v = 0; v < kWarpsG; ++v) {
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
    any |= have > 0;
    const int all = (have + kChunk - 1) / kChunk, chunks = all > crank ? (all - 1 - crank) / csize + 1 : 0;
    const auto token = [&](int e) { return w0 + (e < have ? (ad.of_token != nullptr ? (int)sh.list[e] : e) : 0); };
    // z and scales of this CTA's chunk c
    const auto fetch_chunk = [&](int c) {
      const int e0 = (crank + c * csize) * kChunk;
      for (int i = threadIdx.x; i < kChunk * 4 * kRT; i += kThreadsG) {
        const int e = e0 + i / (4 * kRT), r = 4 * (i % (4 * kRT));
        const bool on = e < have && r0 + r < rank;
        copy_16(zraw + i / (4 * kRT) * kZRow + r, z + token(e) * rank + (on ? r0 + r : 0), on ? 16 : 0);
      }
      if constexpr (kFormat >= 0) {
        const int64_t first = col0 / kCkptBlock, last = (cols + kCkptBlock - 1) / kCkptBlock;
        for (int i = threadIdx.x; i < kChunk * 2; i += kThreadsG) {
          const int e = e0 + i / 2, b = 4 * (i % 2);
          const uint8_t* src = rows.scale_row(token(e)) + first;
          uint8_t* dst = &sh.scales[c & 1][i / 2][b];
          if (rows.words) {
            const bool on = e < have && first + b < last;
            copy_4(dst, on ? src + b : rows.ckpt.scales, on ? 4 : 0);
          } else {
            for (int k = 0; k < 4; ++k) dst[k] = e < have && first + b + k < last ? __ldg(src + b + k) : (uint8_t)0;
          }
        }
      }
    };
    // rows of this warp's k-th unit
    const auto fetch_rows = [&](int k, int stage) {
      if (k < chunks * kTurns) {
        const int e0 = (crank + k / kTurns * csize) * kChunk + (sub + k % kTurns * kSub) * 16 + 2 * q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = e0 + (i & 1) + 8 * (i >> 1);  // slots 2 q, 2 q + 1, 2 q + 8, 2 q + 9
          rows.copy(ring + stage * kUnitBytes + i * kRow, rows.row(token(e)), colin, e < have ? colbytes : 0);
        }
      }
      copies_end();
    };
    if (chunks > 0) fetch_chunk(0);
#pragma unroll
    for (int i = 0; i < kUnits - 1; ++i) fetch_rows(i, i);
    int stage = 0, k = 0;
    for (int c = 0; c < chunks; ++c) {
      // chunk c's copies are older than the latest kUnits - 2 units' (the first chunk's came with the first unit's)
      copies_wait<kUnits - 2>();
      __syncthreads();
      uint8_t* frag = frags + (c & 1) * frag_bytes<kRT>();
      for (int i = threadIdx.x; i < kChunk / 16 * kRT * 32; i += kThreadsG) {
        // unit i / (32 kRT), ranks 16 m .., as this lane of the warps will read them: rows fg | fg + 8, slots
        // (2 fq, 2 fq + 1) | (2 fq + 8, 2 fq + 9)
        const int l = i & 31, m = i / 32 % kRT, u = i / (32 * kRT), fg = l >> 2, fq = l & 3;
        const float* src = zraw + (16 * u + 2 * fq) * kZRow + 16 * m + fg;
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const float z0 = src[8 * s * kZRow + 8 * h], z1 = src[(8 * s + 1) * kZRow + 8 * h];
            const uint32_t p = pack_bf16(z0, z1);
            hi[2 * s + h] = p;
            lo[2 * s + h] = pack_bf16(z0 - bf16_lo(p), z1 - bf16_hi(p));
          }
        uint4* dst = reinterpret_cast<uint4*>(frag) + (u * kRT + m) * 64 + l;
        dst[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        dst[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
      __syncthreads();
      if (c + 1 < chunks) fetch_chunk(c + 1);
      for (int turn = 0; turn < kTurns; ++turn, ++k) {
        fetch_rows(k + kUnits - 1, stage == 0 ? kUnits - 1 : stage - 1);
        copies_wait<kUnits - 1>();
        const int u = sub + turn * kSub;
        if ((crank + c * csize) * kChunk + 16 * u < have) {
          uint32_t v[4][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint8_t* src = ring + stage * kUnitBytes + i * kRow;
            uint4 x;
            if constexpr (kFormat < 0) {
              x = *reinterpret_cast<const uint4*>(src);
            } else {
              const uint32_t byte = sh.scales[c & 1][16 * u + 2 * q + (i & 1) + 8 * (i >> 1)][block];
              x = Rows<kFormat>::values(*reinterpret_cast<const uint2*>(src), ckpt_scale(byte));
            }
            v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
          }
          const uint4* fsrc = reinterpret_cast<const uint4*>(frag) + u * kRT * 64 + lane;
#pragma unroll
          for (int i = 0; i < kRT; ++i) {
            const uint4 h4 = fsrc[64 * i], l4 = fsrc[64 * i + 32];
            const uint32_t hi[4] = {h4.x, h4.y, h4.z, h4.w}, lo[4] = {l4.x, l4.y, l4.z, l4.w};
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
        stage = stage + 1 == kUnits ? 0 : stage + 1;
      }
    }
  }
  // acc[i][j]: ranks 16 i + g (e 0, 1) and + 8 (e 2, 3), N slots 2 q, 2 q + 1 of column tile j, which are columns
  // 8 (2 q) + j and 8 (2 q + 1) + j of the warp's 64.  The sets' partials: [set][rank][column].
  constexpr int kSize = 16 * kRT * kPitch;
  float* part = reinterpret_cast<float*>(smem);
  if (any) {
    copies_wait<0>();
    __syncthreads();  // the partials take the rings' place
  #pragma unroll
    for (int i = 0; i < kRT; ++i)
  #pragma unroll
      for (int j = 0; j < 8; ++j)
  #pragma unroll
        for (int e = 0; e < 4; ++e)
          part[sub * kSize + (16 * i + 8 * (e >> 1) + g) * kPitch + 64 * (warp & 3) + 8 * (2 * q + (e & 1)) + j] = acc[i][j][e];
    __syncthreads();
  }
  // `width` columns from c0 on; value(at): the sum at `at` of a partial
  const auto finish = [&](int c0, int width, auto value) {
    for (int i = threadIdx.x; i < 16 * kRT * width; i += kThreadsG) {
      // dA's rows run along the columns, dB's along the ranks
      const int rr = kRankMajor ? i / width : i % (16 * kRT), cc = c0 + (kRankMajor ? i % width : i / (16 * kRT));
      const int r = r0 + rr;
      const int64_t c = col0 + cc;
      if (r >= rank || c >= cols) continue;
      const float s = any ? value(rr * kPitch + cc) : 0.0f;
      out[kRankMajor ? ((int64_t)a * rank + r) * cols + c : ((int64_t)a * cols + c) * rank + r] = __float2bfloat16_rn(s);
    }
  };
  const auto sum_sets = [&](int at) {
    float s = part[at];
#pragma unroll
    for (int v = 1; v < kSub; ++v) s += part[v * kSize + at];
    return s;
  };
  if (csize == 1) {
    finish(0, kColumns, sum_sets);
    return;
  }
  // a rank of the cluster finishes a share of the columns
  if (any) {
    for (int i = threadIdx.x; i < kSize; i += kThreadsG) part[i] = sum_sets(i);
    cluster_sync();
  }
  const int share = (kColumns / 8 + csize - 1) / csize * 8, c0 = crank * share;
  finish(c0, min(share, kColumns - c0), [&](int at) {
    float s = ld_cluster(part + at, 0);
    for (int d = 1; d < csize; ++d) s += ld_cluster(part + at, (uint32_t)d);
    return s;
  });
  cluster_sync();
}

// blockIdx.x / csize: the column tiles of dA (tiles_a of them), then those of dB.
struct GradArgs {
  Adapters ad;
  int64_t tokens;
  const float *z, *dz;
  __nv_bfloat16 *da, *db;
  int csize, tiles_a;
};
template <int kFormat, int kRT, int kSets>
__global__ void __launch_bounds__(128 * kSets, grad_ctas(kRT, kSets)) grad_kernel(Rows<kFormat> x, Rows<-1> dy, GradArgs p) {
  extern __shared__ __align__(16) uint8_t grad_smem[];
  __shared__ GradShared sh;
  const int crank = p.csize > 1 ? (int)cluster_rank() : 0, tile = blockIdx.x / p.csize, r0 = blockIdx.z * 16 * kRT;
  if (tile < p.tiles_a)
    grad_tile<kFormat, true, kRT, kSets>(x, p.tokens, p.ad, p.dz, p.da, (int64_t)tile * kColumns, blockIdx.y, r0, p.csize, crank, grad_smem,
                                  sh);
  else
    grad_tile<-1, false, kRT, kSets>(dy, p.tokens, p.ad, p.z, p.db, (int64_t)(tile - p.tiles_a) * kColumns, blockIdx.y, r0, p.csize,
                              crank, grad_smem, sh);
}

template <int kFormat, int kRT, int kSets>
cudaError_t launch_grad_of(const Rows<kFormat>& x, const Rows<-1>& dy, GradArgs p, int64_t tiles, int passes, int sms,
                           cudaStream_t stream) {
  auto kernel = grad_kernel<kFormat, kRT, kSets>;
  constexpr int kCtas = grad_ctas(kRT, kSets);
  constexpr int kSmem = std::max(kSets * 16 * kRT * kPitch * 4, grad_smem_bytes<kRT, kSets>());
  static_assert(kCtas * (kSmem + sizeof(GradShared) + 1024) <= 228 * 1024, "shared memory");
  cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), kSmem);
  if (err != cudaSuccess) return err;
  // the tokens split (by up to four: clusters of eight CTAs that fill an SM each leave many SMs out) while a CTA an
  // SM holds all, and an adapter's share has a chunk of them
  const int64_t used = used_adapters(p.ad);
  p.csize = 1;
  while (p.csize < 4 && tiles * used * passes * (p.csize + 1) <= kCtas * sms && p.tokens / used > (int64_t)p.csize * kChunk)
    ++p.csize;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * p.csize), (unsigned)p.ad.count, (unsigned)passes);
  cfg.blockDim = dim3(128 * kSets, 1, 1);
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

template <int kFormat, int kRT>
cudaError_t launch_grad(const Rows<kFormat>& x, const Rows<-1>& dy, GradArgs p, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  p.tiles_a = p.da != nullptr ? (int)((x.cols + kColumns - 1) / kColumns) : 0;
  const int64_t tiles = p.tiles_a + (p.db != nullptr ? (dy.cols + kColumns - 1) / kColumns : 0);
  const int passes = (p.ad.rank + 16 * kRT - 1) / (16 * kRT), sms = info.sm_count;
  if constexpr (kRT == 4) {
    return launch_grad_of<kFormat, kRT, 2>(x, dy, p, tiles, passes, sms, stream);
  } else {
    // with more CTAs than SMs, two an SM (2048 tokens on 32 adapters, 1024 x 4096: 62 -> 52 us); with fewer, each the faster
    // the more warps it has (300 tokens on 4, 2048 x 2048: 25.7 us and 24.7)
    return tiles * used_adapters(p.ad) * passes > sms ? launch_grad_of<kFormat, kRT, 2>(x, dy, p, tiles, passes, sms, stream)
                                                     : launch_grad_of<kFormat, kRT, 4>(x, dy, p, tiles, passes, sms, stream);
  }
}

Rows<-1> bf16_rows(const void* x, int64_t ld, int64_t cols) { return {static_cast<const uint16_t*>(x), ld, {}, cols, 1, false}; }

template <int kFormat>
Rows<kFormat> ckpt_rows(const Checkpoint& c, int64_t cols) {
  const uintptr_t base = reinterpret_cast<uintptr_t>(c.codes);
  const int vec = base % 16 == 0 && c.ld_codes % 16 == 0 ? 16 : base % 8 == 0 && c.ld_codes % 8 == 0 ? 8 : 1;
  const bool words = reinterpret_cast<uintptr_t>(c.scales) % 4 == 0 && c.ld_scales % 4 == 0 && cols % 128 == 0;
  return {nullptr, 0, c, cols, vec, words};
}

template <int kFormat>
cudaError_t backward_products(const Checkpoint& c, int64_t n, const Rows<-1>& dy, const ShrinkArgs& p, cudaStream_t stream) {
  return launch_shrink<kFormat>(ckpt_rows<kFormat>(c, n), dy, p, stream);
}
template <int kFormat>
cudaError_t gradients(const Checkpoint& c, int64_t n, const Rows<-1>& dy, const GradArgs& p, cudaStream_t stream) {
  const Rows<kFormat> x = ckpt_rows<kFormat>(c, n);
  if (p.ad.rank <= 16) return launch_grad<kFormat, 1>(x, dy, p, stream);
  return p.ad.rank <= 32 ? launch_grad<kFormat, 2>(x, dy, p, stream) : launch_grad<kFormat, 4>(x, dy, p, stream);
}

}  // namespace

cudaError_t launch_adapter_down(const void* x, int64_t ld_x, int64_t tokens, int64_t n, const Adapters& ad,
                                const float* global_scale, float* z, uint32_t* z_split, cudaStream_t stream) {
  const ShrinkArgs p = {ad, tokens, global_scale, z, nullptr, z_split, nullptr, 1, 1, 0};
  return launch_shrink<-1>(bf16_rows(x, ld_x, n), bf16_rows(nullptr, 0, 0), p, stream);
}

cudaError_t launch_adapter_backward(const Checkpoint& x, int format, int64_t n, const void* dy, int64_t ld_dy, int64_t m,
                                    int64_t tokens, const Adapters& ad, const float* global_scale, float* z, float* dz,
                                    uint32_t* dz_split, cudaStream_t stream) {
  const ShrinkArgs p = {ad, tokens, global_scale, z, dz, nullptr, dz_split, 1, 1, 1};
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
