// experts.cu -- a layer of experts with packed NVFP4 weights on the tcgen05 tensor cores:
//   y_t = sum_j w_tj D_e (act(G_e x_t) * (U_e x_t)),  e = ids[t, j]
// Steps, each launched while the one before it runs: the slots (token, j) are grouped by expert; their x is laid out in that
// order, in fp16 (experts.cuh); the first product makes h = act(G x) * (U x) in fp16 under powers of two of 32 outputs; h is
// moved under a power of two of its row; the second product makes D h of each slot in fp32; a token's slots are
// weighted and added up in order, and rounded once.
//
// The products.  Tile: 256 rows of weights as two halves of 128 (128 rows of G and the same 128 of U, or 256 rows of
// D) x up to kN slots of one expert, K in blocks of 64.  24 warps:
//   0      TMA loads of the slots' tile, K-major, 128-byte swizzle
//   1      MMAs
//   2-5    epilogue (lane = row of weights, columns = slots)
//   6-21   unpacking: a group of four for each half and every other block; a thread has one row, and writes 64 fp16
//          weights a block into tensor memory, from where the MMAs take their A operand: shared memory, which both
//          operands would saturate, holds the slots' tile and the packed rows alone
//   22-23  the packed rows, 256 columns a stage, as many stages ahead as fit (experts.cuh: how they come)
// A block's 16384 weights cost the unpacking warps some 1200 instructions, 300 cycles at best; its bytes take 390 cycles at the
// card's bandwidth, its MMAs 512 at 128 slots.  So few slots are bound by memory (16 tokens of 64 experts, 4096 x 2048, k 8:
// 147 us, 5.4 TB/s of weights, the launches around the products among them), many by the tensor cores (32768 slots: 1.65 PFLOP/s
// in the first product, 1.45 in the second, whose K is half as long; the rest is the epilogue, for which tensor memory has
// no second accumulator at 128 slots: the unpacking warps take part in it).  One token: latency, of six launches one
// behind another and of each product's first loads.
//
// A packed stage is given back only when its values have been used: an arrival right behind the loads had TMA
// overwrite rows that were still being read.  The plan is complete before a product's kernel may start, so its weights come
// while the kernel before it still runs.
//
// Every wait is bounded; a CTA in which one ran out writes NaN for what it owed and sets the error flag.
#include <algorithm>
#include <type_traits>

#include "chained_launch.h"
#include "experts.cuh"
#include "hscale_internal.h"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace hscale {
namespace {

__device__ uint32_t g_experts_flags = 0;

constexpr int kSpreadKept = 4;  // 16-byte pieces of a row that a thread keeps in registers: 8192 columns

// ---------------------------------------------------------------- grouping
constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kPlanAhead = 8;  // ids a lane has in flight: one at a time, 32768 slots took 56 us

constexpr int64_t kPlanSlots = 4096;  // of a CTA, where there are more

// An expert's chunks: nearly the same size, whole 16s.
__device__ __forceinline__ void cut(int expert, int first, int total, int pieces, Chunk* to) {
  const int each = pieces ? ((total + pieces - 1) / pieces + 15) / 16 * 16 : 0;
  for (int c = 0; c < pieces; ++c) {
    const int from = min(total, c * each), end = min(total, from + each);
    to[c] = {expert, first + from, end - from, 0};
  }
}

// The slots of each expert in each run of kPlanSlots slots: counts [runs][experts].
__global__ void __launch_bounds__(kPlanThreads) count_kernel(const int32_t* __restrict__ ids, int64_t slots, int experts,
                                                             int32_t* __restrict__ counts) {
  __shared__ int32_t mine[kRouteExperts];
  pdl_launch_dependents();
  for (int e = threadIdx.x; e < experts; e += kPlanThreads) mine[e] = 0;
  __syncthreads();
  const int64_t s0 = (int64_t)blockIdx.x * kPlanSlots, s1 = min(slots, s0 + kPlanSlots);
  for (int64_t s = s0 + threadIdx.x; s < s1; s += kPlanThreads) {
    const int id = ids[s];
    if ((unsigned)id < (unsigned)experts) atomicAdd(&mine[id], 1);  // whole numbers
  }
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kPlanThreads) counts[(int64_t)blockIdx.x * experts + e] = mine[e];
}

// A stable counting sort: each warp counts a run of slots, the warps' counts are summed up expert by expert, and each
// warp then places its run.  By one CTA, or a CTA for each run of count_kernel's (run_counts; one CTA alone took 32768 slots 36 us).
// Integers only: equal calls give equal plans.
// wide: chunks of another width over the same positions (its chunks and their number alone; nullptr: none).
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const int32_t* ids, int64_t slots, int experts, int width, Plan plan,
                                                            int wide_width, Plan wide, const int32_t* run_counts) {
  extern __shared__ int32_t counts[];  // [kPlanWarps][experts], then each expert's first position
  int32_t* first = counts + kPlanWarps * experts;
  __shared__ int32_t warp_total[kPlanWarps], warp_chunks[kPlanWarps], warp_wide[kPlanWarps];
  if (run_counts != nullptr) pdl_wait_primary();
  pdl_launch_dependents();
  if (slots <= 32) {
    // a warp's: an expert's place by the slots of lower ones
    if (threadIdx.x >= 32) return;
    const int lane = threadIdx.x, id = lane < slots ? ids[lane] : -1;
    const bool on = (unsigned)id < (unsigned)experts;
    const uint32_t alike = __match_any_sync(0xFFFFFFFFu, on ? id : -1), below = (1u << lane) - 1u;
    const bool leads = on && (alike & below) == 0u;
    const int total = __popc(alike), pieces = leads ? (total + width - 1) / width : 0;
    const int wide_pieces = leads ? (total + wide_width - 1) / wide_width : 0;
    int at = 0, chunk = 0, wide_chunk = 0, chunks = 0, wide_chunks = 0;
    for (int j = 0; j < (int)slots; ++j) {
      const int other = __shfl_sync(0xFFFFFFFFu, on ? id : INT32_MAX, j), n = __shfl_sync(0xFFFFFFFFu, pieces, j),
                w = __shfl_sync(0xFFFFFFFFu, wide_pieces, j);
      if (other < id) ++at, chunk += n, wide_chunk += w;
      chunks += n, wide_chunks += w;
    }
    if (on) plan.slot_of[at + __popc(alike & below)] = lane;
    if (lane < slots) plan.pos_of[lane] = on ? at + __popc(alike & below) : -1;
    if (leads) {
      cut(id, at, total, pieces, plan.chunks + chunk);
      if (wide.header != nullptr) cut(id, at, total, wide_pieces, wide.chunks + wide_chunk);
    }
    const uint32_t placed = __ballot_sync(0xFFFFFFFFu, on);
    if (lane == 0) {
      plan.header[0] = chunks, plan.header[1] = __popc(placed);
      if (wide.header != nullptr) wide.header[0] = wide_chunks;
    }
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t begin = run_counts != nullptr ? blockIdx.x * kPlanSlots : 0;
  const int64_t stop = run_counts != nullptr ? min(slots, begin + kPlanSlots) : slots;
  const int64_t run = (stop - begin + kPlanWarps - 1) / kPlanWarps, s0 = begin + warp * run, s1 = min(stop, s0 + run);
  for (int i = threadIdx.x; i < kPlanWarps * experts; i += kPlanThreads) counts[i] = 0;
  __syncthreads();
  int32_t* mine = counts + warp * experts;
  for (int64_t s = s0; s < s1; s += 32 * kPlanAhead) {
    int id[kPlanAhead];
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) id[u] = s + 32 * u + lane < s1 ? ids[s + 32 * u + lane] : -1;
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) {
      if (s + 32 * u >= s1) break;
      const bool on = (unsigned)id[u] < (unsigned)experts;
      if (on) atomicAdd(&mine[id[u]], 1);  // the warp's own, whole numbers
    }
  }
  __syncthreads();
  // expert e = threadIdx.x (at most 1024): its slots, then the experts' first positions and first chunks
  int total = 0, before = 0;  // before: in the runs before this CTA's
  if ((int)threadIdx.x < experts) {
    for (int w = 0; w < kPlanWarps; ++w) {
      const int c = counts[w * experts + threadIdx.x];
      counts[w * experts + threadIdx.x] = total;
      total += c;
    }
    if (run_counts != nullptr) {
      total = 0;
      for (int g = 0; g < (int)gridDim.x; ++g) {
        const int c = run_counts[(int64_t)g * experts + threadIdx.x];
        if (g < (int)blockIdx.x) before += c;
        total += c;
      }
    }
  }
  const int pieces = (total + width - 1) / width, wide_pieces = (total + wide_width - 1) / wide_width;
  int at = total, chunk = pieces, wide_chunk = wide_pieces;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int a = __shfl_up_sync(0xFFFFFFFFu, at, d), b = __shfl_up_sync(0xFFFFFFFFu, chunk, d), c = __shfl_up_sync(0xFFFFFFFFu, wide_chunk, d);
    if (lane >= d) at += a, chunk += b, wide_chunk += c;
  }
  if (lane == 31) warp_total[warp] = at, warp_chunks[warp] = chunk, warp_wide[warp] = wide_chunk;
  __syncthreads();
  for (int w = 0; w < warp; ++w) at += warp_total[w], chunk += warp_chunks[w], wide_chunk += warp_wide[w];
  if (threadIdx.x == kPlanThreads - 1 && blockIdx.x == 0) {
    plan.header[0] = chunk, plan.header[1] = at;
    if (wide.header != nullptr) wide.header[0] = wide_chunk;
  }
  at -= total, chunk -= pieces, wide_chunk -= wide_pieces;
  if ((int)threadIdx.x < experts) {
    first[threadIdx.x] = at + before;
    if (blockIdx.x == 0) {
      cut((int)threadIdx.x, at, total, pieces, plan.chunks + chunk);
      if (wide.header != nullptr) cut((int)threadIdx.x, at, total, wide_pieces, wide.chunks + wide_chunk);
    }
  }
  __syncthreads();
  for (int64_t s = s0; s < s1; s += 32 * kPlanAhead) {
    int id[kPlanAhead];
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) id[u] = s + 32 * u + lane < s1 ? ids[s + 32 * u + lane] : -1;
#pragma unroll
    for (int u = 0; u < kPlanAhead; ++u) {
      if (s + 32 * u >= s1) break;
      const bool on = (unsigned)id[u] < (unsigned)experts;
      const uint32_t alike = __match_any_sync(0xFFFFFFFFu, on ? id[u] : -1);
      int pos = -1;
      if (on) {
        pos = first[id[u]] + mine[id[u]] + __popc(alike & ((1u << lane) - 1u));
        plan.slot_of[pos] = (int32_t)(s + 32 * u + lane);
      }
      if (s + 32 * u + lane < s1) plan.pos_of[s + 32 * u + lane] = pos;
      __syncwarp();
      if (on && __ffs(alike) - 1 == lane) mine[id[u]] += __popc(alike);
      __syncwarp();
    }
  }
}

// A token's row in fp16 (experts.cuh) to the positions of its slots, with the row's amax; a row of h begins with none.
// Where weight_of is not nullptr, the slots' weights too.
// gridDim.y of them: of x, and of the backward pass's dy.
struct Spread {
  const uint4* x;
  int64_t ld;
  uint4* out;
  uint32_t* amax;
};
__global__ void __launch_bounds__(256) spread_kernel(Spread first, Spread second, int64_t pieces, int k, Plan plan, uint32_t* h_amax,
                                                     const float* weights, float* weight_of) {
  __shared__ uint32_t warp_max[8];
  pdl_wait_primary();
  pdl_launch_dependents();
  const Spread& s = blockIdx.y ? second : first;
  uint4* out = s.out;
  uint32_t* amax = s.amax;
  const int64_t t = blockIdx.x;
  const uint4* row = s.x + t * s.ld;
  uint4 kept[kSpreadKept];
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < kSpreadKept; ++i) {
    const int64_t at = threadIdx.x + 256 * i;
    if (at < pieces) m = max(m, amax_bf16(kept[i] = row[at]));
  }
  for (int64_t at = threadIdx.x + 256 * kSpreadKept; at < pieces; at += 256) m = max(m, amax_bf16(row[at]));
  m = __reduce_max_sync(0xFFFFFFFFu, m);
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, warp_max[i]);
  const float down = exp2_int(-row_exponent(m));
#pragma unroll
  for (int i = 0; i < kSpreadKept; ++i) kept[i] = bf16_to_f16(kept[i], down);
  for (int j = 0; j < k; ++j) {
    const int64_t pos = plan.pos_of[t * k + j];
    if (pos < 0) continue;
    if (threadIdx.x == 0) {
      amax[pos] = m;
      if (h_amax != nullptr) h_amax[pos] = 0u;
      if (weight_of != nullptr) weight_of[pos] = weights[t * k + j];
    }
    uint4* to = out + pos * pieces;
#pragma unroll
    for (int i = 0; i < kSpreadKept; ++i)
      if (threadIdx.x + 256 * i < pieces) to[threadIdx.x + 256 * i] = kept[i];
    for (int64_t at = threadIdx.x + 256 * kSpreadKept; at < pieces; at += 256) to[at] = bf16_to_f16(row[at], down);
  }
}

// Rows of fp16 from their groups' powers of two to the row's, in place, 16 bytes a thread: exact but where a number is below
// 2^-14 then.  A row is `pieces` of 16 bytes in parts of `part`, which have the same groups; those under the row's power
// already are neither read nor written.
__global__ void __launch_bounds__(256) level_kernel(uint4* h, int64_t pieces, int64_t part, Plan plan, const uint32_t* amax, const int8_t* groups) {
  pdl_launch_dependents();  // the next product's weights may come; it waits for this kernel before it reads h
  pdl_wait_primary();
  const int64_t total = plan.header[1] * pieces, per = (part + 3) / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / pieces;
    const uint32_t at = (uint32_t)(i - row * pieces);
    const int e = (int)groups[row * per + at % (uint32_t)part / 4] - row_exponent(amax[row]);
    if (e == 0) continue;
    const float f = exp2_int(max(e, -126));
    const uint4 v = h[i];
    const auto move = [&](uint32_t w) {
      const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w));
      return pack_f16(x.x * f, x.y * f);
    };
    h[i] = make_uint4(move(v.x), move(v.y), move(v.z), move(v.w));
  }
}

// out_t = the sum of the token's slots' rows (part, and more where it is not nullptr) times their weights (nullptr: 1), in order;
// four columns a thread.  The threads behind them, where there are dots: dweights of each slot, the sum of its position's `parts` partial
// sums, in order, and 0 of a slot without an expert.
struct Combine {
  const float *part, *more, *weights;
  __nv_bfloat16* out;
  int64_t n, ld, tokens;
  int32_t k;
  const float* dots;
  int32_t parts;
  float* dweights;
};
__global__ void __launch_bounds__(256) combine_kernel(const __grid_constant__ Combine c, Plan plan) {
  pdl_wait_primary();
  const int64_t per = c.out != nullptr ? c.n / 4 : 0;
  int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= c.tokens * per) {
    i -= c.tokens * per;
    const int64_t slots = c.tokens * c.k;
    if (c.dots == nullptr || i >= slots) return;
    if (plan.pos_of[i] < 0) c.dweights[i] = 0.0f;
    if (i >= plan.header[1]) return;
    // position i's, so that a warp's are side by side
    float s = 0.0f;
#pragma unroll 8
    for (int q = 0; q < c.parts; ++q) s += c.dots[(int64_t)q * slots + i];
    c.dweights[plan.slot_of[i]] = s;
    return;
  }
  const int64_t t = i / per, col = (i - t * per) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int j = 0; j < c.k; ++j) {
    const int64_t pos = plan.pos_of[t * c.k + j];
    if (pos < 0) continue;
    const float w = c.weights == nullptr ? 1.0f : c.weights[t * c.k + j];
    float4 v = *reinterpret_cast<const float4*>(c.part + pos * c.n + col);
    if (c.more != nullptr) {
      const float4 m = *reinterpret_cast<const float4*>(c.more + pos * c.n + col);
      v.x += m.x, v.y += m.y, v.z += m.z, v.w += m.w;
    }
    s.x = fmaf(w, v.x, s.x), s.y = fmaf(w, v.y, s.y), s.z = fmaf(w, v.z, s.z), s.w = fmaf(w, v.w, s.w);
  }
  uint2 r;
  r.x = pack_bf16(s.x, s.y), r.y = pack_bf16(s.z, s.w);
  *reinterpret_cast<uint2*>(c.out + t * c.ld + col) = r;
}

// ---------------------------------------------------------------- the products
constexpr int kBM = 128, kBK = 64, kHalves = 2;
constexpr int kEpilogueWarp0 = 2, kUnpackWarp0 = 6, kUnpackWarps = 16, kWeightsWarp0 = 22;
constexpr int kThreads = 768;
constexpr int kModeHidden = 0, kModeRaw = 1, kModeDown = 2;
// A packed block: kQuad blocks of K of the tile's rows, 128 bytes a row, and 16 bytes of their codes (20 where they are
// copied as whole words from any address).
constexpr int kQuad = 4;
constexpr uint32_t kRowBytes = kPackedRow;
static_assert(kRowBytes == kQuad * kBK / 2, "a packed stage's rows");
constexpr uint32_t kHalfBytes = kBM * kPairRow, kHalfCodes = kBM * kCodeRow;
constexpr uint32_t kPackedBytes = kHalves * (kHalfBytes + kHalfCodes);

template <int kN>
struct Tile {
  static constexpr int kStages = kN <= 32 ? 6 : 4;  // unpacked blocks and blocks of the slots' tile
  static constexpr int kAccs = kN <= 64 ? 2 : 1;
  static constexpr bool kHelp = kAccs == 1;  // the unpacking warps take part in the epilogue
  static constexpr int kPackedStages = kN == 16 ? 5 : kN <= 64 ? 4 : 3;
  static constexpr int kEpilogueWarps = kHelp ? 4 + kUnpackWarps : 4;
  static constexpr uint32_t kBBytes = kN * kBK * 2;
  static constexpr uint32_t kTurnBytes = kEpilogueWarps * 1024;
  static constexpr uint32_t kSmemBytes = kStages * kBBytes + kPackedStages * kPackedBytes + 1024 /* alignment */ + 512 /* barriers */ + kTurnBytes;
  static constexpr uint32_t kAcc = kHalves * kN;                // columns of an accumulator
  static constexpr uint32_t kA0 = kAccs * kAcc;                 // the weights' first column
  static constexpr uint32_t kAStage = kHalves * kBK / 2;
  static_assert(kA0 + kStages * kAStage <= 512, "tensor memory");
  static_assert(kSmemBytes <= 232448, "shared memory");
};

struct GemmArgs {
  ExpertMatrix a, b;  // the tile's halves
  int64_t rows, cols;  // of an expert's matrix
  int32_t kb_total, tiles_o, tile_rows;  // tile_rows: between the tiles' first rows
  int32_t segments, kb_segment;          // of kModeRaw: K's segments, and their K blocks (whole stages; the last has fewer)
  int32_t activation;
  int32_t path;  // packed_path
  int64_t all_rows;  // of all experts
  Plan plan;
  const uint32_t* amax;  // of each position's row of the slots' tile
  uint32_t* h_amax;      // of each position's h
  int8_t* h_groups;      // [positions, level_groups(rows)] powers of two of h
  void* out;
};

// D[tmem] (+)= A[tmem] * B[smem]^T: A's row in its lane, two elements of K a column.
__device__ __forceinline__ void umma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// kPath: how the packed rows are read: kBulk, kMixed (kCopies too), kPairs or kDirect.  (A branch on it in the unpacking
// cost a decoding batch 7%.)
template <int kMode, int kN, int kPath>
__global__ void __launch_bounds__(kThreads, 1)
gemm_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap,
            const __grid_constant__ CUtensorMap acodes, const __grid_constant__ CUtensorMap bcodes, const __grid_constant__ GemmArgs p) {
  using T = Tile<kN>;
  constexpr int kStages = T::kStages, kAccs = T::kAccs, kPackedStages = T::kPackedStages;
  extern __shared__ __align__(16) uint8_t dynamic_smem[];
  uint8_t* smem = dynamic_smem + ((1024u - (smem_addr(dynamic_smem) & 1023u)) & 1023u);
  uint8_t* tile_b = smem;
  uint8_t* packed = smem + kStages * T::kBBytes;                                    // [stages][halves]
  uint8_t* packed_codes = packed + kPackedStages * kHalves * kHalfBytes;            // [stages][halves]
  uint8_t* rest = packed_codes + kPackedStages * kHalves * kHalfCodes;
  uint64_t* full = reinterpret_cast<uint64_t*>(rest);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + kAccs;
  uint64_t* packed_full = acc_empty + kAccs;
  uint64_t* packed_empty = packed_full + kPackedStages;
  uint64_t* mma_done = packed_empty + kPackedStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  uint32_t* failed = tmem_slot + 1;

  const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1 + kHalves * 4);  // the TMA load and the warps of the halves' groups
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kPackedStages; ++s) {
      mbar_init(&packed_full[s], (p.path == kBulk ? 0 : 2 * 32) + (p.path >= kMixed ? 1 : 0));
      mbar_init(&packed_empty[s], kUnpackWarps);
    }
    for (int i = 0; i < kAccs; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], T::kEpilogueWarps);
    }
    mbar_init(mma_done, 1);
    *failed = 0u;
    mbar_fence_init();
    prefetch_tensormap(&vmap);
    if (p.path >= kMixed) prefetch_tensormap(&amap), prefetch_tensormap(&bmap);
    if (p.path == kBulk) prefetch_tensormap(&acodes), prefetch_tensormap(&bcodes);
  }
  if (warp == 1) {
    tmem_alloc(smem_addr(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  // The plan is there: the kernel that this one may run beside has waited for it.  What that kernel writes (the slots'
  // tile, and the rows' amax) is waited for where it is read; the weights begin to come meanwhile.

  // The CTA's tile i.  In kModeRaw a tile's segments of K are tiles one after another, each summed up from zero and added to
  // what the ones before left (gate_up_segments).
  const int segments = kMode == kModeRaw ? p.segments : 1;
  const int tiles = p.plan.header[0] * p.tiles_o, step = (int)gridDim.x, first = (int)blockIdx.x;
  const int ntiles = tiles > first ? (tiles - first + step - 1) / step * segments : 0;
  const auto tile_of = [&](int i) { return first + (kMode == kModeRaw ? i / segments : i) * step; };
  const auto kb_first = [&](int i) { return kMode == kModeRaw ? i % segments * p.kb_segment : 0; };
  const auto kb_count = [&](int i) { return kMode == kModeRaw ? min(p.kb_segment, p.kb_total - kb_first(i)) : p.kb_total; };
  const uint32_t quarter = (uint32_t)(warp & 3), lane_base = (quarter * 32u) << 16;
  const int row_in_half = (int)quarter * 32 + lane;
  bool have = true;  // of the warps of the epilogue: no wait for an accumulator has run out

  // What a warp's epilogue of the CTA's tile i needs, fetched before its time: the chunk, the matrices' scales, and the power
  // of two of the rows of its first 16 slots and its second (lane j: slot j's).
  struct Finish {
    Chunk c;
    float scale_a, scale_b, up0, up1;
  };
  constexpr int kWorkers = T::kEpilogueWarps / 4;
  const auto up_of = [&](const Chunk& c, int j) { return lane < 16 && j + lane < c.count ? exp2_int(row_exponent(p.amax[c.first + j + lane])) : 0.0f; };
  const auto prepare = [&](int i, int who) {
    Finish f;
    f.c = p.plan.chunks[tile_of(i) / p.tiles_o];
    f.scale_a = p.a.scale[f.c.expert], f.scale_b = p.b.scale[f.c.expert];
    f.up0 = up_of(f.c, 16 * who), f.up1 = up_of(f.c, 16 * (who + kWorkers));
    return f;
  };
  const auto release = [&](uint32_t acc) {
    tc_fence_before_sync();
    __syncwarp();
    // a warp that writes NaN runs ahead of the others: its arrivals would stand for theirs, and the next tile's MMAs overwrite
    // what they still read
    if (lane == 0 && have) mbar_arrive(&acc_empty[acc]);
  };
  // The epilogue: 16 slots a time, those of this warp (one of kWorkers of its quarter).
  const auto finish = [&](int i, int who, uint32_t* turn, const Finish& f) {
    const int t = tile_of(i);
    const Chunk& c = f.c;
    const int64_t o0 = (int64_t)(t % p.tiles_o) * p.tile_rows, o = o0 + row_in_half;
    const uint32_t acc = (uint32_t)i % kAccs, d = tmem + acc * T::kAcc + lane_base;
    const float scale_a = f.scale_a, scale_b = f.scale_b;
    const float nan = __int_as_float(0x7FC00000);
    if (have) have = __all_sync(0xFFFFFFFFu, mbar_wait_acc(&acc_full[acc], (uint32_t)(i / kAccs) & 1u));
    tc_fence_after_sync();
#pragma unroll 1
    for (int j0 = 16 * who, turns = 0; j0 < c.count; j0 += 16 * kWorkers, ++turns) {
      const int left = min(16, c.count - j0);
      const float my_up = turns == 0 ? f.up0 : turns == 1 ? f.up1 : up_of(c, j0);
      uint32_t a[16], b[16];
      tmem_ld_32x32b_x16(d + (uint32_t)j0, a);
      tmem_ld_32x32b_x16(d + (uint32_t)(kN + j0), b);
      tmem_ld_wait();
      // the warp's last columns: the next tile's MMAs need not wait for what is done with them
      if (j0 + 16 * kWorkers >= c.count) release(acc);
      if constexpr (kMode == kModeHidden) {
        // rounded (lane j: slot j's power of two) and turned, so that a lane stores 8 outputs of a slot at once
        const float my_a = have ? my_up * scale_a : nan, my_b = my_up * scale_b;
        const auto hidden = [&](auto kind) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            a[j] = __float_as_uint(activate_fast<decltype(kind)::value>(__uint_as_float(a[j]) * __shfl_sync(0xFFFFFFFFu, my_a, j)) *
                                   (__uint_as_float(b[j]) * __shfl_sync(0xFFFFFFFFu, my_b, j)));
        };
        if (p.activation == kActSilu)
          hidden(std::integral_constant<int, kActSilu>{});
        else
          hidden(std::integral_constant<int, kActGeluTanh>{});
        uint32_t most = 0u;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t m = __reduce_max_sync(0xFFFFFFFFu, o < p.rows ? a[j] & 0x7FFFFFFFu : 0u);
          if (lane == j) most = m >> 16;
        }
        const int e = row_exponent(most);
        const float down = exp2_int(-e);
        const int64_t at32 = o0 + quarter * 32;
        if (lane < left && at32 < p.rows) {
          const int64_t pos = c.first + j0 + lane;
          p.h_groups[pos * level_groups(p.rows) + at32 / kLevel] = (int8_t)e;
          atomicMax(&p.h_amax[pos], most);
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          turn[j * 32 + lane] = pack_f16(__uint_as_float(a[2 * j]) * __shfl_sync(0xFFFFFFFFu, down, 2 * j),
                                         __uint_as_float(a[2 * j + 1]) * __shfl_sync(0xFFFFFFFFu, down, 2 * j + 1));
        __syncwarp();
        const int pair = lane >> 2;
        const uint4 q0 = reinterpret_cast<const uint4*>(turn)[2 * lane], q1 = reinterpret_cast<const uint4*>(turn)[2 * lane + 1];
        const int64_t at = at32 + (lane & 3) * 8;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t pick = e ? 0x7632u : 0x5410u;
          const uint4 r = make_uint4(__byte_perm(q0.x, q0.y, pick), __byte_perm(q0.z, q0.w, pick), __byte_perm(q1.x, q1.y, pick),
                                     __byte_perm(q1.z, q1.w, pick));
          // rows are a multiple of 16: 8 outputs are all there or none is
          const int64_t pos = c.first + j0 + 2 * pair + e;
          if (2 * pair + e < left && at < p.rows) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + pos * p.rows + at) = r;
        }
      } else if constexpr (kMode == kModeRaw) {
        // 32 outputs of a slot side by side, g with u
        float2* out = static_cast<float2*>(p.out) + (int64_t)(c.first + j0) * p.rows + o;
        const bool on = o < p.rows;
        const bool add = kb_first(i) > 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float up = __shfl_sync(0xFFFFFFFFu, my_up, j), upn = have ? up : nan;
          const float vg = __uint_as_float(a[j]) * (scale_a * upn), vu = __uint_as_float(b[j]) * (scale_b * upn);
          if (j < left && on) {
            // to what this thread wrote there before, in that order: no other adds
            if (add)
              asm volatile("red.relaxed.gpu.global.add.v2.f32 [%0], {%1, %2};" ::"l"(out), "f"(vg), "f"(vu) : "memory");
            else
              *out = make_float2(vg, vu);
          }
          out += p.rows;
        }
      } else {
        // 32 outputs of a slot side by side
        float* out = static_cast<float*>(p.out) + (int64_t)(c.first + j0) * p.rows + o;
        const bool on_a = o < p.rows, on_b = o + kBM < p.rows;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float up = have ? __shfl_sync(0xFFFFFFFFu, my_up, j) : nan;
          if (j < left && on_a) out[0] = __uint_as_float(a[j]) * (scale_a * up);
          if (j < left && on_b) out[kBM] = __uint_as_float(b[j]) * (scale_b * up);
          out += p.rows;
        }
      }
    }
    if (16 * who >= c.count) release(acc);
  };
  const auto turn_at = [&](int worker) { return reinterpret_cast<uint32_t*>(rest + 512 + worker * 1024); };

  if (warp == 0) {
    pdl_wait_primary();
    pdl_launch_dependents();
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      const Chunk c = p.plan.chunks[tile_of(i) / p.tiles_o];
      const int kb0 = kb_first(i), kbs = kb_count(i);
      for (int kb = 0; kb < kbs; ++kb) {
        if (!mbar_wait_warp(&empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(&full[s], T::kBBytes);
          tma_load_2d(tile_b + s * T::kBBytes, &vmap, (kb0 + kb) * kBK, c.first, &full[s], policy);
        }
        __syncwarp();
        if (++s == kStages) s = 0, parity ^= 1u;
      }
    }
    ring_drain(full, kStages, s, parity);
  } else if (warp == 1) {
    uint32_t s = 0, parity = 0;
    bool ok = true;
    for (int i = 0; i < ntiles && ok; ++i) {
      const Chunk c = p.plan.chunks[tile_of(i) / p.tiles_o];
      const int kbs = kb_count(i);
      const uint32_t idesc = warp_uniform(idesc_f16_f32(kBM, (uint32_t)((c.count + 15) & ~15)));
      const uint32_t acc = (uint32_t)i % kAccs, d = tmem + acc * T::kAcc;
      if (i >= kAccs && !mbar_wait_warp(&acc_empty[acc], (uint32_t)(i / kAccs - 1) & 1u)) {
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
          const uint64_t bd = smem_desc_k_sw128(smem_addr(tile_b + s * T::kBBytes));
          const uint32_t a = tmem + T::kA0 + s * T::kAStage;
#pragma unroll
          for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int kk = 0; kk < kBK / 16; ++kk)
              umma_f16_ts(d + half * kN, a + half * (kBK / 2) + 8 * kk, bd + 2 * kk, idesc, (uint32_t)(kb > 0 || kk > 0));
          umma_commit(smem_addr(&empty[s]));
        }
        __syncwarp();
        if (++s == kStages) s = 0, parity ^= 1u;
      }
      if (ok && elect_one()) umma_commit(smem_addr(&acc_full[acc]));
      __syncwarp();
    }
    if (!ok && lane == 0) atomicOr(failed, 1u);
    __syncwarp();
    umma_drain(mma_done);
  } else if (warp < kUnpackWarp0) {
    pdl_wait_primary();
    Finish f = {};
    if (ntiles > 0) f = prepare(0, 0);
    for (int i = 0; i < ntiles; ++i) {
      finish(i, 0, turn_at(warp - kEpilogueWarp0), f);
      if (i + 1 < ntiles) f = prepare(i + 1, 0);
    }
    if (!have && lane == 0) atomicOr(failed, 1u);
  } else if (warp < kWeightsWarp0) {
    // group: the half it unpacks, of every other K block
    const int group = (warp - kUnpackWarp0) >> 2, half = group & 1, odd = group >> 1;
    const ExpertMatrix& w = half ? p.b : p.a;
    const int64_t cols = p.cols, half_cols = cols >> 1, code_cols = cols >> 4;
    const int row_in_tile = row_in_half + (kMode == kModeDown && half ? kBM : 0);
    const uint32_t src = smem_addr(packed + half * kHalfBytes);
    const uint32_t code_src = smem_addr(packed_codes + half * kHalfCodes);
    uint32_t* turn = turn_at(T::kHelp ? 4 + warp - kUnpackWarp0 : 0);
    bool go = true;
    int owed = 0;  // the first tile whose epilogue these warps still owe
    // the packed stage that is read next; the stage of unpacked blocks that this group writes next
    uint32_t stage = 0, parity_p = 0, slot = (uint32_t)odd, parity = 1;
    const uint32_t tmem_a = tmem + T::kA0 + (uint32_t)half * (kBK / 2) + lane_base;
    for (int i = 0; i < ntiles && go; ++i) {
      const int kb0 = kb_first(i), kbs = kb_count(i), quads = (kbs + kQuad - 1) / kQuad;
      int64_t row = 0;
      uint32_t shift = 0;  // bits that a row's codes begin into a word
      if constexpr (kPath != kBulk) {
        // rows past the end are read as the last one, or as what is behind it, and not stored
        const int t = tile_of(i);
        const int64_t in_tile = (int64_t)(t % p.tiles_o) * p.tile_rows + row_in_tile;
        row = (int64_t)p.plan.chunks[t / p.tiles_o].expert * p.rows;
        if (kPath != kDirect)
          shift = (uint32_t)((row + in_tile) * code_cols & 3) * 8;
        else
          row += min(in_tile, p.rows - 1);
      }
      int kb = odd;
      for (int quad = 0; quad < quads && go; ++quad) {
        Finish f;
        if (T::kHelp && quad == 0 && i > 0) {
          if (i == 1) pdl_wait_primary();
          f = prepare(i - 1, 1 + group);
        }
        uint32_t code[2] = {0u, 0u};
        const uint32_t from = src + stage * (kHalves * kHalfBytes);
        if constexpr (kPath != kDirect) {
          if (!mbar_wait_unpack(&packed_full[stage], parity_p, parity_p != 0)) {
            go = false;
            break;
          }
          const uint32_t at = code_src + stage * (kHalves * kHalfCodes) + row_in_half * (kPath == kBulk ? 16u : kCodeRow);
          uint32_t c[4];
          if constexpr (kPath == kBulk) {
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3]) : "r"(at));
            code[0] = odd ? c[1] : c[0], code[1] = odd ? c[3] : c[2];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(c[e]) : "r"(at + 4 * (odd + e)));
            code[0] = __funnelshift_r(c[0], c[1], shift), code[1] = __funnelshift_r(c[2], c[3], shift);
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (kb >= kbs || !go) break;
          uint32_t q[8];
          if constexpr (kPath != kDirect) {
            read_packed(q, from, row_in_half, kBM, 2 * (odd + 2 * u), kPath == kPairs);
          } else {
            // blocks past the end of K are zeros; so is the slots' tile there
            const uint8_t *wp = w.packed + row * half_cols + ((int64_t)(kb0 + kb) << 5);
            const uint8_t* cp = w.codes + row * code_cols + ((int64_t)(kb0 + kb) << 2);
            uint32_t c[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              c[e] = q[2 * e] = q[2 * e + 1] = 0u;
              const bool on = (int64_t)(kb0 + kb) * kBK + 16 * e < cols;
              ld_8_ahead(on, wp + 8 * e, q[2 * e], q[2 * e + 1]);
              ld_1_ahead(on, cp + e, c[e]);
            }
            code[u] = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
          }
          if (!mbar_wait_unpack(&empty[slot], parity)) {
            go = false;
            break;
          }
          tc_fence_after_sync();
          const uint32_t dst = tmem_a + slot * T::kAStage;
          uint32_t ca, cb;
          codes_f16(code[u], ca, cb);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[16];
#pragma unroll
            for (int e = 0; e < 4; ++e) unpack_f16(q[4 * h + e], __byte_perm(h ? cb : ca, 0u, (e & 2) ? 0x3232 : 0x1010), r + 4 * e);
            tmem_st_32x32b_x16(dst + 16 * h, r);
          }
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[slot]);
          // this group's next block, two further, or in the next tile
          const int ahead = kb + 2 < kbs ? 2 : kbs - kb + odd;
          kb += 2;
          slot += (uint32_t)ahead;
          while (slot >= kStages) slot -= kStages, parity ^= 1u;
        }
        if (kPath != kDirect && go) {
          // only now have the loads' values been used: an arrival does not wait for loads still under way (one right behind
          // them had TMA overwrite rows that were being read)
          __syncwarp();
          if (lane == 0) mbar_arrive(&packed_empty[stage]);
          if (++stage == kPackedStages) stage = 0, parity_p ^= 1u;
        }
        // the tile before, once this one's first blocks are there for the MMAs
        if (T::kHelp && quad == 0 && i > 0) finish(owed++, 1 + group, turn, f);
      }
      if (odd >= kbs) {  // a tile of one block has none for the odd groups
        slot += (uint32_t)kbs;
        while (slot >= kStages) slot -= kStages, parity ^= 1u;
      }
    }
    if constexpr (T::kHelp) {
      // the last tile; after a wait that ran out every tile that is left, as NaN
      have = have && go;
      pdl_wait_primary();
#pragma unroll 1
      for (; owed < ntiles; ++owed) finish(owed, 1 + group, turn, prepare(owed, 1 + group));
    }
    if ((!go || !have) && lane == 0) atomicOr(failed, 1u);
  } else if (p.path != kDirect && (warp == kWeightsWarp0 || p.path != kBulk)) {
    // the packed weights.  In small tiles an expert's only chunk reads them, once; in large ones others read them again,
    // from L2
    const int half = warp - kWeightsWarp0;  // whose copies are this warp's
    const ExpertMatrix& w = half ? p.b : p.a;
    const bool loads = p.path >= kMixed && half == 0, copies = p.path != kBulk;
    uint64_t policy;
    if constexpr (kN <= 32)
      policy = l2_evict_first_policy();
    else
      asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      const int t = tile_of(i), quad0 = kb_first(i) / kQuad, quads = quad0 + (kb_count(i) + kQuad - 1) / kQuad;
      const int64_t row_a = (int64_t)p.plan.chunks[t / p.tiles_o].expert * p.rows + (int64_t)(t % p.tiles_o) * p.tile_rows;
      const int64_t row_b = row_a + (kMode == kModeDown ? kBM : 0), row = half ? row_b : row_a;
      for (int quad = quad0; quad < quads; ++quad) {
        if (!mbar_wait_warp(&packed_empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        uint8_t *to = packed + s * (kHalves * kHalfBytes), *codes_to = packed_codes + s * (kHalves * kHalfCodes);
        if (loads && elect_one()) {
          if (kPath == kPairs) {
            // the even rows of each half, then the odd ones, which begin row_bytes further
            const int x = quad * (int)kRowBytes, odd_x = (int)(p.cols >> 1) - 8 + x;
            mbar_arrive_expect_tx(&packed_full[s], kHalves * kBM * kPairRow);
            tma_load_2d(to, &amap, x, (int)(row_a >> 1), &packed_full[s], policy);
            tma_load_2d(to + kHalfBytes / 2, &amap, odd_x, (int)(row_a >> 1), &packed_full[s], policy);
            tma_load_2d(to + kHalfBytes, &bmap, x, (int)(row_b >> 1), &packed_full[s], policy);
            tma_load_2d(to + kHalfBytes + kHalfBytes / 2, &bmap, odd_x, (int)(row_b >> 1), &packed_full[s], policy);
          } else {
            mbar_arrive_expect_tx(&packed_full[s], kHalves * kBM * (kRowBytes + (p.path == kBulk ? 16 : 0)));
            tma_load_2d(to, &amap, quad * (int)kRowBytes, (int)row_a, &packed_full[s], policy);
            tma_load_2d(to + kHalfBytes, &bmap, quad * (int)kRowBytes, (int)row_b, &packed_full[s], policy);
          }
          if (p.path == kBulk) {
            tma_load_2d(codes_to, &acodes, quad * 16, (int)row_a, &packed_full[s], policy);
            tma_load_2d(codes_to + kHalfCodes, &bcodes, quad * 16, (int)row_b, &packed_full[s], policy);
          }
        }
        __syncwarp();
        if (copies) {
          if (p.path == kCopies)
            copy_packed<kBM>(w.packed, p.cols >> 1, p.all_rows, row, (int64_t)quad * kRowBytes, smem_addr(to + half * kHalfBytes), 0, lane);
          copy_codes<kBM>(w.codes, p.cols >> 4, p.all_rows, row, (int64_t)quad * 16, smem_addr(codes_to + half * kHalfCodes), 0, lane);
          copies_arrive(smem_addr(&packed_full[s]));
        }
        if (++s == kPackedStages) s = 0, parity ^= 1u;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    ring_drain(packed_full, kPackedStages, s, parity);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
  if (threadIdx.x == 0 && *failed) atomicOr(&g_experts_flags, kErrMbarTimeout);
}

cudaError_t slots_map(CUtensorMap* map, const void* v, int64_t cols, int64_t rows, int width) {
  EncodeTiledFn encode = nullptr;
  const cudaError_t err = encode_tiled_fn(&encode);
  if (err != cudaSuccess) return err;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)cols * 2};
  const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)width};
  const cuuint32_t estr[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(v), dims, strides, box, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

template <int kMode, int kN>
cudaError_t launch_gemm_n(const void* v, int64_t slots, int64_t experts, GemmArgs p, int64_t most_tiles, int sms, cudaStream_t stream) {
  CUtensorMap map;
  cudaError_t err = slots_map(&map, v, p.cols, slots, kN);
  if (err != cudaSuccess) return err;
  p.all_rows = experts * p.rows;
  p.path = packed_path(p.a, p.b, p.cols, p.all_rows);
  CUtensorMap maps[4] = {map, map, map, map};
  if (p.path >= kMixed) {
    const bool pairs = p.path == kPairs;
    const int64_t bytes = pairs ? p.cols : p.cols / 2, rows = pairs ? p.all_rows / 2 : p.all_rows;
    const uint32_t width = pairs ? kPairRow : kRowBytes, height = pairs ? kBM / 2 : kBM;
    if ((err = bytes_map(&maps[0], p.a.packed, bytes, rows, width, height)) != cudaSuccess) return err;
    if ((err = bytes_map(&maps[1], p.b.packed, bytes, rows, width, height)) != cudaSuccess) return err;
  }
  if (p.path == kBulk) {
    if ((err = bytes_map(&maps[2], p.a.codes, p.cols / 16, p.all_rows, 16, kBM)) != cudaSuccess) return err;
    if ((err = bytes_map(&maps[3], p.b.codes, p.cols / 16, p.all_rows, 16, kBM)) != cudaSuccess) return err;
  }
  const auto launch = [&](auto kernel) {
    const cudaError_t set = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)Tile<kN>::kSmemBytes);
    if (set != cudaSuccess) return set;
    return launch_chained(kernel, dim3((unsigned)std::min<int64_t>(most_tiles, sms)), kThreads, (int)Tile<kN>::kSmemBytes, stream, map,
                          maps[0], maps[1], maps[2], maps[3], p);
  };
  switch (p.path) {
    case kBulk: return launch(gemm_kernel<kMode, kN, kBulk>);
    case kPairs: return launch(gemm_kernel<kMode, kN, kPairs>);
    case kDirect: return launch(gemm_kernel<kMode, kN, kDirect>);
    default: return launch(gemm_kernel<kMode, kN, kMixed>);
  }
}
template <int kMode>
cudaError_t launch_gemm(int width, const void* v, int64_t slots, int64_t experts, GemmArgs p, int64_t chunks, int sms,
                        cudaStream_t stream) {
  p.tile_rows = kMode == kModeDown ? 2 * kBM : kBM;
  p.tiles_o = (int32_t)((p.rows + p.tile_rows - 1) / p.tile_rows);
  p.kb_total = (int32_t)((p.cols + kBK - 1) / kBK);
  const int wanted = kMode == kModeRaw ? gate_up_segments(p.cols) : 1;
  p.kb_segment = ((p.kb_total + wanted - 1) / wanted + kQuad - 1) / kQuad * kQuad;
  p.segments = (p.kb_total + p.kb_segment - 1) / p.kb_segment;
  const int64_t tiles = chunks * p.tiles_o;
  if (tiles * p.kb_total > INT32_MAX) return cudaErrorInvalidValue;
  switch (width) {
    case 16: return launch_gemm_n<kMode, 16>(v, slots, experts, p, tiles, sms, stream);
    case 32: return launch_gemm_n<kMode, 32>(v, slots, experts, p, tiles, sms, stream);
    case 64: return launch_gemm_n<kMode, 64>(v, slots, experts, p, tiles, sms, stream);
    default: return launch_gemm_n<kMode, 128>(v, slots, experts, p, tiles, sms, stream);
  }
}

inline int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

// Bytes [rows, bytes] in boxes of `width` x `height`.
cudaError_t bytes_map(CUtensorMap* map, const void* v, int64_t bytes, int64_t rows, uint32_t width, uint32_t height) {
  EncodeTiledFn encode = nullptr;
  const cudaError_t err = encode_tiled_fn(&encode);
  if (err != cudaSuccess) return err;
  const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)bytes};
  const cuuint32_t box[2] = {width, height};
  const cuuint32_t estr[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(v), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                width == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

// Slots a tile: as many as an expert has on average, so that a tile's weights serve them all.  Measured on both sides, 32 experts
// of 4096 x 2048, as many slots each (and, behind the stroke, uneven ones as routers give), us:
//   slots    16 wide     32 wide     64 wide    128 wide
//     10    118 / 118   120 / 118   122 / 123   126 / 129
//     16    132 / 134   120 / 120   122 / 124   128 / 129
//     24    173 / 172   124 / 137   128 / 126   131 / 134
//     32    211 / 209   139 / 137   134 / 128   136 / 140
//     56                183 / 201   138 / 153   147 / 151
//     72                247 / 244   183 / 182   159 / 157
int experts_width(int64_t slots, int64_t experts) {
  const int64_t each = (slots + experts - 1) / experts;
  return each <= 10 ? 16 : each <= 24 ? 32 : each <= 56 ? 64 : 128;
}

static int64_t plan_runs(int64_t slots) { return (slots + kPlanSlots - 1) / kPlanSlots; }

int64_t experts_plan_bytes(int64_t slots, int64_t experts) {
  return 256 + 2 * round256(plan_chunks(slots, experts, 16) * (int64_t)sizeof(Chunk)) + 2 * round256(slots * 4) +
         round256(plan_runs(slots) * experts * 4);
}

Plan experts_plan_at(void* workspace, int64_t slots, int64_t experts) {
  uint8_t* p = static_cast<uint8_t*>(workspace);
  Plan plan;
  plan.header = reinterpret_cast<int32_t*>(p);
  plan.chunks = reinterpret_cast<Chunk*>(p + 256);
  p += 256 + 2 * round256(plan_chunks(slots, experts, 16) * (int64_t)sizeof(Chunk));
  plan.slot_of = reinterpret_cast<int32_t*>(p);
  plan.pos_of = reinterpret_cast<int32_t*>(p + round256(slots * 4));
  return plan;
}

Plan experts_wide_plan(const Plan& plan, int64_t slots, int64_t experts) {
  Plan wide = plan;
  wide.header = plan.header + 2;
  wide.chunks = reinterpret_cast<Chunk*>(reinterpret_cast<uint8_t*>(plan.chunks) +
                                         round256(plan_chunks(slots, experts, 16) * (int64_t)sizeof(Chunk)));
  return wide;
}

cudaError_t launch_experts_plan(const Routing& r, int64_t experts, int width, const Plan& plan, int wide_width, const Plan* wide,
                                cudaStream_t stream) {
  const int smem = (int)((kPlanWarps + 1) * experts * 4);
  // set once, for every call's size
  const cudaError_t err = ensure_dynamic_smem(reinterpret_cast<const void*>(plan_kernel), (kPlanWarps + 1) * (int)kRouteExperts * 4);
  if (err != cudaSuccess) return err;
  const int64_t slots = r.tokens * r.k, runs = plan_runs(slots);
  const Plan none = {}, &second = wide != nullptr ? *wide : none;
  if (runs == 1) {
    plan_kernel<<<1, kPlanThreads, smem, stream>>>(r.ids, slots, (int)experts, width, plan, wide_width, second, nullptr);
    return cudaGetLastError();
  }
  int32_t* counts = plan.pos_of + round256(slots * 4) / 4;
  count_kernel<<<(unsigned)runs, kPlanThreads, 0, stream>>>(r.ids, slots, (int)experts, counts);
  if (const cudaError_t count = cudaGetLastError(); count != cudaSuccess) return count;
  return launch_chained(plan_kernel, dim3((unsigned)runs), kPlanThreads, smem, stream, r.ids, slots, (int)experts, width, plan, wide_width,
                        second, static_cast<const int32_t*>(counts));
}

cudaError_t launch_experts_spread(const void* x, int64_t ld, void* out, uint32_t* amax, const void* dy, int64_t ld_dy, void* dy_out,
                                  uint32_t* dy_amax, int64_t n, const Routing& r, const Plan& plan, uint32_t* h_amax, float* weight_of,
                                  cudaStream_t stream) {
  const Spread first = {static_cast<const uint4*>(x), ld / 8, static_cast<uint4*>(out), amax};
  const Spread second = {static_cast<const uint4*>(dy), ld_dy / 8, static_cast<uint4*>(dy_out), dy_amax};
  return launch_chained(spread_kernel, dim3((unsigned)r.tokens, dy != nullptr ? 2 : 1), 256, 0, stream, first, second, n / 8, r.k, plan,
                        h_amax, r.weights, weight_of);
}

// h: [positions, parts, cols] of fp16, groups: [positions, level_groups(cols)]
cudaError_t launch_experts_level(void* h, int64_t slots, int64_t cols, int parts, const Plan& plan, const uint32_t* amax, const int8_t* groups,
                                 cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int64_t pieces = parts * (cols / 8), blocks = std::min<int64_t>(8 * info.sm_count, (slots * pieces + 255) / 256);
  return launch_chained(level_kernel, dim3((unsigned)blocks), 256, 0, stream, static_cast<uint4*>(h), pieces, cols / 8, plan, amax, groups);
}

cudaError_t launch_experts_combine(const float* part, const float* more, const Routing& r, const float* weights, const Plan& plan, int64_t n,
                                   void* out, int64_t ld, const float* dots, int parts, float* dweights, cudaStream_t stream) {
  const Combine c = {part, more, weights, static_cast<__nv_bfloat16*>(out), n, ld, r.tokens, r.k, dots, parts, dweights};
  const int64_t threads = (out != nullptr ? r.tokens * (n / 4) : 0) + (dots != nullptr ? r.tokens * r.k : 0);
  return launch_chained(combine_kernel, dim3((unsigned)((threads + 255) / 256)), 256, 0, stream, c, plan);
}

cudaError_t launch_experts_raw(const void* xs, const uint32_t* amax, int64_t slots, const Experts& w, const Plan& plan, int width,
                               float* raw, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  GemmArgs p = {};
  p.a = w.gate, p.b = w.up, p.rows = w.inner, p.cols = w.n, p.activation = w.activation, p.plan = plan, p.amax = amax, p.out = raw;
  return launch_gemm<kModeRaw>(width, xs, slots, w.count, p, plan_chunks(slots, w.count, width), info.sm_count, stream);
}

int64_t experts_workspace(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  const int64_t slots = tokens * k;
  return experts_plan_bytes(slots, experts) + 2 * round256(slots * 4) + round256(slots * n * 2) + round256(slots * inner * 2) +
         round256(slots * n * 4) + round256(slots * level_groups(inner));
}

cudaError_t launch_experts(const void* x, int64_t ld_x, const Routing& r, const Experts& w, void* y, int64_t ld_y, void* workspace,
                           cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int64_t slots = r.tokens * r.k;
  const int width = experts_width(slots, w.count);
  const Plan plan = experts_plan_at(workspace, slots, w.count);
  uint8_t* at = static_cast<uint8_t*>(workspace) + experts_plan_bytes(slots, w.count);
  uint32_t* amax = reinterpret_cast<uint32_t*>(at);
  uint32_t* h_amax = reinterpret_cast<uint32_t*>(at + round256(slots * 4));
  uint8_t* xs = at + 2 * round256(slots * 4);
  uint8_t* h = xs + round256(slots * w.n * 2);
  float* part = reinterpret_cast<float*>(h + round256(slots * w.inner * 2));
  int8_t* groups = reinterpret_cast<int8_t*>(part) + round256(slots * w.n * 4);
  const int64_t chunks = plan_chunks(slots, w.count, width);
  if ((err = launch_experts_plan(r, w.count, width, plan, width, nullptr, stream)) != cudaSuccess) return err;
  if ((err = launch_experts_spread(x, ld_x, xs, amax, nullptr, 0, nullptr, nullptr, w.n, r, plan, h_amax, nullptr, stream)) != cudaSuccess) return err;
  GemmArgs p = {};
  p.a = w.gate, p.b = w.up, p.rows = w.inner, p.cols = w.n, p.activation = w.activation, p.plan = plan;
  p.amax = amax, p.h_amax = h_amax, p.h_groups = groups, p.out = h;
  if ((err = launch_gemm<kModeHidden>(width, xs, slots, w.count, p, chunks, info.sm_count, stream)) != cudaSuccess) return err;
  if ((err = launch_experts_level(h, slots, w.inner, 1, plan, h_amax, groups, stream)) != cudaSuccess) return err;
  p.a = p.b = w.down, p.rows = w.n, p.cols = w.inner, p.amax = h_amax, p.out = part;
  if ((err = launch_gemm<kModeDown>(width, h, slots, w.count, p, chunks, info.sm_count, stream)) != cudaSuccess) return err;
  return launch_experts_combine(part, nullptr, r, r.weights, plan, w.n, y, ld_y, nullptr, 0, nullptr, stream);
}

cudaError_t read_experts_device_error(uint32_t* flags) {
  uint32_t v = 0;
  cudaError_t err = cudaMemcpyFromSymbol(&v, g_experts_flags, sizeof v);
  if (err != cudaSuccess) return err;
  *flags = v;
  if (v) {
    const uint32_t zero = 0;
    err = cudaMemcpyToSymbol(g_experts_flags, &zero, sizeof zero);
  }
  return err;
}

}  // namespace hscale
