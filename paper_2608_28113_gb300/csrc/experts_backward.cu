// experts_backward.cu -- the gradients of a layer of experts with packed NVFP4 weights:
//   dh = D_e^T dy_t,  dw = h . dh,  dx_t = sum_j w_tj (G_e^T (dh u act'(g)) + U_e^T (dh act(g)))
// The slots are grouped as in the forward pass (experts.cu), x and dy laid out in that order in fp16, and g and u made again
// in fp32.  Two products by transposed weights follow: the first (K = n) makes dh and, as it leaves tensor memory, dw's
// partial sums and the two factors of dx, with G's and U's global scales in them, in fp16 (experts.cuh); the second (K =
// G's rows, then U's) makes each slot's part of dx in fp32; a token's slots are added up in order and rounded once.
//
// The transposed products.  Tile: 256 outputs (columns of the weights) as two halves of 128 x up to kN slots, K in blocks
// of 64 rows.  The packed rows, unpacked as they are stored, make the weights' tile MN-major in shared memory
// (tensor memory would take it K-major only).  24 warps, as in the forward pass: TMA loads of the slots' tile, MMAs,
// four of the epilogue, two groups of eight that unpack every other K block (a thread: 64 outputs of a row of
// K), and two that fetch the packed blocks.
// Bound by shared memory, which carries both operands, the packed blocks and the unpacking: of 128 bytes a
// cycle, a K block takes some 1010 cycles at 128 slots against 512 of MMAs, and 1416 at 256 against 1024; so an expert
// with enough slots takes 256 a tile, and the unpacking warps then take part in its epilogue.  4096 slots of 8 experts,
// 4096 x 14336: g and u 803 us, first product 745, second 797 (1.21 PFLOP/s).  Segments of K (experts.cuh) are 200 us
// of the first and 200 of g and u: a segment more is an epilogue more, of 65536 numbers a tile at some 45 instructions
// each in the last one, and at this width there is no second accumulator to go on with.  The factors under their row's power
// of two: 74 us.
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

__device__ uint32_t g_experts_backward_flags = 0;

constexpr int kBM = 128, kBK = 64, kHalves = 2;
constexpr int kEpilogueWarp0 = 2, kUnpackWarp0 = 6, kUnpackWarps = 16, kWeightsWarp0 = 22;
constexpr int kThreads = 768;
constexpr int kModeHidden = 0, kModeInput = 1;
constexpr uint32_t kGroupBytes = 64 * kBK * 2;  // 64 outputs x 64 rows of K
constexpr uint32_t kHalfBytes = 2 * kGroupBytes;
// A packed block: 64 rows of K, 128 bytes (256 outputs) each, and 16 bytes of their codes (20 where they are copied
// as whole words from any address).
constexpr uint32_t kRowBytes = kPackedRow;
static_assert(kRowBytes == kHalves * kBM / 2, "a packed stage's rows");
constexpr uint32_t kPackedBytes = kBK * kPairRow, kCodeBytes = kBK * kCodeRow;

template <int kN>
struct Tile {
  static constexpr int kStages = kN == 256 ? 2 : kN == 128 ? 3 : 4;
  static constexpr int kPackedStages = 6;
  static constexpr int kAccs = kN == 256 ? 1 : 2;
  static constexpr bool kHelp = kAccs == 1;  // the unpacking warps take part in the epilogue
  static constexpr int kEpilogueWarps = kHelp ? 4 + kUnpackWarps : 4;
  static constexpr uint32_t kABytes = kHalves * kHalfBytes, kBBytes = kN * kBK * 2;
  static constexpr uint32_t kTurnBytes = kEpilogueWarps * 512;
  static constexpr uint32_t kSmemBytes = kStages * (kABytes + kBBytes) + kPackedStages * (kPackedBytes + kCodeBytes) + 1024 /* alignment */ +
                                         512 /* barriers */ + kTurnBytes;
  static constexpr uint32_t kAcc = kHalves * kN, kTmemCols = kAccs * kAcc;
  static_assert(kSmemBytes <= 232448, "shared memory");
};

struct BackArgs {
  ExpertMatrix a, b;    // the weights of the first and the second half of K (down twice where there is one)
  int64_t rows, cols;   // of an expert's matrix: K and the outputs
  int32_t kb_part, parts, tiles_o, path;
  int32_t segments, kb_segment;  // of kModeHidden: K's segments, and their K blocks (the last has fewer)
  float* held;       // [positions, cols]: dh of the segments before
  int32_t splits;    // 2: the halves of K are tiles of their own, into part and more
  int64_t all_rows;  // of all experts
  int32_t activation;
  Plan plan;
  const float* weight_of;    // of each position
  const uint32_t* amax;      // of each position's dy, or of its factors
  const float2* raw;         // g and u, [positions, cols]
  const float *gate_scale, *up_scale;
  uint16_t* factors;         // fp16 [positions, 2, cols], or nullptr
  int8_t* groups;            // [positions, level_groups(cols)] powers of two of the factors, and the rows' amax
  uint32_t* factor_amax;
  float* dots;               // [8 tiles_o, slots] partial sums of h . dh, or nullptr
  int64_t slots;
  float *part, *more;        // [slots, cols]
};

// Eight columns' sums over a warp's lanes: every lane has that of column_of(lane).
__device__ __forceinline__ float sum_columns(float (&v)[8], int lane) {
#pragma unroll
  for (int n = 4, d = 16; n > 0; n >>= 1, d >>= 1) {
    const bool upper = (lane & d) != 0;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float send = upper ? v[j] : v[j + n], keep = upper ? v[j + n] : v[j];
      v[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, d);
    }
  }
  v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], 2);
  return v[0] + __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
}
__device__ __forceinline__ int column_of(int lane) { return lane >> 2; }

// Eight slots of 32 outputs (a slot's in neighbouring lanes) times the power of two in lane j, rounded to fp16 and stored,
// 8 outputs of a slot a lane.
__device__ __forceinline__ void store_rows(const float (&v)[8], float down, uint32_t* turn, uint16_t* out, int64_t stride, int64_t at0,
                                           int64_t cols, int left, int lane) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j)
    turn[j * 32 + lane] = pack_f16(v[2 * j] * __shfl_sync(0xFFFFFFFFu, down, 2 * j), v[2 * j + 1] * __shfl_sync(0xFFFFFFFFu, down, 2 * j + 1));
  __syncwarp();
  const int odd = lane >> 4, j = 2 * ((lane >> 2) & 3) + odd;
  const uint4 q0 = reinterpret_cast<const uint4*>(turn)[2 * (lane & 15)], q1 = reinterpret_cast<const uint4*>(turn)[2 * (lane & 15) + 1];
  const uint32_t pick = odd ? 0x7632u : 0x5410u;
  const uint4 r = make_uint4(__byte_perm(q0.x, q0.y, pick), __byte_perm(q0.z, q0.w, pick), __byte_perm(q1.x, q1.y, pick),
                             __byte_perm(q1.z, q1.w, pick));
  const int64_t at = at0 + (lane & 3) * 8;
  // cols is a multiple of 16: 8 outputs are all there or none is
  if (j < left && at < cols) *reinterpret_cast<uint4*>(out + j * stride + at) = r;
}

__device__ __forceinline__ void tmem_ld_32x32b_x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}

template <int kMode, int kN, bool kPairRows>
__global__ void __launch_bounds__(kThreads, 1)
back_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap amap, const __grid_constant__ CUtensorMap bmap,
            const __grid_constant__ CUtensorMap acodes, const __grid_constant__ CUtensorMap bcodes, const __grid_constant__ BackArgs p) {
  using T = Tile<kN>;
  constexpr int kStages = T::kStages, kPackedStages = T::kPackedStages, kAccs = T::kAccs;
  extern __shared__ __align__(16) uint8_t dynamic_smem[];
  uint8_t* smem = dynamic_smem + ((1024u - (smem_addr(dynamic_smem) & 1023u)) & 1023u);
  uint8_t* tile_a = smem;
  uint8_t* tile_b = smem + kStages * T::kABytes;
  uint8_t* packed = tile_b + kStages * T::kBBytes;
  uint8_t* packed_codes = packed + kPackedStages * kPackedBytes;
  uint8_t* rest = packed_codes + kPackedStages * kCodeBytes;
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
      mbar_init(&full[s], 1 + kUnpackWarps / 2);  // the TMA load and the warps of a group
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kPackedStages; ++s) {
      mbar_init(&packed_full[s], (p.path == kBulk ? 0 : 2 * 32) + (p.path >= kMixed ? 1 : 0));
      mbar_init(&packed_empty[s], kUnpackWarps / 2);
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
    tmem_alloc(smem_addr(tmem_slot), T::kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  // The plan is there: the kernel that this one may run beside has waited for it.  What that kernel writes (the slots'
  // tile, g and u) is waited for where it is read; the weights begin to come meanwhile.

  const int tiles = p.plan.header[0] * p.tiles_o * p.splits, step = (int)gridDim.x, first = (int)blockIdx.x;
  // in kModeHidden a tile's segments of K are tiles one after another (hidden_segments)
  const int segments = kMode == kModeHidden ? p.segments : 1;
  const int ntiles = tiles > first ? (tiles - first + step - 1) / step * segments : 0;
  const int kb_all = p.kb_part * p.parts / p.splits;
  const auto kb_first = [&](int i) { return kMode == kModeHidden ? i % segments * p.kb_segment : 0; };
  const auto kb_count = [&](int i) { return kMode == kModeHidden ? min(p.kb_segment, kb_all - kb_first(i)) : kb_all; };
  // the CTA's tile i: split, chunk, outputs
  struct Where {
    int split, chunk, to;
  };
  const auto where = [&](int i) {
    const int t = first + (kMode == kModeHidden ? i / segments : i) * step, u = t / p.splits;
    return Where{t - u * p.splits, u / p.tiles_o, u % p.tiles_o};
  };
  const uint32_t quarter = (uint32_t)(warp & 3), lane_base = (quarter * 32u) << 16;
  bool have = true;  // of the warps of the epilogue: no wait for an accumulator has run out

  // the next tile's MMAs need not wait for what is done with a warp's last columns
  const auto release = [&](uint32_t acc) {
    tc_fence_before_sync();
    __syncwarp();
    // a warp that writes NaN runs ahead of the others: its arrivals would stand for theirs, and the next tile's MMAs overwrite
    // what they still read
    if (lane == 0 && have) mbar_arrive(&acc_empty[acc]);
  };
  // The epilogue of the CTA's tile i: eight slots of a half a time, those of this warp.
  const auto finish = [&](int i, int who, uint32_t* turn) {
    constexpr int kWorkers = T::kEpilogueWarps / 4;
    const Where at = where(i);
    const int to = at.to;
    const Chunk c = p.plan.chunks[at.chunk];
    const uint32_t acc = (uint32_t)i % kAccs, d = tmem + acc * T::kAcc + lane_base;
    const float scale = kMode == kModeHidden ? p.a.scale[c.expert] : 1.0f;
    const float sg = kMode == kModeHidden ? p.gate_scale[c.expert] : 0.0f, su = kMode == kModeHidden ? p.up_scale[c.expert] : 0.0f;
    const float nan = __int_as_float(0x7FC00000);
    const int each = (c.count + 7) / 8, pieces = kHalves * each;
    const int segment = kMode == kModeHidden ? i % segments : 0;
    const bool last = segment == segments - 1;
    float g[8], u[8];
    const auto fetch = [&](int piece) {
      if (kMode != kModeHidden || piece >= pieces || !last) return;
      const int half = piece >= each ? 1 : 0, j0 = (piece - half * each) * 8;
      const int64_t o = (int64_t)to * (kHalves * kBM) + half * kBM + quarter * 32 + lane;
      const float2* raw = p.raw + (int64_t)(c.first + j0) * p.cols + o;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 v = j0 + j < c.count && o < p.cols ? *raw : make_float2(0.0f, 0.0f);
        g[j] = v.x, u[j] = v.y;
        raw += p.cols;
      }
    };
    fetch(who);
    if (have) have = __all_sync(0xFFFFFFFFu, mbar_wait_acc(&acc_full[acc], (uint32_t)(i / kAccs) & 1u));
    tc_fence_after_sync();
#pragma unroll 1
    for (int piece = who; piece < pieces; piece += kWorkers) {
      const int half = piece >= each ? 1 : 0, j0 = (piece - half * each) * 8, left = min(8, c.count - j0);
      const int64_t at0 = (int64_t)to * (kHalves * kBM) + half * kBM + quarter * 32, o = at0 + lane, pos = c.first + j0;
      const bool on = o < p.cols;
      uint32_t a[8];
      tmem_ld_32x32b_x8(d + (uint32_t)(half * kN + j0), a);
      if (kMode == kModeHidden && segments > 1) {
        // the segment's dh to what the thread left there of those before
        float* held = p.held + pos * p.cols + o;
        float before[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) before[j] = segment > 0 && j < left && on ? held[j * p.cols] : 0.0f;
        const float my_up = !have ? nan : lane < left ? scale * exp2_int(row_exponent(p.amax[pos + lane])) : 0.0f;
        tmem_ld_wait();
        if (piece + kWorkers >= pieces) release(acc);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float dh = fmaf(__uint_as_float(a[j]), __shfl_sync(0xFFFFFFFFu, my_up, j), before[j]);
          if (last)
            a[j] = __float_as_uint(dh);
          else if (j < left && on)
            held[j * p.cols] = dh;
        }
        if (!last) continue;
      }
      if constexpr (kMode == kModeHidden) {
        // lane j: slot j's weight times G's and U's scales, and the power of two of its row of dy times D's
        const float my_w = lane < left ? p.weight_of[pos + lane] : 0.0f, my_g = my_w * sg, my_u = my_w * su;
        float my_up = 1.0f;
        if (segments == 1) {
          my_up = !have ? nan : lane < left ? scale * exp2_int(row_exponent(p.amax[pos + lane])) : 0.0f;
          tmem_ld_wait();
          if (piece + kWorkers >= pieces) release(acc);
        }
        float dot[8], dg[8], du[8];
        // (outputs past the end have g = u = 0, and are not stored)
        const auto factors = [&](auto kind) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float dh = __uint_as_float(a[j]) * __shfl_sync(0xFFFFFFFFu, my_up, j);
            const float2 act = activate<decltype(kind)::value>(g[j]);
            dot[j] = dh * (act.x * u[j]);
            dg[j] = dh * __shfl_sync(0xFFFFFFFFu, my_g, j) * (u[j] * act.y);
            du[j] = dh * __shfl_sync(0xFFFFFFFFu, my_u, j) * act.x;
          }
        };
        if (p.activation == kActSilu)
          factors(std::integral_constant<int, kActSilu>{});
        else
          factors(std::integral_constant<int, kActGeluTanh>{});
        fetch(piece + kWorkers);
        if (p.factors != nullptr) {
          uint32_t most = 0u;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint32_t m = max(__float_as_uint(dg[j]) & 0x7FFFFFFFu, __float_as_uint(du[j]) & 0x7FFFFFFFu);
            const uint32_t all = __reduce_max_sync(0xFFFFFFFFu, on ? m : 0u);
            if (lane == j) most = all >> 16;
          }
          const int e = row_exponent(most);
          if (lane < left && at0 < p.cols) {
            p.groups[(pos + lane) * level_groups(p.cols) + at0 / kLevel] = (int8_t)e;
            atomicMax(&p.factor_amax[pos + lane], most);
          }
          uint16_t* out = p.factors + pos * 2 * p.cols;
          store_rows(dg, exp2_int(-e), turn, out, 2 * p.cols, at0, p.cols, left, lane);
          store_rows(du, exp2_int(-e), turn, out + p.cols, 2 * p.cols, at0, p.cols, left, lane);
        }
        if (p.dots != nullptr) {
          const float s = sum_columns(dot, lane);
          const int j = column_of(lane);
          if ((lane & 3) == 0 && j < left) p.dots[((int64_t)(to * kHalves + half) * 4 + quarter) * p.slots + pos + j] = s;
        }
      } else {
        const float my_up = !have ? nan : lane < left ? exp2_int(row_exponent(p.amax[pos + lane])) : 0.0f;
        tmem_ld_wait();
        if (piece + kWorkers >= pieces) release(acc);
        float* out = (at.split ? p.more : p.part) + pos * p.cols + o;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float up = __shfl_sync(0xFFFFFFFFu, my_up, j);
          if (j < left && on) *out = __uint_as_float(a[j]) * up;
          out += p.cols;
        }
      }
    }
    if (who >= pieces) release(acc);
  };
  const auto turn_at = [&](int worker) { return reinterpret_cast<uint32_t*>(rest + 512 + worker * 512); };

  if (warp == 0) {
    pdl_wait_primary();
    pdl_launch_dependents();
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      const Where at = where(i);
      const Chunk c = p.plan.chunks[at.chunk];
      const int kb1 = kb_first(i) + kb_count(i);
      for (int kb = kb_first(i); kb < kb1; ++kb) {
        if (!mbar_wait_warp(&empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(&full[s], T::kBBytes);
          const int part = at.split || kb >= p.kb_part ? 1 : 0;
          tma_load_3d(tile_b + s * T::kBBytes, &vmap, (kb - (kb >= p.kb_part ? p.kb_part : 0)) * kBK, part, c.first, &full[s], policy);
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
      const Chunk c = p.plan.chunks[where(i).chunk];
      const int kbs = kb_count(i);
      const uint32_t slots = (uint32_t)((c.count + 15) & ~15);
      const uint32_t idesc = warp_uniform(idesc_f16_f32(kBM, slots) | 1u << 15);
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
#pragma unroll
          for (int half = 0; half < kHalves; ++half) {
            const uint64_t ad = smem_desc_mn_sw128(smem_addr(tile_a + s * T::kABytes + half * kHalfBytes), kGroupBytes);
#pragma unroll
            for (int kk = 0; kk < kBK / 16; ++kk)
              umma_bf16(d + half * kN, ad + 128 * kk, bd + 2 * kk, idesc, (uint32_t)(kb > 0 || kk > 0));
          }
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
    for (int i = 0; i < ntiles; ++i) finish(i, 0, turn_at(warp - kEpilogueWarp0));
    if (!have && lane == 0) atomicOr(failed, 1u);
  } else if (warp < kWeightsWarp0) {
    // group: every other K block; a thread: 64 outputs (`part64` of four) of one row of K
    const int group = (warp - kUnpackWarp0) >> 3, line = ((warp - kUnpackWarp0) & 7) * 32 + lane, row = line & 63, part64 = line >> 6;
    const int64_t cols = p.cols, half_cols = cols >> 1, code_cols = cols >> 4;
    const uint32_t swizzle = (uint32_t)row & 7u;  // of the unpacked tile
    uint32_t* turn = turn_at(T::kHelp ? 4 + warp - kUnpackWarp0 : 0);
    // after a wait that ran out: how far before the next tile the first one lies whose epilogue is owed
    int back = 0;
    // blocks of all tiles, one after another: this group's are group, group + 2, ...
    int kb = group;
    uint32_t block = (uint32_t)group;
    int i = 0;
    for (; i < ntiles && back == 0; kb -= kb_count(i), ++i) {
      const int kbs = kb_count(i), kb0 = kb_first(i);
      const Where at = where(i);
      const int64_t e = p.plan.chunks[at.chunk].expert, o0 = (int64_t)at.to * (kHalves * kBM) + part64 * 64;
      const int64_t row0 = e * p.rows + row;
      // bits that a row's codes begin into a word: the same for rows 64 apart
      const uint32_t shift = p.path != kDirect && p.path != kBulk ? (uint32_t)(row0 * code_cols & 3) * 8 : 0u;
      int done = 0;
      for (; kb < kbs && back == 0; kb += 2, block += 2) {
        const uint32_t ps = block % kPackedStages, parity_p = (block / kPackedStages) & 1u;
        uint32_t q[8], code;
        if (p.path != kDirect) {
          if (!mbar_wait_unpack(&packed_full[ps], parity_p, parity_p != 0)) {
            back = done == 0 ? 2 : 1;
            break;
          }
          read_packed(q, smem_addr(packed + ps * kPackedBytes), row, kBK, 2 * part64, kPairRows);
          const uint32_t code_at = smem_addr(packed_codes + ps * kCodeBytes) + row * (p.path == kBulk ? 16u : kCodeRow) + 4 * part64;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(code) : "r"(code_at));
          if (p.path != kBulk) {
            uint32_t more;
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(more) : "r"(code_at + 4));
            code = __funnelshift_r(code, more, shift);
          }
        } else {
          // rows past the end of K are read as the last one (the slots' tile is zeros there), outputs past the end are zeros, and not
          // stored
          const int part = at.split || kb >= p.kb_part ? 1 : 0;
          const int64_t f = e * p.rows + min((int64_t)(kb0 + kb - (kb >= p.kb_part ? p.kb_part : 0)) * kBK + row, p.rows - 1);
          const uint8_t *wp = (part ? p.b.packed : p.a.packed) + f * half_cols + (o0 >> 1),
                        *cp = (part ? p.b.codes : p.a.codes) + f * code_cols + (o0 >> 4);
          uint32_t c[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            c[h] = q[2 * h] = q[2 * h + 1] = 0u;
            ld_8_ahead(o0 + 16 * h < cols, wp + 8 * h, q[2 * h], q[2 * h + 1]);
            ld_1_ahead(o0 + 16 * h < cols, cp + h, c[h]);
          }
          code = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
        }
        const uint32_t s = block % kStages;
        if (!mbar_wait_unpack(&empty[s], ((block / kStages) & 1u) ^ 1u)) {
          back = done == 0 ? 2 : 1;
          break;
        }
        uint8_t* dst = tile_a + s * T::kABytes + part64 * kGroupBytes + row * 128;
        uint32_t ca, cb;
        codes_f16(code, ca, cb);
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          uint32_t r[4];
          const uint32_t scale = __byte_perm(h < 4 ? ca : cb, 0u, (h & 2) ? 0x3232 : 0x1010);
          unpack_f16(q[h], scale, r);
          *reinterpret_cast<uint4*>(dst + (((uint32_t)h ^ swizzle) << 4)) = make_uint4(r[0], r[1], r[2], r[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&full[s]);
          if (p.path != kDirect) mbar_arrive(&packed_empty[ps]);  // the loads' values have been used
        }
        // the tile before, once this one's first blocks are there for the MMAs
        if (T::kHelp && done == 0 && i == 1) pdl_wait_primary();
        if (T::kHelp && done++ == 0 && i > 0) finish(i - 1, 1 + ((warp - kUnpackWarp0) >> 2), turn);
      }
      // (a tile of one K block has none of this group's)
      if (T::kHelp && done == 0 && i == 1) pdl_wait_primary();
      if (T::kHelp && done == 0 && i > 0 && back == 0) finish(i - 1, 1 + ((warp - kUnpackWarp0) >> 2), turn);
    }
    if constexpr (T::kHelp) {
      // the last tile; after a wait that ran out all that are owed, as NaN
      have = have && back == 0;
      pdl_wait_primary();
#pragma unroll 1
      for (int j = max(0, back == 0 ? ntiles - 1 : i - back); j < ntiles; ++j) finish(j, 1 + ((warp - kUnpackWarp0) >> 2), turn);
    }
    if ((back != 0 || !have) && lane == 0) atomicOr(failed, 1u);
  } else if (p.path != kDirect && (warp == kWeightsWarp0 || p.path != kBulk)) {
    const int who = warp - kWeightsWarp0;  // whose copies are 32 of the 64 rows
    const bool loads = p.path >= kMixed && who == 0, copies = p.path != kBulk;
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      const Where at = where(i);
      const int to = at.to;
      const int64_t row0 = (int64_t)p.plan.chunks[at.chunk].expert * p.rows;
      const int kb1 = kb_first(i) + kb_count(i);
      for (int kb = kb_first(i); kb < kb1; ++kb) {
        if (!mbar_wait_warp(&packed_empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        const bool second = at.split || kb >= p.kb_part;
        const int64_t row = row0 + (int64_t)(kb - (kb >= p.kb_part ? p.kb_part : 0)) * kBK;
        uint8_t *packed_to = packed + s * kPackedBytes, *codes_to = packed_codes + s * kCodeBytes;
        if (loads && elect_one()) {
          const CUtensorMap* map = second ? &bmap : &amap;
          if (kPairRows) {
            // the even rows, then the odd ones, which begin row_bytes further
            mbar_arrive_expect_tx(&packed_full[s], kBK * kPairRow);
            tma_load_2d(packed_to, map, to * (int)kRowBytes, (int)(row >> 1), &packed_full[s], policy);
            tma_load_2d(packed_to + kPackedBytes / 2, map, (int)(p.cols >> 1) - 8 + to * (int)kRowBytes, (int)(row >> 1), &packed_full[s], policy);
          } else {
            mbar_arrive_expect_tx(&packed_full[s], kBK * (kRowBytes + (p.path == kBulk ? 16 : 0)));
            tma_load_2d(packed_to, map, to * (int)kRowBytes, (int)row, &packed_full[s], policy);
          }
          if (p.path == kBulk) tma_load_2d(codes_to, second ? &bcodes : &acodes, to * 16, (int)row, &packed_full[s], policy);
        }
        __syncwarp();
        if (copies) {
          const ExpertMatrix& w = second ? p.b : p.a;
          if (p.path == kCopies)
            copy_packed<32>(w.packed, p.cols >> 1, p.all_rows, row + 32 * who, (int64_t)to * kRowBytes, smem_addr(packed_to), 32 * who, lane);
          copy_codes<32>(w.codes, p.cols >> 4, p.all_rows, row + 32 * who, (int64_t)to * 16, smem_addr(codes_to), 32 * who, lane);
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
    tmem_dealloc(tmem, T::kTmemCols);
  }
  if (threadIdx.x == 0 && *failed) atomicOr(&g_experts_backward_flags, kErrMbarTimeout);
}

template <int kMode, int kN>
cudaError_t launch_back_n(const void* v, int64_t depth, int64_t experts, BackArgs p, int64_t most_tiles, int sms, cudaStream_t stream) {
  const int parts = p.parts;
  EncodeTiledFn encode = nullptr;
  cudaError_t err = encode_tiled_fn(&encode);
  if (err != cudaSuccess) return err;
  CUtensorMap map;
  const cuuint64_t dims[3] = {(cuuint64_t)depth, (cuuint64_t)parts, (cuuint64_t)p.slots};
  const cuuint64_t strides[2] = {(cuuint64_t)depth * 2, (cuuint64_t)(depth * parts * 2)};
  const cuuint32_t box[3] = {(cuuint32_t)kBK, 1, (cuuint32_t)kN};
  const cuuint32_t estr[3] = {1, 1, 1};
  if (encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(v), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  p.all_rows = experts * p.rows;
  p.path = packed_path(p.a, p.b, p.cols, p.all_rows);
  CUtensorMap maps[4] = {map, map, map, map};
  if (p.path >= kMixed) {
    const bool pairs = p.path == kPairs;
    const int64_t bytes = pairs ? p.cols : p.cols / 2, rows = pairs ? p.all_rows / 2 : p.all_rows;
    const uint32_t width = pairs ? kPairRow : kRowBytes, height = pairs ? kBK / 2 : kBK;
    if ((err = bytes_map(&maps[0], p.a.packed, bytes, rows, width, height)) != cudaSuccess) return err;
    if ((err = bytes_map(&maps[1], p.b.packed, bytes, rows, width, height)) != cudaSuccess) return err;
  }
  if (p.path == kBulk) {
    if ((err = bytes_map(&maps[2], p.a.codes, p.cols / 16, p.all_rows, 16, kBK)) != cudaSuccess) return err;
    if ((err = bytes_map(&maps[3], p.b.codes, p.cols / 16, p.all_rows, 16, kBK)) != cudaSuccess) return err;
  }
  const auto launch = [&](auto kernel) {
    const cudaError_t set = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)Tile<kN>::kSmemBytes);
    if (set != cudaSuccess) return set;
    return launch_chained(kernel, dim3((unsigned)std::min<int64_t>(most_tiles, sms)), kThreads, (int)Tile<kN>::kSmemBytes, stream, map,
                          maps[0], maps[1], maps[2], maps[3], p);
  };
  return p.path == kPairs ? launch(back_kernel<kMode, kN, true>) : launch(back_kernel<kMode, kN, false>);
}
// chunks: at most; expected: about how many there are
template <int kMode>
cudaError_t launch_back(int width, const void* v, int parts, int64_t experts, BackArgs& p, int64_t chunks, int64_t expected, int sms,
                        cudaStream_t stream) {
  p.parts = parts;
  p.kb_part = (int32_t)((p.rows + kBK - 1) / kBK);
  p.splits = 1;
  const int wanted = kMode == kModeHidden ? hidden_segments(p.rows) : 1;
  p.kb_segment = (p.kb_part + wanted - 1) / wanted;
  p.segments = (p.kb_part + p.kb_segment - 1) / p.kb_segment;
  p.tiles_o = (int32_t)((p.cols + kHalves * kBM - 1) / (kHalves * kBM));
  int64_t tiles = chunks * p.tiles_o;
  // G's and U's rows as tiles of their own where that fills the last round of tiles better (by more than the second
  // sum costs): 320 tiles of 256 x 256 x 28672 on 152 SMs, 973 us in three rounds, 797 as 640.  dx's bits go by the choice, since one
  // accumulator cuts its sums off elsewhere than two; tiles of their own always would cost up to a quarter of a call where inner
  // is short (4096 tokens on 8 of 64 experts, 8192 x 256: 1450 us, 1820), the two added in the tile's epilogue 1 to 9%
  if (parts == 2) {
    const int64_t likely = std::max<int64_t>(1, expected * p.tiles_o);
    const int64_t whole = 2 * ((likely + sms - 1) / sms), halves = (2 * likely + sms - 1) / sms;
    if (halves < whole) p.splits = 2, tiles *= 2;
  }
  if (tiles * p.kb_part * parts > INT32_MAX) return cudaErrorInvalidValue;
  switch (width) {
    case 32: return launch_back_n<kMode, 32>(v, p.rows, experts, p, tiles, sms, stream);
    case 64: return launch_back_n<kMode, 64>(v, p.rows, experts, p, tiles, sms, stream);
    case 128: return launch_back_n<kMode, 128>(v, p.rows, experts, p, tiles, sms, stream);
    default: return launch_back_n<kMode, 256>(v, p.rows, experts, p, tiles, sms, stream);
  }
}

inline int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }
// Slots a tile of the transposed products.  Measured as in experts_width, whole backward pass, us:
//   slots    32 wide     64 wide    128 wide    256 wide
//     24    251 / 295   259 / 278   261 / 303   326 / 350
//     32    326 / 323   280 / 295   295 / 324   336 / 347
//     56    416 / 443   341 / 402   351 / 385   379 / 396
//     72    528 / 525   444 / 445   400 / 420   423 / 446
//     96                517 / 536   465 / 517   465 / 538
//    144                759 / 753   696 / 665   587 / 628
//    176                821 / 829   767 / 747   647 / 646
// (At 128 to 144 slots 256 wide would be 6 to 16 % faster already.)
inline int back_width(int64_t slots, int64_t experts) {
  const int64_t each = (slots + experts - 1) / experts;
  return each <= 24 ? 32 : each <= 56 ? 64 : each <= 144 ? 128 : 256;
}
inline int64_t raw_bytes(int64_t slots, int64_t n, int64_t inner) { return round256(slots * std::max(8 * inner, 4 * n)); }
inline int64_t held_bytes(int64_t slots, int64_t n, int64_t inner) { return hidden_segments(n) > 1 ? round256(slots * inner * 4) : 0; }
inline int64_t dot_parts(int64_t inner) { return (inner + kHalves * kBM - 1) / (kHalves * kBM) * kHalves * 4; }

}  // namespace

int64_t experts_backward_workspace(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  const int64_t slots = tokens * k;
  // x and dy in order, whose place the slots' parts of dx take afterwards; g and u, whose place a second sum of them takes;
  // the factors; the dots; dh of K's segments before the last; the factors' amax, the slots' weights and
  // the factors' powers of two
  return experts_plan_bytes(slots, experts) + 2 * round256(slots * 4) + 2 * round256(slots * n * 2) + raw_bytes(slots, n, inner) + round256(slots * inner * 4) +
         round256(dot_parts(inner) * slots * 4) + held_bytes(slots, n, inner) + 2 * round256(slots * 4) +
         round256(slots * level_groups(inner));
}

cudaError_t launch_experts_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const Routing& r, const Experts& w,
                                    void* dx, int64_t ld_dx, float* dweights, void* workspace, cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int64_t slots = r.tokens * r.k;
  const int width = experts_width(slots, w.count), wide_width = back_width(slots, w.count);
  const Plan plan = experts_plan_at(workspace, slots, w.count);
  uint32_t* amax = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + experts_plan_bytes(slots, w.count));
  uint32_t* dy_amax = amax + round256(slots * 4) / 4;
  uint8_t* xs = reinterpret_cast<uint8_t*>(dy_amax) + round256(slots * 4);
  uint8_t* dys = xs + round256(slots * w.n * 2);
  uint8_t* raw = dys + round256(slots * w.n * 2);
  uint8_t* factors = raw + raw_bytes(slots, w.n, w.inner);
  uint8_t* dots = factors + round256(slots * w.inner * 4);
  uint8_t* held = dots + round256(dot_parts(w.inner) * slots * 4);
  uint32_t* factor_amax = reinterpret_cast<uint32_t*>(held + held_bytes(slots, w.n, w.inner));
  float* weight_of = reinterpret_cast<float*>(factor_amax) + round256(slots * 4) / 4;
  int8_t* groups = reinterpret_cast<int8_t*>(weight_of) + round256(slots * 4);
  const Plan wide = experts_wide_plan(plan, slots, w.count);
  const int64_t chunks = plan_chunks(slots, w.count, wide_width);
  const int64_t expected = slots / wide_width + std::min<int64_t>(slots, w.count) / 2;  // half a chunk an expert is not full
  if ((err = launch_experts_plan(r, w.count, width, plan, wide_width, &wide, stream)) != cudaSuccess) return err;
  err = launch_experts_spread(x, ld_x, xs, amax, dy, ld_dy, dys, dy_amax, w.n, r, plan, factor_amax, weight_of, stream);
  if (err != cudaSuccess) return err;
  if ((err = launch_experts_raw(xs, amax, slots, w, plan, width, reinterpret_cast<float*>(raw), stream)) != cudaSuccess) return err;
  BackArgs p = {};
  p.a = p.b = w.down, p.rows = w.n, p.cols = w.inner, p.activation = w.activation, p.plan = wide, p.weight_of = weight_of, p.amax = dy_amax;
  p.raw = reinterpret_cast<const float2*>(raw), p.gate_scale = w.gate.scale, p.up_scale = w.up.scale, p.slots = slots;
  p.factors = dx != nullptr ? reinterpret_cast<uint16_t*>(factors) : nullptr;
  p.groups = groups, p.factor_amax = factor_amax;
  p.dots = dweights != nullptr ? reinterpret_cast<float*>(dots) : nullptr;
  p.held = reinterpret_cast<float*>(held);
  if ((err = launch_back<kModeHidden>(wide_width, dys, 1, w.count, p, chunks, expected, info.sm_count, stream)) != cudaSuccess) return err;
  if (dx != nullptr) {
    if ((err = launch_experts_level(factors, slots, w.inner, 2, plan, factor_amax, groups, stream)) != cudaSuccess) return err;
    p.amax = factor_amax;
    p.a = w.gate, p.b = w.up, p.rows = w.inner, p.cols = w.n, p.part = reinterpret_cast<float*>(xs), p.more = reinterpret_cast<float*>(raw);
    if ((err = launch_back<kModeInput>(wide_width, factors, 2, w.count, p, chunks, expected, info.sm_count, stream)) != cudaSuccess) return err;
  }
  return launch_experts_combine(p.part, p.splits == 2 ? p.more : nullptr, r, nullptr, plan, w.n, dx, ld_dx, p.dots, (int)dot_parts(w.inner),
                                dweights, stream);
}

cudaError_t read_experts_backward_device_error(uint32_t* flags) {
  uint32_t v = 0;
  cudaError_t err = cudaMemcpyFromSymbol(&v, g_experts_backward_flags, sizeof v);
  if (err != cudaSuccess) return err;
  *flags = v;
  if (v) {
    const uint32_t zero = 0;
    err = cudaMemcpyToSymbol(g_experts_backward_flags, &zero, sizeof zero);
  }
  return err;
}

}  // namespace hscale
