// experts_backward.cu -- the gradients of a layer of experts with packed NVFP4 weights:
//   dh = D_e^T dy_t,  dw = h . dh,  dx_t = sum_j w_tj (G_e^T (dh u act'(g)) + U_e^T (dh act(g)))
// The slots are grouped as in the forward pass (experts.cu), x and dy laid out in that order, and g and u made again in
// fp32.  Two products by transposed weights follow: the first (K = n) makes dh and, as it leaves tensor memory, dw and the two factors
// of dx, rounded to bf16 with G's and U's global scales in them; the second (K = G's rows, then U's) makes each slot's
// part of dx in fp32; a token's slots are added up in order and rounded once.
//
// The transposed products.  Tile: 256 outputs (columns of the weights) as two halves of 128 x up to kN slots, K in blocks
// of 64 rows.  The packed rows, unpacked as they are stored, make the weights' tile MN-major in shared memory
// (tensor memory would take it K-major only).  18 warps, as in the forward pass: TMA loads of the slots' tile, MMAs,
// epilogue, and three groups of four that unpack the halves' blocks in turn: a thread has 64 outputs of a row of K.
// Bound by shared memory, which carries both operands: at 128 slots some 875 cycles a K block against 512 of MMAs.
//
// Every wait is bounded; a CTA in which one ran out writes NaN for what it owed and sets the error flag.
#include <algorithm>

#include "chained_launch.h"
#include "experts.cuh"
#include "hscale_internal.h"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace hscale {
namespace {

__device__ uint32_t g_experts_backward_flags = 0;

constexpr int kBM = 128, kBK = 64, kHalves = 2;
constexpr int kThreads = 576;
constexpr int kUnpackWarp0 = 6, kUnpackGroups = 3;
constexpr int kAhead = 2;  // blocks of its own that a group has in flight
constexpr int kModeHidden = 0, kModeInput = 1;
constexpr uint32_t kGroupBytes = 64 * kBK * 2;  // 64 outputs x 64 rows of K
constexpr uint32_t kHalfBytes = 2 * kGroupBytes;
constexpr uint32_t kTurnBytes = 4 * 2048;

template <int kN>
struct Tile {
  static constexpr int kStages = kN == 128 ? 4 : 5;
  static constexpr uint32_t kABytes = kHalves * kHalfBytes, kBBytes = kN * kBK * 2;
  static constexpr uint32_t kSmemBytes = kStages * (kABytes + kBBytes) + 1024 /* alignment */ + 256 /* barriers */ + kTurnBytes;
  static constexpr uint32_t kAcc = kHalves * kN, kTmemCols = 2 * kAcc;
};

struct BackArgs {
  ExpertMatrix a, b;    // the weights of the first and the second half of K (down twice where there is one)
  int64_t rows, cols;   // of an expert's matrix: K and the outputs
  int32_t kb_part, parts, tiles_o;
  int32_t activation;
  Plan plan;
  const float* weights;
  const uint32_t* amax;      // of each position's dy
  const float* raw;          // g and u, [positions, 2, cols]
  const float *gate_scale, *up_scale;
  __nv_bfloat16* factors;    // [positions, 2, cols], or nullptr
  float* dots;               // [8 tiles_o, slots] partial sums of h . dh, or nullptr
  int64_t slots;
  float* part;               // [slots, cols]
};

__device__ __forceinline__ void unpack8(uint32_t w, uint32_t scale, uint32_t (&r)[4]) {
  constexpr uint32_t kSign = 0x80008000u, kMag = 0x01C001C0u;
  const uint32_t up = w << 4;
  const uint32_t a = __byte_perm(up, w, 0x5410), b = __byte_perm(up, w, 0x7632);
  r[0] = mul_bf16x2(((a << 8) & kSign) | ((a << 2) & kMag), scale);
  r[1] = mul_bf16x2((a & kSign) | ((a >> 6) & kMag), scale);
  r[2] = mul_bf16x2(((b << 8) & kSign) | ((b << 2) & kMag), scale);
  r[3] = mul_bf16x2((b & kSign) | ((b >> 6) & kMag), scale);
}

// 16 columns' sums over a warp's lanes: lane l, even, has that of column_of(l).
__device__ __forceinline__ float sum_columns(float (&v)[16], int lane) {
#pragma unroll
  for (int n = 8, d = 16; n > 0; n >>= 1, d >>= 1) {
    const bool upper = (lane & d) != 0;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float send = upper ? v[j] : v[j + n], keep = upper ? v[j + n] : v[j];
      v[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, d);
    }
  }
  return v[0] + __shfl_xor_sync(0xFFFFFFFFu, v[0], 1);
}
__device__ __forceinline__ int column_of(int lane) { return (lane >> 1 & 8) | (lane >> 1 & 4) | (lane >> 1 & 2) | (lane >> 1 & 1); }

// 16 slots of 32 outputs (a slot's in neighbouring lanes) rounded and stored, 8 outputs a lane.
__device__ __forceinline__ void store_rows(const float (&v)[16], uint32_t* turn, __nv_bfloat16* out, int64_t stride, int64_t at0,
                                           int64_t cols, int left, int lane) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 8; ++j) turn[j * 32 + lane] = pack_bf16(v[2 * j], v[2 * j + 1]);
  __syncwarp();
  const int pair = lane >> 2;
  const uint4 q0 = reinterpret_cast<const uint4*>(turn)[2 * lane], q1 = reinterpret_cast<const uint4*>(turn)[2 * lane + 1];
  const int64_t at = at0 + (lane & 3) * 8;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t pick = e ? 0x7632u : 0x5410u;
    const uint4 r = make_uint4(__byte_perm(q0.x, q0.y, pick), __byte_perm(q0.z, q0.w, pick), __byte_perm(q1.x, q1.y, pick),
                               __byte_perm(q1.z, q1.w, pick));
    // cols is a multiple of 16: 8 outputs are all there or none is
    if (2 * pair + e < left && at < cols) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(out) + (2 * pair + e) * stride + at) = r;
  }
}

template <int kMode, int kN>
__global__ void __launch_bounds__(kThreads, 1) back_kernel(const __grid_constant__ CUtensorMap vmap, const __grid_constant__ BackArgs p) {
  using T = Tile<kN>;
  constexpr int kStages = T::kStages;
  extern __shared__ __align__(16) uint8_t dynamic_smem[];
  uint8_t* smem = dynamic_smem + ((1024u - (smem_addr(dynamic_smem) & 1023u)) & 1023u);
  uint8_t* tile_a = smem;
  uint8_t* tile_b = smem + kStages * T::kABytes;
  uint8_t* rest = tile_b + kStages * T::kBBytes;
  uint64_t* full = reinterpret_cast<uint64_t*>(rest);
  uint64_t* empty = full + kStages;
  uint64_t* acc_full = empty + kStages;
  uint64_t* acc_empty = acc_full + 2;
  uint64_t* mma_done = acc_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  uint32_t* failed = tmem_slot + 1;
  uint32_t* turn = reinterpret_cast<uint32_t*>(rest + 256) + (threadIdx.x >> 5 & 3) * (kTurnBytes / 16);

  const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1 + kHalves * 4);  // the TMA load and the warps of the halves' groups
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 128);
    }
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
  const uint32_t tmem = warp_uniform(*tmem_slot);
  pdl_wait_primary();  // the plan, the slots' tile, g and u

  const int tiles = p.plan.header[0] * p.tiles_o, step = (int)gridDim.x, first = (int)blockIdx.x;
  const int ntiles = tiles > first ? (tiles - first + step - 1) / step : 0;
  const int kbs = p.kb_part * p.parts;
  const uint32_t quarter = (uint32_t)(warp & 3), lane_base = (quarter * 32u) << 16;

  if (warp == 0) {
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    uint32_t s = 0, parity = 1;
    bool go = true;
    for (int i = 0; i < ntiles && go; ++i) {
      const Chunk c = p.plan.chunks[(first + i * step) / p.tiles_o];
      for (int kb = 0; kb < kbs; ++kb) {
        if (!mbar_wait_warp(&empty[s], parity)) {
          if (lane == 0) atomicOr(failed, 1u);
          go = false;
          break;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(&full[s], T::kBBytes);
          const int part = kb >= p.kb_part ? 1 : 0;
          tma_load_3d(tile_b + s * T::kBBytes, &vmap, (kb - part * p.kb_part) * kBK, part, c.first, &full[s], policy);
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
      const Chunk c = p.plan.chunks[(first + i * step) / p.tiles_o];
      const uint32_t idesc = warp_uniform((kMode == kModeHidden ? idesc_f16_f32(kBM, (uint32_t)((c.count + 15) & ~15))
                                                                   : idesc_bf16_f32(kBM, (uint32_t)((c.count + 15) & ~15))) | 1u << 15);
      const uint32_t acc = (uint32_t)i & 1u, d = tmem + acc * T::kAcc;
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
    bool have = true;
    const float nan = __int_as_float(0x7FC00000);
    for (int i = 0; i < ntiles; ++i) {
      const int t = first + i * step, to = t % p.tiles_o;
      const Chunk c = p.plan.chunks[t / p.tiles_o];
      const uint32_t acc = (uint32_t)i & 1u, d = tmem + acc * T::kAcc + lane_base;
      const float scale = kMode == kModeHidden ? p.a.scale[c.expert] : kWeightUnit;
      if (have) have = __all_sync(0xFFFFFFFFu, mbar_wait_acc(&acc_full[acc], (uint32_t)(i >> 1) & 1u));
      tc_fence_after_sync();
#pragma unroll 1
      for (int half = 0; half < kHalves; ++half) {
        const int64_t at0 = (int64_t)to * (kHalves * kBM) + half * kBM + quarter * 32, o = at0 + lane;
        const bool on = o < p.cols;
#pragma unroll 1
        for (int j0 = 0; j0 < kN; j0 += 16) {
          if (j0 >= c.count) break;
          uint32_t a[16];
          tmem_ld_32x32b_x16(d + (uint32_t)(half * kN + j0), a);
          tmem_ld_wait();
          if (half == kHalves - 1 && j0 + 16 >= c.count) {
            tc_fence_before_sync();
            mbar_arrive(&acc_empty[acc]);
          }
          const int left = min(16, c.count - j0);
          const int64_t pos = c.first + j0;
          if constexpr (kMode == kModeHidden) {
            const int my_slot = lane < left ? p.plan.slot_of[pos + lane] : 0;
            const float sg = p.gate_scale[c.expert], su = p.up_scale[c.expert];
            const float my_w = lane < left ? p.weights[my_slot] : 0.0f;
            const float my_up = lane < left ? exp2_int(row_exponent(p.amax[pos + lane])) : 0.0f;
            float dg[16], du[16];
            const float* raw = p.raw + pos * 2 * p.cols + o;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              dg[j] = j < left && on ? raw[(int64_t)(2 * j) * p.cols] : 0.0f;
              du[j] = j < left && on ? raw[(int64_t)(2 * j + 1) * p.cols] : 0.0f;
            }
            float dot[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float dh = have ? __uint_as_float(a[j]) * (scale * __shfl_sync(0xFFFFFFFFu, my_up, j)) : nan, w = __shfl_sync(0xFFFFFFFFu, my_w, j);
              const float2 act = activate(p.activation, dg[j]);
              const float u = du[j];
              dot[j] = j < left && on ? dh * (act.x * u) : 0.0f;
              dg[j] = w * dh * u * act.y * sg;
              du[j] = w * dh * act.x * su;
            }
            if (p.factors != nullptr) {
              __nv_bfloat16* out = p.factors + pos * 2 * p.cols;
              store_rows(dg, turn, out, 2 * p.cols, at0, p.cols, left, lane);
              store_rows(du, turn, out + p.cols, 2 * p.cols, at0, p.cols, left, lane);
            }
            if (p.dots != nullptr) {
              const float s = sum_columns(dot, lane);
              const int j = column_of(lane);
              if ((lane & 1) == 0 && j < left) p.dots[((int64_t)(to * kHalves + half) * 4 + quarter) * p.slots + pos + j] = s;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              if (j < left && on) p.part[(pos + j) * p.cols + o] = have ? __uint_as_float(a[j]) * scale : nan;
            }
          }
        }
      }
    }
    if (!have && lane == 0) atomicOr(failed, 1u);
  } else {
    // a thread: 64 outputs of one row of K
    const int tid = (int)threadIdx.x - kUnpackWarp0 * 32;
    const int group = tid >> 7, line = tid & 127, row = line & 63;
    const int64_t cols = p.cols, half_cols = cols >> 1, code_cols = cols >> 4;
    const bool wide = (cols & 63) == 0 && ((reinterpret_cast<uintptr_t>(p.a.packed) | reinterpret_cast<uintptr_t>(p.b.packed)) & 31) == 0 &&
                      ((reinterpret_cast<uintptr_t>(p.a.codes) | reinterpret_cast<uintptr_t>(p.b.codes)) & 3) == 0;
    // job j: half j % 2 of K block j / 2, over the CTA's tiles; this group's are group, group + 3, ...
    const int per_tile = kHalves * kbs;
    const int64_t total = (int64_t)ntiles * per_tile;
    int li = 0, lj = group;  // the next job to load
    uint32_t ring[kAhead][8], codes[kAhead][4];
    auto load = [&](uint32_t (&q)[8], uint32_t (&c)[4]) {
      while (lj >= per_tile) lj -= per_tile, ++li;
      if (li >= ntiles) return;
      const int t = first + li * step, block = lj >> 1, part = block >= p.kb_part ? 1 : 0;
      const int64_t e = p.plan.chunks[t / p.tiles_o].expert;
      const int64_t o0 = (int64_t)(t % p.tiles_o) * (kHalves * kBM) + (lj & 1) * kBM + (line >> 6) * 64;
      // rows past the end of K are read as the last one (the slots' tile is zeros there), outputs past the end as
      // the last 64 or as zeros, and not stored
      const int64_t f = e * p.rows + min((int64_t)(block - part * p.kb_part) * kBK + row, p.rows - 1);
      const int64_t oin = min(o0, (cols - 1) & ~(int64_t)63);
      const uint8_t* w = (part ? p.b.packed : p.a.packed) + f * half_cols + (oin >> 1);
      const uint8_t* code = (part ? p.b.codes : p.a.codes) + f * code_cols + (oin >> 4);
      if (wide) {
        ld_32_ahead(w, q);
        ld_4_ahead(true, code, c[0]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = q[2 * i] = q[2 * i + 1] = 0u;
          ld_8_ahead(o0 + 16 * i < cols, w + 8 * i, q[2 * i], q[2 * i + 1]);
          ld_1_ahead(o0 + 16 * i < cols, code + i, c[i]);
        }
      }
      lj += kUnpackGroups;
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int i = 0; i < 4; ++i) codes[u][i] = 0u;
      load(ring[u], codes[u]);
    }
    bool go = true;
    for (int64_t base = group; base < total && go; base += kAhead * kUnpackGroups) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t job = base + u * kUnpackGroups;
        if (job >= total || !go) break;
        const uint32_t block = (uint32_t)(job >> 1), s = block % kStages, parity = ((block / kStages) & 1u) ^ 1u;
        if (!mbar_wait_warp(&empty[s], parity)) {
          go = false;
          break;
        }
        uint8_t* dst = tile_a + s * T::kABytes + (uint32_t)(job & 1) * kHalfBytes + line * 128;
        const uint32_t code = wide ? codes[u][0] : codes[u][0] | codes[u][1] << 8 | codes[u][2] << 16 | codes[u][3] << 24;
        uint32_t ca, cb;
        if constexpr (kMode == kModeHidden)
          codes_f16(code, ca, cb);
        else
          ca = unpack_codes(code & 0xFFFFu), cb = unpack_codes(code >> 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          uint32_t r[4];
          const uint32_t scale = __byte_perm(i < 4 ? ca : cb, 0u, (i & 2) ? 0x3232 : 0x1010);
          if constexpr (kMode == kModeHidden)
            unpack_f16(ring[u][i], scale, r);
          else
            unpack8(ring[u][i], scale, r);
          *reinterpret_cast<uint4*>(dst + ((i ^ (row & 7)) << 4)) = make_uint4(r[0], r[1], r[2], r[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full[s]);
        load(ring[u], codes[u]);
      }
    }
    if (!go && lane == 0) atomicOr(failed, 1u);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, T::kTmemCols);
  }
  if (threadIdx.x == 0 && *failed) atomicOr(&g_experts_backward_flags, kErrMbarTimeout);
}

// dweights of each slot: the sum of its position's partial sums, in order; 0 for a slot without an expert.
__global__ void __launch_bounds__(256) dweights_kernel(const float* dots, int parts, int64_t slots, const int32_t* ids,
                                                       int experts, Plan plan, float* dweights) {
  pdl_wait_primary();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= slots) return;
  if ((unsigned)ids[i] >= (unsigned)experts) dweights[i] = 0.0f;
  if (i < plan.header[1]) {
    float s = 0.0f;
    for (int q = 0; q < parts; ++q) s += dots[(int64_t)q * slots + i];
    dweights[plan.slot_of[i]] = s;
  }
}

template <int kMode, int kN>
cudaError_t launch_back_n(const void* v, int64_t depth, int parts, const BackArgs& p, int64_t most_tiles, int sms, cudaStream_t stream) {
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
  auto kernel = back_kernel<kMode, kN>;
  err = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), (int)Tile<kN>::kSmemBytes);
  if (err != cudaSuccess) return err;
  return launch_chained(kernel, dim3((unsigned)std::min<int64_t>(most_tiles, sms)), kThreads, (int)Tile<kN>::kSmemBytes, stream, map, p);
}
template <int kMode>
cudaError_t launch_back(int width, const void* v, int parts, BackArgs p, int64_t chunks, int sms, cudaStream_t stream) {
  p.parts = parts;
  p.kb_part = (int32_t)((p.rows + kBK - 1) / kBK);
  p.tiles_o = (int32_t)((p.cols + kHalves * kBM - 1) / (kHalves * kBM));
  const int64_t tiles = chunks * p.tiles_o;
  if (tiles > INT32_MAX) return cudaErrorInvalidValue;
  switch (width) {
    case 32: return launch_back_n<kMode, 32>(v, p.rows, parts, p, tiles, sms, stream);
    case 64: return launch_back_n<kMode, 64>(v, p.rows, parts, p, tiles, sms, stream);
    default: return launch_back_n<kMode, 128>(v, p.rows, parts, p, tiles, sms, stream);
  }
}

inline int64_t round256(int64_t bytes) { return (bytes + 255) / 256 * 256; }
inline int64_t dot_parts(int64_t inner) { return (inner + kHalves * kBM - 1) / (kHalves * kBM) * kHalves * 4; }

}  // namespace

int64_t experts_backward_workspace(int64_t tokens, int64_t k, int64_t n, int64_t inner, int64_t experts) {
  const int64_t slots = tokens * k;
  // x and dy in order, whose place the slots' parts of dx take afterwards; g and u; the factors; the dots
  return experts_plan_bytes(slots, experts) + 2 * round256(slots * 4) + 2 * round256(slots * n * 2) + round256(slots * inner * 8) + round256(slots * inner * 4) +
         round256(dot_parts(inner) * slots * 4);
}

cudaError_t launch_experts_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const Routing& r, const Experts& w,
                                    void* dx, int64_t ld_dx, float* dweights, void* workspace, cudaStream_t stream) {
  DeviceInfo info;
  cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  const int64_t slots = r.tokens * r.k;
  const int width = std::max(32, experts_width(slots, w.count));
  const Plan plan = experts_plan_at(workspace, slots, w.count);
  uint32_t* amax = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + experts_plan_bytes(slots, w.count));
  uint32_t* dy_amax = amax + round256(slots * 4) / 4;
  uint8_t* xs = reinterpret_cast<uint8_t*>(dy_amax) + round256(slots * 4);
  uint8_t* dys = xs + round256(slots * w.n * 2);
  uint8_t* raw = dys + round256(slots * w.n * 2);
  uint8_t* factors = raw + round256(slots * w.inner * 8);
  uint8_t* dots = factors + round256(slots * w.inner * 4);
  const int64_t chunks = plan_chunks(slots, w.count, width);
  if ((err = launch_experts_plan(r, w.count, width, plan, stream)) != cudaSuccess) return err;
  if ((err = launch_experts_spread(x, ld_x, w.n, r, plan, xs, amax, nullptr, stream)) != cudaSuccess) return err;
  if ((err = launch_experts_spread(dy, ld_dy, w.n, r, plan, dys, dy_amax, nullptr, stream)) != cudaSuccess) return err;
  if ((err = launch_experts_raw(xs, amax, slots, w, plan, width, reinterpret_cast<float*>(raw), stream)) != cudaSuccess) return err;
  BackArgs p = {};
  p.a = p.b = w.down, p.rows = w.n, p.cols = w.inner, p.activation = w.activation, p.plan = plan, p.weights = r.weights, p.amax = dy_amax;
  p.raw = reinterpret_cast<const float*>(raw), p.gate_scale = w.gate.scale, p.up_scale = w.up.scale, p.slots = slots;
  p.factors = dx != nullptr ? reinterpret_cast<__nv_bfloat16*>(factors) : nullptr;
  p.dots = dweights != nullptr ? reinterpret_cast<float*>(dots) : nullptr;
  if ((err = launch_back<kModeHidden>(width, dys, 1, p, chunks, info.sm_count, stream)) != cudaSuccess) return err;
  if (dx != nullptr) {
    p.a = w.gate, p.b = w.up, p.rows = w.inner, p.cols = w.n, p.part = reinterpret_cast<float*>(xs);
    if ((err = launch_back<kModeInput>(width, factors, 2, p, chunks, info.sm_count, stream)) != cudaSuccess) return err;
    if ((err = launch_experts_combine(p.part, r, nullptr, plan, w.n, dx, ld_dx, stream)) != cudaSuccess) return err;
  }
  if (dweights == nullptr) return cudaSuccess;
  return launch_chained(dweights_kernel, dim3((unsigned)((slots + 255) / 256)), 256, 0, stream, reinterpret_cast<const float*>(dots),
                        (int)dot_parts(w.inner), slots, r.ids, w.count, plan, dweights);
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
