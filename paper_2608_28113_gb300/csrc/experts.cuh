// experts.cuh -- what the kernels of a mixture of experts share: its weights, the grouping of its tokens, its
// activations.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "hscale_device.cuh"
#include "nvfp4_weight.cuh"

namespace hscale {

// One NVFP4 matrix per expert: packed [experts, rows, cols / 2], codes [experts, rows, cols / 16], scale [experts].
struct ExpertMatrix {
  const uint8_t* packed;
  const uint8_t* codes;
  const float* scale;
};

// gate and up [inner, n], down [n, inner] of each expert.
struct Experts {
  ExpertMatrix gate, up, down;
  int64_t n, inner;
  int32_t count, activation;
};

// Slot t k + j is token t's j-th expert.  An id outside [0, experts) is none.
struct Routing {
  const int32_t* ids;
  const float* weights;
  int64_t tokens;
  int32_t k;
};

// The slots grouped by their experts (experts.cu): slot_of[pos], the experts one after another, slots ascending; chunks of
// at most `width` positions of one expert.
struct Chunk {
  int32_t expert, first, count, pad;
};
struct Plan {
  int32_t* header;  // chunks, positions
  Chunk* chunks;
  int32_t *slot_of, *pos_of;  // pos_of: -1 for a slot without an expert
};
inline __host__ __device__ int64_t plan_chunks(int64_t slots, int64_t experts, int64_t width) {
  return (slots < experts ? slots : experts) + slots / width;
}

constexpr int kActSilu = 0, kActGeluTanh = 1;

// act(g) = g s(q) with s the logistic function and q = g (silu) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (the tanh form of
// gelu); approximate exponential and quotient (some 2^-20), for values that are rounded to 16 bits next.
template <int kKind>
__device__ __forceinline__ float activate_fast(float g) {
  const float q = kKind == kActSilu ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
  return __fdividef(g, 1.0f + __expf(-q));
}
// act(g) and its derivative in fp32: the exponential of a number that is not positive and the quotient are off by a few
// 2^-23 (of 1, the derivative; of max(1, |g|), the activation).
template <int kKind>
__device__ __forceinline__ float2 activate(float g) {
  const float q = kKind == kActSilu ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
  const float e = __expf(-fabsf(q)), part = __fdividef(1.0f, 1.0f + e), other = e * part;
  const float s = q >= 0.0f ? part : other, a = g * s;
  if (kKind == kActSilu) return make_float2(a, fmaf(a, q >= 0.0f ? other : part, s));  // part other = s (1 - s)
  const float dq = 1.5957691216057308f * fmaf(0.134145f * g, g, 1.0f);
  return make_float2(a, s + (other > 0.0f ? g * dq * (part * other) : 0.0f));  // other may be 0 where dq is infinite
}

// Segments of K that the sums behind dweights (fp32) are formed in, each from zero.  The tensor cores cut off a sum's low bits
// at each step of 16, always toward zero: of sums of random numbers 2.5e-7 is lost over 1024 columns and 2e-6 over 8192 (of
// positive ones five times that), where fp32 sums that round are off by 3e-7 to 7e-7.  dweights takes the losses of g, of
// u and of dh: with these segments 8e-7 at 4096 columns as at 8192 (whole sums: 2.9e-6 and 4.6e-6; 1408 and 2048 columns:
// 1.2e-6; fp32 sums 0.6e-6 to 1.9e-6).  A step of 2048 tokens takes 2530 us with them, some 2080 without, 2390 with those
// longer ones.  Results in bf16 do not feel the loss, and hscale_experts has no segments.
inline int gate_up_segments(int64_t cols) { return (int)((cols + 1023) / 1024); }
inline int hidden_segments(int64_t cols) { return (int)((cols + 1407) / 1408); }

// Asynchronous copies of 4 or 8 bytes, of which `bytes` are read and the rest zeros.
__device__ __forceinline__ void copy_4_async(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_8_async(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Arrives, as one of the barrier's count, once this thread's copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// How a product's packed weights come to shared memory, a row's 128 bytes (256 weights) a stage:
//   kBulk    by TMA, their codes too (rows of codes of whole 16 bytes);
//   kMixed   by TMA, the codes by two warps' asynchronous copies;
//   kPairs   as kMixed, where a row is 8 bytes more than whole 16s, which TMA cannot step by: two rows are one of its
//            rows.  The odd ones begin 8 bytes into a piece of 16: their boxes begin 8 bytes earlier, and all are 144 wide;
//   kCopies  by the two warps' copies too (weights at an address of 8 bytes);
//   kDirect  not at all, they are read where they are unpacked (codes at an odd address).
// 16 tokens of 64 experts, 4096 x 2048, first product: 101 us, 118 (kMixed), 184 (kCopies).
constexpr int kDirect = 0, kCopies = 1, kMixed = 2, kPairs = 3, kBulk = 4;
constexpr uint32_t kPackedRow = 128, kPairRow = 144, kCodeRow = 20;  // bytes of a row in a stage, and its codes' words

// A lane's 32 bytes, the 16-byte pieces `piece` and `piece` + 1 of row `row` of `rows` (swizzled as TMA does; pairs: even
// rows first).
__device__ __forceinline__ void read_packed(uint32_t (&q)[8], uint32_t stage, int row, int rows, int piece, bool pairs) {
  if (!pairs) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(q[4 * e]), "=r"(q[4 * e + 1]), "=r"(q[4 * e + 2]), "=r"(q[4 * e + 3])
                   : "r"(stage + (uint32_t)row * kPackedRow + ((((uint32_t)(piece + e)) ^ ((uint32_t)row & 7u)) << 4)));
  } else {
    const uint32_t from = stage + (uint32_t)((row & 1) * (rows >> 1) + (row >> 1)) * kPairRow + (row & 1) * 8 + piece * 16;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(q[2 * e]), "=r"(q[2 * e + 1]) : "r"(from + 8 * e));
  }
}

// kRows rows of 128 bytes, from byte `from` of row `row` on, to rows first, first + 1, ... of a stage whose 16-byte
// pieces are swizzled as TMA does.  By a warp, 8 bytes a lane; first % 8 == 0.  Bytes past a row's end are zeros.
template <int kRows>
__device__ __forceinline__ void copy_packed(const uint8_t* packed, int64_t half_cols, int64_t all_rows, int64_t row, int64_t from,
                                            uint32_t stage, int first, int lane) {
  const int sub = lane >> 4, piece = lane & 15;
  const bool on = from + piece * 8 < half_cols;
  const uint8_t* src = on ? packed + (row + sub) * half_cols + from + piece * 8 : packed;
  const int64_t step = on ? 2 * half_cols : 0;
  uint32_t to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    to[i] = stage + (uint32_t)(first + 2 * i + sub) * kPackedRow + (((uint32_t)(piece >> 1) ^ (uint32_t)(2 * i + sub)) << 4) + (piece & 1) * 8;
  if (row + kRows <= all_rows) {
#pragma unroll 4
    for (int r = 0; r < kRows; r += 8)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        copy_8_async(to[i] + r * kPackedRow, src, on ? 8u : 0u);
        src += step;
      }
  } else {
    for (int r = 0; r < kRows; r += 8)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = on && row + r + 2 * i + sub < all_rows;
        copy_8_async(to[i] + r * kPackedRow, there ? src : packed, there ? 8u : 0u);
        src += step;
      }
  }
}
// The words that the codes from byte `from` of these rows on are in: four, and the one that they end in.  (A row's
// codes may begin inside a word; eight rows further it is the same place in the word.)
template <int kRows>
__device__ __forceinline__ void copy_codes(const uint8_t* codes, int64_t code_cols, int64_t all_rows, int64_t row, int64_t from,
                                           uint32_t stage, int first, int lane) {
  const int64_t end = all_rows * code_cols;
  if ((row + kRows - 1) * code_cols + from + 20 <= end) {
    const uint8_t* src = codes + (((row + (lane >> 2)) * code_cols + from) & ~(int64_t)3) + 4 * (lane & 3);
    const uint32_t to = stage + (uint32_t)(first + (lane >> 2)) * kCodeRow + 4 * (lane & 3);
#pragma unroll 4
    for (int r = 0; r < kRows; r += 8) {
      copy_4_async(to + r * kCodeRow, src, 4u);
      src += 8 * code_cols;
    }
#pragma unroll
    for (int r = 0; r < kRows; r += 32)
      copy_4_async(stage + (uint32_t)(first + r + lane) * kCodeRow + 16,
                   codes + (((row + r + lane) * code_cols + from) & ~(int64_t)3) + 16, 4u);
  } else {
    for (int r = lane; r < kRows; r += 32) {
      const int64_t word = ((row + r) * code_cols + from) & ~(int64_t)3;
#pragma unroll
      for (int e = 0; e < 5; ++e) {
        const int64_t left = end - (word + 4 * e);
        copy_4_async(stage + (uint32_t)(first + r) * kCodeRow + 4 * e, left > 0 ? codes + word + 4 * e : codes,
                     left <= 0 ? 0u : left < 4 ? (uint32_t)left : 4u);
      }
    }
  }
}
// The path for matrices a and b: a product's rows are `cols` long, all_rows of them.
inline int packed_path(const ExpertMatrix& a, const ExpertMatrix& b, int64_t cols, int64_t all_rows) {
  const auto both = [](const void* p, const void* q, uintptr_t n) {
    return reinterpret_cast<uintptr_t>(p) % n == 0 && reinterpret_cast<uintptr_t>(q) % n == 0;
  };
  if (!both(a.codes, b.codes, 4)) return kDirect;
  if (!both(a.packed, b.packed, 16) || all_rows > INT32_MAX - 512) return kCopies;
  if (cols % 32 != 0) return kPairs;
  return cols % 256 == 0 && both(a.codes, b.codes, 16) ? kBulk : kMixed;
}

// Weights as fp16: E2M1 times E4M3 has at most 6 significant bits, from 2^-10 to 2688, so a weight without its global
// scale is exact.  The card converts two nibbles in one instruction, and to fp16 only: 85 weights a cycle and
// SM with their scales, against 43 by the bit operations that make bf16.

// Four code bytes as two pairs of fp16, read as the rest of the library reads codes: sign cleared, in [1, 126] (byte
// 127, NaN, is left by the minimum).
__device__ __forceinline__ void codes_f16(uint32_t c4, uint32_t& lo, uint32_t& hi) {
  c4 &= 0x7F7F7F7Fu;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t"
      "min.f16x2 %0, %0, %3;\n\tmin.f16x2 %1, %1, %3;\n\tmax.f16x2 %0, %0, %4;\n\tmax.f16x2 %1, %1, %4;\n\t}"
      : "=&r"(lo), "=&r"(hi)
      : "r"(c4), "r"(0x5F005F00u /* 448 */), "r"(0x18001800u /* 2^-9 */));
}
// Eight nibbles times a scale (both halves), pairs (0, 1), (2, 3), (4, 5), (6, 7).
__device__ __forceinline__ void unpack_f16(uint32_t w, uint32_t scale, uint32_t* r) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t.reg .b32 p, q, s, t;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 p, a;\n\tcvt.rn.f16x2.e2m1x2 q, b;\n\tcvt.rn.f16x2.e2m1x2 s, c;\n\tcvt.rn.f16x2.e2m1x2 t, d;\n\t"
      "mul.rn.f16x2 %0, p, %5;\n\tmul.rn.f16x2 %1, q, %5;\n\tmul.rn.f16x2 %2, s, %5;\n\tmul.rn.f16x2 %3, t, %5;\n\t}"
      : "=&r"(r[0]), "=&r"(r[1]), "=&r"(r[2]), "=&r"(r[3])
      : "r"(w), "r"(scale));
}

// The slots' operand is fp16 too, under a power of two of its row: with amax (the bits of the row's largest bf16
// magnitude, 2^p <= amax < 2^(p + 1)) elements are held as v 2^-E, E = p - 14, so the largest is below 2^15.  fp16 has
// 24 binades below 2^0 and bf16's 8 bits fit its 11: an element loses bits only where it is below 2^-31 of the largest, and
// 2^-39 of the largest at most.  E >= -112: bf16's smallest numbers are still exact then.  A row with an Inf or NaN is taken as
// it is.
__device__ __forceinline__ int row_exponent(uint32_t amax) {
  return amax >= 0x7F80u ? 0 : max((int)(amax >> 7) - 127 - 14, -112);
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// two bf16 numbers times 2^-E as fp16
__device__ __forceinline__ uint32_t bf16_to_f16(uint32_t v, float down) {
  const __half2 h = __floats2half2_rn(bf16_lo(v) * down, bf16_hi(v) * down);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 bf16_to_f16(const uint4& v, float down) {
  return make_uint4(bf16_to_f16(v.x, down), bf16_to_f16(v.y, down), bf16_to_f16(v.z, down), bf16_to_f16(v.w, down));
}
// h and the factors of dx, made in fp32, are rounded to fp16 as they are made, 32 outputs of a slot under their own power of
// two E (a row's largest is not known yet), and moved under the row's afterwards (launch_experts_level): 11 bits, and as
// above a number loses more only below 2^-29 of its row's largest.  (As bf16 they were half of y's and dx's error.)
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
constexpr int kLevel = 32;  // outputs under one power of two
inline __host__ __device__ int64_t level_groups(int64_t cols) { return (cols + kLevel - 1) / kLevel; }
// the largest magnitude of eight bf16 numbers, as bits
__device__ __forceinline__ uint32_t amax_bf16(const uint4& v) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
  return max(m & 0xFFFFu, m >> 16);
}

}  // namespace hscale
