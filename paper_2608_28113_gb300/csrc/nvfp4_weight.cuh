// nvfp4_weight.cuh -- the packed NVFP4 weight and the 8-bit checkpoint as kernels read them.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "hscale_device.cuh"

namespace hscale {

// W_hat[f, k] = s_g * E4M3(code[f, k / 16]) * E2M1(nibble[f, k]); n % 16 == 0.
struct Nvfp4Weight {
  const uint8_t* packed;      // [m, n / 2], 8-byte aligned
  const uint8_t* codes;       // [m, n / 16]
  const float* global_scale;  // device scalar
  int64_t m, n;
};

// Weights as bf16.  E2M1 times E4M3 has at most 6 significant bits, so a weight without s_g is exact in bf16; the
// kernels hold 2^-7 of it (kWeightUnit) and multiply their sums by 128 s_g.
constexpr float kWeightUnit = 128.0f;

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Two code bytes as bf16x2 E4M3 2^119, read as the rest of the library reads codes: sign cleared, in [1, 126].
// A byte shifted to bf16's mantissa and low exponent bits reads as
// E4M3 2^-120, subnormals included (the formats' subnormal boundaries line up).
__device__ __forceinline__ uint32_t unpack_codes(uint32_t c2) {
  uint32_t c = (c2 & 0x7Fu) | ((c2 & 0x7F00u) << 8);
  c = __vminu2(__vmaxu2(c, 0x00010001u), kE4M3MaxCode * 0x00010001u);
  return mul_bf16x2(mul_bf16x2(c << 4, 0x7F007F00u /* 2^127 */), 0x77807780u /* 2^112 */);
}


// Loads that stay where they are written, so that several are in flight, and that leave the registers as they are
// where `on` is false (a branch around a load would have the result moved, and the move waits for it).
__device__ __forceinline__ void ld_32_ahead(const void* p, uint32_t (&r)[8]) {
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "l"(p));
}
__device__ __forceinline__ void ld_16_ahead(bool on, const void* p, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
               : "+r"(a), "+r"(b), "+r"(c), "+r"(d)
               : "l"(p), "r"((uint32_t)on));
}
__device__ __forceinline__ void ld_8_ahead(bool on, const void* p, uint32_t& a, uint32_t& b) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\t@p ld.global.nc.v2.u32 {%0, %1}, [%2];\n\t}"
               : "+r"(a), "+r"(b)
               : "l"(p), "r"((uint32_t)on));
}
__device__ __forceinline__ void ld_4_ahead(bool on, const void* p, uint32_t& a) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.nc.u32 %0, [%1];\n\t}"
               : "+r"(a)
               : "l"(p), "r"((uint32_t)on));
}
__device__ __forceinline__ void ld_2_ahead(bool on, const void* p, uint32_t& a) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.nc.u16 %0, [%1];\n\t}"
               : "+r"(a)
               : "l"(p), "r"((uint32_t)on));
}
__device__ __forceinline__ void ld_1_ahead(bool on, const void* p, uint32_t& a) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.nc.u8 %0, [%1];\n\t}"
               : "+r"(a)
               : "l"(p), "r"((uint32_t)on));
}

// The low-rank adapters of a call: A [count, rank, n], B [count, m, rank], alpha [count], and the
// adapter of each token (nullptr: adapter 0 for all).
struct Adapters {
  const __nv_bfloat16* a;
  const __nv_bfloat16* b;
  const float* alpha;
  const int32_t* of_token;
  int32_t count, rank;
};

// The adapter of token t, or -1 for none.
__device__ __forceinline__ int adapter_of(const Adapters& ad, int64_t t) {
  if (ad.count == 0) return -1;
  if (ad.of_token == nullptr) return 0;
  const int a = ad.of_token[t];
  return (unsigned)a < (unsigned)ad.count ? a : -1;
}

// Activations in 8 bits: codes [tokens, cols] and a power-of-two scale byte per 32 channels.
constexpr int kCkptBlock = 32;
constexpr int kCkptInt8 = 0, kCkptE4M3 = 1;
struct Checkpoint {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t ld_codes, ld_scales;
};

// 2^(byte - 127) in both halves, exact; byte 255 is NaN, and byte 0, which no save writes, 0.
__device__ __forceinline__ uint32_t ckpt_scale(uint32_t byte) {
  return (byte == 255u ? 0x7FC0u : byte << 7) * 0x00010001u;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two elements (bytes 2 kPair, 2 kPair + 1 of `four`) as the values they stand for: bf16x2, every step exact.
template <int kFormat, int kPair>
__device__ __forceinline__ uint32_t ckpt_values(uint32_t four, uint32_t scale) {
  if constexpr (kFormat == kCkptInt8) {
    // the low 7 bits u of a byte in the mantissa of 128 read as 128 + u; its sign bit one place further up makes 128 256
    const uint32_t p = __byte_perm(four, 0u, kPair ? 0x4342 : 0x4140);
    const uint32_t m = (p & 0x007F007Fu) | 0x43004300u, c = (p & 0x00800080u) | 0x43004300u;
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(m), "r"(c));
    return mul_bf16x2(r, scale);
  } else {
    // exponent and mantissa moved to bf16's low exponent bits and mantissa read as E4M3 2^-120
    const uint32_t p = __byte_perm(four, 0u, kPair ? 0x3424 : 0x1404);
    return mul_bf16x2(mul_bf16x2((p & 0x80008000u) | ((p >> 4) & 0x07F007F0u), 0x7B807B80u /* 2^120 */), scale);
  }
}

}  // namespace hscale
