// grad_norm.cu -- the 2-norm over many tensors, and the tensors scaled to a largest norm.
//   norm = sqrt(sum of all squares);  out = g * min(1, max_norm / norm), as they are where the norm is not finite.
//
// Bound by bandwidth: every gradient is read for the norm and once more to be scaled, by then from L2 if it is among the
// last ones read (1120 tensors of fp32, 1.8 GB: 860 us, 6.3 TB/s over the 5.4 GB of both reads and the write; 14 small ones: 10 us,
// the call and its two launches).  The tensors' addresses and sizes are kernel parameters (no copy to the GPU, and a graph keeps its own);
// a call of more tensors than a table holds goes in several launches.  A CTA takes pieces of kPiece elements, whichever tensors
// they are in, found by bisection of the table's running counts.
//
// Squares of a piece's 16 elements are summed in fp32 where the sum lies well inside fp32's range; elements whose
// squares leave it are taken again, scaled by a power of two.  A thread adds up kRun pieces in fp32, and these sums, the CTAs' and
// the launches' in fp64, each in a fixed order, so equal calls give equal bits.  (One fp32 sum a thread was off by 2^-13 after
// 20000 equal pieces.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstdint>

#include "chained_launch.h"
#include "hscale_device.cuh"
#include "hscale_internal.h"
#include "tma.cuh"

namespace hscale {
namespace {

constexpr int kThreads = 256, kPer = 16, kPiece = kThreads * kPer;  // elements a thread and a CTA take at once
constexpr int kMaxParts = kGradParts;
constexpr int kRun = 64;

template <int kTensors>
struct Table {
  const void* in[kTensors];
  void* out[kTensors];
  int64_t size[kTensors];
  int32_t end[kTensors];    // pieces up to and with this tensor
  uint8_t type[kTensors];
  int32_t count, parts;
  bool first;
  float max_norm;
};

__device__ __forceinline__ float half_to_float(uint32_t bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }

// A thread's 16 elements of a piece: four (fp32) or two (16 bits) vectors of 16 bytes, each beside its neighbours' so
// that a warp's loads are whole lines.  Elements behind the end are zeros.
template <int kWide>
__device__ __forceinline__ int64_t place(int64_t first, int i) { return first + ((int64_t)i * kThreads + threadIdx.x) * kWide; }

__device__ __forceinline__ void load(const void* in, int type, int64_t first, int64_t size, float (&v)[kPer]) {
  const bool even = (reinterpret_cast<uintptr_t>(in) & 15) == 0;
  if (type == kGradF32) {
    const float* p = static_cast<const float*>(in);
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const int64_t at = place<4>(first, i);
      if (even && at + 4 <= size) {
        const float4 q = *reinterpret_cast<const float4*>(p + at);
        v[4 * i] = q.x, v[4 * i + 1] = q.y, v[4 * i + 2] = q.z, v[4 * i + 3] = q.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * i + j] = at + j < size ? p[at + j] : 0.0f;
      }
    }
    return;
  }
  const uint16_t* p = static_cast<const uint16_t*>(in);
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int64_t at = place<8>(first, i);
    uint32_t w[4];
    if (even && at + 8 <= size) {
      const uint4 q = *reinterpret_cast<const uint4*>(p + at);
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = (at + 2 * j < size ? (uint32_t)p[at + 2 * j] : 0u) | (at + 2 * j + 1 < size ? (uint32_t)p[at + 2 * j + 1] << 16 : 0u);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[8 * i + 2 * j] = type == kGradBF16 ? bf16_lo(w[j]) : half_to_float(w[j] & 0xFFFFu);
      v[8 * i + 2 * j + 1] = type == kGradBF16 ? bf16_hi(w[j]) : half_to_float(w[j] >> 16);
    }
  }
}

__device__ __forceinline__ uint32_t to_half_bits(int type, float v) {
  return type == kGradBF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}

__device__ __forceinline__ void store(void* out, int type, int64_t first, int64_t size, const float (&v)[kPer]) {
  const bool even = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
  if (type == kGradF32) {
    float* p = static_cast<float*>(out);
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      const int64_t at = place<4>(first, i);
      if (even && at + 4 <= size) {
        *reinterpret_cast<float4*>(p + at) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + j < size) p[at + j] = v[4 * i + j];
      }
    }
    return;
  }
  uint16_t* p = static_cast<uint16_t*>(out);
#pragma unroll
  for (int i = 0; i < kPer / 8; ++i) {
    const int64_t at = place<8>(first, i);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = to_half_bits(type, v[8 * i + 2 * j]) | to_half_bits(type, v[8 * i + 2 * j + 1]) << 16;
    if (even && at + 8 <= size) {
      *reinterpret_cast<uint4*>(p + at) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (at + j < size) p[at + j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  }
}

// The tensor that a piece is in; i: the one before's.
template <int kTensors>
__device__ __forceinline__ int tensor_of(const Table<kTensors>& t, int piece, int i) {
  if (piece < t.end[i] && (i == 0 || piece >= t.end[i - 1])) return i;
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (piece < t.end[mid]) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// The sum of a value over the CTA, in every thread.
__device__ __forceinline__ double block_sum(double v, double* shared) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) s += shared[i];
  return s;
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads) squares_kernel(const __grid_constant__ Table<kTensors> t, double* parts) {
  __shared__ double shared[kThreads / 32];
  // sums of squares, of squares of v 2^-70 (where v^2 may leave fp32's range), and of v 2^90 (where it may vanish)
  float mid = 0.0f, high = 0.0f, low = 0.0f;
  double total = 0.0;
  const int pieces = t.end[t.count - 1];
  int i = 0, run = kRun;
  for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    if (--run < 0) {
      total += (double)mid + (double)high * 0x1p140 + (double)low * 0x1p-180;
      mid = high = low = 0.0f, run = kRun - 1;
    }
    i = tensor_of(t, piece, i);
    float v[kPer];
    load(t.in[i], t.type[i], (int64_t)(piece - (i ? t.end[i - 1] : 0)) * kPiece, t.size[i], v);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) s = fmaf(v[j], v[j], s);
    // an element whose square vanishes is nothing beside such a sum
    if (s > 0x1p-90f && s < 0x1p100f) {
      mid += s;
    } else if (s <= 0x1p-90f) {
      float q = 0.0f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) q = fmaf(v[j] * 0x1p90f, v[j] * 0x1p90f, q);
      low += q;
    } else {
      float q = 0.0f;
#pragma unroll
      for (int j = 0; j < kPer; ++j) q = fmaf(v[j] * 0x1p-70f, v[j] * 0x1p-70f, q);
      high += q;
    }
  }
  const double sum = block_sum(total + ((double)mid + (double)high * 0x1p140 + (double)low * 0x1p-180), shared);
  if (threadIdx.x == 0) parts[blockIdx.x] = t.first ? sum : parts[blockIdx.x] + sum;
}

// The norm of the CTAs' parts, which every CTA adds up alike.
__device__ __forceinline__ float norm_of(const double* parts, int count) {
  __shared__ double shared[kThreads / 32];
  double s = 0.0;
  for (int i = threadIdx.x; i < count; i += kThreads) s += parts[i];
  return (float)sqrt(block_sum(s, shared));
}

__global__ void __launch_bounds__(kThreads) norm_kernel(const double* parts, int count, float* norm) {
  pdl_wait_primary();
  const float v = norm_of(parts, count);
  if (threadIdx.x == 0) *norm = v;
}

template <int kTensors>
__global__ void __launch_bounds__(kThreads) clip_kernel(const __grid_constant__ Table<kTensors> t, const double* parts, float* norm) {
  pdl_wait_primary();
  const float v = norm_of(parts, t.parts);
  if (t.first && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
  const bool scaled = v > t.max_norm && v < INFINITY;
  const float factor = scaled ? t.max_norm / v : 1.0f;
  // below fp32's normal numbers the factor has few bits or none, although the scaled elements may be among them
  const bool tiny = factor < 0x1p-126f && t.max_norm > 0.0f;
  const double wide = tiny ? (double)t.max_norm / (double)v : 0.0;
  const int pieces = t.end[t.count - 1];
  int i = 0;
  // the last pieces first: the norm's pass read them last, so they may still be in L2
  for (int piece = pieces - 1 - (int)blockIdx.x; piece >= 0; piece -= gridDim.x) {
    i = tensor_of(t, piece, i);
    if (!scaled && t.in[i] == t.out[i]) continue;
    const int64_t first = (int64_t)(piece - (i ? t.end[i - 1] : 0)) * kPiece;
    float x[kPer];
    load(t.in[i], t.type[i], first, t.size[i], x);
    if (tiny) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] = (float)((double)x[j] * wide);
    } else if (scaled) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] *= factor;
    }
    store(t.out[i], t.type[i], first, t.size[i], x);
  }
}

template <int kTensors>
cudaError_t run(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int64_t count, bool clip,
                float max_norm, float* norm, double* parts, int sms, cudaStream_t stream) {
  Table<kTensors> t;
  int64_t all = 0;
  for (int64_t i = 0; i < count; ++i) all += (sizes[i] + kPiece - 1) / kPiece;
  // CTAs of the norm's launches, and so parts: the first launch writes them all, the others add to them
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)kMaxParts, (int64_t)4 * sms, all}));
  for (int pass = 0; pass < (clip ? 2 : 1); ++pass) {
    bool first = true;
    int64_t i = 0;
    while (i < count || first) {
      int n = 0;
      int64_t pieces = 0;
      for (; i < count && n < kTensors; ++i) {
        const int64_t p = (sizes[i] + kPiece - 1) / kPiece;
        if (p == 0) continue;
        if (pieces + p > ((int64_t)1 << 30)) {  // a piece's number and a grid's step stay within 32 bits
          if (n == 0) return cudaErrorInvalidValue;
          break;
        }
        pieces += p;
        t.in[n] = in[i], t.out[n] = out ? out[i] : const_cast<void*>(in[i]), t.size[n] = sizes[i], t.type[n] = (uint8_t)types[i];
        t.end[n] = (int32_t)pieces;
        ++n;
      }
      if (n == 0) {
        if (!first) break;
        t.in[0] = t.out[0] = nullptr, t.size[0] = 0, t.type[0] = 0, t.end[0] = 0, n = 1;
      }
      t.count = n, t.parts = most, t.first = first, t.max_norm = max_norm;
      cudaError_t err;
      if (pass == 0) {
        squares_kernel<kTensors><<<most, kThreads, 0, stream>>>(t, parts);
        err = cudaGetLastError();
      } else {
        err = launch_chained(clip_kernel<kTensors>, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(most, pieces))), kThreads,
                             0, stream, t, parts, norm);
      }
      if (err != cudaSuccess) return err;
      first = false;
    }
  }
  if (clip) return cudaSuccess;
  return launch_chained(norm_kernel, dim3(1), kThreads, 0, stream, parts, most, norm);
}

}  // namespace

cudaError_t launch_grad_norm(const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, int64_t count,
                             bool clip, float max_norm, float* norm, double* parts, cudaStream_t stream) {
  DeviceInfo info;
  const cudaError_t err = current_device_info(&info);
  if (err != cudaSuccess) return err;
  // a small table where it is enough: a launch's parameters are copied
  return count <= 64 ? run<64>(in, out, sizes, types, count, clip, max_norm, norm, parts, info.sm_count, stream)
                     : run<1000>(in, out, sizes, types, count, clip, max_norm, norm, parts, info.sm_count, stream);
}

}  // namespace hscale
