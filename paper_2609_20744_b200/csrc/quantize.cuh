// Cast to 8-bit floating point (e4m3) with a scale for each block of 128 channels: the operands of the block-scaled product.
//
//   s_b = the smallest power of two with max |x_b| <= 448 s_b  (1 for a block of zeros),   x8 = rn(x / s_b)
//
// b is 128 channels of one token, or 128 x 128 weights.  Dividing by a power of two is exact, so the only rounding is the one to
// 8 bits, and the scale needs no division: it is the exponent field of the maximum, moved by 8 (448 = 1.75 * 2^8).
// Bound by HBM: an element is read once (2 or 4 bytes) and written once (1 byte).
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace vdn {

constexpr int kScaleBlock = 128;

// n / d for n < 2^32 by one multiplication: `factor` = floor(2^64 / d) + 1 (0 stands for d = 1) is off by less than 2^-64 d, and
// n d < 2^64.
struct FastDivide {
  uint32_t d;
  uint64_t factor;
};
inline FastDivide fast_divide(uint32_t d) { return FastDivide{d, d <= 1 ? 0 : ~0ull / d + 1}; }
__device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDivide& f) {
  return f.factor ? (uint32_t)__umul64hi(n, f.factor) : n;
}

struct QuantizeArgs {
  const void* x;
  uint8_t* x8;
  float* scale;
  long long rows, x_stride, out_stride;   // elements from one row to the next
  int cols, col_blocks;
  uint32_t items;                         // rows * col_blocks of this launch (tile 1)
  FastDivide per_row;                     // by col_blocks
};

// Scale of a block with the largest magnitude `amax` (finite), and its reciprocal.  2^-126 at least, so that both are normal.
__device__ __forceinline__ float block_scale(float amax, float& inverse) {
  const uint32_t u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = u == 0 ? 127 : max(e, 1);
  inverse = __uint_as_float((uint32_t)(254 - e) << 23);
  return __uint_as_float((uint32_t)e << 23);
}

// N consecutive elements as floats; those from `valid` on are zero.  WIDE: the address is a multiple of 16 bytes.
template <typename Tio, int N, bool WIDE>
__device__ __forceinline__ void load_run(const Tio* p, int valid, float (&x)[N]) {
  if (WIDE && valid >= N) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = load4(p + i);
      x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = i < valid ? to_float(p[i]) : 0.f;
  }
}
// (one 16-byte load where eight elements are asked for)
template <>
__device__ __forceinline__ void load_run<__nv_bfloat16, 8, true>(const __nv_bfloat16* p, int valid, float (&x)[8]) {
  if (valid >= 8) {
    const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i < valid ? to_float(p[i]) : 0.f;
  }
}

// (fmaxf passes over NaN, which the maximum therefore must not begin with)
template <int N>
__device__ __forceinline__ float largest(const float (&x)[N]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) a = fmaxf(a, fabsf(x[i]));
  return a;
}
// ... and infinities made NaN and passed over too: 8 bits have no infinity
template <int N>
__device__ __forceinline__ float largest_finite(float (&x)[N]) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (isinf(x[i])) x[i] = __int_as_float(0x7fffffff);
    a = fmaxf(a, fabsf(x[i]));
  }
  return a;
}

template <int N>
__device__ __forceinline__ void store_run(uint8_t* p, int valid, const float (&x)[N], float inverse) {
  static_assert(N % 4 == 0, "whole words");
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * inverse, x[4 * i + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * inverse, x[4 * i + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
    w[i] = lo | (hi << 16);
  }
  if (valid >= N) {
    if constexpr (N == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < valid) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// Scales of 128 channels of a token.  A block goes to as many lanes as 16-byte pieces make it up (16 of bf16, 32 of f32), a lane
// keeps ITEMS blocks in flight.
template <typename Tio, bool WIDE>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantizeArgs a) {
  constexpr int N = 16 / sizeof(Tio), LANES = kScaleBlock / N, GROUPS = 256 / LANES, ITEMS = 4;
  const int lane = threadIdx.x % LANES;
  const uint32_t first = blockIdx.x * (uint32_t)(GROUPS * ITEMS) + threadIdx.x / LANES;
  float x[ITEMS][N];
  uint32_t row[ITEMS];
  int col[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint32_t item = first + i * GROUPS;
    row[i] = quotient(item, a.per_row);
    col[i] = (int)(item - row[i] * a.per_row.d) * kScaleBlock + lane * N;
    const int valid = item < a.items ? a.cols - col[i] : 0;
    load_run<Tio, N, WIDE>(static_cast<const Tio*>(a.x) + (valid > 0 ? row[i] * a.x_stride + col[i] : 0), valid, x[i]);
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    float amax = largest(x[i]);
#pragma unroll
    for (int o = LANES / 2; o > 0; o /= 2) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o, LANES));
    if (__any_sync(0xffffffffu, isinf(amax))) {
      amax = largest_finite(x[i]);
#pragma unroll
      for (int o = LANES / 2; o > 0; o /= 2) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o, LANES));
    }
    const uint32_t item = first + i * GROUPS;
    if (item >= a.items) continue;
    float inverse;
    const float s = block_scale(amax, inverse);
    if (lane == 0) a.scale[item] = s;
    const int valid = a.cols - col[i];
    if (valid > 0) store_run<N>(a.x8 + row[i] * a.out_stride + col[i], valid, x[i], inverse);
  }
}

// One scale for 128 rows of 128 channels: a CTA to a block, its elements in registers between the maximum and the cast.
template <typename Tio, bool WIDE>
__global__ void __launch_bounds__(512) quantize_square_kernel(QuantizeArgs a) {
  constexpr int N = 16 / sizeof(Tio), LANES = kScaleBlock / N, GROUPS = 512 / LANES, ITEMS = kScaleBlock / GROUPS;
  const long long row0 = (long long)(blockIdx.x / a.col_blocks) * kScaleBlock;
  const int col = (int)(blockIdx.x % a.col_blocks) * kScaleBlock + (int)(threadIdx.x % LANES) * N;
  __shared__ float part[16];
  float x[ITEMS][N];
  int valid[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const long long row = row0 + i * GROUPS + threadIdx.x / LANES;
    valid[i] = row < a.rows ? max(a.cols - col, 0) : 0;
    load_run<Tio, N, WIDE>(static_cast<const Tio*>(a.x) + (valid[i] ? row * a.x_stride + col : 0), valid[i], x[i]);
  }
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) amax = fmaxf(amax, largest(x[i]));
  if (__syncthreads_or(isinf(amax))) {
    amax = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) amax = fmaxf(amax, largest_finite(x[i]));
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = amax;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) amax = fmaxf(amax, part[i]);
  float inverse;
  const float s = block_scale(amax, inverse);
  if (threadIdx.x == 0) a.scale[blockIdx.x] = s;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const long long row = row0 + i * GROUPS + threadIdx.x / LANES;
    if (valid[i]) store_run<N>(a.x8 + row * a.out_stride + col, valid[i], x[i], inverse);
  }
}

}  // namespace vdn
