// Cast to 8-bit floating point (e4m3) with a scale for each block of 128 channels: the operands of the block-scaled product.
//
//   s_b = the smallest power of two with max |x_b| <= 448 s_b  (1 for a block of zeros),   x8 = rn(x / s_b)
//
// b is 128 channels of one token, or 128 x 128 weights.  Dividing by a power of two is exact, so the only rounding is the one to
// 8 bits, and the scale needs no division: it is the exponent field of the maximum, moved by 8 (448 = 1.75 * 2^8).
// Bound by HBM: an element is read once (2 or 4 bytes) and written once (1 byte).  350880 x 5120 bf16: 770 us, 7.0 TB/s.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace vdn {

constexpr int kScaleBlock = 128;

// n / d for n < 2^32 by one multiplication: `factor` = ceil(2^64 / d) (0 stands for d = 1) is 2^64 / d + e / d with e < d, so n factor is
// n / d of 2^64 and at most n more, which is less than the 2^64 / d that would take it to the next whole number, since n d < 2^64.
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

// Scale of a block with the largest magnitude `u` (the bits of a finite fp32 number), and its reciprocal.  2^-126 at least, so that both
// are normal.
__device__ __forceinline__ float block_scale(uint32_t u, float& inverse) {
  int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = u == 0 ? 127 : max(e, 1);
  inverse = __uint_as_float((uint32_t)(254 - e) << 23);
  return __uint_as_float((uint32_t)e << 23);
}

// A lane's share of a block's row: 16 consecutive elements, those from `valid` on zero.  Magnitudes are compared as bit patterns of fp32;
// patterns from kInfinity on are not finite.
constexpr int kQuantizeLanes = kScaleBlock / 16, kQuantizeItems = 4;
constexpr uint32_t kInfinity = 0x7F800000u;

template <typename Tio>
struct Run16;

template <>
struct Run16<__nv_bfloat16> {                   // in pairs all the way: half the instructions
  uint32_t w[8];
  template <bool WIDE>
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int valid) {
    if (WIDE && valid >= 16) {
      const uint4 a = *reinterpret_cast<const uint4*>(p), b = *reinterpret_cast<const uint4*>(p + 8);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    } else {
      const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
      if (valid >= 16) {                        // rows that begin anywhere: whole words, and the ends by themselves where words begin odd
        if ((reinterpret_cast<uintptr_t>(p) & 2) == 0) {
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint32_t*>(u + 2 * i);
        } else {
          uint32_t mid[7];
#pragma unroll
          for (int i = 0; i < 7; ++i) mid[i] = *reinterpret_cast<const uint32_t*>(u + 2 * i + 1);
          w[0] = (uint32_t)u[0] | (mid[0] << 16);
#pragma unroll
          for (int i = 1; i < 7; ++i) w[i] = __funnelshift_l(mid[i - 1], mid[i], 16);
          w[7] = (mid[6] >> 16) | ((uint32_t)u[15] << 16);
        }
        return;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        w[i] = (2 * i < valid ? (uint32_t)u[2 * i] : 0u) | (2 * i + 1 < valid ? (uint32_t)u[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    return max(m >> 16, m & 0xFFFFu) << 16;
  }
  // what is not finite becomes NaN (8 bits have no infinity) and no maximum
  __device__ __forceinline__ uint32_t largest_finite() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool hi = (w[i] & 0x7F800000u) == 0x7F800000u, lo = (w[i] & 0x7F80u) == 0x7F80u;
      w[i] |= (hi ? 0x7FFF0000u : 0u) | (lo ? 0x7FFFu : 0u);
      m = __vmaxu2(m, w[i] & (hi ? 0u : 0x7FFF0000u) | w[i] & (lo ? 0u : 0x7FFFu));
    }
    return max(m >> 16, m & 0xFFFFu) << 16;
  }
  // elements 4 i .. 4 i + 3 times a power of two, in 8 bits (exact in bf16 but for what is zero in 8 bits)
  __device__ __forceinline__ uint32_t cast(int i, float inverse) const {
    const uint32_t f = __byte_perm(__float_as_uint(inverse), 0, 0x3232);
    uint32_t r[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t y;
      asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(w[2 * i + j]), "r"(f));
      r[j] = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(y << 16), __uint_as_float(y & 0xFFFF0000u)), __NV_SATFINITE, __NV_E4M3);
    }
    return r[0] | (r[1] << 16);
  }
};

template <>
struct Run16<float> {
  float x[16];
  template <bool WIDE>
  __device__ __forceinline__ void load(const float* p, int valid) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      if (WIDE && valid >= i + 4) {
        const float4 v = load4(p + i);
        x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
      } else {
#pragma unroll
        for (int j = i; j < i + 4; ++j) x[j] = j < valid ? p[j] : 0.f;
      }
    }
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return m;
  }
  __device__ __forceinline__ uint32_t largest_finite() {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
      if (u >= kInfinity) x[i] = __int_as_float(0x7FFFFFFF);
      else m = max(m, u);
    }
    return m;
  }
  __device__ __forceinline__ uint32_t cast(int i, float inverse) const {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i] * inverse, x[4 * i + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(x[4 * i + 2] * inverse, x[4 * i + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
};

template <typename Tio>
__device__ __forceinline__ void put_run(const Run16<Tio>& x, uint8_t* p, int valid, float inverse) {
  const uint32_t w[4] = {x.cast(0, inverse), x.cast(1, inverse), x.cast(2, inverse), x.cast(3, inverse)};
  if (valid >= 16) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < valid) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// Scales of 128 channels of a token: eight lanes to a block, a lane keeps ITEMS blocks in flight.  Sixteen elements a lane, bf16 compared
// and multiplied in pairs: with eight elements, each widened first, the instructions bound it (1313 us at the size above).  Rows
// that begin anywhere: 100000 x 2501 bf16 202 us, 3.7 TB/s.
template <typename Tio, bool WIDE>
__global__ void __launch_bounds__(256) quantize_rows_kernel(QuantizeArgs a) {
  constexpr int GROUPS = 256 / kQuantizeLanes, ITEMS = kQuantizeItems;
  const int lane = threadIdx.x % kQuantizeLanes;
  const uint32_t first = blockIdx.x * (uint32_t)(GROUPS * ITEMS) + threadIdx.x / kQuantizeLanes;
  Run16<Tio> x[ITEMS];
  uint32_t row[ITEMS];
  int col[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const uint32_t item = first + i * GROUPS;
    row[i] = quotient(item, a.per_row);
    col[i] = (int)(item - row[i] * a.per_row.d) * kScaleBlock + lane * 16;
    const int valid = item < a.items ? a.cols - col[i] : 0;
    x[i].template load<WIDE>(static_cast<const Tio*>(a.x) + (valid > 0 ? row[i] * a.x_stride + col[i] : 0), valid);
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    auto of_block = [](uint32_t m) {
#pragma unroll
      for (int o = kQuantizeLanes / 2; o > 0; o /= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, o, kQuantizeLanes));
      return m;
    };
    uint32_t top = of_block(x[i].largest());
    if (__any_sync(0xffffffffu, top >= kInfinity)) top = of_block(x[i].largest_finite());
    const uint32_t item = first + i * GROUPS;
    if (item >= a.items) continue;
    float inverse;
    const float s = block_scale(top, inverse);
    if (lane == 0) a.scale[item] = s;
    const int valid = a.cols - col[i];
    if (valid > 0) put_run(x[i], a.x8 + row[i] * a.out_stride + col[i], valid, inverse);
  }
}

// One scale for 128 rows of 128 channels: a CTA to a block, its elements in registers between the maximum and the cast.  5000 x 2600
// f32: 12.5 us, 5.2 TB/s: 2.8 waves of CTAs, two on an SM (64 registers, with a spill of 12 to 20 bytes), that each wait for their loads
// once.  bf16 takes 91 registers and has an SM to itself: 5120 x 5120 20.7 us, 3.8 TB/s, where two CTAs of 64 registers would take 14.6.
template <typename Tio, bool WIDE>
__global__ void __launch_bounds__(512, sizeof(Tio) == 4 ? 2 : 1) quantize_square_kernel(QuantizeArgs a) {
  constexpr int GROUPS = 512 / kQuantizeLanes, ITEMS = kScaleBlock / GROUPS;
  const long long row0 = (long long)(blockIdx.x / a.col_blocks) * kScaleBlock;
  const int col = (int)(blockIdx.x % a.col_blocks) * kScaleBlock + (int)(threadIdx.x % kQuantizeLanes) * 16;
  __shared__ uint32_t part[16];
  Run16<Tio> x[ITEMS];
  int valid[ITEMS];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const long long row = row0 + i * GROUPS + threadIdx.x / kQuantizeLanes;
    valid[i] = row < a.rows ? max(a.cols - col, 0) : 0;
    x[i].template load<WIDE>(static_cast<const Tio*>(a.x) + (valid[i] ? row * a.x_stride + col : 0), valid[i]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) top = max(top, x[i].largest());
  if (__syncthreads_or(top >= kInfinity)) {
    top = 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) top = max(top, x[i].largest_finite());
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, part[i]);
  float inverse;
  const float s = block_scale(top, inverse);
  if (threadIdx.x == 0) a.scale[blockIdx.x] = s;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const long long row = row0 + i * GROUPS + threadIdx.x / kQuantizeLanes;
    if (valid[i]) put_run(x[i], a.x8 + row * a.out_stride + col, valid[i], inverse);
  }
}

}  // namespace vdn
