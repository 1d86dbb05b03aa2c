// Block-scaled 8-bit product in plain fp32 arithmetic: the second opinion beside the tensor-core kernels (VDN_FLAG_FORCE_SIMT).
//   out[m, n] = sum_b sa[m, b] sw[n / 128, b] sum_{k in block b} a[m, k] w[n, k]  + bias[n] + add[m, n]
// 64 x 64 outputs a CTA, 4 x 4 a thread, 32 channels at a time in shared memory; a block's sum is kept apart until its scales.
#pragma once
#include "quantize.cuh"

namespace vdn {

struct MatmulArgs {
  const uint8_t* a;
  const uint8_t* w;
  const float* a_scale;       // [M, blocks]
  const float* w_scale;       // [ceil(N / 128), blocks]
  const float* bias;          // [N] or null
  const void* add;            // [M, N] or null; may be out
  void* out;
  long long M, a_stride, w_stride, add_stride, out_stride;
  int N, K, blocks;
};

__device__ __forceinline__ float2 from_e4m3x2(uint32_t x) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)x, __NV_E4M3);
  return __half22float2(__half2(h));
}

// The two scales of a block as one factor: the result, with `first` = 1.  Where their product is no normal number although what it stands
// for may well be (a block's sum is 0 or 2^-18 .. 2^24.6), it is two: the sum times `first`, then times the result.  The larger goes first
// where the product is too small, the smaller where it is too large, so that the step between leaves the range only if the end does.
__device__ __forceinline__ bool normal_number(float x) { return (__float_as_uint(x) & 0x7FFFFFFFu) - 0x00800000u < 0x7F000000u; }
__device__ __forceinline__ float join_scales(float sa, float sw, float& first) {
  const float s = sa * sw;
  first = 1.f;
  if (normal_number(s) || sa == 0.f || sw == 0.f) return s;
  const bool a_first = (fabsf(sa) > fabsf(sw)) == (fabsf(s) < 1.f);
  first = a_first ? sa : sw;
  return a_first ? sw : sa;
}

template <typename Tio>
__global__ void __launch_bounds__(256) matmul_simt_kernel(MatmulArgs p) {
  constexpr int TILE = 64, KC = 32;
  __shared__ float sa[KC][TILE + 4], sw[KC][TILE + 4];
  const long long m0 = (long long)blockIdx.x * TILE;
  const int n0 = blockIdx.y * TILE, ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  const int lr = threadIdx.x / 4, lc = (threadIdx.x % 4) * 8;          // the row and the eight channels that this thread fetches
  float acc[4][4] = {};
  for (int b = 0; b < p.blocks; ++b) {
    float part[4][4] = {};
    for (int k0 = b * kScaleBlock; k0 < min((b + 1) * kScaleBlock, p.K); k0 += KC) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = k0 + lc + i;
        sa[lc + i][lr] = m0 + lr < p.M && k < p.K ? from_e4m3x2(p.a[(m0 + lr) * p.a_stride + k]).x : 0.f;
        sw[lc + i][lr] = n0 + lr < p.N && k < p.K ? from_e4m3x2(p.w[(n0 + lr) * p.w_stride + k]).x : 0.f;
      }
      __syncthreads();
#pragma unroll 8
      for (int k = 0; k < KC; ++k) {
        const float4 x = *reinterpret_cast<const float4*>(&sa[k][ty * 4]), y = *reinterpret_cast<const float4*>(&sw[k][tx * 4]);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(xs[i], ys[j], part[i][j]);
      }
    }
    const float ws = p.w_scale[(long long)(n0 / kScaleBlock) * p.blocks + b];   // (64 features lie in one block of 128)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long long m = m0 + ty * 4 + i;
      float first, s = join_scales(m < p.M ? p.a_scale[m * p.blocks + b] : 0.f, ws, first);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(part[i][j] * first, s, acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long m = m0 + ty * 4 + i;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tx * 4 + j;
      if (m >= p.M || n >= p.N) continue;
      float y = acc[i][j];
      if (p.bias) y += p.bias[n];
      if (p.add) y += to_float(static_cast<const Tio*>(p.add)[m * p.add_stride + n]);
      static_cast<Tio*>(p.out)[m * p.out_stride + n] = from_float<Tio>(y);
    }
  }
}

}  // namespace vdn
