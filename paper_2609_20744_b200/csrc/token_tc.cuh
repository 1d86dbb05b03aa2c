// Token-wise gated delta rule (Eq. 2) on the tensor cores, in chunks of C = 64 tokens; bf16 I/O, d = 128.
//
// Inside a chunk, with G_i the running sum of log_alpha, r_i the optional 1 / |k_i| and S the state before the chunk,
// the rule is a unit lower triangular system for the written differences U:
//        (I + L) U = Diag(beta) X,      L_ij = beta_i e^{G_i - G_j} r_i r_j k_i.k_j  (j < i),
//        X = V - Diag(e^{G} r) K S^T,
//        S' = e^{G_C} S + U^T Diag(e^{G_C - G} r) K,
//        O  = scale (Diag(e^{G}) Q S^T + M U),      M_ij = e^{G_i - G_j} r_j q_i.k_j  (j <= i).
// Everything that does not depend on S is formed beforehand for all chunks at once (token_prep_kernel):
//        E = K^T Diag(e^{G_C - G} r) (I + L)^{-1} Diag(beta)      [d_k x C],  two bf16 parts
//        P = scale M (I + L)^{-1} Diag(beta)                      [C x C],    bf16
// so that a chunk's step of the sequential kernel (token_chain_kernel) is two dependent products,
//        X^T = V^T - (S K^T) Diag(e^G r),      S <- e^{G_C} S + X^T E^T,      O^T = (S Q^T) Diag(scale e^G) + X^T P^T.
//
// Precision.  K and Q are bf16 as given and enter exactly.  S, X, E and the triangular inverse are fp32 and enter the
// products that reach the state as two bf16 parts (16 bits; products of the two low parts are left out: 2^-16 of the
// whole), accumulated in fp32; S itself is carried in fp32 registers.  What only the rounded output sees (S Q^T, X^T P^T)
// takes the high parts alone.
#pragma once
#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"
#include "tc_common.cuh"
#include "token_rule.cuh"

namespace vdn {

// ---------------------------------------------------------------------------------------------- layout of a call
// Chunk c of sequence s (first row `start`) has the place start / 64 + s + c: no two chunks share one, because
// floor(a) + ceil(b) <= floor(a + b) + 1, and there are n_tokens / 64 + S places.  The offsets can so stay on the device.
struct TokenTc {
  static constexpr int C = 64, D = 128;
  static constexpr int E_PART = D * C * 2;            // one part of E: 128 rows of 128 bytes, as the swizzled operand lies in shared memory
  static constexpr int E_BYTES = 2 * E_PART;
  static constexpr int P_BYTES = C * C * 2;
  // per-token factors: e^G r [64], scale r_q e^G [64], e^{G_C}, padding
  static constexpr int F_FLOATS = 132, F_BYTES = F_FLOATS * 4;
};

struct TokenTcArgs {
  TokenArgs t;
  unsigned char* e;          // [places * H] E_BYTES
  unsigned char* p;          // ... P_BYTES
  unsigned char* f;          // ... F_BYTES
  long long places;
};

// The sequence that owns place x, places being `unit` rows wide: the last one whose first place is not behind x.
__device__ __forceinline__ int token_seq_of(const TokenArgs& t, long long x, int unit) {
  int lo = 0, hi = t.S - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    long long start;
    int len;
    token_range(t.cu_seqlens, mid, t.per, t.n_tokens, start, len);
    if (start / unit + mid <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

namespace tc {

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
               ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(src), "r"(bytes)
               : "memory");
}

// D[tmem] (+)= A[tmem] * B[smem]: A has its rows in the lanes and two K elements to a 32-bit column.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Two floats at once (the packed fp32 pipe).
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t r, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// x = hi + lo + rest, |rest| <= 2^-16 |x|, both parts rounded to nearest, two neighbours packed.  The high part comes from
// Dekker's splitting (c = (2^16 + 1) x, hi = c - (c - x)), which keeps NaN a NaN (rounding the bit pattern by an
// integer addition would turn the pattern 0x7FFFFFFF into -0); |x| must stay below 2^110.
__device__ __forceinline__ void split2_pair(uint64_t x, uint32_t& hi, uint32_t& lo) {
  const uint64_t minus = f2_pack(-1.f, -1.f);
  const uint64_t c = mul2(x, f2_pack(65537.f, 65537.f));
  const uint64_t t = fma2(x, minus, c);
  const uint64_t h = fma2(t, minus, c);
  const uint64_t r = fma2(h, minus, x);
  float h0, h1, r0, r1;
  f2_unpack(h, h0, h1);
  f2_unpack(r, r0, r1);
  hi = __byte_perm(__float_as_uint(h0), __float_as_uint(h1), 0x7632);
  lo = __byte_perm(__float_as_uint(r0) + 0x8000u, __float_as_uint(r1) + 0x8000u, 0x7632);
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace tc

// ---------------------------------------------------------------------------------------------- chunk operators
// One CTA (four warps) per (place, head).  [K; Q] K^T is one MMA chain with the keys in rows 0..63 and the queries in rows
// 64..127 of one operand, so that lane i of tensor memory holds row i of K K^T and lane 64 + i row i of Q K^T.  The inverse
// of the unit lower triangular I + L is a forward substitution in fp32, a thread to a column: its 64 rows stay in
// registers, and the rows of L are broadcast from shared memory.  A thread's column is a row of the (K-major) B operand
// of the two last products, so no transpose is needed.
struct TokenPrep {
  static constexpr int THREADS = 128;
  static constexpr int OFF_KQ = 0;                    // [K; Q]: two 64-channel boxes of 128 rows; later the parts of E
  static constexpr int OFF_T = 32768;                 // inverse times factors: high, low; inverse times beta; (first: L)
  static constexpr int OFF_M = OFF_T + 3 * 8192;      // scale M
  static constexpr int OFF_F = OFF_M + 8192;          // G high, G low, beta, r, weight [64] each, then the factors
  static constexpr int OFF_BAR = OFF_F + 5 * 256 + 640;
  static constexpr int SMEM_BYTES = OFF_BAR + 64 + 1024;
  static constexpr int L_PITCH = 68;                  // floats: 16-byte rows, lanes' rows four banks apart
};

__global__ void __launch_bounds__(TokenPrep::THREADS, 3)
token_prep_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ, const TokenTcArgs a,
                  tc::DevStatus ds) {
  using namespace tc;
  using S = TokenPrep;
  constexpr int C = TokenTc::C;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* bp = smem_dyn + (base - smem_u32(smem_dyn));
  const TokenArgs& t = a.t;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = (int)(blockIdx.x % t.H);
  const long long place = blockIdx.x / t.H;

  const int seq = token_seq_of(t, place, C);
  long long start;
  int len;
  token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
  const long long chunk = place - (start / C + seq);
  if (chunk < 0 || chunk * C >= len) return;          // a place that no chunk has
  const long long row0 = start + chunk * C;
  const int n = min(C, len - (int)(chunk * C));

  const uint32_t bar_load = base + S::OFF_BAR, bar_mma = bar_load + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bp + S::OFF_BAR + 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + S::OFF_BAR + 24);
  const WaitCtx wc(abort_flag, ds);
  float* g_hi = reinterpret_cast<float*>(bp + S::OFF_F);
  float* g_lo = g_hi + 64;
  float* beta = g_hi + 128;
  float* rk = g_hi + 192;
  float* wgt = g_hi + 256;
  float* fac = g_hi + 320;

  if (tid == 0) {
    mbar_init(bar_load, 1);
    mbar_init(bar_mma, 1);
    *abort_flag = 0;
    mbar_fence_init();
    const int hk = h / (t.H / t.Hk);
    mbar_arrive_expect_tx(bar_load, 32768);
    tma_load_2d(base, &tmK, bar_load, hk * 128, (int)row0);
    tma_load_2d(base + 16384, &tmK, bar_load, hk * 128 + 64, (int)row0);
    tma_load_2d(base + 8192, &tmQ, bar_load, hk * 128, (int)row0);
    tma_load_2d(base + 24576, &tmQ, bar_load, hk * 128 + 64, (int)row0);
  }
  if (warp == 1) {
    // running sum of the decay in 64 bits, kept as two floats: a difference of two of them is then good to fp32's
    // rounding however far the sum has run.  A token's log decay counts down to -104 (e^-104 is 0 in fp32), so that -infinity
    // leaves the differences finite.
    double x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * lane + i;
      float g = j < n && t.log_alpha ? t.log_alpha[(row0 + j) * t.H + h] : 0.f;
      x[i] = g < -104.f ? -104.0 : (double)g;
    }
    double sum = x[0] + x[1];
    const double own = sum;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const double y = __shfl_up_sync(0xFFFFFFFFu, sum, m);
      if (lane >= m) sum += y;
    }
    const double g0 = sum - own + x[0], g1 = sum;
    g_hi[2 * lane] = (float)g0;     g_lo[2 * lane] = (float)(g0 - (double)(float)g0);
    g_hi[2 * lane + 1] = (float)g1; g_lo[2 * lane + 1] = (float)(g1 - (double)(float)g1);
  } else if (warp >= 2) {
    const int j = tid - 64;
    beta[j] = j < n ? t.beta[(row0 + j) * t.H + h] : 0.f;
    rk[j] = 1.f;
  } else {
    __syncwarp();
    tmem_alloc(smem_u32(tmem_slot), 128);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
  bool ok = mbar_wait(bar_load, 0, wc);
  if (n < C && ok) {
    // keys behind the sequence are the next one's (or nothing's): they must not enter a sum, not even times zero
    for (int e = tid; e < (C - n) * 16; e += S::THREADS) {
      const int r = n + e / 16, c = e % 16;
      *reinterpret_cast<uint4*>(bp + (c >> 3) * 16384 + r * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
  }
  if (!__syncthreads_or(!ok)) {
    if (tid == 0) {
      constexpr uint32_t idesc = make_idesc_bf16(128, 64, false, false);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t at = base + (k >> 2) * 16384 + (k & 3) * 32;
        mma_bf16_ss(tmem, make_smem_desc(at, 16, 1024), make_smem_desc(at, 16, 1024), idesc, k ? 1u : 0u);
      }
      mma_commit(bar_mma);
    }
    const bool is_q = warp >= 2;
    const int i = tid & 63;                           // token of this thread's row
    float rq = 1.f;
    if (is_q && t.l2_eps > 0.f) {
      float ss = 0.f;
#pragma unroll 4
      for (int c = 0; c < 16; ++c) {
        const uint4 w = *reinterpret_cast<const uint4*>(bp + (c >> 3) * 16384 + (64 + i) * 128 + (((c & 7) ^ (i & 7)) << 4));
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = __uint_as_float(v[e] << 16), hi = __uint_as_float(v[e] & 0xFFFF0000u);
          ss = fmaf(lo, lo, fmaf(hi, hi, ss));
        }
      }
      rq = rsqrtf(ss + t.l2_eps);
    }
    ok = mbar_wait(bar_mma, 0, wc);
    if (!__syncthreads_or(!ok)) {
      tc_fence_after_sync();
      float x[64];
      tmem_ld32(lanes, *reinterpret_cast<float(*)[32]>(x));
      tmem_ld32(lanes + 32, *reinterpret_cast<float(*)[32]>(x + 32));
      tmem_wait_ld();
      if (t.l2_eps > 0.f) {                           // a key's squared norm is the diagonal of K K^T
        if (!is_q) {
          float kk = 0.f;
#pragma unroll
          for (int j = 0; j < 64; ++j) kk = j == i ? x[j] : kk;
          rk[i] = rsqrtf(kk + t.l2_eps);
        }
        __syncthreads();
      }
      const float gi_hi = g_hi[i], gi_lo = g_lo[i];
      const float row = is_q ? t.scale * rq : beta[i] * rk[i];
      const int last = is_q ? i : i - 1;              // L is strictly lower, M has its diagonal
#pragma unroll
      for (int j = 0; j < 64; j += 4) {
        const float4 gh = *reinterpret_cast<const float4*>(g_hi + j), gl = *reinterpret_cast<const float4*>(g_lo + j);
        const float4 rr = *reinterpret_cast<const float4*>(rk + j);
        x[j] = j <= last ? row * rr.x * __expf((gi_hi - gh.x) + (gi_lo - gl.x)) * x[j] : 0.f;
        x[j + 1] = j + 1 <= last ? row * rr.y * __expf((gi_hi - gh.y) + (gi_lo - gl.y)) * x[j + 1] : 0.f;
        x[j + 2] = j + 2 <= last ? row * rr.z * __expf((gi_hi - gh.z) + (gi_lo - gl.z)) * x[j + 2] : 0.f;
        x[j + 3] = j + 3 <= last ? row * rr.w * __expf((gi_hi - gh.w) + (gi_lo - gl.w)) * x[j + 3] : 0.f;
      }
      float* L = reinterpret_cast<float*>(bp + S::OFF_T);
      if (!is_q) {
#pragma unroll
        for (int j = 0; j < 64; j += 4)
          *reinterpret_cast<float4*>(L + i * S::L_PITCH + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
        const float eg = __expf(gi_hi + gi_lo);
        wgt[i] = rk[i] * __expf((g_hi[63] - gi_hi) + (g_lo[63] - gi_lo));
        fac[i] = eg * rk[i];
        if (i == 0) fac[128] = __expf(g_hi[63] + g_lo[63]);
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c)
          *reinterpret_cast<uint4*>(bp + S::OFF_M + i * 128 + ((c ^ (i & 7)) << 4)) =
              make_uint4(bf16_pair(x[8 * c], x[8 * c + 1]), bf16_pair(x[8 * c + 2], x[8 * c + 3]),
                         bf16_pair(x[8 * c + 4], x[8 * c + 5]), bf16_pair(x[8 * c + 6], x[8 * c + 7]));
        fac[64 + i] = t.scale * rq * __expf(gi_hi + gi_lo);
      }
      __syncthreads();
      const long long unit = place * t.H + h;
      if (!is_q) {
        // forward substitution: column i of (I + L)^-1;  columns from 32 on have nothing above row 32
        float y[64];
#pragma unroll
        for (int r = 0; r < 64; ++r) y[r] = 0.f;
        auto solve = [&](auto first) {
          constexpr int R0 = decltype(first)::value;
#pragma unroll
          for (int r = R0; r < 64; ++r) {
            float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
            for (int j = R0; j < r; j += 4) {
              const float4 l = *reinterpret_cast<const float4*>(L + r * S::L_PITCH + j);
              s0 = fmaf(l.x, y[j], s0);
              s1 = fmaf(l.y, y[j + 1], s1);
              s2 = fmaf(l.z, y[j + 2], s2);
              s3 = fmaf(l.w, y[j + 3], s3);
            }
            y[r] = (r == i ? 1.f : 0.f) - ((s0 + s1) + (s2 + s3));
          }
        };
        if (warp == 0) solve(std::integral_constant<int, 0>{});
        else solve(std::integral_constant<int, 32>{});
        named_barrier_sync(1, 64);                    // L is read, its place is taken by the operands
        const float b = beta[i];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          uint32_t hi[4], lo[4], one[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 8 * c + 2 * e;
            const float u0 = y[r] * b, u1 = y[r + 1] * b;
            split2_pair(f2_pack(wgt[r] * u0, wgt[r + 1] * u1), hi[e], lo[e]);
            one[e] = bf16_pair(u0, u1);
          }
          unsigned char* at = bp + S::OFF_T + i * 128 + ((c ^ (i & 7)) << 4);
          *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(at + 8192) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          *reinterpret_cast<uint4*>(at + 16384) = make_uint4(one[0], one[1], one[2], one[3]);
        }
      } else {
        float* f = reinterpret_cast<float*>(a.f + (size_t)unit * TokenTc::F_BYTES);
        f[i] = fac[i];
        f[64 + i] = fac[64 + i];
        if (i == 0) f[128] = fac[128];
      }
      fence_proxy_async_smem();
      tc_fence_before_sync();
      __syncthreads();
      tc_fence_after_sync();
      if (tid == 0) {
        // E [128 x 64] = K^T (M rows = channels, read MN-major) times the two parts
        constexpr uint32_t ide = make_idesc_bf16(128, 64, true, false);
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16_ss(tmem + 64, make_smem_desc(base + k * 2048, 16384, 1024),
                        make_smem_desc(base + S::OFF_T + part * 8192 + k * 32, 16, 1024), ide, part || k ? 1u : 0u);
        // P: rows 64..127 of the A operand are scale M, the rows before it are of no interest
        constexpr uint32_t idp = make_idesc_bf16(128, 64, false, false);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16_ss(tmem, make_smem_desc(base + S::OFF_M - 8192 + k * 32, 16, 1024),
                      make_smem_desc(base + S::OFF_T + 16384 + k * 32, 16, 1024), idp, k ? 1u : 0u);
        mma_commit(bar_mma);
      }
      ok = mbar_wait(bar_mma, 1, wc);
      if (!__syncthreads_or(!ok)) {
        tc_fence_after_sync();
        tmem_ld32(lanes + 64, *reinterpret_cast<float(*)[32]>(x));
        tmem_ld32(lanes + 96, *reinterpret_cast<float(*)[32]>(x + 32));
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 8; ++c) {                 // row tid of E: channel tid
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) split2_pair(f2_pack(x[8 * c + 2 * e], x[8 * c + 2 * e + 1]), hi[e], lo[e]);
          unsigned char* at = bp + S::OFF_KQ + tid * 128 + ((c ^ (tid & 7)) << 4);
          *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(at + TokenTc::E_PART) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        if (is_q) {
          tmem_ld32(lanes, *reinterpret_cast<float(*)[32]>(x));
          tmem_ld32(lanes + 32, *reinterpret_cast<float(*)[32]>(x + 32));
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < 8; ++c)
            *reinterpret_cast<uint4*>(bp + S::OFF_T + i * 128 + ((c ^ (i & 7)) << 4)) =
                make_uint4(bf16_pair(x[8 * c], x[8 * c + 1]), bf16_pair(x[8 * c + 2], x[8 * c + 3]),
                           bf16_pair(x[8 * c + 4], x[8 * c + 5]), bf16_pair(x[8 * c + 6], x[8 * c + 7]));
        }
        fence_proxy_async_smem();
        __syncthreads();
        if (tid == 0) {
          bulk_store(a.e + (size_t)unit * TokenTc::E_BYTES, base + S::OFF_KQ, TokenTc::E_BYTES);
          bulk_store(a.p + (size_t)unit * TokenTc::P_BYTES, base + S::OFF_T, TokenTc::P_BYTES);
          tma_store_commit();
          tma_store_wait_all<0>();
        }
      }
    }
  } else if (!ok && tid == 0) {
    mbar_drain(bar_load, 0);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 128);
  }
}

// ---------------------------------------------------------------------------------------------- chunk after chunk
// One CTA per (sequence, head).  Everything is transposed: value channels are the rows (lanes) of tensor memory, so S, X
// and O keep one row per thread and both factors a product needs from the previous one (the parts of S, the parts of X)
// are written by the threads that own the rows, as A operands in tensor memory: nothing of the recurrence passes
// through shared memory.  Roles: one thread feeds the loads (two stages, three groups of operands with their own
// barriers), one issues the MMAs, eight warps own the state (two threads a row: 64 key channels each), four write out.
struct TokenChain {
  static constexpr int STATE_WARPS = 8, OUT_WARPS = 4;
  static constexpr int THREADS = 64 + 32 * (STATE_WARPS + OUT_WARPS);
  static constexpr int OFF_K = 0, OFF_Q = 16384, OFF_V = 32768, OFF_E = 49152, OFF_P = 81920, OFF_F = 90112;
  static constexpr int STAGE = 91136;
  static constexpr int OFF_BAR = 2 * STAGE;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  // tensor memory columns
  static constexpr uint32_t S_HI = 0, S_LO = 64, DS = 128, D_K = 256, X_HI = 320, X_LO = 352, D_Q = 384, D_O = 448;
};

__global__ void __launch_bounds__(TokenChain::THREADS, 1)
token_chain_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ,
                   const __grid_constant__ CUtensorMap tmV, const TokenTcArgs a, tc::DevStatus ds) {
  using namespace tc;
  using S = TokenChain;
  constexpr int C = TokenTc::C, D = TokenTc::D;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* bp = smem_dyn + (base - smem_u32(smem_dyn));
  const TokenArgs& t = a.t;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = (int)(blockIdx.x % t.H), seq = (int)(blockIdx.x / t.H);

  long long start;
  int len;
  token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
  const int steps = (len + C - 1) / C;
  const long long place0 = start / C + seq;

  const uint32_t bar0 = base + S::OFF_BAR;
  enum { KQ = 0, V = 1, E = 2 };
  auto FULL = [&](int g, int st) { return bar0 + 8u * (g * 4 + st); };
  auto FREE = [&](int g, int st) { return bar0 + 8u * (g * 4 + 2 + st); };
  const uint32_t S_READY = bar0 + 96, DK_FULL = bar0 + 104, DQ_FULL = bar0 + 112, X_READY = bar0 + 120, DS_FULL = bar0 + 128,
                 DO_FULL = bar0 + 136, O_FREE = bar0 + 144;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bp + S::OFF_BAR + 160);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + S::OFF_BAR + 168);
  const WaitCtx wc(abort_flag, ds);
  // a whole warp waits, and goes on or gives up together (tensor memory is accessed by whole warps)
  auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, wc)) != 0; };

  if (threadIdx.x == 0) {
    for (int st = 0; st < 2; ++st) {
      for (int g = 0; g < 3; ++g) {
        mbar_init(FULL(g, st), 1);
        mbar_init(FREE(g, st), g == V ? S::STATE_WARPS + S::OUT_WARPS : 1);
      }
    }
    mbar_init(S_READY, S::STATE_WARPS);
    mbar_init(X_READY, S::STATE_WARPS);
    mbar_init(O_FREE, S::OUT_WARPS);
    mbar_init(DK_FULL, 1); mbar_init(DQ_FULL, 1); mbar_init(DS_FULL, 1); mbar_init(DO_FULL, 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ loads
    if (lane == 0) {
      const int hk = h / (t.H / t.Hk);
      uint32_t issued[3] = {0u, 0u, 0u};
      bool ok = true;
      for (int s = 0; s < steps && ok; ++s) {
        const int st = s & 1, row = (int)(start + (long long)s * C);
        const uint32_t at = base + st * S::STAGE, par = ((s >> 1) & 1) ^ 1;
        const size_t unit = (size_t)(place0 + s) * t.H + h;
        if (s >= 2 && !(ok = mbar_wait(FREE(KQ, st), par, wc))) break;
        mbar_arrive_expect_tx(FULL(KQ, st), 32768);
        tma_load_2d(at + S::OFF_K, &tmK, FULL(KQ, st), hk * 128, row);
        tma_load_2d(at + S::OFF_K + 8192, &tmK, FULL(KQ, st), hk * 128 + 64, row);
        tma_load_2d(at + S::OFF_Q, &tmQ, FULL(KQ, st), hk * 128, row);
        tma_load_2d(at + S::OFF_Q + 8192, &tmQ, FULL(KQ, st), hk * 128 + 64, row);
        issued[KQ] = s + 1;
        if (s >= 2 && !(ok = mbar_wait(FREE(V, st), par, wc))) break;
        mbar_arrive_expect_tx(FULL(V, st), 16384 + TokenTc::F_BYTES);
        tma_load_2d(at + S::OFF_V, &tmV, FULL(V, st), h * 128, row);
        bulk_load(at + S::OFF_F, a.f + unit * TokenTc::F_BYTES, TokenTc::F_BYTES, FULL(V, st));
        issued[V] = s + 1;
        if (s >= 2 && !(ok = mbar_wait(FREE(E, st), par, wc))) break;
        mbar_arrive_expect_tx(FULL(E, st), TokenTc::E_BYTES + TokenTc::P_BYTES);
        bulk_load(at + S::OFF_E, a.e + unit * TokenTc::E_BYTES, TokenTc::E_BYTES, FULL(E, st));
        bulk_load(at + S::OFF_P, a.p + unit * TokenTc::P_BYTES, TokenTc::P_BYTES, FULL(E, st));
        issued[E] = s + 1;
      }
      // Whoever gives up, and when: copies in flight get a bounded chance to land before the CTA retires.
      for (int g = 0; g < 3; ++g) mbar_drain_ring(FULL(g, 0), 2, issued[g]);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint32_t id64 = make_idesc_bf16(128, 64, false, false), id128 = make_idesc_bf16(128, 128, false, false);
      for (int s = 0; s < steps; ++s) {
        const int st = s & 1;
        const uint32_t at = base + st * S::STAGE, par = (s >> 1) & 1;
        if (!mbar_wait(FULL(KQ, st), par, wc) || !mbar_wait(S_READY, s & 1, wc)) break;
        tc_fence_after_sync();
        // S K^T, small part first
#pragma unroll
        for (int part = 1; part >= 0; --part)
#pragma unroll
          for (int k = 0; k < 8; ++k)
            mma_bf16_ts(tmem + S::D_K, tmem + (part ? S::S_LO : S::S_HI) + k * 8,
                        make_smem_desc(at + S::OFF_K + (k >> 2) * 8192 + (k & 3) * 32, 16, 1024), id64, part == 1 && k == 0 ? 0u : 1u);
        mma_commit(DK_FULL);
        if (s > 0) {
          if (!mbar_wait(O_FREE, (s - 1) & 1, wc)) break;
          tc_fence_after_sync();
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          mma_bf16_ts(tmem + S::D_Q, tmem + S::S_HI + k * 8,
                      make_smem_desc(at + S::OFF_Q + (k >> 2) * 8192 + (k & 3) * 32, 16, 1024), id64, k ? 1u : 0u);
        mma_commit(DQ_FULL);
        mma_commit(FREE(KQ, st));
        if (!mbar_wait(FULL(E, st), par, wc) || !mbar_wait(X_READY, s & 1, wc)) break;
        tc_fence_after_sync();
        // X^T E^T: low X high E, high X low E, high X high E
#pragma unroll
        for (int term = 0; term < 3; ++term)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16_ts(tmem + S::DS, tmem + (term == 0 ? S::X_LO : S::X_HI) + k * 8,
                        make_smem_desc(at + S::OFF_E + (term == 1 ? TokenTc::E_PART : 0) + k * 32, 16, 1024), id128,
                        term || k ? 1u : 0u);
        mma_commit(DS_FULL);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16_ts(tmem + S::D_O, tmem + S::X_HI + k * 8, make_smem_desc(at + S::OFF_P + k * 32, 16, 1024), id64, k ? 1u : 0u);
        mma_commit(DO_FULL);
        mma_commit(FREE(E, st));
      }
    }
  } else if (warp < 2 + S::STATE_WARPS) {
    // ------------------------------------------------------------------ state
    const int qd = warp & 3, half = (warp - 2) >> 2;
    const int row = qd * 32 + lane;                   // value channel
    const uint32_t tl = tmem + ((uint32_t)(qd * 32) << 16);
    uint64_t sv[32];                                  // S[row][64 half ..], two to a register pair
    {
      const float* src = t.state_in ? t.state_in + (((size_t)seq * t.H + h) * D + row) * D + half * 64 : nullptr;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float4 x = src ? *reinterpret_cast<const float4*>(src + 4 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
        sv[2 * e] = f2_pack(x.x, x.y);
        sv[2 * e + 1] = f2_pack(x.z, x.w);
      }
    }
    auto publish = [&]() {
#pragma unroll
      for (int part = 0; part < 2; ++part) {          // 32 key channels at a time: fewer live registers
        float hi[16], lo[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          uint32_t u, v;
          split2_pair(sv[part * 16 + e], u, v);
          hi[e] = __uint_as_float(u);
          lo[e] = __uint_as_float(v);
        }
        tmem_st16(tl + S::S_HI + half * 32 + part * 16, hi);
        tmem_st16(tl + S::S_LO + half * 32 + part * 16, lo);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive_warp(S_READY);
    };
    if (steps > 0) publish();
    for (int s = 0; s < steps; ++s) {
      const int st = s & 1;
      const int n = min(C, len - s * C) - half * 32;  // tokens of this half that exist
      const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(bp + st * S::STAGE + S::OFF_V) + half * 32 * D + row;
      const float* f = reinterpret_cast<const float*>(bp + st * S::STAGE + S::OFF_F);
      if (!warp_wait(FULL(V, st), (s >> 1) & 1)) break;
      const float whole = f[128];
      if (!warp_wait(DK_FULL, s & 1)) break;
      tc_fence_after_sync();
      float x[32];
      tmem_ld32(tl + S::D_K + half * 32, x);
      tmem_wait_ld();
      float hi[16], lo[16];
#pragma unroll
      for (int j = 0; j < 32; j += 4) {
        const float4 fj = *reinterpret_cast<const float4*>(f + half * 32 + j);
        const float e[4] = {fj.x, fj.y, fj.z, fj.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j + i] = fmaf(-e[i], x[j + i], __bfloat162float(v[(j + i) * D]));
        if (n < C / 2) {                              // rows behind the sequence: whatever they hold, X is zero there
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (j + i >= n) x[j + i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          uint32_t p, q;
          split2_pair(f2_pack(x[j + i], x[j + i + 1]), p, q);
          hi[(j + i) / 2] = __uint_as_float(p);
          lo[(j + i) / 2] = __uint_as_float(q);
        }
      }
      tmem_st16(tl + S::X_HI + half * 16, hi);
      tmem_st16(tl + S::X_LO + half * 16, lo);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive_warp(X_READY);
      mbar_arrive_warp(FREE(V, st));
      if (!warp_wait(DS_FULL, s & 1)) break;
      tc_fence_after_sync();
      const uint64_t w2 = f2_pack(whole, whole);
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        tmem_ld32(tl + S::DS + half * 64 + part * 32, x);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[part * 16 + e] = fma2(w2, sv[part * 16 + e], f2_pack(x[2 * e], x[2 * e + 1]));
      }
      if (s + 1 < steps) publish();
    }
    if (t.state_out) {
      float* dst = t.state_out + (((size_t)seq * t.H + h) * D + row) * D + half * 64;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float4 x;
        f2_unpack(sv[2 * e], x.x, x.y);
        f2_unpack(sv[2 * e + 1], x.z, x.w);
        *reinterpret_cast<float4*>(dst + 4 * e) = x;
      }
    }
  } else {
    // ------------------------------------------------------------------ output: lanes are value channels, 64 bytes a warp and token
    const int qd = warp & 3;
    const uint32_t tl = tmem + ((uint32_t)(qd * 32) << 16);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(t.out) + start * t.out_stride + h * D + qd * 32 + lane;
    for (int s = 0; s < steps; ++s) {
      const int st = s & 1;
      const int n = min(C, len - s * C);
      const float* f = reinterpret_cast<const float*>(bp + st * S::STAGE + S::OFF_F) + 64;
      if (!warp_wait(FULL(V, st), (s >> 1) & 1) || !warp_wait(DQ_FULL, s & 1)) break;
      tc_fence_after_sync();
      float o[64];
      tmem_ld32(tl + S::D_Q, *reinterpret_cast<float(*)[32]>(o));
      tmem_ld32(tl + S::D_Q + 32, *reinterpret_cast<float(*)[32]>(o + 32));
      tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 64; j += 4) {
        const float4 e = *reinterpret_cast<const float4*>(f + j);
        o[j] *= e.x; o[j + 1] *= e.y; o[j + 2] *= e.z; o[j + 3] *= e.w;
      }
      mbar_arrive_warp(FREE(V, st));
      if (!warp_wait(DO_FULL, s & 1)) break;
      tc_fence_after_sync();
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        float x[32];
        tmem_ld32(tl + S::D_O + part * 32, x);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 32; ++j) o[part * 32 + j] += x[j];
      }
      tc_fence_before_sync();
      mbar_arrive_warp(O_FREE);
#pragma unroll
      for (int j = 0; j < 64; ++j)
        if (j < n) out[j * t.out_stride] = __float2bfloat16_rn(o[j]);
      out += C * t.out_stride;
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace vdn
