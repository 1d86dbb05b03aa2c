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
// Precision.  K and Q are bf16 as given and enter exactly.  Every other factor -- S, X, E, P, M, the triangular inverse -- is fp32 and
// enters its product as two bf16 parts (16 bits; products of the two low parts are left out: 2^-16 of the whole),
// accumulated in fp32; S itself is carried in fp32 registers.  One part would do for what only the rounded output sees where keys
// differ (read-out off by 3.4e-3, 1.7e-3 of which is its rounding), but not where they are alike and beta is near 1, where
// M times the inverse cancels: 2.3e-2 with one key throughout, 1.1e-1 with keys of length 1.2; 1.7e-3 everywhere with two.
// They cost 10 % (65536 tokens x 32 heads, a call: 1.43 -> 1.59 ms).
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
  static constexpr int P_PART = C * C * 2, P_BYTES = 2 * P_PART;
  // per-token factors: e^G r [64], scale r_q e^G [64], e^{G_C}, padding
  static constexpr int F_FLOATS = 132, F_BYTES = F_FLOATS * 4;
};

struct TokenTcArgs : TokenParts {
  TokenArgs t;
  unsigned char* e;          // [places * H] E_BYTES
  unsigned char* p;          // ... P_BYTES
  unsigned char* f;          // ... F_BYTES
  int places;                // of chunks
  int* order;                // [S] the sequences, longest first, or null: as they come
};

// More chains than SMs run one after another on an SM; the longest ones first, or the last to start would end long after
// the others (13 prompts of 0 .. 1244 tokens, 32 heads: 100 -> 87 us).  Lengths stay on the device, so a CTA of the
// first kernel ranks them, a thread to a sequence.
constexpr int kOrderMax = 256;
__device__ __forceinline__ void token_order(const TokenArgs& t, int* order, int* lens) {
  const int s = threadIdx.x;
  long long start;
  if (s < t.S) token_range(t.cu_seqlens, s, t.per, t.n_tokens, start, lens[s]);
  __syncthreads();
  if (s < t.S) {
    const int own = lens[s];
    int rank = 0;
    for (int j = 0; j < t.S; ++j) rank += lens[j] > own || (lens[j] == own && j < s);
    order[rank] = s;
  }
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

// 32 lanes x 8 consecutive columns.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float* r) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}

__device__ __forceinline__ void tmem_st4(uint32_t taddr, const float* r) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};"
               ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3])
               : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
               : "r"(taddr)
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

// x = hi + lo + rest, |rest| <= 2^-16 |x|, both parts rounded to nearest, two neighbours packed.  The packed conversion takes
// two cycles a warp and keeps NaN (rounding the bit pattern by an integer addition would turn 0x7FFFFFFF into -0):
// 7 cycles a pair in all, against 12 for Dekker's splitting in packed fp32 arithmetic.
__device__ __forceinline__ void split2_pair(float x0, float x1, uint32_t& hi, uint32_t& lo) {
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(x1), "f"(x0));
  const float r0 = x0 - __uint_as_float(hi << 16), r1 = x1 - __uint_as_float(hi & 0xFFFF0000u);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(r1), "f"(r0));
}
// The same in packed fp32 arithmetic: these kernels are short of issue slots.
__device__ __forceinline__ void split2_pair(uint64_t x, uint32_t& hi, uint32_t& lo) {
  float x0, x1, r0, r1;
  f2_unpack(x, x0, x1);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(x1), "f"(x0));
  f2_unpack(f2_fma(f2_pack(__uint_as_float(hi << 16), __uint_as_float(hi & 0xFFFF0000u)), f2_pack(-1.f, -1.f), x), r0, r1);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(r1), "f"(r0));
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

}  // namespace tc

// ---------------------------------------------------------------------------------------------- chunk operators
// One CTA (eight warps) per (place, head).  [K; Q] K^T is one MMA chain with the keys in rows 0..63 and the queries in rows
// 64..127 of one operand, so that lane i of tensor memory holds row i of K K^T and lane 64 + i row i of Q K^T.
// The inverse of the unit lower triangular I + L is formed in fp32 in shared memory, block by block: the four 16 x 16 blocks on
// the diagonal by forward substitution (a warp to a block, a lane to a column, 16 rows in registers), then pairs of
// blocks are merged, [T11 0; -T22 L21 T11, T22], to 32 and to 64 rows, all threads at once.  A thread to a column over all 64
// rows needs no products, but 2016 steps in straight line: half as fast again, most of it waiting for
// instructions.  Everything that could be a long straight line is a loop over 16 columns for the same reason.
// Measured on 65536 tokens x 32 heads (33 000 chunks): 724 us, 3.7 TB/s of the 81 KB a chunk reads and writes; four CTAs an SM use about half of
// the issue slots and two thirds of the shared-memory pipe (ncu) and wait at barriers for the rest.
struct TokenPrep {
  static constexpr int THREADS = 256, CTAS = 4;       // a CTA's phases are short and end at barriers: four of them side by side
  // [K; Q]: two 64-channel boxes of 128 rows, the queries in their lower halves.  Once the queries' product is formed, the
  // two parts of M take the queries' places; in the end the two parts of E take all of it.
  static constexpr int OFF_KQ = 0, OFF_M = 8192, OFF_M_LOW = 24576;
  // L and its inverse; then the inverse times beta, high and low (for P), and the same times factors (for E); then P
  static constexpr int OFF_T = 32768;
  static constexpr int L_PITCH = 68, W_PITCH = 36;    // floats: 16-byte rows, lanes' rows four banks apart
  static constexpr int OFF_W = OFF_T + 64 * L_PITCH * 4;   // products on the way to the inverse
  // per token, exponents in units of ln 2: from the start of its 16 tokens; back to it; to their end; factor of a column as a whole;
  // distances between blocks of 16 (all these are used up when W grows over them); to the chunk's end (later the weight
  // r e^{G_C - G}); from the chunk's start; beta; r of keys and queries.  LOW: what their rounding to fp32 left, plus a key's log2 r
  static constexpr int F_UP = 0, F_UP_LOW = 64, F_DOWN = 128, F_DOWN_LOW = 192, F_END = 256, F_END_LOW = 320, F_COL = 384, F_DIST = 448,
                       F_LAST = 464, F_ALL = 528, F_BETA = 592, F_R = 656, F_FLOATS = 784;
  static constexpr int OFF_F = OFF_W + 32 * W_PITCH * 4 - F_LAST * 4;
  static constexpr int OFF_BAR = OFF_F + F_FLOATS * 4;
  static constexpr int SMEM_BYTES = OFF_BAR + 64 + 1024;
};

// c += A B for one 16 x 8 tile of small fp32 matrices in shared memory (row-major, pitches in floats), 8 `ksteps` deep, on the
// warp-level tensor instruction: each factor as two tf32 parts (the instruction looks at the upper 19 bits), low times low left
// out: 2^-20 of a product.  A 32-row merge is 14 of these steps; with one multiply-add a thread and LDS.128 for two
// operands it kept the shared-memory pipe 80 % busy.
__device__ __forceinline__ void tile_product(float (&c)[4], const float* A, int pa, const float* B, int pb, int ksteps) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  const float* ar = A + g * pa + t;
  const float* br = B + t * pb + g;
#pragma unroll 2
  for (int k = 0; k < ksteps; ++k) {
    const float av[4] = {ar[0], ar[8 * pa], ar[4], ar[8 * pa + 4]}, bv[2] = {br[0], br[4 * pb]};
    uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ah[i] = __float_as_uint(av[i]) & 0xFFFFE000u;
      al[i] = __float_as_uint(av[i] - __uint_as_float(ah[i]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bh[i] = __float_as_uint(bv[i]) & 0xFFFFE000u;
      bl[i] = __float_as_uint(bv[i] - __uint_as_float(bh[i]));
    }
    auto mma = [&](const uint32_t (&x)[4], const uint32_t (&y)[2]) {
      asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                   : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                   : "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(y[0]), "r"(y[1]));
    };
    mma(al, bh);
    mma(ah, bl);
    mma(ah, bh);
    ar += 8;
    br += 8 * pb;
  }
}
__device__ __forceinline__ void tile_store(float* D, int pd, float sign, const float (&c)[4]) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  *reinterpret_cast<float2*>(D + g * pd + 2 * t) = make_float2(sign * c[0], sign * c[1]);
  *reinterpret_cast<float2*>(D + (g + 8) * pd + 2 * t) = make_float2(sign * c[2], sign * c[3]);
}

__global__ void __launch_bounds__(TokenPrep::THREADS, TokenPrep::CTAS)
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
  const int h = (int)(blockIdx.x % (unsigned)t.H);
  const int place = (int)(blockIdx.x / (unsigned)t.H);

  const uint32_t bar_load = base + S::OFF_BAR, bar_mma = bar_load + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bp + S::OFF_BAR + 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + S::OFF_BAR + 24);
  int* where = reinterpret_cast<int*>(bp + S::OFF_BAR + 32);      // first row, tokens (0: no chunk has this place)
  const WaitCtx wc(abort_flag, ds);
  float* fs = reinterpret_cast<float*>(bp + S::OFF_F);
  let_next_kernel_start();
  if (place == a.places) {                            // one CTA behind those of the chunks
    token_order(t, a.order, reinterpret_cast<int*>(bp));
    return;
  }

  if (warp == 0) {
    const int seq = token_seq_of(t, place, C);
    if (lane == 0) {
      long long start;
      int len;
      token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
      const long long chunk = place - (start / C + seq), row0 = start + chunk * C;
      const int n = chunk < 0 || chunk * C >= len ? 0 : min(C, len - (int)(chunk * C));
      where[0] = (int)row0;
      where[1] = n;
      mbar_init(bar_load, 1);
      mbar_init(bar_mma, 1);
      *abort_flag = 0;
      mbar_fence_init();
      if (n > 0) {
        const int ch = h / (t.H / t.Hk) * 128;
        mbar_arrive_expect_tx(bar_load, 32768);
        tma_load_2d(base, &tmK, bar_load, ch, (int)row0);
        tma_load_2d(base + 16384, &tmK, bar_load, ch + 64, (int)row0);
        tma_load_2d(base + 8192, &tmQ, bar_load, ch, (int)row0);
        tma_load_2d(base + 24576, &tmQ, bar_load, ch + 64, (int)row0);
      }
    }
  }
  __syncthreads();
  const int row0 = where[0], n = where[1];
  if (n == 0) return;
  if (warp == 1) {
    // Running sum of the decay, in 64 bits and units of ln 2.  What is kept are differences, each rounded once: to the end of 16
    // tokens, between blocks, to the ends of the chunk; and within 16 tokens as two numbers each, because there the distances
    // of two tokens to the start of the 16 are subtracted: after a few strong decays (a reset counts 150) they are in the hundreds
    // and the difference that matters is small (14 resets and two ordinary tokens: 1.2e-4 off with one number).  A token's log decay
    // counts down to -104 (e^-104 is 0 in fp32), so that -infinity leaves the differences finite.
    double x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * lane + i;
      const float g = j < n && t.log_alpha ? t.log_alpha[(size_t)(row0 + j) * t.H + h] : 0.f;
      x[i] = (g < -104.f ? -104.0 : (double)g) * 1.4426950408889634074;
    }
    double sum = x[0] + x[1];
    const double own = sum;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
      const double y = __shfl_up_sync(0xFFFFFFFFu, sum, m);
      if (lane >= m) sum += y;
    }
    const double end = __shfl_sync(0xFFFFFFFFu, sum, lane | 7);          // of the lane's 16 tokens
    double from = __shfl_sync(0xFFFFFFFFu, sum, (lane & 24) - 1);        // of those before
    if (lane < 8) from = 0.0;
    const double all = __shfl_sync(0xFFFFFFFFu, sum, 31);
    const double g[2] = {sum - own + x[0], sum};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = 2 * lane + i;
      const float up = (float)(g[i] - from), low = (float)(g[i] - from - up);
      fs[S::F_UP + j] = up;
      fs[S::F_UP_LOW + j] = low;
      fs[S::F_DOWN + j] = -up;
      fs[S::F_DOWN_LOW + j] = -low;
      fs[S::F_END + j] = (float)(end - g[i]);
      fs[S::F_LAST + j] = (float)(all - g[i]);
      fs[S::F_ALL + j] = (float)g[i];
    }
    const double e = __shfl_sync(0xFFFFFFFFu, sum, (lane & 3) * 8 + 7);  // end of block J = lane & 3
    const double b = __shfl_sync(0xFFFFFFFFu, sum, max(((lane >> 2) & 3) * 8 - 1, 0));   // end of the block before I = lane / 4
    if (lane < 16) fs[S::F_DIST + lane] = (float)(b - e);                // used for J < I
  } else if (warp == 2 || warp == 3) {
    const int j = tid - 64;
    fs[S::F_BETA + j] = j < n ? t.beta[(size_t)(row0 + j) * t.H + h] : 0.f;
  } else if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 128);
    tmem_relinquish();
  }
  // two warps share a quarter of the lanes and divide the columns between them
  const int qd = warp & 3, part = warp >> 2;
  const int rowid = qd * 32 + lane;                   // lane of tensor memory: a key, or 64 + a query, or a channel
  bool ok = mbar_wait(bar_load, 0, wc);
  if (n < C && ok) {
    // keys behind the sequence are the next one's (or nothing's): they must not enter a sum, not even times zero
    for (int e = tid; e < (C - n) * 16; e += S::THREADS) {
      const int r = n + e / 16, c = e % 16;
      *reinterpret_cast<uint4*>(bp + (c >> 3) * 16384 + r * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
  }
  tc_fence_before_sync();
  if (!__syncthreads_or(!ok)) {
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const uint32_t lanes = tmem + ((uint32_t)(qd * 32) << 16);
    if (tid == 0) {
      constexpr uint32_t idesc = make_idesc_bf16(128, 64, false, false);
      const uint64_t d = make_smem_desc(base, 16, 1024);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint64_t dk = d + ((k >> 2) * (16384 >> 4) + (k & 3) * 2);
        mma_bf16_ss(tmem, dk, dk, idesc, k ? 1u : 0u);
      }
      mma_commit(bar_mma);
    }
    float ss = 1.f;
    if (t.l2_eps > 0.f) {                             // two lanes a row, 64 channels each
      const int r = tid >> 1;
      ss = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 w = *reinterpret_cast<const uint4*>(bp + (tid & 1) * 16384 + r * 128 + ((c ^ (r & 7) ^ ((tid & 1) << 2)) << 4));
        const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = __uint_as_float(v[e] << 16), hi = __uint_as_float(v[e] & 0xFFFF0000u);
          ss = fmaf(lo, lo, fmaf(hi, hi, ss));
        }
      }
      ss += __shfl_xor_sync(0xFFFFFFFFu, ss, 1);
      ss = rsqrtf(ss + t.l2_eps);
    }
    if (!(tid & 1)) {
      const int r = tid >> 1;
      fs[S::F_R + r] = ss;
      if (r < 64) {                                   // a key's r goes with its column's exponents
        const float lg = __log2f(ss);
        fs[S::F_DOWN_LOW + r] += lg;
        fs[S::F_END_LOW + r] = lg;
        fs[S::F_COL + r] = exp2_fast(fs[S::F_END + r] + lg);
        fs[S::F_LAST + r] = ss * exp2_fast(fs[S::F_LAST + r]);
      }
    }
    ok = mbar_wait(bar_mma, 0, wc);
    if (!__syncthreads_or(!ok)) {
      tc_fence_after_sync();
      const bool is_q = qd >= 2;
      const int i = rowid & 63;                       // token of this thread's row
      const float norm = fs[S::F_R + rowid], up = fs[S::F_UP + i], up_low = fs[S::F_UP_LOW + i];
      const float row = is_q ? t.scale * norm : fs[S::F_BETA + i] * norm;
      const int last = is_q ? i : i - 1;              // L is strictly lower, M has its diagonal
      float* L = reinterpret_cast<float*>(bp + S::OFF_T);
      constexpr int LOW = S::OFF_M_LOW - S::OFF_M;
      static_assert(S::F_DOWN_LOW - S::F_DOWN == S::F_END_LOW - S::F_END, "");
#pragma unroll 1
      for (int jb = part * 16; jb < 64; jb += 32) {
        unsigned char* m0 = bp + S::OFF_M + i * 128 + (((jb / 8) ^ (i & 7)) << 4);
        unsigned char* m1 = bp + S::OFF_M + i * 128 + (((jb / 8 + 1) ^ (i & 7)) << 4);
        if (jb > (i | 31)) {                          // nothing of this warp's rows is this far right
          if (is_q)
            *reinterpret_cast<uint4*>(m0) = *reinterpret_cast<uint4*>(m1) = *reinterpret_cast<uint4*>(m0 + LOW) =
                *reinterpret_cast<uint4*>(m1 + LOW) = make_uint4(0, 0, 0, 0);
          continue;
        }
        float x[16];
        tmem_ld16(lanes + jb, x);
        tmem_wait_ld();
        if (jb + 16 <= (i & 32)) {
          // the warp's rows all lie behind these 16 columns: e^{G_i - G_j} is a factor of the row, from the columns' end on, times
          // a factor of the column, up to their end, both at most 1
          const float f = row * exp2_fast(up + fs[S::F_DIST + (i >> 4) * 4 + (jb >> 4)]);
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 c = *reinterpret_cast<const float4*>(fs + S::F_COL + jb + j);
            x[j] *= f * c.x; x[j + 1] *= f * c.y; x[j + 2] *= f * c.z; x[j + 3] *= f * c.w;
          }
        } else {
          // the row's own 16 columns (exponents from their start), or the 16 before them (the columns' end is the rows' start)
          const float* col = fs + ((i >> 4) == (jb >> 4) ? S::F_DOWN : S::F_END) + jb;
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const float4 c = *reinterpret_cast<const float4*>(col + j), r = *reinterpret_cast<const float4*>(col + (S::F_END_LOW - S::F_END) + j);
            const float c4[4] = {c.x, c.y, c.z, c.w}, r4[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[j + e] = jb + j + e <= last ? row * exp2_fast((up + c4[e]) + (up_low + r4[e])) * x[j + e] : 0.f;
          }
        }
        if (is_q) {
          uint32_t hi[8], lo[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) split2_pair(x[2 * e], x[2 * e + 1], hi[e], lo[e]);
          *reinterpret_cast<uint4*>(m0) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(m1) = make_uint4(hi[4], hi[5], hi[6], hi[7]);
          *reinterpret_cast<uint4*>(m0 + LOW) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          *reinterpret_cast<uint4*>(m1 + LOW) = make_uint4(lo[4], lo[5], lo[6], lo[7]);
        } else {
#pragma unroll
          for (int j = 0; j < 16; j += 4)
            *reinterpret_cast<float4*>(L + i * S::L_PITCH + jb + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
        }
      }
      const size_t unit = (size_t)place * t.H + h;
      if (part == 0) {
        float* f = reinterpret_cast<float*>(a.f + unit * TokenTc::F_BYTES);
        f[rowid] = exp2_fast(fs[S::F_ALL + i]) * (is_q ? t.scale * norm : norm);   // keys' factors, then the queries'
        if (tid == 0) f[128] = exp2_fast(fs[S::F_ALL + 63]);
      }
      // ---- inverse: the blocks on the diagonal, in place, by the four warps that formed L (the other four form M meanwhile)
      if (!is_q) {
        named_barrier_sync(1, 128);
        float* Lb = L + ((warp & 1) + 2 * part) * 16 * (S::L_PITCH + 1);
        const int c = lane & 15;
        float y[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float s0 = 0.f, s1 = 0.f;
#pragma unroll
          for (int j = 0; j < r; j += 4) {
            const float4 l = *reinterpret_cast<const float4*>(Lb + r * S::L_PITCH + j);
            s0 = fmaf(l.x, y[j], s0);
            s1 = fmaf(l.y, y[j + 1], s1);
            s0 = fmaf(l.z, y[j + 2], s0);
            s1 = fmaf(l.w, y[j + 3], s1);
          }
          y[r] = (r == c ? 1.f : 0.f) - (s0 + s1);
        }
        __syncwarp();
        if (lane < 16) {
#pragma unroll
          for (int r = 0; r < 16; ++r) Lb[r * S::L_PITCH + c] = y[r];
        }
      }
      __syncthreads();
      float* W = reinterpret_cast<float*>(bp + S::OFF_W);
      if (warp < 4) {
        // ---- pairs of 16: W = L21 T11, then T21 = -T22 W;  a warp to eight columns of a pair, which need nobody else's W
        float* A = L + (warp >> 1) * 32 * (S::L_PITCH + 1);
        float* Wp = W + warp * 16 * 8;
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        tile_product(c, A + 16 * S::L_PITCH, S::L_PITCH, A + (warp & 1) * 8, S::L_PITCH, 2);
        tile_store(Wp, 8, 1.f, c);
        __syncwarp();
        c[0] = c[1] = c[2] = c[3] = 0.f;
        tile_product(c, A + 16 * S::L_PITCH + 16, S::L_PITCH, Wp, 8, 2);
        // (the other warp of the pair still reads these rows of L: wait for it)
        named_barrier_sync(2, 128);
        tile_store(A + 16 * S::L_PITCH + (warp & 1) * 8, S::L_PITCH, -1.f, c);
      }
      __syncthreads();
      {
        // ---- the pair of 32: a warp to 16 rows and 8 columns
        const int m = (warp & 1) * 16, c0 = (warp >> 1) * 8;
        float* A = L + 32 * S::L_PITCH;
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        tile_product(c, A + m * S::L_PITCH, S::L_PITCH, L + c0, S::L_PITCH, 4);
        tile_store(W + m * S::W_PITCH + c0, S::W_PITCH, 1.f, c);
        __syncthreads();
        c[0] = c[1] = c[2] = c[3] = 0.f;
        tile_product(c, A + m * S::L_PITCH + 32, S::L_PITCH, W + c0, S::W_PITCH, m ? 4 : 2);   // T22 is lower triangular
        tile_store(A + m * S::L_PITCH + c0, S::L_PITCH, -1.f, c);
      }
      __syncthreads();
      // ---- operands: column c of the inverse times beta, 16 of its rows a thread; first as it is for P, then with the weights of E
      const int c = tid & 63, r0 = (tid >> 6) * 16;
      uint32_t hi[8], lo[8];
      auto operand = [&]() {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          unsigned char* at = bp + S::OFF_T + c * 128 + (((r0 / 8 + q) ^ (c & 7)) << 4);
          *reinterpret_cast<uint4*>(at) = make_uint4(hi[4 * q], hi[4 * q + 1], hi[4 * q + 2], hi[4 * q + 3]);
          *reinterpret_cast<uint4*>(at + 8192) = make_uint4(lo[4 * q], lo[4 * q + 1], lo[4 * q + 2], lo[4 * q + 3]);
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
      };
      {
        const bool zero = r0 < 32 && c >= 32;         // above the diagonal blocks: never written
        float y[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = zero ? 0.f : fs[S::F_BETA + c] * L[(r0 + r) * S::L_PITCH + c];
#pragma unroll
        for (int e = 0; e < 8; ++e) split2_pair(y[2 * e], y[2 * e + 1], hi[e], lo[e]);
        __syncthreads();                              // the inverse is read, the operand takes its place
        operand();
        if (tid == 0) {
          // P: rows 64..127 of the A operand are scale M, the rows before it (keys) are of no interest.  low high, high low, high high
          constexpr uint32_t idp = make_idesc_bf16(128, 64, false, false);
          const uint64_t dm = make_smem_desc(base + S::OFF_M - 8192, 16, 1024), dl = make_smem_desc(base + S::OFF_M_LOW - 8192, 16, 1024);
          const uint64_t dt = make_smem_desc(base + S::OFF_T, 16, 1024);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            mma_bf16_ss(tmem, dl + k * 2, dt + k * 2, idp, k ? 1u : 0u);
            mma_bf16_ss(tmem, dm + k * 2, dt + (8192 >> 4) + k * 2, idp, 1u);
            mma_bf16_ss(tmem, dm + k * 2, dt + k * 2, idp, 1u);
          }
          mma_commit(bar_mma);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 w = *reinterpret_cast<const float2*>(fs + S::F_LAST + r0 + 2 * e);
          split2_pair(w.x * y[2 * e], w.y * y[2 * e + 1], hi[e], lo[e]);
        }
      }
      ok = mbar_wait(bar_mma, 1, wc);
      if (!__syncthreads_or(!ok)) {
        operand();
        if (tid == 0) {
          // E [128 x 64] = K^T (M rows = channels, read MN-major) times the two parts
          constexpr uint32_t ide = make_idesc_bf16(128, 64, true, false);
          const uint64_t dk = make_smem_desc(base, 16384, 1024), dt = make_smem_desc(base + S::OFF_T, 16, 1024);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            mma_bf16_ss(tmem + 64, dk + (k & 3) * (2048 >> 4), dt + ((k >> 2) * (8192 >> 4) + (k & 3) * 2), ide, k ? 1u : 0u);
          mma_commit(bar_mma);
        }
        ok = mbar_wait(bar_mma, 0, wc);
      }
      if (!__syncthreads_or(!ok)) {
        tc_fence_after_sync();
#pragma unroll 1
        for (int jb = part * 32; jb < part * 32 + 32; jb += 16) {   // a row of E: a channel
          float x[16];
          tmem_ld16(lanes + 64 + jb, x);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) split2_pair(x[8 * c + 2 * e], x[8 * c + 2 * e + 1], hi[e], lo[e]);
            unsigned char* at = bp + S::OFF_KQ + rowid * 128 + (((jb / 8 + c) ^ (rowid & 7)) << 4);
            *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4*>(at + TokenTc::E_PART) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          }
          if (is_q) {
            tmem_ld16(lanes + jb, x);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) split2_pair(x[8 * c + 2 * e], x[8 * c + 2 * e + 1], hi[e], lo[e]);
              unsigned char* at = bp + S::OFF_T + i * 128 + (((jb / 8 + c) ^ (i & 7)) << 4);
              *reinterpret_cast<uint4*>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
              *reinterpret_cast<uint4*>(at + TokenTc::P_PART) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
          }
        }
        fence_proxy_async_smem();
        __syncthreads();
        if (tid == 0) {
          bulk_store(a.e + unit * TokenTc::E_BYTES, base + S::OFF_KQ, TokenTc::E_BYTES);
          bulk_store(a.p + unit * TokenTc::P_BYTES, base + S::OFF_T, TokenTc::P_BYTES);
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
    settle(smem_u32(const_cast<int*>(abort_flag)));
    tc_fence_after_sync();
    tmem_dealloc(*tmem_slot, 128);
  }
}

// ---------------------------------------------------------------------------------------------- chunk after chunk
// One CTA per (sequence, head), or per part of a long sequence.  Everything is transposed: value channels are the rows
// (lanes) of tensor memory, so S, X and O keep one row per thread and both factors a product needs from the previous one
// (the parts of S, the parts of X) are written by the threads that own the rows, as A operands in tensor memory: nothing of the
// recurrence passes through shared memory.  Roles: one thread feeds the loads (two stages, three groups of operands with
// their own barriers), one issues the MMAs of the recurrence and one those of the results, sixteen warps own the state (four
// threads a row: 32 key channels each), four write out.
//
// Measured: 2.3 us a chunk alone (4400 cycles: 830 S K^T, 830 X^T E^T, the rest the state warps' turns and the hand-overs);
// 65536 tokens x 32 heads, a chain after another on every SM: 675 us, 113 KB a chunk, 5.6 TB/s with what shared keys leave to DRAM.
struct TokenChain {
  static constexpr int STATE_WARPS = 16, OUT_WARPS = 4;
  static constexpr int RESULT_WARP = 2 + STATE_WARPS + OUT_WARPS;
  static constexpr int THREADS = 32 * (RESULT_WARP + 1);
  static constexpr int OFF_K = 0, OFF_Q = 16384, OFF_V = 32768, OFF_E = 49152, OFF_P = 81920, OFF_F = 98304;
  static constexpr int STAGE = 99328;
  static constexpr int OFF_O = 2 * STAGE;             // two tiles of results
  static constexpr int OFF_BAR = STAGE + OFF_F + TokenTc::F_BYTES;   // (where the second stage's last kilobyte is free)
  static constexpr int SMEM_BYTES = OFF_O + 2 * 16384 + 1024;
  static_assert(OFF_BAR % 8 == 0 && OFF_BAR + 192 <= OFF_O && SMEM_BYTES <= 227 * 1024, "");
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
  let_next_kernel_start();
  // this CTA's rows, first state and what becomes of its last one
  const int h = (int)blockIdx.x % t.H, x = (int)blockIdx.x / t.H;
  if (a.order) wait_for_kernel_before();              // it is that kernel's work
  const int seq = a.part > 0 ? token_seq_of(t, x, a.part) : a.order ? a.order[x] : x;
  long long start;
  int len;
  token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
  const int parts = token_parts(len, a.part);
  const int pos = a.part > 0 ? x - ((int)(start / a.part) + seq) : 0;
  if (pos < 0 || pos >= parts) { wait_for_kernel_before(); return; }   // a place that no part has
  const float* first = parts > 1 ? a.enter + ((size_t)x * t.H + h) * (D * D)
                                 : t.state_in ? t.state_in + ((size_t)seq * t.H + h) * (D * D) : nullptr;
  float* last = pos + 1 == parts && t.state_out ? t.state_out + ((size_t)seq * t.H + h) * (D * D) : nullptr;
  const long long place0 = start / C + seq + (long long)pos * (a.part / C);
  if (parts > 1) {
    start += (long long)pos * a.part;
    len = min(a.part, len - pos * a.part);
  }
  const int steps = (len + C - 1) / C;

  const uint32_t bar0 = base + S::OFF_BAR;
  enum { KQ = 0, V = 1, E = 2 };
  auto FULL = [&](int g, int st) { return bar0 + 8u * (g * 4 + st); };
  auto FREE = [&](int g, int st) { return bar0 + 8u * (g * 4 + 2 + st); };
  // the parts of S and of X are handed over in two halves each: the MMAs on the first run while the second is formed
  const uint32_t S_READY = bar0 + 96, X_READY = bar0 + 112, DK_FULL = bar0 + 128, DS_FULL = bar0 + 136, DO_FULL = bar0 + 144,
                 O_FREE = bar0 + 152, S_FREE = bar0 + 160;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bp + S::OFF_BAR + 168);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + S::OFF_BAR + 176);
  const WaitCtx wc(abort_flag, ds);
  // a whole warp waits, and goes on or gives up together (tensor memory is accessed by whole warps)
  auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, wc)) != 0; };

  if (threadIdx.x == 0) {
    for (int st = 0; st < 2; ++st) {
      for (int g = 0; g < 3; ++g) {
        mbar_init(FULL(g, st), 1);
        mbar_init(FREE(g, st), g == V ? S::STATE_WARPS + S::OUT_WARPS : g == E ? 2 : 1);
      }
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(S_READY + 8 * i, S::STATE_WARPS);
      mbar_init(X_READY + 8 * i, S::STATE_WARPS);
    }
    mbar_init(O_FREE, S::OUT_WARPS);
    mbar_init(S_FREE, 1); mbar_init(DK_FULL, 1); mbar_init(DS_FULL, 1); mbar_init(DO_FULL, 1);
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
  wait_for_kernel_before();
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
    // ------------------------------------------------------------------ MMAs of the recurrence
    if (lane == 0) {
      constexpr uint32_t id64 = make_idesc_bf16(128, 64, false, false), id128 = make_idesc_bf16(128, 128, false, false);
      // descriptors of the first stage; one step along K is 32 bytes, the other 64 channels a box further on
      const uint64_t dk0 = make_smem_desc(base + S::OFF_K, 16, 1024), de0 = make_smem_desc(base + S::OFF_E, 16, 1024);
      for (int s = 0; s < steps; ++s) {
        const int st = s & 1;
        const uint32_t par = (s >> 1) & 1;
        const uint64_t off = st ? S::STAGE >> 4 : 0;
        const uint64_t dk = dk0 + off, de = de0 + off;
        if (!mbar_wait(FULL(KQ, st), par, wc)) break;
        // S K^T: even steps of 16 key channels (the first half that the state warps hand over), then odd ones
        bool ok = true;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(ok = mbar_wait(S_READY + 8 * half, s & 1, wc))) break;
          tc_fence_after_sync();
#pragma unroll
          for (int k = half; k < 8; k += 2) {
            mma_bf16_ts(tmem + S::D_K, tmem + S::S_LO + k * 8, dk + ((k >> 2) * 512 + (k & 3) * 2), id64, k ? 1u : 0u);
            mma_bf16_ts(tmem + S::D_K, tmem + S::S_HI + k * 8, dk + ((k >> 2) * 512 + (k & 3) * 2), id64, 1u);
          }
        }
        if (!ok) break;
        mma_commit(DK_FULL);
        if (!mbar_wait(FULL(E, st), par, wc)) break;
        // X^T E^T, 32 tokens at a time: low X high E, high X low E, high X high E
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!(ok = mbar_wait(X_READY + 8 * half, s & 1, wc))) break;
          tc_fence_after_sync();
#pragma unroll
          for (int k = 2 * half; k < 2 * half + 2; ++k) {
            mma_bf16_ts(tmem + S::DS, tmem + S::X_LO + k * 8, de + k * 2, id128, k ? 1u : 0u);
            mma_bf16_ts(tmem + S::DS, tmem + S::X_HI + k * 8, de + ((TokenTc::E_PART >> 4) + k * 2), id128, 1u);
            mma_bf16_ts(tmem + S::DS, tmem + S::X_HI + k * 8, de + k * 2, id128, 1u);
          }
        }
        if (!ok) break;
        mma_commit(DS_FULL);
        mma_commit(FREE(E, st));
      }
    }
  } else if (warp < 2 + S::STATE_WARPS) {
    // ------------------------------------------------------------------ state
    const int qd = warp & 3, sl = (warp - 2) >> 2;    // lane quarter; quarter of the key channels and of the chunk's tokens
    const int row = qd * 32 + lane;                   // value channel
    const uint32_t tl = tmem + ((uint32_t)(qd * 32) << 16);
    float sv[32];                                     // S[row][32 sl ..]
    {
      const float* src = first ? first + (size_t)row * D + sl * 32 : nullptr;
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        const float4 x = src ? *reinterpret_cast<const float4*>(src + e) : make_float4(0.f, 0.f, 0.f, 0.f);
        sv[e] = x.x; sv[e + 1] = x.y; sv[e + 2] = x.z; sv[e + 3] = x.w;
      }
    }
    // columns 16 half .. of the thread's 32: one K step of the product
    auto publish = [&](int half) {
      float hl[16];                                   // high words, then low words
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t u, v;
        split2_pair(sv[16 * half + 2 * e], sv[16 * half + 2 * e + 1], u, v);
        hl[e] = __uint_as_float(u);
        hl[8 + e] = __uint_as_float(v);
      }
      tmem_st8(tl + S::S_HI + sl * 16 + half * 8, hl);
      tmem_st8(tl + S::S_LO + sl * 16 + half * 8, hl + 8);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive_warp(S_READY + 8 * half);
    };
    if (steps > 0) { publish(0); publish(1); }
    for (int s = 0; s < steps; ++s) {
      const int st = s & 1;
      const int n = min(C, len - s * C) - sl * 8;     // tokens from this warp's first on; it has 8 there and 8 half a chunk further on
      // what does not depend on the products is fetched while they run: V, two tokens to a register
      if (!warp_wait(FULL(V, st), (s >> 1) & 1)) break;
      const unsigned short* v = reinterpret_cast<const unsigned short*>(bp + st * S::STAGE + S::OFF_V) + sl * 8 * D + row;
      const float* f = reinterpret_cast<const float*>(bp + st * S::STAGE + S::OFF_F);
      uint32_t vv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int at = (j >> 2) * 32 + (j & 3) * 2;
        vv[j] = (uint32_t)v[at * D] | ((uint32_t)v[(at + 1) * D] << 16);
      }
      const float whole = f[128];
      if (!warp_wait(DK_FULL, s & 1)) break;
      tc_fence_after_sync();
      // (X^T P^T of the step before, which another thread issues, must be done with the old parts of X)
      if (s > 0) {
        if (!warp_wait(DO_FULL, (s - 1) & 1)) break;
        tc_fence_after_sync();
      }
      float x[16];
      tmem_ld8(tl + S::D_K + sl * 8, x);
      tmem_ld8(tl + S::D_K + 32 + sl * 8, x + 8);
      tmem_wait_ld();
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float hl[8];                                  // high words, then low words
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 fj = *reinterpret_cast<const float4*>(f + half * 32 + sl * 8 + j);
          float* y = x + half * 8 + j;
          const uint32_t v01 = vv[half * 4 + j / 2], v23 = vv[half * 4 + j / 2 + 1];
          y[0] = fmaf(-fj.x, y[0], __uint_as_float(v01 << 16));
          y[1] = fmaf(-fj.y, y[1], __uint_as_float(v01 & 0xFFFF0000u));
          y[2] = fmaf(-fj.z, y[2], __uint_as_float(v23 << 16));
          y[3] = fmaf(-fj.w, y[3], __uint_as_float(v23 & 0xFFFF0000u));
          if (n < 40) {                               // rows behind the sequence: whatever they hold, X is zero there
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (half * 32 + j + i >= n) y[i] = 0.f;
          }
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            uint32_t u, w;
            split2_pair(y[i], y[i + 1], u, w);
            hl[(j + i) / 2] = __uint_as_float(u);
            hl[4 + (j + i) / 2] = __uint_as_float(w);
          }
        }
        tmem_st4(tl + S::X_HI + half * 16 + sl * 4, hl);
        tmem_st4(tl + S::X_LO + half * 16 + sl * 4, hl + 4);
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive_warp(X_READY + 8 * half);
      }
      mbar_arrive_warp(FREE(V, st));
      if (!warp_wait(DS_FULL, s & 1)) break;
      tc_fence_after_sync();
      bool ok = true;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float d[16];
        tmem_ld16(tl + S::DS + sl * 32 + half * 16, d);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[half * 16 + e] = fmaf(whole, sv[half * 16 + e], d[e]);
        if (half == 0) {                     // S Q^T is done with the old parts of S (and, at the end, with Q's memory)
          if (!(ok = warp_wait(S_FREE, s & 1))) break;
          tc_fence_after_sync();
        }
        if (s + 1 < steps) publish(half);
      }
      if (!ok) break;
    }
    if (last) {
      // rows leave whole: through shared memory (the first stage's keys, queries, values and part of E, which no product reads
      // any more), 16-byte pieces in an order that keeps the banks apart.  Stored from the threads that own the rows, 512 bytes apart, it took 3 us.
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<float4*>(bp + row * 512 + (((sl * 8 + e) ^ lane) << 4)) =
            make_float4(sv[4 * e], sv[4 * e + 1], sv[4 * e + 2], sv[4 * e + 3]);
      named_barrier_sync(1, 32 * S::STATE_WARPS);
      const int tid = (warp - 2) * 32 + lane;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = (tid >> 5) + 16 * e;
        *reinterpret_cast<float4*>(last + (size_t)r * D + lane * 4) = *reinterpret_cast<const float4*>(bp + r * 512 + ((lane ^ (r & 31)) << 4));
      }
    }
  } else if (warp == S::RESULT_WARP) {
    // ------------------------------------------------------------------ MMAs of the results
    // Their own issuer: in the gaps that the recurrence leaves, and what they wait for (the accumulators being read) does not
    // hold the recurrence up.
    if (lane == 0) {
      constexpr uint32_t id64 = make_idesc_bf16(128, 64, false, false);
      const uint64_t dq0 = make_smem_desc(base + S::OFF_Q, 16, 1024), dp0 = make_smem_desc(base + S::OFF_P, 16, 1024);
      for (int s = 0; s < steps; ++s) {
        const int st = s & 1;
        const uint64_t off = st ? S::STAGE >> 4 : 0;
        // (DK_FULL: the keys, the queries and the parts of S are there, and the keys have been used)
        if (!mbar_wait(DK_FULL, s & 1, wc) || (s > 0 && !mbar_wait(O_FREE, (s - 1) & 1, wc))) break;
        tc_fence_after_sync();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          mma_bf16_ts(tmem + S::D_Q, tmem + S::S_LO + k * 8, dq0 + off + ((k >> 2) * 512 + (k & 3) * 2), id64, k ? 1u : 0u);
          mma_bf16_ts(tmem + S::D_Q, tmem + S::S_HI + k * 8, dq0 + off + ((k >> 2) * 512 + (k & 3) * 2), id64, 1u);
        }
        mma_commit(S_FREE);
        mma_commit(FREE(KQ, st));
        if (!mbar_wait(FULL(E, st), (s >> 1) & 1, wc) || !mbar_wait(X_READY, s & 1, wc) || !mbar_wait(X_READY + 8, s & 1, wc)) break;
        tc_fence_after_sync();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          mma_bf16_ts(tmem + S::D_O, tmem + S::X_LO + k * 8, dp0 + off + k * 2, id64, k ? 1u : 0u);
          mma_bf16_ts(tmem + S::D_O, tmem + S::X_HI + k * 8, dp0 + off + (TokenTc::P_PART >> 4) + k * 2, id64, 1u);
          mma_bf16_ts(tmem + S::D_O, tmem + S::X_HI + k * 8, dp0 + off + k * 2, id64, 1u);
        }
        mma_commit(DO_FULL);
        mma_commit(FREE(E, st));
      }
    }
  } else {
    // ------------------------------------------------------------------ output
    // Lanes are value channels: the tile is turned round in shared memory and leaves as whole rows of 256 bytes.
    // (Stored from here, 64 bytes a warp and token, it took 3300 cycles a chunk and held up the MMAs.)
    const int qd = warp & 3, tid = (warp - 2 - S::STATE_WARPS) * 32 + lane;
    const uint32_t tl = tmem + ((uint32_t)(qd * 32) << 16);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(t.out) + (start + 2 * (tid >> 4)) * t.out_stride + h * D + (tid & 15) * 8;
    for (int s = 0; s < steps; ++s) {
      const int st = s & 1;
      const int n = min(C, len - s * C);
      const float* f = reinterpret_cast<const float*>(bp + st * S::STAGE + S::OFF_F) + 64;
      unsigned char* tile = bp + S::OFF_O + st * 16384;
      // (one thread issues S Q^T, then X^T P^T: one barrier says that both are there)
      const bool ok = warp_wait(FULL(V, st), (s >> 1) & 1) && warp_wait(DO_FULL, s & 1);
      if (ok) {
        tc_fence_after_sync();
        // two tokens to a word: [token / 2][channel]
        uint32_t* col = reinterpret_cast<uint32_t*>(tile) + qd * 32 + lane;
#pragma unroll 1
        for (int jb = 0; jb < 64; jb += 32) {
          float x[32], y[32];
          tmem_ld32(tl + S::D_Q + jb, x);
          tmem_ld32(tl + S::D_O + jb, y);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            const float4 e = *reinterpret_cast<const float4*>(f + jb + j);
            col[(jb + j) / 2 * D] = bf16_pair(fmaf(e.x, x[j], y[j]), fmaf(e.y, x[j + 1], y[j + 1]));
            col[((jb + j) / 2 + 1) * D] = bf16_pair(fmaf(e.z, x[j + 2], y[j + 2]), fmaf(e.w, x[j + 3], y[j + 3]));
          }
        }
        tc_fence_before_sync();
        mbar_arrive_warp(O_FREE);
        mbar_arrive_warp(FREE(V, st));
      }
      if (named_barrier_or(2, 32 * S::OUT_WARPS, !ok)) break;
      // two tiles in turn: the next barrier comes after these reads, the next write to this tile after that
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int pair = (tid >> 4) + 8 * r;
        const uint4* w = reinterpret_cast<const uint4*>(tile + pair * 512 + (tid & 15) * 32);
        const uint4 u = w[0], v = w[1];
        __nv_bfloat16* dst = out + 16 * r * t.out_stride;
        if (2 * pair < n)
          *reinterpret_cast<uint4*>(dst) = make_uint4(__byte_perm(u.x, u.y, 0x5410), __byte_perm(u.z, u.w, 0x5410),
                                                      __byte_perm(v.x, v.y, 0x5410), __byte_perm(v.z, v.w, 0x5410));
        if (2 * pair + 1 < n)
          *reinterpret_cast<uint4*>(dst + t.out_stride) = make_uint4(__byte_perm(u.x, u.y, 0x7632), __byte_perm(u.z, u.w, 0x7632),
                                                                     __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x7632));
      }
      out += C * t.out_stride;
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    settle(smem_u32(const_cast<int*>(abort_flag)));
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// ---------------------------------------------------------------------------------------------- parts of a sequence
// Few long sequences would leave most SMs idle.  The rule is linear in the state, S_out = S_in M + J over any stretch, and the rows
// of S go their own ways, so M is what the same recurrence makes of the rows of the identity when nothing is written
// (V = 0).  A sequence is then cut into parts: token_compose_kernel runs all parts but the last side by side, from zero (J; the
// first part from the sequence's first state) and from the identity (M); token_join_kernel passes the state along the parts;
// token_chain_kernel runs all parts from the states they enter with.
//
// J and M of a part share a CTA: the same keys and operators, and two independent chains, so that the MMAs of one run
// while the state warps work on the other -- S K^T of J, of M, X^T E^T of J, of M, and under each the state warps' turn
// that it does not depend on (262144 tokens x 24 heads in 6 parts: 3.49 ms with a CTA to each, 2.23 ms so; the split into bf16
// parts on the packed fp32 pipe is a tenth of that; it is bound by issue slots, 12 000 instructions a step of both chains, 44 % of
// the slots used; 96 registers a thread and 108 bytes of spills).  Tensor memory holds both because each chain has two
// regions only: the parts of S, which X^T E^T overwrites (they are used up by then) and whose place the thread that owns a piece of
// the new state fills again, and S K^T, which the parts of X replace in the same way.
struct TokenCompose {
  static constexpr int STATE_WARPS = 16, THREADS = 64 + 32 * STATE_WARPS, STAGES = 3;
  static constexpr int OFF_K = 0, OFF_V = 16384, OFF_E = 32768, OFF_F = 65536, STAGE = 66560;
  static constexpr int OFF_BAR = STAGES * STAGE;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  // columns of a chain: 128 of S or X^T E^T (32 for each quarter of the key channels: 16 high words, 16 low ones), 64 of S K^T
  // or X (16 for each 16 tokens: 8 high words, 8 low ones)
  static constexpr uint32_t CHAIN = 192, D_K = 128;
};

__global__ void __launch_bounds__(TokenCompose::THREADS, 1)
token_compose_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const TokenTcArgs a,
                     tc::DevStatus ds) {
  using namespace tc;
  using S = TokenCompose;
  constexpr int C = TokenTc::C, D = TokenTc::D;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* bp = smem_dyn + (base - smem_u32(smem_dyn));
  const TokenArgs& t = a.t;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_kernel_start();
  const int h = (int)blockIdx.x % t.H, x = (int)blockIdx.x / t.H;
  const int seq = token_seq_of(t, x, a.part);
  long long start;
  int len;
  token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
  const int parts = token_parts(len, a.part);
  const int pos = x - ((int)(start / a.part) + seq);
  if (pos < 0 || pos + 1 >= parts) { wait_for_kernel_before(); return; }   // no part, or one that nobody follows
  const float* first = pos == 0 && t.state_in ? t.state_in + ((size_t)seq * t.H + h) * (D * D) : nullptr;
  const size_t comp = ((size_t)x * t.H + h) * (D * D);
  const long long place0 = start / C + seq + (long long)pos * (a.part / C);
  start += (long long)pos * a.part;
  const int steps = a.part / C;                       // all parts but the last are whole

  const uint32_t bar0 = base + S::OFF_BAR;
  auto FULL = [&](int st) { return bar0 + 8u * st; };
  auto FREE = [&](int st) { return bar0 + 8u * (S::STAGES + st); };
  // of chain c (0: J, 1: M)
  auto S_READY = [&](int c) { return bar0 + 64u + 8u * c; };
  auto DK_FULL = [&](int c) { return bar0 + 80u + 8u * c; };
  auto X_READY = [&](int c) { return bar0 + 96u + 8u * c; };
  auto DS_FULL = [&](int c) { return bar0 + 112u + 8u * c; };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bp + S::OFF_BAR + 128);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + S::OFF_BAR + 136);
  const WaitCtx wc(abort_flag, ds);
  auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, wc)) != 0; };

  if (threadIdx.x == 0) {
    for (int st = 0; st < S::STAGES; ++st) { mbar_init(FULL(st), 1); mbar_init(FREE(st), 1 + S::STATE_WARPS); }
    for (int c = 0; c < 2; ++c) {
      mbar_init(S_READY(c), S::STATE_WARPS);
      mbar_init(X_READY(c), S::STATE_WARPS);
      mbar_init(DK_FULL(c), 1);
      mbar_init(DS_FULL(c), 1);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  wait_for_kernel_before();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ loads
    if (lane == 0) {
      const int ch = h / (t.H / t.Hk) * 128;
      uint32_t issued = 0;
      for (int s = 0; s < steps; ++s) {
        const int st = s % S::STAGES, row = (int)(start + (long long)s * C);
        if (s >= S::STAGES && !mbar_wait(FREE(st), ((s / S::STAGES) & 1) ^ 1, wc)) break;
        const uint32_t at = base + st * S::STAGE;
        const size_t unit = (size_t)(place0 + s) * t.H + h;
        mbar_arrive_expect_tx(FULL(st), 32768 + TokenTc::E_BYTES + TokenTc::F_BYTES);
        tma_load_2d(at + S::OFF_K, &tmK, FULL(st), ch, row);
        tma_load_2d(at + S::OFF_K + 8192, &tmK, FULL(st), ch + 64, row);
        tma_load_2d(at + S::OFF_V, &tmV, FULL(st), h * 128, row);
        bulk_load(at + S::OFF_E, a.e + unit * TokenTc::E_BYTES, TokenTc::E_BYTES, FULL(st));
        bulk_load(at + S::OFF_F, a.f + unit * TokenTc::F_BYTES, TokenTc::F_BYTES, FULL(st));
        issued = s + 1;
      }
      mbar_drain_ring(FULL(0), S::STAGES, issued);    // copies in flight get a bounded chance to land before the CTA retires
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMAs
    if (lane == 0) {
      constexpr uint32_t id64 = make_idesc_bf16(128, 64, false, false), id128 = make_idesc_bf16(128, 128, false, false);
      const uint64_t dk0 = make_smem_desc(base + S::OFF_K, 16, 1024), de0 = make_smem_desc(base + S::OFF_E, 16, 1024);
      bool ok = true;
      for (int s = 0; s < steps && ok; ++s) {
        const int st = s % S::STAGES;
        const uint64_t off = (uint64_t)(st * (S::STAGE >> 4)), dk = dk0 + off, de = de0 + off;
        if (!mbar_wait(FULL(st), (s / S::STAGES) & 1, wc)) break;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (!(ok = ok && mbar_wait(S_READY(c), s & 1, wc))) break;
          tc_fence_after_sync();
          const uint32_t tc0 = tmem + c * S::CHAIN;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t sp = tc0 + (k >> 1) * 32 + (k & 1) * 8;
            mma_bf16_ts(tc0 + S::D_K, sp + 16, dk + ((k >> 2) * 512 + (k & 3) * 2), id64, k ? 1u : 0u);
            mma_bf16_ts(tc0 + S::D_K, sp, dk + ((k >> 2) * 512 + (k & 3) * 2), id64, 1u);
          }
          mma_commit(DK_FULL(c));
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if (!(ok = ok && mbar_wait(X_READY(c), s & 1, wc))) break;
          tc_fence_after_sync();
          const uint32_t tc0 = tmem + c * S::CHAIN, xp = tc0 + S::D_K;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            mma_bf16_ts(tc0, xp + k * 16 + 8, de + k * 2, id128, k ? 1u : 0u);
            mma_bf16_ts(tc0, xp + k * 16, de + ((TokenTc::E_PART >> 4) + k * 2), id128, 1u);
            mma_bf16_ts(tc0, xp + k * 16, de + k * 2, id128, 1u);
          }
          mma_commit(DS_FULL(c));
        }
        if (ok) mma_commit(FREE(st));
      }
    }
  } else {
    // ------------------------------------------------------------------ state
    const int qd = warp & 3, sl = (warp - 2) >> 2;    // lane quarter; quarter of the key channels and of the chunk's tokens
    const int row = qd * 32 + lane;                   // value channel
    const uint32_t tl = tmem + ((uint32_t)(qd * 32) << 16);
    uint64_t sv[2][16];                               // of both chains: S[row][32 sl ..], two to a register pair
    {
      const float* src = first ? first + (size_t)row * D + sl * 32 : nullptr;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float4 y = src ? *reinterpret_cast<const float4*>(src + 2 * e) : make_float4(0.f, 0.f, 0.f, 0.f);
        sv[0][e] = f2_pack(y.x, y.y);
        sv[0][e + 1] = f2_pack(y.z, y.w);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) sv[1][e] = f2_pack(sl * 32 + 2 * e == row ? 1.f : 0.f, sl * 32 + 2 * e + 1 == row ? 1.f : 0.f);
    }
    auto publish = [&](int c) {
      const uint32_t at = tl + c * S::CHAIN + sl * 32;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float hl[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t u, v;
          split2_pair(sv[c][8 * half + e], u, v);
          hl[e] = __uint_as_float(u);
          hl[8 + e] = __uint_as_float(v);
        }
        tmem_st8(at + half * 8, hl);
        tmem_st8(at + 16 + half * 8, hl + 8);
      }
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive_warp(S_READY(c));
    };
    publish(0);
    publish(1);
    bool ok = true;
    for (int s = 0; s < steps && ok; ++s) {
      const int st = s % S::STAGES;
      if (!warp_wait(FULL(st), (s / S::STAGES) & 1)) break;
      const unsigned short* v = reinterpret_cast<const unsigned short*>(bp + st * S::STAGE + S::OFF_V) + sl * 16 * D + row;
      const float* f = reinterpret_cast<const float*>(bp + st * S::STAGE + S::OFF_F);
      const float whole = f[128];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t vv[8];
        if (c == 0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) vv[j] = (uint32_t)v[2 * j * D] | ((uint32_t)v[(2 * j + 1) * D] << 16);
        }
        if (!(ok = ok && warp_wait(DK_FULL(c), s & 1))) break;
        tc_fence_after_sync();
        float y[16], hl[16];
        const uint32_t at = tl + c * S::CHAIN + S::D_K + sl * 16;
        tmem_ld16(at, y);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const float4 fj = *reinterpret_cast<const float4*>(f + sl * 16 + j);
          const float f4[4] = {fj.x, fj.y, fj.z, fj.w};
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const uint32_t w = c == 0 ? vv[(j + i) / 2] : 0u;
            uint32_t u, l;
            split2_pair(f2_fma(f2_pack(-f4[i], -f4[i + 1]), f2_pack(y[j + i], y[j + i + 1]),
                               f2_pack(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u))), u, l);
            hl[(j + i) / 2] = __uint_as_float(u);
            hl[8 + (j + i) / 2] = __uint_as_float(l);
          }
        }
        tmem_st16(at, hl);
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive_warp(X_READY(c));
      }
      if (!ok) break;
      mbar_arrive_warp(FREE(st));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (!(ok = ok && warp_wait(DS_FULL(c), s & 1))) break;
        tc_fence_after_sync();
        float d[32];
        tmem_ld32(tl + c * S::CHAIN + sl * 32, d);
        tmem_wait_ld();
#pragma unroll
        for (int e = 0; e < 16; ++e) sv[c][e] = f2_fma(f2_pack(whole, whole), sv[c][e], f2_pack(d[2 * e], d[2 * e + 1]));
        if (s + 1 < steps) publish(c);
      }
    }
    // whole rows leave through shared memory (the loads of all steps have been used; the first part's M is not wanted)
    const int tid = (warp - 2) * 32 + lane;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        *reinterpret_cast<ulonglong2*>(bp + c * 65536 + row * 512 + (((sl * 8 + e) ^ lane) << 4)) =
            make_ulonglong2(sv[c][2 * e], sv[c][2 * e + 1]);
    }
    named_barrier_sync(1, 32 * S::STATE_WARPS);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float* dst = (c == 0 ? a.comp_j : a.comp_m) + comp;
      if (c == 1 && pos == 0) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = (tid >> 5) + 16 * e;
        *reinterpret_cast<float4*>(dst + (size_t)r * D + lane * 4) =
            *reinterpret_cast<const float4*>(bp + c * 65536 + r * 512 + ((lane ^ (r & 31)) << 4));
      }
    }
  }

  // ------------------------------------------------------------------ teardown
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    settle(smem_u32(const_cast<int*>(abort_flag)));
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace vdn
