// Token-wise gated delta rule (Eq. 2), token by token, states in registers.
//
// Per value head, with the decay gate alpha_t = exp(log_alpha_t), write gate beta_t, and S [d_v][d_k]:
//        S <- alpha_t S,      u = beta_t (v_t - S k_t),      S <- S + u k_t^T,      o_t = scale S q_t
// (k, q divided by their L2 norms first when l2_eps > 0; value head h reads key head h / (H / Hk)).  Both products are
// taken with the state as it was before the token, so that one pass over the state serves a token:
//        S k and S q reduced together,   o = scale (alpha (S q) + u (k.q)).
//
// Rows of S (value channels) evolve independently.  Eight lanes share a row and hold d/8 columns each, as 16-byte pieces 128
// bytes apart, so that a warp's loads and stores of the state cover whole 128-byte lines and a row's two dot products need
// three shuffle steps.  Two kernels:
//   token_few_kernel   a few tokens a sequence (one above all): a copy of the states through registers, bound by HBM.
//   token_walk_kernel  longer sequences: tokens are fetched in batches ahead of their use, what does not depend on the state is
//                      formed once a batch, and what is left is bound by the latency of a token's step.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"

namespace vdn {

struct TokenArgs {
  const void* q;             // [N, Hk, d], rows of q_stride elements
  const void* k;
  const void* v;             // [N, H, d]
  const float* beta;         // [N, H]
  const float* log_alpha;    // [N, H] or null (no decay)
  void* out;                 // [N, H, d]
  const int* cu_seqlens;     // [S + 1] or null: sequence s is rows s * per .. (s + 1) * per - 1
  const int* index;          // [S] state of each sequence, or null: state s
  const float* state_in;     // [slots, H, d_v, d_k] or null (zero)
  float* state_out;          // ... or null; may be state_in
  long long q_stride, k_stride, v_stride, out_stride;
  long long n_tokens, slots;
  int S, H, Hk, per;
  float scale, l2_eps;
  int* status;
};

constexpr int kStatusInvalidArg = 1;   // mirrors VDN_ERR_INVALID_ARG

// Rows [start, start + len) of sequence s.  The offsets live in device memory, where the host cannot check them: they are
// clamped to the tensor, so that wrong ones give wrong rows but no access outside it.
__device__ __forceinline__ void token_range(const int* cu, int s, int per, long long n, long long& start, int& len) {
  if (cu == nullptr) {
    start = (long long)s * per;
    len = per;
    return;
  }
  const long long a = min(max((long long)cu[s], 0LL), n), b = min(max((long long)cu[s + 1], a), n);
  start = a;
  len = (int)(b - a);
}

// The state of sequence s: its slot, or -1 for an entry that is skipped.  `x` runs over all threads of the block, which come here
// together.
__device__ __forceinline__ long long token_slot(const TokenArgs& a, int s, int x, int threads) {
  const long long slot = a.index ? (long long)a.index[s] : s;
  if (slot < 0 || slot >= a.slots) return -1;            // a padding entry of the batch: nothing is read or written
  if (a.index) {
    // two requests for one state cannot both have it: the first in the batch does, later ones are skipped and reported
    int twice = 0;
    for (int j = x; j < s; j += threads) twice |= a.index[j] == (int)slot;
    if (__syncthreads_or(twice)) {
      if (x == 0) atomicExch(a.status, kStatusInvalidArg);
      return -1;
    }
  }
  return slot;
}

// One CTA to 32 rows of a (sequence, head).
template <typename Tio, int D>
__global__ void __launch_bounds__(256, D == 64 ? 5 : 3) token_few_kernel(const TokenArgs a) {
  constexpr int ROWS = 32, GROUPS = D / ROWS, NE = D / 8, NV = NE / 4;
  const int tid = threadIdx.x, lane8 = tid & 7;
  const int row = (int)(blockIdx.x % GROUPS) * ROWS + (tid >> 3);
  const int h = (int)(blockIdx.x / GROUPS) % a.H, s = (int)(blockIdx.x / GROUPS) / a.H;
  const long long at = a.index ? (long long)a.index[s] : s;
  const size_t soff = (((size_t)at * a.H + h) * D + row) * D + lane8 * 4;
  float4 st[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) st[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.state_in && at >= 0 && at < a.slots) {           // on its way while the slot is being checked
#pragma unroll
    for (int i = 0; i < NV; ++i) st[i] = *reinterpret_cast<const float4*>(a.state_in + soff + i * 32);
  }
  if (token_slot(a, s, tid, 256) < 0) return;
  long long start;
  int len;
  token_range(a.cu_seqlens, s, a.per, a.n_tokens, start, len);
  const int hk = h / (a.H / a.Hk);
  const Tio* qp = static_cast<const Tio*>(a.q) + start * a.q_stride + hk * D + lane8 * 4;
  const Tio* kp = static_cast<const Tio*>(a.k) + start * a.k_stride + hk * D + lane8 * 4;
  const Tio* vp = static_cast<const Tio*>(a.v) + start * a.v_stride + h * D + row;
  Tio* op = static_cast<Tio*>(a.out) + start * a.out_stride + h * D + row;
  for (int t = 0; t < len; ++t) {
    float4 k[NV], q[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) { k[i] = load4(kp + i * 32); q[i] = load4(qp + i * 32); }
    const float v = to_float(*vp), beta = a.beta[(start + t) * a.H + h];
    const float alpha = a.log_alpha ? expf(a.log_alpha[(start + t) * a.H + h]) : 1.f;
    float sk = 0.f, sq = 0.f, kq = 0.f, kk = 0.f, qq = 0.f;
    auto add = [](float& s, const float4& x, const float4& y) {
      s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s); s = fmaf(x.z, y.z, s); s = fmaf(x.w, y.w, s);
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) { add(sk, st[i], k[i]); add(sq, st[i], q[i]); add(kq, k[i], q[i]); }
    if (a.l2_eps > 0.f) {
#pragma unroll
      for (int i = 0; i < NV; ++i) { add(kk, k[i], k[i]); add(qq, q[i], q[i]); }
    }
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {
      sk += __shfl_xor_sync(0xFFFFFFFFu, sk, m);
      sq += __shfl_xor_sync(0xFFFFFFFFu, sq, m);
      kq += __shfl_xor_sync(0xFFFFFFFFu, kq, m);
      if (a.l2_eps > 0.f) {
        kk += __shfl_xor_sync(0xFFFFFFFFu, kk, m);
        qq += __shfl_xor_sync(0xFFFFFFFFu, qq, m);
      }
    }
    const float rk = a.l2_eps > 0.f ? rsqrtf(kk + a.l2_eps) : 1.f;
    const float rq = a.l2_eps > 0.f ? rsqrtf(qq + a.l2_eps) : 1.f;
    const float uk = beta * (v - alpha * rk * sk) * rk;
    if (lane8 == 0) *op = from_float<Tio>(a.scale * rq * fmaf(uk, kq, alpha * sq));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      st[i].x = fmaf(uk, k[i].x, alpha * st[i].x); st[i].y = fmaf(uk, k[i].y, alpha * st[i].y);
      st[i].z = fmaf(uk, k[i].z, alpha * st[i].z); st[i].w = fmaf(uk, k[i].w, alpha * st[i].w);
    }
    qp += a.q_stride; kp += a.k_stride; vp += a.v_stride; op += a.out_stride;
  }
  if (a.state_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i) *reinterpret_cast<float4*>(a.state_out + soff + i * 32) = st[i];
  }
}

// One CTA (four warps) to 16 rows of a (sequence, head): a warp to a scheduler, and as many CTAs as rows allow, since a step is a
// chain of latencies (dot products, shuffles, update).  Four tokens make one step.  With P_i = alpha_1 .. alpha_i and
// A_ij = alpha_{j+1} .. alpha_i (products, so that nothing is divided), S the state before the four:
//        u_i = beta_i (v_i - P_i S k_i - sum_{j<i} A_ij (k_i.k_j) u_j),    o_i = P_i S q_i + sum_{j<=i} A_ij (q_i.k_j) u_j,
//        S' = P_4 S + sum_j A_4j u_j k_j^T.
// The coefficients are formed once a batch, a warp to each four tokens.  A row is shared by 16 lanes, which hold two rows each;
// the sixteen dot products of a step are reduced together, each lane ending with one of them (15 shuffles instead of 64).
// Measured, d = 128, one sequence: FIXME.
template <typename Tio, int D>
struct TokenWalk {
  static constexpr int THREADS = 128, ROWS = 16, BATCH = 16;
  static constexpr int PIECE = 16 / (int)sizeof(Tio);            // elements of a 16-byte copy
  struct Stage {
    Tio k[BATCH][D], q[BATCH][D], v[BATCH][ROWS];
    float beta[BATCH], log_alpha[BATCH];
  };
  struct Batch {            // the batch being walked, as the steps want it
    float k[BATCH][D], q[BATCH][D];
    float4 a[BATCH];        // beta P r, beta, (i,0), (i,1) of the first sum
    float4 b[BATCH];        // (i,2); A_4i r_i; scale r_q P; P_4
    float4 c[BATCH];        // (i,0) .. (i,3) of the second sum, times scale
    float v[BATCH][ROWS];
  };
  struct Smem {
    Stage st[2];
    Batch now;
  };
};

template <typename Tio, int D>
__global__ void __launch_bounds__(128) token_walk_kernel(const TokenArgs a) {
  using W = TokenWalk<Tio, D>;
  constexpr int ROWS = W::ROWS, GROUPS = D / ROWS, B = W::BATCH, PIECE = W::PIECE;
  constexpr int NE = D / 16, NV = NE / 4;                // columns of a lane, in 16-byte pieces 256 bytes apart
  extern __shared__ __align__(16) unsigned char walk_smem[];
  typename W::Smem& sm = *reinterpret_cast<typename W::Smem*>(walk_smem);
  const int tid = threadIdx.x, lane = tid & 31, l16 = lane & 15;
  const int row0 = (int)(blockIdx.x % GROUPS) * ROWS;
  const int r = (tid >> 4) * 2;                          // this lane's rows: row0 + r, row0 + r + 1
  const int h = (int)(blockIdx.x / GROUPS) % a.H, s = (int)(blockIdx.x / GROUPS) / a.H;
  const long long slot = token_slot(a, s, tid, W::THREADS);
  if (slot < 0) return;
  long long start;
  int len;
  token_range(a.cu_seqlens, s, a.per, a.n_tokens, start, len);
  const int hk = h / (a.H / a.Hk);
  const Tio* qp = static_cast<const Tio*>(a.q) + start * a.q_stride + hk * D;
  const Tio* kp = static_cast<const Tio*>(a.k) + start * a.k_stride + hk * D;
  const Tio* vp = static_cast<const Tio*>(a.v) + start * a.v_stride + h * D + row0;
  const size_t gate0 = (size_t)start * a.H + h;

  auto fetch = [&](int t0, typename W::Stage& st) {      // tokens t0 .. of the sequence, those that exist
    const int n = min(B, len - t0);
    for (int e = tid; e < n * (D / PIECE); e += W::THREADS) {
      const int j = e / (D / PIECE), c = e % (D / PIECE) * PIECE;
      cp_async16(&st.k[j][c], kp + (size_t)(t0 + j) * a.k_stride + c);
      cp_async16(&st.q[j][c], qp + (size_t)(t0 + j) * a.q_stride + c);
    }
    for (int e = tid; e < n * (ROWS / PIECE); e += W::THREADS) {
      const int j = e / (ROWS / PIECE), c = e % (ROWS / PIECE) * PIECE;
      cp_async16(&st.v[j][c], vp + (size_t)(t0 + j) * a.v_stride + c);
    }
    if (tid < n) {
      cp_async4(&st.beta[tid], a.beta + gate0 + (size_t)(t0 + tid) * a.H);
      if (a.log_alpha) cp_async4(&st.log_alpha[tid], a.log_alpha + gate0 + (size_t)(t0 + tid) * a.H);
      else st.log_alpha[tid] = 0.f;
    }
    cp_async_commit();
  };

  if (len > 0) fetch(0, sm.st[0]);
  const size_t soff = (((size_t)slot * a.H + h) * D + row0 + r) * D + l16 * 4;
  float x[2][NE];                                        // the state
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const float4 y = a.state_in ? *reinterpret_cast<const float4*>(a.state_in + soff + i * D + c * 64) : make_float4(0.f, 0.f, 0.f, 0.f);
      x[i][4 * c] = y.x; x[i][4 * c + 1] = y.y; x[i][4 * c + 2] = y.z; x[i][4 * c + 3] = y.w;
    }
  auto columns = [&](const float* p, float (&y)[NE]) {
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const float4 z = *reinterpret_cast<const float4*>(p + l16 * 4 + c * 64);
      y[4 * c] = z.x; y[4 * c + 1] = z.y; y[4 * c + 2] = z.z; y[4 * c + 3] = z.w;
    }
  };
  for (int t0 = 0, b = 0; t0 < len; t0 += B, b ^= 1) {
    const typename W::Stage& st = sm.st[b];
    const int n = min(B, len - t0);
    if (t0 + B < len) { fetch(t0 + B, sm.st[b ^ 1]); cp_async_wait<1>(); }
    else cp_async_wait<0>();
    __syncthreads();                                     // the stage is there, the batch before has been walked
    {
      // ---- coefficients: a warp to four tokens, eight lanes to a token.  Tokens that do not exist count as keys and queries of
      // zero that are not written and do not decay.
      constexpr int ME = D / 8;
      const int j = tid >> 3, l8 = tid & 7, i4 = j & 3, g0 = j & ~3;
      float kk[4] = {0.f, 0.f, 0.f, 0.f}, qk[4] = {0.f, 0.f, 0.f, 0.f}, qq = 0.f;
      const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
      auto dot = [](float s, const float4& x, const float4& y) { return fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, s)))); };
#pragma unroll
      for (int i = 0; i < ME / 4; ++i) {
        const int c = l8 * 4 + i * 32;
        const float4 k = j < n ? load4(&st.k[j][c]) : none, q = j < n ? load4(&st.q[j][c]) : none;
        *reinterpret_cast<float4*>(&sm.now.k[j][c]) = k;
        *reinterpret_cast<float4*>(&sm.now.q[j][c]) = q;
        qq = dot(qq, q, q);
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          const float4 ko = g0 + o < n ? load4(&st.k[g0 + o][c]) : none;
          kk[o] = dot(kk[o], k, ko);
          qk[o] = dot(qk[o], q, ko);
        }
      }
#pragma unroll
      for (int m = 1; m < 8; m <<= 1) {
        qq += __shfl_xor_sync(0xFFFFFFFFu, qq, m);
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          kk[o] += __shfl_xor_sync(0xFFFFFFFFu, kk[o], m);
          qk[o] += __shfl_xor_sync(0xFFFFFFFFu, qk[o], m);
        }
      }
      const float own = i4 == 0 ? kk[0] : i4 == 1 ? kk[1] : i4 == 2 ? kk[2] : kk[3];
      const float rk = a.l2_eps > 0.f ? rsqrtf(own + a.l2_eps) : 1.f;
      const float rq = a.l2_eps > 0.f ? rsqrtf(qq + a.l2_eps) : 1.f;
      const float alpha = j < n ? expf(st.log_alpha[j]) : 1.f, beta = j < n ? st.beta[j] : 0.f;
      float al[4], ro[4];
#pragma unroll
      for (int o = 0; o < 4; ++o) {
        al[o] = __shfl_sync(0xFFFFFFFFu, alpha, o * 8);
        ro[o] = __shfl_sync(0xFFFFFFFFu, rk, o * 8);
      }
      sm.now.v[j][l8] = j < n ? to_float(st.v[j][l8]) : 0.f;
      sm.now.v[j][l8 + 8] = j < n ? to_float(st.v[j][l8 + 8]) : 0.f;
      if (l8 == 0) {
        float first[3], second[4], pi = 1.f, to_end = 1.f;
#pragma unroll
        for (int o = 0; o < 4; ++o) {
          pi *= o <= i4 ? al[o] : 1.f;
          to_end *= o > i4 ? al[o] : 1.f;
          float dec = 1.f;                               // A_{i4, o}
#pragma unroll
          for (int m = 0; m < 4; ++m) dec *= m > o && m <= i4 ? al[m] : 1.f;
          if (o < 3) first[o] = o < i4 ? beta * rk * ro[o] * dec * kk[o] : 0.f;
          second[o] = o <= i4 ? a.scale * rq * ro[o] * dec * qk[o] : 0.f;
        }
        sm.now.a[j] = make_float4(beta * pi * rk, beta, first[0], first[1]);
        sm.now.b[j] = make_float4(first[2], to_end * rk, a.scale * rq * pi, pi * to_end);
        sm.now.c[j] = make_float4(second[0], second[1], second[2], second[3]);
      }
    }
    __syncthreads();
    for (int g = 0; g < n; g += 4) {
      float k[4][NE];
#pragma unroll
      for (int i = 0; i < 4; ++i) columns(sm.now.k[g + i], k[i]);
      float d[16];                                       // [row][S k_1 .. S k_4, S q_1 .. S q_4], this lane's columns
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float q[NE];
        columns(sm.now.q[g + i], q);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float sk = 0.f, sq = 0.f;
#pragma unroll
          for (int e = 0; e < NE; ++e) { sk = fmaf(x[w][e], k[i][e], sk); sq = fmaf(x[w][e], q[e], sq); }
          d[8 * w + i] = sk;
          d[8 * w + 4 + i] = sq;
        }
      }
      // reduce: at each step a lane keeps the half of its values that its bit names and adds its partner's
      const bool b3 = l16 & 8, b2 = l16 & 4, b1 = l16 & 2, b0 = l16 & 1;
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = (b3 ? d[8 + i] : d[i]) + __shfl_xor_sync(0xFFFFFFFFu, b3 ? d[i] : d[8 + i], 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = (b2 ? d[4 + i] : d[i]) + __shfl_xor_sync(0xFFFFFFFFu, b2 ? d[i] : d[4 + i], 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) d[i] = (b1 ? d[2 + i] : d[i]) + __shfl_xor_sync(0xFFFFFFFFu, b1 ? d[i] : d[2 + i], 2);
      const float mine = (b0 ? d[1] : d[0]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? d[0] : d[1], 1);
      // lane (row, query?, token) has its product; the keys' ones go to all lanes
      float u[2][4];
      const float4 a0 = sm.now.a[g], a1 = sm.now.a[g + 1], a2 = sm.now.a[g + 2], a3 = sm.now.a[g + 3];
      const float4 b3v = sm.now.b[g + 3];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        float sk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sk[i] = __shfl_sync(0xFFFFFFFFu, mine, (lane & 16) + 8 * w + i);
        u[w][0] = a0.y * sm.now.v[g][r + w] - a0.x * sk[0];
        u[w][1] = a1.y * sm.now.v[g + 1][r + w] - a1.x * sk[1] - a1.z * u[w][0];
        u[w][2] = a2.y * sm.now.v[g + 2][r + w] - a2.x * sk[2] - a2.z * u[w][0] - a2.w * u[w][1];
        u[w][3] = a3.y * sm.now.v[g + 3][r + w] - a3.x * sk[3] - a3.z * u[w][0] - a3.w * u[w][1] - b3v.x * u[w][2];
      }
      {
        const int i = g + (l16 & 3);
        if (b2 && i < n) {
          const float4 c = sm.now.c[i];
          const float o = fmaf(sm.now.b[i].z, mine, fmaf(c.x, b3 ? u[1][0] : u[0][0], fmaf(c.y, b3 ? u[1][1] : u[0][1],
                          fmaf(c.z, b3 ? u[1][2] : u[0][2], c.w * (b3 ? u[1][3] : u[0][3])))));
          static_cast<Tio*>(a.out)[(size_t)(start + t0 + i) * a.out_stride + h * D + row0 + r + (b3 ? 1 : 0)] = from_float<Tio>(o);
        }
      }
      float e4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e4[i] = sm.now.b[g + i].y;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[w][i] *= e4[i];
#pragma unroll
        for (int e = 0; e < NE; ++e)
          x[w][e] = fmaf(u[w][3], k[3][e], fmaf(u[w][2], k[2][e], fmaf(u[w][1], k[1][e], fmaf(u[w][0], k[0][e], b3v.w * x[w][e]))));
      }
    }
  }
  if (a.state_out) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < NV; ++c)
        *reinterpret_cast<float4*>(a.state_out + soff + i * D + c * 64) =
            make_float4(x[i][4 * c], x[i][4 * c + 1], x[i][4 * c + 2], x[i][4 * c + 3]);
  }
}

}  // namespace vdn
