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

// One CTA (four warps) to 16 rows of a (sequence, head): a warp to a scheduler, and as many CTAs as rows allow, since a token's
// step is a chain of latencies.
template <typename Tio, int D>
struct TokenWalk {
  static constexpr int THREADS = 128, ROWS = 16, BATCH = 16;
  static constexpr int PIECE = 16 / (int)sizeof(Tio);            // elements of a 16-byte copy
  struct Stage {
    Tio k[BATCH][D], q[BATCH][D], v[BATCH][ROWS];
    float beta[BATCH], log_alpha[BATCH];
  };
  struct Smem {
    Stage st[2];
    float4 f[BATCH];        // alpha, alpha r_k, beta, r_k
    float2 g[BATCH];        // of the read-out: scale r_q alpha, scale r_q r_k (k.q)
  };
};

template <typename Tio, int D>
__global__ void __launch_bounds__(128) token_walk_kernel(const TokenArgs a) {
  using W = TokenWalk<Tio, D>;
  constexpr int ROWS = W::ROWS, GROUPS = D / ROWS, NE = D / 8, NV = NE / 4, B = W::BATCH, PIECE = W::PIECE;
  __shared__ __align__(16) typename W::Smem sm;
  const int tid = threadIdx.x, lane8 = tid & 7, r = tid >> 3;
  const int row0 = (int)(blockIdx.x % GROUPS) * ROWS;
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
  Tio* op = static_cast<Tio*>(a.out) + start * a.out_stride + h * D + row0 + r;

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
  const size_t soff = (((size_t)slot * a.H + h) * D + row0 + r) * D + lane8 * 4;
  float x[NE];                                           // the state
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const float4 y = a.state_in ? *reinterpret_cast<const float4*>(a.state_in + soff + i * 32) : make_float4(0.f, 0.f, 0.f, 0.f);
    x[4 * i] = y.x; x[4 * i + 1] = y.y; x[4 * i + 2] = y.z; x[4 * i + 3] = y.w;
  }
  auto columns = [&](const Tio* p, float (&y)[NE]) {     // this lane's columns of a token's row in shared memory
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float4 z = load4(p + lane8 * 4 + i * 32);
      y[4 * i] = z.x; y[4 * i + 1] = z.y; y[4 * i + 2] = z.z; y[4 * i + 3] = z.w;
    }
  };
  for (int t0 = 0, b = 0; t0 < len; t0 += B, b ^= 1) {
    const typename W::Stage& st = sm.st[b];
    const int n = min(B, len - t0);
    if (t0 + B < len) { fetch(t0 + B, sm.st[b ^ 1]); cp_async_wait<1>(); }
    else cp_async_wait<0>();
    __syncthreads();
    {
      // what does not depend on the state: eight lanes a token
      float k[NE], q[NE], kq = 0.f, kk = 0.f, qq = 0.f;
      columns(st.k[r], k);                               // (rows of tokens that do not exist hold anything: their factors are not used)
      columns(st.q[r], q);
#pragma unroll
      for (int i = 0; i < NE; ++i) { kq = fmaf(k[i], q[i], kq); kk = fmaf(k[i], k[i], kk); qq = fmaf(q[i], q[i], qq); }
#pragma unroll
      for (int m = 1; m < 8; m <<= 1) {
        kq += __shfl_xor_sync(0xFFFFFFFFu, kq, m);
        kk += __shfl_xor_sync(0xFFFFFFFFu, kk, m);
        qq += __shfl_xor_sync(0xFFFFFFFFu, qq, m);
      }
      if (lane8 == 0) {
        const float rk = a.l2_eps > 0.f ? rsqrtf(kk + a.l2_eps) : 1.f;
        const float rq = a.l2_eps > 0.f ? rsqrtf(qq + a.l2_eps) : 1.f;
        const float alpha = expf(st.log_alpha[r]);
        sm.f[r] = make_float4(alpha, alpha * rk, st.beta[r], rk);
        sm.g[r] = make_float2(a.scale * rq * alpha, a.scale * rq * rk * kq);
      }
    }
    __syncthreads();
    float k[NE], q[NE];
    columns(st.k[0], k);
    columns(st.q[0], q);
    float v = to_float(st.v[0][r]);
    float4 f = sm.f[0];
#pragma unroll 2
    for (int j = 0; j < n; ++j) {
      float sk[4] = {0.f, 0.f, 0.f, 0.f}, sq[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        sk[i & 3] = fmaf(x[i], k[i], sk[i & 3]);
        sq[i & 1] = fmaf(x[i], q[i], sq[i & 1]);
      }
      float dk = (sk[0] + sk[1]) + (sk[2] + sk[3]), dq = sq[0] + sq[1];
#pragma unroll
      for (int m = 1; m < 8; m <<= 1) {
        dk += __shfl_xor_sync(0xFFFFFFFFu, dk, m);
        dq += __shfl_xor_sync(0xFFFFFFFFu, dq, m);
      }
      const float u = f.z * (v - f.y * dk), uk = u * f.w;
#pragma unroll
      for (int i = 0; i < NE; ++i) x[i] = fmaf(uk, k[i], f.x * x[i]);
      if (lane8 == 0) {
        const float2 g = sm.g[j];
        *op = from_float<Tio>(fmaf(g.y, u, g.x * dq));
      }
      op += a.out_stride;
      if (j + 1 < n) {                                   // the next token, under the latencies of this one
        columns(st.k[j + 1], k);
        columns(st.q[j + 1], q);
        v = to_float(st.v[j + 1][r]);
        f = sm.f[j + 1];
      }
    }
    __syncthreads();                                     // the stage and the factors may be replaced
  }
  if (a.state_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      *reinterpret_cast<float4*>(a.state_out + soff + i * 32) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
}

}  // namespace vdn
