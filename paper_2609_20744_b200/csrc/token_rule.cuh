// Token-wise gated delta rule (Eq. 2), token by token, states in registers.
//
// Per value head, with the decay gate alpha_t = exp(log_alpha_t), write gate beta_t, and S [d_v][d_k]:
//        S <- alpha_t S,      u = beta_t (v_t - S k_t),      S <- S + u k_t^T,      o_t = scale S q_t
// (k, q divided by their L2 norms first when l2_eps > 0; value head h reads key head h / (H / Hk)).  Both products are
// taken with the state as it was before the token, so that one pass over the state serves a token:
//        S k and S q reduced together,   o = scale (alpha (S q) + u (k.q)).
//
// Rows of S (value channels) evolve independently.  A CTA owns 32 rows of one (sequence, head) state; eight lanes share a
// row and hold d/8 columns each, as 16-byte pieces 128 bytes apart, so that a warp's loads and stores cover whole 128-byte
// lines and a row's two dot products need three shuffle steps.  For one token a request the kernel is a copy of the states
// through registers and bound by HBM; for longer sequences it is bound by the latency of a token's step.
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

template <typename Tio, int D>
__global__ void __launch_bounds__(256) token_rule_kernel(const TokenArgs a) {
  constexpr int ROWS = 32, GROUPS = D / ROWS, NE = D / 8, NV = NE / 4;
  const int tid = threadIdx.x, lane8 = tid & 7;
  const int row = (int)(blockIdx.x % GROUPS) * ROWS + (tid >> 3);
  const int h = (int)(blockIdx.x / GROUPS) % a.H, s = (int)(blockIdx.x / GROUPS) / a.H;
  const long long slot = a.index ? (long long)a.index[s] : s;
  if (slot < 0 || slot >= a.slots) return;               // a padding entry of the batch: nothing is read or written

  const size_t soff = (((size_t)slot * a.H + h) * D + row) * D + lane8 * 4;
  float st[NE];
  if (a.state_in) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(a.state_in + soff + i * 32);
      st[4 * i] = x.x; st[4 * i + 1] = x.y; st[4 * i + 2] = x.z; st[4 * i + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NE; ++i) st[i] = 0.f;
  }
  if (a.index) {
    // two requests for one state cannot both have it: the first in the batch does, later ones are skipped and reported
    int twice = 0;
    for (int j = tid; j < s; j += 256) twice |= a.index[j] == (int)slot;
    if (__syncthreads_or(twice)) {
      if (tid == 0) atomicExch(a.status, kStatusInvalidArg);
      return;
    }
  }
  long long start;
  int len;
  token_range(a.cu_seqlens, s, a.per, a.n_tokens, start, len);

  const int hk = h / (a.H / a.Hk);
  const Tio* qp = static_cast<const Tio*>(a.q) + start * a.q_stride + hk * D + lane8 * 4;
  const Tio* kp = static_cast<const Tio*>(a.k) + start * a.k_stride + hk * D + lane8 * 4;
  const Tio* vp = static_cast<const Tio*>(a.v) + start * a.v_stride + h * D + row;
  Tio* op = static_cast<Tio*>(a.out) + start * a.out_stride + h * D + row;
  const float* bp = a.beta + start * a.H + h;
  const float* gp = a.log_alpha ? a.log_alpha + start * a.H + h : nullptr;

  float4 kn[NV], qn[NV];
  float vn = 0.f, bn = 0.f, gn = 0.f;
  auto fetch = [&]() {                                   // the next token, one step ahead of its use
#pragma unroll
    for (int i = 0; i < NV; ++i) { kn[i] = load4(kp + i * 32); qn[i] = load4(qp + i * 32); }
    vn = to_float(*vp);
    bn = *bp;
    gn = gp ? *gp : 0.f;
    kp += a.k_stride; qp += a.q_stride; vp += a.v_stride; bp += a.H;
    if (gp) gp += a.H;
  };
  if (len > 0) fetch();
  for (int t = 0; t < len; ++t) {
    float k[NE], q[NE];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      k[4 * i] = kn[i].x; k[4 * i + 1] = kn[i].y; k[4 * i + 2] = kn[i].z; k[4 * i + 3] = kn[i].w;
      q[4 * i] = qn[i].x; q[4 * i + 1] = qn[i].y; q[4 * i + 2] = qn[i].z; q[4 * i + 3] = qn[i].w;
    }
    const float v = vn, beta = bn, alpha = expf(gn);
    if (t + 1 < len) fetch();
    float sk = 0.f, sq = 0.f, kq = 0.f, kk = 0.f, qq = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      sk = fmaf(st[i], k[i], sk);
      sq = fmaf(st[i], q[i], sq);
      kq = fmaf(k[i], q[i], kq);
      kk = fmaf(k[i], k[i], kk);
      qq = fmaf(q[i], q[i], qq);
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
    const float u = beta * (v - alpha * rk * sk), uk = u * rk;
    if (lane8 == 0) *op = from_float<Tio>(a.scale * rq * fmaf(uk, kq, alpha * sq));
    op += a.out_stride;
#pragma unroll
    for (int i = 0; i < NE; ++i) st[i] = fmaf(uk, k[i], alpha * st[i]);
  }
  if (a.state_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      *reinterpret_cast<float4*>(a.state_out + soff + i * 32) =
          make_float4(st[4 * i], st[4 * i + 1], st[4 * i + 2], st[4 * i + 3]);
  }
}

}  // namespace vdn
