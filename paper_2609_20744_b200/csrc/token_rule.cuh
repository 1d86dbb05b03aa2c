// Token-wise gated delta rule (Eq. 2), token by token, states in registers.
//
// Per value head, with the decay gate alpha_t = exp(log_alpha_t), write gate beta_t, and S [d_v][d_k]:
//        S <- alpha_t S,      u = beta_t (v_t - S k_t),      S <- S + u k_t^T,      o_t = scale S q_t
// (k, q divided by their L2 norms first when l2_eps > 0; value head h reads key head h / (H / Hk)).  Both products are
// taken with the state as it was before the token, so that one pass over the state serves a token:
//        S k and S q reduced together,   o = scale (alpha (S q) + u (k.q)).
//
// Rows of S (value channels) evolve independently.  The kernels:
//   token_few_kernel   a few tokens a sequence (one above all): a copy of the states through registers, bound by HBM.  Eight lanes
//                      share a row and hold d/8 columns each, as 16-byte pieces 128 bytes apart, so that a warp's loads and
//                      stores cover whole 128-byte lines and a row's two dot products need three shuffle steps.
//   token_coef_kernel, token_walk_kernel  longer sequences: what does not depend on the state is formed first, for all tokens;
//                      what is left is bound by the latency of a step, or by issue slots when all SMs are busy.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"
#include "tc_common.cuh"

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

// Long sequences may be cut into parts of `part` rows (0: none is).  Part x of head h has, at (x * H + h) d d,
struct TokenParts {
  int part;
  float* enter;              // the state it starts from
  float* comp_j;             // what it writes on its own: its last state from zero (the first part: from the sequence's first state)
  float* comp_m;             // what it makes of an entering state: S -> S M
};

// Parts a sequence of `len` rows is cut into.  Two would gain nothing: composing the first and then running both takes as long as
// one after the other.
__host__ __device__ inline int token_parts(int len, int part) {
  return part > 0 && len > 2 * part ? (len + part - 1) / part : 1;
}

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
      if (x == 0) atomicCAS(a.status, 0, kStatusInvalidArg);   // (a timeout that nobody has read yet says more)
      return -1;
    }
  }
  return slot;
}

// A factor that every token multiplies the state with must not be off by the same part of a step each time: with a constant gate near
// 1 (log_alpha = -1e-6, 3000 tokens, d = 128) the state was off by 2.3e-5, without a gate by 4e-7.  So where a gate is above a
// half the state x becomes x + (alpha - 1) x, or alpha x + (what alpha lost) x; below, it forgets too fast for that to matter,
// and alpha - 1 would have lost alpha's last bits.
__device__ __forceinline__ bool slow_decay(float log_alpha) { return fabsf(log_alpha) < 0.69f; }

// One CTA to 32 R rows of a (sequence, head), R of them to a thread.  R = d / 32, a whole state to a CTA, where there are states
// enough to fill the GPU: more bytes on their way, keys and queries read once.  256 requests x 32 heads of 128 x 128 take 232 us
// with R = 1, 201 with 2 and 179 with 4 (the bytes alone: 165); 40 states are faster on four CTAs each.
template <typename Tio, int D, int R>
__global__ void __launch_bounds__(256, R == 4 ? 2 : 3) token_few_kernel(const TokenArgs a) {
  constexpr int ROWS = 32 * R, GROUPS = D / ROWS, NE = D / 8, NV = NE / 4;
  const int tid = threadIdx.x, lane8 = tid & 7;
  const int row = (int)(blockIdx.x % GROUPS) * ROWS + (tid >> 3);
  const int h = (int)(blockIdx.x / GROUPS) % a.H, s = (int)(blockIdx.x / GROUPS) / a.H;
  const long long at = a.index ? (long long)a.index[s] : s;
  const size_t soff = (((size_t)at * a.H + h) * D + row) * D + lane8 * 4;
  float4 st[R][NV];
#pragma unroll
  for (int w = 0; w < R; ++w)
#pragma unroll
    for (int i = 0; i < NV; ++i) st[w][i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.state_in && at >= 0 && at < a.slots) {           // on its way while the slot is being checked
#pragma unroll
    for (int w = 0; w < R; ++w)
#pragma unroll
      for (int i = 0; i < NV; ++i) st[w][i] = *reinterpret_cast<const float4*>(a.state_in + soff + w * 32 * D + i * 32);
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
    float v[R];
#pragma unroll
    for (int w = 0; w < R; ++w) v[w] = to_float(vp[w * 32]);
    const float beta = a.beta[(start + t) * a.H + h], ga = a.log_alpha ? a.log_alpha[(start + t) * a.H + h] : 0.f;
    const bool slow = slow_decay(ga);                    // (the same for all threads)
    const float less = slow ? expm1f(ga) : 0.f, alpha = slow ? 1.f + less : expf(ga);   // less: alpha - 1
    float sk[R], sq[R], kq = 0.f, kk = 0.f, qq = 0.f;
    auto add = [](float& s, const float4& x, const float4& y) {
      s = fmaf(x.x, y.x, s); s = fmaf(x.y, y.y, s); s = fmaf(x.z, y.z, s); s = fmaf(x.w, y.w, s);
    };
#pragma unroll
    for (int w = 0; w < R; ++w) {
      sk[w] = sq[w] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) { add(sk[w], st[w][i], k[i]); add(sq[w], st[w][i], q[i]); }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) add(kq, k[i], q[i]);
    if (a.l2_eps > 0.f) {
#pragma unroll
      for (int i = 0; i < NV; ++i) { add(kk, k[i], k[i]); add(qq, q[i], q[i]); }
    }
#pragma unroll
    for (int m = 1; m < 8; m <<= 1) {
#pragma unroll
      for (int w = 0; w < R; ++w) {
        sk[w] += __shfl_xor_sync(0xFFFFFFFFu, sk[w], m);
        sq[w] += __shfl_xor_sync(0xFFFFFFFFu, sq[w], m);
      }
      kq += __shfl_xor_sync(0xFFFFFFFFu, kq, m);
      if (a.l2_eps > 0.f) {
        kk += __shfl_xor_sync(0xFFFFFFFFu, kk, m);
        qq += __shfl_xor_sync(0xFFFFFFFFu, qq, m);
      }
    }
    const float rk = a.l2_eps > 0.f ? rsqrtf(kk + a.l2_eps) : 1.f;
    const float rq = a.l2_eps > 0.f ? rsqrtf(qq + a.l2_eps) : 1.f;
    float uk[R];
#pragma unroll
    for (int w = 0; w < R; ++w) {
      uk[w] = beta * (v[w] - alpha * rk * sk[w]) * rk;
      if (lane8 == 0) op[w * 32] = from_float<Tio>(a.scale * rq * fmaf(uk[w], kq, alpha * sq[w]));
    }
    if (slow) {
#pragma unroll
      for (int w = 0; w < R; ++w)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float4& y = st[w][i];
          y.x = fmaf(uk[w], k[i].x, fmaf(less, y.x, y.x)); y.y = fmaf(uk[w], k[i].y, fmaf(less, y.y, y.y));
          y.z = fmaf(uk[w], k[i].z, fmaf(less, y.z, y.z)); y.w = fmaf(uk[w], k[i].w, fmaf(less, y.w, y.w));
        }
    } else {
#pragma unroll
      for (int w = 0; w < R; ++w)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float4& y = st[w][i];
          y.x = fmaf(uk[w], k[i].x, alpha * y.x); y.y = fmaf(uk[w], k[i].y, alpha * y.y);
          y.z = fmaf(uk[w], k[i].z, alpha * y.z); y.w = fmaf(uk[w], k[i].w, alpha * y.w);
        }
    }
    qp += a.q_stride; kp += a.k_stride; vp += a.v_stride; op += a.out_stride;
  }
  if (a.state_out) {
#pragma unroll
    for (int w = 0; w < R; ++w)
#pragma unroll
      for (int i = 0; i < NV; ++i) *reinterpret_cast<float4*>(a.state_out + soff + w * 32 * D + i * 32) = st[w][i];
  }
}

// The kernels of one call overlap at their edges: each lets the next one start early, and each first gets ready and then waits
// for the one before to be done.  Every thread waits, also of a CTA that has nothing to do: a kernel that did not wait could be
// done before its predecessor, and its successor would then read unfinished results.
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// The sequence that owns place x, places being `unit` rows wide: the last one whose first place is not behind x.  A whole
// warp looks at 32 offsets at a time: a round trip to memory for 32 sequences, two for a thousand.
__device__ __forceinline__ int token_seq_of(const TokenArgs& t, long long x, int unit) {
  int lo = 0, n = t.S;                                // the answer lies in [lo, lo + n), and sequence lo qualifies
  const int lane = threadIdx.x & 31;
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int s = lo + lane * step;
    bool fits = false;
    if (s < lo + n) {
      long long start;
      int len;
      token_range(t.cu_seqlens, s, t.per, t.n_tokens, start, len);
      fits = start / unit + s <= x;
    }
    const unsigned m = __ballot_sync(0xFFFFFFFFu, fits) | 1u;
    const int k = 31 - __clz(m);
    n = min(step, lo + n - (lo + k * step));
    lo += k * step;
  }
  return lo;
}

// Longer sequences: four tokens make one step.  With P_i = alpha_1 .. alpha_i and A_ij = alpha_{j+1} .. alpha_i (products, so that
// nothing is divided), S the state before the four:
//        u_i = beta_i (v_i - P_i S k_i - sum_{j<i} A_ij (k_i.k_j) u_j),    o_i = P_i S q_i + sum_{j<=i} A_ij (q_i.k_j) u_j,
//        S' = P_4 S + sum_j A_4j u_j k_j^T.
// The coefficients do not depend on the state: token_coef_kernel forms them for all tokens, twelve numbers each, a warp to four
// tokens of a head, eight lanes to a token.  (Formed by the walking CTAs, eight of which share a head's tokens at d = 128, they took a
// fifth of the time.)
//   [0] beta P r, beta, (i,0), (i,1) of the first sum;  [1] (i,2), A_4i r_i, scale r_q P, P_4;  [2] (i,0) .. (i,3) of the second, times scale
// The first of the four has no (i,2): there stands what P_4 lost when it was rounded (slow_decay).  (A branch on the size, as below, is
// slower here by 4 %: 9000 tokens, 36 heads, f32, d = 128.  As it is it costs 4 % there, 1 to 2 % with fewer heads.)
constexpr int kCoefFloats = 12;

template <typename Tio, int D>
__global__ void __launch_bounds__(256) token_coef_kernel(const TokenArgs a, float4* coef, long long warps) {
  const int lane = threadIdx.x & 31, l8 = lane & 7, i4 = lane >> 3;
  const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (w >= warps) return;
  const int h = (int)(w % a.H);
  const long long place = w / a.H;
  const int seq = token_seq_of(a, place, 4);
  long long start;
  int len;
  token_range(a.cu_seqlens, seq, a.per, a.n_tokens, start, len);
  const long long g0 = (place - (start / 4 + seq)) * 4;  // first token of the four, in the sequence
  if (g0 < 0 || g0 >= len) return;
  const int n = (int)min(4LL, len - g0);
  const int hk = h / (a.H / a.Hk);
  const Tio* kp = static_cast<const Tio*>(a.k) + (start + g0) * a.k_stride + hk * D + l8 * 4;
  const Tio* qp = static_cast<const Tio*>(a.q) + (start + g0 + i4) * a.q_stride + hk * D + l8 * 4;
  const bool there = i4 < n;
  float kk[4] = {0.f, 0.f, 0.f, 0.f}, qk[4] = {0.f, 0.f, 0.f, 0.f}, qq = 0.f;
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  auto dot = [](float s, const float4& x, const float4& y) { return fmaf(x.w, y.w, fmaf(x.z, y.z, fmaf(x.y, y.y, fmaf(x.x, y.x, s)))); };
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const float4 q = there ? load4(qp + i * 32) : none;
    float4 k[4];
#pragma unroll
    for (int o = 0; o < 4; ++o) k[o] = o < n ? load4(kp + o * a.k_stride + i * 32) : none;
    const float4 own = i4 == 0 ? k[0] : i4 == 1 ? k[1] : i4 == 2 ? k[2] : k[3];
    qq = dot(qq, q, q);
#pragma unroll
    for (int o = 0; o < 4; ++o) { kk[o] = dot(kk[o], own, k[o]); qk[o] = dot(qk[o], q, k[o]); }
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
  const size_t gate = (size_t)(start + g0 + i4) * a.H + h;
  const float ga = there && a.log_alpha ? a.log_alpha[gate] : 0.f, alpha = expf(ga), beta = there ? a.beta[gate] : 0.f;
  float al[4], ro[4], four = ga;
  four += __shfl_xor_sync(0xFFFFFFFFu, four, 8);
  four += __shfl_xor_sync(0xFFFFFFFFu, four, 16);
#pragma unroll
  for (int o = 0; o < 4; ++o) {
    al[o] = __shfl_sync(0xFFFFFFFFu, alpha, o * 8);
    ro[o] = __shfl_sync(0xFFFFFFFFu, rk, o * 8);
  }
  if (l8 == 0 && there) {
    float first[3], second[4], pi = 1.f, to_end = 1.f;
#pragma unroll
    for (int o = 0; o < 4; ++o) {
      pi *= o <= i4 ? al[o] : 1.f;
      to_end *= o > i4 ? al[o] : 1.f;
      float dec = 1.f;                                   // A_{i4, o}
#pragma unroll
      for (int m = 0; m < 4; ++m) dec *= m > o && m <= i4 ? al[m] : 1.f;
      if (o < 3) first[o] = o < i4 ? beta * rk * ro[o] * dec * kk[o] : 0.f;
      second[o] = o <= i4 ? a.scale * rq * ro[o] * dec * qk[o] : 0.f;
    }
    float p4 = pi * to_end, rest = 0.f;
    if (slow_decay(four)) {
      const float less = expm1f(four);
      p4 = 1.f + less;
      rest = less - (p4 - 1.f);                          // exact
    }
    float4* c = coef + gate * (kCoefFloats / 4);
    c[0] = make_float4(beta * pi * rk, beta, first[0], first[1]);
    c[1] = make_float4(i4 > 0 ? first[2] : rest, to_end * rk, a.scale * rq * pi, p4);
    c[2] = make_float4(second[0], second[1], second[2], second[3]);
  }
}

// Two fp32 numbers worked on by one instruction: the fp32 pipe is no faster so, but half as many instructions are issued.
namespace tc {
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t r, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(r)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
}  // namespace tc

// One CTA (four warps, one to a scheduler) to 8 R rows of a (sequence, head), since a step is a chain of latencies (dot products,
// shuffles, update).  A row is shared by 16 lanes, which hold R rows each; the 8 R dot products of a step are reduced together,
// each lane ending with one of them (15 shuffles instead of 64).  R = 2 does the least work; R = 1 shortens a step, with twice the CTAs,
// where SMs would be left over.  Batches of 16 tokens -- keys, queries, this CTA's values, coefficients -- arrive by four tile
// copies each, which a fifth warp issues, three batches ahead.
// Measured, one sequence of 1024 tokens, 2 heads, d = 128, bf16: 119 us, both kernels (R = 2: 150); a token at a time it took 289.
// Long sequences of few (sequence, head)s: with COMPOSE the kernel makes, side by side, of each part what it writes by itself (J) and
// what it makes of an entering state (M, rows of the identity walked without values); token_join_kernel passes the states along, and
// the parts are walked from those.  9000 tokens, 1 head, d = 128, f32: 921 us whole, 170 in 33 parts (compose 70, join 51, walk 55).
// Many heads (9000 tokens, 36, d = 128, f32): 1620 us (1540 with decays rounded to one number); 1720 with queries fetched one by one and single fp32 instructions, about 60 % of
// the issue slots and of the shared-memory pipe either way.
template <typename Tio, int D, int R, bool COMPOSE = false>
struct TokenWalk {
  static constexpr int WALKERS = 128, THREADS = WALKERS + 32, ROWS = 8 * R, BATCH = 16, STAGES = 3;
  struct alignas(128) Stage {
    Tio k[BATCH][D], v[BATCH][ROWS];
    float4 c[BATCH][kCoefFloats / 4];
    Tio q[COMPOSE ? 1 : BATCH][D];                       // (composing reads none)
  };
  static constexpr int SMEM_BYTES = STAGES * (int)sizeof(Stage) + 64 + 128;
};

template <typename Tio, int D, int R, bool COMPOSE>
__global__ void __launch_bounds__(160) token_walk_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmQ,
                                                         const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmC,
                                                         const TokenArgs a, const TokenParts cut, tc::DevStatus ds) {
  using namespace tc;
  using W = TokenWalk<Tio, D, R, COMPOSE>;
  constexpr int ROWS = W::ROWS, GROUPS = D / ROWS, B = W::BATCH;
  constexpr int NE = D / 16, NV = NE / 4;                // columns of a lane, in pieces of four, 64 apart
  extern __shared__ unsigned char walk_smem[];
  unsigned char* bp = walk_smem + ((128u - (smem_u32(walk_smem) & 127u)) & 127u);
  typename W::Stage* stages = reinterpret_cast<typename W::Stage*>(bp);
  const uint32_t bars = smem_u32(bp) + W::STAGES * (uint32_t)sizeof(typename W::Stage);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bp + W::STAGES * sizeof(typename W::Stage) + 16 * W::STAGES);
  const WaitCtx wc(abort_flag, ds);
  const int tid = threadIdx.x, lane = tid & 31, l16 = lane & 15;
  const int row0 = (int)(blockIdx.x % GROUPS) * ROWS;
  const int r = ((tid >> 4) & 7) * R;                    // a walker's rows: row0 + r ..
  const int h = (int)(blockIdx.x / GROUPS) % a.H, y = (int)(blockIdx.x / GROUPS) / a.H;
  const bool of_m = COMPOSE && (y & 1);                  // M's rows, or J's
  const int p = COMPOSE ? y >> 1 : y;                    // the part, or the sequence where none is cut
  const int s = cut.part > 0 ? token_seq_of(a, p, cut.part) : p;
  long long start;
  int len;
  token_range(a.cu_seqlens, s, a.per, a.n_tokens, start, len);
  const int parts = token_parts(len, cut.part);
  const int pos = cut.part > 0 ? p - ((int)(start / cut.part) + s) : 0;
  // not every sequence fills its places; nothing follows the last part, and nothing enters the first
  if (pos < 0 || pos >= parts || (COMPOSE && (pos + 1 == parts || (of_m && pos == 0)))) return;
  if (parts > 1) {
    start += (long long)pos * cut.part;
    len = min(cut.part, len - pos * cut.part);
  }
  if (tid == 0) {
    for (int i = 0; i < W::STAGES; ++i) { mbar_init(bars + 8 * i, 1); mbar_init(bars + 8 * (W::STAGES + i), W::WALKERS / 32); }
    *abort_flag = 0;
    mbar_fence_init();
  }
  __syncthreads();
  const int batches = (len + B - 1) / B;
  if (tid >= W::WALKERS) {
    // one thread keeps two batches on their way (issuing the copies takes a walker 600 cycles of a batch's 4500)
    if (tid == W::WALKERS) {
      const typename W::Stage& st0 = stages[0];
      const int kc = h / (a.H / a.Hk) * D;
      const int bytes = (int)(sizeof(st0.k) + sizeof(st0.c) + (COMPOSE ? 0 : sizeof(st0.q)) + (of_m ? 0 : sizeof(st0.v)));
      auto fetch = [&](int b) {
        const int st = b % W::STAGES, row = (int)start + b * B;
        const uint32_t bar = bars + 8 * st;
        mbar_arrive_expect_tx(bar, bytes);
        tma_load_2d(smem_u32(stages[st].k), &tmK, bar, kc, row);
        if (!COMPOSE) tma_load_2d(smem_u32(stages[st].q), &tmQ, bar, kc, row);
        if (!of_m) tma_load_2d(smem_u32(stages[st].v), &tmV, bar, h * D + row0, row);
        tma_load_2d(smem_u32(stages[st].c), &tmC, bar, h * kCoefFloats, row);
      };
      uint32_t issued = 0;
      for (int b = 0; b < batches; ++b) {
        // a stage is free once the four walking warps have left it
        if (b >= W::STAGES && !mbar_wait(bars + 8 * (W::STAGES + b % W::STAGES), ((b / W::STAGES) & 1) ^ 1, wc)) break;
        fetch(b);
        issued = b + 1;
      }
      mbar_drain_ring(bars, W::STAGES, issued);          // copies in flight get a bounded chance to land before the CTA retires
    }
    return;
  }
  const size_t own = (size_t)(row0 + r) * D + l16 * 4;
  const size_t of_seq = ((size_t)s * a.H + h) * (D * D) + own, of_part = ((size_t)p * a.H + h) * (D * D) + own;
  const float* first = !COMPOSE && parts > 1 ? cut.enter + of_part : pos == 0 && a.state_in ? a.state_in + of_seq : nullptr;
  float* last = COMPOSE ? (of_m ? cut.comp_m : cut.comp_j) + of_part : pos + 1 == parts && a.state_out ? a.state_out + of_seq : nullptr;
  uint64_t x[R][NE / 2];                                 // the state, in pairs
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const float4 y = first ? *reinterpret_cast<const float4*>(first + i * D + c * 64) : make_float4(0.f, 0.f, 0.f, 0.f);
      x[i][2 * c] = f2_pack(y.x, y.y);
      x[i][2 * c + 1] = f2_pack(y.z, y.w);
      if (of_m) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = l16 * 4 + c * 64 + 2 * e;
          x[i][2 * c + e] = f2_pack(col == row0 + r + i ? 1.f : 0.f, col + 1 == row0 + r + i ? 1.f : 0.f);
        }
      }
    }
  auto columns = [&](const Tio* p, uint64_t (&y)[NE / 2]) {
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const float4 z = load4(p + l16 * 4 + c * 64);
      y[2 * c] = f2_pack(z.x, z.y);
      y[2 * c + 1] = f2_pack(z.z, z.w);
    }
  };
  for (int b = 0; b < batches; ++b) {
    typename W::Stage& st = stages[b % W::STAGES];
    const int t0 = b * B, n = min(B, len - t0);
    // a warp waits, and goes on or gives up together; it needs nothing of the other warps
    if (!__all_sync(0xFFFFFFFFu, mbar_wait(bars + 8 * (b % W::STAGES), (b / W::STAGES) & 1, wc))) break;
    for (int g = 0; g < n; g += 4) {
      if (g + 4 > n) {
        // the end of the sequence: what lies behind it is the next one's.  Tokens that do not exist count as keys and queries
        // of zero that are not written and do not decay; the state's factor is that of the last one that exists.  (All four
        // warps write the same; a warp reads what it wrote itself.)
        if (lane >= n - g && lane < 4) {
          st.c[g + lane][0] = st.c[g + lane][2] = make_float4(0.f, 0.f, 0.f, 0.f);
          st.c[g + lane][1] = make_float4(0.f, 0.f, 0.f, st.c[n - 1][1].w);
        }
        for (int e = lane; e < (g + 4 - n) * D; e += 32) {
          st.k[n + e / D][e % D] = from_float<Tio>(0.f);
          if (!COMPOSE) st.q[n + e / D][e % D] = from_float<Tio>(0.f);
        }
        for (int e = lane; e < (g + 4 - n) * ROWS; e += 32) st.v[n + e / ROWS][e % ROWS] = from_float<Tio>(0.f);
        __syncwarp();
      }
      uint64_t k[4][NE / 2], q[4][NE / 2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        columns(st.k[g + i], k[i]);
        if (!COMPOSE) columns(st.q[g + i], q[i]);
      }
      constexpr int N = COMPOSE ? 4 : 8;
      float d[N * R];                                    // [row][S k_1 .. S k_4, S q_1 .. S q_4], this lane's columns
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 0; w < R; ++w) {
          uint64_t sk = 0, sq = 0;
#pragma unroll
          for (int e = 0; e < NE / 2; ++e) {
            sk = f2_fma(x[w][e], k[i][e], sk);
            if (!COMPOSE) sq = f2_fma(x[w][e], q[i][e], sq);
          }
          float lo, hi;
          f2_unpack(sk, lo, hi);
          d[N * w + i] = lo + hi;
          if (!COMPOSE) {
            f2_unpack(sq, lo, hi);
            d[N * w + 4 + i] = lo + hi;
          }
        }
      }
      // reduce: at each step a lane keeps the half of its values that its bit names and adds its partner's; where that
      // leaves one before the last bits, they are sums of the same
      int m = 8;                                         // the bit, from the highest
#pragma unroll
      for (int half = N * R / 2; half > 0; half >>= 1, m >>= 1) {
        const bool upper = l16 & m;
#pragma unroll
        for (int i = 0; i < half; ++i) d[i] = (upper ? d[half + i] : d[i]) + __shfl_xor_sync(0xFFFFFFFFu, upper ? d[i] : d[half + i], m);
      }
      constexpr int LOW = N * R == 16 ? 0 : N * R == 8 ? 1 : 2;   // bits of the lane below those that say (row, query?, token)
      float mine = d[0];
#pragma unroll
      for (int low = LOW - 1; low >= 0; --low) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, 1 << low);
      const int what = l16 >> LOW;
      // lane (row, query?, token) has its product; the keys' ones go to all lanes
      float u[R][4];
      const float4 a0 = st.c[g][0], a1 = st.c[g + 1][0], a2 = st.c[g + 2][0], a3 = st.c[g + 3][0];
      const float4 tail = st.c[g + 3][1];
      auto value = [&](int i, int w) { return of_m ? 0.f : to_float(st.v[i][r + w]); };
#pragma unroll
      for (int w = 0; w < R; ++w) {
        float sk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sk[i] = __shfl_sync(0xFFFFFFFFu, mine, (lane & 16) + ((N * w + i) << LOW));
        u[w][0] = a0.y * value(g, w) - a0.x * sk[0];
        u[w][1] = a1.y * value(g + 1, w) - a1.x * sk[1] - a1.z * u[w][0];
        u[w][2] = a2.y * value(g + 2, w) - a2.x * sk[2] - a2.z * u[w][0] - a2.w * u[w][1];
        u[w][3] = a3.y * value(g + 3, w) - a3.x * sk[3] - a3.z * u[w][0] - a3.w * u[w][1] - tail.x * u[w][2];
      }
      if (!COMPOSE) {
        const int i = g + (what & 3);
        const bool second = R == 2 && (what & 8);        // of the lane's two rows
        if ((what & 4) && (R == 2 || !(l16 & 1)) && i < n) {
          const float4 c = st.c[i][2];
          // Tokens behind this one have coefficients of zero, but what they write need not be finite: left out, not multiplied.
          // (As predicated steps it costs nothing; with zeros selected for what they write, 9000 tokens, 36 heads, f32, d = 128 took
          // 1.87 ms instead of 1.62.)
          auto from = [&](int t) { return second ? u[R - 1][t] : u[0][t]; };
          float o = 0.f;
          if ((what & 3) == 3) o = c.w * from(3);
          if (what & 2) o = fmaf(c.z, from(2), o);
          if (what & 3) o = fmaf(c.y, from(1), o);
          o = fmaf(st.c[i][1].z, mine, fmaf(c.x, from(0), o));
          static_cast<Tio*>(a.out)[(size_t)(start + t0 + i) * a.out_stride + h * D + row0 + r + (second ? 1 : 0)] = from_float<Tio>(o);
        }
      }
      const uint64_t p4 = f2_pack(tail.w, tail.w), rest = f2_pack(st.c[g][1].x, st.c[g][1].x);
      float e4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e4[i] = st.c[g + i][1].y;
#pragma unroll
      for (int w = 0; w < R; ++w) {
        uint64_t uu[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) uu[i] = f2_pack(u[w][i] * e4[i], u[w][i] * e4[i]);
#pragma unroll
        for (int e = 0; e < NE / 2; ++e)
          x[w][e] = f2_fma(uu[3], k[3][e], f2_fma(uu[2], k[2][e], f2_fma(uu[1], k[1][e],
                    f2_fma(uu[0], k[0][e], f2_fma(p4, x[w][e], f2_fma(rest, x[w][e], 0ull))))));
      }
    }
    mbar_arrive_warp(bars + 8 * (W::STAGES + b % W::STAGES));
  }
  if (last) {
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < NV; ++c)
      {
        float4 y;
        f2_unpack(x[i][2 * c], y.x, y.y);
        f2_unpack(x[i][2 * c + 1], y.z, y.w);
        *reinterpret_cast<float4*>(last + i * D + c * 64) = y;
      }
  }
}

// ---------------------------------------------------------------------------------------------- part after part
// The states the parts of a cut sequence enter with: enter_0 the first one, enter_1 = J_0, enter_{i+1} = enter_i M_i + J_i.  Rows
// go their own ways: a CTA has 8 of a (sequence, head).  Eight groups of d/4 threads divide M's rows, d/8 each, so that each element of M is
// fetched once, into registers and a part ahead of its use; their partial products are added through shared memory.  Plain
// fp32.  Bound by the chain of parts.
template <int D>
struct TokenJoin {
  static constexpr int THREADS = 2 * D, ROWS = 8;
};
template <int D>
__global__ void __launch_bounds__(TokenJoin<D>::THREADS) token_join_kernel(const TokenArgs t, const TokenParts a) {
  constexpr int ROWS = TokenJoin<D>::ROWS, GROUPS = D / ROWS, LANES = D / 4, K = D / 8;
  __shared__ float sm[ROWS][D];                       // the state's rows
  __shared__ float4 partial[8][ROWS][LANES];
  const int r0 = (int)(blockIdx.x % GROUPS) * ROWS, h = (int)(blockIdx.x / GROUPS) % t.H, seq = (int)(blockIdx.x / GROUPS) / t.H;
  long long start;
  int len;
  token_range(t.cu_seqlens, seq, t.per, t.n_tokens, start, len);
  const int parts = token_parts(len, a.part);
  let_next_kernel_start();
  wait_for_kernel_before();
  if (parts == 1) return;
  const int group = (int)threadIdx.x / LANES, lane = (int)threadIdx.x % LANES;
  const size_t x0 = (size_t)(start / a.part + seq), step = (size_t)t.H * D * D, base = (x0 * t.H + h) * (D * D);
  // the thread's own four elements of the state: row r0 + group, columns 4 lane ..
  const size_t own = base + (size_t)(r0 + group) * D + lane * 4;
  const float* mp = a.comp_m + base + (size_t)(group * K) * D + lane * 4;
  {
    const float* s0 = t.state_in ? t.state_in + ((size_t)seq * t.H + h) * (D * D) + (size_t)(r0 + group) * D + lane * 4 : nullptr;
    *reinterpret_cast<float4*>(a.enter + own) = s0 ? *reinterpret_cast<const float4*>(s0) : make_float4(0.f, 0.f, 0.f, 0.f);
    const float4 j = *reinterpret_cast<const float4*>(a.comp_j + own);
    *reinterpret_cast<float4*>(a.enter + own + step) = j;
    *reinterpret_cast<float4*>(&sm[group][lane * 4]) = j;
  }
  float4 m[K], next[K], j = make_float4(0.f, 0.f, 0.f, 0.f), jn = j;
  auto fetch = [&](int p) {
#pragma unroll
    for (int k = 0; k < K; ++k) next[k] = __ldg(reinterpret_cast<const float4*>(mp + p * step + (size_t)k * D));
    jn = __ldg(reinterpret_cast<const float4*>(a.comp_j + own + p * step));
  };
  if (parts > 2) fetch(1);
  for (int p = 1; p + 1 < parts; ++p) {
#pragma unroll
    for (int k = 0; k < K; ++k) m[k] = next[k];
    j = jn;
    if (p + 2 < parts) fetch(p + 1);
    __syncthreads();                                  // the state is there
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < K; k += 4) {
        const float4 s = *reinterpret_cast<const float4*>(&sm[r][group * K + k]);
        const float s4[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc.x = fmaf(s4[e], m[k + e].x, acc.x); acc.y = fmaf(s4[e], m[k + e].y, acc.y);
          acc.z = fmaf(s4[e], m[k + e].z, acc.z); acc.w = fmaf(s4[e], m[k + e].w, acc.w);
        }
      }
      partial[group][r][lane] = acc;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const float4 q = partial[w][group][lane];
      j.x += q.x; j.y += q.y; j.z += q.z; j.w += q.w;
    }
    *reinterpret_cast<float4*>(a.enter + own + (p + 1) * step) = j;
    *reinterpret_cast<float4*>(&sm[group][lane * 4]) = j;
  }
}

}  // namespace vdn
