// Attention of each query to all the states of its batch row's encoder, in plain fp32 arithmetic: f32 I/O, single tokens, and the
// second opinion beside the tensor-core kernel.
//
//   z_j = scale q . k_j over the keys that count,   lse = log sum_j e^{z_j},   out = sum_j e^{z_j - lse} v_j
//
// One pass over the keys with the running maximum m and, relative to it, the sum l and the weighted values o (in base 2: the
// logarithms carry a factor log2 e).  No key that counts: out = 0, lse = -inf.
// The rows of a key head are its queries times the heads of its group, so K and V are read once for all of them.  Long encoders are
// cut into parts that leave (m, l, o) in the workspace, joined by cross_join_kernel.
// A key that does not count is told by its place, never by its score, and enters with zeros in the place of k and v: what stands
// behind a sequence or under the mask may be anything, NaN too.
#pragma once
#include "common.cuh"
#include "token_rule.cuh"

namespace vdn {

struct CrossArgs {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;                 // [B * Lq, H] or null
  const int* cu_seqlens;      // [B + 1]: keys packed one behind another; null: B rows of Lk
  const int* lengths;         // [B] or null
  const uint8_t* mask;        // [keys of all rows] or null; zero: does not count
  float* part_o;              // [B * Lq * H][parts][d]
  float2* part_ml;            // [B * Lq * H][parts] maximum (base 2) and sum
  long long q_stride, k_stride, v_stride, out_stride;
  long long n_keys;           // rows of k and v in all
  long long Lk;               // keys of a batch row (not packed)
  int B, Lq, H, Hk, group;    // group = H / Hk
  int parts;                  // each batch row's keys are cut into so many
  float scale_log2;           // scale * log2(e)
};

constexpr float kLn2 = 0.69314718055994531f;

// The keys of batch row b: first row and number.  Whatever the offsets and lengths say, no more than the tensor has.
__device__ __forceinline__ void cross_range(const CrossArgs& a, int b, long long& start, int& len) {
  if (a.cu_seqlens) {
    const long long lo = min(max((long long)a.cu_seqlens[b], 0LL), a.n_keys), hi = min(max((long long)a.cu_seqlens[b + 1], lo), a.n_keys);
    start = lo;
    len = (int)(hi - lo);
  } else {
    start = b * a.Lk;
    len = (int)(a.lengths ? min(max((long long)a.lengths[b], 0LL), a.Lk) : a.Lk);
  }
}
// Part `p` of `parts` of a row's keys, whole tiles of `tile` keys each.
__device__ __forceinline__ void cross_part(int len, int p, int parts, int tile, int& lo, int& hi) {
  const int tiles = (len + tile - 1) / tile;
  lo = min(len, (int)((long long)tiles * p / parts) * tile);
  hi = min(len, (int)((long long)tiles * (p + 1) / parts) * tile);
}
__device__ __forceinline__ bool key_counts(const CrossArgs& a, long long row) { return !a.mask || a.mask[row]; }

// Subtracted from scores: the running maximum, or zero while every score has been -inf (then all of them give e^-inf = 0).
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float lse_of(float m, float l) { return kLn2 * (m + log2f(l)); }

// What is left of a (token, head) when its keys are done: the result itself, or a part's share of it.
template <typename Tio, int N>
__device__ __forceinline__ void cross_put(const CrossArgs& a, long long token, int head, int c, const float (&o)[N], float m, float l,
                                          int part, int d) {
  if (a.parts > 1) {
    const long long at = (token * a.H + head) * a.parts + part;
#pragma unroll
    for (int i = 0; i < N; i += 4) store4(a.part_o + at * d + c + i, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
    if (c == 0) a.part_ml[at] = make_float2(m, l);
  } else {
    const float r = l == 0.f ? 0.f : 1.f / l;
    Tio* p = static_cast<Tio*>(a.out) + token * a.out_stride + (long long)head * d + c;
#pragma unroll
    for (int i = 0; i < N; i += 4) store4(p + i, make_float4(o[i] * r, o[i + 1] * r, o[i + 2] * r, o[i + 3] * r));
    if (c == 0 && a.lse) a.lse[token * a.H + head] = lse_of(m, l);
  }
}

// ---------------------------------------------------------------------------------------------- few rows
// R rows of one key head, a CTA of eight warps over a part of the keys.  A key's channels lie across as many lanes as 16-byte
// pieces make them up, so a warp holds 1 to 4 keys at once, U of them one behind another in flight; every such slot keeps its own
// (m, l, o), joined at the end.  Bound by the keys' and values' bytes.
template <typename Tio, int D, int R>
__global__ void __launch_bounds__(256) cross_few_kernel(CrossArgs a) {
  constexpr int N = 16 / sizeof(Tio), LANES = D / N, SLOTS = 32 / LANES, WARPS = 8, U = R <= 2 ? 4 : 2;
  constexpr int STEP = WARPS * SLOTS * U;
  __shared__ float so[WARPS][R][D];
  __shared__ float2 sml[WARPS][R];
  if (a.parts > 1) let_next_kernel_start();
  const int tiles = (a.Lq * a.group + R - 1) / R;
  long long unit = blockIdx.x;
  const int part = (int)(unit % a.parts); unit /= a.parts;
  const int row0 = (int)(unit % tiles) * R; unit /= tiles;
  const int hk = (int)(unit % a.Hk), b = (int)(unit / a.Hk);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, slot = lane / LANES, c = (lane % LANES) * N;
  const int rows = min(R, a.Lq * a.group - row0);
  long long start;
  int len, lo, hi;
  cross_range(a, b, start, len);
  cross_part(len, part, a.parts, STEP, lo, hi);

  float q[R][N], o[R][N] = {}, m[R], l[R] = {};
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    const int row = row0 + min(r, rows - 1), i = row / a.group;
    const Tio* p = static_cast<const Tio*>(a.q) + ((long long)b * a.Lq + i) * a.q_stride + (long long)(hk * a.group + row - i * a.group) * D + c;
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const float4 x = load4(p + j);
      q[r][j] = x.x * a.scale_log2; q[r][j + 1] = x.y * a.scale_log2; q[r][j + 2] = x.z * a.scale_log2; q[r][j + 3] = x.w * a.scale_log2;
    }
  }
  const Tio* kp = static_cast<const Tio*>(a.k) + start * a.k_stride + (long long)hk * D + c;
  const Tio* vp = static_cast<const Tio*>(a.v) + start * a.v_stride + (long long)hk * D + c;
  for (int j0 = lo + (warp * SLOTS + slot); j0 - (warp * SLOTS + slot) < hi; j0 += STEP) {
    float k[U][N], v[U][N];
    bool on[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * WARPS * SLOTS;
      on[u] = j < hi && key_counts(a, start + j);
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        const float4 x = on[u] ? load4(kp + j * a.k_stride + i) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float4 y = on[u] ? load4(vp + j * a.v_stride + i) : make_float4(0.f, 0.f, 0.f, 0.f);
        k[u][i] = x.x; k[u][i + 1] = x.y; k[u][i + 2] = x.z; k[u][i + 3] = x.w;
        v[u][i] = y.x; v[u][i + 1] = y.y; v[u][i + 2] = y.z; v[u][i + 3] = y.w;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float z[U], top = m[r];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        z[u] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) z[u] = fmaf(q[r][i], k[u][i], z[u]);
#pragma unroll
        for (int s = LANES / 2; s > 0; s /= 2) z[u] += __shfl_xor_sync(0xffffffffu, z[u], s);
        if (!on[u]) z[u] = -INFINITY;
        top = fmaxf(top, z[u]);
      }
      const float base = finite_max(top), keep = exp2_fast(m[r] - base);
      m[r] = top;
      l[r] *= keep;
#pragma unroll
      for (int i = 0; i < N; ++i) o[r][i] *= keep;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float p = exp2_fast(z[u] - base);
        l[r] += p;
#pragma unroll
        for (int i = 0; i < N; ++i) o[r][i] = fmaf(p, v[u][i], o[r][i]);
      }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {                                          // the slots of a warp
#pragma unroll
    for (int s = LANES; s < 32; s *= 2) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[r], s), lo_ = __shfl_xor_sync(0xffffffffu, l[r], s);
      const float top = fmaxf(m[r], mo), base = finite_max(top), x = exp2_fast(m[r] - base), y = exp2_fast(mo - base);
      l[r] = l[r] * x + lo_ * y;
#pragma unroll
      for (int i = 0; i < N; ++i) o[r][i] = o[r][i] * x + __shfl_xor_sync(0xffffffffu, o[r][i], s) * y;
      m[r] = top;
    }
    if (slot == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) so[warp][r][c + i] = o[r][i];
      if (lane == 0) sml[warp][r] = make_float2(m[r], l[r]);
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < rows * (D / 4); t += 256) {              // the warps
    const int r = t / (D / 4), cc = (t % (D / 4)) * 4;
    float top = -INFINITY, sum = 0.f, x[4] = {};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, sml[w][r].x);
    const float base = finite_max(top);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = exp2_fast(sml[w][r].x - base);
      sum += sml[w][r].y * f;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = fmaf(so[w][r][cc + i], f, x[i]);
    }
    const int row = row0 + r, i = row / a.group;
    cross_put<Tio>(a, (long long)b * a.Lq + i, hk * a.group + row - i * a.group, cc, x, top, sum, part, D);
  }
}

// ---------------------------------------------------------------------------------------------- many rows
// 64 rows of one key head against 64 keys at a time, in shared memory as fp32; keys and then values in the same place, so that two
// CTAs fit on an SM with d = 128.  A thread has 4 x 4 scores (rows of its own, keys 16 apart: reads without bank conflicts) and
// 4 x D/16 results, both as pairs for packed arithmetic (scores: sums over even and odd channels); the 16 threads of a row lie side
// by side in a warp.  Bound by the multiply-adds.
template <int D>
struct CrossPlain {
  static constexpr int ROWS = 64, KEYS = 64, PITCH = D + 4, P_PITCH = KEYS + 4;
  static constexpr int OFF_KV = ROWS * PITCH, OFF_P = OFF_KV + KEYS * PITCH, OFF_ON = OFF_P + ROWS * P_PITCH;
  static constexpr int SMEM_BYTES = (OFF_ON + KEYS) * 4;
};

template <typename Tio, int D>
__global__ void __launch_bounds__(256, 2) cross_plain_kernel(CrossArgs a) {
  using namespace tc;
  using S = CrossPlain<D>;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *skv = smem + S::OFF_KV, *sp = smem + S::OFF_P;
  int* son = reinterpret_cast<int*>(smem + S::OFF_ON);
  if (a.parts > 1) let_next_kernel_start();
  const int tiles = (int)(((long long)a.Lq * a.group + S::ROWS - 1) / S::ROWS);
  long long unit = blockIdx.x;
  const int part = (int)(unit % a.parts); unit /= a.parts;
  const int row0 = (int)(unit % tiles) * S::ROWS; unit /= tiles;
  const int hk = (int)(unit % a.Hk), b = (int)(unit / a.Hk);
  const int rows = min(S::ROWS, a.Lq * a.group - row0);
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
  long long start;
  int len, lo, hi;
  cross_range(a, b, start, len);
  cross_part(len, part, a.parts, S::KEYS, lo, hi);

  for (int t = threadIdx.x; t < S::ROWS * (D / 4); t += 256) {
    const int r = t / (D / 4), c = (t % (D / 4)) * 4, row = row0 + min(r, rows - 1), i = row / a.group;
    float4 x = load4(static_cast<const Tio*>(a.q) + ((long long)b * a.Lq + i) * a.q_stride + (long long)(hk * a.group + row - i * a.group) * D + c);
    x.x *= a.scale_log2; x.y *= a.scale_log2; x.z *= a.scale_log2; x.w *= a.scale_log2;
    store4(sq + r * S::PITCH + c, x);
  }
  uint64_t o[4][D / 32];
  float m[4], l[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[i][c] = 0ull;
  }
  for (int j0 = lo; j0 < hi; j0 += S::KEYS) {
    __syncthreads();
    if (threadIdx.x < S::KEYS) son[threadIdx.x] = j0 + (int)threadIdx.x < hi && key_counts(a, start + j0 + threadIdx.x);
    __syncthreads();
    auto fetch = [&](const void* from, long long stride) {
#pragma unroll 4
      for (int t = threadIdx.x; t < S::KEYS * (D / 4); t += 256) {
        const int r = t / (D / 4), c = (t % (D / 4)) * 4;
        store4(skv + r * S::PITCH + c, son[r] ? load4(static_cast<const Tio*>(from) + (start + j0 + r) * stride + (long long)hk * D + c)
                                              : make_float4(0.f, 0.f, 0.f, 0.f));
      }
      __syncthreads();
    };
    fetch(a.k, a.k_stride);
    uint64_t z2[4][4] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      ulonglong2 x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(sq + (ty * 4 + i) * S::PITCH + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const ulonglong2*>(skv + (tx + 16 * j) * S::PITCH + c);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) z2[i][j] = f2_fma(x[i].y, y[j].y, f2_fma(x[i].x, y[j].x, z2[i][j]));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float z[4], top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float z0, z1;
        f2_unpack(z2[i][j], z0, z1);
        z[j] = son[tx + 16 * j] ? z0 + z1 : -INFINITY;
        top = fmaxf(top, z[j]);
      }
#pragma unroll
      for (int s = 8; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
      const float base = finite_max(top), keep = exp2_fast(m[i] - base);
      m[i] = top;
      l[i] *= keep;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2_fast(z[j] - base);
        l[i] += p;                                                       // (this thread's keys; the row's 16 are added at the end)
        sp[(ty * 4 + i) * S::P_PITCH + tx + 16 * j] = p;
      }
      const uint64_t keep2 = f2_pack(keep, keep);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[i][c] = f2_fma(o[i][c], keep2, 0ull);
    }
    __syncthreads();                                                     // all have read the keys
    fetch(a.v, a.v_stride);
#pragma unroll 2
    for (int j = 0; j < S::KEYS; j += 4) {
      float4 p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = load4(sp + (ty * 4 + i) * S::P_PITCH + j);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(skv + (j + u) * S::PITCH + c * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
            const uint64_t w2 = f2_pack(w, w);
            o[i][2 * c] = f2_fma(w2, y.x, o[i][2 * c]);
            o[i][2 * c + 1] = f2_fma(w2, y.y, o[i][2 * c + 1]);
          }
        }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int s = 8; s > 0; s /= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], s);
    const int r = ty * 4 + i;
    if (r >= rows) continue;
    const int row = row0 + r, t = row / a.group;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      float x[4];
      f2_unpack(o[i][2 * c], x[0], x[1]);
      f2_unpack(o[i][2 * c + 1], x[2], x[3]);
      cross_put<Tio>(a, (long long)b * a.Lq + t, hk * a.group + row - t * a.group, c * 64 + tx * 4, x, m[i], l[i], part, D);
    }
  }
}

// ---------------------------------------------------------------------------------------------- parts
// A warp to a (token, head).  Starts while its predecessor runs.
template <typename Tio, int D>
__global__ void __launch_bounds__(256) cross_join_kernel(CrossArgs a) {
  constexpr int N = D / 32;
  wait_for_kernel_before();
  const long long at = (long long)blockIdx.x * 8 + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  if (at >= (long long)a.B * a.Lq * a.H) return;
  const float2* ml = a.part_ml + at * a.parts;
  const float* o = a.part_o + at * a.parts * D + lane * N;
  float top = -INFINITY, sum = 0.f, x[N] = {};
  for (int p = lane; p < a.parts; p += 32) top = fmaxf(top, ml[p].x);
#pragma unroll
  for (int s = 16; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  const float base = finite_max(top);
  for (int p = 0; p < a.parts; ++p) {
    const float2 y = ml[p];
    const float f = exp2_fast(y.x - base);
    sum = fmaf(y.y, f, sum);
    // (a part without a key that counts has left zeros)
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(o[(long long)p * D + i], f, x[i]);
  }
  const float r = sum == 0.f ? 0.f : 1.f / sum;
  const long long token = at / a.H;
  Tio* out = static_cast<Tio*>(a.out) + token * a.out_stride + (at - token * a.H) * D + lane * N;
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = from_float<Tio>(x[i] * r);
  if (lane == 0 && a.lse) a.lse[at] = lse_of(top, sum);
}

}  // namespace vdn
