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
  float* long_o;              // tensor cores, long parts: sums of the keys so far, [CTA][d + 2][256]
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

// 16 bytes as floats.
template <typename Tio>
__device__ __forceinline__ void piece_floats(const uint4& r, float (&x)[16 / sizeof(Tio)]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(Tio) == 4) {
      x[i] = __uint_as_float(w[i]);
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}

// ---------------------------------------------------------------------------------------------- few rows
// R rows of one key head, a CTA of eight warps over a part of the keys.  A key's channels lie across as many lanes as 16-byte
// pieces make them up, so a warp holds 1 to 4 keys at once, U of them one behind another in flight; every such slot keeps its own
// (m, l, o), joined at the end.  Bound by the keys' and values' bytes: 32 requests of 32 heads, 1500 keys, d = 128: 134 us, 5.9 TB/s (182
// without fetching a step ahead); one request of 40 heads, 512 keys: 7.1 us, latencies.
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
  struct Step { uint4 k[U], v[U]; bool on[U]; };
  auto fetch = [&](int first, Step& x) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = first + u * WARPS * SLOTS;
      x.on[u] = j < hi && key_counts(a, start + j);
      x.k[u] = x.v[u] = make_uint4(0, 0, 0, 0);
      if (x.on[u]) {
        x.k[u] = *reinterpret_cast<const uint4*>(kp + j * a.k_stride);
        x.v[u] = *reinterpret_cast<const uint4*>(vp + j * a.v_stride);
      }
    }
  };
  const int mine = warp * SLOTS + slot;
  Step next;
  fetch(lo + mine, next);
  for (int j0 = lo; j0 < hi; j0 += STEP) {
    const Step x = next;
    if (j0 + STEP < hi) fetch(j0 + STEP + mine, next);                    // while these are worked on
    float k[U][N], v[U][N];
    const bool (&on)[U] = x.on;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      piece_floats<Tio>(x.k[u], k[u]);
      piece_floats<Tio>(x.v[u], v[u]);
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
// 128 rows of one key head (64 where that leaves SMs without work) against 64 keys at a time, in shared memory as fp32; values arrive while scores are formed, the next keys
// while the values are summed (f32: by asynchronous copies).  A thread has 4 x 4 scores (rows of its own, keys 16 apart: reads
// without bank conflicts) and 4 x D/16 results, both as pairs for packed arithmetic (scores: sums over even and odd channels); the
// 16 threads of a row lie side by side in a warp.  64 rows and d = 128 leave room for one CTA on an SM (119 KB; the bound of 128 registers
// is for two, as with d = 64: 16 batch rows of 40 queries x 1500 keys x 8 heads 219 us, without it 215).  Bound by the multiply-adds and the shared-memory reads that feed them: 4096 x 4096 x
// 8 heads, f32: d = 128 1825 us, 38 TFLOP/s, d = 64 1053 us, 33 TFLOP/s.  (8 x 4 scores a thread, half as many threads: 2890 us.)
template <int D, int TILE>
struct CrossPlain {
  static constexpr int ROWS = TILE, KEYS = 64, THREADS = 4 * ROWS, PITCH = D + 4, P_PITCH = KEYS + 4;
  static constexpr int OFF_K = ROWS * PITCH, OFF_V = OFF_K + KEYS * PITCH, OFF_P = OFF_V + KEYS * PITCH;
  static constexpr int SMEM_BYTES = (OFF_P + ROWS * P_PITCH) * 4;
};

// 16 bytes of shared memory from global memory, or zeros.
__device__ __forceinline__ void cp_async16_or_zero(void* smem_dst, const void* gmem_src, bool on) {
  const uint32_t s = (uint32_t)__cvta_generic_to_shared(smem_dst);
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(s), "l"(gmem_src), "r"(on ? 16 : 0) : "memory");
}

template <typename Tio, int D, int TILE>
__global__ void __launch_bounds__(CrossPlain<D, TILE>::THREADS, 512 / CrossPlain<D, TILE>::THREADS) cross_plain_kernel(CrossArgs a) {
  using namespace tc;
  using S = CrossPlain<D, TILE>;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = smem + S::OFF_K, *sv = smem + S::OFF_V, *sp = smem + S::OFF_P;
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

  auto fetch = [&](float* to, const void* from, long long stride, int j0) {
#pragma unroll
    for (int t = threadIdx.x; t < S::KEYS * (D / 4); t += S::THREADS) {
      const int r = t / (D / 4), c = (t % (D / 4)) * 4;
      const bool on = j0 + r < hi && key_counts(a, start + j0 + r);
      const Tio* p = static_cast<const Tio*>(from) + (on ? (start + j0 + r) * stride + (long long)hk * D + c : 0);
      if constexpr (sizeof(Tio) == 4) cp_async16_or_zero(to + r * S::PITCH + c, p, on);
      else store4(to + r * S::PITCH + c, on ? load4(p) : make_float4(0.f, 0.f, 0.f, 0.f));
    }
    cp_async_commit();
  };
  if (lo < hi) fetch(sk, a.k, a.k_stride, lo);
  for (int t = threadIdx.x; t < S::ROWS * (D / 4); t += S::THREADS) {
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
    fetch(sv, a.v, a.v_stride, j0);
    bool on[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) on[j] = j0 + tx + 16 * j < hi && key_counts(a, start + j0 + tx + 16 * j);
    cp_async_wait<1>();                                                  // the keys
    __syncthreads();
    float keep[4];
    uint64_t z2[4][4] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      ulonglong2 x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const ulonglong2*>(sq + (ty * 4 + i) * S::PITCH + c);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const ulonglong2*>(sk + (tx + 16 * j) * S::PITCH + c);
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
        z[j] = on[j] ? z0 + z1 : -INFINITY;
        top = fmaxf(top, z[j]);
      }
#pragma unroll
      for (int s = 8; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
      const float base = finite_max(top);
      keep[i] = exp2_fast(m[i] - base);
      m[i] = top;
      float sum = 0.f;                                                   // (this thread's keys; the row's 16 are added at the end)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2_fast(z[j] - base);
        sum += p;
        sp[(ty * 4 + i) * S::P_PITCH + tx + 16 * j] = p;
      }
      l[i] = fmaf(l[i], keep[i], sum);
    }
    __syncthreads();                                                     // all have read the keys
    if (j0 + S::KEYS < hi) fetch(sk, a.k, a.k_stride, j0 + S::KEYS);
    else cp_async_commit();
    cp_async_wait<1>();                                                  // the values
    __syncthreads();
    // a tile's values by themselves first: what is small beside a long sum would get lost in it
    uint64_t t[4][D / 32] = {};
#pragma unroll 2
    for (int j = 0; j < S::KEYS; j += 4) {
      float4 p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = load4(sp + (ty * 4 + i) * S::P_PITCH + j);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(sv + (j + u) * S::PITCH + c * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
            const uint64_t w2 = f2_pack(w, w);
            t[i][2 * c] = f2_fma(w2, y.x, t[i][2 * c]);
            t[i][2 * c + 1] = f2_fma(w2, y.y, t[i][2 * c + 1]);
          }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[i][c] = f2_fma(o[i][c], f2_pack(keep[i], keep[i]), t[i][c]);
    __syncthreads();                                                     // ... and the values
  }
  cp_async_wait<0>();
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
// A warp to 32 channels of a (token, head), eight parts in flight (rows are few where parts are many).  Starts while its predecessor runs.
template <typename Tio, int D>
__global__ void __launch_bounds__(256) cross_join_kernel(CrossArgs a) {
  constexpr int PER = D / 32, BATCH = 8;
  wait_for_kernel_before();
  const long long unit = (long long)blockIdx.x * 8 + threadIdx.x / 32, at = unit / PER;
  const int lane = threadIdx.x % 32, c = (int)(unit % PER) * 32 + lane;
  if (at >= (long long)a.B * a.Lq * a.H) return;
  const float2* ml = a.part_ml + at * a.parts;
  const float* o = a.part_o + at * a.parts * D + c;
  float top = -INFINITY, sum = 0.f, x = 0.f;
  for (int p = lane; p < a.parts; p += 32) top = fmaxf(top, ml[p].x);
#pragma unroll
  for (int s = 16; s > 0; s /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  const float base = finite_max(top);
  for (int p0 = 0; p0 < a.parts; p0 += BATCH) {
    float2 y[BATCH];
    float z[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const bool on = p0 + i < a.parts;
      y[i] = on ? ml[p0 + i] : make_float2(-INFINITY, 0.f);
      z[i] = on ? o[(long long)(p0 + i) * D] : 0.f;
    }
    // (a part without a key that counts has left zeros)
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float f = exp2_fast(y[i].x - base);
      sum = fmaf(y[i].y, f, sum);
      x = fmaf(z[i], f, x);
    }
  }
  const float r = sum == 0.f ? 0.f : 1.f / sum;
  const long long token = at / a.H;
  static_cast<Tio*>(a.out)[token * a.out_stride + (at - token * a.H) * D + c] = from_float<Tio>(x * r);
  if (c == 0 && a.lse) a.lse[at] = lse_of(top, sum);
}

}  // namespace vdn
