// Rotary positions on three axes (time, height, width) for queries and keys, with an optional RMSNorm of each head's
// channels before the rotation.
//
// Pair p of a head's channels is turned by the angle  position(token, axis[p]) * freq[p].  The angle is formed in 64
// bits, as turns, and only its fraction of a turn is rounded to 32 bits: at position 10^5 a 32-bit product would be off by
// up to 4e-3 radians.  A CTA first writes the cosines and sines of its tokens to shared memory -- they are the same for
// all heads of the queries and the keys -- and then streams the heads through registers: a lane holds two 16-byte
// pieces, which are the two halves of its pairs (HALF) or hold whole neighbouring pairs.  Bound by HBM: each tensor is
// read once and written once.  768p clip, 40 heads of queries and of keys: 2.10 ms on the same tensors again and again, 2.16 ms on others in
// turn (6.7 TB/s; the measured copy: 6.6); 480p clip, 8 and 2 heads: 37 us without norm, 43 with it, where a plain copy of as many
// bytes takes 31: with the norm it is short of issue slots (64 % used, DRAM 37 %).
#pragma once
#include <cuda_bf16.h>

#include <type_traits>

#include "common.cuh"

namespace vdn {

struct RotaryArgs {
  const void* in[2];         // queries, keys (or null)
  void* out[2];
  const float* weight[2];    // [d] or null
  long long in_stride[2], out_stride[2];   // elements from one token to the next
  int heads[2];              // 0 for keys left out
  const double* freq;        // [pairs]
  const int* axis;           // [pairs]; anything but 0, 1, 2 leaves the pair as it is
  const int* positions;      // [3][n_tokens] or null: frame t0 + t, row, column of the token's grid place
  long long n_tokens;
  int pairs, T, F, X, t0, tile;
  unsigned per_row;          // rotary_per_row
  float norm_eps;            // > 0: RMSNorm first
  float sign;                // -1: rotate back
};

struct Rotary {
  static constexpr int THREADS = 256;
  static constexpr int MAX_TILE = 32;      // tokens a CTA covers
  static constexpr int UNROLL = 2;         // head rows a lane has in flight
};

// A tile's head rows are counted through, `rows` (all heads of queries and keys) to a token: row t belongs to token t / rows.
// Division by multiplication with ceil(2^32 / rows) = (2^32 + e) / rows, e < rows: right while t * e < 2^32, and a tile of more than
// one token has fewer than 512 rows to a token and 32 tokens at most.  One row to a token (queries of one head alone) has no such
// factor in 32 bits, and needs none; nor does a tile of one token, whose rows may be many.
__host__ __device__ inline unsigned rotary_per_row(int rows, int tile) {
  return tile > 1 && rows > 1 ? (unsigned)((0x100000000ULL + rows - 1) / rows) : 0u;
}
__host__ __device__ inline int rotary_token(int t, int rows, unsigned per_row) {
  return rows == 1 ? t : (int)(((unsigned long long)(unsigned)t * per_row) >> 32);
}

// 16 bytes of a head's channels as floats, and back
__device__ __forceinline__ void unpack16(const uint4& r, float (&x)[4], const float*) {
  x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack16(const uint4& r, float (&x)[8], const __nv_bfloat16*) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack16(const float (&x)[4], const float*) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack16(const float (&x)[8], const __nv_bfloat16*) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename Tio, int D, bool HALF, bool NORM>
__global__ void __launch_bounds__(Rotary::THREADS, 4) rotary_kernel(const RotaryArgs a) {
  constexpr int VEC = 16 / (int)sizeof(Tio);       // channels of a 16-byte piece
  constexpr int LPH = D / (2 * VEC);               // lanes of a head
  constexpr int NP = VEC;                          // pairs of a lane
  constexpr int P4 = NP / 2;                       // float4's (two pairs each) of a lane's cosines and sines
  constexpr int STEP = Rotary::THREADS / LPH;      // head rows side by side
  constexpr int U = Rotary::UNROLL;
  // 1 for a pair that is turned, in the order the lanes take them; the channels of the others are copied, not computed: times 1 and
  // 0 an infinite partner would make them NaN
  __shared__ alignas(8) unsigned char on_axis[D / 2];
  // [token][pair / 2 mod P4][lane][cos, sin, cos, sin]: the lanes of a head read 16-byte pieces side by side
  extern __shared__ float4 table[];
  // of queries and keys, in the order the lanes take them: [4 channels of the first piece .. of the second][lane]
  __shared__ float4 weight[NORM ? 2 : 1][NORM ? VEC / 2 : 1][LPH];
  const long long n0 = (long long)blockIdx.x * a.tile;
  const int nt = (int)min((long long)a.tile, a.n_tokens - n0);

  // heads: task = (token of the tile, head row of queries then keys, lane)
  const int rows = a.heads[0] + a.heads[1];
  const int tasks = nt * rows;
  const int l = threadIdx.x % LPH, first = (int)threadIdx.x / LPH;
  // first channel of the lane's two pieces
  int c0 = 2 * l * VEC, c1 = c0 + VEC;
  if (HALF && l * VEC < a.pairs) { c0 = l * VEC; c1 = c0 + a.pairs; }
  bool turned;
  // ---- cosines and sines: a thread has one place lp = lane * NP + pair of the lane, and every (256 / places)-th token
  {
    constexpr int PLACES = D / 2, TOKENS = Rotary::THREADS / PLACES;
    const int lp = threadIdx.x % PLACES, tl = lp / NP, ti = lp % NP;
    // the pair that the place stands for; HALF: lanes past the rotated channels pass theirs through
    const int p = HALF ? (tl * VEC < a.pairs ? lp : a.pairs) : lp;
    const int ax = p < a.pairs ? a.axis[p] : -1;
    turned = ax >= 0 && ax <= 2;
    if (threadIdx.x < PLACES) on_axis[lp] = turned;
    const double turn = turned ? a.freq[p] * 0.15915494309189533577 : 0.0;   // 1 / (2 pi)
    for (int j = (int)threadIdx.x / PLACES; j < nt; j += TOKENS) {
      float c = 1.f, s = 0.f;
      if (turned) {
        const long long n = n0 + j;
        int pos;
        if (a.positions) {
          pos = a.positions[(size_t)ax * a.n_tokens + n];
        } else {
          const unsigned fr = (unsigned)n / (unsigned)a.F, u = (unsigned)n - fr * (unsigned)a.F;
          pos = ax == 0 ? a.t0 + (int)(fr % (unsigned)a.T) : ax == 1 ? (int)(u / (unsigned)a.X) : (int)(u % (unsigned)a.X);
        }
        const double turns = (double)pos * turn;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        s *= a.sign;
      }
      float* t = reinterpret_cast<float*>(&table[(j * P4 + ti / 2) * LPH + tl]);
      *reinterpret_cast<float2*>(t + (ti & 1) * 2) = make_float2(c, s);
    }
  }
  if constexpr (NORM) {
    if (threadIdx.x < 2 * (VEC / 2) * LPH) {
      const int w = (int)threadIdx.x / (VEC / 2 * LPH), k = (int)threadIdx.x / LPH % (VEC / 2);   // l is the thread's own lane
      const int c = k < VEC / 4 ? c0 + 4 * k : c1 + 4 * (k - VEC / 4);
      const float* g = a.weight[w];
      weight[w][k][l] = g ? make_float4(g[c], g[c + 1], g[c + 2], g[c + 3]) : make_float4(1.f, 1.f, 1.f, 1.f);
    }
  }
  const bool all = __syncthreads_and(turned);
  const unsigned char* on = on_axis + l * NP;

  // whole: every pair is turned.  A loop of its own: asked for each head row it cost 2 % (768p) to 5 % (480p, norms); a block with
  // pairs that are not turned pays 2 to 3 % for copying them (160 000 tokens x 48 heads, 32 of 64 pairs: 594 -> 608 us).
  auto heads = [&](auto whole) {
    for (int base = first; base < tasks + first; base += STEP * U) {   // (all lanes together: the norm shuffles)
      uint4 x0[U], x1[U];
      int token[U], head[U];
      bool key[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = base + u * STEP;
        x0[u] = x1[u] = make_uint4(0, 0, 0, 0);
        token[u] = head[u] = 0;
        key[u] = false;
        if (t < tasks) {
          token[u] = rotary_token(t, rows, a.per_row);
          head[u] = t - token[u] * rows;
          key[u] = head[u] >= a.heads[0];
          if (key[u]) head[u] -= a.heads[0];
          const Tio* src = static_cast<const Tio*>(a.in[key[u]]) + (size_t)(n0 + token[u]) * a.in_stride[key[u]] + head[u] * D;
          x0[u] = *reinterpret_cast<const uint4*>(src + c0);
          x1[u] = *reinterpret_cast<const uint4*>(src + c1);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool live = base + u * STEP < tasks;
        const int j = token[u], w = key[u];
        float y0[VEC], y1[VEC];
        unpack16(x0[u], y0, static_cast<const Tio*>(nullptr));
        unpack16(x1[u], y1, static_cast<const Tio*>(nullptr));
        if constexpr (NORM) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < VEC; ++i) ss += y0[i] * y0[i] + y1[i] * y1[i];
#pragma unroll
          for (int m = 1; m < LPH; m <<= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, m);
          const float rn = rsqrtf(ss * (1.f / D) + a.norm_eps);
#pragma unroll
          for (int i = 0; i < VEC; i += 4) {
            const float4 g = weight[w][i / 4][l], k = weight[w][VEC / 4 + i / 4][l];
            y0[i] *= rn * g.x; y0[i + 1] *= rn * g.y; y0[i + 2] *= rn * g.z; y0[i + 3] *= rn * g.w;
            y1[i] *= rn * k.x; y1[i + 1] *= rn * k.y; y1[i + 2] *= rn * k.z; y1[i + 3] *= rn * k.w;
          }
        }
#pragma unroll
        for (int i = 0; i < NP; i += 2) {
          const float4 cs = table[(j * P4 + i / 2) * LPH + l];
          // HALF: pair i is channel i of either piece; else pairs i, i + 1 are channels 2i .. 2i + 3 of the 2 VEC neighbouring ones
          float* y = HALF ? &y0[i] : 2 * i < VEC ? &y0[(2 * i) % VEC] : &y1[(2 * i) % VEC];
          float& a0 = y[0];
          float& b0 = HALF ? y1[i] : y[1];
          float& a1 = HALF ? y[1] : y[2];
          float& b1 = HALF ? y1[i + 1] : y[3];
          const float p0 = a0, z0 = b0, p1 = a1, z1 = b1;
          if (whole || on[i]) { a0 = p0 * cs.x - z0 * cs.y; b0 = p0 * cs.y + z0 * cs.x; }
          if (whole || on[i + 1]) { a1 = p1 * cs.z - z1 * cs.w; b1 = p1 * cs.w + z1 * cs.z; }
        }
        if (live) {
          Tio* dst = static_cast<Tio*>(a.out[w]) + (size_t)(n0 + j) * a.out_stride[w] + head[u] * D;
          *reinterpret_cast<uint4*>(dst + c0) = pack16(y0, static_cast<const Tio*>(nullptr));
          *reinterpret_cast<uint4*>(dst + c1) = pack16(y1, static_cast<const Tio*>(nullptr));
        }
      }
    }
  };
  if (all) heads(std::true_type());
  else heads(std::false_type());
}

}  // namespace vdn
