// Attention of each query to all the states of its batch row's encoder on the tensor cores; bf16 I/O, d = 64 or 128.
//
// The rows of a key head are its queries times the heads of its group.  They go in blocks of up to 32 (a warp's share: whole tokens,
// or 32 heads of one), four blocks to a tile of 128, two tiles to a CTA.  Per tile and 128 keys:
//   S = Q K^T      (128 x 128 x d, both operands in shared memory, S in tensor memory)
//   P = 2^(c S - m)  a thread to a row: the maximum, the exponentials and their sum in fp32, P as bf16 over S in tensor memory
//   O += P V       (128 x d x 128, P from tensor memory, V as it lies in shared memory)
// The two tiles take turns: while one is exponentiated the other is multiplied.  O stays in tensor memory; it is brought to a new
// maximum only where that has grown by more than 2^8 (else P goes up to 2^8, which bf16 and fp32 hold as well), by the
// warp that found it, between its tile's products.
// Keys that do not count: their scores are replaced by -inf, their rows of V by zeros in shared memory (zero times what may
// be anything is not zero).
#pragma once
#include "cross_simt.cuh"
#include "tc_common.cuh"
#include "token_rule.cuh"
#include "token_tc.cuh"

namespace vdn {

struct CrossTcShape {
  int hb, tb;                 // heads and tokens of a row block
  int head_blocks;            // ceil(group / hb)
  int pairs;                  // pairs of tiles of a (batch row, key head)
  long long items;            // B * Hk * pairs * parts
};

template <int D>
struct CrossTc {
  static constexpr int KEYS = 128, THREADS = 384, CHUNKS = D / 64;
  static constexpr int TILE_BYTES = 128 * D * 2, CHUNK_BYTES = 128 * 128, OUT_BYTES = 32 * 128;
  static constexpr int STAGES = D == 128 ? 2 : 4;                       // of keys, and of values
  static constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + STAGES * TILE_BYTES, OFF_OUT = OFF_V + STAGES * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_OUT + 8 * OUT_BYTES;
  static constexpr int BARS = 2 + 2 + 5 * STAGES + 2 + 4 + 2 + 2;
  static constexpr int USED_BYTES = OFF_BAR + 8 * BARS + 16, SMEM_BYTES = USED_BYTES + 1024;
  static constexpr int COL_S = 0, COL_O = 256, COLS = 512;              // tensor memory: S of both tiles, O of both
};
static_assert(CrossTc<128>::SMEM_BYTES <= 232448, "shared memory of a CTA");

// What every role of the CTA derives of an item.
struct CrossItem {
  int b, hk, pair, part, lo, hi, tiles;        // keys lo .. hi-1 of the batch row, in so many tiles
  long long start;
  bool second;                                  // the pair's second tile has rows
};
__device__ __forceinline__ CrossItem cross_item(const CrossArgs& a, const CrossTcShape& s, long long item) {
  CrossItem x;
  x.part = (int)(item % a.parts); item /= a.parts;
  x.pair = (int)(item % s.pairs); item /= s.pairs;
  x.hk = (int)(item % a.Hk);
  x.b = (int)(item / a.Hk);
  int len;
  cross_range(a, x.b, x.start, len);
  cross_part(len, x.part, a.parts, 128, x.lo, x.hi);
  x.tiles = (x.hi - x.lo + 127) / 128;
  const long long blocks = (long long)((a.Lq + s.tb - 1) / s.tb) * s.head_blocks;
  x.second = ((long long)x.pair * 2 + 1) * 4 < blocks;
  return x;
}

template <int D>
__global__ void __launch_bounds__(CrossTc<D>::THREADS, 1)
cross_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                const __grid_constant__ CUtensorMap tmOut, const CrossArgs a, const CrossTcShape s, tc::DevStatus ds) {
  using namespace tc;
  using G = CrossTc<D>;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + G::OFF_BAR;
  auto Q_FULL = [&](int c) { return bar0 + 8u * c; };
  auto Q_EMPTY = [&](int c) { return bar0 + 8u * (2 + c); };
  auto K_FULL = [&](int i) { return bar0 + 8u * (4 + i); };
  auto K_EMPTY = [&](int i) { return bar0 + 8u * (4 + G::STAGES + i); };
  auto V_FULL = [&](int i) { return bar0 + 8u * (4 + 2 * G::STAGES + i); };
  auto V_READY = [&](int i) { return bar0 + 8u * (4 + 3 * G::STAGES + i); };
  auto V_EMPTY = [&](int i) { return bar0 + 8u * (4 + 4 * G::STAGES + i); };
  auto S_FULL = [&](int c) { return bar0 + 8u * (4 + 5 * G::STAGES + c); };
  auto P_READY = [&](int c) { return bar0 + 8u * (6 + 5 * G::STAGES + c); };
  auto O_FULL = [&](int c) { return bar0 + 8u * (10 + 5 * G::STAGES + c); };
  auto O_EMPTY = [&](int c) { return bar0 + 8u * (12 + 5 * G::STAGES + c); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + G::OFF_BAR + 8 * G::BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const WaitCtx wc(abort_flag, ds);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int c = 0; c < 2; ++c) {
      mbar_init(Q_FULL(c), 1); mbar_init(Q_EMPTY(c), 1);
      mbar_init(S_FULL(c), 1);
      mbar_init(P_READY(2 * c), 4); mbar_init(P_READY(2 * c + 1), 4);   // a warp an arrival
      mbar_init(O_FULL(c), 1); mbar_init(O_EMPTY(c), 4);
    }
    for (int i = 0; i < G::STAGES; ++i) {
      mbar_init(K_FULL(i), 1); mbar_init(K_EMPTY(i), 1);
      mbar_init(V_FULL(i), 1); mbar_init(V_READY(i), 1); mbar_init(V_EMPTY(i), 1);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(tmem_slot), G::COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const int block_rows = s.hb * s.tb;

  if (warp >= 8) {
    registers_fewer<72>();
    if (warp == 8) {
      // ------------------------------------------------------------------ copies
      if (lane == 0) {
        uint32_t kv = 0, q[2] = {0, 0};
        bool ok = true;
        for (long long item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
          const CrossItem x = cross_item(a, s, item);
          if (x.tiles == 0) continue;
          auto load_q = [&](int c) {
            if (!mbar_wait(Q_EMPTY(c), (q[c] & 1) ^ 1, wc)) return false;
            mbar_arrive_expect_tx(Q_FULL(c), 4 * G::CHUNKS * block_rows * 128);
            for (int w = 0; w < 4; ++w) {
              const int rb = (x.pair * 2 + c) * 4 + w;
              const int tok = rb / s.head_blocks * s.tb, head = rb % s.head_blocks * s.hb;
              for (int i = 0; i < G::CHUNKS; ++i)
                tma_load_5d(base + G::OFF_Q + c * G::TILE_BYTES + i * G::CHUNK_BYTES + w * 32 * 128, &tmQ, Q_FULL(c), i * 64, head, x.hk, tok, x.b);
            }
            ++q[c];
            return true;
          };
          auto load = [&](const CUtensorMap* m, uint32_t full, uint32_t empty, int off, int j) {
            if (!mbar_wait(empty, ((kv / G::STAGES) & 1) ^ 1, wc)) return false;
            mbar_arrive_expect_tx(full, G::TILE_BYTES);
            for (int i = 0; i < G::CHUNKS; ++i)
              tma_load_3d(base + off + (kv % G::STAGES) * G::TILE_BYTES + i * G::CHUNK_BYTES, m, full, i * 64, x.hk, (int)(x.start + x.lo + j * 128));
            return true;
          };
          ok = load_q(0);
          for (int j = 0; j < x.tiles && ok; ++j, ++kv) {
            const int st = kv % G::STAGES;
            ok = load(&tmK, K_FULL(st), K_EMPTY(st), G::OFF_K, j);
            if (ok && j == 0 && x.second) ok = load_q(1);
            if (ok) ok = load(&tmV, V_FULL(st), V_EMPTY(st), G::OFF_V, j);
          }
        }
        if (!ok) {
          // a bounded chance for what is under way to land (the last tile of values may not have been asked for: bounded all the same)
          for (int c = 0; c < 2; ++c)
            if (q[c]) mbar_drain(Q_FULL(c), (q[c] - 1) & 1);
          mbar_drain_ring(K_FULL(0), G::STAGES, kv);
          mbar_drain_ring(V_FULL(0), G::STAGES, kv);
        }
      }
    } else if (warp == 9) {
      // ------------------------------------------------------------------ products
      constexpr uint32_t id_s = make_idesc_bf16(128, 128, false, false), id_o = make_idesc_bf16(128, D, false, true);
      uint32_t kv = 0, n_item[2] = {0, 0}, n_p[2] = {0, 0};
      bool ok = true;
      auto scores = [&](int c, uint32_t at) {
        const uint32_t st = at % G::STAGES;
        const uint64_t dq = make_smem_desc(base + G::OFF_Q + c * G::TILE_BYTES, 16, 1024);
        const uint64_t dk = make_smem_desc(base + G::OFF_K + st * G::TILE_BYTES, 16, 1024);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (k >> 2) * (G::CHUNK_BYTES >> 4) + (k & 3) * 2;
            mma_bf16_ss(tmem + G::COL_S + c * 128, dq + off, dk + off, id_s, k ? 1u : 0u);
          }
          mma_commit(S_FULL(c));
        }
        __syncwarp();
      };
      auto commit = [&](uint32_t bar) {
        if (elect_one()) mma_commit(bar);
        __syncwarp();
      };
      for (long long item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
        const CrossItem x = cross_item(a, s, item);
        if (x.tiles == 0) continue;
        const int chains = x.second ? 2 : 1;
        for (int c = 0; c < chains && ok; ++c) {
          ok = mbar_wait_warp(Q_FULL(c), n_item[c] & 1, wc) && mbar_wait_warp(K_FULL(kv % G::STAGES), (kv / G::STAGES) & 1, wc);
          if (!ok) break;
          tc_fence_after_sync();
          scores(c, kv);
        }
        if (!ok) break;
        commit(K_EMPTY(kv % G::STAGES));
        if (x.tiles == 1)
          for (int c = 0; c < chains; ++c) commit(Q_EMPTY(c));
        for (int j = 0; j < x.tiles && ok; ++j, ++kv) {
          const uint32_t st = kv % G::STAGES, next = kv + 1;
          const uint64_t dv = make_smem_desc(base + G::OFF_V + st * G::TILE_BYTES, G::CHUNK_BYTES, 1024);
          for (int c = 0; c < chains; ++c) {
            ok = mbar_wait_warp(V_READY(st), (kv / G::STAGES) & 1, wc) && (j > 0 || mbar_wait_warp(O_EMPTY(c), (n_item[c] & 1) ^ 1, wc));
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              ok = ok && mbar_wait_warp(P_READY(2 * c + half), n_p[c] & 1, wc);
              if (!ok) break;
              tc_fence_after_sync();
              if (elect_one()) {
#pragma unroll
                for (int k = half * 4; k < half * 4 + 4; ++k)
                  mma_bf16_ts(tmem + G::COL_O + c * D, tmem + G::COL_S + c * 128 + k * 8, dv + k * (2048 >> 4), id_o, k || j ? 1u : 0u);
                if (half == 1) {
                  if (j + 1 == x.tiles) mma_commit(O_FULL(c));
                  if (c + 1 == chains) mma_commit(V_EMPTY(st));
                }
              }
              __syncwarp();
            }
            if (!ok) break;
            ++n_p[c];
            if (j + 1 < x.tiles) {
              ok = mbar_wait_warp(K_FULL(next % G::STAGES), (next / G::STAGES) & 1, wc);
              if (!ok) break;
              tc_fence_after_sync();
              scores(c, next);
              if (c + 1 == chains) commit(K_EMPTY(next % G::STAGES));
              if (j + 2 == x.tiles) commit(Q_EMPTY(c));
            }
          }
        }
        for (int c = 0; c < chains; ++c) ++n_item[c];
      }
    } else if (warp == 10) {
      // ------------------------------------------------------------------ values that do not count become zeros
      uint32_t kv = 0;
      bool ok = true;
      for (long long item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
        const CrossItem x = cross_item(a, s, item);
        for (int j = 0; j < x.tiles && ok; ++j, ++kv) {
          const uint32_t st = kv % G::STAGES;
          uint32_t on[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = x.lo + j * 128 + i * 32 + lane;
            on[i] = __ballot_sync(0xffffffffu, key < x.hi && key_counts(a, x.start + key));
          }
          ok = __all_sync(0xffffffffu, mbar_wait(V_FULL(st), (kv / G::STAGES) & 1, wc));
          if (!ok) break;
          if ((on[0] & on[1] & on[2] & on[3]) != 0xffffffffu) {
            unsigned char* v = base_ptr + G::OFF_V + st * G::TILE_BYTES;
            for (int r = lane / 8; r < 128; r += 4)                 // eight lanes to a row's 128 bytes
              if (!((on[r >> 5] >> (r & 31)) & 1u))
                for (int i = 0; i < G::CHUNKS; ++i) *reinterpret_cast<uint4*>(v + i * G::CHUNK_BYTES + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
          }
          mbar_arrive_warp(V_READY(st));
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ exponentials, and the results
    registers_more<216>();
    const int c = warp >> 2, qd = warp & 3;
    const uint32_t ts = tmem + ((uint32_t)(qd * 32) << 16) + G::COL_S + c * 128, to = tmem + ((uint32_t)(qd * 32) << 16) + G::COL_O + c * D;
    const uint32_t out_smem = base + G::OFF_OUT + warp * G::OUT_BYTES;
    unsigned char* out_row = base_ptr + G::OFF_OUT + warp * G::OUT_BYTES + lane * 128;
    const float sl = a.scale_log2;
    uint32_t n_s = 0, n_item = 0;
    bool ok = true;
    for (long long item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
      const CrossItem x = cross_item(a, s, item);
      if (c == 1 && !x.second) continue;
      const int rb = (x.pair * 2 + c) * 4 + qd;
      const int tok0 = rb / s.head_blocks * s.tb, head0 = rb % s.head_blocks * s.hb;
      const int head_in = head0 + lane % s.hb, tok = tok0 + lane / s.hb;
      const bool row_on = lane < block_rows && head_in < a.group && tok < a.Lq;
      float ms = -INFINITY, l = 0.f;                           // the maximum times sl, the sum relative to it
      for (int j = 0; j < x.tiles; ++j, ++n_s) {
        const int key0 = x.lo + j * 128;
        uint32_t on[4];
        bool all = key0 + 128 <= x.hi;
        if (a.mask || !all) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + i * 32 + lane;
            on[i] = __ballot_sync(0xffffffffu, key < x.hi && key_counts(a, x.start + key));
          }
          all = (on[0] & on[1] & on[2] & on[3]) == 0xffffffffu;
        }
        if (!mbar_wait(S_FULL(c), n_s & 1, wc)) { ok = false; break; }
        tc_fence_after_sync();
        uint64_t v[64];                                        // two neighbouring scores each
        tmem_ld128_pairs(ts, v);
        if (!all) {
#pragma unroll
          for (int i = 0; i < 64; ++i) {
            float x0, x1;
            f2_unpack(v[i], x0, x1);
            if (!((on[i >> 4] >> (2 * i & 31)) & 1u)) x0 = -INFINITY;
            if (!((on[i >> 4] >> ((2 * i + 1) & 31)) & 1u)) x1 = -INFINITY;
            v[i] = f2_pack(x0, x1);
          }
        }
        float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 64; ++i) {
          float x0, x1;
          f2_unpack(v[i], x0, x1);
          tops[i & 3] = fmaxf(fmaxf(tops[i & 3], x0), x1);
        }
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * sl;
        // the first finite maximum is taken over as it is (O is zero, or about to be overwritten), a later one if it is much larger
        const bool grown = ms != -INFINITY && top > ms + 8.f;
        if (__any_sync(0xffffffffu, grown)) {
          const float keep = grown ? exp2_fast(ms - top) : 1.f;
          l *= keep;
#pragma unroll 1
          for (int i = 0; i < D; i += 16) {
            float o[16];
            tmem_ld16(to + i, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= keep;
            tmem_st16(to + i, o);
          }
          tmem_wait_st();
        }
        if (ms == -INFINITY || grown) ms = fmaxf(ms, top);
        const float neg = -finite_max(ms);
        const uint64_t sl2 = f2_pack(sl, sl), neg2 = f2_pack(neg, neg);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int h = 0; h < 4; ++h) {                          // 32 keys; the products may begin with the first 64
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float p0, p1;
            f2_unpack(f2_fma(v[h * 16 + i], sl2, neg2), p0, p1);
            p0 = exp2_fast(p0);
            p1 = exp2_fast(p1);
            sum[i & 1] = f2_add(sum[i & 1], f2_pack(p0, p1));
            p[i] = bf16_pair(p0, p1);
          }
          tmem_st16(ts + h * 16, *reinterpret_cast<float (*)[16]>(p));
          if (h & 1) {
            tmem_wait_st();
            tc_fence_before_sync();
            mbar_arrive_warp(P_READY(c * 2 + (h >> 1)));
          }
        }
        float s0, s1;
        f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      if (!ok) break;
      if (x.tiles > 0) {
        if (!mbar_wait(O_FULL(c), n_item & 1, wc)) { ok = false; break; }
        ++n_item;
        tc_fence_after_sync();
      }
      const long long token = (long long)x.b * a.Lq + tok;
      const int head = x.hk * a.group + head_in;
      const long long at = token * a.H + head;
      const float r = a.parts > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
      for (int i = 0; i < G::CHUNKS; ++i) {
        float o[64];
        if (x.tiles > 0) {
          tmem_ld32(to + i * 64, *reinterpret_cast<float (*)[32]>(o));
          tmem_ld32(to + i * 64 + 32, *reinterpret_cast<float (*)[32]>(o + 32));
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 64; ++e) o[e] = 0.f;
        }
        if (a.parts > 1) {
          if (row_on) {
            float* dst = a.part_o + (at * a.parts + x.part) * D + i * 64;
#pragma unroll
            for (int e = 0; e < 64; e += 4) store4(dst + e, make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]));
          }
        } else {
          tma_store_wait_read<0>();                            // (only lane 0 has any) the store that last read this buffer
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(out_row + ((e ^ (lane & 7)) * 16)) =
                make_uint4(bf16_pair(o[8 * e] * r, o[8 * e + 1] * r), bf16_pair(o[8 * e + 2] * r, o[8 * e + 3] * r),
                           bf16_pair(o[8 * e + 4] * r, o[8 * e + 5] * r), bf16_pair(o[8 * e + 6] * r, o[8 * e + 7] * r));
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (tok0 < a.Lq) tma_store_5d(&tmOut, out_smem, i * 64, head0, x.hk, tok0, x.b);
            tma_store_commit();
          }
        }
      }
      if (x.tiles > 0) {
        tc_fence_before_sync();
        mbar_arrive_warp(O_EMPTY(c));
      }
      if (row_on) {
        if (a.parts > 1) a.part_ml[at * a.parts + x.part] = make_float2(ms, l);
        else if (a.lse) a.lse[at] = lse_of(ms, l);
      }
    }
    tma_store_wait_all<0>();
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, G::COLS);
  }
}

}  // namespace vdn
