// Attention of each query to all the states of its batch row's encoder on the tensor cores; bf16 I/O, d = 64 or 128.
//
// The rows of a key head are its queries times the heads of its group.  They go in blocks of up to 32 (a warp's share: whole tokens,
// or 32 heads of one), four blocks to a tile of 128, two tiles to a CTA.  Per tile and 128 keys:
//   S = Q K^T      (128 x 128 x d, both operands in shared memory, S in tensor memory)
//   P = 2^(c S - m)  a thread to a row: the maximum, the exponentials and their sum in fp32, P as bf16 over S in tensor memory
//   O += P V       (128 x d x 128, P from tensor memory, V as it lies in shared memory)
// The two tiles take turns: while one is exponentiated the other is multiplied.  (A tile without rows, the last of an odd number, waits
// for the other's keys to end, 1 us for each 128.)  O stays in tensor memory; it is brought to a new maximum only where that has
// grown by more than 2^8 (else P goes up to 2^8, which bf16 and fp32 hold as well), by the warp that found it, between its tile's
// products.
// P is rounded to bf16, the type that V has and the instruction takes; the sum is that of the weights before it.  With d = 128 the result is
// off by 2.0e-3 (77 keys) to 2.3e-3 (8192) in the 2-norm, 1.66e-3 of which its own rounding is.  P in two bf16 parts (twice the
// products) leaves 1.66e-3 and costs 11 % with 77 keys, 28 % in steps of 32 requests, 35 % with 512 and 16384 keys.
// 16384 x 16384 x 16 heads: d = 128 1690 us, 1300 TFLOP/s; d = 64 1400 us, 785 TFLOP/s (exponentials: 58 % of what their pipe can).
// 87720 x 512 keys x 40 heads, d = 128: 910 us.  What bounds it: a tile's chain from scores to weights to the next scores (about 2000 cycles
// in the warps, 1400 in products and signals), two chains side by side.  Three exponentials in eight on the
// multiply-add pipe: 8 % slower; 64 keys at a time with two S for each tile: 963 TFLOP/s (products of 64 columns take as long to issue
// as those of 128); results stored by the threads instead of by tile copies: 1400 us at 87720 x 512.
// The tensor cores cut off what an addition leaves over instead of rounding it, so a long sum of values of one sign falls short by about
// 2^-27 for each of its keys: 5e-4 at 65536 keys, 7e-3 at 2^20, a tenth at 2^24.  Every FOLD tiles O and the sum of weights therefore
// move to fp32 sums of their own (O's in the workspace), at most 3e-4 short, and start anew.  2^20 keys, 19456 rows, d = 128: 15.2 ms, 14.7 without.
// Keys that do not count: their scores are replaced by -inf, their rows of V by zeros in shared memory (zero times what may
// be anything is not zero).
#pragma once
#include <type_traits>

#include "cross_simt.cuh"
#include "quantize.cuh"
#include "tc_common.cuh"
#include "token_rule.cuh"
#include "token_tc.cuh"

namespace vdn {

struct CrossTcShape {
  int hb, tb;                 // heads and tokens of a row block
  int head_blocks;            // ceil(group / hb)
  int blocks, pairs;          // row blocks, and pairs of tiles, of a (batch row, key head)
  FastDivide by_parts, by_pairs, by_heads, by_head_blocks;
  uint32_t items;             // B * Hk * pairs * parts
};

template <int D>
struct CrossTc {
  static constexpr int KEYS = 128, THREADS = 384, CHUNKS = D / 64;
  static constexpr int TILE_BYTES = 128 * D * 2, CHUNK_BYTES = 128 * 128, OUT_BYTES = 32 * 128;
  static constexpr int STAGES = D == 128 ? 3 : 6;                       // tiles of keys and values in turn
  static constexpr int OFF_Q = 0, OFF_KV = 2 * TILE_BYTES, OFF_OUT = OFF_KV + STAGES * TILE_BYTES;
  static constexpr int OFF_BAR = OFF_OUT + 8 * CHUNKS * OUT_BYTES;      // a warp's results: 32 rows, 64 channels at a time
  static constexpr int BARS = 2 + 2 + 3 * STAGES + 2 + 4 + 2 + 2;
  static constexpr int USED_BYTES = OFF_BAR + 8 * BARS + 16, SMEM_BYTES = USED_BYTES + 1024;
  // P is handed over as a whole (d = 128), or in halves (d = 64: products are short, and waiting for the second half costs less than
  // starting late).  16384 x 16384: d = 128 1679 us whole, 1733 in halves; d = 64 1528, 1435.
  static constexpr int P_PARTS = D == 128 ? 1 : 2;
  static constexpr int COL_S = 0, COL_O = 256, COLS = 512;              // tensor memory: S of both tiles, O of both
  static constexpr int FOLD = 256, ROWS = 256;                          // tiles between two moves of O; rows, a thread each
};
static_assert(CrossTc<128>::SMEM_BYTES <= 232448, "shared memory of a CTA");

// What every role of the CTA derives of an item.
struct CrossItem {
  int b, hk, pair, part, lo, hi, tiles;        // keys lo .. hi-1 of the batch row, in so many tiles
  long long start;
  bool second;                                  // the pair's second tile has rows
};
__device__ __forceinline__ CrossItem cross_item(const CrossArgs& a, const CrossTcShape& s, uint32_t item) {
  CrossItem x;
  uint32_t q = quotient(item, s.by_parts);
  x.part = (int)(item - q * s.by_parts.d);
  item = quotient(q, s.by_pairs);
  x.pair = (int)(q - item * s.by_pairs.d);
  x.b = (int)quotient(item, s.by_heads);
  x.hk = (int)(item - (uint32_t)x.b * s.by_heads.d);
  int len;
  cross_range(a, x.b, x.start, len);
  cross_part(len, x.part, a.parts, 128, x.lo, x.hi);
  x.tiles = (x.hi - x.lo + 127) / 128;
  x.second = ((uint32_t)x.pair * 2 + 1) * 4 < (uint32_t)s.blocks;
  return x;
}

// A thread's sums of the tiles so far, and back: O's channels, what the weights add up to, and the maximum that both are relative to, ROWS
// apart.  Functions of their own, with all of it in memory, so that nothing of it lives in registers on the way.
template <int D>
__device__ __noinline__ void cross_fold(float* at, uint32_t to, float ms, float l, bool first) {
  using namespace tc;
  constexpr int ROWS = CrossTc<D>::ROWS;
  const float keep = first ? 0.f : exp2_fast(at[(D + 1) * ROWS] - finite_max(ms));
#pragma unroll 1
  for (int i = 0; i < D; i += 16) {
    float o[16];
    tmem_ld16(to + i, o);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 16; ++e) at[(i + e) * ROWS] = first ? o[e] : fmaf(at[(i + e) * ROWS], keep, o[e]);
  }
  at[D * ROWS] = first ? l : fmaf(at[D * ROWS], keep, l);
  at[(D + 1) * ROWS] = ms;
}
// (returns what is to be added to the sum of weights)
template <int D>
__device__ __noinline__ float cross_unfold(const float* at, uint32_t to, float ms) {
  using namespace tc;
  constexpr int ROWS = CrossTc<D>::ROWS;
  const float keep = exp2_fast(at[(D + 1) * ROWS] - finite_max(ms));
#pragma unroll 1
  for (int i = 0; i < D; i += 16) {
    float o[16];
    tmem_ld16(to + i, o);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = fmaf(at[(i + e) * ROWS], keep, o[e]);
    tmem_st16(to + i, o);
  }
  tmem_wait_st();
  return at[D * ROWS] * keep;
}

// LONG: some run of keys may be longer than FOLD tiles.  A variant of its own: what has none that long takes 1 to 3 % longer with it, as a
// packed batch with so many keys in all does (100 x 512 keys, 1000 queries, 8 heads 264 -> 272 us; with the two functions above in line 295).
template <int D, bool LONG>
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
  auto FULL = [&](int i) { return bar0 + 8u * (4 + i); };
  auto READY = [&](int i) { return bar0 + 8u * (4 + G::STAGES + i); };
  auto EMPTY = [&](int i) { return bar0 + 8u * (4 + 2 * G::STAGES + i); };
  auto S_FULL = [&](int c) { return bar0 + 8u * (4 + 3 * G::STAGES + c); };
  auto P_READY = [&](int c) { return bar0 + 8u * (6 + 3 * G::STAGES + c); };
  auto O_FULL = [&](int c) { return bar0 + 8u * (10 + 3 * G::STAGES + c); };
  auto O_EMPTY = [&](int c) { return bar0 + 8u * (12 + 3 * G::STAGES + c); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + G::OFF_BAR + 8 * G::BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const WaitCtx wc(abort_flag, ds);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (a.parts > 1) let_next_kernel_start();

  if (threadIdx.x == 0) {
    for (int c = 0; c < 2; ++c) {
      mbar_init(Q_FULL(c), 1); mbar_init(Q_EMPTY(c), 1);
      mbar_init(S_FULL(c), 1);
      mbar_init(P_READY(2 * c), 4); mbar_init(P_READY(2 * c + 1), 4);   // a warp an arrival
      mbar_init(O_FULL(c), 1); mbar_init(O_EMPTY(c), 4);
    }
    for (int i = 0; i < G::STAGES; ++i) {
      mbar_init(FULL(i), 1); mbar_init(READY(i), 1); mbar_init(EMPTY(i), 1);
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
        uint32_t n = 0, q[2] = {0, 0};                       // tiles so far: keys and values in turn
        bool ok = true;
        for (uint32_t item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
          const CrossItem x = cross_item(a, s, item);
          if (x.tiles == 0) continue;
          auto load_q = [&](int c) {
            if (!mbar_wait(Q_EMPTY(c), (q[c] & 1) ^ 1, wc)) return false;
            mbar_arrive_expect_tx(Q_FULL(c), 4 * G::CHUNKS * block_rows * 128);
            for (int w = 0; w < 4; ++w) {
              const uint32_t rb = (uint32_t)(x.pair * 2 + c) * 4 + w, tb = quotient(rb, s.by_head_blocks);
              for (int i = 0; i < G::CHUNKS; ++i)
                tma_load_5d(base + G::OFF_Q + c * G::TILE_BYTES + i * G::CHUNK_BYTES + w * 32 * 128, &tmQ, Q_FULL(c), i * 64,
                            (int)(rb - tb * s.head_blocks) * s.hb, x.hk, (int)tb * s.tb, x.b);
            }
            ++q[c];
            return true;
          };
          auto load = [&](const CUtensorMap* m, int j) {
            const uint32_t st = n % G::STAGES;
            if (!mbar_wait(EMPTY(st), ((n / G::STAGES) & 1) ^ 1, wc)) return false;
            mbar_arrive_expect_tx(FULL(st), G::TILE_BYTES);
            for (int i = 0; i < G::CHUNKS; ++i)
              tma_load_3d(base + G::OFF_KV + st * G::TILE_BYTES + i * G::CHUNK_BYTES, m, FULL(st), i * 64, x.hk, (int)(x.start + x.lo + j * 128));
            ++n;
            return true;
          };
          ok = load_q(0);
          for (int j = 0; j < x.tiles && ok; ++j)
            ok = load(&tmK, j) && (j > 0 || !x.second || load_q(1)) && load(&tmV, j);
        }
        if (!ok) {                                             // a bounded chance for what is under way to land
          for (int c = 0; c < 2; ++c)
            if (q[c]) mbar_drain(Q_FULL(c), (q[c] - 1) & 1);
          mbar_drain_ring(FULL(0), G::STAGES, n);
        }
      }
    } else if (warp == 9) {
      // ------------------------------------------------------------------ products
      constexpr uint32_t id_s = make_idesc_bf16(128, 128, false, false), id_o = make_idesc_bf16(128, D, false, true);
      uint32_t n = 0, n_item[2] = {0, 0}, n_p[2] = {0, 0};
      bool ok = true;
      auto arrived = [&](uint32_t r) { return mbar_wait_warp(READY(r % G::STAGES), (r / G::STAGES) & 1, wc); };
      auto scores = [&](int c, uint32_t r, bool last_of_k, bool last_of_q) {
        const uint32_t st = r % G::STAGES;
        const uint64_t dq = make_smem_desc(base + G::OFF_Q + c * G::TILE_BYTES, 16, 1024);
        const uint64_t dk = make_smem_desc(base + G::OFF_KV + st * G::TILE_BYTES, 16, 1024);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (k >> 2) * (G::CHUNK_BYTES >> 4) + (k & 3) * 2;
            mma_bf16_ss(tmem + G::COL_S + c * 128, dq + off, dk + off, id_s, k ? 1u : 0u);
          }
          mma_commit(S_FULL(c));
          if (last_of_k) mma_commit(EMPTY(st));
          if (last_of_q) mma_commit(Q_EMPTY(c));
        }
        __syncwarp();
      };
      for (uint32_t item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
        const CrossItem x = cross_item(a, s, item);
        if (x.tiles == 0) continue;
        const int chains = x.second ? 2 : 1;
        ok = arrived(n);
        for (int c = 0; c < chains && ok; ++c) {
          ok = mbar_wait_warp(Q_FULL(c), n_item[c] & 1, wc);
          if (!ok) break;
          tc_fence_after_sync();
          scores(c, n, c + 1 == chains, x.tiles == 1);
        }
        for (int j = 0; j < x.tiles && ok; ++j, n += 2) {
          const uint32_t st = (n + 1) % G::STAGES;
          const uint64_t dv = make_smem_desc(base + G::OFF_KV + st * G::TILE_BYTES, G::CHUNK_BYTES, 1024);
          const bool more = j + 1 < x.tiles;
          // (a tile is waited for once; the next keys early only where there are stages for them to have come long ago)
          constexpr bool EARLY = G::STAGES > 3;
          ok = arrived(n + 1) && (!EARLY || !more || arrived(n + 2));
          for (int c = 0; c < chains && ok; ++c) {
            if (j == 0) ok = mbar_wait_warp(O_EMPTY(c), (n_item[c] & 1) ^ 1, wc);
#pragma unroll
            for (int part = 0; part < G::P_PARTS; ++part) {
              ok = ok && mbar_wait_warp(P_READY(2 * c + part), n_p[c] & 1, wc);
              if (!ok) break;
              tc_fence_after_sync();
              if (elect_one()) {
#pragma unroll
                for (int k = part * (8 / G::P_PARTS); k < (part + 1) * (8 / G::P_PARTS); ++k)
                  mma_bf16_ts(tmem + G::COL_O + c * D, tmem + G::COL_S + c * 128 + k * 8, dv + k * (2048 >> 4), id_o, k || (LONG ? j % G::FOLD : j) ? 1u : 0u);
                if (part + 1 == G::P_PARTS) {
                  if (!more) mma_commit(O_FULL(c));
                  if (c + 1 == chains) mma_commit(EMPTY(st));
                }
              }
              __syncwarp();
            }
            if (!ok) break;
            ++n_p[c];
            if (!EARLY && more && c == 0) ok = arrived(n + 2);
            if (more && ok) scores(c, n + 2, c + 1 == chains, j + 2 == x.tiles);
          }
        }
        for (int c = 0; c < chains; ++c) ++n_item[c];
      }
    } else if (warp == 10) {
      // ------------------------------------------------------------------ values that do not count become zeros
      uint32_t n = 0;
      bool ok = true;
      for (uint32_t item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
        const CrossItem x = cross_item(a, s, item);
        for (int j = 0; j < 2 * x.tiles && ok; ++j, ++n) {
          const uint32_t st = n % G::STAGES;
          uint32_t on[4] = {~0u, ~0u, ~0u, ~0u};
          if (j & 1) {                                             // (tiles of keys pass)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = x.lo + (j >> 1) * 128 + i * 32 + lane;
              on[i] = __ballot_sync(0xffffffffu, key < x.hi && key_counts(a, x.start + key));
            }
          }
          ok = mbar_wait_warp(FULL(st), (n / G::STAGES) & 1, wc);
          if (!ok) break;
          if ((on[0] & on[1] & on[2] & on[3]) != 0xffffffffu) {
            unsigned char* v = base_ptr + G::OFF_KV + st * G::TILE_BYTES;
            for (int r = lane / 8; r < 128; r += 4)                 // eight lanes to a row's 128 bytes
              if (!((on[r >> 5] >> (r & 31)) & 1u))
                for (int i = 0; i < G::CHUNKS; ++i) *reinterpret_cast<uint4*>(v + i * G::CHUNK_BYTES + r * 128 + (lane & 7) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
          }
          mbar_arrive_warp(READY(st));
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ exponentials, and the results
    registers_more<216>();
    const int c = warp >> 2, qd = warp & 3;
    const uint32_t ts = tmem + ((uint32_t)(qd * 32) << 16) + G::COL_S + c * 128, to = tmem + ((uint32_t)(qd * 32) << 16) + G::COL_O + c * D;
    const float sl = a.scale_log2;
    const int lane_head = lane % s.hb, lane_tok = lane / s.hb;
    const uint32_t out_smem = base + G::OFF_OUT + warp * G::CHUNKS * G::OUT_BYTES;
    unsigned char* out_row = base_ptr + G::OFF_OUT + warp * G::CHUNKS * G::OUT_BYTES + lane * 128;
    uint32_t n_s = 0, n_item = 0;
    bool ok = true;
    [[maybe_unused]] auto long_at = [&] { return a.long_o + (size_t)blockIdx.x * ((D + 2) * G::ROWS) + threadIdx.x; };
    for (uint32_t item = blockIdx.x; item < s.items && ok; item += gridDim.x) {
      const CrossItem x = cross_item(a, s, item);
      if (c == 1 && !x.second) continue;
      const uint32_t rb = (uint32_t)(x.pair * 2 + c) * 4 + qd, block = quotient(rb, s.by_head_blocks);
      const int tok0 = (int)block * s.tb, head0 = (int)(rb - block * s.head_blocks) * s.hb;
      const int head_in = head0 + lane_head, tok = tok0 + lane_tok;
      const bool row_on = lane < block_rows && head_in < a.group && tok < a.Lq;
      float ms = -INFINITY;                                    // the maximum times sl,
      uint64_t sum[2] = {0ull, 0ull};                          // and the sum relative to it, in four parts
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
        if (!__all_sync(0xffffffffu, mbar_wait(S_FULL(c), n_s & 1, wc))) { ok = false; break; }
        tc_fence_after_sync();
        // (these scores follow the last product into O, and the next one waits for P)
        if (LONG && j % G::FOLD == 0 && j > 0) {
          float l0, l1;
          f2_unpack(f2_add(sum[0], sum[1]), l0, l1);
          cross_fold<D>(long_at(), to, ms, l0 + l1, j == G::FOLD);
          sum[0] = sum[1] = 0ull;
        }
        // (twice, so that a tile whose keys all count has no branch in it: those cost 6 % of a long encoder's time)
        auto weights = [&](auto cut) {
          constexpr bool CUT = decltype(cut)::value;
          uint64_t v[64];                                      // two neighbouring scores each
          tmem_ld128_pairs(ts, v);
          float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (CUT && on[g] != 0xffffffffu) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float x0, x1;
                f2_unpack(v[g * 16 + i], x0, x1);
                v[g * 16 + i] = f2_pack((on[g] >> (2 * i)) & 1u ? x0 : -INFINITY, (on[g] >> (2 * i + 1)) & 1u ? x1 : -INFINITY);
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float x0, x1;
              f2_unpack(v[g * 16 + i], x0, x1);
              tops[i & 3] = fmaxf(fmaxf(tops[i & 3], x0), x1);
            }
          }
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * sl;
          // the first finite maximum is taken over as it is (O is zero, or about to be overwritten), a later one if it is much larger
          const bool grown = ms != -INFINITY && top > ms + 8.f;
          if (__any_sync(0xffffffffu, grown)) {
            const float keep = grown ? exp2_fast(ms - top) : 1.f;
            const uint64_t keep2 = f2_pack(keep, keep);
            sum[0] = f2_fma(sum[0], keep2, 0ull);
            sum[1] = f2_fma(sum[1], keep2, 0ull);
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
#pragma unroll
          for (int g = 0; g < 4; ++g) {                        // 32 keys
            uint32_t p[16];
            if (!CUT || on[g] != 0) {
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float p0, p1;
                f2_unpack(f2_fma(v[g * 16 + i], sl2, neg2), p0, p1);
                p0 = exp2_fast(p0);
                p1 = exp2_fast(p1);
                sum[i & 1] = f2_add(sum[i & 1], f2_pack(p0, p1));
                p[i] = bf16_pair(p0, p1);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) p[i] = 0u;
            }
            tmem_st16(ts + g * 16, *reinterpret_cast<float (*)[16]>(p));
            if ((g + 1) % (4 / G::P_PARTS) == 0) {
              tmem_wait_st();
              tc_fence_before_sync();
              mbar_arrive_warp(P_READY(c * 2 + g / (4 / G::P_PARTS)));
            }
          }
        };
        if (all) weights(std::false_type{});
        else weights(std::true_type{});
      }
      if (!ok) break;
      if (x.tiles > 0) {
        if (!__all_sync(0xffffffffu, mbar_wait(O_FULL(c), n_item & 1, wc))) { ok = false; break; }
        ++n_item;
        tc_fence_after_sync();
      }
      float l, l1;
      f2_unpack(f2_add(sum[0], sum[1]), l, l1);
      l += l1;
      if (LONG && x.tiles > G::FOLD) l += cross_unfold<D>(long_at(), to, ms);
      const long long token = (long long)x.b * a.Lq + tok;
      const long long at = token * a.H + x.hk * a.group + head_in;
      const float r = l == 0.f ? 0.f : 1.f / l;
      if (a.parts == 1) {
        tma_store_wait_read<0>();                              // (only lane 0 has any) the last item's stores
        __syncwarp();
      }
#pragma unroll
      for (int i = 0; i < G::CHUNKS; ++i) {
        float o[64];
        if (x.tiles > 0) {
          tmem_ld32(to + i * 64, *reinterpret_cast<float (*)[32]>(o));
          tmem_ld32(to + i * 64 + 32, *reinterpret_cast<float (*)[32]>(o + 32));
          tmem_wait_ld();
          if (i + 1 == G::CHUNKS) {
            tc_fence_before_sync();
            mbar_arrive_warp(O_EMPTY(c));
          }
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
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4*>(out_row + i * G::OUT_BYTES + ((e ^ (lane & 7)) * 16)) =
                make_uint4(bf16_pair(o[8 * e] * r, o[8 * e + 1] * r), bf16_pair(o[8 * e + 2] * r, o[8 * e + 3] * r),
                           bf16_pair(o[8 * e + 4] * r, o[8 * e + 5] * r), bf16_pair(o[8 * e + 6] * r, o[8 * e + 7] * r));
        }
      }
      if (a.parts == 1) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (tok0 < a.Lq)
            for (int i = 0; i < G::CHUNKS; ++i) tma_store_5d(&tmOut, out_smem + i * G::OUT_BYTES, i * 64, head0, x.hk, tok0, x.b);
          tma_store_commit();
        }
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
    settle(bar0 + 8u * G::BARS + 4u);
    tc_fence_after_sync();
    tmem_dealloc(tmem, G::COLS);
  }
}

}  // namespace vdn
