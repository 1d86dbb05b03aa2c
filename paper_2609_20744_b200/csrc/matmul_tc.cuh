// Block-scaled 8-bit product on the tensor cores.
//   out[m, n] = sum_b sa[m, b] sw[n / 128, b] sum_{k in block b} a[m, k] w[n, k]  + bias[n] + add[m, n]
// The scales are any fp32 numbers, so a block's sum (128 channels: four instructions of 32) leaves tensor memory, is multiplied by
// its scale and added to the others in fp32 registers, while the next block's sum is formed in another accumulator.
#pragma once
#include "matmul_simt.cuh"
#include "tc_common.cuh"
#include "token_rule.cuh"

namespace vdn {

// ---------------------------------------------------------------------------------------------- large
// 256 x 256 outputs to a pair of CTAs (128 rows in either's tensor memory), persistent.  Per block of channels a CTA fetches 128 rows of
// a and 128 of w (32 KB); one CTA alone would need 48 KB for as much work, more than L2 gives 148 SMs at the tensor
// cores' rate.  Warps 0-7 take the block sums out, a thread a row and 128 of the 256 columns, and write the tile;
// warp 8 issues the copies, warp 9 (of the even CTA) the products.  Registers: 384 threads start with 168 each; the four warps that
// copy and issue keep 40, the eight others get 232 (128 of them sums): 256 * 232 + 128 * 40 = 384 * 168.
// 32768 x 5120 x 5120: 746 us, 2300 TFLOP/s.  What bounds it: an accumulator's round trip (products, signal, read, signal back)
// with two of them.  In copies of this kernel one accumulator over all channels took 591 us, the round trip without the
// multiply-adds 671.  Columns in two halves with four accumulators: 1014 us (the products of 128 columns wait for shared memory);
// sixteen warps of 64 columns: 877.
struct MatmulPair {
  static constexpr int ROWS = 128, COLS = 256, STAGES = 5, THREADS = 384;
  static constexpr int A_BYTES = ROWS * 128, STAGE_BYTES = A_BYTES + COLS / 2 * 128;
  static constexpr int OUT_BYTES = 32 * 128;                       // one warp's rows, 128 bytes of each
  static constexpr int OFF_OUT = STAGES * STAGE_BYTES, OFF_BAR = OFF_OUT + 8 * 2 * OUT_BYTES;
  static constexpr int BARS = 2 * STAGES + 4 + 16, USED_BYTES = OFF_BAR + 8 * BARS + 16;
  static constexpr int SMEM_BYTES = USED_BYTES + 1024;
};
static_assert(MatmulPair::SMEM_BYTES <= 232448, "shared memory of a CTA");

__device__ __forceinline__ uint32_t bf16_word(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// bias of columns n .. n+31 (of N).
__device__ __forceinline__ void add_bias(const MatmulArgs& p, int n, float (&x)[32]) {
  if (p.bias) {
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] += n + i < p.N ? __ldg(p.bias + n + i) : 0.f;
  }
}

// An accumulator's sums times `factor(column)`, where they lie: what blocks need whose scales do not make one factor, out of the way of
// those that the rest of the loop is laid out for (the same in its registers: 32768 x 5120 x 5120 3 % slower, 128 rows 18.9 -> 23.1 us).
template <int COLS, typename F>
__device__ __forceinline__ void scale_in_place(uint32_t taddr, F factor) {
#pragma unroll 1
  for (int c = 0; c < COLS; c += 16) {
    float v[16];
    tc::tmem_ld16(taddr + c, v);
    tc::tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= factor(c + i);
    tc::tmem_st16(taddr + c, v);
    tc::tmem_wait_st();
  }
}

// How results leave: by tile copies; by tile copies, `add` coming the same way; or element by element, where one of them has rows that no tile
// copy can reach, or that end inside 16 bytes.  Variants of their own: in common code the first takes 6 % longer with the second's (753 -> 800 us at
// 32768 x 5120 x 5120), and spills with the third's.
enum MatmulOut { kOutTiles, kOutTilesAdd, kOutElements };
template <typename Tio, int MODE>
__global__ void __launch_bounds__(MatmulPair::THREADS, 1) __cluster_dims__(2, 1, 1)
matmul_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                   const __grid_constant__ CUtensorMap tmOut, const __grid_constant__ CUtensorMap tmAdd, const MatmulArgs p,
                   tc::DevStatus ds) {
  using namespace tc;
  using G = MatmulPair;
  constexpr bool ADD = MODE == kOutTilesAdd;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + G::OFF_BAR;
  auto FULL = [&](int i) { return bar0 + 8u * i; };
  auto EMPTY = [&](int i) { return bar0 + 8u * (G::STAGES + i); };
  auto ACCFULL = [&](int i) { return bar0 + 8u * (2 * G::STAGES + i); };
  auto ACCEMPTY = [&](int i) { return bar0 + 8u * (2 * G::STAGES + 2 + i); };
  auto ADDED = [&](int i) { return bar0 + 8u * (2 * G::STAGES + 4 + i); };       // 16: a warp's two staging tiles
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + G::OFF_BAR + 8 * G::BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const WaitCtx wc(abort_flag, ds);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();

  if (threadIdx.x == 0) {
    for (int i = 0; i < G::STAGES; ++i) { mbar_init(FULL(i), 1); mbar_init(EMPTY(i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(ACCFULL(i), 1); mbar_init(ACCEMPTY(i), 16); }   // a warp an arrival, of both CTAs
    for (int i = 0; i < 16; ++i) mbar_init(ADDED(i), 1);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmW);
  }
  if (warp == 9) {
    tmem_alloc_pair(smem_u32(tmem_slot), 512);
    tmem_relinquish_pair();
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  const int tiles_n = (p.N + G::COLS - 1) / G::COLS;
  const long long tiles = (p.M + 2 * G::ROWS - 1) / (2 * G::ROWS) * tiles_n;
  const long long first = blockIdx.x / 2, step = gridDim.x / 2;

  if (warp >= 8) {
    registers_fewer<40>();
    if (warp == 8) {
      if (lane == 0) {
        uint32_t it = 0;
        bool ok = true;
        for (long long t = first; t < tiles && ok; t += step) {
          const int m0 = (int)(t / tiles_n) * 2 * G::ROWS + (int)rank * G::ROWS;
          const int n0 = (int)(t % tiles_n) * G::COLS + (int)rank * (G::COLS / 2);
          for (int b = 0; b < p.blocks; ++b, ++it) {
            const int st = it % G::STAGES;
            if (!mbar_wait(EMPTY(st), ((it / G::STAGES) & 1) ^ 1, wc)) { ok = false; break; }
            if (rank == 0) mbar_arrive_expect_tx(FULL(st), 2 * G::STAGE_BYTES);
            const uint32_t dst = base + st * G::STAGE_BYTES, bar = rank_address(FULL(st), 0);
            tma_load_2d_pair(dst, &tmA, bar, b * kScaleBlock, m0);
            tma_load_2d_pair(dst + G::A_BYTES, &tmW, bar, b * kScaleBlock, n0);
          }
        }
        // (the even CTA's barriers count the copies of both)
        if (!ok && rank == 0) mbar_drain_ring(FULL(0), G::STAGES, it);
      }
    } else if (warp == 9 && rank == 0) {
      constexpr uint32_t idesc = make_idesc_e4m3(2 * G::ROWS, G::COLS);
      uint32_t it = 0;
      bool ok = true;
      for (long long t = first; t < tiles && ok; t += step) {
        for (int b = 0; b < p.blocks; ++b, ++it) {
          const int st = it % G::STAGES, a = it & 1;
          ok = mbar_wait_warp(ACCEMPTY(a), ((it >> 1) & 1) ^ 1, wc) && mbar_wait_warp(FULL(st), (it / G::STAGES) & 1, wc);
          if (!ok) break;
          tc_fence_after_sync();
          const uint64_t da = make_smem_desc(base + st * G::STAGE_BYTES, 16, 1024);
          const uint64_t dw = make_smem_desc(base + st * G::STAGE_BYTES + G::A_BYTES, 16, 1024);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_e4m3_pair(tmem + a * G::COLS, da + k * 2, dw + k * 2, idesc, k ? 1u : 0u);
            mma_commit_pair(EMPTY(st));
            mma_commit_pair(ACCFULL(a));
          }
          __syncwarp();
        }
      }
    }
  } else {
    registers_more<232>();
    const int qd = warp & 3, half = warp >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(qd * 32) << 16) + half * 128;
    const uint32_t out_smem = base + G::OFF_OUT + warp * 2 * G::OUT_BYTES;
    unsigned char* out_ptr = base_ptr + G::OFF_OUT + warp * 2 * G::OUT_BYTES;
    constexpr int PER = 128 / (int)sizeof(Tio), SLICES = 128 / PER;
    // Whether this lane's waits for sums have all ended in time.  No lane acts on that by itself: the vote on the next block's scales carries
    // it, and until then sums that are not there are added like others.  (A vote of its own at the wait: 1 % longer; one for both there: 1 to
    // 3 %, 10 % where results and add leave element by element.)
    bool in_time = true;
    uint32_t it = 0, phase = 0;                          // phase: of the two staging tiles' barriers, a bit each
    bool ok = true;
    for (long long t = first; t < tiles && ok; t += step) {
      const long long m = (t / tiles_n) * 2 * G::ROWS + rank * G::ROWS + qd * 32 + lane;
      const int n0 = (int)(t % tiles_n) * G::COLS + half * 128;
      const bool inside = m < p.M && n0 < p.N;
      const float* sa = p.a_scale + (inside ? m * p.blocks : 0);
      const float* sw = p.w_scale + (inside ? (long long)(n0 / kScaleBlock) * p.blocks : 0);
      // What is to be added comes into the staging tiles the results will leave from, the first two slices while the sums are formed.
      const bool here = m - lane < p.M;
      auto fetch = [&](int c) {
        const int n = n0 + c * PER, bar = warp * 2 + (c & 1);
        if (!ADD || !here || n >= p.N || lane != 0) return;
        mbar_arrive_expect_tx(ADDED(bar), G::OUT_BYTES);
        tma_load_2d(out_smem + (c & 1) * G::OUT_BYTES, &tmAdd, ADDED(bar), n, (int)m);
      };
      if constexpr (ADD) {
        tma_store_wait_read<0>();                        // (only lane 0 has any) the last tile's stores have read them
        __syncwarp();
        fetch(0);
        fetch(1);
      }
      uint64_t acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0ull;
      float s = __ldg(sa) * __ldg(sw), xa = 0.f, xw = 0.f;
      bool odd = __any_sync(0xffffffffu, !normal_number(s));   // anything out of the ordinary
      for (int b = 0; b < p.blocks; ++b, ++it) {
        const int a = it & 1;
        if (b + 1 < p.blocks) { xa = __ldg(sa + b + 1); xw = __ldg(sw + b + 1); }
        in_time = mbar_wait(ACCFULL(a), (it >> 1) & 1, wc) && in_time;
        tc_fence_after_sync();
        if (odd) {
          if (__any_sync(0xffffffffu, !in_time)) break;
          float first;
          s = join_scales(__ldg(sa + b), __ldg(sw + b), first);
          if (__any_sync(0xffffffffu, first != 1.f)) scale_in_place<128>(taddr + a * G::COLS, [&](int) { return first; });
        }
        // The accumulator is free once it has been read: half of it waits in registers (there is no room for all), and only that half
        // is added before the rest has been fetched.
        const uint64_t s2 = f2_pack(s, s);
        uint64_t v[32];
        tmem_ld64_pairs(taddr + a * G::COLS, v);
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] = f2_fma(v[i], s2, acc[i]);
        tmem_ld64_pairs(taddr + a * G::COLS + 64, v);
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(rank_address(ACCEMPTY(a), 0));
        s = xa * xw;                                       // the next block's
        odd = __any_sync(0xffffffffu, !normal_number(s) || !in_time);
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[32 + i] = f2_fma(v[i], s2, acc[32 + i]);
      }
      if (odd) ok = !__any_sync(0xffffffffu, !in_time);
      if (!ok) {
        if (ADD && here)                            // a bounded chance for copies under way to land
          for (int c = 0; c < 2 && n0 + c * PER < p.N; ++c) mbar_drain(ADDED(warp * 2 + c), (phase >> c) & 1);
        break;
      }
      if constexpr (MODE == kOutElements) {
        // results, or what is added to them, that no tile copy can reach (rows at any address): 32 columns at a time in fp32 through
        // shared memory, so that a warp reads and writes neighbouring elements
        const long long mw = m - lane;
        const int rows = (int)max(0LL, min(32LL, p.M - mw));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int n = n0 + c * 32 + lane;
          const int mine = n < p.N ? rows : 0;
          float x[32];
#pragma unroll
          for (int i = 0; i < 16; ++i) f2_unpack(acc[c * 16 + i], x[2 * i], x[2 * i + 1]);
          add_bias(p, n0 + c * 32, x);
          unsigned char* tile = out_ptr + (c & 1) * G::OUT_BYTES;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<float4*>(tile + lane * 128 + ((i ^ (lane & 7)) * 16)) = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
          __syncwarp();                                  // (the other of the two tiles is written next: all have read it by then)
          Tio* q = static_cast<Tio*>(p.out) + mw * p.out_stride + n;
          auto result = [&](int r) { return *reinterpret_cast<const float*>(tile + r * 128 + (((lane >> 2) ^ (r & 7)) * 16) + (lane & 3) * 4); };
          if (p.add) {                                   // (sixteen rows fetched before the first is written: out may be add)
            const Tio* w = static_cast<const Tio*>(p.add) + mw * p.add_stride + n;
#pragma unroll 1
            for (int r0 = 0; r0 < mine; r0 += 16) {
              float z[16];
#pragma unroll
              for (int i = 0; i < 16; ++i, w += p.add_stride) z[i] = r0 + i < mine ? to_float(*w) : 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i, q += p.out_stride)
                if (r0 + i < mine) *q = from_float<Tio>(result(r0 + i) + z[i]);
            }
          } else {
#pragma unroll 8
            for (int r = 0; r < mine; ++r, q += p.out_stride) *q = from_float<Tio>(result(r));
          }
        }
        __syncwarp();
      } else {
        // the tile: this warp's 32 rows, 128 bytes of each at a time through shared memory (16-byte pieces turned by the row, as the
        // copy's swizzle has them), so that whole lines leave
#pragma unroll
        for (int c = 0; c < SLICES; ++c) {
          const uint32_t slot = c & 1;
          if (c >= 2 || !ADD) {
            tma_store_wait_read<1>();                      // the store that last read this buffer
            __syncwarp();
            if (c >= 2) fetch(c);
          }
          const int n = n0 + c * PER;
          const bool by_tile = ADD && here && n < p.N;
          if (by_tile) {
            if (!mbar_wait_warp(ADDED(warp * 2 + slot), (phase >> slot) & 1, wc)) { ok = false; break; }
            phase ^= 1u << slot;
          }
          unsigned char* row = out_ptr + slot * G::OUT_BYTES + lane * 128;
#pragma unroll
          for (int g = 0; g < PER / 32; ++g) {
            float x[32];
#pragma unroll
            for (int i = 0; i < 16; ++i) f2_unpack(acc[(c * PER + g * 32) / 2 + i], x[2 * i], x[2 * i + 1]);
            add_bias(p, n + g * 32, x);
            if constexpr (sizeof(Tio) == 4) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                float4* at = reinterpret_cast<float4*>(row + ((i ^ (lane & 7)) * 16));
                const float4 y = by_tile ? *at : make_float4(0.f, 0.f, 0.f, 0.f);
                *at = make_float4(x[4 * i] + y.x, x[4 * i + 1] + y.y, x[4 * i + 2] + y.z, x[4 * i + 3] + y.w);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint4* at = reinterpret_cast<uint4*>(row + (((g * 4 + i) ^ (lane & 7)) * 16));
                if (by_tile) {
                  const uint4 y = *at;
                  const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    x[8 * i + 2 * e] += __uint_as_float(w[e] << 16);
                    x[8 * i + 2 * e + 1] += __uint_as_float(w[e] & 0xFFFF0000u);
                  }
                }
                *at = make_uint4(bf16_word(x[8 * i], x[8 * i + 1]), bf16_word(x[8 * i + 2], x[8 * i + 3]), bf16_word(x[8 * i + 4], x[8 * i + 5]),
                                 bf16_word(x[8 * i + 6], x[8 * i + 7]));
              }
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (here && n < p.N) tma_store_2d(&tmOut, out_smem + slot * G::OUT_BYTES, n, (int)m);
            tma_store_commit();
          }
        }
      }
    }
    tma_store_wait_all<0>();
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();
  if (warp == 9) {
    settle(bar0 + 8u * G::BARS + 4u);
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem, 512);
  }
  cluster_sync();
}

// ---------------------------------------------------------------------------------------------- few rows
// Few tokens: bound by the weights' bytes.  The weights take the place of A (128 features in the lanes of tensor memory), TOK tokens
// that of B, so that a product's size goes with the tokens; the channels are cut among the CTAs of a cluster, which add their
// sums through each other's shared memory, in the order of their ranks.  Warps 0-3 take the block sums out, a thread a feature; warp 4
// copies, warp 5 issues products.
// 5120 x 5120: one row 9.4 us (the weights alone 4.1 at the copy's rate; the rest is the launch, the first load's and the joining's
// latency), 48 rows 11.5, 128 rows 17.9.
template <int TOK>
struct MatmulSlim {
  static constexpr int THREADS = 192, STAGE_BYTES = 128 * 128 + TOK * 128;
  static constexpr int STAGES = TOK <= 32 ? 5 : TOK <= 64 ? 4 : 3;             // two CTAs to an SM
  static constexpr int OFF_SCALE = STAGES * STAGE_BYTES, OFF_BAR = OFF_SCALE + 3 * TOK * 4;
  static constexpr int USED_BYTES = OFF_BAR + 8 * (2 * STAGES + 4) + 16;
  static constexpr int SMEM_BYTES = USED_BYTES + 1024;
  static constexpr int TMEM_COLS = 2 * TOK < 32 ? 32 : 2 * TOK;
  static_assert(TOK * 128 * 4 <= OFF_SCALE, "the partial sums take the place of the stages");
};

template <typename Tio, int TOK>
__global__ void __launch_bounds__(192, 2)
matmul_slim_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW, const MatmulArgs p, const int parts,
                   const int wide, tc::DevStatus ds) {
  using namespace tc;
  using G = MatmulSlim<TOK>;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t base = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - smem_u32(smem_dyn));
  const uint32_t bar0 = base + G::OFF_BAR;
  auto FULL = [&](int i) { return bar0 + 8u * i; };
  auto EMPTY = [&](int i) { return bar0 + 8u * (G::STAGES + i); };
  auto ACCFULL = [&](int i) { return bar0 + 8u * (2 * G::STAGES + i); };
  auto ACCEMPTY = [&](int i) { return bar0 + 8u * (2 * G::STAGES + 2 + i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + G::OFF_BAR + 8 * (2 * G::STAGES + 4));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const WaitCtx wc(abort_flag, ds);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = (int)cluster_rank();
  const int n0 = (int)(blockIdx.x / parts) * 128;
  const long long m0 = (long long)blockIdx.y * TOK;
  const int b_lo = (int)((long long)p.blocks * part / parts), b_hi = (int)((long long)p.blocks * (part + 1) / parts);

  if (threadIdx.x == 0) {
    for (int i = 0; i < G::STAGES; ++i) { mbar_init(FULL(i), 1); mbar_init(EMPTY(i), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(ACCFULL(i), 1); mbar_init(ACCEMPTY(i), 4); }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmW);
  }
  if (warp == 5) {
    tmem_alloc(smem_u32(tmem_slot), G::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;

  float* sums = reinterpret_cast<float*>(base_ptr);
  if (warp == 4) {
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int b = b_lo; b < b_hi; ++b, ++it) {
        const int st = it % G::STAGES;
        if (!mbar_wait(EMPTY(st), ((it / G::STAGES) & 1) ^ 1, wc)) { ok = false; break; }
        mbar_arrive_expect_tx(FULL(st), G::STAGE_BYTES);
        const uint32_t dst = base + st * G::STAGE_BYTES;
        tma_load_2d(dst, &tmW, FULL(st), b * kScaleBlock, n0);
        tma_load_2d(dst + 128 * 128, &tmA, FULL(st), b * kScaleBlock, (int)m0);
      }
      if (!ok) mbar_drain_ring(FULL(0), G::STAGES, it);
    }
  } else if (warp == 5) {
    constexpr uint32_t idesc = make_idesc_e4m3(128, TOK);
    uint32_t it = 0;
    for (int b = b_lo; b < b_hi; ++b, ++it) {
      const int st = it % G::STAGES, a = it & 1;
      if (!mbar_wait_warp(ACCEMPTY(a), ((it >> 1) & 1) ^ 1, wc) || !mbar_wait_warp(FULL(st), (it / G::STAGES) & 1, wc)) break;
      tc_fence_after_sync();
      const uint64_t dw = make_smem_desc(base + st * G::STAGE_BYTES, 16, 1024);
      const uint64_t da = make_smem_desc(base + st * G::STAGE_BYTES + 128 * 128, 16, 1024);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_e4m3_ss(tmem + a * TOK, dw + k * 2, da + k * 2, idesc, k ? 1u : 0u);
        mma_commit(EMPTY(st));
        mma_commit(ACCFULL(a));
      }
      __syncwarp();
    }
  } else {
    // The factors of a block, one for each token, go through shared memory: a thread brings one token's and reads all.
    const uint32_t taddr = tmem + ((uint32_t)(warp * 32) << 16);
    float* factors = reinterpret_cast<float*>(base_ptr + G::OFF_SCALE);    // [2][TOK]
    float* firsts = factors + 2 * TOK;                                     // [TOK], where a token's are two
    const bool mine = (int)threadIdx.x < TOK && m0 + threadIdx.x < p.M;
    const float* sa = p.a_scale + (mine ? (m0 + threadIdx.x) * p.blocks : 0);
    const float* sw = p.w_scale + (long long)(n0 / kScaleBlock) * p.blocks;
    constexpr int W = TOK < 32 || TOK > 64 ? 16 : 32;                     // columns read at a time (registers)
    float acc[TOK];
#pragma unroll
    for (int i = 0; i < TOK; ++i) acc[i] = 0.f;
    float xa = mine && b_lo < b_hi ? __ldg(sa + b_lo) : 0.f, xw = mine && b_lo < b_hi ? __ldg(sw + b_lo) : 0.f;
    uint32_t it = 0;
    bool ok = true;
    for (int b = b_lo; b < b_hi; ++b, ++it) {
      const int a = it & 1;
      float first;
      const float s = join_scales(xa, xw, first);
      if ((int)threadIdx.x < TOK) factors[a * TOK + threadIdx.x] = s;
      if (mine && b + 1 < b_hi) { xa = __ldg(sa + b + 1); xw = __ldg(sw + b + 1); }
      ok = mbar_wait(ACCFULL(a), (it >> 1) & 1, wc);
      // (one barrier for both pieces of news; which of them it is, a second one tells)
      if (named_barrier_or(1, 128, !ok || first != 1.f)) {
        if ((int)threadIdx.x < TOK) firsts[threadIdx.x] = first;
        if (named_barrier_or(1, 128, !ok)) { ok = false; break; }
        tc_fence_after_sync();
        scale_in_place<TOK>(taddr + a * TOK, [&](int i) { return firsts[i]; });
      }
      tc_fence_after_sync();
#pragma unroll
      for (int c = 0; c < TOK / W; ++c) {
        float v[W];
        if constexpr (W == 16) tmem_ld16(taddr + a * TOK + c * W, v);
        else tmem_ld32(taddr + a * TOK + c * W, v);
        tmem_wait_ld();
        if (c == TOK / W - 1) {
          tc_fence_before_sync();
          mbar_arrive_warp(ACCEMPTY(a));
        }
#pragma unroll
        for (int i = 0; i < W; i += 4) {
          const float4 f = *reinterpret_cast<const float4*>(factors + a * TOK + c * W + i);
          acc[c * W + i] = fmaf(v[i], f.x, acc[c * W + i]);
          acc[c * W + i + 1] = fmaf(v[i + 1], f.y, acc[c * W + i + 1]);
          acc[c * W + i + 2] = fmaf(v[i + 2], f.z, acc[c * W + i + 2]);
          acc[c * W + i + 3] = fmaf(v[i + 3], f.w, acc[c * W + i + 3]);
        }
      }
    }
    // every product has been read, so nothing is on its way into the stages any more (after a wait that ran out something may be:
    // nothing is put there then)
    if (ok) {
#pragma unroll
      for (int i = 0; i < TOK; ++i) sums[i * 128 + threadIdx.x] = acc[i];
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync();
  // A rank's share of the tokens: four neighbouring features of one to a thread, from all ranks.
  const int lo = TOK * part / parts, hi = (int)min((long long)(TOK * (part + 1) / parts), p.M - m0);
#pragma unroll 2
  for (int t = (int)threadIdx.x; t < (hi - lo) * 32; t += G::THREADS) {
    const int i = lo + t / 32, n = n0 + (t % 32) * 4;
    const uint32_t at = base + (uint32_t)(i * 128 + (t % 32) * 4) * 4;
    float4 x[8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r < parts) x[r] = ld_cluster4(rank_address(at, r));
    float y[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
#pragma unroll
    for (int r = 1; r < 8; ++r)
      if (r < parts) { y[0] += x[r].x; y[1] += x[r].y; y[2] += x[r].z; y[3] += x[r].w; }
    Tio* out = static_cast<Tio*>(p.out) + (m0 + i) * p.out_stride + n;
    const Tio* add = static_cast<const Tio*>(p.add) + (m0 + i) * p.add_stride + n;
    if (p.bias) {
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += n + j < p.N ? __ldg(p.bias + n + j) : 0.f;
    }
    if (wide && n + 4 <= p.N) {
      if (p.add) {
        const float4 z = load4(add);
        y[0] += z.x; y[1] += z.y; y[2] += z.z; y[3] += z.w;
      }
      store4(out, make_float4(y[0], y[1], y[2], y[3]));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n + j < p.N) out[j] = from_float<Tio>(y[j] + (p.add ? to_float(add[j]) : 0.f));
    }
  }
  __syncwarp();
  if (warp == 5) {
    settle(bar0 + 8u * (2 * G::STAGES + 4) + 4u);
    tc_fence_after_sync();
    tmem_dealloc(tmem, G::TMEM_COLS);
  }
  cluster_sync();
}

}  // namespace vdn
