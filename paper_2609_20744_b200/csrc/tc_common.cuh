// Blackwell (sm_100a) building blocks used by the tensor-core kernels: mbarriers with bounded waits,
// TMA tile copies, tcgen05 MMA / TMEM access, shared-memory matrix descriptors.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace vdn {
namespace tc {

constexpr int kStatusTimeout = 6;   // mirrors VDN_ERR_TIMEOUT
constexpr int kStatusInternal = 7;  // mirrors VDN_ERR_INTERNAL

// What every tensor-core kernel is handed for error reporting: the handle's host-mapped status word and the
// time any single wait may take before the CTA gives up.
struct DevStatus {
  int* word;
  unsigned long long wait_ns;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ uint64_t global_timer_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}

// ---------------------------------------------------------------------------------------------- mbarrier
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// One arrival for a whole warp: every lane has made its writes visible (its own fences), the warp converges, one
// lane arrives.  An mbarrier arrival is an atomic on shared memory; hundreds of them per phase serialise.
__device__ __forceinline__ void mbar_arrive_warp(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// Every wait in these kernels goes through here.  It gives up after limit_ns of wall time (2 s unless the
// caller of the library chose otherwise), or as soon as another thread of the CTA has given up; it then records
// the timeout in the host-visible status word and raises the CTA-wide abort flag, after which every role leaves
// its loops and the CTA tears down.
struct WaitCtx {
  volatile int* abort_flag;  // shared memory
  int* status;               // host-mapped status word
  unsigned long long limit_ns;
  __device__ WaitCtx(volatile int* f, const DevStatus& ds) : abort_flag(f), status(ds.word), limit_ns(ds.wait_ns) {}
};
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const WaitCtx& w) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 0u) {
      if (*w.abort_flag) return false;
      if (global_timer_ns() - t0 > w.limit_ns) {
        *w.abort_flag = 1;
        atomicExch(w.status, kStatusTimeout);
        return false;
      }
    }
  }
}

// The wait of a whole warp.  mbar_wait answers each lane by itself, and a barrier may complete between one lane's giving up and another's
// look at it; lanes that disagreed and met in an instruction of the whole warp (tensor memory, votes, __syncwarp) would stand there
// for ever.  So a warp that goes on as a whole decides as a whole.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, const WaitCtx& w) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, w));
}

// After a wait gave up: the copy last issued on `bar` completes the phase of parity `parity`; give it a bounded
// chance to land before the CTA retires and its shared memory goes to another CTA.  (Asking for either parity would
// return at once: the phase before the current one always counts as complete.)
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
  for (int spin = 0; spin < 4096 && !mbar_try_wait(bar, parity); ++spin) {}
}
// ... for a ring of `stages` barriers (`first` + 8 * stage) on which `issued` copies went out round-robin, copy j on
// stage j % stages completing that stage's phase j / stages
__device__ __forceinline__ void mbar_drain_ring(uint32_t first, uint32_t stages, uint32_t issued) {
  for (uint32_t st = 0; st < stages && st < issued; ++st) {
    const uint32_t j = ((issued - 1 - st) / stages) * stages + st;      // the last copy issued on this stage
    mbar_drain(first + 8u * st, (j / stages) & 1u);
  }
}

// Between a CTA's last barrier and its end, by the warp that gives the tensor memory back: where a wait ran out, copies, products and their
// signals may still be on their way into this CTA (or, of a pair, into the other), also those of roles that had nothing left to wait
// for.  Milliseconds are more than any of them takes.  `flag` is the abort flag's shared-memory address.
__device__ __forceinline__ void settle(uint32_t flag) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b32 f;\n\t"
      "ld.volatile.shared.b32 f, [%0];\n\t"
      "setp.ne.u32 p, f, 0;\n\t"
      "@p nanosleep.u32 1000000;\n\t@p nanosleep.u32 1000000;\n\t@p nanosleep.u32 1000000;\n\t}"
      ::"r"(flag)
      : "memory");
  __syncwarp();
}

// ---------------------------------------------------------------------------------------------- proxies
__device__ __forceinline__ void fence_proxy_async_smem() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ---------------------------------------------------------------------------------------------- TMA
__device__ __forceinline__ void tma_prefetch_desc(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1,
                                            int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
__device__ __forceinline__ void tma_store_5d(const CUtensorMap* m, uint32_t src, int c0, int c1, int c2, int c3,
                                             int c4) {
  asm volatile("cp.async.bulk.tensor.5d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5, %6}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
               : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void tma_store_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void tma_store_wait_all() {
  asm volatile("cp.async.bulk.wait_group %0;" ::"n"(N) : "memory");
}

// ---------------------------------------------------------------------------------------------- TMEM
__device__ __forceinline__ void tmem_alloc(uint32_t smem_result, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(ncols)
               : "memory");
}
__device__ __forceinline__ void tmem_relinquish() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tc_fence_before_sync() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after_sync() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 32 lanes x 32 consecutive 32-bit columns: thread l of the warp receives row (lane base + l).
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&r)[32]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
        "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]),
        "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]),
        "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr)
      : "memory");
}

__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 lanes x 64 or 128 columns, complete when it returns, two neighbours to a 64-bit register: what packed fp32 arithmetic takes.
// (Packed behind the load, the pairs cost a move each.)
__device__ __forceinline__ void tmem_ld64_pairs(uint32_t taddr, uint64_t (&r)[32]) {
  asm volatile(
      "{\n\t.reg .b32 a<64>;\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "a0, a1, a2, a3, a4, a5, a6, a7, a8, a9, a10, a11, a12, a13, a14, a15, "
      "a16, a17, a18, a19, a20, a21, a22, a23, a24, a25, a26, a27, a28, a29, a30, a31, "
      "a32, a33, a34, a35, a36, a37, a38, a39, a40, a41, a42, a43, a44, a45, a46, a47, "
      "a48, a49, a50, a51, a52, a53, a54, a55, a56, a57, a58, a59, a60, a61, a62, a63}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;\n\t"
      "mov.b64 %0, {a0, a1}; mov.b64 %1, {a2, a3}; mov.b64 %2, {a4, a5}; mov.b64 %3, {a6, a7};\n\t"
      "mov.b64 %4, {a8, a9}; mov.b64 %5, {a10, a11}; mov.b64 %6, {a12, a13}; mov.b64 %7, {a14, a15};\n\t"
      "mov.b64 %8, {a16, a17}; mov.b64 %9, {a18, a19}; mov.b64 %10, {a20, a21}; mov.b64 %11, {a22, a23};\n\t"
      "mov.b64 %12, {a24, a25}; mov.b64 %13, {a26, a27}; mov.b64 %14, {a28, a29}; mov.b64 %15, {a30, a31};\n\t"
      "mov.b64 %16, {a32, a33}; mov.b64 %17, {a34, a35}; mov.b64 %18, {a36, a37}; mov.b64 %19, {a38, a39};\n\t"
      "mov.b64 %20, {a40, a41}; mov.b64 %21, {a42, a43}; mov.b64 %22, {a44, a45}; mov.b64 %23, {a46, a47};\n\t"
      "mov.b64 %24, {a48, a49}; mov.b64 %25, {a50, a51}; mov.b64 %26, {a52, a53}; mov.b64 %27, {a54, a55};\n\t"
      "mov.b64 %28, {a56, a57}; mov.b64 %29, {a58, a59}; mov.b64 %30, {a60, a61}; mov.b64 %31, {a62, a63};\n\t"
      "}"
      : "=l"(r[0]), "=l"(r[1]), "=l"(r[2]), "=l"(r[3]), "=l"(r[4]), "=l"(r[5]), "=l"(r[6]), "=l"(r[7]),
        "=l"(r[8]), "=l"(r[9]), "=l"(r[10]), "=l"(r[11]), "=l"(r[12]), "=l"(r[13]), "=l"(r[14]), "=l"(r[15]),
        "=l"(r[16]), "=l"(r[17]), "=l"(r[18]), "=l"(r[19]), "=l"(r[20]), "=l"(r[21]), "=l"(r[22]), "=l"(r[23]),
        "=l"(r[24]), "=l"(r[25]), "=l"(r[26]), "=l"(r[27]), "=l"(r[28]), "=l"(r[29]), "=l"(r[30]), "=l"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld128_pairs(uint32_t taddr, uint64_t (&r)[64]) {
  asm volatile(
      "{\n\t.reg .b32 a<128>;\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x128.b32 {"
      "a0, a1, a2, a3, a4, a5, a6, a7, a8, a9, a10, a11, a12, a13, a14, a15, "
      "a16, a17, a18, a19, a20, a21, a22, a23, a24, a25, a26, a27, a28, a29, a30, a31, "
      "a32, a33, a34, a35, a36, a37, a38, a39, a40, a41, a42, a43, a44, a45, a46, a47, "
      "a48, a49, a50, a51, a52, a53, a54, a55, a56, a57, a58, a59, a60, a61, a62, a63, "
      "a64, a65, a66, a67, a68, a69, a70, a71, a72, a73, a74, a75, a76, a77, a78, a79, "
      "a80, a81, a82, a83, a84, a85, a86, a87, a88, a89, a90, a91, a92, a93, a94, a95, "
      "a96, a97, a98, a99, a100, a101, a102, a103, a104, a105, a106, a107, a108, a109, a110, a111, "
      "a112, a113, a114, a115, a116, a117, a118, a119, a120, a121, a122, a123, a124, a125, a126, a127}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;\n\t"
      "mov.b64 %0, {a0, a1}; mov.b64 %1, {a2, a3}; mov.b64 %2, {a4, a5}; mov.b64 %3, {a6, a7};\n\t"
      "mov.b64 %4, {a8, a9}; mov.b64 %5, {a10, a11}; mov.b64 %6, {a12, a13}; mov.b64 %7, {a14, a15};\n\t"
      "mov.b64 %8, {a16, a17}; mov.b64 %9, {a18, a19}; mov.b64 %10, {a20, a21}; mov.b64 %11, {a22, a23};\n\t"
      "mov.b64 %12, {a24, a25}; mov.b64 %13, {a26, a27}; mov.b64 %14, {a28, a29}; mov.b64 %15, {a30, a31};\n\t"
      "mov.b64 %16, {a32, a33}; mov.b64 %17, {a34, a35}; mov.b64 %18, {a36, a37}; mov.b64 %19, {a38, a39};\n\t"
      "mov.b64 %20, {a40, a41}; mov.b64 %21, {a42, a43}; mov.b64 %22, {a44, a45}; mov.b64 %23, {a46, a47};\n\t"
      "mov.b64 %24, {a48, a49}; mov.b64 %25, {a50, a51}; mov.b64 %26, {a52, a53}; mov.b64 %27, {a54, a55};\n\t"
      "mov.b64 %28, {a56, a57}; mov.b64 %29, {a58, a59}; mov.b64 %30, {a60, a61}; mov.b64 %31, {a62, a63};\n\t"
      "mov.b64 %32, {a64, a65}; mov.b64 %33, {a66, a67}; mov.b64 %34, {a68, a69}; mov.b64 %35, {a70, a71};\n\t"
      "mov.b64 %36, {a72, a73}; mov.b64 %37, {a74, a75}; mov.b64 %38, {a76, a77}; mov.b64 %39, {a78, a79};\n\t"
      "mov.b64 %40, {a80, a81}; mov.b64 %41, {a82, a83}; mov.b64 %42, {a84, a85}; mov.b64 %43, {a86, a87};\n\t"
      "mov.b64 %44, {a88, a89}; mov.b64 %45, {a90, a91}; mov.b64 %46, {a92, a93}; mov.b64 %47, {a94, a95};\n\t"
      "mov.b64 %48, {a96, a97}; mov.b64 %49, {a98, a99}; mov.b64 %50, {a100, a101}; mov.b64 %51, {a102, a103};\n\t"
      "mov.b64 %52, {a104, a105}; mov.b64 %53, {a106, a107}; mov.b64 %54, {a108, a109}; mov.b64 %55, {a110, a111};\n\t"
      "mov.b64 %56, {a112, a113}; mov.b64 %57, {a114, a115}; mov.b64 %58, {a116, a117}; mov.b64 %59, {a118, a119};\n\t"
      "mov.b64 %60, {a120, a121}; mov.b64 %61, {a122, a123}; mov.b64 %62, {a124, a125}; mov.b64 %63, {a126, a127};\n\t"
      "}"
      : "=l"(r[0]), "=l"(r[1]), "=l"(r[2]), "=l"(r[3]), "=l"(r[4]), "=l"(r[5]), "=l"(r[6]), "=l"(r[7]),
        "=l"(r[8]), "=l"(r[9]), "=l"(r[10]), "=l"(r[11]), "=l"(r[12]), "=l"(r[13]), "=l"(r[14]), "=l"(r[15]),
        "=l"(r[16]), "=l"(r[17]), "=l"(r[18]), "=l"(r[19]), "=l"(r[20]), "=l"(r[21]), "=l"(r[22]), "=l"(r[23]),
        "=l"(r[24]), "=l"(r[25]), "=l"(r[26]), "=l"(r[27]), "=l"(r[28]), "=l"(r[29]), "=l"(r[30]), "=l"(r[31]),
        "=l"(r[32]), "=l"(r[33]), "=l"(r[34]), "=l"(r[35]), "=l"(r[36]), "=l"(r[37]), "=l"(r[38]), "=l"(r[39]),
        "=l"(r[40]), "=l"(r[41]), "=l"(r[42]), "=l"(r[43]), "=l"(r[44]), "=l"(r[45]), "=l"(r[46]), "=l"(r[47]),
        "=l"(r[48]), "=l"(r[49]), "=l"(r[50]), "=l"(r[51]), "=l"(r[52]), "=l"(r[53]), "=l"(r[54]), "=l"(r[55]),
        "=l"(r[56]), "=l"(r[57]), "=l"(r[58]), "=l"(r[59]), "=l"(r[60]), "=l"(r[61]), "=l"(r[62]), "=l"(r[63])
      : "r"(taddr)
      : "memory");
}

// 32 lanes x 16 consecutive columns.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16]) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
        "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float (&r)[16]) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
        "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&r)[32]) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]),
        "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]),
        "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]),
        "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]), "r"(u[31])
      : "memory");
}

// ---------------------------------------------------------------------------------------------- MMA
// Shared-memory matrix descriptor, 128-byte swizzle (layout type 2), descriptor version 1.
// lbo / sbo are byte offsets (multiples of 16).  For a K-major operand sbo is the distance between
// 8-row groups and lbo is unused; for an MN-major operand lbo is the distance between 64-element
// chunks along M/N and sbo the distance between 8-deep groups along K.
__device__ __forceinline__ uint64_t make_smem_desc(uint32_t smem_addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Instruction descriptor for kind::f16 with bf16 operands and fp32 accumulation.
__host__ __device__ constexpr uint32_t make_idesc_bf16(int M, int N, bool a_mn_major, bool b_mn_major) {
  return (1u << 4)                          // D format: f32
         | (1u << 7)                        // A format: bf16
         | (1u << 10)                       // B format: bf16
         | ((a_mn_major ? 1u : 0u) << 15)   // A major
         | ((b_mn_major ? 1u : 0u) << 16)   // B major
         | ((uint32_t)(N >> 3) << 17)       // N / 8
         | ((uint32_t)(M >> 4) << 24);      // M / 16
}

// D[tmem] (+)= A[smem] * B[smem]; issued by one thread.
__device__ __forceinline__ void mma_bf16_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// One lane of a converged warp.  A warp that issues products runs as a whole up to here, so that what it works out for them (descriptors,
// addresses) is known to be the same for all lanes and stays in the uniform registers that the instruction reads; under a test
// of the lane every product first has its operands moved there, some 50 cycles each.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// mbarrier arrive once every MMA issued so far by this thread has completed.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---------------------------------------------------------------------------------------------- 8-bit operands, clusters
// Instruction descriptor for kind::f8f6f4 with e4m3 operands, both K-major, and fp32 accumulation.
__host__ __device__ constexpr uint32_t make_idesc_e4m3(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void mma_e4m3_ss(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// A cluster of CTAs on neighbouring SMs: `rank_address` is where a shared-memory address of this CTA lies in the CTA `rank`.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t rank_address(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// (after cluster_sync, before which the other CTA has written them)
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr));
  return x;
}
// Every thread of every CTA of the cluster arrives and waits; nothing before it can be left undone by a wait that ran out, since all
// of those are bounded.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// An arrival in another CTA that hands over tensor memory only, whose reads are complete (tcgen05.wait::ld): it releases nothing else, and
// a release at the cluster's scope would wait for every load under way (block-scaled product, 32768 x 5120 x 5120: 1807 -> 972 us).
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// A warpgroup's registers a thread, from here on; all its warps come here.  What some gain others must have given up, counted from what
// the CTA was launched with.
template <int N>
__device__ __forceinline__ void registers_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void registers_fewer() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// Two CTAs of a cluster as one: the even one's thread issues products of 256 rows, 128 in either's tensor memory, from both CTAs'
// shared memory (its own rows of A, half of the rows of B); the hand-over barriers of both are signalled at once.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_result, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(ncols) : "memory");
}
__device__ __forceinline__ void tmem_relinquish_pair() {
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ void mma_e4m3_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
// A tile of this CTA's own, counted on a barrier that may lie in the other CTA of the pair (`bar`: rank_address).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1)
      : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(src), "r"(c0), "r"(c1)
               : "memory");
}

// x -> three bf16 parts with x = x1 + x2 + x3 exactly, for two neighbouring elements at once (packed as
// bf16x2 words, element 0 in the low half).  Each part is the remainder truncated to its top 8 mantissa bits
// (a mask on the fp32 bit pattern), so three parts hold all 24 bits and the remainders are formed without
// rounding error.  Only integer/FMA-pipe instructions: the float->bf16 conversion instruction is an order of
// magnitude slower per warp on this GPU and sat on the critical path of the scan and the resolve.
__device__ __forceinline__ void split3_pair(float x0, float x1, uint32_t& p1, uint32_t& p2, uint32_t& p3) {
  uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
  p1 = __byte_perm(u0, u1, 0x7632);                       // {hi16(x1), hi16(x0)}
  x0 -= __uint_as_float(u0 & 0xFFFF0000u);
  x1 -= __uint_as_float(u1 & 0xFFFF0000u);
  u0 = __float_as_uint(x0); u1 = __float_as_uint(x1);
  p2 = __byte_perm(u0, u1, 0x7632);
  x0 -= __uint_as_float(u0 & 0xFFFF0000u);
  x1 -= __uint_as_float(u1 & 0xFFFF0000u);
  p3 = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
}

__device__ __forceinline__ void named_barrier_sync(int id, int nthreads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(nthreads) : "memory");
}

// A block-level barrier that also tells every participant whether any of them has given up on a wait.  A thread whose
// wait ran out does not leave at once -- the others, whose wait may have been satisfied a moment earlier, would then
// stand at their next bar.sync for ever -- but comes to that barrier with `gave_up` set, and all leave together.
__device__ __forceinline__ bool named_barrier_or(int id, int nthreads, bool gave_up) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %3, 0;\n\t"
      "bar.red.or.pred p, %1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(any)
      : "r"(id), "r"(nthreads), "r"(gave_up ? 1u : 0u)
      : "memory");
  return any != 0;
}

}  // namespace tc
}  // namespace vdn
