// PTX wrappers shared by the kernels: mbarriers with bounded waits, TMA loads, cluster barriers.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

namespace psgd {

constexpr unsigned FU_WAIT_LIMIT = 1u << 20;   // polls of one mbarrier wait before giving up
constexpr int FU_W_TIMEOUT = 4;                // == PSGD_W_TIMEOUT
#ifndef PSGD_WARP_WAIT_LIMIT
#define PSGD_WARP_WAIT_LIMIT FU_WAIT_LIMIT     // of mbar_wait_warp; a build with 0 gives up every such wait at once (test of what then happens)
#endif

// ---- PTX wrappers ---------------------------------------------------------------------------
__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(unsigned bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_expect_tx(unsigned bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(unsigned bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(unsigned bar, unsigned parity) {
    unsigned ok;
    asm volatile(
        "{\n.reg .pred p;\n"
#ifdef PSGD_MBAR_TEST_WAIT
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
#else
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
#endif
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait: gives up after FU_WAIT_LIMIT polls, records it and lets the caller go on; a thread
// that has given up once no longer waits at all (`dead`), so a broken pipeline still ends quickly.
__device__ __forceinline__ void mbar_wait(unsigned bar, unsigned parity, int* flags, bool& dead) {
    if (dead) return;
    for (unsigned it = 0; it < FU_WAIT_LIMIT; ++it)
        if (mbar_try_wait(bar, parity)) return;
    dead = true;
    atomicOr(flags, FU_W_TIMEOUT);
}
__device__ __forceinline__ bool mbar_test(unsigned bar, unsigned parity) {   // never blocks
    unsigned ok;
    asm volatile(
        "{\n.reg .pred p;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// For a role played by a single thread whose barrier has usually completed already: a non-blocking test first.
__device__ __forceinline__ void mbar_wait_ready(unsigned bar, unsigned parity, int* flags, bool& dead) {
    if (!mbar_test(bar, parity)) mbar_wait(bar, parity, flags, dead);
}
// The same wait for a whole warp (all 32 lanes must call it): lane 0 polls, pausing between polls, so that a waiting
// warp puts one request at a time on the barrier instead of 32 (many warps polling at full rate slow down every other
// barrier operation of the CTA, the single MMA-issuing thread's first of all); once the phase has completed every lane
// observes it itself with one more try_wait, which returns at once and gives that lane its own acquire.
__device__ __forceinline__ void mbar_wait_warp(unsigned bar, unsigned parity, int* flags, bool& dead) {
    if (dead) return;                        // (uniform across the warp: set from lane 0 below)
    int gave_up = 0;
    if ((threadIdx.x & 31) == 0) {
        bool ok = false;
        for (unsigned it = 0; it < PSGD_WARP_WAIT_LIMIT && !ok; ++it) {
            ok = mbar_try_wait(bar, parity);
            if (!ok) __nanosleep(40);
        }
        if (!ok) { gave_up = 1; atomicOr(flags, FU_W_TIMEOUT); }
    }
    gave_up = __shfl_sync(0xffffffffu, gave_up, 0);
    if (gave_up) { dead = true; return; }
#ifndef PSGD_MBAR_NO_REWAIT
    (void)mbar_try_wait(bar, parity);
#endif
}
// TMA: one tile {x: columns, y: rows, z: (matrix, node)} of a rank-3 tensor map into shared memory.
// x must be a multiple of 4 floats (16 bytes); coordinates past the extents read zeros.
__device__ __forceinline__ void tma_load_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_arrive_release() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void cluster_wait_acquire() {
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void st_cluster_f32(unsigned local_addr, unsigned rank, float v) {
    unsigned remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(remote) : "r"(local_addr), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(remote), "f"(v) : "memory");
}

}  // namespace psgd
