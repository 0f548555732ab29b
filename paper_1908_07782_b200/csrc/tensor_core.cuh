// Blackwell's tensor cores by inline PTX: mbarriers, tiled TMA loads, tcgen05 products with accumulators in TMEM.
// CG = 1: a CTA by itself; CG = 2: a pair of CTAs (a cluster of two) forms one product of twice the height, each with
// its half of both operands and of the accumulator; the pair's even CTA, the leader, issues the products.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace combo_tc {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// One thread of the warp, the same at every call: the whole warp asks.  What it issues alone stands under this test and
// not under a comparison of lane numbers, which would have the compiler expect many threads there (100 cycles a copy).
__device__ __forceinline__ bool elect() {
    uint32_t p;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// The same place in the shared memory of the pair's leader, as a cluster address.
__device__ __forceinline__ uint32_t at_leader(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}

// Arrivals on an own barrier, or (`bar` a cluster address; an own address is one) on any.  Cluster-wide release costs about a microsecond, so it
// is asked for only where a thread's own writes are handed over: bytes that TMA brings are published by the barrier
// itself, and TMEM by tcgen05's fences.
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_release(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

constexpr uint32_t kPolls = 1u << 22;        // polls before a wait is given up: 17 s, a poll being suspended for 4 us by the hardware
// Waits for the phase of that parity; false if it is given up, or if `dead` was set meanwhile.  CLUSTER: what threads of
// the other CTA wrote before they arrived is seen behind the wait.
template <bool CLUSTER> __device__ __forceinline__ bool mbar_poll(uint32_t bar, uint32_t parity, const volatile int* dead) {
    uint32_t ok;
#pragma unroll 1
    for (uint32_t it = 1; it <= kPolls; ++it) {
        if constexpr (CLUSTER)
            asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                         : "=r"(ok)
                         : "r"(bar), "r"(parity)
                         : "memory");
        else
            asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                         : "=r"(ok)
                         : "r"(bar), "r"(parity)
                         : "memory");
        if (ok) return true;
        if (it % 1024 == 0 && *dead) return false;
    }
    return false;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const volatile int* dead) { return mbar_poll<false>(bar, parity, dead); }
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, const volatile int* dead) { return mbar_poll<true>(bar, parity, dead); }

// ---- TMA: boxes of global memory into this CTA's shared memory; bytes are counted on `bar` (CG = 2: the leader's)
template <int CG> __device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y)
                     : "memory");
}
template <int CG> __device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
                     : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int u, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(u)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                     "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(u)
                     : "memory");
}
// A box of this CTA's shared memory to global memory; the thread that asked may wait until it has been read (the memory may be
// used again), or is there.  Outside the map nothing is written, but for a line that ends inside 16 bytes: those are written whole
// (measured: lines of 773 floats, the three behind each).
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t from, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y), "r"(z)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// The same, added to what is there.
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* map, uint32_t from, int x, int y, int z) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y), "r"(z)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// what threads wrote to shared memory becomes visible to the tensor cores and to TMA
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- TMEM
template <int CG> __device__ __forceinline__ void tmem_alloc(uint32_t where, uint32_t columns) {
    if constexpr (CG == 1) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    else asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
}
template <int CG> __device__ __forceinline__ void tmem_release(uint32_t base, uint32_t columns) {
    if constexpr (CG == 1) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    }
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: v[c] of a lane is (its row, column c)
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
}
// All loads so far have arrived in `v`: naming the registers keeps their uses behind the wait.
__device__ __forceinline__ void tmem_load_wait(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                   "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                   "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                   "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}

// 16 columns of the warp's 32 lanes: v becomes what is at `from`, added to what is at `to` if `add`, and is left at `to`.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                   "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}
__device__ __forceinline__ void tmem_fold16(uint32_t from, uint32_t to, bool add) {
    uint32_t v[16];
    tmem_load16(from, v);
    if (add) {
        uint32_t m[16];
        tmem_load16(to, m);
        tmem_load_wait(v);
        tmem_load_wait(m);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + __uint_as_float(m[e]));
    } else {
        tmem_load_wait(v);
    }
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
        "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
        "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(to)
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- products
// Shared-memory operand, 128-byte swizzle (8 lines of 128 bytes to an atom).
// Contiguous along r: a line is one i with 64 values of r; atoms of 8 values of i lie 1024 bytes apart.
// Contiguous along i: a line is one r with 64 values of i; atoms of 8 values of r lie 1024 bytes apart, blocks of 64
// values of i `block` bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool along_r, uint32_t block) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)((along_r ? 16u : block) >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 |
           1ull << 46 | 2ull << 61;
}
// Shared-memory operand without swizzle: pieces of 8 x 16 bytes, 128 bytes each, `next_r` bytes from one to the next along r,
// `next_i` along its own index (either index may be the one that 16 bytes run along).
__device__ __forceinline__ uint64_t operand_plain(uint32_t addr, uint32_t next_r, uint32_t next_i) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(next_r >> 4) << 16 | (uint64_t)(next_i >> 4) << 32 | 1ull << 46;
}
// bytes from one step of 16 values of r to the next
__host__ __device__ constexpr uint32_t step16(bool along_r) { return along_r ? 32u : 2048u; }
// bfloat16 times bfloat16 into binary32, m x n outputs
__device__ __forceinline__ uint32_t product_kind(int m, int n, bool a_along_r, bool b_along_r) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (a_along_r ? 0u : 1u << 15) | (b_along_r ? 0u : 1u << 16) | (uint32_t)(n >> 3) << 17 |
           (uint32_t)(m >> 4) << 24;
}
// the same for float16
__device__ __forceinline__ uint32_t product_kind_half(int m, int n, bool a_along_r, bool b_along_r) { return product_kind(m, n, a_along_r, b_along_r) & ~(1u << 7 | 1u << 10); }
template <int CG> __device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
    if constexpr (CG == 1)
        asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a),
                     "l"(b), "r"(kind), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a),
                     "l"(b), "r"(kind), "r"((uint32_t)add)
                     : "memory");
}
// An arrival on `bar` (CG = 2: at the same place in both CTAs) when this thread's products so far are done.
template <int CG> __device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((unsigned short)3)
                     : "memory");
}

}  // namespace combo_tc
