// Tensor-core (tcgen05) and tensor-map copy helpers, and the descriptors of operands in shared memory.
#pragma once

#include "ciera_pipe.cuh"

namespace ciera {

// Two blocks of threads on neighbouring SMs (a cluster of 2) work on one product: each holds its own 128 rows of the one
// operand, half of the other, and its rows' sums; one thread of the first block starts the products of both.

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the first block's address of something that lies at `p` in each block
__device__ __forceinline__ uint32_t in_first_block(const void* p) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(p)));
    return a;
}
// Arrivals on a barrier of either block, for work that the other block starts, so both sides have the cluster's scope.  With what
// the warp has written to its own shared memory (behind a fence_async_shared), which is all that the release is for: a full one waits
// for results on their way to memory too (weights' gradient of 32768 rows 270 us with it) ...
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("fence.release.sync_restrict::shared::cta.cluster;\n\t"
                 "mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
}
// ... and with tensor memory that has been read, which a tensor_fence_before orders
__device__ __forceinline__ void mbar_arrive_cluster_read(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// behind a mbar_wait_cluster: what the other block's warps have written to shared memory
__device__ __forceinline__ void fence_acquire_shared() { asm volatile("fence.acquire.sync_restrict::shared::cluster.cluster;" ::: "memory"); }
// true in one lane of the warp, the same one every time.  Tensor work and tensor-map copies are started under this, by a warp that
// otherwise runs as one: under `lane == 0` the compiler does not see that one thread is left, and starting a stage's products
// took longer than the products (8192^3 507 us, 403 with this).
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
// mbar_wait for phases that are mostly over or about to be: without the suspension of its polls at first, which wakes up late
// (32768 rows of 64 experts 185 us with it, 175 without)
__device__ __forceinline__ bool mbar_wait_soon(uint64_t* bar, uint32_t parity, volatile int* abort, int32_t* status,
                                               uint32_t max_polls = kMaxBarrierPolls) {
    for (int i = 0; i < 256; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
    }
    return mbar_wait(bar, parity, abort, status, max_polls);
}

// mbar_wait_soon for a barrier on which the other block's threads arrive
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, volatile int* abort, int32_t* status) {
    for (uint32_t i = 0; i < 256 + kMaxBarrierPolls; ++i) {
        uint32_t ok;
        if (i < 256)
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(ok)
                : "r"(smem_u32(bar)), "r"(parity)
                : "memory");
        else
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(ok)
                : "r"(smem_u32(bar)), "r"(parity), "r"(kSuspendNs)
                : "memory");
        if (ok) return true;
        if (i >= 256 && *abort) return false;
    }
    *abort = 1;
    if (status) atomicCAS(status, 0, (int32_t)CIERA_ERR_TIMEOUT);
    return false;
}

// ---- tensor memory: 128 lanes x 512 columns of 32 bits in each block; an address is lane << 16 | column

__device__ __forceinline__ void tmem_alloc(uint32_t* where, uint32_t columns) {  // a whole warp of each block
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(where)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {  // the same warps
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// arrives on the barrier at `bar` in both blocks when all the thread's tensor work so far has finished
__device__ __forceinline__ void tensor_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
// 32 columns of the warp's 32 lanes: lane i gets its lane's values
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(at));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- operands in shared memory

// Rows of 128 bytes along the contraction, written by a tensor map with 128-byte swizzle: groups of 8 rows 1024 bytes apart;
// the tile starts at a multiple of 1024.  The next 32 bytes of the contraction are 2 further on (units of 16 bytes).
__device__ __forceinline__ uint64_t operand_descriptor(const void* tile) {
    return (uint64_t)((smem_u32(tile) & 0x3ffff) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// 32 rows of 16 bytes, one behind the other
__device__ __forceinline__ uint64_t scales_descriptor(const void* rows) {
    return (uint64_t)((smem_u32(rows) & 0x3ffff) >> 4) | 1ull << 16 | (uint64_t)(128 >> 4) << 32 | 1ull << 46;
}
// 32 rows of 128 bits to 4 columns, the same in each quarter of the lanes; in both blocks, each from its own shared memory
__device__ __forceinline__ void tmem_copy_scales(uint32_t to, uint64_t rows) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(rows) : "memory");
}

// e4m3 operands with a power of two for each row and 32 values of the contraction, fp32 sums; the scales are byte `byte` of
// the words in tensor memory
__host__ __device__ constexpr uint32_t mx_byte(uint32_t byte) { return byte << 4 | byte << 29; }
__host__ __device__ constexpr uint32_t mx_instruction(uint32_t m, uint32_t n, uint32_t byte) {
    return (n >> 3) << 17 | 1u << 23 /* scales are powers of two */ | (m >> 4) << 24 | mx_byte(byte);
}
__device__ __forceinline__ void tensor_mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t a_scales,
                                              uint32_t b_scales, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(instruction), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
        : "memory");
}

// e2m1 operands with a power of two for each row and 32 values of the contraction, 64 of which an instruction takes; the scales
// are two bytes of the words in tensor memory, from byte 0 or (mx_byte(2)) 2 on
__host__ __device__ constexpr uint32_t mx4_instruction(uint32_t m, uint32_t n) {
    return 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 /* scales are powers of two */ | (m >> 7) << 27;
}
__device__ __forceinline__ void tensor_mma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t a_scales,
                                               uint32_t b_scales, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(instruction), "r"(a_scales), "r"(b_scales), "r"((uint32_t)add)
        : "memory");
}

// ---- tensor maps

__device__ __forceinline__ void prefetch_map(const void* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// to the block's own shared memory; `bar`: a barrier of either block
__device__ __forceinline__ void map_load3(void* dst, const void* map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void map_load4(void* dst, const void* map, int32_t x, int32_t y, int32_t z, int32_t w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            smem_u32(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}

}  // namespace ciera
