// sm_103a building blocks of the expert products: barriers in shared memory with
// bounded waits, tile loads by the TMA unit, and the fifth-generation tensor cores
// (tcgen05) used by one CTA or by pairs (kCtas: 1 or 2).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace gnmr_mma {

__device__ __forceinline__ uint32_t smem_addr(const void *p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}

// The same shared-memory address in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One lane of a converged warp, the same one each time.
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes != 0;
}

// ---- barriers ---------------------------------------------------------------

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void barrier_init_fence()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

// Arrivals on a barrier of any CTA of the cluster (an address from in_cta).  The
// plain one hands over tensor memory and nothing else, between tcgen05.wait and fence_before on this
// side and fence_after on the other, which order it: a release would wait for the outputs' stores
// too (49152 x 2048 -> 1408 over 64 experts 558 us with releases, 290 without).
__device__ __forceinline__ void arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// After shared memory was read that will be written anew, or was written and, past fence_async_proxy, the
// tensor cores will read.  On a barrier of this CTA (its own address), for a thread of it that waits; or on one
// of the pair's first CTA (from in_cta), where the thread that waits is: the narrower scope says nothing about
// that one.  (The wider one takes 2,000 cycles, so that a loop of every stage keeps to its own CTA.)
__device__ __forceinline__ void release(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void release_in_pair(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void arrive_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}

// Whether a phase is complete, for a whole warp, after a nap of the hardware's choosing.  kPaired: a barrier
// on which the other CTA arrives too, or its multiplies.
template <bool kPaired> __device__ __forceinline__ bool complete(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    if (kPaired)
        asm volatile("{\n.reg .pred p;\n"
                     "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                     "selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done)
                     : "r"(bar), "r"(parity)
                     : "memory");
    else
        asm volatile("{\n.reg .pred p;\n"
                     "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n"
                     "selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done)
                     : "r"(bar), "r"(parity)
                     : "memory");
    return __all_sync(~0u, done);
}

__device__ __forceinline__ uint64_t nanoseconds()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// Every wait ends: after `most` nanoseconds it returns false, and its caller leaves its
// loop.  By a whole warp, which goes on or gives up as one.
template <bool kPaired> __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, uint64_t most)
{
    if (complete<kPaired>(bar, parity))
        return true;
    for (const uint64_t since = nanoseconds(); !complete<kPaired>(bar, parity);)
        if (__any_sync(~0u, nanoseconds() - since >= most))
            return false;
    return true;
}

// Registers a thread of this warpgroup may use from here on.
template <int kRegisters> __device__ __forceinline__ void more_registers()
{
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegisters));
}

template <int kRegisters> __device__ __forceinline__ void fewer_registers()
{
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegisters));
}

// ---- tile loads ---------------------------------------------------------------
// In a pair, the barrier may be the other CTA's.

template <int kCtas>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int x, int y, int block, int z, uint32_t bar)
{
    if (kCtas == 1) {
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                     "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(block), "r"(z), "r"(bar)
                     : "memory");
        return;
    }
    asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(block), "r"(z), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// What generic stores wrote to shared memory, for the tensor cores to read.
__device__ __forceinline__ void fence_async_proxy()
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ---- tensor memory and tensor cores ----------------------------------------------

template <int kCtas> __device__ __forceinline__ void tmem_alloc(uint32_t smem_result, uint32_t columns)
{
    if (kCtas == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        return;
    }
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_result), "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

template <int kCtas> __device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns)
{
    if (kCtas == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
        return;
    }
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory operand in 128-byte swizzled rows.
//   rows along the contraction (K-major): 8 rows of 64 elements are 1,024 bytes,
//     `stride` the bytes to the next 8 rows; `lead` is not used;
//   rows along the lanes or columns (MN-major): each 128-byte row is 64 of them at
//     one place of the contraction, `stride` the bytes to the next 8 places,
//     `lead` those to the next 64 lanes or columns.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead, uint32_t stride)
{
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | static_cast<uint64_t>((lead >> 4) & 0x3fff) << 16 |
           static_cast<uint64_t>((stride >> 4) & 0x3fff) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// 128 lanes in each CTA by `columns`, 16-bit operands of one type, fp32 sums.
template <int kCtas>
__device__ __forceinline__ uint32_t shape(bool bf16, bool a_along_lanes, bool b_along_columns, uint32_t columns)
{
    const uint32_t type = bf16 ? 1 : 0;
    return 1u << 4 | type << 7 | type << 10 | (a_along_lanes ? 1u << 15 : 0) | (b_along_columns ? 1u << 16 : 0) |
           (columns >> 3) << 17 | (128u * kCtas >> 4) << 24;
}

// One step of 16 along the contraction, by one thread, of a pair's first CTA for both.
__device__ __forceinline__ void multiply(uint32_t tmem, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(tmem),
                 "l"(a), "l"(b), "r"(shape), "r"(static_cast<uint32_t>(add))
                 : "memory");
}

// The same with A's 16 elements of each lane in tensor memory, two to a column.
template <int kCtas>
__device__ __forceinline__ void multiply(uint32_t tmem, uint32_t a, uint64_t b, uint32_t shape, bool add)
{
    if (kCtas == 1) {
        asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(tmem),
                     "r"(a), "l"(b), "r"(shape), "r"(static_cast<uint32_t>(add))
                     : "memory");
        return;
    }
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(tmem),
                 "r"(a), "l"(b), "r"(shape), "r"(static_cast<uint32_t>(add))
                 : "memory");
}

// Arrives on `bar`, in both CTAs of a pair, once every multiply issued so far is done.
template <int kCtas> __device__ __forceinline__ void commit(uint32_t bar)
{
    if (kCtas == 1) {
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
        return;
    }
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
}

// 16 columns of this warp's 32 lanes; complete after load_wait.
__device__ __forceinline__ void load16(uint32_t tmem, uint32_t (&v)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(tmem));
}

// Until the last load16 of this thread is in; v is named so that nothing reads it earlier.
__device__ __forceinline__ void load_wait(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

// 32 columns of this warp's 32 lanes; complete after store_wait.
__device__ __forceinline__ void store32(uint32_t tmem, const uint32_t (&v)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 :
                 : "r"(tmem), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
                 : "memory");
}

__device__ __forceinline__ void store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

}  // namespace gnmr_mma
