// Inline-PTX wrappers of the fifth-generation tensor cores as a pair of blocks uses them (tcgen05, cta_group::2):
// tensor memory, matrix instructions on operands in shared memory, tensor copies, barriers across the pair.
#ifndef NBOS_TENSOR_CUH_
#define NBOS_TENSOR_CUH_

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "nbos_ptx.cuh"

namespace nbos {
namespace tensor {

__device__ __forceinline__ uint32_t pair_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// address of the same place in the shared memory of block `rank` of the cluster
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void barriers_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// A barrier anywhere in the cluster. What is handed over here is tensor memory, whose accesses the tcgen05 fences order: a release to the
// whole cluster would wait for all of the thread's memory accesses besides.
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity)
{
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
// Bounded, as mbar_wait: false when the wait ran out or another thread of the block gave up.
static __device__ __noinline__ bool wait_cluster_slow(uint32_t bar, uint32_t parity, volatile unsigned int *abort_flag, unsigned long long limit_ns)
{
    const unsigned long long t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 32; ++i)
            if (try_wait_cluster(bar, parity)) return true;
        if (*abort_flag) return false;
        if (global_timer_ns() - t0 > limit_ns) {
            *abort_flag = 1u;
            return false;
        }
    }
}
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile unsigned int *abort_flag, unsigned long long limit_ns)
{
    if (try_wait_cluster(bar, parity)) return true;
    return wait_cluster_slow(bar, parity, abort_flag, limit_ns);
}

// ---- tensor copies ------------------------------------------------------------------------------------------
// A box of a three-dimensional map to this block's shared memory; the bytes count on a barrier of the pair (no multicast).
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t cluster_bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(cluster_bar)
        : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, int x, int y, int z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void stores_read_wait()   // until their shared memory may be written again
{
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
}
__device__ __forceinline__ void stores_drain() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---- tensor memory ------------------------------------------------------------------------------------------
// A warp of each block of the pair calls these, after a barrier of the pair and before one: both blocks have to be there. `at` is a word of
// shared memory that gets the address.
__device__ __forceinline__ void tmem_alloc(uint32_t at, int columns)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, int columns)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 32 neighbouring columns of this warp's 32 lanes: one row a thread
__device__ __forceinline__ void tmem_load32(uint32_t (&v)[32], uint32_t at)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(at)
        : "memory");
}
// The loaded registers pass through, so that nothing that uses them moves before the wait.
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                   "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]),
                   "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]),
                   "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :
                 : "memory");
}

// one column of this warp's 32 lanes
__device__ __forceinline__ void tmem_load1(uint32_t &v, uint32_t at)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t &v) { asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v) : : "memory"); }

// 32 neighbouring columns of 16 lanes: thread t has v[4 j + 2 r + e] = lane t / 4 + 8 r, column 8 j + 2 (t % 4) + e
__device__ __forceinline__ void tmem_load16(uint32_t (&v)[16], uint32_t at)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&v)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                   "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}

// ---- matrix instructions ------------------------------------------------------------------------------------
// Operand tiles lie in shared memory in rows of 128 bytes, eight rows to an atom of 1,024 bytes whose 16-byte
// pieces are swizzled (the tensor copies' 128-byte swizzle).
//   along K:  a row is 64 values of K of one M (or N): atoms follow one another along M; 16 values of K are 32 bytes
//   along MN: a row is 64 values of M (or N) for one K: atoms follow one another along K, blocks of 64 of M at `next`
__device__ __forceinline__ uint64_t operand_base(bool along_k, uint32_t next)
{
    const uint64_t leading = along_k ? 1u : (next >> 4), step = 1024u >> 4;
    return leading << 16 | step << 32 | 1ull << 46 /* version */ | 2ull << 61 /* 128-byte swizzle */;
}
__device__ __forceinline__ uint64_t operand(uint64_t base, uint32_t addr) { return base | ((addr >> 4) & 0x3FFF); }

template <typename T> constexpr uint32_t kOperandType = 0;                      // f16
template <> constexpr uint32_t kOperandType<__nv_bfloat16> = 1;
// D (32 bits) = A B: an M x N tile of the pair
template <typename T>
__host__ __device__ constexpr uint32_t instruction(int m, int n, bool a_along_k, bool b_along_k)
{
    return 1u << 4 | kOperandType<T> << 7 | kOperandType<T> << 10 | (a_along_k ? 0u : 1u) << 15 | (b_along_k ? 0u : 1u) << 16 |
           (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
__device__ __forceinline__ void mma(uint32_t tmem, uint64_t a, uint64_t b, uint32_t instr, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)add)
        : "memory");
}
// Once the matrix instructions so far have finished, one arrival at this place in both blocks.
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3)
                 : "memory");
}

}  // namespace tensor
}  // namespace nbos
#endif
