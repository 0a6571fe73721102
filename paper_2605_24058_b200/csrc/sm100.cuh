// sm_100a building blocks of the product kernels: mbarriers with bounded waits, tiled copies, tcgen05.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "lordba_internal.h"

namespace lordba {
namespace sm100 {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---- clusters -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t v;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(v));
    return v;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of the same shared-memory location in another CTA of the cluster
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint4 load_peer_v4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void store_peer(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// ---- mbarriers -------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_init_fence()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\n"
                 "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
                 "selp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}

// Every wait is bounded: the thread that gives up records a code in the device status word and raises the
// CTA's abort flag, after which all waits return false at once and the roles walk on to the kernel's end.
struct Bounded {
    volatile int *abort_flag;   // shared memory
    int *status;                // global

    __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, int code) const
    {
        if (bar_try(bar, parity)) return *abort_flag == 0;
        const long long start = clock64();
        for (uint32_t spins = 0;; ++spins) {
            if (bar_try(bar, parity)) return *abort_flag == 0;
            if ((spins & 15u) == 15u) {
                if (*abort_flag) return false;
                if (clock64() - start > kWaitLimitCycles) {
                    atomicCAS(status, 0, code);
                    *abort_flag = 1;
                    return false;
                }
            }
        }
    }
};

// Position in a ring of `size` stages and the parity of its barriers.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int size)
    {
        if (++stage == size) { stage = 0; phase ^= 1u; }
    }
};

// ---- tiled copies: x along a row (its byte offset a multiple of 16), y the row -----------------------------
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y) : "memory");
}
// the same, completing on a barrier of either CTA of a pair (cluster address)
__device__ __forceinline__ void load_tile_pair(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t cluster_bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(cluster_bar), "r"(x), "r"(y) : "memory");
}
// A stage written by ordinary stores: they are made visible to the tensor core before the arrival.
__device__ __forceinline__ void store_shared_v4(uint32_t addr, uint4 v)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 load_shared_v4(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// Sixteen bytes from an aligned global address, asynchronously; zeros (nothing is read) where !in.
__device__ __forceinline__ void fetch16(uint32_t to, uintptr_t from, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void fetch_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// wait until at most `left` (0 ... 5) of this thread's groups are in flight
__device__ __forceinline__ void fetch_wait(int left)
{
    if (left == 5) asm volatile("cp.async.wait_group 5;" ::: "memory");
    else if (left == 4) asm volatile("cp.async.wait_group 4;" ::: "memory");
    else if (left == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (left == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The tile at `from` to memory; what lies outside of the matrix is left out.  One thread.
__device__ __forceinline__ void store_tile(const CUtensorMap *map, uint32_t from, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(from), "r"(x), "r"(y) : "memory");
}
// The thread's stores since the last call become a group (an empty one where there were none): the waits below
// count groups.
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read_but_one() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void stores_complete() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// ---- tcgen05 ---------------------------------------------------------------------------------------------
// PAIR = 1: one CTA's tensor core; 2: those of a CTA pair (M = 256, both CTAs' shared memory and TMEM).
template <int PAIR>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns)
{
    if constexpr (PAIR == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int PAIR>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns)
{
    if constexpr (PAIR == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory matrix descriptors of 128-byte swizzled tiles, as (low, high) words; advancing the start by
// n bytes adds n / 16 to the low word.
//   contraction contiguous: rows of 128 bytes, eight of them a swizzle atom, atoms 1024 bytes apart;
//   m (n) contiguous: a row is 64 elements of one contraction index, eight rows an atom, atoms 1024 bytes
//     apart along the contraction, groups of 64 columns `group` bytes apart.
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t group = 0) { return ((addr >> 4) & 0x3fffu) | (group >> 4) << 16; }
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;      // stride of the atoms, version, 128-byte swizzle

// Instruction descriptors: type of the sum, of A and B, which of them are m (n) contiguous, the tile.
constexpr uint32_t kSumF32 = 1u << 4, kSumS32 = 2u << 4;
__host__ __device__ constexpr uint32_t instr_desc(bool int8, bool bf16, bool a_mn, bool b_mn, int m, int n)
{
    return (int8 ? kSumS32 | 1u << 7 | 1u << 10 : kSumF32 | (bf16 ? 1u << 7 | 1u << 10 : 0u)) | (a_mn ? 1u << 15 : 0u) |
           (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}

template <int PAIR, bool INT8>
__device__ __forceinline__ void mma(uint32_t d, uint32_t a_low, uint32_t b_low, uint32_t idesc, uint32_t accumulate)
{
#define LORDBA_MMA(GROUP, KIND)                                                                                     \
    asm volatile("{\n.reg .pred p;\n.reg .b64 da, db;\nsetp.ne.b32 p, %5, 0;\n"                                     \
                 "mov.b64 da, {%1, %4};\nmov.b64 db, {%2, %4};\n"                                                   \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], da, db, %3, p;\n}"                          \
                 ::"r"(d), "r"(a_low), "r"(b_low), "r"(idesc), "r"(kDescHigh), "r"(accumulate) : "memory")
    if constexpr (PAIR == 2 && INT8) LORDBA_MMA("2", "i8");
    else if constexpr (PAIR == 2) LORDBA_MMA("2", "f16");
    else if constexpr (INT8) LORDBA_MMA("1", "i8");
    else LORDBA_MMA("1", "f16");
#undef LORDBA_MMA
}
// Arrive on a barrier once the MMAs issued so far are complete; in a pair, on the barrier of both CTAs.
template <int PAIR>
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    if constexpr (PAIR == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// Sixteen columns of the warp's 32 lanes.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t r[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

}  // namespace sm100
}  // namespace lordba
