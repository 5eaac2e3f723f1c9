// Shared-memory barriers, TMA loads, tensor-memory reads and operand descriptors used by every
// tensor-core kernel of the library (tcgen05, sm_100a).
#pragma once
#include <cuda.h>

#include <atomic>

#include "device_utils.cuh"

namespace stmoe_dev {

// the float4 (or float) at this CTA's shared-memory address, read from CTA `rank` of the cluster
__device__ __forceinline__ float4 ld_cluster4(uint32_t smem, int rank)
{
    uint32_t remote;
    float4 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote));
    return v;
}
__device__ __forceinline__ float ld_cluster(uint32_t smem, int rank)
{
    uint32_t remote;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote));
    return v;
}

constexpr int kDenseSpinLimit = 1 << 22;
// Polls after which a wait of the operators' kernels gives up, for the launches to come (tests lower it).
inline std::atomic<int> g_mx4_polls{kDenseSpinLimit};

__device__ __forceinline__ uint32_t dsmem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void dmbar_init(uint64_t *bar, int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(dsmem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void dmbar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(dsmem_u32(bar)) : "memory");
}
// One lane of a converged warp.  The TMA and tcgen05 instructions take their operands from uniform
// registers: under a plain `lane == 0` the compiler cannot tell that one lane is left and wraps each of
// them in a loop over the active lanes' values (measured: 75-130 cycles an instruction).  Where such
// instructions follow one another closely (the MMA loop) even one elected lane is slow, because inside
// its branch every operand is moved to a uniform register first; there the whole warp walks the loop
// and the elected lane is a predicate of the instruction.
__device__ __forceinline__ bool elect_one()
{
    uint32_t mine;
    asm volatile(
        "{.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;}"
        : "=r"(mine));
    return mine != 0;
}
__device__ __forceinline__ bool dmbar_try(uint64_t *bar, uint32_t parity)
{
    uint32_t done;
    asm volatile(
        "{.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;}"
        : "=r"(done)
        : "r"(dsmem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// bounded wait on a phase parity; false when the limit ran out or another thread gave up
__device__ __forceinline__ bool dmbar_wait(uint64_t *bar, uint32_t parity, volatile int *dead,
                                           int spin_limit = kDenseSpinLimit)
{
    for (int spins = 0; spins < spin_limit; ++spins) {
        if (dmbar_try(bar, parity)) return true;
        if (*dead) return false;
    }
    *dead = 1;
    return false;
}

// Behind a wait that ran out, before a block gives its shared and tensor memory back: time for the copies
// and MMAs that it still has in flight, whose barriers may never complete any more (a copy takes
// microseconds; 1 ms by the clock, and a bounded number of looks at it).  Not inlined: kernels that it is
// never called in pay for every line of code that they fetch.
inline __device__ __noinline__ void settle_in_flight()
{
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
    for (int i = 0; i < 1 << 16; ++i) {
        asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
        if (t - t0 > 1000000ull) break;
        __nanosleep(1000);
    }
}

// K-major, no-swizzle shared-memory matrix descriptor: 8-row groups `sbo` bytes apart, the two
// 16-byte K chunks of one MMA `lbo` bytes apart (descriptor version 1 = sm_100).
__device__ __forceinline__ uint64_t umma_desc(uint32_t smem_addr, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((smem_addr >> 4) & 0x3FFFu) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)((sbo >> 4) & 0x3FFFu) << 32) | (1ull << 46);
}
__device__ __forceinline__ void umma_commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(dsmem_u32(bar))
                 : "memory");
}
// the same from a whole warp, by the lane that `leader` names
__device__ __forceinline__ void umma_commit_if(bool leader, uint64_t *bar)
{
    asm volatile(
        "{.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];}" ::"r"(dsmem_u32(bar)),
        "r"((uint32_t)leader)
        : "memory");
}
// tensor memory -> registers, eight columns of this thread's lane; the values are there after tmem_ld_wait
__device__ __forceinline__ void tmem_ld8_start(uint32_t addr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float (&v)[8])
{
    uint32_t r[8];
    tmem_ld8_start(addr, r);
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async;" ::: "memory"); }

__device__ __forceinline__ void dmbar_expect_tx(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(dsmem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int c0, int c1, int c2, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dsmem_u32(dst)), "l"(map), "r"(dsmem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d_at(uint32_t dst, const CUtensorMap *map, int c0, int c1, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(dsmem_u32(bar)), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void tma_load_2d(void *dst, const CUtensorMap *map, int c0, int c1, uint64_t *bar)
{
    tma_load_2d_at(dsmem_u32(dst), map, c0, c1, bar);
}
// K-major operand tile in the 128-byte swizzled layout (rows of 128 bytes, 8-row groups 1024
// bytes apart, tile base 1024-byte aligned); kstep = which 32-byte slice of the row (one MMA's
// reduction depth: 16 two-byte or 32 one-byte elements).
__device__ __forceinline__ uint64_t umma_desc_sw128(uint32_t smem_addr, int kstep)
{
    return (uint64_t)(((smem_addr + kstep * 32) >> 4) & 0x3FFFu) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// The two descriptor forms by their low words (address and leading offset); the high words are constant.
constexpr uint32_t kDescHighSw128 = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t kDescHighScales = (128u >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_low_sw128(uint32_t smem_addr) { return ((smem_addr >> 4) & 0x3FFFu) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_low_scales(uint32_t smem_addr) { return ((smem_addr >> 4) & 0x3FFFu) | ((128u >> 4) << 16); }
}  // namespace stmoe_dev
