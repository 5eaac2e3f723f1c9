// MX4 product on the tensor cores (tcgen05.mma kind::mxf4, block scales in tensor memory):
//
//   out[t][i] = sum_k a[t][k] * b_e(t)[i][k]
//
// with both operands in MX4 (mx4.cuh).  The rows of a (tokens) are sorted by expert: counts[e] rows
// belong to matrix e of b, in order; without counts there is one matrix and every row belongs to it.
// The products of codes and scales are exact, sums are fp32 in tensor memory, the result is rounded
// once.
//
// The rows of b are the MMA's M (128 a tile), the tokens its N (a tile of up to 192, multiples of
// 16), and a stage holds 256 elements of the reduction: 128 bytes of codes a row, the width of the
// swizzled operand layout, four MMAs of depth 64.
//   warp 0      one thread loads the code tiles by TMA
//   warp 1      one thread copies a stage's scales into tensor memory (tcgen05.cp), issues its four
//               MMAs and frees the stage; the warp owns the tensor-memory allocation
//   warps 2-5   epilogue, from two accumulator buffers
//   warps 6-9   scales, a warp every fourth stage: a lane reads eight scale bytes of the rows lane,
//               lane + 32, ... (its next stage's before it waits for this one's place in the ring, in the
//               other of two register sets) and writes them where the copy expects them: for 128 rows and four blocks 512 bytes, row r
//               at (r % 32) * 16 + (r / 32) * 4, so four rows of a lane are one 16-byte store.  A
//               warp a stage keeps four stages' loads in flight.
// Warps 0 and 1 elect their thread (elect.sync): under lane == 0 each TMA and tcgen05 instruction took
// 75 to 130 cycles, and 8192 x 14336 x 4096 with its quantisation 454 us against 370.
// The scales of a stage have their own columns in tensor memory, as many sets as there are stages:
// a set is rewritten only after the commit that frees its stage, so no copy can overtake an MMA
// that still reads the set.
//
// Few tokens: the product is bound by reading b, and one tile per SM leaves SMs idle, so the
// reduction is split over a cluster of CTAs that exchange their partial sums through distributed
// shared memory and add them in the order of the ranks (no workspace, no atomics, the same bits
// every time).
// Every wait is bounded; where one runs out the error word is set and the affected outputs are NaN: the
// loaders, the scale warps and the MMA warp stop, and an epilogue warp that has given up walks the tasks
// that are left and writes NaN.  It arrives at no barrier of the pipeline any more, so no accumulator is
// overwritten under a warp that still reads it, and it meets the others at every barrier of theirs.
#pragma once
#include <atomic>

#include "mx4.cuh"
#include "tcgen05_utils.cuh"

namespace stmoe_dev {

constexpr int kMmThreads = 320;
constexpr int kMmRows = 128;              // rows of b in a tile (MMA M)
constexpr int kMmMaxTokens = 192;         // tokens in a tile (MMA N)
constexpr int kMmStageBlocks = 8;         // scale blocks of a stage (256 elements, 128 bytes of codes)
constexpr int kMmABytes = kMmRows * 128;
constexpr int kMmMaxStages = 12;
constexpr int kMmMaxSplits = 8;           // portable cluster size
constexpr int kMmMaxGroups = 256;
constexpr int kMmSmemBytes = 224 * 1024;  // dynamic; one CTA per SM
constexpr int kMmStageOut = 2048;         // epilogue: bytes of shared memory of a warp
constexpr int kMmAccStride = kMmMaxTokens;
constexpr int kMmScaleCol = 2 * kMmAccStride;   // scale sets start behind the accumulators

// rows of 128 tokens whose scales a stage copies, bytes and tensor-memory columns of a stage
__host__ __device__ constexpr int mm_token_atoms(int bn) { return (bn + 127) / 128; }
__host__ __device__ constexpr int mm_stage_bytes(int bn) { return kMmABytes + bn * 128 + 1024 + 1024 * mm_token_atoms(bn); }
__host__ __device__ constexpr int mm_scale_cols(int bn) { return 8 + 8 * mm_token_atoms(bn); }
__host__ __device__ constexpr int mm_slot_bytes(int bn) { return (mm_stage_bytes(bn) + 1023) / 1024 * 1024; }
__host__ __device__ constexpr int mm_stages(int bn)
{
    const int by_smem = (kMmSmemBytes - 1024 - 4 * kMmStageOut) / mm_slot_bytes(bn), by_tmem = (512 - kMmScaleCol) / mm_scale_cols(bn);
    const int n = by_smem < by_tmem ? by_smem : by_tmem;
    return n < kMmMaxStages ? n : kMmMaxStages;
}

// a scale warp waits for step i + 4 knowing that step i - NS has been consumed: with four stages or more
// it is never two phases ahead of a barrier, whose parity would then deceive it
static_assert(mm_stages(16) >= 4 && mm_stages(128) >= 4 && mm_stages(kMmMaxTokens) >= 4, "");

// Polls after which a wait gives up, for the launches to come (tests lower it).
inline std::atomic<int> g_mx4_polls{kDenseSpinLimit};

struct Mx4MatmulArgs {
    const uint8_t *a_scales, *b_scales;
    long long a_scale_stride, b_scale_stride;  // bytes
    const int *counts;      // [groups] rows of a per matrix of b, or nullptr
    int groups, m, n;
    int blocks;             // scale blocks of a row (reduction length / 32)
    int bn, splits;
    void *out;
    long long out_stride;   // elements
    bool out_wide;          // rows of out start on 16-byte boundaries
    unsigned *err;          // may be nullptr
    int a_align, b_align;   // what scale rows are aligned to: 8, 4 or 1 bytes
    int polls;              // limit of every wait
};

// mxf4 descriptor: e2m1 x e2m1, e8m0 scales, both K-major, M = 128, N = n; which half of a scale
// word (two blocks) the MMA takes, for both operands
__device__ __forceinline__ uint32_t umma_idesc_mxf4(int n, int half)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(kMmRows >> 7) << 27) |
           ((uint32_t)(2 * half) << 4) | ((uint32_t)(2 * half) << 29);
}
// from a whole warp, issued by the lane that `leader` names; a, b: low words of swizzled descriptors
__device__ __forceinline__ void umma_mxf4(bool leader, uint32_t tmem_d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sfa,
                                          uint32_t sfb, bool accumulate)
{
    asm volatile(
        "{.reg .pred p, q;\n\t"
        ".reg .b64 da, db;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "setp.ne.b32 p, %7, 0;\n\t"
        "mov.b64 da, {%2, %8};\n\t"
        "mov.b64 db, {%3, %8};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%1], da, db, %4, [%5], [%6], p;}"
        :
        : "r"((uint32_t)leader), "r"(tmem_d), "r"(a), "r"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate),
          "n"(kDescHighSw128)
        : "memory");
}
// 32 rows x 16 bytes of shared memory into four columns, repeated in each quarter of the lanes; low:
// low word of the descriptor
__device__ __forceinline__ void umma_copy_scales(bool leader, uint32_t tmem, uint32_t low)
{
    asm volatile(
        "{.reg .pred q;\n\t"
        ".reg .b64 d;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "mov.b64 d, {%2, %3};\n\t"
        "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%1], d;}" ::"r"((uint32_t)leader), "r"(tmem), "r"(low), "n"(kDescHighScales)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16])
{
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// Eight scale bytes, from block kb on, of G rows of a lane (row(r): address of row r's first scale; rows
// whose `on` bit is clear read nothing).  Blocks past the end read as 1.0: their codes are zero, and zero
// times a NaN scale would not be.  One branch around all loads, and the loads predicated inside: with a
// branch at each of them they waited for one another (11 cold loads, 8 us in front of the first MMA).
// Volatile, as the kernel before may have written the scales: the loads must stay behind pdl_wait (an
// __ldg or a plain asm may move across it).
__device__ __forceinline__ uint2 ld_scales8_if(bool on, const uint8_t *p)
{
    uint2 v;
    asm volatile("{.reg .pred p;\n\t"
        "setp.ne.b32 p, %3, 0;\n\t"
        "mov.b32 %0, 0x7f7f7f7f;\n\t"
        "mov.b32 %1, 0x7f7f7f7f;\n\t"
        "@p ld.global.nc.v2.u32 {%0, %1}, [%2];}"
        : "=&r"(v.x), "=&r"(v.y)
        : "l"(p), "r"((uint32_t)on));
    return v;
}
__device__ __forceinline__ uint32_t ld_scales4_if(bool on, const uint8_t *p)
{
    uint32_t v;
    asm volatile("{.reg .pred p;\n\t"
        "setp.ne.b32 p, %2, 0;\n\t"
        "mov.b32 %0, 0x7f7f7f7f;\n\t"
        "@p ld.global.nc.u32 %0, [%1];}"
        : "=&r"(v)
        : "l"(p), "r"((uint32_t)on));
    return v;
}
template <int G, typename Row>
__device__ __forceinline__ void load_scales(uint2 (&v)[G], Row row, uint32_t on, int kb, int blocks, int align)
{
    if (align == 8 && kb + 8 <= blocks) {
#pragma unroll
        for (int r = 0; r < G; ++r) v[r] = ld_scales8_if(on >> r & 1, row(r) + kb);
    } else if (align >= 4 && blocks % 4 == 0) {   // whole words, the second perhaps past the end
#pragma unroll
        for (int r = 0; r < G; ++r) {
            v[r].x = ld_scales4_if(on >> r & 1, row(r) + kb);
            v[r].y = ld_scales4_if((on >> r & 1) && kb + 4 < blocks, row(r) + kb + 4);
        }
    } else {
#pragma unroll
        for (int r = 0; r < G; ++r) {
            const uint8_t *p = row(r) + kb;
            uint32_t b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = (on >> r & 1) && kb + i < blocks ? (uint32_t)p[i] : 0x7fu;
            v[r] = make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
        }
    }
}
// What a lane has read of G row groups (rows lane, lane + 32, ...), into the atoms of 128 rows x four
// blocks: first half at st, second half of the stage's blocks `half` bytes behind it
template <int G> __device__ __forceinline__ void store_scales(uint8_t *st, int half, int lane, const uint2 (&v)[G])
{
#pragma unroll
    for (int a = 0; a < (G + 3) / 4; ++a) {
        uint32_t x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = 4 * a + i < G ? v[(4 * a + i) % G].x : 0u;   // (no index past the array, even unused)
            y[i] = 4 * a + i < G ? v[(4 * a + i) % G].y : 0u;
        }
        *reinterpret_cast<uint4 *>(st + 512 * a + 16 * lane) = make_uint4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint4 *>(st + half + 512 * a + 16 * lane) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

// Which rows a task multiplies.
struct Mx4Task {
    int expert, row0;      // matrix of b and its first row
    int tok0, count;       // first token and how many of the tile's are this expert's
};

// s_off: first token of every group (groups + 1 entries), s_tile: token tiles before it
__device__ __forceinline__ Mx4Task mm_task(const Mx4MatmulArgs &a, const int *s_off, const int *s_tile, int task)
{
    const int wt = (a.n + kMmRows - 1) / kMmRows;
    const int t = task / wt;  // which token tile the task would be if every group's came first
    int lo = 0, hi = a.groups - 1;
    while (lo < hi) {         // last group with s_tile[g] <= t and tiles of its own
        const int mid = (lo + hi + 1) / 2;
        if (s_tile[mid] <= t) lo = mid; else hi = mid - 1;
    }
    // a group's tasks: its row tiles, and for each of them its token tiles, so that a tile of b is
    // read by consecutive tasks
    const int tiles = s_tile[lo + 1] - s_tile[lo], r = task - s_tile[lo] * wt;
    Mx4Task k;
    k.expert = lo;
    k.row0 = (r / tiles) * kMmRows;
    k.tok0 = s_off[lo] + (r % tiles) * a.bn;
    k.count = min(a.bn, s_off[lo + 1] - k.tok0);
    return k;
}

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
// How many clusters of 2, 4 and 8 CTAs of a kernel run at a time: fewer than the SMs would suggest, as a
// cluster has to fit one of the GPU's processor clusters.
struct MmClusters {
    int fit[3];
};
template <typename... P> inline bool mm_clusters(void (*kernel)(P...), int threads, MmClusters *c)
{
    for (int i = 0; i < 3; ++i) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 2u << i, at[0].val.clusterDim.y = 1, at[0].val.clusterDim.z = 1;
        cfg.gridDim = dim3(2u << i), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = kMmSmemBytes;
        cfg.attrs = at, cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&c->fit[i], kernel, &cfg) != cudaSuccess) {
            (void)cudaGetLastError();
            return false;
        }
    }
    return true;
}
// Splits of a reduction of `steps` stages over a cluster, for `tasks` tiles: a power of two whose clusters
// all run at once, as long as the stages saved (0.26 us each, latency) outweigh the exchange (about
// 1 us).  Measured at 5 x 2816 outputs: reduction 2048 (8 stages) 6.1 us unsplit, 5.3 by 4; 16 x 512,
// reduction 14336: 17.3 and 7.0 by 8; 60 x 2048, reduction 2048, 16 clusters of 8 in two rounds: 6.6 and 12.4.
inline int mm_splits(int64_t tasks, int steps, const MmClusters &c)
{
    int best = 1;
    float cost = 0.26f * steps;
    for (int i = 0; i < 3; ++i) {
        const int z = 2 << i;
        const float t = 0.26f * ((steps + z - 1) / z) + 1.f;
        if (z <= steps && tasks <= c.fit[i] && t < cost) cost = t, best = z;
    }
    return best;
}

template <int ODT>
__global__ void __launch_bounds__(kMmThreads, 1)
mx4_matmul_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Mx4MatmulArgs a)
{
    using E = Elem<ODT>;
    extern __shared__ uint8_t dsm_raw[];
    __shared__ uint64_t full[kMmMaxStages], empty[kMmMaxStages], tfull[2], tempty[2];
    __shared__ int s_off[kMmMaxGroups + 1], s_tile[kMmMaxGroups + 1];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp;
    uint8_t *dsm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dsm_raw) + 1023) & ~(uintptr_t)1023);
    const int NS = mm_stages(a.bn), slot = mm_slot_bytes(a.bn), bn = a.bn;
    uint8_t *stage_out = dsm + NS * slot;
    const int sfa_at = kMmABytes + bn * 128, sfb_at = sfa_at + 1024, atoms = mm_token_atoms(bn);

    if (tid == 0) {
        s_dead = 0;
        for (int s = 0; s < NS; ++s) dmbar_init(&full[s], 2), dmbar_init(&empty[s], 1);
        for (int b = 0; b < 2; ++b) dmbar_init(&tfull[b], 1), dmbar_init(&tempty[b], 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dsmem_u32(&s_tmem)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();   // all that is read may be the kernel before's
    pdl_launch_dependents();
    if (warp == 2) {  // group offsets; a count that is negative or leaves the rows of a is cut
        int off = 0, tiles = 0;
        if (lane == 0) s_off[0] = s_tile[0] = 0;
        for (int g0 = 0; g0 < a.groups; g0 += kWarp) {
            const int g = g0 + lane;
            int c = g < a.groups ? (a.counts ? max(0, a.counts[g]) : a.m) : 0;
            c = min(c, a.m);
            long long at = c;
#pragma unroll
            for (int o = 1; o < kWarp; o <<= 1) {
                const long long t = __shfl_up_sync(kFull, at, o);
                if (lane >= o) at += t;
            }
            const int end = (int)min((long long)a.m, off + at);
            const int beg = (int)min((long long)a.m, off + at - c);
            int t = (end - beg + bn - 1) / bn;
#pragma unroll
            for (int o = 1; o < kWarp; o <<= 1) {
                const int u = __shfl_up_sync(kFull, t, o);
                if (lane >= o) t += u;
            }
            if (g < a.groups) s_off[g + 1] = end, s_tile[g + 1] = tiles + t;
            off = __shfl_sync(kFull, end, kWarp - 1);
            tiles += __shfl_sync(kFull, t, kWarp - 1);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int *dead = &s_dead;

    const int n_tasks = s_tile[a.groups] * ((a.n + kMmRows - 1) / kMmRows);
    const int rank = blockIdx.x % a.splits, first = blockIdx.x / a.splits, step = gridDim.x / a.splits;
    const int n_steps = (a.blocks + kMmStageBlocks - 1) / kMmStageBlocks;
    const int k_beg = (int)((long long)n_steps * rank / a.splits), k_end = (int)((long long)n_steps * (rank + 1) / a.splits);

    if (warp == 0) {
        if (elect_one()) {
            int s = 0, issued = 0;
            uint32_t par = 0;
            for (int task = first; task < n_tasks && !*dead; task += step) {
                const Mx4Task t = mm_task(a, s_off, s_tile, task);
                for (int k = k_beg; k < k_end; ++k, ++issued) {
                    if (!dmbar_wait(&empty[s], par ^ 1u, dead, a.polls)) break;
                    uint8_t *st = dsm + (size_t)s * slot;
                    dmbar_expect_tx(&full[s], (uint32_t)(kMmABytes + bn * 128));
                    tma_load_2d(st, &map_b, k * 128, t.expert * a.n + t.row0, &full[s]);
                    tma_load_2d(st + kMmABytes, &map_a, k * 128, t.tok0, &full[s]);
                    if (++s == NS) s = 0, par ^= 1u;
                }
            }
            // every load that was issued lands before the CTA may exit (the wait has an end of its own, as
            // the error word would cut it short; behind an error settle_in_flight has the last word)
            int none = 0;
            for (int i = 0; i < min(issued, NS); ++i) {
                if (s == 0) s = NS, par ^= 1u;
                --s;
                dmbar_wait(&full[s], par, &none, 1 << 14);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // the whole warp walks the loop, one lane issues
        const bool leader = elect_one();
        const uint32_t id0 = umma_idesc_mxf4(bn, 0), id1 = umma_idesc_mxf4(bn, 1);
        const int cols = mm_scale_cols(bn);
        const uint32_t ring = dsmem_u32(dsm);
        int s = 0, it = 0;
        uint32_t par = 0;
        bool ok = true;
        for (int task = first; task < n_tasks && ok; task += step, ++it) {
            const int ab = it & 1;
            if (!(ok = __all_sync(kFull, dmbar_wait(&tempty[ab], ((uint32_t)(it >> 1) & 1u) ^ 1u, dead, a.polls)))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + ab * kMmAccStride;
            for (int k = k_beg; k < k_end; ++k) {
                if (!(ok = __all_sync(kFull, dmbar_wait(&full[s], par, dead, a.polls)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t st = ring + s * slot;
                const uint32_t sf = tmem + kMmScaleCol + s * cols;  // this stage's set of scale columns
                const uint32_t da = desc_low_sw128(st), db = desc_low_sw128(st + kMmABytes);
                const uint32_t ds = desc_low_scales(st + sfa_at);   // 512 bytes a copy: 32 address units
#pragma unroll
                for (int q = 0; q < 2; ++q) {                       // four blocks each
                    umma_copy_scales(leader, sf + 4 * q, ds + 32 * q);
                    umma_copy_scales(leader, sf + 8 + 4 * q * atoms, ds + 64 + 32 * q * atoms);
                    if (atoms == 2) umma_copy_scales(leader, sf + 12 + 8 * q, ds + 96 + 64 * q);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    umma_mxf4(leader, acc, da + 2 * j, db + 2 * j, j & 1 ? id1 : id0, sf + 4 * (j / 2), sf + 8 + 4 * (j / 2) * atoms,
                              k > k_beg || j > 0);
                umma_commit_if(leader, &empty[s]);
                if (++s == NS) s = 0, par ^= 1u;
            }
            if (ok) umma_commit_if(leader, &tfull[ab]);
        }
        __syncwarp();
    } else if (warp < 6) {
        const int lg = warp % 4;  // the quarter of the lanes this warp may read
        int it = 0;
        bool ok = true;
        for (int task = first; task < n_tasks; task += step, ++it) {
            const int ab = it & 1;
            const Mx4Task t = mm_task(a, s_off, s_tile, task);
            ok = ok && __all_sync(kFull, dmbar_wait(&tfull[ab], (uint32_t)(it >> 1) & 1u, dead, a.polls));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + ab * kMmAccStride + ((uint32_t)(lg * kWarp) << 16);
            const int row = t.row0 + lg * kWarp + lane;
            if (a.splits == 1) {
                using T = typename E::T;
                T *out = reinterpret_cast<T *>(a.out) + (long long)t.tok0 * a.out_stride + (row - lane);
                if (a.out_wide && t.row0 + kMmRows <= a.n) {
                    // A lane has one column of out for every token.  Stored like that, 192 tokens are 192
                    // two-byte stores of a warp (17000 cycles, twice the tile's MMAs); through shared memory
                    // the four warps' 128 columns of a token become whole lines.
                    constexpr int kRow = kMmRows * (int)sizeof(T), kLanes = kRow / 16, kTok = 4 * kMmStageOut / kRow;  // 256 or 512 bytes a token
                    T *tile = reinterpret_cast<T *>(stage_out);
                    const int id = lg * kWarp + lane, tk = id / kLanes, piece = (id % kLanes) * (16 / (int)sizeof(T));
                    constexpr int kHop = 4 * kWarp / kLanes;   // tokens that the four warps store at a time
                    T *to = reinterpret_cast<T *>(a.out) + (long long)(t.tok0 + tk) * a.out_stride + t.row0 + piece;
                    for (int j0 = 0; j0 < t.count; j0 += kTok) {
#pragma unroll
                        for (int h = 0; h < kTok; h += 16) {
                            float v[16];
                            tmem_ld16(acc + j0 + h, v);
#pragma unroll
                            for (int j = 0; j < 16; ++j) tile[(h + j) * kMmRows + id] = E::from_f32(ok ? v[j] : __uint_as_float(0x7fffffffu));
                        }
                        asm volatile("bar.sync 2, 128;" ::: "memory");
#pragma unroll
                        for (int h = 0; h < kTok; h += kHop) {
                            if (j0 + h + tk < t.count)
                                *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(tile + (h + tk) * kMmRows + piece);
                            to += kHop * a.out_stride;
                        }
                        asm volatile("bar.sync 2, 128;" ::: "memory");
                    }
                } else {
                    T *to = out + lane;
                    for (int j0 = 0; j0 < t.count; j0 += 16) {
                        float v[16];
                        tmem_ld16(acc + j0, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            if (row < a.n && j0 + j < t.count) *to = E::from_f32(ok ? v[j] : __uint_as_float(0x7fffffffu));
                            to += a.out_stride;
                        }
                    }
                }
            } else {
                // the ring is idle once the last MMA has been committed: the partial tile takes its place
                // (NaN, where that was not waited for, once nothing can land on top of it)
                if (!ok) settle_in_flight();
                float *part = reinterpret_cast<float *>(dsm);
                for (int j0 = 0; j0 < bn; j0 += 16) {
                    float v[16];
                    tmem_ld16(acc + j0, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) part[(j0 + j) * kMmRows + lg * kWarp + lane] = ok ? v[j] : __uint_as_float(0x7fffffffu);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (ok && lane == 0) dmbar_arrive(&tempty[ab]);
        }
    } else {
        // scales: this warp's stages are the CTA's steps w, w + 4, ... across its tasks
        const int w = warp - 6, per_task = k_end - k_beg;
        int task = first, k = k_beg + w;   // step i of the CTA, and the next of this warp's
        Mx4Task t = {0, 0, 0, 0};
        if (first < n_tasks) t = mm_task(a, s_off, s_tile, first);
        auto load = [&](uint2 (&vb)[4], uint2 (&va)[6]) {
            bool entered = false;
            for (; task < n_tasks && k >= k_end; task += step) k -= per_task, entered = true;
            if (task >= n_tasks) return false;
            if (entered) t = mm_task(a, s_off, s_tile, task);
            const int kb = k * kMmStageBlocks;
            k += 4;
            const uint8_t *pb = a.b_scales + (long long)t.expert * a.n * a.b_scale_stride;
            load_scales<4>(vb, [&](int r) { return pb + (long long)min(t.row0 + 32 * r + lane, a.n - 1) * a.b_scale_stride; }, 15u, kb,
                           a.blocks, a.b_align);
            load_scales<6>(va, [&](int r) { return a.a_scales + (long long)min(t.tok0 + 32 * r + lane, a.m - 1) * a.a_scale_stride; },
                           (1u << ((bn + 31) / 32)) - 1, kb, a.blocks, a.a_align);
            return true;
        };
        uint32_t i = w;
        auto put = [&](const uint2 (&vb)[4], const uint2 (&va)[6]) {   // step i
            const int s = (int)(i % NS);
            if (!__all_sync(kFull, dmbar_wait(&empty[s], ((i / NS) & 1u) ^ 1u, dead, a.polls))) return false;   // its place may be in use
            uint8_t *st = dsm + (size_t)s * slot;
            store_scales<4>(st + sfa_at, 512, lane, vb);
            if (atoms == 1) {
                const uint2 v4[4] = {va[0], va[1], va[2], va[3]};
                store_scales<4>(st + sfb_at, 512, lane, v4);
            } else {
                store_scales<6>(st + sfb_at, 1024, lane, va);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) dmbar_arrive(&full[s]);
            i += 4;
            return true;
        };
        // two sets of registers in turn: copying one into the other would wait for its loads
        uint2 b0[4], a0[6], b1[4], a1[6];
        bool more = load(b0, a0);
        while (more) {
            const bool next = load(b1, a1);
            if (!put(b0, a0) || !next) break;
            more = load(b0, a0);
            if (!put(b1, a1)) break;
        }
    }
    if (a.splits > 1 && first < n_tasks) {  // one task per cluster, the same for all its CTAs
        __syncwarp();
        cluster_sync();
        const Mx4Task t = mm_task(a, s_off, s_tile, first);
        const uint32_t part = dsmem_u32(dsm);
        // a warp a token, four rows a lane; the ranks' loads are under way together
        using T = typename E::T;
        const int row = t.row0 + 4 * lane;
        for (int j = rank + a.splits * warp; j < t.count; j += a.splits * (kMmThreads / kWarp)) {
            float4 v[kMmMaxSplits];
#pragma unroll
            for (int z = 0; z < kMmMaxSplits; ++z)
                if (z < a.splits) v[z] = ld_cluster4(part + (uint32_t)(j * kMmRows + 4 * lane) * 4, z);
            float y[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
            for (int z = 1; z < kMmMaxSplits; ++z)
                if (z < a.splits) y[0] += v[z].x, y[1] += v[z].y, y[2] += v[z].z, y[3] += v[z].w;
            T *to = reinterpret_cast<T *>(a.out) + (long long)(t.tok0 + j) * a.out_stride + row;
            T q[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) q[r] = E::from_f32(y[r]);
            if (a.out_wide && row + 4 <= a.n) {
                if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(q);
                else *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(q);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (row + r < a.n) to[r] = q[r];
            }
        }
        cluster_sync();  // nobody leaves while its partial tile is read
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    if (tid == 0 && s_dead && a.err) *a.err = 1u;
}

}  // namespace stmoe_dev
