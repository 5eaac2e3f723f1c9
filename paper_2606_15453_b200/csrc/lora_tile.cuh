// The adapters' two products for many rows (lora.cuh has the formulas and the kernels for few): tiles of up to 128
// positions of one adapter on tcgen05.mma, accumulators in tensor memory.
//
//   lora_down_tile_kernel   D[128][r] = X A^T, one tile and one part of the inner dimension a CTA.  Rows of x are gathered through the
//                           grouping's order; four warps copy 64 inner elements a stage (cp.async into the 128-byte swizzled layout), one
//                           issues the MMAs.
//   lora_up_tile_kernel     D[128][128] = H B^T, H in 16-bit planes that lie one after the other in the inner dimension, the same
//                           B tile against each.  A CTA takes a run of (tile, columns) units, so that the planes are made once for most of
//                           its units.
//
// Both are the memory's work: x once, B and A once a tile, base and out once.  What the design has to keep up is bytes in flight.  In the
// first that is stages of x, two CTAs an SM.  In the second the base's rows come by asynchronous copies into a ring of units in shared
// memory, three units ahead of the one in work, so that they cost neither registers nor waits (8192 rows, 4096 -> 14336: with the rows in
// the registers of eight warps and two CTAs an SM 215 us, spills and all; as a bulk copy of 256 bytes a row 265 us, a lane's bulk copy
// taking some 75 cycles to issue; like this 106 us).  Two sets of four warps take units in turn.  B's rows are permuted on their way to
// shared memory so that a lane finds sixteen neighbouring outputs in its accumulator registers and stores them at once.
// Rows that are not 16-byte aligned go another way: the sums pass through the same shared memory in fp32, and each warp adds and stores
// its rows element by element, lanes side by side.
#pragma once
#include <atomic>

#include "lora.cuh"

namespace stmoe_dev {

constexpr int kTileRows = 128, kTileMaxRank = 128;
constexpr int kDownMaxSplits = 8;          // parts of the inner dimension: a portable cluster
constexpr int kDownTileThreads = 160;       // warps 0-3 copy and store, warp 4 issues
constexpr int kUpTileThreads = 416;         // warps 0-7 add and store, 8-11 copy B and the base, 12 issues
constexpr int kUpRowBytes = 256, kUpPitch = kUpRowBytes + 16;   // of a unit's row, and from one to the next in shared memory
constexpr int kUnitBytes = kTileRows * kUpPitch;
constexpr int kCopyWarps = 4;
constexpr int kSlabBytes = kTileRows * 128; // 128 rows of 64 inner elements

__host__ __device__ constexpr int lora_r16(int r) { return (r + 15) / 16 * 16; }
__host__ __device__ constexpr int lora_slabs(int r) { return (r + 63) / 64; }
__host__ __device__ constexpr int down_stage_bytes(int r) { return kSlabBytes + (lora_r16(r) * 128 + 1023) / 1024 * 1024; }
__host__ __device__ constexpr int down_stages(int r) { return 96 * 1024 / down_stage_bytes(r); }
// outputs of a unit (128 16-bit or 64 fp32 ones), bytes of a B tile, B tiles and units in shared memory (an even number, so that a set of
// warps keeps its own)
template <int DO> __host__ __device__ constexpr int up_cols() { return kUpRowBytes / (DO == 0 ? 4 : 2); }
template <int DO> __host__ __device__ constexpr int up_b_bytes(int r) { return lora_slabs(r) * up_cols<DO>() * 128; }
__host__ __device__ constexpr int up_stages(int r) { return lora_slabs(r) == 1 ? 3 : 2; }
__host__ __device__ constexpr int up_units(int r) { return lora_slabs(r) == 1 ? 4 : 2; }
template <int DO, int PL> __host__ __device__ constexpr int up_smem(int r)
{
    return 1024 + PL * lora_slabs(r) * kSlabBytes + up_stages(r) * up_b_bytes<DO>(r) + up_units(r) * kUnitBytes;
}
static_assert(up_smem<1, 2>(64) <= 227 * 1024 && up_smem<1, 2>(128) <= 227 * 1024 && up_smem<0, 3>(64) <= 227 * 1024 && up_smem<0, 3>(128) <= 227 * 1024, "");

// 16-bit operands of one type (DT) -> fp32, both K-major, M = 128
template <int DT> __host__ __device__ constexpr uint32_t umma_idesc_16(int n)
{
    constexpr uint32_t t = DT == 1 ? 1 : 0;
    return (1u << 4) | (t << 7) | (t << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
}
// from a whole warp, by the lane that `leader` names
__device__ __forceinline__ void umma_16(bool leader, uint32_t tmem_d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile(
        "{.reg .pred p, q;\n\t"
        "setp.ne.b32 q, %0, 0;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], %2, %3, %4, p;}" ::"r"((uint32_t)leader),
        "r"(tmem_d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// Sixteen lanes by 64 columns of tensor memory: register 4 j + i holds column 8 j + 2 (lane % 4) + i % 2 of lane lane / 4 + 8 (i / 2).
__device__ __forceinline__ void tmem_ld_16x64(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
        "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}

// First tile of every adapter (s_tile[n]: of the rows without one, s_tile[n + 1]: all), by the first 128 threads, eight adapters each.
__device__ __forceinline__ void lora_tiles(const LoraArgs &a, int *s_tile, int *s_sum)
{
    constexpr int kEach = kLoraMaxAdapters / 128;
    const int tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp;
    int mine[kEach], all = 0, up = 0;
    if (tid < 128) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int g = tid * kEach + i;
            mine[i] = g < a.n ? (min(max(a.counts[g], 0), a.T) + kTileRows - 1) / kTileRows : 0;
            all += mine[i];
        }
        up = all;
#pragma unroll
        for (int o = 1; o < kWarp; o <<= 1) {
            const int t = __shfl_up_sync(kFull, up, o);
            if (lane >= o) up += t;
        }
        if (lane == kWarp - 1) s_sum[warp] = up;
    }
    __syncthreads();
    if (tid < 128) {
        int at = up - all;
        for (int w = 0; w < warp; ++w) at += s_sum[w];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int g = tid * kEach + i;
            if (g <= a.n) s_tile[g] = at;       // [n]: behind the last adapter's
            at += mine[i];
        }
    }
    if (tid == 0 && a.n == kLoraMaxAdapters) s_tile[a.n] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    __syncthreads();
    if (tid == 0) s_tile[a.n + 1] = s_tile[a.n] + (a.T - min(max(a.starts[a.n], 0), a.T) + kTileRows - 1) / kTileRows;
    __syncthreads();
}
struct LoraTile {
    int g, begin, count;        // adapter (n: none), first position, positions
};
__device__ __forceinline__ LoraTile lora_tile_at(const LoraArgs &a, const int *s_tile, int t)
{
    int lo = 0, hi = a.n;       // last g with s_tile[g] <= t
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (s_tile[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int at = (t - s_tile[lo]) * kTileRows, begin = min(max(a.starts[lo], 0), a.T);
    const int all = lo < a.n ? a.counts[lo] : a.T - begin;
    return {lo, begin + at, max(0, min(min(kTileRows, all - at), a.T - begin - at))};
}

// Eight elements of a row (zeros behind its end) into shared memory: in flight until the group is waited for where rows are aligned.
template <int DT, bool VEC> __device__ __forceinline__ void put8(uint32_t dst, const typename Elem<DT>::T *row, int k, int n, bool on)
{
    if constexpr (VEC) {
        const bool some = on && k < n;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(some ? row + k : row), "r"(some ? 16 : 0) : "memory");
    } else {
        const uint4 q = lora_load8<DT, false>(row, k, n, on);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
    }
}
// place of 16-byte piece c of row i in a slab
__device__ __forceinline__ uint32_t slab_at(int i, int c) { return i * 128 + ((c ^ (i & 7)) << 4); }

__device__ __forceinline__ void tmem_alloc(int *s_tmem, int cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dsmem_u32(s_tmem)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, int cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
}

template <int DT, bool XVEC, bool WVEC> __global__ void __launch_bounds__(kDownTileThreads, 2) lora_down_tile_kernel(const LoraArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int kLag = 2;                 // stages that a copying warp leaves in flight behind the one it issues
    constexpr int kMaxStages = 5;
    extern __shared__ uint8_t dsm_raw[];
    __shared__ int s_tile[kLoraMaxAdapters + 2], s_sum[4], s_tmem, s_row[kTileRows];
    __shared__ int s_dead;
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], done;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp;
    const int r16 = lora_r16(a.r), NS = down_stages(a.r), slot = down_stage_bytes(a.r);
    int cols = 32;
    while (cols < r16) cols *= 2;
    if (!a.early) pdl_wait();
    lora_tiles(a, s_tile, s_sum);
    if (a.early) pdl_wait();
    pdl_launch_dependents();
    // the parts of a tile's inner dimension are a cluster
    const int rank = blockIdx.x % a.splits, from = rank * a.steps, to = min(from + a.steps, (a.I + 63) / 64);
    if ((int)blockIdx.x / a.splits >= s_tile[a.n]) return;
    const LoraTile t = lora_tile_at(a, s_tile, blockIdx.x / a.splits);
    uint8_t *const dsm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dsm_raw) + 1023) & ~(uintptr_t)1023);
    if (tid == 0) {
        s_dead = 0;
        for (int s = 0; s < NS; ++s) dmbar_init(&full[s], 4), dmbar_init(&empty[s], 1);
        dmbar_init(&done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid < kTileRows) s_row[tid] = tid < t.count ? lora_row(a, t.begin + tid) : -1;
    if (warp == 4) tmem_alloc(&s_tmem, cols);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int *const dead = &s_dead;
    const int n = to - from;
    bool ok = true;
    if (warp < 4) {
        // eight lanes a row: piece c of rows tid / 8 + 16 j.  Rows that the tile does not have keep what was there: a row of D depends on its own
        // row of x alone, and is not stored.
        const int c = tid % 8, i0 = tid / 8;
        const T *const x = reinterpret_cast<const T *>(a.x);
        const T *const w = reinterpret_cast<const T *>(a.a) + t.g * a.a_group;
        const T *rows[kTileRows / 16];
#pragma unroll
        for (int j = 0; j < kTileRows / 16; ++j) {
            const int row = s_row[i0 + 16 * j];
            rows[j] = row >= 0 ? x + row * a.x_stride : nullptr;
        }
        auto arrive = [&](int s) {          // what this warp wrote into the stage is there
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) dmbar_arrive(&full[s]);
        };
        int s = 0, par = 0, ready = 0;
        for (int i = 0; i < n; ++i) {
            if (!(ok = __all_sync(kFull, dmbar_wait(&empty[s], par ^ 1, dead, a.polls)))) break;
            const uint32_t st = dsmem_u32(dsm) + s * slot;
            const int k = (from + i) * 64 + c * 8;
#pragma unroll
            for (int j = 0; j < kTileRows / 16; ++j)
                if (rows[j]) put8<DT, XVEC>(st + slab_at(i0 + 16 * j, c), rows[j], k, a.I, true);
            for (int r = i0; r < r16; r += 16) put8<DT, WVEC>(st + kSlabBytes + slab_at(r, c), w + (r < a.r ? r : 0) * a.a_row, k, a.I, r < a.r);
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (i >= kLag) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kLag) : "memory");
                arrive(ready);
                if (++ready == NS) ready = 0;
            }
            if (++s == NS) s = 0, par ^= 1;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (ok)
            for (int i = max(0, n - kLag); i < n; ++i) {
                arrive(ready);
                if (++ready == NS) ready = 0;
            }
        ok = ok && __all_sync(kFull, dmbar_wait(&done, 0, dead, a.polls));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        // a thread a position: one part goes to memory, several to shared memory, where every stage has been read.  Should a wait have run out, a
        // warp that is still copying would write over the others' NaN: all four are behind their copies first.
        if (a.splits > 1) asm volatile("bar.sync 1, 128;" ::: "memory");
        const int i = warp * kWarp + lane;
        float *const to_row = a.splits == 1 ? a.part + (long long)(t.begin + i) * a.rp : reinterpret_cast<float *>(dsm) + i * (r16 + 4);
        for (int r = 0; r < a.rp; r += 8) {
            float v[8];
            if (ok) tmem_ld8(tmem + ((uint32_t)(warp * kWarp) << 16) + r, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = ok ? v[j] : NAN;
            if (i < t.count) {
                *reinterpret_cast<float4 *>(to_row + r) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(to_row + r + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
        }
    } else {
        const bool leader = elect_one();
        const uint32_t idesc = umma_idesc_16<DT>(r16);
        int s = 0, par = 0;
        for (int i = 0; i < n && ok; ++i) {
            if (!(ok = __all_sync(kFull, dmbar_wait(&full[s], par, dead, a.polls)))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t st = dsmem_u32(dsm) + s * slot;
#pragma unroll
            for (int j = 0; j < 4; ++j) umma_16(leader, tmem, umma_desc_sw128(st, j), umma_desc_sw128(st + kSlabBytes, j), idesc, i > 0 || j > 0);
            umma_commit_if(leader, &empty[s]);
            if (++s == NS) s = 0, par ^= 1;
        }
        if (ok) umma_commit_if(leader, &done);
    }
    if (a.splits > 1) {
        __syncwarp();
        cluster_sync();
        const int pieces = a.rp / 4;
        for (int e = rank * kDownTileThreads + tid; e < t.count * pieces; e += a.splits * kDownTileThreads) {
            const int i = e / pieces, r = e % pieces * 4;
            const uint32_t at = dsmem_u32(dsm) + (i * (r16 + 4) + r) * 4;
            float4 v[kDownMaxSplits];
#pragma unroll
            for (int z = 0; z < kDownMaxSplits; ++z)
                if (z < a.splits) v[z] = ld_cluster4(at, z);
#pragma unroll
            for (int z = 1; z < kDownMaxSplits; ++z)
                if (z < a.splits) v[0].x += v[z].x, v[0].y += v[z].y, v[0].z += v[z].z, v[0].w += v[z].w;
            *reinterpret_cast<float4 *>(a.part + (long long)(t.begin + i) * a.rp + r) = v[0];
        }
        cluster_sync();                     // nobody leaves while its part is read
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 4) tmem_free(tmem, cols);
}

// ROWS rows of B, r16 ranks each, by the copying warps together: LP lanes a row.  PERM: row 16 q + 2 j + b of each 64 stands at 8 j + 2 q + b, so
// that the accumulator's lanes (tmem_ld_16x64) hold sixteen neighbouring outputs.
template <int DT, bool WVEC, bool PERM, int ROWS, int LP>
__device__ __forceinline__ void put_unit(const LoraArgs &a, uint32_t st, const typename Elem<DT>::T *w, int row0, int warp, int lane)
{
    constexpr int kRows = kWarp / LP;
    const int c = lane % LP, n0 = warp * (ROWS / kCopyWarps) + lane / LP;
    if (c * 8 >= lora_r16(a.r)) return;
    const typename Elem<DT>::T *row = w + (long long)(row0 + n0) * a.b_row;
    const int left = a.O - row0 - n0;
    auto place = [](int n) { return PERM ? (n & 64) | (n & 14) << 2 | (n & 48) >> 3 | (n & 1) : n; };
    const int at0 = place(n0);
#pragma unroll
    for (int i = 0; i < ROWS / kCopyWarps; i += kRows)       // n0 and i take different bits
        put8<DT, WVEC>(st + (c / 8) * ROWS * 128 + slab_at(at0 | place(i), c % 8), i < left ? row + (long long)i * a.b_row : w, c * 8, a.r, i < left);
}

// DO: type of base and out.  PL: planes of h.  WVEC: rows of B are 16-byte aligned; OVEC: rows of base and out.
template <int DT, int DO, int PL, bool WVEC, bool OVEC> __global__ void __launch_bounds__(kUpTileThreads, 1) lora_up_tile_kernel(const LoraArgs a)
{
    using T = typename Elem<DT>::T;
    using TO = typename Elem<DO>::T;
    constexpr int kStages = 3, kUnits = 4, kCols = up_cols<DO>(), kTmem = 4 * kCols;    // two accumulators a set
    extern __shared__ uint8_t dsm_raw[];
    __shared__ int s_tile[kLoraMaxAdapters + 2], s_sum[4], s_tmem;
    __shared__ float s_factor[kTileRows];
    __shared__ int s_dead;
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], tfull[4], tempty[4], planes, bfull[kUnits], bfree[kUnits];
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp;
    const int slabs = lora_slabs(a.r), r16 = lora_r16(a.r), NS = up_stages(a.r), NU = up_units(a.r);
    lora_tiles(a, s_tile, s_sum);
    // units of this CTA: whole tiles' columns, tile after tile
    const int per_tile = (a.O + kCols - 1) / kCols;
    const int units = s_tile[a.keep && !a.hidden ? a.n : a.n + 1] * per_tile;      // < 2^31: checked by the host
    const int first = (int)((long long)units * blockIdx.x / gridDim.x), count = (int)((long long)units * (blockIdx.x + 1) / gridDim.x) - first;
    if (count <= 0) {
        pdl_wait();
        return;
    }
    uint8_t *const dsm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dsm_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t h_at = dsmem_u32(dsm), b_at = h_at + PL * slabs * kSlabBytes;
    uint8_t *const units_at = dsm + PL * slabs * kSlabBytes + NS * up_b_bytes<DO>(a.r);
    if (tid == 0) {
        s_dead = 0;
        for (int s = 0; s < NS; ++s) dmbar_init(&full[s], kCopyWarps * kWarp), dmbar_init(&empty[s], 1);
        for (int b = 0; b < 4; ++b) dmbar_init(&tfull[b], 1), dmbar_init(&tempty[b], 4);
        for (int s = 0; s < NU; ++s) dmbar_init(&bfull[s], kCopyWarps * kWarp), dmbar_init(&bfree[s], 4);
        dmbar_init(&planes, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tmem_alloc(&s_tmem, kTmem);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int *const dead = &s_dead;
    int tile = first / per_tile, col = first % per_tile;
    bool fresh = true;                       // the unit begins a tile (or the run)
    LoraTile t = lora_tile_at(a, s_tile, tile);
    auto step = [&](int u) {                 // to the unit behind u
        fresh = false;
        if (u + 1 < count && ++col == per_tile) {
            col = 0, ++tile, fresh = true;
            t = lora_tile_at(a, s_tile, tile);
        }
    };
    const TO *const base = reinterpret_cast<const TO *>(a.base);
    TO *const out = reinterpret_cast<TO *>(a.out);
    if (warp < 8) {
        const int set = warp / 4, i = tid % kTileRows;      // set u % 2 takes unit u; thread i its position i
        bool ok = true;
        uint32_t used = 0;                                   // units that this set took from the tensor cores
        int row = -1;
        // OVEC: a lane's four rows are o + 8 j + 16 h of its warp's 32, where its sixteen outputs of each 64 begin at 16 q
        const int q = lane % 4, o = lane / 4;
        TO *to[2][2];
        pdl_wait();                                          // h is the kernel before's
        pdl_launch_dependents();
        for (int u = 0; u < count; step(u), ++u) {
            const bool some = t.g < a.n;
            if (fresh) {
                row = i < t.count ? lora_row(a, t.begin + i) : -1;
                if (OVEC) {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int of = __shfl_sync(kFull, some || !a.keep ? row : -1, h * 16 + j * 8 + o);
                            to[h][j] = of >= 0 ? out + of * a.out_stride + q * 16 : nullptr;
                        }
                }
                if (some) {
                    // both sets are behind the tile before, so its MMAs have read the planes.  16 or 32 lanes a position, four ranks each; eight
                    // positions' loads under way together
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    const int lanes = slabs * 16, rows = 256 / lanes, k = tid % lanes * 4;
                    const float c = a.alpha * (a.scale ? a.scale[t.g] : 1.f);
                    for (int i0 = tid / lanes; i0 < kTileRows; i0 += 8 * rows) {
                        float4 sum[8];
                        const float *const p = a.part + (long long)(t.begin + i0) * a.rp + k;
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            sum[j] = i0 + j * rows < t.count && k < a.rp ? ld_f4(p + j * rows * a.rp) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int pos = i0 + j * rows;
                            float f[4] = {sum[j].x, sum[j].y, sum[j].z, sum[j].w}, up = 1.f;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (k + e >= a.r) f[e] = 0.f;
                            if (DT != 1) {
                                float most = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
                                for (int s = lanes / 2; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, s));
                                up = plane_scale<DT>(most);
                            }
                            uint16_t pl[4][PL];
#pragma unroll
                            for (int e = 0; e < 4; ++e) planes_of<DT, PL>(f[e] * up, pl[e]);
#pragma unroll
                            for (int e = 0; e < PL; ++e)
                                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(h_at + (e * slabs + k / 64) * kSlabBytes + slab_at(pos, k % 64 / 8) + k % 8 * 2),
                                             "r"(pl[0][e] | (uint32_t)pl[1][e] << 16), "r"(pl[2][e] | (uint32_t)pl[3][e] << 16) : "memory");
                            if (k == 0) s_factor[pos] = c / up;
                            if (a.hidden && col == 0 && pos < t.count) {
                                const int to = lora_row(a, t.begin + pos);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (to >= 0 && k + e < a.r) a.hidden[(long long)to * a.r + k + e] = f[e];
                            }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (lane == 0) dmbar_arrive(&planes);
                } else if (a.hidden && col == 0 && set == 0 && row >= 0) {
                    for (int r = 0; r < a.r; ++r) a.hidden[(long long)row * a.r + r] = 0.f;
                }
            }
            if ((u & 1) != set) continue;
            const int o0 = col * kCols, here = min(kCols, a.O - o0), slot = u % NU;
            uint8_t *const unit = units_at + slot * kUnitBytes;
            const bool write = row >= 0 && (some || !a.keep);
            const int ab = set * 2 + (used & 1);
            if (some) {
                ok = ok && __all_sync(kFull, dmbar_wait(&tfull[ab], used >> 1 & 1, dead, a.polls));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                ++used;
            }
            if (OVEC && base) ok = ok && __all_sync(kFull, dmbar_wait(&bfull[slot], u / NU & 1, dead, a.polls));
            const uint32_t acc = tmem + ((uint32_t)(i / kWarp * kWarp) << 16) + ab * kCols;
            auto taken = [&] {                              // the accumulator has been read
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) dmbar_arrive(&tempty[ab]);
            };
            if (!ok) {                                       // a wait ran out: what depends on it is NaN
                if (write)
                    for (int c = 0; c < here; ++c)
                        out[row * a.out_stride + o0 + c] = some ? Elem<DO>::from_f32(NAN) : base ? base[row * a.base_stride + o0 + c] : Elem<DO>::from_f32(0.f);
            } else if constexpr (OVEC) {
                constexpr int V = Elem<DO>::kVec, G = 16 / V;
                const uint8_t *const was = unit + (i / kWarp * kWarp + o) * kUpPitch + q * 16 * (int)sizeof(TO);
                const float fs[2][2] = {{some ? s_factor[i / kWarp * kWarp + o] : 0.f, some ? s_factor[i / kWarp * kWarp + o + 8] : 0.f},
                                        {some ? s_factor[i / kWarp * kWarp + o + 16] : 0.f, some ? s_factor[i / kWarp * kWarp + o + 24] : 0.f}};
#pragma unroll
                for (int c = 0; c < kCols; c += 64)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t d[32];
                        if (some) tmem_ld_16x64(acc + ((uint32_t)(h * 16) << 16) + c, d);
                        uint4 v[2][G];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int g = 0; g < G; ++g)
                                v[j][g] = base ? *reinterpret_cast<const uint4 *>(was + (h * 16 + j * 8) * kUpPitch + c * (int)sizeof(TO) + g * 16) : make_uint4(0, 0, 0, 0);
                        if (some) tmem_ld_wait();
                        if (c + 64 == kCols && h == 1) {     // the accumulator and the base have been read
                            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                            __syncwarp();
                            if (lane == 0 && some) dmbar_arrive(&tempty[ab]);
                            if (lane == 0) dmbar_arrive(&bfree[slot]);
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int g = 0; g < G; ++g) {
                                float x[V];
                                bal_widen<DO>(v[j][g], reinterpret_cast<float2 *>(x));
                                if (some) {
#pragma unroll
                                    for (int e = 0; e < V; ++e) {
                                        const int n = g * V + e;          // output 16 q + n: column 8 (n / 2) + 2 q + n % 2
                                        x[e] = fmaf(fs[h][j], __uint_as_float(d[n / 2 * 4 + j * 2 + n % 2]), x[e]);
                                    }
                                }
                                if (to[h][j] && c + q * 16 + g * V < here)
                                    *reinterpret_cast<uint4 *>(to[h][j] + o0 + c + g * V) = bal_narrow<DO>(reinterpret_cast<const float2 *>(x));
                            }
                    }
            } else {
                const float f = some ? s_factor[i] : 0.f;
                // 64 columns at a time: a thread leaves its row's products as fp32, then each warp adds and stores its 32 rows
                constexpr int kPitch = 65;
                float *const sums = reinterpret_cast<float *>(unit);
                static_assert(kTileRows * kPitch * 4 <= kUnitBytes, "");
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += 64) {
                    __syncwarp();
                    if (some) {
#pragma unroll
                        for (int c = 0; c < 64; c += 32) {
                            uint32_t d[4][8];
#pragma unroll
                            for (int j = 0; j < 4; ++j) tmem_ld8_start(acc + c0 + c + j * 8, d[j]);
                            tmem_ld_wait();
                            if (c0 + c + 32 == kCols) taken();
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                sums[i * kPitch + c + j] = f * __uint_as_float(d[j / 8][j % 8]);
                        }
                    }
                    __syncwarp();
                    const int left = here - c0;             // columns: lane and lane + 32
                    for (int r0 = 0; r0 < kWarp; r0 += 8) {
                        float v[8][2];
                        int at[8];
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            at[r] = __shfl_sync(kFull, write ? row : -1, r0 + r);
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                v[r][h] = base && at[r] >= 0 && lane + h * kWarp < left ? Elem<DO>::to_f32(base[at[r] * a.base_stride + o0 + c0 + lane + h * kWarp]) : 0.f;
                        }
#pragma unroll
                        for (int r = 0; r < 8; ++r)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const float s = some ? sums[(i / kWarp * kWarp + r0 + r) * kPitch + lane + h * kWarp] : 0.f;
                                if (at[r] >= 0 && lane + h * kWarp < left) out[at[r] * a.out_stride + o0 + c0 + lane + h * kWarp] = Elem<DO>::from_f32(v[r][h] + s);
                            }
                    }
                }
            }
        }
    } else if (warp < 8 + kCopyWarps) {
        // The base: 32 rows a warp, two at a time, sixteen lanes each: where this lane's come from (their first output), or nullptr.  Kept as
        // addresses: made anew for every unit they took 130 cycles a copy, which was the whole kernel's time (230 us).
        const int mine = warp - 8, piece = lane % 16, elem = piece * Elem<DO>::kVec, row0 = mine * kWarp + lane / 16;
        const TO *from[kWarp / 2];
        int s = 0, par = 0, ahead = -1;
        for (int u = 0; u < count; step(u), ++u) {
            const int slot = u % NU, o0 = col * kCols;
            if (t.g < a.n) {
                if (!__all_sync(kFull, dmbar_wait(&empty[s], par ^ 1, dead, a.polls))) break;
                const T *const w = reinterpret_cast<const T *>(a.b) + t.g * a.b_group;
                const uint32_t st = b_at + s * up_b_bytes<DO>(a.r);
                if (r16 <= 16) put_unit<DT, WVEC, OVEC, kCols, 2>(a, st, w, o0, mine, lane);
                else if (r16 <= 32) put_unit<DT, WVEC, OVEC, kCols, 4>(a, st, w, o0, mine, lane);
                else if (r16 <= 64) put_unit<DT, WVEC, OVEC, kCols, 8>(a, st, w, o0, mine, lane);
                else put_unit<DT, WVEC, OVEC, kCols, 16>(a, st, w, o0, mine, lane);
                if (WVEC) asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(dsmem_u32(&full[s])) : "memory");
                else dmbar_arrive(&full[s]);
                if (++s == NS) s = 0, par ^= 1;
            }
            if (!base) continue;
            if constexpr (!OVEC) {
                // the base is read by the warps that add, element by element: here it is asked into L2, a lane a row
                if (fresh) {
                    const int i = mine * kWarp + lane;
                    ahead = i < t.count && (t.g < a.n || !a.keep) ? lora_row(a, t.begin + i) : -1;
                }
                if (ahead >= 0) {
                    const TO *const p = base + ahead * a.base_stride + o0;
                    const int last = min(kCols, a.O - o0) - 1;
                    prefetch_l2(p), prefetch_l2(p + min(last, kCols / 2)), prefetch_l2(p + last);
                }
                continue;
            }
            if (fresh) {
#pragma unroll
                for (int r = 0; r < kWarp / 2; ++r) {
                    const int i = row0 + 2 * r, row = i < t.count && (t.g < a.n || !a.keep) ? lora_row(a, t.begin + i) : -1;
                    from[r] = row >= 0 ? base + row * a.base_stride + elem : nullptr;
                }
            }
            if (!__all_sync(kFull, dmbar_wait(&bfree[slot], ((u / NU) & 1) ^ 1, dead, a.polls))) break;
            const uint32_t at = dsmem_u32(units_at) + slot * kUnitBytes + row0 * kUpPitch + piece * 16;
#pragma unroll
            for (int r = 0; r < kWarp / 2; ++r)
                if (from[r] && o0 + elem < a.O)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + r * 2 * kUpPitch), "l"(from[r] + o0) : "memory");
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(dsmem_u32(&bfull[slot])) : "memory");
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        const bool leader = elect_one();
        const uint32_t idesc = umma_idesc_16<DT>(kCols);
        bool ok = true;
        int s = 0, par = 0;
        uint32_t tiles = 0, used[2] = {0, 0};
        for (int u = 0; u < count && ok; step(u), ++u) {
            if (t.g >= a.n) continue;
            if (fresh) ok = __all_sync(kFull, dmbar_wait(&planes, tiles++ & 1, dead, a.polls));
            const uint32_t n = u & 1 ? used[1]++ : used[0]++;
            const int ab = (u & 1) * 2 + (n & 1);
            ok = ok && __all_sync(kFull, dmbar_wait(&tempty[ab], (n >> 1 & 1) ^ 1, dead, a.polls));
            ok = ok && __all_sync(kFull, dmbar_wait(&full[s], par, dead, a.polls));
            if (!ok) break;
            // B was copied by ordinary accesses, the tensor cores read through the asynchronous proxy
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t st = b_at + s * up_b_bytes<DO>(a.r);
            for (int p = 0; p < PL; ++p)
                for (int k = 0; k < r16; k += 16)
                    umma_16(leader, tmem + ab * kCols, umma_desc_sw128(h_at + (p * slabs + k / 64) * kSlabBytes, k % 64 / 16),
                            umma_desc_sw128(st + k / 64 * (kCols * 128), k % 64 / 16), idesc, p > 0 || k > 0);
            umma_commit_if(leader, &empty[s]);
            umma_commit_if(leader, &tfull[ab]);
            if (++s == NS) s = 0, par ^= 1;
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 12) tmem_free(tmem, kTmem);
}

}  // namespace stmoe_dev
