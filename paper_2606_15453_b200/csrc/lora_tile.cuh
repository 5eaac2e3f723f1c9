// The adapters' two products for many rows (lora.cuh has the formulas and the kernels for few): tiles of up to 128
// positions of one adapter on tcgen05.mma, accumulators in tensor memory.
//
//   lora_down_tile_kernel   D[128][r] = X A^T, one tile and one part of the inner dimension a CTA.  Rows of x are gathered through the
//                           grouping's order; four warps copy 64 inner elements a stage (cp.async into the 128-byte swizzled layout), one
//                           issues the MMAs.
//   lora_up_tile_kernel     D[128][128] = H B^T, H in 16-bit planes that lie one after the other in the inner dimension, the same
//                           B tile against each.  A CTA takes a run of (tile, 128 outputs) units, so that the planes are made once for
//                           most of its units; eight warps add the base and store, one copies B tiles, one issues the MMAs.
//
// Both are the memory's work: x once, B and A once a tile, base and out once.  What the design has to keep up is bytes in
// flight: stages of x in the first, the base's rows in the registers of eight warps, asked for before the accumulator is waited for, in
// the second, and two CTAs an SM in both.
#pragma once
#include <atomic>

#include "lora.cuh"

namespace stmoe_dev {

constexpr int kTileRows = 128, kTileMaxRank = 128;
constexpr int kDownTileThreads = 160;       // warps 0-3 copy and store, warp 4 issues
constexpr int kUpTileThreads = 320;         // warps 0-7 store, 8 copies, 9 issues
constexpr int kUpCols = 128;                // outputs of a unit
constexpr int kSlabBytes = kTileRows * 128; // 128 rows of 64 inner elements

__host__ __device__ constexpr int lora_r16(int r) { return (r + 15) / 16 * 16; }
__host__ __device__ constexpr int lora_slabs(int r) { return (r + 63) / 64; }
__host__ __device__ constexpr int down_stage_bytes(int r) { return kSlabBytes + (lora_r16(r) * 128 + 1023) / 1024 * 1024; }
__host__ __device__ constexpr int down_stages(int r) { return 96 * 1024 / down_stage_bytes(r); }
__host__ __device__ constexpr int up_stages(int r) { return lora_slabs(r) == 1 ? 3 : 2; }
__host__ __device__ constexpr int up_smem(int r, int planes) { return 1024 + (planes + up_stages(r)) * lora_slabs(r) * kSlabBytes; }

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
__device__ __forceinline__ void tmem_ld_16x64(uint32_t addr, float (&v)[32])
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
        "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
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
    pdl_wait();
    pdl_launch_dependents();
    lora_tiles(a, s_tile, s_sum);
    const int from = blockIdx.y * a.steps, to = min(from + a.steps, (a.I + 63) / 64);
    if ((int)blockIdx.x >= s_tile[a.n] || from >= to) return;
    const LoraTile t = lora_tile_at(a, s_tile, blockIdx.x);
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
        // a thread a position
        const int i = warp * kWarp + lane;
        float *const part = a.part + ((long long)blockIdx.y * a.T + t.begin + i) * a.rp;
        for (int r = 0; r < a.rp; r += 8) {
            float v[8];
            if (ok) tmem_ld8(tmem + ((uint32_t)(warp * kWarp) << 16) + r, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = ok ? v[j] : NAN;
            if (i < t.count) {
                *reinterpret_cast<float4 *>(part + r) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4 *>(part + r + 4) = make_float4(v[4], v[5], v[6], v[7]);
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
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 4) tmem_free(tmem, cols);
}

// DO: type of base and out.  PL: planes of h.  WVEC: rows of B are 16-byte aligned.
template <int DT, int DO, int PL, bool WVEC> __global__ void __launch_bounds__(kUpTileThreads, 2) lora_up_tile_kernel(const LoraArgs a)
{
    using T = typename Elem<DT>::T;
    using TO = typename Elem<DO>::T;
    constexpr int kStages = 3, kTmem = 256;
    extern __shared__ uint8_t dsm_raw[];
    __shared__ int s_tile[kLoraMaxAdapters + 2], s_sum[4], s_tmem, s_row[kTileRows];
    __shared__ float s_factor[kTileRows];
    __shared__ int s_dead;
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], tfull[2], tempty[2], planes;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp;
    const int slabs = lora_slabs(a.r), r16 = lora_r16(a.r), NS = up_stages(a.r);
    pdl_wait();
    pdl_launch_dependents();
    lora_tiles(a, s_tile, s_sum);
    // units of this CTA: whole tiles' 128-output columns, tile after tile
    const int per_tile = (a.O + kUpCols - 1) / kUpCols;
    const int units = s_tile[a.keep && !a.hidden ? a.n : a.n + 1] * per_tile;      // < 2^31: checked by the host
    const int first = (int)((long long)units * blockIdx.x / gridDim.x), last = (int)((long long)units * (blockIdx.x + 1) / gridDim.x);
    if (first >= last) return;
    uint8_t *const dsm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dsm_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t h_at = dsmem_u32(dsm), b_at = h_at + PL * slabs * kSlabBytes;
    if (tid == 0) {
        s_dead = 0;
        for (int s = 0; s < NS; ++s) dmbar_init(&full[s], 1), dmbar_init(&empty[s], 1);
        for (int b = 0; b < 2; ++b) dmbar_init(&tfull[b], 1), dmbar_init(&tempty[b], 8);
        dmbar_init(&planes, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) tmem_alloc(&s_tmem, kTmem);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int *const dead = &s_dead;
    int tile = first / per_tile, col = first % per_tile;
    LoraTile t = lora_tile_at(a, s_tile, tile);
    auto step = [&]() {                      // to the next unit; whether it begins a tile
        if (++col < per_tile) return false;
        col = 0, ++tile;
        return true;
    };
    const bool wide = a.out_vec;             // lanes hold neighbouring outputs
    if (warp < 8) {
        const int quad = warp % 4, half = warp / 4, q = lane % 4, o = lane / 4;
        bool ok = true, fresh = true;
        uint32_t it = 0;
        for (int u = first; u < last; ++u) {
            const bool some = t.g < a.n;
            if (fresh) {
                // the unit before is behind all warps, and its MMAs have read the planes
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (tid < kTileRows) s_row[tid] = tid < t.count ? lora_row(a, t.begin + tid) : -1;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (some) {
                    // 16 or 32 lanes a position, four ranks each; eight positions' loads under way together
                    const int lanes = slabs * 16, rows = 256 / lanes, k = tid % lanes * 4;
                    const float c = a.alpha * (a.scale ? a.scale[t.g] : 1.f);
                    for (int i0 = tid / lanes; i0 < kTileRows; i0 += 8 * rows) {
                        float4 sum[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                        const float *p = a.part + (long long)(t.begin + i0) * a.rp + k;
                        for (int s = 0; s < a.splits; ++s, p += (long long)a.T * a.rp) {
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (i0 + i * rows < t.count && k < a.rp) {
                                    const float4 v = *reinterpret_cast<const float4 *>(p + i * rows * a.rp);
                                    sum[i].x += v.x, sum[i].y += v.y, sum[i].z += v.z, sum[i].w += v.w;
                                }
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int pos = i0 + i * rows;
                            float f[4] = {sum[i].x, sum[i].y, sum[i].z, sum[i].w}, up = 1.f;
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (k + j >= a.r) f[j] = 0.f;
                            if (DT != 1) {
                                float most = fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
                                for (int s = lanes / 2; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(kFull, most, s));
                                up = plane_scale<DT>(most);
                            }
                            uint16_t pl[4][PL];
#pragma unroll
                            for (int j = 0; j < 4; ++j) planes_of<DT, PL>(f[j] * up, pl[j]);
#pragma unroll
                            for (int j = 0; j < PL; ++j)
                                asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(h_at + (j * slabs + k / 64) * kSlabBytes + slab_at(pos, k % 64 / 8) + k % 8 * 2),
                                             "r"(pl[0][j] | (uint32_t)pl[1][j] << 16), "r"(pl[2][j] | (uint32_t)pl[3][j] << 16) : "memory");
                            if (k == 0) s_factor[pos] = c / up;
                            if (a.hidden && col == 0 && s_row[pos] >= 0) {
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    if (k + j < a.r) a.hidden[(long long)s_row[pos] * a.r + k + j] = f[j];
                            }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (lane == 0) dmbar_arrive(&planes);
                } else if (a.hidden && col == 0) {
                    for (int i = tid; i < t.count * a.r; i += 256)
                        if (s_row[i / a.r] >= 0) a.hidden[(long long)s_row[i / a.r] * a.r + i % a.r] = 0.f;
                }
            }
            const int ab = it & 1, o0 = col * kUpCols + half * 64;
            // lane: rows o and o + 8 of each half of the quadrant, 16 outputs: 16 q + i, or 8 (i / 2) + 2 q + i % 2 where rows are not aligned
            int rows[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 2; ++j) rows[h][j] = some || !a.keep ? s_row[quad * 32 + h * 16 + j * 8 + o] : -1;
            const TO *const base = a.base ? reinterpret_cast<const TO *>(a.base) + o0 : nullptr;
            TO *const out = reinterpret_cast<TO *>(a.out) + o0;
            const int here = min(64, a.O - o0);
            constexpr int V = Elem<DO>::kVec, G = 16 / V;
            uint4 ahead[2][2][G];            // the base, asked for before the accumulator is waited for
            const bool whole = wide && 16 * q + 16 <= here;
            auto ask = [&](int h) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        ahead[h][j][g] = whole && base && rows[h][j] >= 0 ? *reinterpret_cast<const uint4 *>(base + rows[h][j] * a.base_stride + 16 * q + g * V) : make_uint4(0, 0, 0, 0);
            };
            ask(0);
            if (DO != 0) ask(1);             // fp32: twice the registers, one half at a time
            if (some) {
                ok = ok && __all_sync(kFull, dmbar_wait(&tfull[ab], (it >> 1) & 1, dead, a.polls));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (DO == 0 && h == 1) ask(1);
                float d[32];
                if (some && ok) tmem_ld_16x64(tmem + ((uint32_t)(quad * 32 + h * 16) << 16) + ab * kUpCols + half * 64, d);
                if (some && h == 1) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) dmbar_arrive(&tempty[ab]);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (rows[h][j] < 0) continue;
                    TO *const to = out + rows[h][j] * a.out_stride;
                    const float f = some ? ok ? s_factor[quad * 32 + h * 16 + j * 8 + o] : NAN : 0.f;
                    float v[16];
                    if (whole) {
#pragma unroll
                        for (int g = 0; g < G; ++g) bal_widen<DO>(ahead[h][j][g], reinterpret_cast<float2 *>(v + g * V));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int at = wide ? 16 * q + i : 8 * (i / 2) + 2 * q + i % 2;
                            v[i] = at < here && base ? Elem<DO>::to_f32(base[rows[h][j] * a.base_stride + at]) : 0.f;
                        }
                    }
                    if (some) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = ok ? fmaf(f, d[i / 2 * 4 + j * 2 + i % 2], v[i]) : NAN;
                    }
                    if (whole) {
#pragma unroll
                        for (int g = 0; g < G; ++g) *reinterpret_cast<uint4 *>(to + 16 * q + g * V) = bal_narrow<DO>(reinterpret_cast<const float2 *>(v + g * V));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int at = wide ? 16 * q + i : 8 * (i / 2) + 2 * q + i % 2;
                            if (at < here) to[at] = Elem<DO>::from_f32(v[i]);
                        }
                    }
                }
            }
            if (some) ++it;
            fresh = u + 1 < last && step();
            if (fresh) t = lora_tile_at(a, s_tile, tile);
        }
    } else if (warp == 8) {
        // B tiles: row n of the unit at its place in the MMA's columns
        int s = 0, par = 0, ready = 0, pending = 0;
        auto arrive = [&](int at) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) dmbar_arrive(&full[at]);
        };
        for (int u = first; u < last; ++u) {
            if (t.g < a.n) {
                if (!__all_sync(kFull, dmbar_wait(&empty[s], par ^ 1, dead, a.polls))) break;
                const T *const w = reinterpret_cast<const T *>(a.b) + t.g * a.b_group;
                const uint32_t st = b_at + s * slabs * kSlabBytes;
                const int pieces = r16 / 8;
#pragma unroll 4
                for (int i = lane; i < kUpCols * pieces; i += kWarp) {
                    const int n = i / pieces, c = i % pieces, row = col * kUpCols + n;
                    // 16 q + 2 j + b -> 8 j + 2 q + b within each 64
                    const int at = wide ? (n & 64) | (n & 14) << 2 | (n & 48) >> 3 | (n & 1) : n;
                    put8<DT, WVEC>(st + (c / 8) * kSlabBytes + slab_at(at, c % 8), w + (row < a.O ? row : 0) * a.b_row, c * 8, a.r, row < a.O);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (++s == NS) s = 0, par ^= 1;
                if (++pending == 2) {       // one unit's tile stays in flight
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    arrive(ready);
                    if (++ready == NS) ready = 0;
                    --pending;
                }
            }
            if (u + 1 < last && step()) t = lora_tile_at(a, s_tile, tile);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (pending && !*dead) arrive(ready);
    } else {
        const bool leader = elect_one();
        const uint32_t idesc = umma_idesc_16<DT>(kUpCols);
        bool ok = true, fresh = true;
        int s = 0, par = 0;
        uint32_t it = 0, made = 0;
        for (int u = first; u < last && ok; ++u) {
            if (t.g < a.n) {
                if (fresh) ok = __all_sync(kFull, dmbar_wait(&planes, made++ & 1, dead, a.polls));
                const int ab = it & 1;
                ok = ok && __all_sync(kFull, dmbar_wait(&tempty[ab], ((it >> 1) & 1) ^ 1, dead, a.polls));
                ok = ok && __all_sync(kFull, dmbar_wait(&full[s], par, dead, a.polls));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t st = b_at + s * slabs * kSlabBytes;
                for (int p = 0; p < PL; ++p)
                    for (int k = 0; k < r16; k += 16)
                        umma_16(leader, tmem + ab * kUpCols, umma_desc_sw128(h_at + (p * slabs + k / 64) * kSlabBytes, k % 64 / 16),
                                umma_desc_sw128(st + k / 64 * kSlabBytes, k % 64 / 16), idesc, p > 0 || k > 0);
                umma_commit_if(leader, &empty[s]);
                umma_commit_if(leader, &tfull[ab]);
                if (++s == NS) s = 0, par ^= 1;
                ++it;
            }
            fresh = u + 1 < last && step();
            if (fresh) t = lora_tile_at(a, s_tile, tile);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 9) tmem_free(tmem, kTmem);
}

}  // namespace stmoe_dev
