// Routed SwiGLU expert FFN over 4-bit expert images (MX4 weights, fp32 hidden state):
//
//   h'[b] = h[b] + r * sum_k w[b][k] * W_d ( silu(W_g x_b) * (W_u x_b) ),   x_b = h[b] * inv_rms[b]
//
// A decode step is bound by reading the routed experts' images once (51/32 bytes per hidden x inter
// element).  The codes go from HBM to the tensor cores as they are (tcgen05.mma kind::mxf4, TMA in
// the 128-byte swizzled layout, block scales through tensor memory as in mx4_matmul.cuh): unpacking
// them to fp32 would cost the CUDA cores two conversions and an FMA per weight and token, three times
// what they can issue at 6.5 TB/s of 4-bit weights.
//
// The tensor cores' 4-bit form takes 4-bit activations, which alone would be far too coarse.  So an
// activation is written as a sum of eight e2m1 values (planes) under scales that fall by a fixed
// amount, a fixed-point expansion of the block:
//   e_0: the smallest exponent with amax <= 6 * 2^e_0;   e_1 = e_0 - 2;   e_p = e_(p-1) - 3
// Rounding at plane 0 leaves at most 2^e_0 = 4 * 2^e_1 (e2m1 steps by 2 up to 6), rounding a value of
// at most 4 leaves at most 1/2, which is 4 units three binary orders below.  After eight planes the
// residue is at most 2^(e_0 - 21), below 2^-22 of the block's largest magnitude: the precision of the
// fp32 values they stand for.  The exponents do not depend on the residues, so all planes of a block
// follow from one maximum.  The planes are further columns of the MMA's N: a token is eight of them,
// and eight rows of 128 bytes are exactly one atom of the swizzled operand layout, so an entry's
// tokens are gathered by one TMA load each.  The epilogue adds a token's eight columns in fp32,
// smallest plane first.
//
//   mx4_planes_kernel    hidden state -> planes; the work-list entries, one line of memory each
//   mx4_ffn_kernel<2>    gate and up tiles of 128 rows; epilogue: SiLU(g) * u as planes (a warp's 32
//                        rows are one block of the next reduction, so a block maximum is one
//                        warp reduction)
//   mx4_ffn_kernel<1>    down tiles -> partial sums [pair][split][H]
//   mx4_combine_kernel   weighted sum and residual in a fixed order
// Every launch may start while the one before drains (programmatic dependent launch) and waits for
// its results itself.  Sums have a fixed order: the same call gives the same bits.
#pragma once
#include "ffn.cuh"
#include "mx4.cuh"
#include "mx4_matmul.cuh"

namespace stmoe_dev {

constexpr int kPlanes = 8;
constexpr int kMxfTokens = 12;                          // tokens of a work-list entry: 96 MMA columns
constexpr int kMxfCols = kMxfTokens * kPlanes;
constexpr int kMxfAccStride = 2 * kMxfCols;             // two accumulator buffers of (gate, up)
constexpr int kMxfScaleCol = 2 * kMxfAccStride;
constexpr int kMxfMaxStages = 12;
// warps: 0 weights, 1 MMA, 2-5 and 6-9 epilogues (a group an accumulator buffer: with few reduction steps
// a task, as in the down projection of narrow experts, one group was slower than the MMAs), 10-13 scales
constexpr int kMxfThreads = 448;
constexpr int kMxfScaleWarp = 10;

// the B tile of a launch whose entries hold at most mt tokens: N is a multiple of 16
__host__ __device__ constexpr int mxf_cols(int tokens) { return (tokens * kPlanes + 15) / 16 * 16; }
__host__ __device__ constexpr int mxf_slot_bytes(int nmat, int mt)
{
    return nmat * (kMmABytes + 1024) + mxf_cols(mt) * 128 + 1024;   // codes and scales of both operands
}
__host__ __device__ constexpr int mxf_stages(int nmat, int mt)
{
    const int by_smem = (kMmSmemBytes - 1024) / mxf_slot_bytes(nmat, mt), by_tmem = (512 - kMxfScaleCol) / (8 * nmat + 8);
    const int n = by_smem < by_tmem ? by_smem : by_tmem;
    return n < kMxfMaxStages ? n : kMxfMaxStages;
}

static_assert(mxf_stages(2, kMxfTokens) >= 4 && mxf_stages(1, kMxfTokens) >= 4 && mxf_stages(2, 1) >= 4, "");  // scale warps

// Byte offsets inside an MX4 expert image: codes of gate [I][H/2], up, down [H][I/2], then the
// scales of the three in the same order.
__host__ __device__ inline size_t mx4_image_codes(int H, int I, int mat) { return (size_t)mat * ((size_t)H * I / 2); }
__host__ __device__ inline size_t mx4_image_scales(int H, int I, int mat)
{
    return 3 * ((size_t)H * I / 2) + (size_t)mat * ((size_t)H * I / 32);
}

// ---- activations as planes ---------------------------------------------------------------------

// The planes of one block: every lane holds one element, returns the word of its eight codes (plane p
// in bits 4p) and the scale byte of plane 0.
__device__ __forceinline__ uint32_t planes_of(float v, uint32_t &byte)
{
    const uint32_t m = __reduce_max_sync(kFull, __float_as_uint(v) & 0x7fffffffu);
    const int ef = (int)(m >> 23);
    if (ef == 255) {  // infinity or NaN: the block is NaN in every plane
        byte = 255;
        return 0;
    }
    // amax = f * 2^(ef-127), f in [1,2): f <= 1.5 fits under 6 * 2^(ef-129), else one binary order more
    byte = (uint32_t)max(ef - 2 + ((m & 0x7fffffu) > 0x400000u ? 1 : 0), 0);
    uint32_t codes = 0;
    const int b = (int)byte;
    const float up = __uint_as_float((uint32_t)(254 - b) << 23);   // 2^-(b-127): b <= 253, so a normal number
    v *= up;
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) {
        uint32_t c, f;
        asm("{.reg .b8 q;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 q, %2, %2;\n\t"
            "cvt.rn.f16x2.e2m1x2 %1, q;\n\t"
            "cvt.u32.u8 %0, q;}"
            : "=r"(c), "=r"(f)
            : "f"(v));
        const int off = p == 0 ? 0 : 3 * p - 1;
        if (b >= off) codes |= (c & 15u) << (4 * p);   // a plane below the smallest scale is dropped
        v -= __low2float(*reinterpret_cast<const __half2 *>(&f));   // exact: at most half a step is left
        v *= p == 0 ? 4.f : 8.f;                                    // to the next plane's units
    }
    return codes;
}
// scale byte of plane p: exponents fall by 2, then by 3
__device__ __forceinline__ uint32_t plane_byte(uint32_t byte, int p)
{
    return byte == 255 ? 255u : (uint32_t)max((int)byte - (p == 0 ? 0 : 3 * p - 1), 0);
}
// A warp stores block `blk` of row `row` (token or pair): codes [row][8][blocks*16], scales [row][8][blocks].
__device__ __forceinline__ void planes_store(float v, uint8_t *codes, uint8_t *scales, long long row, int blk, int blocks, int lane)
{
    uint32_t byte;
    const uint32_t w = transpose_nibbles(planes_of(v, byte), lane);   // plane lane%8 of elements 8 (lane/8) .. +7
    const int p = lane % kPlanes;
    *reinterpret_cast<uint32_t *>(codes + ((row * kPlanes + p) * blocks + blk) * 16 + 4 * (lane / kPlanes)) = w;
    if (lane < kPlanes) scales[(row * kPlanes + lane) * blocks + blk] = (uint8_t)plane_byte(byte, lane);
}

// What the projections need to know of a work-list entry (one expert, up to kMxfTokens of its pairs), in
// one line of memory: gathered from the router's lists it would be a chain of three dependent loads at
// every task of every warp.
struct alignas(128) Mx4Entry {
    const uint8_t *img;            // expert image
    int32_t img_index;             // its place in the store that the tensor maps cover
    int16_t count;                 // pairs
    int16_t shared;                // 1: in the store of the shared experts
    uint16_t token[kMxfTokens];    // sequence
    uint16_t slot[kMxfTokens];     // row of the activation and partial-sum buffers
    float inv[kMxfTokens];         // the sequence's RMSNorm factor
};
static_assert(sizeof(Mx4Entry) == 128, "");

struct Mx4PlanesArgs {
    const float *h, *inv_rms;
    int B, H;
    uint8_t *codes, *scales;
    Mx4Entry *entries;
    int *n_entries;
    const uint8_t *store[2];       // first image of the maps: routed experts, shared ones
    unsigned long long img_bytes;
    int E, K, mt;
    // entries from given ids (stand-alone call, by the first CTA) ...
    const int32_t *ids;
    // ... or from the router's work list
    WorkList wl;
    const uint8_t *const *blob;    // image of every expert of the step
};

// Entries of at most mt tokens per expert from given ids, pairs of an expert in index order.  ids
// outside [0, E) have no entry.  One CTA of 256 threads.  A pair's place among its expert's pairs is its
// rank in its chunk of 32 (one match per warp) behind the chunks before it: a thread per expert that
// walked all pairs took 40 us at 64 sequences x 6 experts.
// s_cnt: [chunks][256], pairs of an expert in a chunk, then behind all chunks before it.
__device__ __forceinline__ void entries_from_ids(const Mx4PlanesArgs &a, uint16_t *s_cnt, int *s_g, int *s_first)
{
    const int e = threadIdx.x, n = a.B * a.K, chunks = (n + kWarp - 1) / kWarp;
    const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp;
    for (int c = 0; c < chunks; ++c) s_cnt[c * 256 + e] = 0;
    __syncthreads();
    for (int c = warp; c < chunks; c += 8) {
        const int i = c * kWarp + lane;
        const int id = i < n ? a.ids[i] : -1;
        const unsigned same = __match_any_sync(kFull, id);
        if ((unsigned)id < (unsigned)a.E && lane == __ffs(same) - 1) s_cnt[c * 256 + id] = (uint16_t)__popc(same);
    }
    __syncthreads();
    int cnt = 0;
    for (int c = 0; c < chunks; ++c) {
        const int k = s_cnt[c * 256 + e];
        s_cnt[c * 256 + e] = (uint16_t)cnt;   // at most 64 * 32 pairs
        cnt += k;
    }
    const int mine = (cnt + a.mt - 1) / a.mt;
    int g = mine;                             // inclusive prefix sum over the experts
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
        const int t = __shfl_up_sync(kFull, g, o);
        if (lane >= o) g += t;
    }
    if (lane == kWarp - 1) s_g[warp] = g;
    __syncthreads();
    for (int w = 0; w < warp; ++w) g += s_g[w];
    if (e == 255) *a.n_entries = g;
    g -= mine;
    s_first[e] = g;
    for (int q = 0; q < mine; ++q) {
        Mx4Entry &x = a.entries[g + q];
        x.img = a.store[0] + (size_t)e * a.img_bytes, x.img_index = e;
        x.count = (int16_t)min(a.mt, cnt - q * a.mt), x.shared = 0;
    }
    __syncthreads();
    for (int c = warp; c < chunks; c += 8) {
        const int i = c * kWarp + lane;
        const int id = i < n ? a.ids[i] : -1;
        const unsigned same = __match_any_sync(kFull, id);
        if ((unsigned)id < (unsigned)a.E) {
            const int at = s_cnt[c * 256 + id] + __popc(same & ((1u << lane) - 1)), b = i / a.K;
            Mx4Entry &x = a.entries[s_first[id] + at / a.mt];
            const int q = at % a.mt;
            x.token[q] = (uint16_t)b, x.slot[q] = (uint16_t)i, x.inv[q] = a.inv_rms ? a.inv_rms[b] : 1.f;
        }
    }
}

// One warp, one entry of the router's work list.
__device__ __forceinline__ void entry_from_list(const Mx4PlanesArgs &a, int g, int lane)
{
    const int ge = a.wl.g_expert[g], start = a.wl.g_start[g], cnt = a.wl.g_count[g], shared = ge >= a.E;
    Mx4Entry &x = a.entries[g];
    if (lane == 0) {
        const uint8_t *img = a.blob[ge];
        x.img = img, x.img_index = (int)((unsigned long long)(img - a.store[shared]) / a.img_bytes);
        x.count = (int16_t)cnt, x.shared = (int16_t)shared;
    }
    if (lane < cnt) {
        const int b = a.wl.pair_token[start + lane];
        x.token[lane] = (uint16_t)b, x.slot[lane] = (uint16_t)a.wl.pair_slot[start + lane];
        x.inv[lane] = a.inv_rms ? a.inv_rms[b] : 1.f;
    }
}

__global__ void __launch_bounds__(256) mx4_planes_kernel(const Mx4PlanesArgs a)
{
    extern __shared__ uint16_t s_cnt[];   // [chunks of 32 pairs][256]; only with ids
    __shared__ int s_g[8], s_first[256];
    pdl_launch_dependents();
    pdl_wait();
    const int blocks = a.H / kMxBlock, lane = threadIdx.x % kWarp, n = a.B * blocks;
    int cta = blockIdx.x, ctas = gridDim.x;
    if (a.ids) {
        if (cta == 0) {
            entries_from_ids(a, s_cnt, s_g, s_first);
            return;
        }
        --cta, --ctas;
    }
    const int warp = cta * (256 / kWarp) + threadIdx.x / kWarp, step = ctas * (256 / kWarp);
    for (int i = warp; i < n; i += step) {
        const int b = i / blocks, blk = i % blocks;
        planes_store(a.h[(size_t)b * a.H + blk * kMxBlock + lane], a.codes, a.scales, b, blk, blocks, lane);
    }
    if (!a.ids) {
        const int entries = *a.wl.n_groups;
        if (warp == 0 && lane == 0) *a.n_entries = entries;
        for (int g = warp; g < entries; g += step) entry_from_list(a, g, lane);
    }
}

// ---- the two projections ------------------------------------------------------------------------

inline int mxf_align(int blocks) { return blocks % 8 == 0 ? 8 : blocks % 4 == 0 ? 4 : 1; }

struct Mx4FfnArgs {
    const Mx4Entry *entries;
    const int *n_entries;
    long long scale_off[2];              // scales of the one or two matrices inside an image
    int rows, blocks;                    // rows of a matrix, scale blocks of its row
    int last_task;                       // of the most that the call can have
    int mt, splits;                      // splits: of the reduction, over a cluster (gate/up) or over tasks (down)
    const uint8_t *x_scales;             // planes of the activations, [row][8][blocks]
    // gate/up
    uint8_t *act_codes, *act_scales;     // [pair][8][rows/32 * 16], [pair][8][rows/32]
    // down
    float *part;                         // [pair][splits][rows]
    unsigned *err;
    int polls;                           // limit of every wait
};

struct Mx4FfnTask {
    int g, row0, z;
};
template <int NMAT> __device__ __forceinline__ Mx4FfnTask mxf_task(const Mx4FfnArgs &a, int task)
{
    const int tiles = (a.rows + kMmRows - 1) / kMmRows, zs = NMAT == 1 ? a.splits : 1;
    Mx4FfnTask t;
    t.g = task / (tiles * zs);
    const int r = task - t.g * tiles * zs;
    t.row0 = (r / zs) * kMmRows;
    t.z = r % zs;
    return t;
}

// SiLU(g) * u for 32 consecutive rows of one pair, as planes; inv: the token's RMSNorm factor, applied
// to the sums: W (inv * h) = inv * (W h)
__device__ __forceinline__ void mxf_store_act(const Mx4FfnArgs &a, float g, float u, int slot, float inv, int row, int lane)
{
    g *= inv, u *= inv;
    planes_store(g / (1.f + expf(-g)) * u, a.act_codes, a.act_scales, slot, row / kMxBlock, a.rows / kMxBlock, lane);
}

// kAlign: what scale rows are aligned to (mxf_align), of weights and planes alike; as a template
// parameter because a kernel of some tens of microseconds pays for every line of code it fetches
template <int NMAT, int kAlign>
__global__ void __launch_bounds__(kMxfThreads, 1)
mx4_ffn_kernel(const __grid_constant__ CUtensorMap map_w0, const __grid_constant__ CUtensorMap map_w1,
               const __grid_constant__ CUtensorMap map_s0, const __grid_constant__ CUtensorMap map_s1,
               const __grid_constant__ CUtensorMap map_x, const Mx4FfnArgs a)
{
    extern __shared__ uint8_t dsm_raw[];
    __shared__ uint64_t full[kMxfMaxStages], empty[kMxfMaxStages], tfull[2], tempty[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_dead;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp;
    uint8_t *dsm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dsm_raw) + 1023) & ~(uintptr_t)1023);
    const int NS = mxf_stages(NMAT, a.mt), slot = mxf_slot_bytes(NMAT, a.mt);
    const int x_at = NMAT * kMmABytes, sfa_at = x_at + mxf_cols(a.mt) * 128, sfb_at = sfa_at + NMAT * 1024;
    constexpr int kSetCols = 8 * NMAT + 8;   // tensor-memory columns of a stage's scales

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
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    volatile int *dead = &s_dead;
    // Gate/up: the work list and the planes are the kernel before's.  Down: only the activations are (the
    // gate/up kernel lets its successor start after its own wait, so the work list is complete); its first
    // weights are on their way while gate/up finishes elsewhere, and the warps that read activations wait.
    // The work list is read from L2, as an L1 line could be older than this launch.
    if (NMAT == 2) pdl_wait();
    pdl_launch_dependents();

    const int ranks = NMAT == 2 ? a.splits : 1;   // CTAs of a cluster that share a task's reduction
    const int tiles = (a.rows + kMmRows - 1) / kMmRows;
    const int n_tasks = __ldcg(a.n_entries) * tiles * (NMAT == 1 ? a.splits : 1);
    const int per_entry = tiles * (NMAT == 1 ? a.splits : 1);
    const int rank = blockIdx.x % ranks, first = blockIdx.x / ranks, step = gridDim.x / ranks;
    const int n_steps = (a.blocks + kMmStageBlocks - 1) / kMmStageBlocks;
    auto k_range = [&](int z, int &beg, int &end) {
        const int q = NMAT == 2 ? rank : z;
        beg = n_steps * q / a.splits, end = n_steps * (q + 1) / a.splits;   // at most 2^20 steps, 8 splits
    };

    if (warp == 0) {
        // the scale warps' first loads go ahead of the flood of weights, or the first stage would wait
        // behind it
        asm volatile("bar.sync 1, 160;" ::: "memory");
        if (elect_one()) {
            int s = 0, issued = 0, img_next = 0;
            bool shared_next = false;
            uint32_t par = 0;
            auto fetch = [&](int task) {   // a task's entry is asked for one task ahead
                const Mx4Entry &en = a.entries[min(task, a.last_task) / per_entry];
                img_next = __ldcg(&en.img_index), shared_next = __ldcg(&en.shared) != 0;
            };
            fetch(first);
            for (int task = first; task < n_tasks && !*dead; task += step) {
                const Mx4FfnTask t = mxf_task<NMAT>(a, task);
                const int img = img_next;
                const bool shared = shared_next;
                fetch(task + step);
                const CUtensorMap *w0 = shared ? &map_s0 : &map_w0, *w1 = shared ? &map_s1 : &map_w1;
                int k_beg, k_end;
                k_range(t.z, k_beg, k_end);
                for (int k = k_beg; k < k_end; ++k, ++issued) {
                    if (!dmbar_wait(&empty[s], par ^ 1u, dead, a.polls)) break;
                    uint8_t *st = dsm + (size_t)s * slot;
                    dmbar_expect_tx(&full[s], (uint32_t)(NMAT * kMmABytes));
                    tma_load_3d(st, w0, k * 128, t.row0, img, &full[s]);
                    if (NMAT == 2) tma_load_3d(st + kMmABytes, w1, k * 128, t.row0, img, &full[s]);
                    if (++s == NS) s = 0, par ^= 1u;
                }
            }
            // every load that was issued lands before the CTA may exit; the token loads of a stage complete
            // on the same barrier (behind an error, where a stage may have token loads and no weights, its
            // barrier never completes: see settle_in_flight)
            int none = 0;
            for (int i = 0; i < min(issued, NS); ++i) {
                if (s == 0) s = NS, par ^= 1u;
                --s;
                dmbar_wait(&full[s], par, &none, 1 << 14);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const bool leader = elect_one();   // the whole warp walks the loop, one lane issues
        const uint32_t ring = dsmem_u32(dsm);
        int s = 0, it = 0;
        uint32_t par = 0;
        bool ok = true;
        int count = __ldcg(&a.entries[min(first, a.last_task) / per_entry].count);
        for (int task = first; task < n_tasks && ok; task += step, ++it) {
            const Mx4FfnTask t = mxf_task<NMAT>(a, task);
            const int n = mxf_cols(count);
            count = __ldcg(&a.entries[min(task + step, a.last_task) / per_entry].count);   // the next task's
            const uint32_t id0 = umma_idesc_mxf4(n, 0), id1 = umma_idesc_mxf4(n, 1);
            const int ab = it & 1;
            if (!(ok = __all_sync(kFull, dmbar_wait(&tempty[ab], ((uint32_t)(it >> 1) & 1u) ^ 1u, dead, a.polls)))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + ab * kMxfAccStride;
            int k_beg, k_end;
            k_range(t.z, k_beg, k_end);
            for (int k = k_beg; k < k_end; ++k) {
                if (!(ok = __all_sync(kFull, dmbar_wait(&full[s], par, dead, a.polls)))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t st = ring + s * slot;
                const uint32_t sf = tmem + kMxfScaleCol + s * kSetCols, sfb = sf + 8 * NMAT;
                const uint32_t dw = desc_low_sw128(st), dx = desc_low_sw128(st + x_at);
                const uint32_t dsw = desc_low_scales(st + sfa_at), dsx = desc_low_scales(st + sfb_at);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) umma_copy_scales(leader, sf + 8 * m + 4 * q, dsw + 64 * m + 32 * q);
                    umma_copy_scales(leader, sfb + 4 * q, dsx + 32 * q);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int m = 0; m < NMAT; ++m)
                        umma_mxf4(leader, acc + m * kMxfCols, dw + m * (kMmABytes >> 4) + 2 * j, dx + 2 * j, j & 1 ? id1 : id0,
                                  sf + 8 * m + 4 * (j / 2), sfb + 4 * (j / 2), k > k_beg || j > 0);
                umma_commit_if(leader, &empty[s]);
                if (++s == NS) s = 0, par ^= 1u;
            }
            if (ok) umma_commit_if(leader, &tfull[ab]);
        }
        __syncwarp();
    } else if (warp < kMxfScaleWarp) {
        const int lg = warp % 4, ab = (warp - 2) / 4;   // quarter of the lanes, accumulator buffer
        float *part = reinterpret_cast<float *>(dsm);   // cluster: this rank's sums [mat][token][128], in the idle ring
        uint32_t use = 0;
        bool ok = true;   // once false, this warp's tasks that are left are NaN (see mx4_matmul.cuh)
        for (int task = first + ab * step; task < n_tasks; task += 2 * step, ++use) {
            const Mx4FfnTask t = mxf_task<NMAT>(a, task);
            const Mx4Entry &en = a.entries[t.g];
            const int cnt = __ldcg(&en.count), own = min(lane, kMxfTokens - 1);
            const int slot_l = __ldcg(&en.slot[own]);      // lane i: the i-th pair's, fetched while the MMAs run
            const float inv_l = en.inv[own];
            ok = ok && __all_sync(kFull, dmbar_wait(&tfull[ab], use & 1u, dead, a.polls));
            if (NMAT == 2 && ranks > 1 && !ok) settle_in_flight();   // its sums take the ring's place
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + ab * kMxfAccStride + ((uint32_t)(lg * kWarp) << 16);
            const int row = t.row0 + lg * kWarp + lane;
            // a few tokens at a time: their chains (loads, sums, reductions, conversions) overlap
            constexpr int kTok = NMAT == 1 ? 4 : 2;
            const long long hop = (long long)a.splits * a.rows;
            for (int i0 = 0; i0 < cnt; i0 += kTok) {
                uint32_t raw[kTok][NMAT][8];
                float y[kTok][NMAT];
#pragma unroll
                for (int q = 0; q < kTok; ++q)
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) tmem_ld8_start(acc + m * kMxfCols + (i0 + q) * kPlanes, raw[q][m]);
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < kTok; ++q)
#pragma unroll
                    for (int m = 0; m < NMAT; ++m) {
                        y[q][m] = __uint_as_float(raw[q][m][7]);   // smallest plane first
#pragma unroll
                        for (int p = 6; p >= 0; --p) y[q][m] += __uint_as_float(raw[q][m][p]);
                        if (!ok) y[q][m] = __uint_as_float(0x7fffffffu);
                    }
                // behind the last pair the columns hold what nobody wrote: not used
#pragma unroll
                for (int q = 0; q < kTok; ++q) {
                    const int slot = __shfl_sync(kFull, slot_l, i0 + q);
                    if (i0 + q >= cnt) break;
                    if (NMAT == 1) {
                        if (row < a.rows) a.part[slot * hop + (long long)t.z * a.rows + row] = y[q][0];
                    } else if (ranks > 1) {
#pragma unroll
                        for (int m = 0; m < NMAT; ++m) part[(m * kMxfTokens + i0 + q) * kMmRows + lg * kWarp + lane] = y[q][m];
                    } else if (t.row0 + lg * kWarp < a.rows) {   // rows are a multiple of 32: the whole warp or none of it
                        mxf_store_act(a, y[q][0], y[q][NMAT - 1], slot, __shfl_sync(kFull, inv_l, i0 + q), row, lane);
                    }
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (ok && lane == 0) dmbar_arrive(&tempty[ab]);
        }
    } else {
        // scales and the tokens' codes, a warp every fourth stage (see mx4_matmul.cuh; up to twelve loads a
        // stage by one thread would hold the weights' back).  A task's steps may differ by one between
        // splits, so the position is walked, not computed
        const int w = warp - kMxfScaleWarp;
        // what a warp knows of the task its next step belongs to, and of the one after (asked for at the
        // start of this one)
        struct Info {
            const uint8_t *img;
            int cnt, row;                 // row: lane i: token or slot of pair i
        };
        struct Pos {
            int task, k, end, row0;
            Info in, ahead;
        };
        auto ask = [&](int task) {
            const Mx4Entry &en = a.entries[min(task, a.last_task) / per_entry];
            const int own = min(lane, kMxfTokens - 1);
            const auto img = __ldcg(reinterpret_cast<const unsigned long long *>(&en.img));
            return Info{reinterpret_cast<const uint8_t *>(img), __ldcg(&en.count), __ldcg(NMAT == 2 ? &en.token[own] : &en.slot[own])};
        };
        auto enter = [&](Pos &p) {   // first step of task p.task
            if (p.task >= n_tasks) return;
            const Mx4FfnTask t = mxf_task<NMAT>(a, p.task);
            p.in = p.ahead, p.row0 = t.row0;
            p.ahead = ask(p.task + step);
            k_range(t.z, p.k, p.end);
        };
        auto forward = [&](Pos &p, int by) {
            p.k += by;
            while (p.task < n_tasks && p.k >= p.end) {
                const int over = p.k - p.end;
                p.task += step;
                enter(p);
                p.k += over;
            }
        };
        auto load_w = [&](const Pos &p, uint2 (&vw)[4 * NMAT]) {
            load_scales<4 * NMAT>(vw, [&](int i) {
                return p.in.img + a.scale_off[i / 4] + (long long)min(p.row0 + 32 * (i % 4) + lane, a.rows - 1) * a.blocks;
            }, (1u << (4 * NMAT)) - 1, p.k * kMmStageBlocks, a.blocks, kAlign);
        };
        auto load_x = [&](const Pos &p, uint2 (&vx)[3]) {
            int row[3];   // rows of the B tile: plane q % 8 of token q / 8
            uint32_t on = 0;
#pragma unroll
            for (int r = 0; r < 3; ++r) {
                const int q = 32 * r + lane;
                row[r] = __shfl_sync(kFull, p.in.row, q / kPlanes) * kPlanes + q % kPlanes;
                if (q < p.in.cnt * kPlanes) on |= 1u << r;
            }
            load_scales<3>(vx, [&](int r) { return a.x_scales + (long long)row[r] * a.blocks; }, on, p.k * kMmStageBlocks, a.blocks, kAlign);
        };
        uint2 vw[4 * NMAT], vx[3], nw[4 * NMAT], nx[3];
        Pos p = {first, 0, 0, 0, {}, ask(first)};
        enter(p);
        forward(p, w);
        if (p.task < n_tasks) load_w(p, vw);
        asm volatile("bar.sync 1, 160;" ::: "memory");
        if (NMAT == 1) pdl_wait();   // the activations
        if (p.task < n_tasks) load_x(p, vx);
        for (int i = w; p.task < n_tasks; i += 4) {
            const int k = p.k, cnt = p.in.cnt, xrow = p.in.row;
            forward(p, 4);
            if (p.task < n_tasks) load_w(p, nw), load_x(p, nx);
            const int s = i % NS;
            if (!__all_sync(kFull, dmbar_wait(&empty[s], ((uint32_t)(i / NS) & 1u) ^ 1u, dead, a.polls))) break;   // its place may be in use
            uint8_t *st = dsm + (size_t)s * slot;
#pragma unroll
            for (int m = 0; m < NMAT; ++m) {
                const uint2 v[4] = {vw[4 * m], vw[4 * m + 1], vw[4 * m + 2], vw[4 * m + 3]};
                store_scales<4>(st + sfa_at + 1024 * m, 512, lane, v);
            }
            store_scales<3>(st + sfb_at, 512, lane, vx);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            const uint32_t xst = dsmem_u32(st + x_at);
            if (elect_one()) dmbar_expect_tx(&full[s], (uint32_t)(cnt * kPlanes * 128));
            for (int q = 0; q < cnt; ++q) {
                const int row = __shfl_sync(kFull, xrow, q) * kPlanes;
                if (elect_one()) tma_load_2d_at(xst + q * kPlanes * 128, &map_x, k * 128, row, &full[s]);
            }
#pragma unroll
            for (int r = 0; r < 4 * NMAT; ++r) vw[r] = nw[r];
#pragma unroll
            for (int r = 0; r < 3; ++r) vx[r] = nx[r];
        }
    }
    if (NMAT == 2 && ranks > 1 && first < n_tasks) {   // one task per cluster
        __syncwarp();
        cluster_sync();
        const Mx4FfnTask t = mxf_task<NMAT>(a, first);
        const Mx4Entry &en = a.entries[t.g];
        const int cnt = en.count;
        const uint32_t part = dsmem_u32(dsm);
        // (token, 32 rows) units, dealt to the ranks and their warps
        for (int u = rank + ranks * warp; u < cnt * 4; u += ranks * (kMxfThreads / kWarp)) {
            const int i = u / 4, r0 = (u % 4) * kWarp;
            if (t.row0 + r0 >= a.rows) continue;
            const int slot_i = en.slot[i];
            const float inv_i = en.inv[i];
            float gz[kMmMaxSplits], vz[kMmMaxSplits];   // the ranks' loads are under way together
#pragma unroll
            for (int z = 0; z < kMmMaxSplits; ++z)
                if (z < ranks) {
                    gz[z] = ld_cluster(part + (uint32_t)(i * kMmRows + r0 + lane) * 4, z);
                    vz[z] = ld_cluster(part + (uint32_t)((kMxfTokens + i) * kMmRows + r0 + lane) * 4, z);
                }
            float g = gz[0], v = vz[0];
#pragma unroll
            for (int z = 1; z < kMmMaxSplits; ++z)
                if (z < ranks) g += gz[z], v += vz[z];
            mxf_store_act(a, g, v, slot_i, inv_i, t.row0 + r0 + lane, lane);
        }
        cluster_sync();
    }
    if (NMAT == 1) pdl_wait();   // a CTA without tasks too: the grid's end then means that gate/up has ended
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (s_dead) settle_in_flight();
    if (warp == 1) {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    if (tid == 0 && s_dead && a.err) *a.err = 1u;
}

// h_out[b][c] = h[b][c] + r * (weighted sum of the down projection's partial sums), in a fixed order:
// shared experts, then routed ones, splits innermost.  ids (stand-alone call): a pair whose id names
// no expert has no partial sums and adds nothing; what lies in its place is read and dropped, so that no
// load waits for another.
template <int S> __device__ __forceinline__ float mx4_combine_sum(const FfnArgs &a, const int32_t *ids, int b, int c)
{
    constexpr int Q = S >= 8 ? 1 : 8 / S;   // slots whose loads are under way together
    const int KS = a.K + a.n_shared;
    const float *part = a.part + (long long)b * KS * S * a.H + c;
    float y = 0.f;
    for (int q0 = 0; q0 < KS; q0 += Q) {
        float v[Q][S], w[Q];
        bool in[Q];
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            const int q = min(q0 + j, KS - 1), k = q < a.n_shared ? a.K + q : q - a.n_shared;
            in[j] = q0 + j < KS && !(ids && (unsigned)ids[b * a.K + k] >= (unsigned)a.E);
            w[j] = q < a.n_shared ? 1.f : a.w[b * a.K + k];
#pragma unroll
            for (int z = 0; z < S; ++z) v[j][z] = __ldcg(part + (long long)(k * S + z) * a.H);
        }
#pragma unroll
        for (int j = 0; j < Q; ++j) {
            float p = v[j][0];
#pragma unroll
            for (int z = 1; z < S; ++z) p += v[j][z];
            if (in[j]) y = fmaf(w[j], p, y);
        }
    }
    return y;
}
__global__ void __launch_bounds__(256) mx4_combine_kernel(const FfnArgs a, const int32_t *ids)
{
    pdl_launch_dependents();
    pdl_wait();
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < a.B * a.H; i += gridDim.x * blockDim.x) {
        const int b = i / a.H, c = i % a.H;
        const float h = a.h[i];
        float y;
        switch (a.S) {
        case 1: y = mx4_combine_sum<1>(a, ids, b, c); break;
        case 2: y = mx4_combine_sum<2>(a, ids, b, c); break;
        case 3: y = mx4_combine_sum<3>(a, ids, b, c); break;
        case 4: y = mx4_combine_sum<4>(a, ids, b, c); break;
        case 5: y = mx4_combine_sum<5>(a, ids, b, c); break;
        case 6: y = mx4_combine_sum<6>(a, ids, b, c); break;
        case 7: y = mx4_combine_sum<7>(a, ids, b, c); break;
        default: y = mx4_combine_sum<8>(a, ids, b, c); break;
        }
        a.h_out[i] = fmaf(a.residual_scale, y, h);
    }
}

}  // namespace stmoe_dev
