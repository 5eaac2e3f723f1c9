// Low-rank adapters of many requests beside a shared projection, and their gradients.
//
//   out[t] = base[t] + c_g h[t] B_g^T,   h[t] = x[t] A_g^T,   g = adapter of row t, c_g its scale
//   A_g [r][I], B_g [O][r], x [T][I], out [T][O]; rows without an adapter: out = base
//   u[t] = dout[t] B_g,  dx[t] = c_g u[t] A_g,  dA_g = c_g sum_t u[t]^T x[t],  dB_g = c_g sum_t dout[t]^T h[t]
//
// Rows are visited in the order of a grouping by adapter (group_rows.cuh), so that rows of one adapter meet in one tile
// and its matrices are read once for all of them.  The rank is small: 2 r operations to each element of x and of out
// leave every size in the range of ranks that adapters have bound by the bytes of x, base and out, or, with few rows, by those of A and B.
//
// h and u are kept in fp32; their products with 16-bit matrices run on the tensor cores as a sum of two 16-bit
// planes (three where the result is fp32), which leaves 2^-17 (2^-25) of a bf16 value behind, 2^-22 of an fp16 one: less than a 128th of the
// result's own rounding, of which it turns a few in a thousand (bf16, against fp32 throughout: 0.1 to 0.5 % of the results are the other neighbour, errors
// against 64 bits are the same to two digits).  fp16 planes hold a power-of-two multiple of the values, whose largest then lies in [2^14, 2^15): the largest
// of a row in the products, in the gradients of A and B the largest so far among the rows and ranks of a task.  Values far below it
// keep what a step of 2^-24 leaves of them: 2^-39 of that largest.
// The inner dimension of the first product may be split; its parts are added in a fixed order.  No
// floating-point atomics: the same call gives the same bits.
#pragma once
#include "row_utils.cuh"
#include "tcgen05_utils.cuh"

namespace stmoe_dev {

constexpr int kLoraThreads = 256, kLoraWarps = kLoraThreads / kWarp;
constexpr int kLoraMaxRank = 256, kLoraMaxAdapters = 1024;
constexpr int kLoraPos = 8;         // rows of a tile of the kernels for few rows: one MMA's columns
constexpr int kLoraStep = 32;       // inner elements of a step: 16 bytes a lane, four lanes a row
constexpr int kLoraRankBlock = 64;  // ranks of a CTA
constexpr int kLoraOutBlock = 512;  // outputs of a CTA

struct LoraArgs {
    const void *x;          // [T][I]
    long long x_stride;     // elements, as all strides here
    const void *a, *b;      // [n][r][I], [n][O][r]
    long long a_group, a_row, b_group, b_row;
    const int *order, *ids; // row at a position; adapter of a row
    const int *counts;      // [n]
    const int *starts;      // [n + 1]
    const float *scale;     // [n] or nullptr (1)
    float alpha;
    int T, n, r, I, O;
    int splits;             // of I
    int steps;              // steps of a split
    int rp;                 // ranks of a row of part: r rounded up to 8
    float *part;            // [splits][T][rp], by position (tile kernels: [T][rp], the parts added up)
    const void *base;       // [T][O] or nullptr
    long long base_stride;
    void *out;              // [T][O]
    long long out_stride;
    bool out_vec;           // rows of base and out are 16-byte aligned
    bool keep;              // out is base: rows without an adapter are there already
    float *hidden;          // [T][r] or nullptr: h by row
    int polls;              // limit of every wait of the tile kernels
    bool b_padded;          // rows of B hold zeros up to a multiple of 8 ranks
    bool early;             // the kernel before in the stream is one of this call's (see below)
};

// Ahead of pdl_wait: every kernel here waits for the one before it and only then lets the one behind it start.  So when a kernel of this
// call starts behind another one of this call, all that ran before that other one is complete, and the grouping, the operands and
// the base, which none of them writes, can be read at once; only what the kernel before wrote, and all writing, stays behind
// the wait.

// D += A B for one 16 x 8 x 16 step (A 16 x 16 by rows, B 16 x 8 by columns); F32 accumulators.
template <int DT> __device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (DT == 1)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// One step of 32 inner elements: every lane holds eight neighbouring ones of its row (16 bytes).  Which of them stands in
// which inner slot of the MMA does not matter as long as both operands agree.
template <int DT> __device__ __forceinline__ void mma32(float (&d)[4], const uint4 &lo, const uint4 &hi, const uint4 &b)
{
    mma16<DT>(d, lo.x, hi.x, lo.y, hi.y, b.x, b.y);
    mma16<DT>(d, lo.z, hi.z, lo.w, hi.w, b.z, b.w);
}

// Elements k .. k+7 of a row of n, zeros behind its end (or all, if off).  VEC: rows 16-byte aligned, n a multiple of 8.
template <int DT, bool VEC> __device__ __forceinline__ uint4 lora_load8(const typename Elem<DT>::T *row, int k, int n, bool on)
{
    uint4 q = make_uint4(0, 0, 0, 0);
    if constexpr (VEC) {
        if (on && k < n) q = *reinterpret_cast<const uint4 *>(row + k);
    } else {
        uint32_t w[4] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (on && k + i < n) w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[k + i] << (16 * (i & 1));
        q = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return q;
}

// Row at a position (-1: none) and its adapter (-1: none).
__device__ __forceinline__ int lora_row(const LoraArgs &a, int p)
{
    const int row = p < a.T ? a.order[p] : -1;
    return (unsigned)row < (unsigned)a.T ? row : -1;
}
__device__ __forceinline__ int lora_adapter(const LoraArgs &a, int row)
{
    const int g = row >= 0 ? a.ids[row] : -1;
    return (unsigned)g < (unsigned)a.n ? g : -1;
}
// The tile that begins at position p, of up to eight positions within one block of eight and one adapter: how many, 0 if p is
// not its first.  row, g: those of position p + lane % 8.
__device__ __forceinline__ int lora_tile(const LoraArgs &a, int p, int lane, int &row, int &g, int &first)
{
    const int at = p + lane % kLoraPos;
    row = at <= (p | (kLoraPos - 1)) ? lora_row(a, at) : -1;
    g = lora_adapter(a, row);
    first = __shfl_sync(kFull, g, 0);
    if (p % kLoraPos && lora_adapter(a, lora_row(a, p - 1)) == first) return 0;
    const uint32_t other = __ballot_sync(kFull, row < 0 || g != first) & ((1u << kLoraPos) - 1);
    return other ? __ffs(other) - 1 : kLoraPos;
}

// h of a tile of up to eight positions, for one part of the inner dimension and up to 64 ranks: part[split][p][r].  Ranks are the
// MMA's rows and positions its columns; A and x go from memory to the operands' registers, no shared memory between, since neither
// is read twice.  Warps take steps in turn and add their sums through shared memory in order.
template <int DT, bool VEC> __global__ void __launch_bounds__(kLoraThreads) lora_down_kernel(const LoraArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int kTiles = kLoraRankBlock / 16;
    __shared__ float s_sum[kLoraWarps][kLoraPos][kLoraRankBlock + 1];
    const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp, q = lane % 4, o = lane / 4;
    pdl_wait();
    pdl_launch_dependents();
    const int p = blockIdx.x, r0 = blockIdx.z * kLoraRankBlock;
    int row8, g8, g;
    const int count = lora_tile(a, p, lane, row8, g8, g);
    if (count == 0 || g < 0) return;
    const int row = __shfl_sync(kFull, row8, o);
    const bool there = o < count;
    const T *const x = reinterpret_cast<const T *>(a.x) + (there ? row : 0) * a.x_stride;
    const T *const w = reinterpret_cast<const T *>(a.a) + g * a.a_group;
    const int tiles = min(kTiles, (a.r - r0 + 15) / 16);
    float d[kTiles][4] = {};
    const int from = blockIdx.y * a.steps, to = min(from + a.steps, (a.I + kLoraStep - 1) / kLoraStep);
#pragma unroll 2
    for (int s = from + warp; s < to; s += kLoraWarps) {
        const int k = s * kLoraStep + q * 8;
        const uint4 xv = lora_load8<DT, VEC>(x, k, a.I, there);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
            if (i < tiles) {
                const int ra = r0 + i * 16 + o, rb = ra + 8;
                const uint4 lo = lora_load8<DT, VEC>(w + ra * a.a_row, k, a.I, ra < a.r), hi = lora_load8<DT, VEC>(w + rb * a.a_row, k, a.I, rb < a.r);
                mma32<DT>(d[i], lo, hi, xv);
            }
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
        if (i < tiles) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s_sum[warp][2 * q + (j & 1)][i * 16 + o + (j & 2) * 4] = d[i][j];
        }
    __syncthreads();
    const int cols = min(tiles * 16, a.rp - r0);
    for (int i = threadIdx.x; i < count * cols; i += kLoraThreads) {
        const int pos = i / cols, r = i % cols;
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < kLoraWarps; ++v) sum += s_sum[v][pos][r];
        a.part[((long long)blockIdx.y * a.T + p + pos) * a.rp + r0 + r] = sum;
    }
}

// The power of two that brings `most` into [2^14, 2^15) (fp16 planes; 1 for bf16, which has fp32's range).
template <int DT> __device__ __forceinline__ float plane_scale(float most)
{
    if (DT == 1 || !(most > 0.f) || most == INFINITY) return 1.f;
    const int e = (int)(__float_as_uint(most) >> 23) - 127;      // floor(log2), -127 for denormals
    return __uint_as_float((uint32_t)(min(14 - e, 100) + 127) << 23);
}
// v as a sum of 16-bit values; nothing is added to an infinity.
template <int DT, int PL> __device__ __forceinline__ void planes_of(float v, uint16_t (&out)[PL])
{
    using T = typename Elem<DT>::T;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        const T h = Elem<DT>::from_f32(v);
        out[i] = *reinterpret_cast<const uint16_t *>(&h);
        const float f = Elem<DT>::to_f32(h);
        v = fabsf(f) == INFINITY ? 0.f : v - f;
    }
}

// out = base + c h B^T for a tile of up to eight positions and 512 outputs, which are the MMA's rows.  Sums leave through shared
// memory in whole lines.
template <int DT, int DO, int PL, bool VEC> __global__ void __launch_bounds__(kLoraThreads) lora_up_kernel(const LoraArgs a)
{
    using T = typename Elem<DT>::T;
    using TO = typename Elem<DO>::T;
    constexpr int kTiles = kLoraOutBlock / 16 / kLoraWarps, kPitch = kLoraMaxRank + 8;
    __shared__ __align__(16) uint16_t s_h[PL][kLoraPos][kPitch];
    __shared__ __align__(16) float s_out[kLoraPos][kLoraOutBlock + 4];
    __shared__ float s_factor[kLoraPos];
    __shared__ int s_row[kLoraPos];
    const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp, q = lane % 4, o = lane / 4;
    const int p = blockIdx.x, o0 = blockIdx.y * kLoraOutBlock;
    int row8, g8, g;
    const int count = lora_tile(a, p, lane, row8, g8, g);
    const T *const w = reinterpret_cast<const T *>(a.b) + max(g, 0) * a.b_group;
    uint4 lo[kTiles], hi[kTiles];
    auto load_b = [&](int k) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            const int oa = o0 + (warp + i * kLoraWarps) * 16 + o, ob = oa + 8;
            lo[i] = lora_load8<DT, VEC>(w + oa * a.b_row, k + q * 8, a.r, oa < a.O);
            hi[i] = lora_load8<DT, VEC>(w + ob * a.b_row, k + q * 8, a.r, ob < a.O);
        }
    };
    if (count > 0 && g >= 0) load_b(0);
    pdl_wait();
    pdl_launch_dependents();
    const bool keep = g < 0 && a.keep;          // nothing of out to write; hidden still gets its zeros
    if (count == 0 || (keep && !(a.hidden && blockIdx.y == 0))) return;
    if (warp == 0 && lane < kLoraPos) s_row[lane] = row8;
    if (g >= 0) {
        // a warp a position: its ranks' sum over the parts, then the planes
        const int wide = (a.r + kLoraStep - 1) / kLoraStep * kLoraStep;
        float h[kLoraMaxRank / kWarp], most = 0.f;
#pragma unroll
        for (int i = 0; i < kLoraMaxRank / kWarp; ++i) {
            const int r = i * kWarp + lane;
            h[i] = 0.f;
            if (warp < count && r < a.r) {
                const float *const part = a.part + (long long)(p + warp) * a.rp + r;
#pragma unroll 8
                for (int s = 0; s < a.splits; ++s) h[i] += part[(long long)s * a.T * a.rp];
            }
            most = fmaxf(most, fabsf(h[i]));
        }
        most = warp_max(most);
        const float up = plane_scale<DT>(most);
        const int row = __shfl_sync(kFull, row8, warp);
#pragma unroll
        for (int i = 0; i < kLoraMaxRank / kWarp; ++i) {
            const int r = i * kWarp + lane;
            if (r < wide) {
                uint16_t pl[PL];
                planes_of<DT, PL>(h[i] * up, pl);
#pragma unroll
                for (int j = 0; j < PL; ++j) s_h[j][warp][r] = pl[j];
            }
            if (a.hidden && blockIdx.y == 0 && warp < count && r < a.r) a.hidden[(long long)row * a.r + r] = h[i];
        }
        if (lane == 0) s_factor[warp] = a.alpha * (a.scale ? a.scale[g] : 1.f) / up;
        __syncthreads();
        float d[kTiles][4] = {};
        for (int k0 = 0; k0 < wide; k0 += kLoraStep) {
            if (k0 > 0) load_b(k0);
#pragma unroll
            for (int j = 0; j < PL; ++j) {
                const uint4 hv = *reinterpret_cast<const uint4 *>(&s_h[j][o][k0 + q * 8]);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) mma32<DT>(d[i], lo[i], hi[i], hv);
            }
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s_out[2 * q + (j & 1)][(warp + i * kLoraWarps) * 16 + o + (j & 2) * 4] = d[i][j];
    } else if (a.hidden && blockIdx.y == 0) {
        for (int i = threadIdx.x; i < count * a.r; i += kLoraThreads) {
            const int row = lora_row(a, p + i / a.r);
            if (row >= 0) a.hidden[(long long)row * a.r + i % a.r] = 0.f;
        }
        if (keep) return;
    }
    __syncthreads();
    const int here = min(kLoraOutBlock, a.O - o0);
    for (int i = threadIdx.x; i < count * (kLoraOutBlock / 8); i += kLoraThreads) {
        const int pos = i / (kLoraOutBlock / 8), c = i % (kLoraOutBlock / 8) * 8;
        if (c >= here) continue;
        const long long row = s_row[pos];
        float v[8] = {};
        if (a.base) row_load8<DO>(reinterpret_cast<const TO *>(a.base) + row * a.base_stride + o0, c, here, a.out_vec, v);
        if (g >= 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf(s_factor[pos], s_out[pos][c + j], v[j]);
        }
        row_store8<DO>(reinterpret_cast<TO *>(a.out) + row * a.out_stride + o0, c, here, a.out_vec, v);
    }
}

// ---- gradients of A and B ------------------------------------------------------------------------

// m [n][rows][cols] -> t [n][cols][ld], two such in one launch
struct LoraTransposeArgs {
    const uint16_t *m[2];
    uint16_t *t[2];
    long long m_group[2], m_row[2], t_row[2];
    int rows[2], cols[2], tiles[2];     // tiles of 32 x 32 in one of the n matrices
};
__global__ void __launch_bounds__(kLoraThreads) lora_transpose_kernel(const LoraTransposeArgs a)
{
    __shared__ uint16_t s[32][33];
    pdl_wait();
    pdl_launch_dependents();
    const int w = (int)blockIdx.x >= a.tiles[0], tile = blockIdx.x - (w ? a.tiles[0] : 0), across = (a.cols[w] + 31) / 32;
    const int r0 = tile / across * 32, c0 = tile % across * 32, x = threadIdx.x % 32, y = threadIdx.x / 32;
    const uint16_t *const m = a.m[w] + blockIdx.y * a.m_group[w];
    uint16_t *const t = a.t[w] + blockIdx.y * a.t_row[w] * a.cols[w];
#pragma unroll
    for (int i = y; i < 32; i += kLoraWarps)
        if (r0 + i < a.rows[w] && c0 + x < a.cols[w]) s[i][x] = m[(r0 + i) * a.m_row[w] + c0 + x];
    __syncthreads();
#pragma unroll
    for (int i = y; i < 32; i += kLoraWarps)
        if (c0 + i < a.cols[w] && r0 + x < a.t_row[w]) t[(c0 + i) * a.t_row[w] + r0 + x] = r0 + x < a.rows[w] ? s[x][i] : 0;   // zeros behind a row
}

// Rows that are not 16-byte aligned, copied into rows of ld (a multiple of 8) with zeros behind them, up to three matrices a launch: by lanes side by
// side once, instead of element by element, sixteen bytes apart, in the products (4318 rows of 5147: 107 us in the first product, so 19 for the copy and 16).
struct LoraPackArgs {
    struct Matrix {
        const uint16_t *from;   // [groups][rows][cols]
        uint16_t *to;           // [groups][rows][ld]
        long long group, row;
        int rows, cols, ld, parts;
        long long tasks;        // warps: groups * rows * parts
    } m[3];
};
constexpr int kPackCols = 512;
__global__ void __launch_bounds__(kLoraThreads) lora_pack_kernel(const __grid_constant__ LoraPackArgs a)
{
    constexpr int kEach = kPackCols / kWarp;
    const int lane = threadIdx.x % kWarp;
    pdl_wait();
    pdl_launch_dependents();
    long long task = (long long)blockIdx.x * kLoraWarps + threadIdx.x / kWarp;
    int w = 0;
    while (w < 2 && task >= a.m[w].tasks) task -= a.m[w++].tasks;
    const LoraPackArgs::Matrix &m = a.m[w];
    if (task >= m.tasks) return;
    const long long row = task / m.parts;
    const int at = (int)(task - row * m.parts) * kPackCols + lane;
    const uint16_t *const from = m.from + row / m.rows * m.group + row % m.rows * m.row + at;
    uint16_t *const to = m.to + row * m.ld + at;
    uint16_t v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = at + i * kWarp < m.cols ? from[i * kWarp] : 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (at + i * kWarp < m.ld) to[i * kWarp] = v[i];
}

constexpr int kGradCols = 256;      // columns of a CTA: 32 a warp
constexpr int kGradPos = 32;        // positions of a step
constexpr int kGradSmem = 87 * 1024;

struct LoraGradArgs {
    const float *u;         // [T][r] by row
    const void *z;          // [T][C]
    long long z_stride;
    const int *order, *counts, *starts;
    const float *scale;
    float alpha;
    int T, n, r, C;
    int task_rows;          // positions of a task, a multiple of kGradPos
    bool vec;               // rows of z are 16-byte aligned
    bool u_vec;             // rows of u are
    bool by_col;            // grad [n][C][r], else [n][r][C]
    void *grad;
    float *part;            // [parts][r * C], laid out as grad: tasks of adapters that have several
    int parts;
};
// The gradients of A and of B in one launch: column blocks of the first, then of the second (either may be left out).
struct LoraGradPair {
    LoraGradArgs g[2];
    int blocks;             // of the first
};

struct LoraTask {
    int g, index, tasks, several;   // adapter, which of its tasks, how many, tasks of earlier adapters that have several
};
// Task t of all (an adapter without rows has one too, which writes zeros); false behind the last.  By the whole CTA.
__device__ __forceinline__ bool lora_task(const LoraGradArgs &a, int t, LoraTask &out)
{
    __shared__ int s_sum[2][kLoraWarps];
    __shared__ LoraTask s_task;
    const int tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp;
    constexpr int kEach = kLoraMaxAdapters / kLoraThreads;
    int mine[kEach], all = 0, several = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int g = tid * kEach + i;
        mine[i] = g < a.n ? max(1, (a.counts[g] + a.task_rows - 1) / a.task_rows) : 0;
        all += mine[i], several += mine[i] > 1 ? mine[i] : 0;
    }
    int x = all, y = several;
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
        const int tx = __shfl_up_sync(kFull, x, o), ty = __shfl_up_sync(kFull, y, o);
        if (lane >= o) x += tx, y += ty;
    }
    if (lane == kWarp - 1) s_sum[0][warp] = x, s_sum[1][warp] = y;
    if (tid == 0) s_task.g = -1;
    __syncthreads();
    int at = x - all, sev = y - several;
    for (int w = 0; w < warp; ++w) at += s_sum[0][w], sev += s_sum[1][w];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (t >= at && t < at + mine[i]) s_task = {tid * kEach + i, t - at, mine[i], sev};
        at += mine[i], sev += mine[i] > 1 ? mine[i] : 0;
    }
    __syncthreads();
    out = s_task;
    return out.g >= 0;
}

__device__ __forceinline__ void ldmatrix4t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

// One task's sum over its positions of z[p][c] u[p][r] for 256 columns and up to 64 ranks.  Columns are the MMA's rows, positions its inner
// dimension: z lies in shared memory as in memory and is read transposed, u as planes by rank, 32 columns a warp.  What bounds it is issue
// slots: every CTA turns the same u into planes, which 256 columns share (with 128, and all 64 ranks converted where there were 24, 4099 rows of 2048
// and 2816 columns took 26 and 37 us, now 31 for both).  A step of 32 positions costs one barrier: behind barrier i the MMAs of step i run while z
// is on its way for steps up to i + 3, u is turned into planes for step i + 1, the largest magnitude of step i + 2 is found (fp16 planes), which the
// next barrier publishes, and u is asked for for step i + 3.  The planes' power of two follows the largest u so far, the sums with it.
template <int DT> __global__ void __launch_bounds__(kLoraThreads, 2) lora_grad_kernel(const __grid_constant__ LoraGradPair pair)
{
    const bool second = (int)blockIdx.y >= pair.blocks;
    const LoraGradArgs &a = pair.g[second];
    const int block = blockIdx.y - (second ? pair.blocks : 0);
    using T = typename Elem<DT>::T;
    constexpr int PL = 2, kTiles = kLoraRankBlock / 8, kZ = kGradCols + 8, kU = kGradPos + 8, kRing = 4;
    struct Steps {
        T z[kRing][kGradPos][kZ];
        uint16_t u[2][PL][kLoraRankBlock][kU];
    };
    extern __shared__ __align__(16) uint8_t smem[];
    Steps &s = *reinterpret_cast<Steps *>(smem);
    float *const s_out = reinterpret_cast<float *>(smem);       // [64][kGradCols + 1], behind the last step
    static_assert(sizeof(Steps) <= kGradSmem && kLoraRankBlock * (kGradCols + 1) * 4 <= kGradSmem, "");
    static_assert(kGradPos == kWarp && kGradCols == 8 * kWarp, "a lane is a position of u, and a piece of a row of z");
    __shared__ float s_most[2][kLoraWarps];
    const int tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp, q = lane % 4, o = lane / 4;
    LoraTask task;
    if (!lora_task(a, blockIdx.x, task) || (task.tasks > 1 && task.several + task.index >= a.parts)) {   // behind the last; counts of more rows than there are
        pdl_wait();
        return;
    }
    const int c0 = block * kGradCols, r0 = blockIdx.z * kLoraRankBlock, here = min(kGradCols, a.C - c0), ranks = min(kLoraRankBlock, a.r - r0);
    const int begin = a.starts[task.g] + task.index * a.task_rows;
    const int count = max(0, min(a.task_rows, a.counts[task.g] - task.index * a.task_rows)), steps = (count + kGradPos - 1) / kGradPos;
    const T *const z = reinterpret_cast<const T *>(a.z) + c0 + lane * 8;
    const int ur = warp * 8;             // u: a lane a position, a warp eight ranks
    auto row_of = [&](int i) {           // row of the lane's position of step i, -1 behind the task's last
        const int at = i * kGradPos + lane, row = at < count && (unsigned)(begin + at) < (unsigned)a.T ? a.order[begin + at] : -1;
        return (unsigned)row < (unsigned)a.T ? row : -1;
    };
    auto fetch = [&](int i, int row) {   // z: a warp a row, positions warp + 8 j
#pragma unroll
        for (int j = 0; j < kGradPos / kLoraWarps; ++j) {
            const int pos = warp + j * kLoraWarps, of = __shfl_sync(kFull, row, pos);
            T *const dst = &s.z[i % kRing][pos][lane * 8];
            const T *const src = z + (of >= 0 ? of : 0) * a.z_stride;
            if (a.vec && lane * 8 + 8 <= here) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dsmem_u32(dst)), "l"(src), "r"(of >= 0 ? 16 : 0) : "memory");
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e] = of >= 0 && lane * 8 + e < here ? src[e] : Elem<DT>::from_f32(0.f);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto load_u = [&](int row, float (&u)[8]) {
        const float *const p = a.u + (long long)(row >= 0 ? row : 0) * a.r + r0 + ur;
        if (a.u_vec && ur + 8 <= ranks) {
            const float4 x = row >= 0 ? ld_f4(p) : float4{}, y = row >= 0 ? ld_f4(p + 4) : float4{};
            u[0] = x.x, u[1] = x.y, u[2] = x.z, u[3] = x.w, u[4] = y.x, u[5] = y.y, u[6] = y.z, u[7] = y.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = row >= 0 && ur + j < ranks ? p[j] : 0.f;
        }
    };
    auto publish = [&](int i, const float (&u)[8]) {
        if (DT == 1) return;
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(u[j]));
        most = warp_max(most);
        if (lane == 0) s_most[i & 1][warp] = most;
    };
    float largest = 0.f;                 // |u| of the steps up to the one whose planes are next
    auto scale_of = [&](int i) {
        if constexpr (DT == 1) return 1.f;
        else {
#pragma unroll
            for (int w = 0; w < kLoraWarps; ++w) largest = fmaxf(largest, s_most[i & 1][w]);
            return plane_scale<DT>(largest);
        }
    };
    auto put_planes = [&](int i, float up, const float (&u)[8]) {
        if (ur >= ranks) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint16_t pl[PL];
            planes_of<DT, PL>(u[j] * up, pl);
#pragma unroll
            for (int p = 0; p < PL; ++p) s.u[i & 1][p][ur + j][lane] = pl[p];
        }
    };
    float sum[2][kTiles][4] = {}, u0[8], u1[8];
    const int row0 = row_of(0), row1 = row_of(1);
    int row = row_of(2);
    fetch(0, row0), fetch(1, row1), fetch(2, row);
    pdl_wait();                          // u and the parts' room may be the kernel before's
    pdl_launch_dependents();
    load_u(row0, u0), load_u(row1, u1);
    publish(0, u0), publish(1, u1);
    __syncthreads();
    float up = scale_of(0), scaled = up;          // of the planes that are next for the MMAs, and of the sums
    put_planes(0, up, u0);
    load_u(row, u0);
    row = row_of(3);
    // convert: u of step i + 1, then of step i + 3; ahead: of step i + 2
    auto step = [&](int i, float (&convert)[8], const float (&ahead)[8]) {
        asm volatile("cp.async.wait_group 2;" ::: "memory");
        __syncthreads();
        fetch(i + 3, row);
        const float next = scale_of(i + 1);
        put_planes(i + 1, next, convert);
        load_u(row, convert);
        row = row_of(i + 4);
        publish(i + 2, ahead);
        if (DT != 1 && up != scaled) {            // a larger u than any before
            const float f = up / scaled;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < kTiles; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[m][j][e] *= f;
            scaled = up;
        }
        up = next;
#pragma unroll
        for (int k = 0; k < kGradPos; k += 16) {
            uint32_t za[2][4];
#pragma unroll
            for (int m = 0; m < 2; ++m) ldmatrix4t(dsmem_u32(&s.z[i % kRing][k + (lane & 7) + (lane & 16) / 2][warp * 32 + m * 16 + (lane & 8)]), za[m]);
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
                if (j * 8 < ranks) {
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        const uint16_t *const col = &s.u[i & 1][p][j * 8 + o][k + 2 * q];
                        const uint32_t b0 = *reinterpret_cast<const uint32_t *>(col), b1 = *reinterpret_cast<const uint32_t *>(col + 8);
#pragma unroll
                        for (int m = 0; m < 2; ++m) mma16<DT>(sum[m][j], za[m][0], za[m][1], za[m][2], za[m][3], b0, b1);
                    }
                }
        }
    };
    for (int i = 0; i < steps; i += 2) {
        step(i, u1, u0);
        if (i + 1 < steps) step(i + 1, u0, u1);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const float c = a.alpha * (a.scale ? a.scale[task.g] : 1.f) / scaled;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 0; m < 2; ++m) s_out[(i * 8 + 2 * q + (j & 1)) * (kGradCols + 1) + warp * 32 + m * 16 + o + (j & 2) * 4] = c * sum[m][i][j];
    __syncthreads();
    const long long size = (long long)a.r * a.C;
    T *const grad = reinterpret_cast<T *>(a.grad) + task.g * size;
    float *const part = a.part + (task.several + task.index) * size;
    for (int i = tid; i < ranks * here; i += kLoraThreads) {
        const int r = a.by_col ? i % ranks : i / here, col = a.by_col ? i / ranks : i % here;
        const float v = s_out[r * (kGradCols + 1) + col];
        const long long at = a.by_col ? (long long)(c0 + col) * a.r + r0 + r : (long long)(r0 + r) * a.C + c0 + col;
        if (task.tasks == 1) grad[at] = Elem<DT>::from_f32(v);
        else part[at] = v;
    }
}

// Adapters of several tasks: their sums, in order.
template <int DT> __global__ void __launch_bounds__(kLoraThreads) lora_grad_sum_kernel(const __grid_constant__ LoraGradPair pair)
{
    const LoraGradArgs &a = pair.g[pair.blocks ? blockIdx.z : 1];
    using T = typename Elem<DT>::T;
    __shared__ int s_sum[kLoraWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int g = blockIdx.x, tasks = max(1, (a.counts[g] + a.task_rows - 1) / a.task_rows);
    if (tasks == 1) return;
    int several = 0;
    for (int e = threadIdx.x; e < g; e += kLoraThreads) {
        const int n = (a.counts[e] + a.task_rows - 1) / a.task_rows;
        several += n > 1 ? n : 0;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) several += __shfl_xor_sync(kFull, several, o);
    if (threadIdx.x % kWarp == 0) s_sum[threadIdx.x / kWarp] = several;
    __syncthreads();
    several = 0;
#pragma unroll
    for (int w = 0; w < kLoraWarps; ++w) several += s_sum[w];
    if (several + tasks > a.parts) return;
    const long long size = (long long)a.r * a.C;
    const float *const part = a.part + several * size;
    T *const grad = reinterpret_cast<T *>(a.grad) + g * size;
    for (long long i = (long long)blockIdx.y * kLoraThreads + threadIdx.x; i < size; i += (long long)gridDim.y * kLoraThreads) {
        float sum = 0.f;
        for (int t = 0; t < tasks; ++t) sum += part[t * size + i];
        grad[i] = Elem<DT>::from_f32(sum);
    }
}

}  // namespace stmoe_dev
