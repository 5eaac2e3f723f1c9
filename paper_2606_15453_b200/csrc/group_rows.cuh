// Rows grouped by expert (or by adapter), carried into that order and back.
//
//   group      ids [T][K] -> counts[g], starts[g] = where group g begins, order[s] = which pair t K + k stands at slot s (stable: pairs of a group in their
//              order; pairs without a group behind the last), slots[t][k] = its slot, -1 without a group
//   dispatch   out[slots[t][k]] = x[t]
//   combine    out[t] = r[t] + c sum_k w[t][k] y[slots[t][k]], in fp32 in the order of k, rounded once
//   backward   dy[slots[t][k]] = c w[t][k] g[t];  dw[t][k] = c <g[t], y[slots[t][k]]>
//
// Grouping is a counting sort.  Every warp owns a stretch of pairs and counts it into its own row of a table in
// shared memory, 32 pairs at a time: lanes with the same id find one another, the first adds their number, so
// neither pass has an atomic and equal ids keep their order.  Running sums down the table and across the groups
// give each warp its place in each group, and a second walk hands the places out.  Few pairs are one CTA's work, more that of a cluster, whose
// CTAs read one another's counts from shared memory; beyond that CTAs count in a first launch and place in a second.
//
// The copies are HBM's work: a row of x is read once and written K times, a row of y is read once.
#pragma once
#include <type_traits>

#include "row_utils.cuh"
#include "tcgen05_utils.cuh"

namespace stmoe_dev {

constexpr int kGrpMaxGroups = 1024;
constexpr int kGrpThreads = 512, kGrpWarps = kGrpThreads / kWarp;
constexpr int kGrpCtaPairs = 4096;  // pairs of a CTA of a cluster, or alone
constexpr int kGrpCluster = 8, kGrpMaxCtas = 128;

struct GroupArgs {
    const int *ids;
    int pairs, G;
    int per_warp;           // pairs of a warp, a multiple of 32
    int *counts, *starts, *order, *slots;
    int *hist;              // [ctas][G + 1], or nullptr: one CTA, or the CTAs of a cluster
};

// Column of a pair: its group, or G without one.
__device__ __forceinline__ int grp_id(const GroupArgs &a, int p)
{
    const int e = a.ids[p];
    return (unsigned)e < (unsigned)a.G ? e : a.G;
}
// Counts of a warp's stretch in its row of the table, columns 0..G.
__device__ __forceinline__ void grp_count(const GroupArgs &a, int first, int lane, int *row)
{
    const int end = min(first + a.per_warp, a.pairs);
    for (int p = first + lane; p - lane < end; p += kWarp) {
        const int e = p < end ? grp_id(a, p) : -1;
        const unsigned same = __match_any_sync(kFull, e);
        if (e >= 0 && lane == __ffs(same) - 1) row[e] += __popc(same);
        __syncwarp();
    }
}
__device__ __forceinline__ int grp_first(const GroupArgs &a, int warp)
{
    const long long p = ((long long)blockIdx.x * kGrpWarps + warp) * a.per_warp;
    return p < a.pairs ? (int)p : a.pairs;
}
// Exclusive running sums over the columns 0..G of total, in place, by the whole CTA.
__device__ __forceinline__ void grp_scan(int *total, int n, int *part)
{
    const int tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp;
    int carry = 0;
    for (int at = 0; at < n; at += kGrpThreads) {
        const int v = at + tid < n ? total[at + tid] : 0;
        int s = v;
#pragma unroll
        for (int o = 1; o < kWarp; o <<= 1) {
            const int t = __shfl_up_sync(kFull, s, o);
            if (lane >= o) s += t;
        }
        if (lane == kWarp - 1) part[warp] = s;
        __syncthreads();
        int before = carry, all = carry;
#pragma unroll
        for (int w = 0; w < kGrpWarps; ++w) {
            if (w < warp) before += part[w];
            all += part[w];
        }
        if (at + tid < n) total[at + tid] = before + s - v;
        carry = all;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kGrpThreads) group_count_kernel(const GroupArgs a)
{
    extern __shared__ int table[];              // [kGrpWarps][G + 1]
    const int n = a.G + 1, tid = threadIdx.x, warp = tid / kWarp;
    for (int i = tid; i < kGrpWarps * n; i += kGrpThreads) table[i] = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    grp_count(a, grp_first(a, warp), tid % kWarp, table + warp * n);
    __syncthreads();
    for (int g = tid; g < n; g += kGrpThreads) {
        int sum = 0;
#pragma unroll
        for (int w = 0; w < kGrpWarps; ++w) sum += table[w * n + g];
        a.hist[blockIdx.x * n + g] = sum;
    }
}

__global__ void __launch_bounds__(kGrpThreads) group_place_kernel(const GroupArgs a)
{
    extern __shared__ int table[];              // [kGrpWarps][G + 1], [G + 1] starts, [G + 1] own counts
    __shared__ int part[kGrpWarps];
    __shared__ int2 sums[kGrpThreads];
    const int n = a.G + 1, tid = threadIdx.x, lane = tid % kWarp, warp = tid / kWarp, ctas = gridDim.x, me = blockIdx.x;
    int *const start = table + kGrpWarps * n, *const own = start + n, *const mine = table + warp * n;
    for (int i = tid; i < kGrpWarps * n; i += kGrpThreads) table[i] = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const int first = grp_first(a, warp), end = min(first + a.per_warp, a.pairs);
    grp_count(a, first, lane, mine);
    __syncthreads();
    if (!a.hist) {
        for (int g = tid; g < n; g += kGrpThreads) {
            int sum = 0;
#pragma unroll
            for (int w = 0; w < kGrpWarps; ++w) sum += table[w * n + g];
            own[g] = sum;
        }
        if (ctas > 1) cluster_sync();
        else __syncthreads();
    }
    // the CTAs' counts of a column, by as many threads as there are for one
    int share = 1;
    while (2 * share * n <= kGrpThreads && share < 8) share *= 2;
    const int columns = kGrpThreads / share, col = tid % columns, of = tid / columns;
    for (int g0 = 0; g0 < n; g0 += columns) {
        const int g = g0 + col;
        int before = 0, total = 0;              // in this group: pairs of the CTAs before this one, of all
        if (g < n) {
            if (a.hist) {
#pragma unroll 16
                for (int c = of; c < ctas; c += share) {
                    const int h = a.hist[c * n + g];
                    before += c < me ? h : 0;
                    total += h;
                }
            } else {
                for (int c = of; c < ctas; c += share) {
                    const int h = ctas == 1 ? own[g] : __float_as_int(ld_cluster(dsmem_u32(own + g), c));
                    before += c < me ? h : 0;
                    total += h;
                }
            }
        }
        if (share > 1) {
            __syncthreads();
            sums[tid] = make_int2(before, total);
            __syncthreads();
            if (of == 0)
                for (int i = 1; i < share; ++i) before += sums[i * columns + col].x, total += sums[i * columns + col].y;
        }
        if (g < n && of == 0) {
            int run = before;
#pragma unroll
            for (int w = 0; w < kGrpWarps; ++w) {
                const int c = table[w * n + g];
                table[w * n + g] = run;
                run += c;
            }
            start[g] = total;
            if (me == 0 && g < a.G) a.counts[g] = total;
        }
    }
    __syncthreads();
    grp_scan(start, n, part);
    if (blockIdx.x == 0)
        for (int g = tid; g < n; g += kGrpThreads) a.starts[g] = start[g];
    for (int p = first + lane; p - lane < end; p += kWarp) {
        const int e = p < end ? grp_id(a, p) : -1;
        const unsigned same = __match_any_sync(kFull, e);
        if (e >= 0) {
            const int s = start[e] + mine[e] + __popc(same & ((1u << lane) - 1));
            a.order[s] = p;
            a.slots[p] = e < a.G ? s : -1;
        }
        __syncwarp();
        if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
        __syncwarp();
    }
    if (!a.hist && ctas > 1) {
        __syncwarp();
        cluster_sync();                         // nobody leaves while its counts are read
    }
}

// ---- rows there and back -------------------------------------------------------------------------

constexpr int kRowThreads = 256;

struct DispatchArgs {
    const uint8_t *x;
    long long x_stride, out_stride, row_bytes;   // bytes
    const int *slots;       // [T][K]
    const int *rows;        // rows in groups; those behind become 0 (nullptr: stay as they were)
    int T, K, out_rows;
    unsigned parts;         // warps that share a row; T * parts < 2^31
    uint8_t *out;
};

// U: widest type that every address of the rows is a multiple of.
template <typename U> __global__ void __launch_bounds__(kRowThreads) dispatch_rows_kernel(const DispatchArgs a)
{
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x % kWarp;
    pdl_wait();
    pdl_launch_dependents();
    const unsigned task = blockIdx.x * (kRowThreads / kWarp) + threadIdx.x / kWarp, t32 = task / a.parts;
    const long long t = t32;
    if (t >= a.T) return;
    const int n = (int)(a.row_bytes / (int)sizeof(U));
    const int first = (int)(task - t32 * a.parts) * kWarp * kAtOnce;
    const unsigned step = a.parts * kWarp * kAtOnce;           // at least n, at most 2^31: at + step is behind the row, and below 2^32
    const U *const src = reinterpret_cast<const U *>(a.x + t * a.x_stride);
    const int *const slots = a.slots + t * a.K;
    const int behind = a.rows ? *a.rows : a.out_rows;
    // one turn, as there are as many parts as it takes; without the loop the compiler asks for fewer registers, and the more CTAs an SM write
    // less evenly (16384 x 2048 bf16, K 8: 95.8 -> 97.2 us)
    for (int at = first; (unsigned)at < (unsigned)n; at = (int)(at + step)) {
        U v[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
            if (at + i * kWarp + lane < n) v[i] = src[at + i * kWarp + lane];
        for (int k = 0; k < a.K; ++k) {
            const int s = slots[k];
            if ((unsigned)s >= (unsigned)a.out_rows) continue;
            U *const dst = reinterpret_cast<U *>(a.out + s * a.out_stride);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (at + i * kWarp + lane < n) dst[at + i * kWarp + lane] = v[i];
        }
        for (long long r = max(t * a.K, (long long)behind); r < min((t + 1) * a.K, (long long)a.out_rows); ++r) {
            U *const dst = reinterpret_cast<U *>(a.out + r * a.out_stride);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (at + i * kWarp + lane < n) dst[at + i * kWarp + lane] = U{};
        }
    }
}

struct CombineArgs {
    const void *y;          // [y_rows][C]
    long long y_stride;     // elements, as all strides here
    const int *slots;       // [T][K]
    const float *w;         // [T][K] or nullptr (1)
    const void *res;        // combine: [T][C] or nullptr; backward: the gradient
    long long res_stride;
    void *out;              // combine: [T][C]; backward: gradient of y
    long long out_stride;
    float *dw;              // backward: [T][K] or nullptr
    const int *rows;        // backward: as in DispatchArgs
    float scale;
    int T, K, C, y_rows;
    unsigned parts;         // warps that share a row; T * parts < 2^31
    bool vec;               // every row is 16-byte aligned
};

// Eight elements of a row of C to a lane: neighbours where rows are aligned (columns c + 8 lane and on), else lanes side by side (c + lane + 32 i), so
// that a row is read in whole lines either way (2047 x 1001 fp16, 16 bytes apart element by element: 49 us both directions, now 35).
// WHOLE: aligned, and all 256 columns are there.
template <int DT, bool WHOLE> struct Lane8 {
    using T = typename Elem<DT>::T;
    static constexpr int V = Elem<DT>::kVec, G = 8 / V;
    uint4 q[WHOLE ? G : 1];
    float f[WHOLE ? 1 : 8];
    __device__ __forceinline__ void load(const T *row, int c, int lane, int C, bool vec, bool on)
    {
        if constexpr (WHOLE) {
#pragma unroll
            for (int g = 0; g < G; ++g) q[g] = on ? *reinterpret_cast<const uint4 *>(row + c + 8 * lane + g * V) : make_uint4(0, 0, 0, 0);
        } else {
            const T *const p = row + c + (vec ? 8 : 1) * lane;
            const int left = on ? C - c - (vec ? 8 : 1) * lane : 0;
            if (vec) {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = i < left ? Elem<DT>::to_f32(p[i]) : 0.f;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = kWarp * i < left ? Elem<DT>::to_f32(p[kWarp * i]) : 0.f;
            }
        }
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const
    {
        if constexpr (WHOLE) {
#pragma unroll
            for (int g = 0; g < G; ++g) bal_widen<DT>(q[g], reinterpret_cast<float2 *>(v) + g * V / 2);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = f[i];
        }
    }
};
template <int DT, bool WHOLE> __device__ __forceinline__ void lane_store8(typename Elem<DT>::T *row, int c, int lane, int C, bool vec, const float (&v)[8])
{
    using T = typename Elem<DT>::T;
    constexpr int V = Elem<DT>::kVec;
    if constexpr (WHOLE) {
#pragma unroll
        for (int g = 0; g < 8 / V; ++g) *reinterpret_cast<uint4 *>(row + c + 8 * lane + g * V) = bal_narrow<DT>(reinterpret_cast<const float2 *>(v) + g * V / 2);
    } else {
        T *const p = row + c + (vec ? 8 : 1) * lane;
        const int left = C - c - (vec ? 8 : 1) * lane;
        if (vec && left >= 8) {
#pragma unroll
            for (int g = 0; g < 8 / V; ++g) *reinterpret_cast<uint4 *>(p + g * V) = bal_narrow<DT>(reinterpret_cast<const float2 *>(v) + g * V / 2);
        } else if (vec) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) p[i] = Elem<DT>::from_f32(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (kWarp * i < left) p[kWarp * i] = Elem<DT>::from_f32(v[i]);
        }
    }
}

// J pieces of 256 columns of a token, from column `first` on; two of its rows at a time in all of them.
template <int DY, int DO, int J, bool WHOLE>
__device__ __forceinline__ void combine_pieces(const CombineArgs &a, long long t, int first, int lane)
{
    using TY = typename Elem<DY>::T;
    using TO = typename Elem<DO>::T;
    const TY *const y = reinterpret_cast<const TY *>(a.y);
    const int *const slots = a.slots + t * a.K;
    float sum[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        Lane8<DO, WHOLE> r;
        r.load(reinterpret_cast<const TO *>(a.res) + t * a.res_stride, first + j * kWarp * 8, lane, a.C, a.vec, a.res != nullptr);
        r.widen(sum[j]);
    }
    for (int k = 0; k < a.K; k += 2) {
        Lane8<DY, WHOLE> row[2][J];
        float w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int s = k + i < a.K ? slots[k + i] : -1;
            const bool there = (unsigned)s < (unsigned)a.y_rows;
            w[i] = there ? a.w ? a.scale * a.w[t * a.K + k + i] : a.scale : 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) row[i][j].load(y + (there ? s : 0) * a.y_stride, first + j * kWarp * 8, lane, a.C, a.vec, there);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float v[8];
                row[i][j].widen(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[j][e] = fmaf(w[i], v[e], sum[j][e]);
            }
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (WHOLE || first + j * kWarp * 8 < a.C)
            lane_store8<DO, WHOLE>(reinterpret_cast<TO *>(a.out) + t * a.out_stride, first + j * kWarp * 8, lane, a.C, a.vec, sum[j]);
}

// DY: type of y, DO: of the residual and the result.  With one piece a warp's loads were too few for its life (16384 x 4096 bf16, K 2: 120 us,
// 70 with four, where the bytes take 62, and three CTAs an SM; a fourth cost registers: 92).
template <int DY, int DO, int J> __global__ void __launch_bounds__(kRowThreads, 3) combine_rows_kernel(const CombineArgs a)
{
    const int lane = threadIdx.x % kWarp;
    pdl_wait();
    pdl_launch_dependents();
    const unsigned task = blockIdx.x * (kRowThreads / kWarp) + threadIdx.x / kWarp, t32 = task / a.parts;
    if (t32 >= (unsigned)a.T) return;
    const int first = (int)(task - t32 * a.parts) * J * kWarp * 8;
    if (a.vec && first + J * kWarp * 8 <= a.C) combine_pieces<DY, DO, J, true>(a, t32, first, lane);
    else combine_pieces<DY, DO, J, false>(a, t32, first, lane);
}

// WPT warps share a token (and reduce its inner products through shared memory, in a fixed order); KB choices at a time, so that a piece of the
// gradient is read once for them and their rows are asked for together.
template <int DY, int DG, int WPT, int KB> __global__ void __launch_bounds__(kRowThreads, KB == 2 ? 5 : 1) combine_rows_backward_kernel(const CombineArgs a)
{
    using TY = typename Elem<DY>::T;
    using TG = typename Elem<DG>::T;
    constexpr int kTokens = kRowThreads / kWarp / WPT;
    __shared__ float s_dot[KB][kRowThreads / kWarp];
    const int lane = threadIdx.x % kWarp, warp = threadIdx.x / kWarp, part = warp % WPT;
    pdl_wait();
    pdl_launch_dependents();
    const long long t = (long long)blockIdx.x * kTokens + warp / WPT;
    const bool on = t < a.T;                    // the CTA's other tokens go on to its barriers
    const TY *const y = reinterpret_cast<const TY *>(a.y);
    TY *const dy = reinterpret_cast<TY *>(a.out);
    const TG *const g = reinterpret_cast<const TG *>(a.res) + t * a.res_stride;
    for (int k = 0; k < a.K; k += KB) {
        int s[KB];
        float w[KB], dot[KB];
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            s[i] = on && k + i < a.K ? a.slots[t * a.K + k + i] : -1;
            if ((unsigned)s[i] >= (unsigned)a.y_rows) s[i] = -1;
            w[i] = s[i] < 0 ? 0.f : a.w ? a.scale * a.w[t * a.K + k + i] : a.scale;
            dot[i] = 0.f;
        }
        auto piece = [&](int c, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            Lane8<DG, WHOLE> graw;
            Lane8<DY, WHOLE> row[KB];
            graw.load(g, c, lane, a.C, a.vec, true);
#pragma unroll
            for (int i = 0; i < KB; ++i) row[i].load(y + (s[i] < 0 ? 0 : s[i]) * a.y_stride, c, lane, a.C, a.vec, s[i] >= 0 && a.dw);
            float gv[8];
            graw.widen(gv);
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                float v[8];
                row[i].widen(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) dot[i] = fmaf(gv[e], v[e], dot[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = w[i] * gv[e];
                if (s[i] >= 0) lane_store8<DY, WHOLE>(dy + s[i] * a.out_stride, c, lane, a.C, a.vec, v);
            }
        };
        constexpr int kStep = WPT * kWarp * 8;
        int c = on ? part * kWarp * 8 : a.C;
        if (a.vec) {
#pragma unroll 2
            for (; c + kWarp * 8 <= a.C; c += kStep) piece(c, std::true_type());
        }
#pragma unroll 2
        for (; c < a.C; c += kStep) piece(c, std::false_type());
        if (a.dw) {
#pragma unroll
            for (int i = 0; i < KB; ++i) dot[i] = warp_sum(dot[i]);
            if (WPT > 1) {
                __syncthreads();
                if (lane == 0) {
#pragma unroll
                    for (int i = 0; i < KB; ++i) s_dot[i][warp] = dot[i];
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < KB; ++i) {
                    dot[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < WPT; ++j) dot[i] += s_dot[i][warp - part + j];
                }
            }
            if (on && part == 0 && lane == 0) {
#pragma unroll
                for (int i = 0; i < KB; ++i)
                    if (k + i < a.K) a.dw[t * a.K + k + i] = s[i] >= 0 ? a.scale * dot[i] : 0.f;
            }
        }
    }
    if (a.rows && on) {
        const float zero[8] = {};
        for (long long r = max(t * a.K, (long long)*a.rows); r < min((t + 1) * a.K, (long long)a.y_rows); ++r)
            for (int c = part * kWarp * 8; c < a.C; c += WPT * kWarp * 8) lane_store8<DY, false>(dy + r * a.out_stride, c, lane, a.C, a.vec, zero);
    }
}

}  // namespace stmoe_dev
