// Balance loss, z loss and per-expert counts of a router over many tokens, and the gradient with
// respect to its logits.
//
//   p_t = softmax(z_t),  lse_t = log sum exp z_t,  n = rows that count
//   c_e = how often expert e stands in the ids of those rows,  f_e = c_e / (n K),  P_e = 1/n sum_t p_te
//   balance = E sum_e f_e P_e          z = 1/n sum_t lse_t^2
//   dz_te = g_balance E/n p_te (f_e - sum_j f_j p_tj) + g_z 2/n lse_t p_te      (c_e held constant)
//
// A row counts unless its mask byte is zero or all its logits are -infinity; other rows are not
// read into any sum (they may hold NaN), and their gradient is zero.
//
// Each direction reads the logits once (and the backward writes the gradient once): HBM's work.  2^j
// lanes share a row, sixteen logits each in registers (eight for rows of up to eight), so one pass gives
// maximum, sum and probabilities, and a row of 8 experts does not leave 31 lanes idle.  What competes
// with the loads is issue slots: with eight logits a lane, library reciprocal and logarithm and 64-bit
// row arithmetic the forward kernel issued 210 instructions per two rows of 128 experts and took 92 us
// for 524288 rows that HBM delivers in 23.  The exponential is exp2 of one fused multiply-add per logit
// (relative error 2^-22 for the terms that matter; the row's sum is formed from the same rounded
// exponents, so a common error of the maximum cancels); reciprocal and logarithm of the sum, which lies
// in [1, 256], are the hardware's (2^-23 relative, 2^-22 absolute).
// Sums over tokens: a lane adds the probabilities of its experts in fp32 over the few hundred rows it
// sees, a CTA adds its lanes in a fixed order, and the CTAs' partial sums are added in fp64 in a fixed
// order by a second launch: no floating-point atomics, the same bits every time.
#pragma once
#include "mx4.cuh"

namespace stmoe_dev {

constexpr int kBalThreads = 256;
constexpr int kBalMaxExperts = 256;
constexpr int kBalRows = 2;         // rows of a lane in flight
constexpr int kBalFinish = 8;       // CTAs of the cluster that adds the partial sums up
constexpr int kBalMaxCtas = 592;   // four a SM: rows of the partial-sum workspace
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// a CTA's partial sums: [E] probabilities, lse^2, then (int) [E] counts, rows
__host__ __device__ inline int bal_part_words(int E) { return 2 * (E + 1); }

struct BalanceArgs {
    const void *logits;
    long long stride;       // elements
    const int *ids;         // [T][K]
    const uint8_t *mask;    // [T] or nullptr
    int T, E, K;
    bool vec;               // rows are 16-byte aligned and E is a multiple of the vector width
    float *part;            // forward: [gridDim.x][bal_part_words(E)]
    int ctas;               // finish: rows of part
    float *loss;            // [2]
    int *counts;            // [E]
    int *rows;              // [1]
    const float *grad;      // backward: [2]
    void *dlogits;
    long long dstride;
    bool dvec;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Where lane l of a row's LPR lanes finds its N logits: in vector order (groups of 16 bytes, lane after
// lane) or one by one.
template <int DT, int LPR> __device__ __forceinline__ int bal_index(int l, int i, bool vec)
{
    constexpr int V = Elem<DT>::kVec;
    return vec ? (i / V) * (LPR * V) + l * V + i % V : i * LPR + l;
}

template <int DT, int LPR, int N>
__device__ __forceinline__ void bal_load(const typename Elem<DT>::T *row, int E, int l, bool vec, float (&z)[N])
{
    using El = Elem<DT>;
    if (vec) {
#pragma unroll
        for (int g = 0; g < N / El::kVec; ++g) {
            const int e = bal_index<DT, LPR>(l, g * El::kVec, true);
            typename El::T t[El::kVec];
            const bool in = e < E;
            if (in) *reinterpret_cast<uint4 *>(t) = ld_stream16(row + e);
#pragma unroll
            for (int i = 0; i < El::kVec; ++i) z[g * El::kVec + i] = in ? El::to_f32(t[i]) : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = i * LPR + l;
            z[i] = e < E ? El::to_f32(row[e]) : -INFINITY;
        }
    }
}

template <int LPR> __device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}
template <int LPR> __device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// z -> exp(z - max) in place, inv: 1 / their sum; returns lse.  live: the row has a logit above
// -infinity (NaN included: then the row's results are NaN, as the formulas say).
template <int LPR, int N> __device__ __forceinline__ float bal_softmax(float (&z)[N], float &inv, bool &live)
{
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    m = lanes_max<LPR>(m);
    const float m2 = m == -INFINITY ? 0.f : m * kLog2e;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = ex2(fmaf(z[i], kLog2e, -m2)), sum += z[i];
    sum = lanes_sum<LPR>(sum);
    live = sum != 0.f;   // 0 where all logits are -infinity (a NaN is not 0)
    inv = __fdividef(1.f, sum);
    return (m2 + __log2f(sum)) * kLn2;
}

// The rows of a lane: first row, rows between two of its own, and its walk through logits, choices and
// masks by pointers (a 64-bit product per row and array would cost as much as the row's exponentials).
template <typename T, int LPR> struct BalWalk {
    static constexpr int RPW = kWarp / LPR;
    long long t, step;
    const T *z;
    const uint8_t *mask;
    long long z_row, z_step;
    bool on[kBalRows];
    __device__ __forceinline__ BalWalk(const BalanceArgs &a, int warp, int sub)
    {
        constexpr int W = kBalThreads / kWarp;
        step = (long long)gridDim.x * W * RPW * kBalRows;
        t = (long long)(blockIdx.x * W + warp) * RPW * kBalRows + sub;
        z_row = RPW * a.stride, z_step = step * a.stride;
        z = reinterpret_cast<const T *>(a.logits) + t * a.stride;
        mask = a.mask ? a.mask + t : nullptr;
        masks(a);
    }
    __device__ __forceinline__ void masks(const BalanceArgs &a)
    {
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) on[r] = t + r * RPW < a.T && (!mask || mask[r * RPW]);
    }
    // to the next rows; their masks are asked for here, a step before the logits that wait for them
    __device__ __forceinline__ void next(const BalanceArgs &a)
    {
        t += step, z += z_step;
        if (mask) mask += step;
        masks(a);
    }
};

// sum: sum_e c_e sum_t p_te; sq: sum_t lse_t^2
__device__ __forceinline__ void bal_write(const BalanceArgs &a, double sum, double sq, int n)
{
    const double rn = n > 0 ? 1. / n : 0.;
    a.loss[0] = (float)(a.E * sum * rn * rn / a.K);
    a.loss[1] = (float)(sq * rn);
    *a.rows = n;
}

// One CTA's sums over its rows.  Alone (gridDim.x = 1) it writes the results, else its partial sums.
template <int DT, int LPR, int N> __global__ void __launch_bounds__(kBalThreads, 3) router_balance_kernel(const BalanceArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int RPW = kWarp / LPR, W = kBalThreads / kWarp;
    __shared__ int s_cnt[kBalMaxExperts];
    __shared__ float s_p[W][LPR * N];
    __shared__ float s_z[W];
    __shared__ int s_n[W];
    __shared__ double s_bal[W];
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    for (int e = tid; e < a.E; e += kBalThreads) s_cnt[e] = 0;
    __syncthreads();
    float p[N] = {}, zz = 0.f;
    int n = 0;
    BalWalk<T, LPR> w(a, warp, sub);
    const int *ids = a.ids + w.t * a.K + l;
    const long long ids_step = w.step * a.K;
    while (w.t - sub < a.T) {
        float z[kBalRows][N];
        int id[kBalRows];
        bool on[kBalRows];
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            on[r] = w.on[r];
            id[r] = -1;
            if (on[r]) {
                bal_load<DT, LPR>(w.z + r * w.z_row, a.E, l, a.vec, z[r]);
                if (l < a.K) id[r] = __ldg(ids + r * RPW * a.K);   // the lane's first choice, with the logits
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) z[r][i] = -INFINITY;
            }
        }
        w.next(a);
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            bool live;
            float inv;
            const float lse = bal_softmax<LPR>(z[r], inv, live);
            if (on[r] && live) {
#pragma unroll
                for (int i = 0; i < N; ++i) p[i] = fmaf(z[r][i], inv, p[i]);
                if (l == 0) zz = fmaf(lse, lse, zz), ++n;
                if ((unsigned)id[r] < (unsigned)a.E) atomicAdd(&s_cnt[id[r]], 1);
                for (int k = LPR; k + l < a.K; k += LPR) {
                    const int e = __ldg(ids + r * RPW * a.K + k);
                    if ((unsigned)e < (unsigned)a.E) atomicAdd(&s_cnt[e], 1);
                }
            }
        }
        ids += ids_step;
    }
    // the rows of a warp first (lanes with the same l), then the warps in order
#pragma unroll
    for (int o = LPR; o < kWarp; o <<= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] += __shfl_xor_sync(kFull, p[i], o);
        zz += __shfl_xor_sync(kFull, zz, o);
        n += __shfl_xor_sync(kFull, n, o);
    }
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s_p[warp][bal_index<DT, LPR>(l, i, a.vec)] = p[i];
        if (l == 0) s_z[warp] = zz, s_n[warp] = n;
    }
    __syncthreads();
    if (gridDim.x > 1) {
        float *part = a.part + (size_t)blockIdx.x * bal_part_words(a.E);
        int *ipart = reinterpret_cast<int *>(part) + a.E + 1;
        for (int e = tid; e <= a.E; e += kBalThreads) {
            float v = 0.f;
            int c = 0;
            for (int q = 0; q < W; ++q) {
                v += e < a.E ? s_p[q][e] : s_z[q];
                if (e == a.E) c += s_n[q];
            }
            part[e] = v;
            ipart[e] = e < a.E ? s_cnt[e] : c;
        }
        return;
    }
    double b = 0.;   // E <= 256 = threads
    if (tid < a.E) {
        float v = 0.f;
        for (int q = 0; q < W; ++q) v += s_p[q][tid];
        b = (double)s_cnt[tid] * (double)v;
        a.counts[tid] = s_cnt[tid];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) b += __shfl_xor_sync(kFull, b, o);
    if (lane == 0) s_bal[warp] = b;
    __syncthreads();
    if (tid == 0) {
        double sum = 0., sq = 0.;
        int rows = 0;
        for (int q = 0; q < W; ++q) sum += s_bal[q], sq += (double)s_z[q], rows += s_n[q];
        bal_write(a, sum, sq, rows);
    }
}

// One cluster: the partial sums of all CTAs, in a fixed order, and the losses.  A CTA of the cluster takes
// every kBalFinish-th row of partial sums, G threads a column; then the threads, then the CTAs in order.
__global__ void __launch_bounds__(1024) router_balance_finish_kernel(const BalanceArgs a)
{
    __shared__ double s_sum[1024];
    __shared__ int s_int[1024];
    __shared__ double s_bal[kWarp];
    const int tid = threadIdx.x, cols = a.E + 1, words = bal_part_words(a.E), rank = blockIdx.x;
    const int G = 1024 / cols, g = tid / cols, e = tid % cols;   // G >= 3: E <= 256
    pdl_wait();
    double v = 0.;
    int c = 0;
    if (g < G)
        for (int b0 = rank + kBalFinish * g; b0 < a.ctas; b0 += 8 * kBalFinish * G) {   // eight rows' words in flight
            float x[8];
            int y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = b0 + j * kBalFinish * G;
                const float *part = a.part + (size_t)b * words;
                x[j] = 0.f, y[j] = 0;
                if (b < a.ctas) x[j] = __ldcg(part + e), y[j] = __ldcg(reinterpret_cast<const int *>(part) + cols + e);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v += (double)x[j], c += y[j];
        }
    s_sum[tid] = v, s_int[tid] = c;
    __syncthreads();
    if (tid < cols) {
        for (int q = 1; q < G; ++q) v += s_sum[q * cols + tid], c += s_int[q * cols + tid];
        s_sum[tid] = v, s_int[tid] = c;   // only this thread reads or writes column tid of group 0
    }
    cluster_sync();
    if (rank == 0 && tid < cols) {
        double dv[kBalFinish];
        int dc[kBalFinish];
#pragma unroll
        for (int z = 1; z < kBalFinish; ++z) {
            uint32_t remote;
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"((uint32_t)__cvta_generic_to_shared(s_sum + tid)), "r"(z));
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(dv[z]) : "r"(remote) : "memory");
            asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"((uint32_t)__cvta_generic_to_shared(s_int + tid)), "r"(z));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(dc[z]) : "r"(remote) : "memory");
        }
#pragma unroll
        for (int z = 1; z < kBalFinish; ++z) v += dv[z], c += dc[z];
        s_sum[tid] = v, s_int[tid] = c;
    }
    cluster_sync();   // nobody leaves while its sums are read
    if (rank != 0) return;
    const int n = s_int[a.E];
    double b = 0.;
    if (tid < a.E) {
        b = (double)s_int[tid] * s_sum[tid];
        a.counts[tid] = s_int[tid];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) b += __shfl_xor_sync(kFull, b, o);
    if (tid % kWarp == 0) s_bal[tid / kWarp] = b;
    __syncthreads();
    if (tid == 0) {
        b = 0.;
        for (int w = 0; w < kBalMaxExperts / kWarp; ++w) b += s_bal[w];
        bal_write(a, b, s_sum[a.E], n);
    }
}

template <int DT, int LPR, int N> __global__ void __launch_bounds__(kBalThreads, 3) router_balance_backward_kernel(const BalanceArgs a)
{
    using El = Elem<DT>;
    using T = typename El::T;
    constexpr int RPW = kWarp / LPR;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    const int n = *a.rows;
    const float rn = n > 0 ? 1.f / (float)n : 0.f;
    const float gb = a.grad[0] * (float)a.E * rn, gz = a.grad[1] * 2.f * rn;
    // logits and gradient may be laid out differently; a lane's experts follow the vector order only
    // where both do
    const bool vec = a.vec && a.dvec;
    float f[N];   // g_balance E/n f_e
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = bal_index<DT, LPR>(l, i, vec);
        f[i] = e < a.E ? gb * ((float)a.counts[e] * rn / (float)a.K) : 0.f;
    }
    BalWalk<T, LPR> w(a, warp, sub);
    T *out = reinterpret_cast<T *>(a.dlogits) + w.t * a.dstride;
    const long long d_row = RPW * a.dstride, d_step = w.step * a.dstride;
    while (w.t - sub < a.T) {
        float z[kBalRows][N];
        bool on[kBalRows];
        const long long t = w.t;
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            on[r] = w.on[r];
            if (on[r]) {
                bal_load<DT, LPR>(w.z + r * w.z_row, a.E, l, vec, z[r]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) z[r][i] = -INFINITY;
            }
        }
        w.next(a);
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            bool live;
            float inv;
            const float lse = bal_softmax<LPR>(z[r], inv, live);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) dot = fmaf(f[i], z[r][i], dot);
            dot = lanes_sum<LPR>(dot);
            const float c = gz * lse - dot * inv;   // dz = p (gb f + gz lse - gb dot)
            const bool counts = on[r] && live;
            if (t + r * RPW >= a.T) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) z[r][i] = counts ? z[r][i] * inv * (f[i] + c) : 0.f;
            T *o = out + r * d_row;
            if (vec) {
#pragma unroll
                for (int g = 0; g < N / El::kVec; ++g) {
                    const int e = bal_index<DT, LPR>(l, g * El::kVec, true);
                    T v[El::kVec];
#pragma unroll
                    for (int i = 0; i < El::kVec; ++i) v[i] = El::from_f32(z[r][g * El::kVec + i]);
                    if (e < a.E) *reinterpret_cast<uint4 *>(o + e) = *reinterpret_cast<const uint4 *>(v);
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i * LPR + l < a.E) o[i * LPR + l] = El::from_f32(z[r][i]);
            }
        }
        out += d_step;
    }
}

}  // namespace stmoe_dev
