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
// Both directions are bound by HBM: the logits are read once (and the gradient written once).
// 2^j lanes share a row, eight logits each in registers, so one pass gives maximum, sum and
// probabilities, and a row of 8 experts does not leave 31 lanes idle.  The exponential is exp2 of
// one fused multiply-add per logit (relative error 2^-22 for the terms that matter; the row's sum is
// formed from the same rounded exponents, so a common error of the maximum cancels).
// Sums over tokens: a lane adds the probabilities of its experts in fp32 over the few hundred rows it
// sees, a CTA adds its lanes in a fixed order, and the CTAs' partial sums are added in fp64 in a fixed
// order by a second launch: no floating-point atomics, the same bits every time.
#pragma once
#include "mx4.cuh"

namespace stmoe_dev {

constexpr int kBalThreads = 256;
constexpr int kBalMaxExperts = 256;
constexpr int kBalRows = 4;         // rows of a lane in flight
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

// Where lane l of a row's lanes finds its eight logits: in vector order (groups of 16 bytes, lane
// after lane) or one by one.
template <int DT, int LPR> __device__ __forceinline__ int bal_index(int l, int i, bool vec)
{
    constexpr int V = Elem<DT>::kVec;
    return vec ? (i / V) * (LPR * V) + l * V + i % V : i * LPR + l;
}

template <int DT, int LPR>
__device__ __forceinline__ void bal_load(const typename Elem<DT>::T *row, int E, int l, bool vec, float (&z)[8])
{
    using El = Elem<DT>;
    if (vec) {
#pragma unroll
        for (int g = 0; g < 8 / El::kVec; ++g) {
            const int e = bal_index<DT, LPR>(l, g * El::kVec, true);
            typename El::T t[El::kVec];
            const bool in = e < E;
            if (in) *reinterpret_cast<uint4 *>(t) = ld_stream16(row + e);
#pragma unroll
            for (int i = 0; i < El::kVec; ++i) z[g * El::kVec + i] = in ? El::to_f32(t[i]) : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
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

// z -> p in place; returns lse.  live: the row has a logit above -infinity (NaN included: then the
// row's results are NaN, as the formulas say).
template <int LPR> __device__ __forceinline__ float bal_softmax(float (&z)[8], bool &live)
{
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, z[i]);
    m = lanes_max<LPR>(m);
    const float m2 = m == -INFINITY ? 0.f : m * kLog2e;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = ex2(fmaf(z[i], kLog2e, -m2)), sum += z[i];
    sum = lanes_sum<LPR>(sum);
    live = sum != 0.f;   // 0 where all logits are -infinity (a NaN is not 0)
    const float inv = 1.f / sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] *= inv;
    return (m2 + log2f(sum)) * kLn2;
}

template <int DT, int LPR> __global__ void __launch_bounds__(kBalThreads) router_balance_kernel(const BalanceArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int RPW = kWarp / LPR, W = kBalThreads / kWarp;
    __shared__ int s_cnt[kBalMaxExperts];
    __shared__ float s_p[W][LPR * 8];
    __shared__ float s_z[W];
    __shared__ int s_n[W];
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    for (int e = tid; e < a.E; e += kBalThreads) s_cnt[e] = 0;
    __syncthreads();
    float p[8] = {}, zz = 0.f;
    int n = 0;
    // kBalRows rows of a lane in flight: one alone leaves the loads' latency bare
    const int stepr = gridDim.x * W * RPW * kBalRows;
    for (long long t0 = (long long)(blockIdx.x * W + warp) * RPW * kBalRows + sub; t0 - sub < a.T; t0 += stepr) {
        float z[kBalRows][8];
        bool on[kBalRows];
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            const long long t = t0 + r * RPW;
            on[r] = t < a.T && (!a.mask || a.mask[t]);
        }
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            if (on[r]) {
                bal_load<DT, LPR>(reinterpret_cast<const T *>(a.logits) + (t0 + r * RPW) * a.stride, a.E, l, a.vec, z[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[r][i] = -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            bool live;
            const float lse = bal_softmax<LPR>(z[r], live);
            if (on[r] && live) {
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] += z[r][i];
                if (l == 0) zz = fmaf(lse, lse, zz), ++n;
                for (int k = l; k < a.K; k += LPR) {
                    const int e = __ldg(a.ids + (t0 + r * RPW) * a.K + k);
                    if ((unsigned)e < (unsigned)a.E) atomicAdd(&s_cnt[e], 1);
                }
            }
        }
    }
    // the rows of a warp first (lanes with the same l), then the warps in order
#pragma unroll
    for (int o = LPR; o < kWarp; o <<= 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] += __shfl_xor_sync(kFull, p[i], o);
        zz += __shfl_xor_sync(kFull, zz, o);
        n += __shfl_xor_sync(kFull, n, o);
    }
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_p[warp][bal_index<DT, LPR>(l, i, a.vec)] = p[i];
        if (l == 0) s_z[warp] = zz, s_n[warp] = n;
    }
    __syncthreads();
    float *part = a.part + (size_t)blockIdx.x * bal_part_words(a.E);
    int *ipart = reinterpret_cast<int *>(part) + a.E + 1;
    for (int e = tid; e <= a.E; e += kBalThreads) {
        float v = 0.f;
        int c = 0;
        for (int w = 0; w < W; ++w) {
            v += e < a.E ? s_p[w][e] : s_z[w];
            if (e == a.E) c += s_n[w];
        }
        part[e] = v;
        ipart[e] = e < a.E ? s_cnt[e] : c;
    }
}

// One CTA: the partial sums of all CTAs, in order, and the losses.
__global__ void __launch_bounds__(1024) router_balance_finish_kernel(const BalanceArgs a)
{
    // a group of threads per column: thread g of G adds the CTAs g, g+G, ...; then the groups in order
    __shared__ double s_sum[1024];
    __shared__ int s_int[1024];
    __shared__ double s_bal[kWarp];
    const int tid = threadIdx.x, cols = a.E + 1, words = bal_part_words(a.E);
    int G = 1024 / cols;   // >= 3: E <= 256
    const int g = tid / cols, e = tid % cols;
    pdl_wait();
    double v = 0.;
    int c = 0;
    if (g < G)
        for (int b0 = g; b0 < a.ctas; b0 += 8 * G) {   // eight CTAs' words in flight
            float x[8];
            int y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float *part = a.part + (size_t)(b0 + j * G) * words;
                x[j] = 0.f, y[j] = 0;
                if (b0 + j * G < a.ctas)
                    x[j] = __ldcg(part + e), y[j] = __ldcg(reinterpret_cast<const int *>(part) + cols + e);
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
    __syncthreads();
    const int n = s_int[a.E];
    double b = 0.;
    for (int i = tid; i < a.E; i += 1024) {
        b += (double)s_int[i] * s_sum[i];
        a.counts[i] = s_int[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) b += __shfl_xor_sync(kFull, b, o);
    if (tid % kWarp == 0) s_bal[tid / kWarp] = b;
    __syncthreads();
    if (tid == 0) {
        b = 0.;
        for (int w = 0; w < kWarp; ++w) b += s_bal[w];
        const double rn = n > 0 ? 1. / n : 0.;
        a.loss[0] = (float)(a.E * b * rn * rn / a.K);
        a.loss[1] = (float)(s_sum[a.E] * rn);
        *a.rows = n;
    }
}

template <int DT, int LPR> __global__ void __launch_bounds__(kBalThreads) router_balance_backward_kernel(const BalanceArgs a)
{
    using El = Elem<DT>;
    using T = typename El::T;
    constexpr int RPW = kWarp / LPR, W = kBalThreads / kWarp;
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    const int n = *a.rows;
    const float rn = n > 0 ? 1.f / (float)n : 0.f;
    const float gb = a.grad[0] * (float)a.E * rn, gz = a.grad[1] * 2.f * rn;
    // logits and gradient may be laid out differently; a lane's experts follow the vector order only
    // where both do
    const bool vec = a.vec && a.dvec;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = bal_index<DT, LPR>(l, i, vec);
        f[i] = e < a.E ? (float)a.counts[e] * rn / (float)a.K : 0.f;
    }
    const int stepr = gridDim.x * W * RPW * kBalRows;
    for (long long t0 = (long long)(blockIdx.x * W + warp) * RPW * kBalRows + sub; t0 - sub < a.T; t0 += stepr) {
        float z[kBalRows][8];
        bool on[kBalRows];
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            const long long t = t0 + r * RPW;
            on[r] = t < a.T && (!a.mask || a.mask[t]);
        }
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            if (on[r]) {
                bal_load<DT, LPR>(reinterpret_cast<const T *>(a.logits) + (t0 + r * RPW) * a.stride, a.E, l, vec, z[r]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) z[r][i] = -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            bool live;
            const float lse = bal_softmax<LPR>(z[r], live);
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) dot = fmaf(f[i], z[r][i], dot);
            dot = lanes_sum<LPR>(dot);
            const float c = fmaf(gz, lse, -gb * dot);   // dz = p (gb f + gz lse - gb dot)
            const long long t = t0 + r * RPW;
            if (t >= a.T) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) z[r][i] = on[r] && live ? z[r][i] * fmaf(gb, f[i], c) : 0.f;
            T *out = reinterpret_cast<T *>(a.dlogits) + t * a.dstride;
            if (vec) {
#pragma unroll
                for (int g = 0; g < 8 / El::kVec; ++g) {
                    const int e = bal_index<DT, LPR>(l, g * El::kVec, true);
                    T o[El::kVec];
#pragma unroll
                    for (int i = 0; i < El::kVec; ++i) o[i] = El::from_f32(z[r][g * El::kVec + i]);
                    if (e < a.E) *reinterpret_cast<uint4 *>(out + e) = *reinterpret_cast<const uint4 *>(o);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i * LPR + l < a.E) out[i * LPR + l] = El::from_f32(z[r][i]);
            }
        }
    }
}

}  // namespace stmoe_dev
