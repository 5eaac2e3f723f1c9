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
// for 524288 rows that HBM delivers in 23.  The exponential is exp2 of one fused multiply-add per logit,
// z log2(e) - fl(m log2(e)) with m the row's maximum (relative error 2^-22 for the terms that matter; the
// row's sum is formed from the same exponents, so what the rounded product of m is off by, less than 0.1
// up to |m| = 2^20, cancels).  Beyond that it would become an exponent of its own and then overflow, so such
// rows, a mask's fill value as a rule, have m subtracted first.  Reciprocal and logarithm of the sum, which
// lies in [0.9, 280], are the hardware's (2^-23 relative, 2^-22 absolute).
// Sums over tokens: a lane adds the probabilities of its experts in fp32 over at most 256 rows (batches that
// would give it more have more CTAs), a CTA adds its lanes in a fixed order, and the CTAs' partial sums are
// added in fp64 in a fixed order by a second launch: no floating-point atomics, the same bits every time, and
// an error that does not grow with the tokens.  (Moving a lane's sums to fp64 inside the loop cost
// registers that the loads need: 92.3 -> 93.9 us for 524288 x 128, both directions.)  lse^2 is summed in fp64 throughout: a
// row at a fill value of 1e20 has one that fp32 does not hold, while the mean over the rows may.
#pragma once
#include "mx4.cuh"

namespace stmoe_dev {

constexpr int kBalThreads = 256;
constexpr int kBalMaxExperts = 256;
constexpr int kBalRows = 2;         // rows of a lane in flight
constexpr int kBalDepth = 3;        // steps of rows in shared memory: one in use, two under way
constexpr int kBalFinish = 8;       // CTAs of the cluster that adds the partial sums up
constexpr int kBalLaneSteps = 128; // steps of a CTA at most: so many times kBalRows rows a lane
constexpr float kBalPlainMax = 1048576.f;   // 2^20: largest |maximum| of a row without a subtraction of its own
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// a CTA's partial sums: [E] probabilities, the low word of lse^2 (fp64), then (int) [E] counts, rows, and
// the high word
__host__ __device__ inline int bal_part_words(int E) { return 2 * (E + 1) + 1; }

struct BalanceArgs {
    const void *logits;
    long long stride;       // elements
    const int *ids;         // [T][K]
    const uint8_t *mask;    // [T] or nullptr
    int T, E, K;
    bool vec;               // rows (of the gradient too) are 16-byte aligned, E a multiple of the vector width
    float *part;            // forward: [gridDim.x][bal_part_words(E)]
    int ctas;               // finish: rows of part
    float *loss;            // [2]
    int *counts;            // [E]
    int *rows;              // [1]
    const float *grad;      // backward: [2]
    void *dlogits;
    long long dstride;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 operations in one instruction (each rounded on its own, as the single ones are).
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*reinterpret_cast<const uint64_t *>(&a)), "l"(*reinterpret_cast<const uint64_t *>(&b)), "l"(*reinterpret_cast<const uint64_t *>(&c)));
    return *reinterpret_cast<const float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<const uint64_t *>(&a)), "l"(*reinterpret_cast<const uint64_t *>(&b)));
    return *reinterpret_cast<const float2 *>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<const uint64_t *>(&a)), "l"(*reinterpret_cast<const uint64_t *>(&b)));
    return *reinterpret_cast<const float2 *>(&r);
}

// Where lane l of a row's LPR lanes finds its N logits: in vector order (groups of 16 bytes, lane after
// lane) or one by one.
template <int DT, int LPR> __device__ __forceinline__ int bal_index(int l, int i, bool vec)
{
    constexpr int V = Elem<DT>::kVec;
    return vec ? (i / V) * (LPR * V) + l * V + i % V : i * LPR + l;
}

// A row read element by element (rows without 16-byte alignment), in lane order.
template <int DT, int LPR, int N> __device__ __forceinline__ void bal_load(const typename Elem<DT>::T *row, int E, int l, float2 (&z)[N / 2])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * LPR + l;
        (i & 1 ? z[i / 2].y : z[i / 2].x) = e < E ? Elem<DT>::to_f32(row[e]) : -INFINITY;
    }
}
// 16 bytes of a row, widened
template <int DT> __device__ __forceinline__ void bal_widen(const uint4 &q, float2 *z)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (DT == 0) {
        z[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
        z[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == 1) z[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
            else z[i] = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        }
    }
}
template <int DT> __device__ __forceinline__ uint4 bal_narrow(const float2 *z)
{
    uint32_t w[4];
    if constexpr (DT == 0) {
        w[0] = __float_as_uint(z[0].x), w[1] = __float_as_uint(z[0].y), w[2] = __float_as_uint(z[1].x), w[3] = __float_as_uint(z[1].y);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == 1) {
                const __nv_bfloat162 h = __float22bfloat162_rn(z[i]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __half2 h = __float22half2_rn(z[i]);
                w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
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
template <int LPR, int P> __device__ __forceinline__ float bal_softmax(float2 (&z)[P], float &inv, bool &live)
{
    float m = fmaxf(z[0].x, z[0].y);
#pragma unroll
    for (int i = 1; i < P; ++i) m = fmaxf(m, fmaxf(z[i].x, z[i].y));
    m = lanes_max<LPR>(m);
    if (m == -INFINITY) m = 0.f;
    float shift = 0.f;
    // a branch of the whole warp (one of the row's lanes cost 3 % of 524288 x 128, this one 0.8 %)
    if (__any_sync(kFull, fabsf(m) > kBalPlainMax)) {
        if (fabsf(m) > kBalPlainMax) shift = m, m = 0.f;
#pragma unroll
        for (int i = 0; i < P; ++i) z[i] = add2(z[i], make_float2(-shift, -shift));
    }
    const float m2 = m * kLog2e;
    const float2 k = make_float2(kLog2e, kLog2e), off = make_float2(-m2, -m2);
    float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        z[i] = fma2(z[i], k, off);
        z[i] = make_float2(ex2(z[i].x), ex2(z[i].y));
        s2 = add2(s2, z[i]);
    }
    const float sum = lanes_sum<LPR>(s2.x + s2.y);
    live = sum != 0.f;   // 0 where all logits are -infinity (a NaN is not 0)
    inv = __fdividef(1.f, sum);
    return fmaf(m2 + __log2f(sum), kLn2, shift);
}

// How rows are read: element by element; 16 bytes at a time; the same with no lane past the last expert
// (n_experts = LPR * N), which needs no checks.
constexpr int kBalScalar = 0, kBalVec = 1, kBalFull = 2;

// The rows of a lane, kBalRows a step.  Where rows are read 16 bytes at a time a lane's part of a row goes
// through shared memory: every lane copies what it will read itself (cp.async, nothing to synchronise),
// two steps ahead of the one it works on, so the loads' latency is hidden at no cost in registers.  Masks
// are asked for one step before the copies that depend on them.  kIds: the lane's first choice of a row
// travels with it.
template <int DT, int LPR, int N, int kRead, bool kIds> struct BalWalk {
    using T = typename Elem<DT>::T;
    static constexpr int RPW = kWarp / LPR, G = N * (int)sizeof(T) / 16;   // 16-byte pieces of a lane's part
    static constexpr bool kRing = kRead != kBalScalar;
    static constexpr uint32_t kBits = (1u << kBalRows) - 1;
    uint32_t t, step, t_ahead;       // row of the step in progress, rows between steps, row of the masks held (T < 2^31)
    const T *z;                      // kRing: of the next copy; else of the step in progress
    const int *ids;
    long long z_row, z_step, ids_step;
    uint32_t on_hist, next_on;       // kBalRows bits a step: the steps under way, newest lowest
    uint32_t ring, slot;             // shared-memory address of this thread's pieces, byte offset of the next stage

    __host__ __device__ static constexpr int stage_bytes() { return kBalRows * (G * 16 + (kIds ? 4 : 0)) * kBalThreads; }
    __device__ __forceinline__ uint32_t ask(const BalanceArgs &a, uint32_t at) const
    {
        uint32_t on = 0;
#pragma unroll
        for (int r = 0; r < kBalRows; ++r)
            if (at + r * RPW < (uint32_t)a.T && (!a.mask || a.mask[at + r * RPW])) on |= 1u << r;
        return on;
    }
    __device__ __forceinline__ uint32_t id_at(int r) const { return ring + kBalRows * G * 16 * kBalThreads - threadIdx.x * 12 + r * kBalThreads * 4; }
    __device__ __forceinline__ void copy(const BalanceArgs &a, int l, uint32_t on)
    {
#pragma unroll
        for (int r = 0; r < kBalRows; ++r)
            if (on >> r & 1) {
                const T *row = z + r * z_row;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const int e = bal_index<DT, LPR>(l, g * Elem<DT>::kVec, true);
                    if (kRead == kBalFull || e < a.E)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + slot + (r * G + g) * kBalThreads * 16), "l"(row + e) : "memory");
                }
                if (kIds && l < a.K) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(id_at(r) + slot), "l"(ids + r * RPW * a.K) : "memory");
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
        z += z_step;
        if (kIds) ids += ids_step;
        slot = slot == (kBalDepth - 1) * stage_bytes() ? 0 : slot + stage_bytes();
    }
    __device__ __forceinline__ BalWalk(const BalanceArgs &a, int warp, int sub, int l, uint8_t *smem)
    {
        constexpr int W = kBalThreads / kWarp;
        step = gridDim.x * W * RPW * kBalRows;
        t = (blockIdx.x * W + warp) * RPW * kBalRows + sub;
        z_row = RPW * a.stride, z_step = step * a.stride;
        z = reinterpret_cast<const T *>(a.logits) + t * a.stride;
        ids = kIds ? a.ids + (long long)t * a.K + l : nullptr, ids_step = (long long)step * a.K;
        ring = (uint32_t)__cvta_generic_to_shared(smem) + threadIdx.x * 16, slot = 0;
        on_hist = 0;
        if (kRing) {
            uint32_t on[kBalDepth];
#pragma unroll
            for (int i = 0; i < kBalDepth; ++i) on[i] = ask(a, t + i * step);
#pragma unroll
            for (int i = 0; i < kBalDepth - 1; ++i) copy(a, l, on[i]), on_hist = on_hist << kBalRows | on[i];
            on_hist = on_hist << kBalRows | on[kBalDepth - 1];   // its copy comes with the first step
            t_ahead = t + kBalDepth * step;
        } else {
            on_hist = ask(a, t);
            t_ahead = t + step;
        }
    }
    __device__ __forceinline__ bool more(const BalanceArgs &a, int sub) const { return t - sub < (uint32_t)a.T; }
    // Begins a step; bit r of the result: row r counts.
    __device__ __forceinline__ uint32_t begin(const BalanceArgs &a, int l)
    {
        const uint32_t newest = on_hist & kBits, now = kRing ? on_hist >> (kBalRows * (kBalDepth - 1)) & kBits : newest;
        if (kRing) copy(a, l, newest);
        next_on = ask(a, t_ahead);
        if (kRing) asm volatile("cp.async.wait_group %0;" ::"n"(kBalDepth - 1) : "memory");
        return now;
    }
    // Row r of the step, which counts, and the lane's first choice.
    __device__ __forceinline__ void row(const BalanceArgs &a, int r, int l, float2 (&v)[N / 2], int &id) const
    {
        if constexpr (kRing) {   // the oldest stage, which the next copy will overwrite
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (kRead == kBalFull || bal_index<DT, LPR>(l, g * Elem<DT>::kVec, true) < a.E) {
                    uint4 q;
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(ring + slot + (r * G + g) * kBalThreads * 16));
                    bal_widen<DT>(q, &v[g * N / 2 / G]);
                } else {
#pragma unroll
                    for (int i = 0; i < N / 2 / G; ++i) v[g * N / 2 / G + i] = make_float2(-INFINITY, -INFINITY);
                }
            }
            if (kIds && l < a.K) asm volatile("ld.shared.s32 %0, [%1];" : "=r"(id) : "r"(id_at(r) + slot));
        } else {
            bal_load<DT, LPR, N>(z + r * z_row, a.E, l, v);
            if (kIds && l < a.K) id = ids[r * RPW * a.K];
        }
    }
    __device__ __forceinline__ void end()
    {
        if (!kRing) {
            z += z_step;
            if (kIds) ids += ids_step;
        }
        on_hist = on_hist << kBalRows | next_on;
        t += step, t_ahead += step;
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
template <int DT, int LPR, int N, int kRead> __global__ void __launch_bounds__(kBalThreads, 3) router_balance_kernel(const BalanceArgs a)
{
    constexpr int W = kBalThreads / kWarp;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ int s_cnt[kBalMaxExperts];
    __shared__ float s_p[W][LPR * N];
    __shared__ double s_z[W];
    __shared__ int s_n[W];
    __shared__ double s_bal[W];
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    for (int e = tid; e < a.E; e += kBalThreads) s_cnt[e] = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    float2 p[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) p[i] = make_float2(0.f, 0.f);
    double zz = 0.;
    int n = 0;
    BalWalk<DT, LPR, N, kRead, true> w(a, warp, sub, l, ring);
    while (w.more(a, sub)) {
        const uint32_t on = w.begin(a, l);
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            float2 z[N / 2];
            int id = -1;
            if (on >> r & 1) {
                w.row(a, r, l, z, id);
            } else {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) z[i] = make_float2(-INFINITY, -INFINITY);
            }
            bool live;
            float inv;
            const float lse = bal_softmax<LPR>(z, inv, live);
            if ((on >> r & 1) && live) {
                const float2 inv2 = make_float2(inv, inv);
#pragma unroll
                for (int i = 0; i < N / 2; ++i) p[i] = fma2(z[i], inv2, p[i]);
                if (l == 0) zz = fma((double)lse, (double)lse, zz), ++n;
                if ((unsigned)id < (unsigned)a.E) atomicAdd(&s_cnt[id], 1);
                for (int k = l + LPR; k < a.K; k += LPR) {
                    const int e = a.ids[(long long)(w.t + r * (kWarp / LPR)) * a.K + k];
                    if ((unsigned)e < (unsigned)a.E) atomicAdd(&s_cnt[e], 1);
                }
            }
        }
        w.end();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // the rows of a warp first (lanes with the same l), then the warps in order
#pragma unroll
    for (int o = LPR; o < kWarp; o <<= 1) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) p[i].x += __shfl_xor_sync(kFull, p[i].x, o), p[i].y += __shfl_xor_sync(kFull, p[i].y, o);
        zz += __shfl_xor_sync(kFull, zz, o);
        n += __shfl_xor_sync(kFull, n, o);
    }
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s_p[warp][bal_index<DT, LPR>(l, i, kRead != kBalScalar)] = i & 1 ? p[i / 2].y : p[i / 2].x;
        if (l == 0) s_z[warp] = zz, s_n[warp] = n;
    }
    __syncthreads();
    if (gridDim.x > 1) {
        float *part = a.part + (size_t)blockIdx.x * bal_part_words(a.E);
        int *ipart = reinterpret_cast<int *>(part) + a.E + 1;
        for (int e = tid; e < a.E; e += kBalThreads) {
            float v = 0.f;
            for (int q = 0; q < W; ++q) v += s_p[q][e];
            part[e] = v;
            ipart[e] = s_cnt[e];
        }
        if (tid == 0) {
            double v = 0.;
            int c = 0;
            for (int q = 0; q < W; ++q) v += s_z[q], c += s_n[q];
            part[a.E] = __int_as_float(__double2loint(v));
            ipart[a.E] = c, ipart[a.E + 1] = __double2hiint(v);
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
        for (int q = 0; q < W; ++q) sum += s_bal[q], sq += s_z[q], rows += s_n[q];
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
    pdl_launch_dependents();
    double v = 0.;
    int c = 0;
    if (g < G)
        for (int b0 = rank + kBalFinish * g; b0 < a.ctas; b0 += 8 * kBalFinish * G) {   // eight rows' words in flight
            float x[8];
            int y[8], hi[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int b = b0 + j * kBalFinish * G;
                const float *part = a.part + (size_t)b * words;
                x[j] = 0.f, y[j] = hi[j] = 0;
                if (b < a.ctas) x[j] = __ldcg(part + e), y[j] = __ldcg(reinterpret_cast<const int *>(part) + cols + e);
                if (b < a.ctas && e == a.E) hi[j] = __ldcg(reinterpret_cast<const int *>(part) + cols + e + 1);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v += e == a.E ? __hiloint2double(hi[j], __float_as_int(x[j])) : (double)x[j], c += y[j];
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

// kRead: how rows of the logits are read and rows of the gradient written
template <int DT, int LPR, int N, int kRead> __global__ void __launch_bounds__(kBalThreads, 3) router_balance_backward_kernel(const BalanceArgs a)
{
    using El = Elem<DT>;
    using T = typename El::T;
    constexpr int RPW = kWarp / LPR, V = El::kVec;
    constexpr bool kVec = kRead != kBalScalar;
    extern __shared__ __align__(16) uint8_t ring[];
    const int tid = threadIdx.x, warp = tid / kWarp, lane = tid % kWarp, l = lane % LPR, sub = lane / LPR;
    pdl_wait();
    pdl_launch_dependents();
    BalWalk<DT, LPR, N, kRead, false> w(a, warp, sub, l, ring);
    const int n = *a.rows;
    const float rn = n > 0 ? 1.f / (float)n : 0.f;
    const float gb = a.grad[0] * (float)a.E * rn, gz = a.grad[1] * 2.f * rn;
    float2 f[N / 2];   // g_balance E/n f_e
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = bal_index<DT, LPR>(l, i, kVec);
        (i & 1 ? f[i / 2].y : f[i / 2].x) = e < a.E ? gb * ((float)a.counts[e] * rn / (float)a.K) : 0.f;
    }
    T *out = reinterpret_cast<T *>(a.dlogits) + w.t * a.dstride;
    const long long d_row = RPW * a.dstride, d_step = w.step * a.dstride;
    while (w.more(a, sub)) {
        const uint32_t on = w.begin(a, l);
#pragma unroll
        for (int r = 0; r < kBalRows; ++r) {
            float2 z[N / 2];
            int id;
            if (on >> r & 1) {
                w.row(a, r, l, z, id);
            } else {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) z[i] = make_float2(-INFINITY, -INFINITY);
            }
            bool live;
            float inv;
            const float lse = bal_softmax<LPR>(z, inv, live);
            float2 d2 = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) d2 = fma2(f[i], z[i], d2);
            const float dot = lanes_sum<LPR>(d2.x + d2.y);
            // dz = p (gb f + c), c = gz lse - gb dot, p = z inv
            const float c = gz * lse - dot * inv;
            const float2 inv2 = make_float2(inv, inv), c2 = make_float2(c * inv, c * inv);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) z[i] = mul2(z[i], fma2(f[i], inv2, c2));
            if (w.t + r * RPW >= (uint32_t)a.T) continue;
            if (!(on >> r & 1) || !live) {   // 0 whatever the losses' gradient is: an infinite one times 0 is NaN
#pragma unroll
                for (int i = 0; i < N / 2; ++i) z[i] = make_float2(0.f, 0.f);
            }
            T *o = out + r * d_row;
            if constexpr (kVec) {
#pragma unroll
                for (int g = 0; g < N / V; ++g) {
                    const int e = bal_index<DT, LPR>(l, g * V, true);
                    if (kRead == kBalFull || e < a.E) *reinterpret_cast<uint4 *>(o + e) = bal_narrow<DT>(&z[g * V / 2]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i * LPR + l < a.E) o[i * LPR + l] = El::from_f32(i & 1 ? z[i / 2].y : z[i / 2].x);
            }
        }
        w.end();
        out += d_step;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace stmoe_dev
