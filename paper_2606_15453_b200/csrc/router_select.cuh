// Choice of experts for many tokens from the router's logits, and the gradient of the chosen weights.
//
//   s = softmax(z) or sigmoid(z)            scores of a row of E logits
//   v = s + bias                            what the choice goes by
//   group score = sum of the best one or two v of a group of E/G neighbours; the best top_groups groups stay
//   ids = the K largest v of the groups that stay, ascending; equal ones: the lower index
//   w = c s[ids], or, renormalised, c s[ids] / sum s[ids]
//   dz: softmax, renormalised   w_k (g_k - sum_j w_j g_j / c) at the chosen, 0 elsewhere
//       sigmoid, renormalised   the same times 1 - s_k
//       softmax                 c s_e ([e chosen] g_e - sum_j s_j g_j) everywhere
//       sigmoid                 w_k (1 - s_k) g_k at the chosen
// Renormalised weights are formed as a softmax over the chosen of log s, which neither underflows nor
// divides zero by zero.
//
// The choice is an integer result, so it has to be that of the formula and not of its rounding.  Without bias and
// with groups ranked by their best member the order of v is that of z, which is compared as it is.  Else
// the kernel chooses by v in fp32 and looks at the border: where a value of the other side lies
// within the error of both (kSelectSlack, derived there), and the values at the border do not all come from the same logit
// and bias (then they are equal, and the index decides), the row is chosen again by v in fp64.
//
// 2^j lanes share a row, eight neighbouring logits each, so a row is read once, 16 bytes at a time, and a warp
// holds 1 to 32 rows.  Choosing takes K rounds of a maximum over the row; these, not the bytes, bound it.
#pragma once
#include <cstddef>

#include "row_utils.cuh"
#include "tcgen05_utils.cuh"

namespace stmoe_dev {

constexpr int kSelThreads = 256;
constexpr int kSelMaxExperts = 256;
constexpr int kSelMaxK = 32;
constexpr int kSelMaxGroups = 32;
constexpr int kSelN = 8;            // logits of a lane
// Two fp32 values of v are told apart when they differ by more than this plus 2^-21 of their magnitude.  A
// sigmoid is off by less than 2^-21: exp2 of a rounded product (|z| 2^-24 relative, which s(1-s) damps to 2^-26), the
// hardware's exp2 and reciprocal (2^-22 and 2^-23).  A softmax probability p is off by p (|z-m| 2^-23 + 2^-22) from
// its exponential, at most 0.37 * 2^-23 + 2^-22, and by 13 * 2^-24 from its sum: less than 2^-19.5.  The sum with the
// bias adds 2^-24 of itself.  So two values are off by 2^-18.5 and 2^-24 of each, and a group's sum of two, its own rounding
// included, by 2^-18.5 and 2^-23 of the magnitudes of its members, which may cancel in it: two groups are told apart by twice the first
// constant and the second of the magnitudes of both groups' members (the quick way: of the largest of any group's, where 2^-22 would do).
constexpr float kSelectSlack = 3.814697265625e-6f, kSelectPart = 4.76837158203125e-7f;   // 2^-18, 2^-21

struct SelectArgs {
    const void *logits;
    long long stride;       // elements
    const float *bias;      // [E] or nullptr
    const uint8_t *mask;    // [T] or nullptr
    int T, E, K, G, top_groups, best;
    bool vec;               // rows (of the gradient too) are 16-byte aligned
    bool sigmoid, renorm, exact;   // exact: the order of v is that of z
    float scale;
    int *ids;               // [T][K]
    float *w;               // [T][K]
    const float *grad;      // backward: [T][K]
    void *dlogits;
    long long dstride;
};

// A lane's logits e0 .. e0+7, -infinity behind the last expert.
template <int DT> __device__ __forceinline__ void sel_load(const typename Elem<DT>::T *row, int e0, int E, bool vec, float (&z)[kSelN])
{
    constexpr int V = Elem<DT>::kVec;
    if (vec && e0 + kSelN <= E) {
#pragma unroll
        for (int g = 0; g < kSelN / V; ++g) bal_widen<DT>(ld_stream16(row + e0 + g * V), reinterpret_cast<float2 *>(z) + g * V / 2);
    } else {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) z[i] = e0 + i < E ? Elem<DT>::to_f32(row[e0 + i]) : -INFINITY;
    }
}

__device__ __forceinline__ float exp_of(float x) { return ex2(x * kLog2e); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

// Order-preserving unsigned keys; 0 stands for "cannot be chosen" (-infinity, NaN).  -0 and +0 are equal.
__device__ __forceinline__ uint32_t sel_key(float v) { return v > -INFINITY ? float_key(v + 0.f) : 0u; }
__device__ __forceinline__ unsigned long long sel_key(double v)
{
    if (!(v > -INFINITY)) return 0;
    const unsigned long long u = __double_as_longlong(v + 0.);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

template <int LPR, typename T> __device__ __forceinline__ T row_max(T v)
{
    if constexpr (LPR == kWarp && sizeof(T) == 4) {
        return __reduce_max_sync(kFull, v);
    } else {
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) {
            const T t = __shfl_xor_sync(kFull, v, o);
            v = t > v ? t : v;
        }
        return v;
    }
}
template <int LPR, typename T> __device__ __forceinline__ T row_sum(T v)
{
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}

// v[i] = what the choice goes by; F: float or double.  m, inv: maximum and 1 / sum of exponentials of the row (softmax).
template <int LPR, typename F> __device__ __forceinline__ void sel_values(const SelectArgs &a, const float (&z)[kSelN], int e0, F (&v)[kSelN], float &m, F &inv)
{
    if (!a.sigmoid) {
        m = z[0];
#pragma unroll
        for (int i = 1; i < kSelN; ++i) m = fmaxf(m, z[i]);
        m = lanes_max<LPR>(m);
        if (m == -INFINITY) m = 0.f;
        F sum = 0;
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = exp_of((F)z[i] - (F)m), sum += v[i];
        inv = (F)1 / row_sum<LPR>(sum);
    }
    if (a.exact) {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = z[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < kSelN; ++i) {
        F s;
        if (!a.sigmoid) s = v[i] * inv;
        else if constexpr (sizeof(F) == 4) s = __fdividef(1.f, 1.f + exp_of(-z[i]));
        else s = 1. / (1. + exp(-(double)z[i]));
        // past 2^126 the hardware's quotient is 0, which is what s is within the slack
        v[i] = z[i] == -INFINITY ? (F)-INFINITY : z[i] != z[i] ? (F)NAN : a.bias && e0 + i < a.E ? s + (F)a.bias[e0 + i] : s;
    }
}

// Groups that stay; members of the others become -infinity.  near: a group of the other side of the border lies within the
// error.  keys, totals, errors: the row's room in shared memory.
template <int LPR, typename F>
__device__ __forceinline__ void sel_groups(const SelectArgs &a, int l, int sub, int e0, F (&v)[kSelN], F *keys, F *totals, float *errors, bool &near)
{
    const int gs = a.E / a.G, lg = gs / kSelN;
    const F lowest = -INFINITY;
    const bool by_order = a.exact || sizeof(F) == 8;      // of the sums as they are: no error to allow for
    auto merge = [&](F &b1, F &b2, F o1, F o2) {
        const F low = b1 < o1 ? b1 : o1;
        b1 = b1 < o1 ? o1 : b1;
        b2 = b2 < o2 ? o2 : b2;
        b2 = b2 < low ? low : b2;
    };
    auto total_of = [&](F b1, F b2) {
        const F t = a.best == 1 || gs == 1 ? b1 : b1 + b2;
        return t > lowest ? t : lowest;       // infinity - infinity: nothing
    };
    // error of a group's sum: its members' are of their own magnitude, also where they cancel
    auto error_of = [&](F total, F b1, F b2) {
        if (by_order || !(total > lowest)) return 0.f;
        return kSelectSlack + (fabsf((float)b1) + (a.best == 1 || gs == 1 ? 0.f : fabsf((float)b2))) * kSelectPart;
    };
    // sure, maybe: groups that are, or may be, ahead of this one
    auto rank_step = [&](F mine, float error, int g, F other, float other_error, int og, int &sure, int &maybe) {
        if (by_order || !(mine > lowest)) {
            const bool ahead = other > mine || (other == mine && og < g);
            sure += ahead, maybe += ahead;
            return;
        }
        const F room = (F)error + (F)other_error;
        sure += other > mine + room;
        maybe += og != g && !(other < mine - room) && other > lowest;
    };
    if (gs % kSelN == 0 && (lg & (lg - 1)) == 0) {   // a group is 2^j whole lanes
        F b1 = lowest, b2 = lowest;
#pragma unroll
        for (int i = 0; i < kSelN; ++i) merge(b1, b2, v[i] > lowest ? v[i] : lowest, lowest);
        for (int o = 1; o < lg; o <<= 1) merge(b1, b2, __shfl_xor_sync(kFull, b1, o), __shfl_xor_sync(kFull, b2, o));
        const F mine = total_of(b1, b2);
        const float error = error_of(mine, b1, b2);
        const int g = l / lg;
        int sure = 0, maybe = 0;
        for (int og = 0; og < a.G; ++og) {
            const int of = sub * LPR + og * lg;
            const F other = __shfl_sync(kFull, mine, of);
            rank_step(mine, error, g, other, by_order ? 0.f : __shfl_sync(kFull, error, of), og, sure, maybe);
        }
        near |= g < a.G && mine > lowest && sure < a.top_groups && maybe >= a.top_groups;
        if (sure >= a.top_groups) {
#pragma unroll
            for (int i = 0; i < kSelN; ++i) v[i] = lowest;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kSelN; ++i) keys[e0 + i] = v[i] > lowest ? v[i] : lowest;
    __syncwarp();
    for (int g = l; g < a.G; g += LPR) {
        F b1 = lowest, b2 = lowest;
        for (int i = 0; i < gs; ++i) merge(b1, b2, keys[g * gs + i], lowest);
        const F t = total_of(b1, b2);
        totals[g] = t;
        if (!by_order) errors[g] = error_of(t, b1, b2);
    }
    __syncwarp();
    uint32_t stay = 0;
    for (int g = l; g < a.G; g += LPR) {
        const F mine = totals[g];
        const float error = by_order ? 0.f : errors[g];
        int sure = 0, maybe = 0;
        for (int og = 0; og < a.G; ++og) rank_step(mine, error, g, totals[og], by_order ? 0.f : errors[og], og, sure, maybe);
        near |= mine > lowest && sure < a.top_groups && maybe >= a.top_groups;
        if (sure < a.top_groups) stay |= 1u << g;
    }
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) stay |= __shfl_xor_sync(kFull, stay, o);
    __syncwarp();   // the room is written again for the next choice
    int g = e0 / gs, left = gs - e0 % gs;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) {
        if (e0 + i < a.E && !(stay >> g & 1)) v[i] = lowest;
        if (--left == 0) ++g, left = gs;
    }
}

// K rounds of "largest, lowest index first": the lane's chosen as bits.  last, next: keys on either side of the border.
template <int LPR, typename U> __device__ __forceinline__ uint32_t sel_rounds(int K, int l, int sub, U (&k)[kSelN], U &last, U &next)
{
    constexpr uint32_t kRowBits = LPR == kWarp ? kFull : (1u << (LPR % kWarp)) - 1;
    uint32_t chosen = 0;
    U m = k[0];
#pragma unroll
    for (int i = 1; i < kSelN; ++i) m = k[i] > m ? k[i] : m;
    U top = row_max<LPR>(m);
    last = 0;
    for (int j = 0; j < K; ++j) {
        if (!__any_sync(kFull, top != 0)) break;
        const uint32_t with = __ballot_sync(kFull, m == top) >> (sub * LPR) & kRowBits;
        if (top != 0 && l == __ffs(with) - 1) {
            bool open = true;
            m = 0;
#pragma unroll
            for (int i = 0; i < kSelN; ++i) {
                const bool hit = open && k[i] == top;
                if (hit) k[i] = 0, chosen |= 1u << i, open = false;
                m = k[i] > m ? k[i] : m;
            }
        }
        last = top;
        top = row_max<LPR>(m);
    }
    next = top;
    return chosen;
}

// The row chosen by v in fp64.
template <int LPR> __device__ __noinline__ uint32_t sel_again(const SelectArgs &a, const float *zp, int l, int sub, double *keys, double *totals)
{
    float z[kSelN], m;
    double v[kSelN], inv;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) z[i] = zp[i];
    sel_values<LPR>(a, z, l * kSelN, v, m, inv);
    bool near = false;
    if (a.G > 1) sel_groups<LPR>(a, l, sub, l * kSelN, v, keys, totals, nullptr, near);
    unsigned long long k[kSelN], last, next;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) k[i] = sel_key(v[i]);
    return sel_rounds<LPR>(a.K, l, sub, k, last, next);
}

// Every value of v within the slack of the border comes from the same logit and the same bias.
template <int LPR> __device__ __forceinline__ bool sel_same(const SelectArgs &a, const float (&z)[kSelN], const float (&v)[kSelN], int e0, float border, float room)
{
    uint32_t zl = 0, zh = 0, bl = 0, bh = 0;     // largest of the complement and of the key: min and max
#pragma unroll
    for (int i = 0; i < kSelN; ++i)
        if (fabsf(v[i] - border) <= room) {
            const uint32_t kz = float_key(z[i] + 0.f), kb = a.bias && e0 + i < a.E ? float_key(a.bias[e0 + i] + 0.f) : 0x80000000u;
            zl = max(zl, ~kz), zh = max(zh, kz), bl = max(bl, ~kb), bh = max(bh, kb);
        }
    zl = row_max<LPR>(zl), zh = row_max<LPR>(zh), bl = row_max<LPR>(bl), bh = row_max<LPR>(bh);
    return ~zl == zh && ~bl == bh;
}

template <int LPR> struct SelShared {
    static constexpr int kRows = kWarp / LPR, kMax = LPR * kSelN < kSelMaxK ? LPR * kSelN : kSelMaxK;
    double keys[kRows * LPR * kSelN];
    union {
        double totals[kRows * kMax];
        struct {
            int id[kRows * kMax];
            float z[kRows * kMax];
        } chosen;
    };
};

// Everything about a row from its logits on (-infinity throughout where it does not count): choice, weights, outputs.
template <int LPR> __device__ __forceinline__ void sel_row(const SelectArgs &a, long long t, const float (&z)[kSelN], int l, int sub, SelShared<LPR> &s)
{
    constexpr uint32_t kRowBits = LPR == kWarp ? kFull : (1u << (LPR % kWarp)) - 1;
    const int e0 = l * kSelN;
    float v[kSelN], m = 0.f, inv = 0.f;
    sel_values<LPR>(a, z, e0, v, m, inv);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) bad |= z[i] != z[i];
    bool near = false, unsure = false;     // the choice's border, the groups'
    double *const keys = s.keys + sub * LPR * kSelN, *const totals = s.totals + sub * SelShared<LPR>::kMax;
    if (a.G > 1) {
        float *const room = reinterpret_cast<float *>(totals);      // as many errors behind the totals
        sel_groups<LPR>(a, l, sub, e0, v, reinterpret_cast<float *>(keys), room, room + SelShared<LPR>::kMax, unsure);
    }
    uint32_t k[kSelN], last, next;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) k[i] = sel_key(v[i]);
    uint32_t chosen = sel_rounds<LPR>(a.K, l, sub, k, last, next);
    if (!a.exact) {
        const float border = key_value(last), room = kSelectSlack + fabsf(border) * kSelectPart;
        near = last != 0 && next != 0 && border - key_value(next) <= room;
        if (__any_sync(kFull, near | unsure)) {
            // a border of equal values needs no second look
            const bool same = sel_same<LPR>(a, z, v, e0, near ? border : INFINITY, room);
            if (__any_sync(kFull, unsure | (near & !same))) {
                float copy[kSelN];
#pragma unroll
                for (int i = 0; i < kSelN; ++i) copy[i] = z[i];
                chosen = sel_again<LPR>(a, copy, l, sub, keys, totals);
            }
        }
    }
    // the chosen side by side, ascending
    const int mine = __popc(chosen);
    int upto = mine;
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) {
        const int t2 = __shfl_up_sync(kFull, upto, o, LPR);
        if (l >= o) upto += t2;
    }
    const int n = __shfl_sync(kFull, upto, LPR - 1, LPR);
    int *const id = s.chosen.id + sub * SelShared<LPR>::kMax;
    float *const zc = s.chosen.z + sub * SelShared<LPR>::kMax;
    __syncwarp();
    int at = upto - mine;
#pragma unroll
    for (int i = 0; i < kSelN; ++i)
        if (chosen >> i & 1) id[at] = e0 + i, zc[at] = z[i], ++at;
    __syncwarp();
    const uint32_t any_bad = __ballot_sync(kFull, bad) >> (sub * LPR) & kRowBits;
    const float poison = any_bad || (!a.sigmoid && inv != inv) ? NAN : 0.f;
    auto log_score = [&](float x) { return a.sigmoid ? fminf(x, 0.f) - log1pf(expf(-fabsf(x))) : x; };
    float top = -INFINITY, sum = 0.f;
    if (a.renorm) {
        for (int j = l; j < n; j += LPR) top = fmaxf(top, log_score(zc[j]));
        top = lanes_max<LPR>(top);
        for (int j = l; j < n; j += LPR) sum += expf(log_score(zc[j]) - top);
        sum = lanes_sum<LPR>(sum);
    }
    if (t < a.T)
        for (int j = l; j < a.K; j += LPR) {
            float w = 0.f;
            if (j < n) {
                if (a.renorm) w = expf(log_score(zc[j]) - top) / sum;
                else w = a.sigmoid ? 1.f / (1.f + expf(-zc[j])) : expf(zc[j] - m) * inv;
            }
            a.ids[t * a.K + j] = j < n ? id[j] : -1;
            a.w[t * a.K + j] = a.scale * w + poison;
        }
}

template <int DT, int LPR> __global__ void __launch_bounds__(kSelThreads, 4) router_select_kernel(const SelectArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int W = kSelThreads / kWarp, RPW = kWarp / LPR;
    __shared__ SelShared<LPR> s_warp[W];
    const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp, l = lane % LPR, sub = lane / LPR;
    pdl_wait();
    pdl_launch_dependents();
    const long long t = ((long long)blockIdx.x * W + warp) * RPW + sub;
    const bool counts = t < a.T && (!a.mask || a.mask[t]);
    float z[kSelN];
    if (counts) sel_load<DT>(reinterpret_cast<const T *>(a.logits) + t * a.stride, l * kSelN, a.E, a.vec, z);
    else {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) z[i] = -INFINITY;
    }
    sel_row<LPR>(a, t, z, l, sub, s_warp[warp]);
}

// ---- one row a warp (more than 128 experts) -----------------------------------------------------
//
// K rounds over eight values a lane are 1400 instructions a row.  Here the K rounds run over one value a lane, the largest of its
// eight: the K-th of these is a lower bound of the row's K-th value, and what reaches it, K values and a few, is brought
// together, a value a lane in ascending order of index, where the few too many are taken away from below (of equal ones the
// highest index first).  Rows that hold an infinity or a NaN, rows with more than 32 values at the bound and rows that have to
// look twice at their border go the general way (131072 x 256, 8 groups, K 8: 259 -> 132 us; what bounds it is issue slots, 630 a row, 70 % of them used).

// 1 / x for 1 <= x <= infinity, to 2^-23
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the same to the last place or two; 0 for infinity
__device__ __forceinline__ float rcp_near(float x)
{
    const float y = rcp(x);
    return x < INFINITY ? fmaf(y, fmaf(-x, y, 1.f), y) : 0.f;
}
__device__ __forceinline__ float redux_max(float v)
{
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float redux_min(float v)
{
    float r;
    asm("redux.sync.min.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

constexpr int kSelLater = INT32_MIN;    // in place of a row's first id

struct SelRoom {
    float z[kWarp * kSelN];     // the row
    float v[kWarp];             // the candidates
    int id[kWarp];
};

// Members of groups that do not stay become -infinity; false where a group's rank is within the error.  A group is lg (2^j) whole lanes.
__device__ __forceinline__ bool sel_groups_quick(const SelectArgs &a, int lane, float (&v)[kSelN])
{
    const int lg = a.E / a.G / kSelN;
    float hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[i] = fmaxf(v[2 * i], v[2 * i + 1]), lo[i] = fminf(v[2 * i], v[2 * i + 1]);
    auto merge = [](float &b1, float &b2, float o1, float o2) {
        b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
        b1 = fmaxf(b1, o1);
    };
    merge(hi[0], lo[0], hi[1], lo[1]), merge(hi[2], lo[2], hi[3], lo[3]), merge(hi[0], lo[0], hi[2], lo[2]);
    for (int o = 1; o < lg; o <<= 1) merge(hi[0], lo[0], __shfl_xor_sync(kFull, hi[0], o), __shfl_xor_sync(kFull, lo[0], o));
    float mine = a.best == 1 ? hi[0] : hi[0] + lo[0];
    // what a sum's error goes by: its members' sizes, which it may be far below
    const float size = lane < a.E / kSelN ? fabsf(hi[0]) + (a.best == 1 ? 0.f : fabsf(lo[0])) : 0.f;
    // the groups that stay, or those that go, whichever are fewer, one after the other; equal ones: the lower index stays
    const bool group = lane < a.E / kSelN, adding = 2 * a.top_groups <= a.G;
    bool stays = !adding;
    float last, next;           // on either side of the border
    if (adding) {
        if (!group) mine = -INFINITY;
        for (int j = 0; j < a.top_groups; ++j) {
            last = redux_max(mine);
            const int first = __ffs(__ballot_sync(kFull, mine == last)) - 1;
            if ((lane ^ first) < lg) stays = true, mine = -INFINITY;
        }
        next = redux_max(mine);
    } else {
        if (!group) mine = INFINITY;
        for (int j = a.top_groups; j < a.G; ++j) {
            next = redux_min(mine);
            const int first = 31 - __clz(__ballot_sync(kFull, mine == next));
            if ((lane ^ first) < lg) stays = false, mine = INFINITY;
        }
        last = redux_min(mine);
    }
    if (!a.exact && last - next <= 2 * kSelectSlack + redux_max(size) * kSelectPart) return false;
    if (!stays) {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = -INFINITY;
    }
    return true;
}

// false: the general way.  bias: -infinity behind the last expert, where z is the lowest finite number.
__device__ __forceinline__ bool sel_row_quick(const SelectArgs &a, long long t, const float (&z)[kSelN], const float (&bias)[kSelN], SelRoom &room)
{
    const int lane = threadIdx.x % kWarp;
    const float lowest = -INFINITY;
    float v[kSelN], m = 0.f, inv = 0.f, probe = 0.f;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) probe = fmaf(z[i], 0.f, probe);
    if (__any_sync(kFull, probe != 0.f)) return false;          // an infinity or a NaN
    if (!a.sigmoid) {
        m = z[0];
#pragma unroll
        for (int i = 1; i < kSelN; ++i) m = fmaxf(m, z[i]);
        m = redux_max(m);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = bias[i] > lowest ? exp_of(z[i] - m) : 0.f, sum += v[i];   // a row may be at the lowest number throughout
        inv = __fdividef(1.f, row_sum<kWarp>(sum));
    }
    if (a.exact) {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = z[i] + bias[i];
    } else if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = rcp(1.f + ex2(z[i] * -kLog2e)) + bias[i];
    } else {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) v[i] = fmaf(v[i], inv, bias[i]);
    }
    if (a.G > 1 && !sel_groups_quick(a, lane, v)) return false;
    float top = v[0];
#pragma unroll
    for (int i = 1; i < kSelN; ++i) top = fmaxf(top, v[i]);
    float bound = lowest;
    for (int j = 0; j < a.K; ++j) {
        bound = redux_max(top);
        const uint32_t with = __ballot_sync(kFull, top == bound);
        if (lane == __ffs(with) - 1) top = lowest;
    }
    bound = fmaxf(bound, -3.402823466e38f);                     // fewer lanes than K with a value: all values
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) mine += v[i] >= bound;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
        const int u = __shfl_up_sync(kFull, upto, o);
        if (lane >= o) upto += u;
    }
    int n = __shfl_sync(kFull, upto, kWarp - 1);
    if (n > kWarp) return false;
    uint32_t at = dsmem_u32(room.v + upto - mine);
#pragma unroll
    for (int i = 0; i < kSelN; ++i)
        asm volatile(
            "{.reg .pred p;\n\t"
            "setp.ge.f32 p, %1, %3;\n\t"
            "@p st.shared.f32 [%0], %1;\n\t"
            "@p st.shared.b32 [%0+%4], %2;\n\t"
            "@p add.u32 %0, %0, 4;}"
            : "+r"(at) : "f"(v[i]), "r"(lane * kSelN + i), "f"(bound), "n"(offsetof(SelRoom, id) - offsetof(SelRoom, v)) : "memory");
    *reinterpret_cast<float4 *>(room.z + lane * kSelN) = make_float4(z[0], z[1], z[2], z[3]);
    *reinterpret_cast<float4 *>(room.z + lane * kSelN + 4) = make_float4(z[4], z[5], z[6], z[7]);
    __syncwarp();
    const float cv = room.v[lane];
    const int id = room.id[lane] & (kWarp * kSelN - 1);          // behind the n-th: what an earlier row left
    const float cz = room.z[id];
    bool there = lane < n;
    float border = lowest;                                      // the largest value on the other side
    if (n > a.K) {
        for (int left = n; left > a.K; --left) {
            border = redux_min(there ? cv : INFINITY);
            const uint32_t with = __ballot_sync(kFull, there && cv == border);
            if (lane == 31 - __clz(with)) there = false;
        }
        n = a.K;
    } else if (!a.exact) {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) border = fmaxf(border, v[i] < bound ? v[i] : lowest);
        border = redux_max(border);
    }
    if (!a.exact && border > lowest) {
        const float last = redux_min(there ? cv : INFINITY);
        if (last - border <= kSelectSlack + fabsf(last) * kSelectPart) return false;
    }
    const uint32_t chosen = __ballot_sync(kFull, there);
    float w = 0.f;
    if (a.renorm) {
        const float far = redux_max(there ? cz : lowest);
        float x;
        if (!a.sigmoid) x = expf(cz - far);
        else if (far > -40.f && !__any_sync(kFull, there && cz < -80.f)) x = rcp_near(1.f + expf(-cz));
        else x = expf(fminf(cz, 0.f) - log1pf(expf(-fabsf(cz))) - fminf(far, 0.f));     // scores so far below 1 that they or their sum underflow: by their logarithms
        x = there ? x : 0.f;
        w = x * rcp_near(row_sum<kWarp>(x));
    } else if (there)
        w = a.sigmoid ? rcp_near(1.f + expf(-cz)) : expf(cz - m) * inv;
    const long long to = t * a.K;
    if (there) {
        const int pos = __popc(chosen & ((1u << lane) - 1));
        a.ids[to + pos] = id;
        a.w[to + pos] = a.scale * w;
    }
    if (lane >= n && lane < a.K) a.ids[to + lane] = -1, a.w[to + lane] = 0.f;
    return true;
}

template <int DT> __global__ void __launch_bounds__(kSelThreads, 4) router_select_wide_kernel(const SelectArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int W = kSelThreads / kWarp, V = Elem<DT>::kVec;
    __shared__ SelShared<kWarp> s_warp[W];
    __shared__ __align__(16) SelRoom s_room[W];
    const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp, e0 = lane * kSelN, valid = a.E - e0;
    const bool whole = a.vec && valid >= kSelN;
    pdl_wait();
    pdl_launch_dependents();
    float bias[kSelN];
    bool odd = false;                       // a bias that is no number, or so large that sums overflow, takes every row the general way
#pragma unroll
    for (int i = 0; i < kSelN; ++i) {
        bias[i] = i >= valid ? -INFINITY : a.bias ? a.bias[e0 + i] : 0.f;
        odd |= i < valid && !(fabsf(bias[i]) < 1e30f);
    }
    odd = __any_sync(kFull, odd);
    const long long step = (long long)gridDim.x * W;
    const T *const logits = reinterpret_cast<const T *>(a.logits) + e0;
    auto counts = [&](long long t) { return t < a.T && (!a.mask || a.mask[t]); };
    // 16-byte pieces of the row after the one in work
    uint4 ahead[kSelN / V];
    auto ask = [&](long long t, bool on) {
#pragma unroll
        for (int g = 0; g < kSelN / V; ++g)
            if (on && whole) ahead[g] = ld_stream16(logits + t * a.stride + g * V);
    };
    long long t = (long long)blockIdx.x * W + warp;
    bool later = false;                     // rows that were marked for the general way, which would cost the loop its registers
    bool on = counts(t);
    ask(t, on);
    for (; t < a.T; t += step) {
        const bool row = on;
        float z[kSelN];
        if (row && whole) {
#pragma unroll
            for (int g = 0; g < kSelN / V; ++g) bal_widen<DT>(ahead[g], reinterpret_cast<float2 *>(z) + g * V / 2);
        } else if (row) {
#pragma unroll
            for (int i = 0; i < kSelN; ++i) z[i] = i < valid ? Elem<DT>::to_f32(logits[t * a.stride + i]) : -3.402823466e38f;
        }
        on = counts(t + step);
        ask(t + step, on);
        if (!row) {
            if (lane < a.K) a.ids[t * a.K + lane] = -1, a.w[t * a.K + lane] = 0.f;
            continue;
        }
        if (odd || !sel_row_quick(a, t, z, bias, s_room[warp])) {
            if (lane == 0) a.ids[t * a.K] = kSelLater;
            later = true;
        }
        __syncwarp();
    }
    if (!later) return;
    for (t = (long long)blockIdx.x * W + warp; t < a.T; t += step) {
        if (*(volatile int *)&a.ids[t * a.K] != kSelLater) continue;
        float z[kSelN];
        sel_load<DT>(logits - e0 + t * a.stride, e0, a.E, a.vec, z);
        __syncwarp();                       // all have seen the mark
        sel_row<kWarp>(a, t, z, lane, 0, s_warp[warp]);
        __syncwarp();
    }
}

// 1 / scale, which turns weights into shares of a row; 0 below 2^-126, where it would overflow: the mean that is left away is below the
// smallest normal number once the scale is back
__device__ __forceinline__ float sel_inverse(float scale) { return fabsf(scale) >= 1.17549435e-38f ? 1.f / scale : 0.f; }

// Gradient of sum grad . w under a plain softmax, which every expert has a part in.
template <int DT, int LPR> __global__ void __launch_bounds__(kSelThreads) router_select_backward_kernel(const SelectArgs a)
{
    using T = typename Elem<DT>::T;
    constexpr int W = kSelThreads / kWarp, RPW = kWarp / LPR, V = Elem<DT>::kVec;
    __shared__ __align__(16) float s_row[W][RPW * LPR * kSelN];
    const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp, l = lane % LPR, sub = lane / LPR, e0 = l * kSelN;
    float *const row = s_row[warp] + sub * LPR * kSelN;
    pdl_wait();
    pdl_launch_dependents();
    const long long t = ((long long)blockIdx.x * W + warp) * RPW + sub;
    const bool there = t < a.T;
    const T *const logits = reinterpret_cast<const T *>(a.logits) + (there ? t : 0) * a.stride;
    *reinterpret_cast<float4 *>(row + e0) = make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4 *>(row + e0 + 4) = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncwarp();
    const float inv_c = sel_inverse(a.scale);
    float mean = 0.f, poison = 0.f;
    bool some = false;
    if (there)
        for (int j = l; j < a.K; j += LPR) {
            const int e = a.ids[t * a.K + j];
            const float w = a.w[t * a.K + j];
            if (w != w) poison = NAN;
            if ((unsigned)e < (unsigned)a.E) mean = fmaf(w * inv_c, a.grad[t * a.K + j], mean), some = true;
        }
    mean = lanes_sum<LPR>(mean), poison = lanes_sum<LPR>(poison);
    some = __ballot_sync(kFull, some) >> (sub * LPR) & (LPR == kWarp ? kFull : (1u << (LPR % kWarp)) - 1);
    if (there)
        for (int j = l; j < a.K; j += LPR) {
            const int e = a.ids[t * a.K + j];
            if ((unsigned)e >= (unsigned)a.E) continue;
            row[e] = a.grad[t * a.K + j];
        }
    __syncwarp();
    float d[kSelN];
    *reinterpret_cast<float4 *>(d) = *reinterpret_cast<const float4 *>(row + e0);
    *reinterpret_cast<float4 *>(d + 4) = *reinterpret_cast<const float4 *>(row + e0 + 4);
    float z[kSelN], v[kSelN], m, inv;
    if (some) sel_load<DT>(logits, e0, a.E, a.vec, z);
    else {
#pragma unroll
        for (int i = 0; i < kSelN; ++i) z[i] = -INFINITY;
    }
    m = z[0];
#pragma unroll
    for (int i = 1; i < kSelN; ++i) m = fmaxf(m, z[i]);
    m = lanes_max<LPR>(m);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) v[i] = z[i] == -INFINITY ? 0.f : exp_of(z[i] - m), sum += v[i];
    inv = a.scale / lanes_sum<LPR>(sum);
#pragma unroll
    for (int i = 0; i < kSelN; ++i) d[i] = z[i] == -INFINITY ? 0.f : v[i] * inv * (d[i] - mean);
    if (!there) return;
#pragma unroll
    for (int i = 0; i < kSelN; ++i) d[i] += poison;
    T *const out = reinterpret_cast<T *>(a.dlogits) + t * a.dstride;
    if (a.vec && e0 + kSelN <= a.E) {
#pragma unroll
        for (int g = 0; g < kSelN / V; ++g) *reinterpret_cast<uint4 *>(out + e0 + g * V) = bal_narrow<DT>(reinterpret_cast<const float2 *>(d) + g * V / 2);
    } else {
#pragma unroll
        for (int i = 0; i < kSelN; ++i)
            if (e0 + i < a.E) out[e0 + i] = Elem<DT>::from_f32(d[i]);
    }
}

// The same where only the chosen have a gradient (all but the plain softmax): up to four rows a warp at a time, a lane a choice, kp (a
// power of two) lanes a row; rows are made in shared memory, which is zero but for the chosen, and go out 16 bytes at a time.  One
// row a warp left each of its four dependent reads to wait alone (131072 x 256, K 8: 67 -> 23 us, where the bytes take 17).
template <int DT> __global__ void __launch_bounds__(kSelThreads) router_select_sparse_backward_kernel(const SelectArgs a, int kp, int rows)
{
    using T = typename Elem<DT>::T;
    constexpr int W = kSelThreads / kWarp, V = Elem<DT>::kVec, kMost = 4;
    __shared__ __align__(16) float s_row[W][kMost][kSelMaxExperts];
    const int warp = threadIdx.x / kWarp, lane = threadIdx.x % kWarp, r = lane / kp, j = lane % kp;
    float(*const row)[kSelMaxExperts] = s_row[warp];
    for (int i = lane; i < kMost * kSelMaxExperts; i += kWarp) row[0][i] = 0.f;
    __syncwarp();
    pdl_wait();
    pdl_launch_dependents();
    const int chunks = (a.E + kSelN - 1) / kSelN;
    const float inv_c = sel_inverse(a.scale);
    const long long step = (long long)gridDim.x * W * rows;
    for (long long t0 = ((long long)blockIdx.x * W + warp) * rows; t0 < a.T; t0 += step) {
        const bool on = r < rows && j < a.K && t0 + r < a.T;
        const long long at = (t0 + r) * a.K + j;
        const int e = on ? a.ids[at] : -1;
        const float w = on ? a.w[at] : 0.f;
        const bool chosen = (unsigned)e < (unsigned)a.E;
        const float g = chosen ? a.grad[at] : 0.f;
        float slope = 1.f;
        if (a.sigmoid && chosen) slope = 1.f / (1.f + expf(Elem<DT>::to_f32(reinterpret_cast<const T *>(a.logits)[(t0 + r) * a.stride + e])));
        float mean = 0.f;
        if (a.renorm) {
            mean = chosen ? w * inv_c * g : 0.f;
            for (int o = kp / 2; o > 0; o >>= 1) mean += __shfl_xor_sync(kFull, mean, o);
        }
        if (chosen) row[r][e] = w * (g - mean) * slope;
        const uint32_t bad = __ballot_sync(kFull, w != w);
        __syncwarp();
        for (int c = lane; c < rows * chunks; c += kWarp) {
            const int rr = c / chunks, e0 = (c - rr * chunks) * kSelN;
            if (t0 + rr >= a.T) break;
            float d[kSelN];
            *reinterpret_cast<float4 *>(d) = *reinterpret_cast<const float4 *>(&row[rr][e0]);
            *reinterpret_cast<float4 *>(d + 4) = *reinterpret_cast<const float4 *>(&row[rr][e0 + 4]);
            if (bad >> (rr * kp) & (kp == kWarp ? kFull : (1u << kp) - 1)) {
#pragma unroll
                for (int i = 0; i < kSelN; ++i) d[i] = NAN;
            }
            T *const out = reinterpret_cast<T *>(a.dlogits) + (t0 + rr) * a.dstride + e0;
            if (a.vec && e0 + kSelN <= a.E) {
#pragma unroll
                for (int i = 0; i < kSelN / V; ++i) *reinterpret_cast<uint4 *>(out + i * V) = bal_narrow<DT>(reinterpret_cast<const float2 *>(d) + i * V / 2);
            } else {
#pragma unroll
                for (int i = 0; i < kSelN; ++i)
                    if (e0 + i < a.E) out[i] = Elem<DT>::from_f32(d[i]);
            }
        }
        __syncwarp();
        if (chosen) row[r][e] = 0.f;
        __syncwarp();
    }
}

}  // namespace stmoe_dev
