// What kernels over rows of logits share: packed fp32 pairs, the hardware's exponential, 16 bytes of a row to and from
// fp32, reductions over the lanes of a row.
#pragma once
#include "mx4.cuh"

namespace stmoe_dev {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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

// Eight neighbouring elements of a row, C of them in all.
template <int DT> __device__ __forceinline__ void row_load8(const typename Elem<DT>::T *row, int c, int C, bool vec, float (&v)[8])
{
    constexpr int V = Elem<DT>::kVec;
    if (vec && c + 8 <= C) {
#pragma unroll
        for (int g = 0; g < 8 / V; ++g) bal_widen<DT>(*reinterpret_cast<const uint4 *>(row + c + g * V), reinterpret_cast<float2 *>(v) + g * V / 2);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < C ? Elem<DT>::to_f32(row[c + i]) : 0.f;
    }
}
template <int DT> __device__ __forceinline__ void row_store8(typename Elem<DT>::T *row, int c, int C, bool vec, const float (&v)[8])
{
    constexpr int V = Elem<DT>::kVec;
    if (vec && c + 8 <= C) {
#pragma unroll
        for (int g = 0; g < 8 / V; ++g) *reinterpret_cast<uint4 *>(row + c + g * V) = bal_narrow<DT>(reinterpret_cast<const float2 *>(v) + g * V / 2);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < C) row[c + i] = Elem<DT>::from_f32(v[i]);
    }
}

}  // namespace stmoe_dev
