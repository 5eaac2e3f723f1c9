// Microscaled 4-bit floating point (MX4): a row is cut into blocks of 32 elements; a block holds
// 32 e2m1 codes (two to a byte, the even element in the low half) under one e8m0 scale byte.
//
//   amax = max |x| over the block
//   byte = clamp(floor(log2 amax) - 2 + 127, 0, 254)   (6 = 1.5 * 2^2 is the largest e2m1 value)
//          255 where the block holds a NaN or an infinity: the whole block reads back as NaN
//   code = x / 2^(byte-127) rounded to the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} with its sign, ties
//          to the even code, values above 6 to 6
//
// A row's last block is filled up with zeros, so a row of codes is a multiple of 16 bytes.
//
// Both directions are bound by HBM: one pass, 16-byte loads of the wide side, 4-byte accesses of
// the codes.  A lane owns 8 consecutive elements of a block, so the block maximum is two shuffles;
// a warp takes 1024 elements of a row, or several short rows, at a time, four independent groups per lane.  Quantising, it asks
// for the next 1024 before it works on these (raw, half the registers of the widened values; without
// that the loads' latency showed: 43 us for 14336 x 4096 bf16).  The arithmetic is exact: the scale is a power of two, its exponent is
// read from the bits of amax, and the only rounding is the conversion to e2m1.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "device_utils.cuh"

namespace stmoe_dev {

constexpr int kMxBlock = 32;        // elements under one scale
constexpr int kMxSeg = 1024;        // elements of a row that a warp takes at a time
constexpr int kMxGroups = kMxSeg / (kWarp * 8);
constexpr int kMxThreads = 256;

// 8 fp32 -> 8 e2m1 codes, element i in bits 4i
__device__ __forceinline__ uint32_t e2m1_pack8(const float (&v)[8])
{
    uint32_t r;
    asm("{.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// 8 codes -> four f16 pairs (exact), element 2i in the low half of h[i]
__device__ __forceinline__ void e2m1_unpack8(uint32_t w, uint32_t (&h)[4])
{
    asm("{.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// 2^(byte-127) as fp32: the byte is the exponent field, except at its ends
__device__ __forceinline__ float e8m0_value(uint32_t byte)
{
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}

// element types of the wide side: 0 fp32, 1 bf16, 4 f16 (the codes of the C boundary)
template <int DT> struct Elem;
template <> struct Elem<0> {
    using T = float;
    static constexpr int kVec = 4;   // elements of a 16-byte access
    __device__ static __forceinline__ float to_f32(T v) { return v; }
    __device__ static __forceinline__ T from_f32(float v) { return v; }
};
template <> struct Elem<1> {
    using T = __nv_bfloat16;
    using T2 = __nv_bfloat162;
    static constexpr int kVec = 8;
    __device__ static __forceinline__ T2 from_bits(uint32_t w) { return *reinterpret_cast<const T2 *>(&w); }
    __device__ static __forceinline__ float2 widen(T2 v)
    {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(&v);
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    __device__ static __forceinline__ float to_f32(T v) { return __bfloat162float(v); }
    __device__ static __forceinline__ T from_f32(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<4> {
    using T = __half;
    using T2 = __half2;
    static constexpr int kVec = 8;
    __device__ static __forceinline__ T2 from_bits(uint32_t w) { return *reinterpret_cast<const T2 *>(&w); }
    __device__ static __forceinline__ float2 widen(T2 v) { return __half22float2(v); }
    __device__ static __forceinline__ float to_f32(T v) { return __half2float(v); }
    __device__ static __forceinline__ T from_f32(float v) { return __float2half_rn(v); }
};

// 8 elements as they lie in memory
template <int DT> struct Raw8 {
    static constexpr int kPieces = 8 / Elem<DT>::kVec;
    uint4 q[kPieces];
};
// from the 16-byte aligned p (valid: how many exist, the others read as 0)
template <int DT> __device__ __forceinline__ void load_raw8(const typename Elem<DT>::T *p, int valid, Raw8<DT> &r)
{
    using T = typename Elem<DT>::T;
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < Raw8<DT>::kPieces; ++i) r.q[i] = ld_stream16(p + i * Elem<DT>::kVec);
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < valid ? p[i] : Elem<DT>::from_f32(0.f);
#pragma unroll
        for (int i = 0; i < Raw8<DT>::kPieces; ++i) r.q[i] = *reinterpret_cast<const uint4 *>(t + i * Elem<DT>::kVec);
    }
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// The 8 values, and the bits of the largest magnitude among the 32 of this lane and its three
// neighbours (infinity and NaN on top).
template <int DT> __device__ __forceinline__ uint32_t widen8(const Raw8<DT> &r, float (&v)[8])
{
    if constexpr (DT == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i] = __uint_as_float(r.q[i].x), v[4 * i + 1] = __uint_as_float(r.q[i].y);
            v[4 * i + 2] = __uint_as_float(r.q[i].z), v[4 * i + 3] = __uint_as_float(r.q[i].w);
        }
        float m = fabsf(v[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max_nan(m, fabsf(v[i]));
        m = max_nan(m, __shfl_xor_sync(kFull, m, 1));
        m = max_nan(m, __shfl_xor_sync(kFull, m, 2));
        return __float_as_uint(m) & 0x7fffffffu;
    } else {
        // two at a time in the 16-bit type, where a maximum is as exact
        using T2 = typename Elem<DT>::T2;
        const uint32_t w[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
        T2 m = Elem<DT>::from_bits(w[0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __hmax2_nan(m, Elem<DT>::from_bits(w[i] & 0x7fff7fffu));
        m = __hmax2_nan(m, __shfl_xor_sync(kFull, m, 1));
        m = __hmax2_nan(m, __shfl_xor_sync(kFull, m, 2));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Elem<DT>::widen(Elem<DT>::from_bits(w[i]));
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
        const float2 f = Elem<DT>::widen(m);
        return __float_as_uint(max_nan(f.x, f.y)) & 0x7fffffffu;
    }
}

template <int DT> __device__ __forceinline__ void store8(typename Elem<DT>::T *p, int valid, const float (&v)[8])
{
    using E = Elem<DT>;
    typename E::T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = E::from_f32(v[i]);
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / E::kVec; ++i)
            *reinterpret_cast<uint4 *>(p + i * E::kVec) = *reinterpret_cast<const uint4 *>(t + i * E::kVec);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = t[i];
    }
}

// From the largest |x| of a block as bits (they order like the values, infinity and NaN on top): the
// scale byte, and what the values are multiplied by.
__device__ __forceinline__ float mx4_inverse_scale(uint32_t m, uint32_t &byte)
{
    const int e = (int)(m >> 23);
    byte = e == 255 ? 255u : (uint32_t)max(e - 2, 0);
    return __uint_as_float((254u - min(byte, 253u)) << 23);  // 2^-(byte-127), always a normal number
}

struct Mx4Rows {
    void *x;                  // wide side [rows][cols]
    uint8_t *codes, *scales;  // [rows][ceil(cols/32)*16], [rows][ceil(cols/32)]
    long long rows, cols;
    long long x_stride;       // elements
    long long code_stride, scale_stride;  // bytes
    bool vec;                 // rows of x start on 16-byte boundaries
    int pack;                 // rows of a task: as many as 1024 elements hold, at least one
};

// A warp's tasks: `pack` short rows, or segments of 1024 elements of a long one, `step` tasks apart.  The
// divisions behind a task's place are done once; from then on it moves by (rows, segments).
struct Mx4Walk {
    long long row, seg, segs, d_row, d_seg;
    int pack;
    __device__ __forceinline__ Mx4Walk(const Mx4Rows &a) : pack(a.pack)
    {
        segs = (a.cols + kMxSeg - 1) / kMxSeg;   // 1 where pack > 1
        const long long task = (long long)blockIdx.x * (kMxThreads / kWarp) + threadIdx.x / kWarp;
        const long long step = (long long)gridDim.x * (kMxThreads / kWarp);
        row = task / segs, seg = task - row * segs, row *= pack;
        d_row = step / segs, d_seg = step - d_row * segs, d_row *= pack;
    }
    __device__ __forceinline__ void next()
    {
        row += d_row, seg += d_seg;
        if (seg >= segs) seg -= segs, row += pack;
    }
};

// A task as its warp sees it: pointers to its first row, elements of a row, rows, blocks of a row.
template <typename T> struct Mx4Piece {
    T *x;
    uint8_t *codes, *scales;
    int cols, rows, per_row;
    __device__ __forceinline__ Mx4Piece(const Mx4Rows &a, const Mx4Walk &w)
    {
        const long long c0 = w.seg * kMxSeg;
        x = reinterpret_cast<T *>(a.x) + w.row * a.x_stride + c0;
        codes = a.codes + w.row * a.code_stride + c0 / 2, scales = a.scales + w.row * a.scale_stride + c0 / kMxBlock;
        cols = (int)min((long long)kMxSeg, a.cols - c0);
        rows = (int)min((long long)w.pack, a.rows - w.row);
        per_row = (cols + kMxBlock - 1) / kMxBlock;
    }
};
// Row and first column of a lane's g-th group of 8 elements (kPack: of a task of several rows; the
// same for all tasks, as they differ in the number of rows alone).
template <bool kPack> struct Mx4Lane {
    int row[kMxGroups], col[kMxGroups];
    __device__ __forceinline__ Mx4Lane(const Mx4Rows &a, int lane)
    {
        const int per_row = kPack ? (int)((a.cols + kMxBlock - 1) / kMxBlock) * 4 : kMxSeg / 8;
#pragma unroll
        for (int g = 0; g < kMxGroups; ++g) {
            const int j = g * kWarp + lane;
            row[g] = kPack ? j / per_row : 0, col[g] = (j - row[g] * per_row) * 8;
        }
    }
};
// 8 x 8 nibbles among eight neighbouring lanes: nibble i of lane l <-> nibble l%8 of lane (l & ~7) + i
__device__ __forceinline__ uint32_t transpose_nibbles(uint32_t x, int lane)
{
    uint32_t r = __shfl_xor_sync(kFull, x, 4);
    x = lane & 4 ? (r >> 16) | (x & 0xffff0000u) : (x & 0x0000ffffu) | (r << 16);
    r = __shfl_xor_sync(kFull, x, 2);
    x = lane & 2 ? ((r >> 8) & 0x00ff00ffu) | (x & 0xff00ff00u) : (x & 0x00ff00ffu) | ((r << 8) & 0xff00ff00u);
    r = __shfl_xor_sync(kFull, x, 1);
    x = lane & 1 ? ((r >> 4) & 0x0f0f0f0fu) | (x & 0xf0f0f0f0u) : (x & 0x0f0f0f0fu) | ((r << 4) & 0xf0f0f0f0u);
    return x;
}

// CTAs an SM is to hold: the two sets of raw values of a lane are 32 registers, or 64 for fp32
template <int DT, bool kVec> constexpr int mx4_quantize_ctas() { return !kVec ? 5 : DT == 0 ? 2 : 4; }

// kVec: rows of x on 16-byte boundaries, a lane owns 8 consecutive elements (four lanes a block).
// Otherwise element by element in lane order, 32 elements (one block) a warp-wide access: with a lane's
// 8 elements read or written one by one, every access of the warp would touch all sectors of 256
// elements.  Eight blocks go together there: a lane has its element of each of them, and one exchange of
// nibbles among eight lanes makes (or takes apart) the words of codes.
// kPack: several short rows a task.
template <int DT, bool kVec, bool kPack>
__global__ void __launch_bounds__(kMxThreads, mx4_quantize_ctas<DT, kVec>()) mx4_quantize_kernel(const Mx4Rows a)
{
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x % kWarp;
    pdl_wait();
    pdl_launch_dependents();
    Mx4Walk w(a);
    if constexpr (kVec) {
        const Mx4Lane<kPack> at(a, lane);
        Raw8<DT> raw[kMxGroups];
        auto fetch = [&]() {
            const Mx4Piece<const T> t(a, w);
#pragma unroll
            for (int g = 0; g < kMxGroups; ++g)
                load_raw8<DT>(t.x + (kPack ? at.row[g] * a.x_stride : 0) + at.col[g], at.row[g] < t.rows ? t.cols - at.col[g] : 0, raw[g]);
        };
        if (w.row < a.rows) fetch();
        while (w.row < a.rows) {
            const Mx4Piece<const T> t(a, w);
            w.next();
            Raw8<DT> now[kMxGroups];
#pragma unroll
            for (int g = 0; g < kMxGroups; ++g) now[g] = raw[g];
            if (w.row < a.rows) fetch();
#pragma unroll
            for (int g = 0; g < kMxGroups; ++g) {
                float v[8];
                uint32_t byte;
                const float inv = mx4_inverse_scale(widen8<DT>(now[g], v), byte);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= inv;
                if (at.col[g] < t.per_row * kMxBlock && at.row[g] < t.rows) {
                    *reinterpret_cast<uint32_t *>(t.codes + (kPack ? at.row[g] * a.code_stride : 0) + at.col[g] / 2) = e2m1_pack8(v);
                    if (lane % 4 == 0) t.scales[(kPack ? at.row[g] * a.scale_stride : 0) + at.col[g] / kMxBlock] = (uint8_t)byte;
                }
            }
        }
    } else {
        for (; w.row < a.rows; w.next()) {
            const Mx4Piece<const T> t(a, w);
            const int blocks = t.per_row * t.rows;
            // the next eight blocks are asked for before these are worked on
            T raw[8];
            int row = 0, blk = 0;   // of the next block to ask for
            auto fetch = [&](int b) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = blk * kMxBlock + lane;
                    raw[i] = b + i < blocks && c < t.cols ? t.x[(kPack ? row * a.x_stride : 0) + c] : Elem<DT>::from_f32(0.f);
                    if (++blk == t.per_row && kPack) blk = 0, ++row;
                }
            };
            fetch(0);
#pragma unroll 1
            for (int b = 0; b < blocks; b += 8) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = Elem<DT>::to_f32(raw[i]);
                fetch(b + 8);
                uint32_t word = 0, mine = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t byte, code;
                    const float inv = mx4_inverse_scale(__reduce_max_sync(kFull, __float_as_uint(v[i]) & 0x7fffffffu), byte);
                    asm("{.reg .b8 q;\n\t"
                        "cvt.rn.satfinite.e2m1x2.f32 q, %1, %1;\n\t"
                        "cvt.u32.u8 %0, q;}"
                        : "=r"(code)
                        : "f"(v[i] * inv));
                    word |= (code & 15u) << (4 * i);
                    mine = lane % 8 == i ? byte : mine;
                }
                word = transpose_nibbles(word, lane);   // elements 8 (lane/8) .. +7 of block b + lane%8
                const int q = b + lane % 8, r = kPack ? q / t.per_row : 0, c = q - r * t.per_row;
                if (q < blocks) {
                    *reinterpret_cast<uint32_t *>(t.codes + (kPack ? r * a.code_stride : 0) + c * 16 + 4 * (lane / 8)) = word;
                    if (lane < 8) t.scales[(kPack ? r * a.scale_stride : 0) + c] = (uint8_t)mine;
                }
            }
        }
    }
}

template <int DT, bool kVec, bool kPack> __global__ void __launch_bounds__(kMxThreads) mx4_dequantize_kernel(const Mx4Rows a)
{
    using T = typename Elem<DT>::T;
    const int lane = threadIdx.x % kWarp;
    pdl_wait();
    pdl_launch_dependents();
    Mx4Walk w(a);
    if constexpr (kVec) {
        const Mx4Lane<kPack> at(a, lane);
        for (; w.row < a.rows; w.next()) {
            const Mx4Piece<T> t(a, w);
            uint32_t word[kMxGroups], byte[kMxGroups];
#pragma unroll
            for (int g = 0; g < kMxGroups; ++g) {
                word[g] = byte[g] = 0;
                if (at.col[g] < t.cols && at.row[g] < t.rows) {
                    word[g] = (*reinterpret_cast<const uint32_t *>(t.codes + (kPack ? at.row[g] * a.code_stride : 0) + at.col[g] / 2));
                    byte[g] = t.scales[(kPack ? at.row[g] * a.scale_stride : 0) + at.col[g] / kMxBlock];
                }
            }
#pragma unroll
            for (int g = 0; g < kMxGroups; ++g) {
                uint32_t h[4];
                e2m1_unpack8(word[g], h);
                const float s = e8m0_value(byte[g]);
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
                    v[2 * i] = f.x * s, v[2 * i + 1] = f.y * s;
                }
                store8<DT>(t.x + (kPack ? at.row[g] * a.x_stride : 0) + at.col[g], at.row[g] < t.rows ? t.cols - at.col[g] : 0, v);
            }
        }
    } else {
        for (; w.row < a.rows; w.next()) {
            const Mx4Piece<T> t(a, w);
            const int blocks = t.per_row * t.rows;
            int row = 0, blk = 0;
#pragma unroll 1
            for (int b = 0; b < blocks; b += 8) {
                const int q = b + lane % 8, qr = kPack ? q / t.per_row : 0, qc = q - qr * t.per_row;
                uint32_t word = 0, byte = 0;
                if (q < blocks) {
                    word = (*reinterpret_cast<const uint32_t *>(t.codes + (kPack ? qr * a.code_stride : 0) + qc * 16 + 4 * (lane / 8)));
                    byte = t.scales[(kPack ? qr * a.scale_stride : 0) + qc];
                }
                const float scale = e8m0_value(byte);
                word = transpose_nibbles(word, lane);   // this lane's element of blocks b .. b+7
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t h;
                    asm("{.reg .b8 q;\n\t"
                        "cvt.u8.u32 q, %1;\n\t"
                        "cvt.rn.f16x2.e2m1x2 %0, q;}"
                        : "=r"(h)
                        : "r"(word >> (4 * i) & 15u));
                    const float v = __low2float(*reinterpret_cast<const __half2 *>(&h)) * __shfl_sync(kFull, scale, i);
                    const int c = blk * kMxBlock + lane;
                    if (b + i < blocks && c < t.cols) t.x[(kPack ? row * a.x_stride : 0) + c] = Elem<DT>::from_f32(v);
                    if (++blk == t.per_row && kPack) blk = 0, ++row;
                }
            }
        }
    }
}

}  // namespace stmoe_dev
