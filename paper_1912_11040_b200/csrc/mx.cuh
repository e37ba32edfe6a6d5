// Microscaled numbers (the OCP microscaling formats MXFP8 with e4m3 elements and MXFP4): along a row, 32 values share
// a scale 2^(byte - 127); the elements have 8 bits (e4m3, largest 448 = 1.75 2^8) or 4 (e2m1, largest 6 = 1.5 2^2).
//
// Rows of codes are padded with zeros to whole groups of 128 values, one 32-bit word of scale bytes each: every
// row starts on a 64-byte boundary (4 bits) and a group's scales are read and written at once.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"

namespace mx {

constexpr int GROUP = 128;
constexpr int EMAX_E4M3 = 8, EMAX_E2M1 = 2;      // exponents of the formats' largest numbers

inline __host__ __device__ int groups(int D) { return (int)(((unsigned)D + GROUP - 1) / GROUP); }

#ifdef __CUDACC__
// The scale byte of a block with this largest magnitude: floor(log2) less the format's largest exponent,
// plus 127; 0 where that falls below it (and for a block of zeros), 255 = NaN where the block is not finite.  All of
// it is exact, so that every way of quantising the same values gives the same codes.
__device__ __forceinline__ unsigned scale_byte(float amax, int emax) {
    const int e = (int)(__float_as_uint(amax) >> 23 & 255u);
    return e == 255 ? 255u : (unsigned)max(e - emax, 0);
}
// 2^(127 - byte), by which the values are multiplied before they are rounded; 0 for a block that is not finite (its
// codes would not mean anything)
__device__ __forceinline__ float inverse_scale(unsigned byte) {
    return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float scale_value(unsigned byte) {
    return byte == 0 ? __uint_as_float(0x00400000u) : byte == 255u ? __uint_as_float(0x7fffffffu)
                                                                   : __uint_as_float(byte << 23);
}
// The larger magnitude; NaN where one is.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Rounding to nearest, ties to even; beyond the largest number that number.
__device__ __forceinline__ unsigned pack4_e4m3(float a, float b, float c, float d) {
    unsigned short lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (unsigned)lo | (unsigned)hi << 16;
}
__device__ __forceinline__ unsigned pack8_e2m1(const float *v) {
    unsigned r;
    asm("{\n"
        ".reg .b8 p, q, s, t;\n"
        "cvt.rn.satfinite.e2m1x2.f32 p, %2, %1;\n"
        "cvt.rn.satfinite.e2m1x2.f32 q, %4, %3;\n"
        "cvt.rn.satfinite.e2m1x2.f32 s, %6, %5;\n"
        "cvt.rn.satfinite.e2m1x2.f32 t, %8, %7;\n"
        "mov.b32 %0, {p, q, s, t};\n"
        "}" : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
__device__ __forceinline__ float2 halves(unsigned h) {       // two fp16 to fp32
    float2 f;
    asm("{\n.reg .f16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
__device__ __forceinline__ float2 unpack2_e4m3(unsigned short c) {
    unsigned h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
    return halves(h);
}
__device__ __forceinline__ void unpack4_e4m3(unsigned c, float *v) {
    const float2 a = unpack2_e4m3((unsigned short)(c & 0xffffu)), b = unpack2_e4m3((unsigned short)(c >> 16));
    v[0] = a.x;
    v[1] = a.y;
    v[2] = b.x;
    v[3] = b.y;
}
// the eight elements of a word
__device__ __forceinline__ void unpack8_e2m1(unsigned c, float *v) {
    unsigned h[4];
    asm("{\n"
        ".reg .b8 p, q, s, t;\n"
        "mov.b32 {p, q, s, t}, %4;\n"
        "cvt.rn.f16x2.e2m1x2 %0, p;\n"
        "cvt.rn.f16x2.e2m1x2 %1, q;\n"
        "cvt.rn.f16x2.e2m1x2 %2, s;\n"
        "cvt.rn.f16x2.e2m1x2 %3, t;\n"
        "}" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(c));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = halves(h[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// ------------------------------------------------------------------ rows in 32 and 16 bits
// Ordinary loads and stores, not through the non-coherent path: a caller may have an operator write over its input,
// row by row.
__device__ __forceinline__ void load8(const float *p, float *v) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    v[0] = a.x;
    v[1] = a.y;
    v[2] = a.z;
    v[3] = a.w;
    v[4] = b.x;
    v[5] = b.y;
    v[6] = b.z;
    v[7] = b.w;
}
__device__ __forceinline__ void unpack8_bf16(uint4 q, float *v) {
    const unsigned w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *v) {
    unpack8_bf16(*reinterpret_cast<const uint4 *>(p), v);
}
__device__ __forceinline__ void store8(float *p, const float *v) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ unsigned pack2_bf16(float a, float b) {
    unsigned r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *v) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]),
                                               pack2_bf16(v[6], v[7]));
}
__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ unsigned bits1(const float *p) { return *reinterpret_cast<const unsigned *>(p); }
__device__ __forceinline__ unsigned bits1(const __nv_bfloat16 *p) { return *reinterpret_cast<const unsigned short *>(p); }
template <typename T>
__device__ __forceinline__ float load1(const T *p) { return as_float(*p); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
#endif

}  // namespace mx

// The padded batch that the operators on rows share: row r is frame r % T_max of utterance r / T_max, and holds
// values where that is below the utterance's frame count (NULL: everywhere).  Row numbers are below 2^30; they are
// divided by T_max with one multiplication: floor(2^(31 + s) / T) + 1 with s the bits of T - 1, good below 2^31.
struct RowBatch {
    const int *counts;
    int T_max;
    int rows;              // B * T_max
    unsigned mul;
    int shift;
    RowBatch(const int *c, int T, int B) : counts(c), T_max(T), rows(B * T), shift(0) {
        while (shift < 31 && (1u << shift) < (unsigned)T) ++shift;
        mul = T == 1 ? 0 : (unsigned)((1ull << (31 + shift)) / (unsigned)T + 1);
        --shift;
    }
#ifdef __CUDACC__
    __device__ __forceinline__ int utterance(int row) const { return mul ? (int)(__umulhi((unsigned)row, mul) >> shift) : row; }
    __device__ __forceinline__ bool holds(int row) const {
        if (row >= rows) return false;
        if (!counts) return true;
        const int b = utterance(row);
        return row - b * T_max < counts[b];
    }
#endif
};

// Checks that all operators on rows share; AUG_OK with *none set where there is nothing to do.
inline int check_rows(const AugCtx *ctx, const int *counts, int B, int T_max, int D, bool *none) {
    *none = false;
    if (!ctx || B < 0 || (reinterpret_cast<uintptr_t>(counts) & 3)) return AUG_EINVAL;
    if (B > ctx->cfg.max_batch) return AUG_ECAP;
    if (T_max <= 0 || D < 1) return AUG_EINVAL;
    if ((int64_t)B * T_max > AUG_MAX_ROWS) return AUG_ECAP;
    *none = B == 0;
    return AUG_OK;
}
inline bool is_row_type(int t) { return t == AUG_ELEM_F32 || t == AUG_ELEM_BF16; }
inline bool is_mx_type(int t) { return t == AUG_ELEM_MX8 || t == AUG_ELEM_MX4; }
inline bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int elem_bytes(int t) { return t == AUG_ELEM_F32 ? 4 : 2; }
