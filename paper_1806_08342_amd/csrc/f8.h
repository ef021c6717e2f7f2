// Operators of language models in 8-bit floating point: what the kernels share.
//
// Codes are e4m3 (four exponent bits, three of mantissa, largest value 448, no infinities, 0x7f and 0xff are NaN).  Activations have one
// binary32 scale per 128 consecutive elements of a row, weights one per block of 128 x 128; a value is code * scale.
#pragma once

#include "halves.h"

namespace qnn {

constexpr int kF8Block = 128;
constexpr float kF8Largest = 448.0f, kF8LeastScale = 0x1p-80f;

using i32x8 = int32_t __attribute__((ext_vector_type(8)));

inline int64_t f8_blocks(int64_t n) { return (n + kF8Block - 1) / kF8Block; }

struct F8Args {
    const uint8_t *x, *w;      // [M][ldx], [N][K]
    const float *xs, *ws;      // [K / 128][ldxs], [N / 128][K / 128]
    const void *bias;          // [N] of the output's type, or null
    void *y;                   // [M][ldy]
    int64_t ldx, ldxs, ldy;
    int32_t M, N, K, type;
};

// outputs of 16 or 32 bits; the type is the same in the whole launch
__device__ __forceinline__ void store_out(void *y, int64_t at, int type, float v)
{
    if (type == QNN_F32) static_cast<float *>(y)[at] = v;
    else static_cast<uint16_t *>(y)[at] = type == QNN_BF16 ? Bf16::narrow(v) : F16::narrow(v);
}
__device__ __forceinline__ float load_out(const void *p, int64_t at, int type)
{
    if (type == QNN_F32) return static_cast<const float *>(p)[at];
    const uint16_t v = static_cast<const uint16_t *>(p)[at];
    return type == QNN_BF16 ? Bf16::widen(v) : F16::widen(v);
}

// Of a row's block of 128 a lane has 16 bytes and those 64 behind them; 16 neighbouring lanes have 16 rows.  A lane loads that of the two first whose
// address has bit 6 as its row's number has bit 0: rows that lie whole blocks apart would keep each load to half of the cache's banks
// (32 x 12288 x 4096 17.9 us without, 12.3 so; 64 x 1000 x 2048 9.1 and 6.0).  in_order puts the two where they belong.
__device__ __forceinline__ uint32_t half_first(uint32_t row_address, int row) { return (row_address >> 6 ^ (uint32_t)row) & 1; }
__device__ __forceinline__ void in_order(const w32x4 (&loaded)[2], uint32_t first, w32x4 (&to)[2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) to[0][i] = first ? loaded[1][i] : loaded[0][i], to[1][i] = first ? loaded[0][i] : loaded[1][i];
}

// eight codes as bfloat16, exactly
__device__ __forceinline__ b16x8 widen_codes(uint32_t low, uint32_t high)
{
    return __builtin_bit_cast(b16x8, w32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.0f, false)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 1.0f, true)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.0f, false)),
                                           __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 1.0f, true))});
}

// Products of 16 x 16 outputs over 128 of K.  A lane has 32 bytes of row lane % 16 of either operand, in two pieces of 16; which 32 of the
// 128 they are does not matter as long as both operands take the same.  Result: column lane % 16 (second operand's row), rows 4 * (lane / 16) + e.
// NARROW: the matrix unit takes the codes; it aligns the products of 8 consecutive k to the largest and cuts them off 13 bits below it, so that sums of
// 128 normal products have a relative error of 1.4e-5, which results of 16 bits do not show.
// Else the codes enter as bfloat16, exactly, at half the rate, and sums are those of binary32 (1e-8).
template <bool NARROW> __device__ __forceinline__ f32x4 f8_products(const w32x4 (&a)[2], const w32x4 (&b)[2])
{
    f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (NARROW) {
        const i32x8 u = __builtin_bit_cast(i32x8, a), v = __builtin_bit_cast(i32x8, b);
        p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, p, 0, 0, 0, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen_codes(a[i >> 1][2 * (i & 1)], a[i >> 1][2 * (i & 1) + 1]),
                                                        widen_codes(b[i >> 1][2 * (i & 1)], b[i >> 1][2 * (i & 1) + 1]), p, 0, 0, 0);
    }
    return p;
}

__device__ __forceinline__ void fma4(f32x4 &acc, const f32x4 p, float s)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = fmaf(p[e], s, acc[e]);
}

} // namespace qnn
