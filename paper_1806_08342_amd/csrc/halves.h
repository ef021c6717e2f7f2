// 16-bit floating types of the kernels for quantized language models, unaligned accesses and lane exchanges.
#pragma once

#include "qnn_device.h"

#include <math.h>

namespace qnn {

using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
using h16x2 = _Float16 __attribute__((ext_vector_type(2)));
using h16x8 = _Float16 __attribute__((ext_vector_type(8)));
using b16x2 = __bf16 __attribute__((ext_vector_type(2)));
using b16x8 = __bf16 __attribute__((ext_vector_type(8)));
using u16x4 = uint16_t __attribute__((ext_vector_type(4)));
using w32x2 = uint32_t __attribute__((ext_vector_type(2)));
using w32x4 = uint32_t __attribute__((ext_vector_type(4)));
using w32x4_at4 = w32x4 __attribute__((aligned(4)));

// the element types of activations: QNN_BF16 and QNN_F16 of the C interface
struct Bf16 {
    using pair = b16x2;
    using eight = b16x8;
    static __device__ __forceinline__ float widen(uint16_t v) { return __builtin_bit_cast(float, (uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); } // to nearest even
};
struct F16 {
    using pair = h16x2;
    using eight = h16x8;
    static __device__ __forceinline__ float widen(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t narrow(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

template <class T> __device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    return (uint32_t)T::narrow(a) | (uint32_t)T::narrow(b) << 16;
}

// loads and stores without an alignment: gfx950 does them in one access
template <class V> __device__ __forceinline__ V load_any(const void *p)
{
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V> __device__ __forceinline__ void store_any(void *p, V v) { __builtin_memcpy(p, &v, sizeof(V)); }

// 16 bytes of a row from byte `at` on where the row ends within them: what lies beyond is zero.  The row's last 16 bytes are
// loaded and moved down (rows shorter than that go byte by byte).
__device__ __forceinline__ w32x4 load_end(const uint8_t *row, int bytes, int at)
{
    w32x4 v = {0u, 0u, 0u, 0u};
    const int have = bytes - at;
    if (have >= 16) return load_any<w32x4>(row + at);
    if (have <= 0) return v;
    if (bytes < 16) {
        for (int b = 0; b < have; ++b) v[b >> 2] |= (uint32_t)row[at + b] << (b & 3) * 8;
        return v;
    }
    const w32x4 last = load_any<w32x4>(row + bytes - 16);
    const int drop = 16 - have, words = drop >> 2, rest = (drop & 3) * 8;
    uint32_t u[5] = {last[0], last[1], last[2], last[3], 0u};
    if (words & 1) u[0] = u[1], u[1] = u[2], u[2] = u[3], u[3] = 0u;
    if (words & 2) u[0] = u[2], u[1] = u[3], u[2] = 0u, u[3] = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (uint32_t)(((uint64_t)u[i + 1] << 32 | u[i]) >> rest);
    return v;
}

// (lanes l, l ^ 16, l ^ 32, l ^ 48 hold the parts of one column)
__device__ __forceinline__ float max_over_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum_over_groups(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// e for the largest |v| of a row, so that v * 2^-e is in the last octave of binary16, from 2^15 on: it then holds what the row holds, but for
// bfloat16 elements below 2^-32 of the row's largest, which keep fewer bits: 256 times less than what a sum in binary32 loses beside the
// largest.  (2^e and 2^-e stay normal numbers.)
__device__ __forceinline__ int row_exponent(float peak)
{
    const int e = (int)(__builtin_bit_cast(uint32_t, peak) >> 23 & 255u) - 142;
    return peak > 0.0f ? max(e, -126) : 0;
}

inline bool bad_half_type(int type) { return type != QNN_BF16 && type != QNN_F16; }

} // namespace qnn
