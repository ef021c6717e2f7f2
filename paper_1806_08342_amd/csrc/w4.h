// Products with 4-bit weights and a scale per group: what the kernels share.
#pragma once

#include "halves.h"

namespace qnn {

struct W4Args {
    const uint16_t *x;
    const uint8_t *codes;
    const uint16_t *scales;
    const int8_t *zeros;
    const uint16_t *bias;
    uint16_t *y;
    int64_t ldx, ldy;
    int32_t M, N, K, group, groups;
    uint32_t group_magic, group_shift; // of the division by 32-weight units of a group
};

__device__ __forceinline__ int group_of(const W4Args &a, int k)
{
    const uint32_t unit = (uint32_t)k >> 5;
    return (int)(a.group_magic ? __umulhi(unit, a.group_magic) >> a.group_shift : unit);
}

// Two nibbles of a dword, 16 bits apart, as 16-bit floats: with bit 3 flipped a nibble is u = c + 8 (one v_bitop3 where mask and
// bits are in registers, see kept()).
template <class T> struct Nibbles;
template <> struct Nibbles<Bf16> {
    static constexpr float kOffset = 128.0f + 8.0f;
    static constexpr uint32_t kBits = 0x43084308u, kOnes = 0x3f803f80u;
    static __device__ __forceinline__ uint32_t two(uint32_t w, uint32_t bits) { return (w & 0x000f000fu) ^ bits; }
    static __device__ __forceinline__ f32x4 mfma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
};
template <> struct Nibbles<F16> {
    static constexpr float kOffset = 8.0f;
    static constexpr uint32_t kBits = 0x64086408u, kOnes = 0x3c003c00u;
    static __device__ __forceinline__ uint32_t two(uint32_t w, uint32_t bits)
    {
        const h16x2 off = {(_Float16)1024.0f, (_Float16)1024.0f};
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, (w & 0x000f000fu) ^ bits) - off);
    }
    static __device__ __forceinline__ f32x4 mfma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
    }
};
// a constant that stays in a vector register: an instruction of three operands takes one other constant only
__device__ __forceinline__ uint32_t kept(uint32_t v)
{
    asm("" : "+v"(v));
    return v;
}
// eight nibbles of a dword in the order 0 4 1 5 2 6 3 7: pairs (i, i + 4)
template <class T> __device__ __forceinline__ w32x4 expand_nibbles(uint32_t w, uint32_t bits)
{
    return w32x4{Nibbles<T>::two(w, bits), Nibbles<T>::two(w >> 4, bits), Nibbles<T>::two(w >> 8, bits), Nibbles<T>::two(w >> 12, bits)};
}
// eight consecutive 16-bit elements in the same order
__device__ __forceinline__ w32x4 pair_order(w32x4 v)
{
    return w32x4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                 __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}

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

// the kernel for many rows (w4_tile.hip), and the scratch that it takes
size_t w4_tile_bytes(int64_t M, int64_t K);
void launch_w4_tile(const W4Args &a, int type, void *workspace, hipStream_t s);

} // namespace qnn
