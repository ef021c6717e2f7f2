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
    int32_t skewed;                    // rows of codes do not all begin at a multiple of 4 bytes
};

__device__ __forceinline__ int group_of(const W4Args &a, int k)
{
    const uint32_t unit = (uint32_t)k >> 5;
    return (int)(a.group_magic ? __umulhi(unit, a.group_magic) >> a.group_shift : unit);
}

// Two nibbles of a dword, 16 bits apart, as 16-bit floats: with bit 3 flipped a nibble is u = c + 8 (one v_bitop3 where mask and
// bits are in registers, see kept()).  bfloat16 reaches to the end of binary32's range: there all stands in units of 2^kUnit, so that
// 128 products with up to 2^8, and their offset, do not pass it where the result does not.
template <class T> struct Nibbles;
template <> struct Nibbles<Bf16> {
    static constexpr float kOffset = 128.0f + 8.0f;
    static constexpr int kUnit = 16;
    static constexpr uint32_t kBits = 0x3b083b08u, kOnes = 0x37803780u; // 2^-9 (with bit 3), 2^-16
    static __device__ __forceinline__ uint32_t two(uint32_t w, uint32_t bits) { return (w & 0x000f000fu) ^ bits; }
    static __device__ __forceinline__ f32x4 mfma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
};
template <> struct Nibbles<F16> {
    static constexpr float kOffset = 8.0f;
    static constexpr int kUnit = 0;
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

// Consecutive dwords of a row of codes.  Where the row does not begin at a multiple of 4 bytes, loads from there take about
// twice as long (1 x 4100 x 4096 8.3 us, 4104 6.1): the dwords that hold them are loaded instead, one more of them,
// and shifted into place when they are used.  Every dword that is read holds a byte of the row.
template <int DWORDS> struct Codes {
    uint32_t w[DWORDS + 1];
    // row: where the lane's part of its row begins
    __device__ __forceinline__ void load(const uint8_t *row, int skewed)
    {
        const uint32_t skew = (uint32_t)(uintptr_t)row & 3u;
        row -= skew;
#pragma unroll
        for (int i = 0; i < DWORDS; i += 4) {
            const w32x4 v = *reinterpret_cast<const w32x4_at4 *>(row + 4 * i);
            w[i] = v[0], w[i + 1] = v[1], w[i + 2] = v[2], w[i + 3] = v[3];
        }
        if (skewed) w[DWORDS] = *reinterpret_cast<const uint32_t *>(row + 4 * DWORDS - (skew == 0 ? 4 : 0));
    }
    // (row: any address with the same last two bits)
    __device__ __forceinline__ void place(const uint8_t *row, int skewed)
    {
        if (!skewed) return;
#pragma unroll
        for (int i = 0; i < DWORDS; ++i) w[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], (uint32_t)(uintptr_t)row);
    }
    // where the row ends within them; at: of the lane's part, from the row's beginning
    __device__ __forceinline__ void load_tail(const uint8_t *row, int bytes, int at, int skewed)
    {
#pragma unroll
        for (int i = 0; i < DWORDS; i += 4) {
            const w32x4 v = load_end(row, bytes, at + 4 * i);
            w[i] = v[0], w[i + 1] = v[1], w[i + 2] = v[2], w[i + 3] = v[3];
        }
        w[DWORDS] = 0;
        if (!skewed) return;
        // as `place` expects them
        const uint32_t skew = (uint32_t)(uintptr_t)(row + at) & 3u;
#pragma unroll
        for (int i = DWORDS; i >= 0; --i) w[i] = (uint32_t)(((uint64_t)w[i] << 32 | (i ? w[i - 1] : 0u)) << 8 * skew >> 32);
    }
};

// Where a lane (of the two of a row) has loaded 32 consecutive bytes, 64 weights, a product of 16 takes a dword of each.  For it to lie
// within a group of 64 or 32 the two lanes exchange dwords; piece_of: the 16-byte piece of x that goes with dword i then.
template <int GS> __device__ __forceinline__ void swap_halves(uint32_t (&w)[8])
{
    if constexpr (GS >= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto r = __builtin_amdgcn_permlane32_swap(w[i], w[i + 4], false, false);
            w[i] = r[0], w[i + 4] = r[1];
        }
    if constexpr (GS == 4)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & 2) == 0) {
                const auto r = __builtin_amdgcn_permlane32_swap(w[i], w[i + 2], false, false);
                w[i] = r[0], w[i + 2] = r[1];
            }
}
template <int GS> __device__ __forceinline__ int piece_of(int i, int hh)
{
    return GS == 1 ? 8 * hh + i : GS == 2 ? 8 * (i >> 2) + 4 * hh + (i & 3) : 4 * (i >> 1) + 2 * hh + (i & 1);
}

// x as the kernels for tens and for many rows take it: binary16, each row scaled by a power of two, which is exact but for bfloat16
// elements below 2^-32 of their row's largest (row_exponent), in the order of expand_nibbles, rows padded with zeros to
// whole 128s
struct W4Prepared {
    uint16_t *x;      // binary16 [M][pitch]
    int32_t *row_exp; // [M], with room for whole tiles
    int32_t pitch;
};

inline W4Prepared prepared(void *workspace, int64_t M, int64_t K)
{
    const int64_t pitch = (K + 127) / 128 * 128;
    W4Prepared p;
    p.x = static_cast<uint16_t *>(workspace);
    p.row_exp = reinterpret_cast<int32_t *>(p.x + M * pitch);
    p.pitch = (int32_t)pitch;
    return p;
}
// scratch of the kernels that take x this way
inline size_t w4_prepared_bytes(int64_t M, int64_t K) { return (size_t)M * ((K + 127) / 128 * 128) * 2 + 4 * (size_t)((M + 127) / 128 * 128); }

void prepare_x(const W4Args &a, int type, const W4Prepared &p, hipStream_t s);
// tens of rows (w4_parts.hip), many (w4_tile.hip)
float w4_parts_us(int64_t M, int64_t N, int64_t K); // estimated time
const char *w4_parts_name(int64_t M, int64_t N, int64_t K);
void launch_w4_parts(const W4Args &a, int type, const W4Prepared &p, hipStream_t s);
void launch_w4_tile(const W4Args &a, int type, const W4Prepared &p, hipStream_t s);

// The unit that accumulators stand in, the scale of the group that they are at, and the largest so far.
struct ScaleUnit {
    float at = 0.0f, most = 0.0f;
};
// The scale of the group that accumulators come to: `ratio` brings them into its unit.  A scale of 0, or less than 2^-80 of the largest before
// it (in whose unit accumulators could overflow, in however many steps they came there), leaves its weights out: all nibbles masked, and
// an offset that takes off what is left.
struct GroupUnit {
    float ratio;
    h16x2 off;
    uint32_t mask;
};
__device__ __forceinline__ GroupUnit enter_group(float s, int z, ScaleUnit &unit)
{
    const bool none = s == 0.0f || fabsf(s) * 0x1p80f < unit.most;
    GroupUnit g;
    g.ratio = none ? 1.0f : unit.at / s;
    unit.at = none ? unit.at : s;
    unit.most = fmaxf(unit.most, fabsf(s));
    const _Float16 o = (_Float16)(1032.0f + (none ? 0.0f : (float)z));
    g.off = h16x2{o, o}, g.mask = none ? 0u : 0x000f000fu;
    return g;
}
// What an accumulator stands for, in a row of x that was scaled by 2^-row_exp: the unit's octave goes with the row's, as either alone may
// lead out of binary32's range.
struct Result {
    float mantissa;
    int octave;
    __device__ __forceinline__ explicit Result(const ScaleUnit &unit) : mantissa(__builtin_amdgcn_frexp_mantf(unit.at)), octave(__builtin_amdgcn_frexp_expf(unit.at)) {}
    __device__ __forceinline__ float of(float acc, int row_exp) const { return ldexpf(acc * mantissa, octave + row_exp); }
};
// eight weights c - z of a dword, in binary16
__device__ __forceinline__ h16x8 whole_weights(uint32_t w, const GroupUnit &g, uint32_t bits)
{
    w32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, (w >> 4 * e & g.mask) ^ bits) - g.off);
    return __builtin_bit_cast(h16x8, v);
}

} // namespace qnn
