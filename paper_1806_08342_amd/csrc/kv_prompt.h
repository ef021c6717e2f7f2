// Attention over the cache for requests with many query rows: 32 rows per wave, keys and values of 64 tokens at a time in LDS, as
// binary16.
//
// 8-bit codes are converted once for all waves of the workgroup, on the way from memory to LDS (two buffers: the codes of the next
// 64 tokens are in flight while these are worked on).  S^T = K q^T and O^T = V^T p^T on 32x32x16 tiles; as in the kernel for few
// rows the tokens' order in a tile is chosen so that the probabilities are the second product's operand in the lane that
// computed them: rows of K in LDS have bits 2 and 3 of the token's number exchanged.
//
// The running maximum and the unit that the accumulators stand in, a value scale, follow lazily: they are kept while a row's scores stay
// below 2^kRoom times the reference and pages' value scales within 2^(kRoom - 1) of the unit at least, so that most units of tokens rescale nothing.  A
// page's value scale is then part of the exponent (p * vs / unit), and the sum of p is corrected once per tile.  Where the scales of
// the two tiles lie further apart, or further from any unit that the accumulators can stand in, probabilities go without them and each tile's
// product is added by itself, with its scale in binary32: a page says nothing about rows that see only others.
//
// Bound by the two things that a wave does in turn: products (4 D flops per row and token, at 38 % of the matrix units' cycles) and the
// softmax between them (an exponential, four more operations and half a conversion per score, 51 % of the vector unit's with the work on addresses); two waves on
// a SIMD seldom overlap them (half a unit apart, or with a higher priority for products, they did not either), and within each of them nearly every product
// waits for the fragment that is read from LDS right before it.  8192 tokens, 32 query
// heads of 128 over 8: 611-650 us, 850-900 TFLOP/s of the half that the mask leaves.  Forms that interleave a unit's products with the next
// one's softmax in a wave, or let the waves of a SIMD alternate, lost more to registers and scalar work than they gained.
#pragma once

#include "kv_attention.h"

namespace qnn {

constexpr float kPromptHead = 6.0f, kRoom = 4.0f; // p * vs / unit stays below 2^(6 + 4 + 4) of binary16's 2^16

// The unit of a wave's accumulators (the same in all lanes, from scales that are): the scale of a page where it can be, so that the probabilities of that
// page's tokens, 2^6 for a row's only one, are not rounded for their scale's sake.  A page's scale is near it from over 2^-4 to just under 2^4 of it.
struct ValueUnit {
    int pattern = 0x3f800000, peak = -127; // of the unit (scales are given as patterns, too); the largest scale's exponent so far
    static __device__ __forceinline__ int exponent(int scale) { return (scale >> 23 & 255) - 127; }
    __device__ __forceinline__ float value() const { return __builtin_bit_cast(float, pattern); }
    __device__ __forceinline__ float of(int scale) const { return __builtin_bit_cast(float, scale) * __builtin_amdgcn_rcpf(value()); } // a scale in units
    __device__ __forceinline__ bool is_near(int scale) const { return (unsigned)(exponent(scale) - exponent(pattern) + 3) <= 6u; }
    // To the scale, as far as accumulators can follow: they are below 2^(10 + 7 + 31) times what the unit lacks of the largest
    // scale, which is at most 2^79, and in units up to 2^20 rows that see only pages of the smallest scales keep them.  Returns what
    // accumulators are to be multiplied with.
    __device__ __forceinline__ float move_to(int scale)
    {
        const float from = value();
        const int e = exponent(scale);
        peak = max(peak, e);
        const int at = min(max(max(e, peak - 60), -60), max(20, peak - 79));
        pattern = at == e ? scale : (at + 127) << 23;
        return from * __builtin_amdgcn_rcpf(value());
    }
};

__device__ __forceinline__ float other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    // r[0]: the low half's value in all lanes, r[1]: the high half's
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

template <class T, int D, int WAVES> __global__ void __launch_bounds__(64 * WAVES, D <= 128 ? 2 : 1) attend_prompt_kernel(const AttendArgs a)
{
    constexpr int BR = 32 * WAVES, KS = D / 16, VT = D / 32;
    constexpr int PIECES = (4 * D + 64 * WAVES - 1) / (64 * WAVES); // 16-byte pieces of 64 tokens' keys (or values) per thread
    constexpr bool EVEN = 4 * D % (64 * WAVES) == 0;
    constexpr int KP = D + 8, VP = 64 + 8; // pitches in LDS: 16 bytes more than the row, so that rows start in different banks
    __shared__ __attribute__((aligned(16))) _Float16 s_k[2][64][KP];
    __shared__ __attribute__((aligned(16))) _Float16 s_v[2][D][VP];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hh = lane >> 5;
    const int heads = a.cache.heads, block = a.cache.block;
    // heads next to each other: workgroups are dealt to the XCDs in turn, so that one XCD's L2 holds few heads' keys and values
    const int h = blockIdx.x % heads, rest = blockIdx.x / heads;
    // the last rows of all requests, which see most tokens, go first
    const int chunk = rest % a.chunks, r = rest / a.chunks % a.requests, rb0 = rest / a.chunks / a.requests;
    const Request rq = request_of<64>(a, r);
    const int rows = rq.n * a.group;
    if (rows <= a.rows_over || rows > a.rows_upto) return;
    const int chunks = chunks_of(a, rq);
    if (chunk >= chunks) return;
    const int blocks = (rows + BR - 1) / BR;

    for (int rb = blocks - 1 - rb0; rb >= 0; rb -= a.row_blocks) {
        const int rt = rb * BR;
        const int64_t pos0 = rq.length - rq.n; // position of the first query
        const int last_row = min(rt + BR, rows) - 1;
        int64_t t0 = rq.low + (int64_t)chunk * a.chunk_tokens;
        const int64_t t1 = min(chunk + 1 < chunks ? min(rq.high, t0 + a.chunk_tokens) : rq.high, pos0 + last_row / a.group + 1);
        if (a.window > 0) t0 = max(t0, (pos0 + rt / a.group - a.window + 1) & ~(int64_t)63);
        const int units = t1 > t0 ? (int)((t1 - t0 + 63) / 64) : 0;

        // this wave's rows
        h16x8 qf[KS];
        float factor;
        int64_t pos, row_id;
        {
            const int row = rt + wave * 32 + c, qi = min(row, rows - 1) / a.group, e = min(row, rows - 1) % a.group;
            pos = row < rows ? pos0 + qi : -1;
            row_id = (rq.row0 + qi) * a.q_heads + h * a.group + e;
            const uint16_t *q = a.q + (rq.row0 + qi) * a.q_token_pitch + (int64_t)(h * a.group + e) * a.q_head_pitch + 8 * hh;
            w32x4 raw[KS];
            float peak = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) raw[k] = load_any<w32x4>(q + 16 * k);
            if constexpr (!std::is_same_v<T, F16>)
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) peak = fmaxf(peak, fabsf(T::widen((uint16_t)(raw[k][i >> 1] >> (i & 1) * 16))));
            const int ex = std::is_same_v<T, F16> ? 0 : row_exponent(fmaxf(peak, other_half(peak)));
            const float down = ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, -ex); // (scores grow with the products: the sign goes to q)
            factor = fabsf(a.scale) * ldexpf(1.0f, ex);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) qf[k][i] = (_Float16)(T::widen((uint16_t)(raw[k][i >> 1] >> (i & 1) * 16)) * down);
        }
        const int wave_row = rt + wave * 32;
        const int64_t wave_first = pos0 + wave_row / a.group, wave_last = pos0 + min(wave_row + 31, rows - 1) / a.group;
        const bool idle = wave_row >= rows;

        f32x16 o[VT];
        float m = kNothing, l = 0.0f;
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[v][i] = 0.0f;
        ValueUnit unit; // that o stands in
        bool far = false; // a row's scores are so large that their products have to be rounded before the maximum is taken off

        // lane i holds place and scales of the i-th of 64 halves (32 tokens)
        int32_t u_page = 0, u_at = 0;
        float u_ks = 0.0f, u_vs = 0.0f;
        int looked = 0;
        auto look_up = [&](int unit) {
            looked = unit;
            const int64_t t = t0 + (int64_t)unit * 64 + lane * 32;
            u_page = -1, u_at = 0, u_ks = 0.0f, u_vs = 0.0f;
            if (t < t1) {
                const int32_t p = a.table[(int64_t)r * a.table_width + t / block];
                u_at = (int32_t)(t % block);
                if ((uint32_t)p < (uint64_t)a.cache.pages) {
                    u_page = p;
                    u_ks = a.cache.k_scales[(int64_t)p * heads + h], u_vs = a.cache.v_scales[(int64_t)p * heads + h];
                }
            }
        };
        w32x4 kr[PIECES], vr[PIECES];
        auto load = [&](int unit) {
            const int i = (unit - looked) * 2;
            const int p[2] = {max(__builtin_amdgcn_readlane(u_page, i), 0), max(__builtin_amdgcn_readlane(u_page, i + 1), 0)};
            const int at[2] = {__builtin_amdgcn_readlane(u_at, i), __builtin_amdgcn_readlane(u_at, i + 1)};
            const int8_t *const kb[2] = {a.cache.k_codes + (((int64_t)p[0] * heads + h) * block + at[0]) * D, a.cache.k_codes + (((int64_t)p[1] * heads + h) * block + at[1]) * D};
            const int8_t *const vb[2] = {a.cache.v_codes + ((int64_t)p[0] * heads + h) * block * D + at[0], a.cache.v_codes + ((int64_t)p[1] * heads + h) * block * D + at[1]};
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                const int piece = x * 64 * WAVES + tid;
                if (!EVEN && piece >= 4 * D) break;
                const int token = piece / (D / 16), d16 = piece % (D / 16);
                kr[x] = *reinterpret_cast<const w32x4 *>((token < 32 ? kb[0] : kb[1]) + (token & 31) * D + 16 * d16);
                const int d = piece >> 2, seg = piece & 3;
                vr[x] = *reinterpret_cast<const w32x4 *>((seg < 2 ? vb[0] : vb[1]) + (int64_t)d * block + 16 * (seg & 1));
            }
        };
        auto stage = [&](int buf) {
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                const int piece = x * 64 * WAVES + tid;
                if (!EVEN && piece >= 4 * D) break;
                const int token = piece / (D / 16), d16 = piece % (D / 16);
                const int row = (token & ~12) | (token & 4) << 1 | (token & 8) >> 1;
                *reinterpret_cast<h16x8 *>(&s_k[buf][row][16 * d16]) = codes_to_halves8(kr[x][0], kr[x][1]);
                *reinterpret_cast<h16x8 *>(&s_k[buf][row][16 * d16 + 8]) = codes_to_halves8(kr[x][2], kr[x][3]);
                const int d = piece >> 2, seg = piece & 3;
                *reinterpret_cast<h16x8 *>(&s_v[buf][d][16 * seg]) = codes_to_halves8(vr[x][0], vr[x][1]);
                *reinterpret_cast<h16x8 *>(&s_v[buf][d][16 * seg + 8]) = codes_to_halves8(vr[x][2], vr[x][3]);
            }
        };

        __syncthreads(); // the buffers' last readers (of the block of rows before) are done
        if (units > 0) {
            look_up(0);
            load(0);
            stage(0);
        }
        __syncthreads();
        for (int u = 0; u < units; ++u) {
            const int buf = u & 1;
            const int64_t t = t0 + (int64_t)u * 64;
            float ks[2];
            int vs[2]; // value scales' patterns (scalar arithmetic)
            bool missing[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int i = (u - looked) * 2 + y;
                missing[y] = __builtin_amdgcn_readlane(u_page, i) < 0;
                ks[y] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u_ks), i));
                vs[y] = __builtin_amdgcn_readlane(__builtin_bit_cast(int, u_vs), i);
            }
            if (u + 1 < units) {
                if (u + 1 - looked == 32) look_up(u + 1);
                load(u + 1);
            }
            if (!idle && t <= wave_last && !(a.window > 0 && t + 63 <= wave_first - a.window)) {
                f32x16 s[2];
                const auto scores = [&] {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.0f;
#pragma unroll
                    for (int k = 0; k < KS; ++k)
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const h16x8 kf = *reinterpret_cast<const h16x8 *>(&s_k[buf][32 * y + c][16 * k + 8 * hh]);
                            s[y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[k], s[y], 0, 0, 0);
                        }
                    if (missing[0] || missing[1] || t + 63 > wave_first || (a.window > 0 && t <= wave_last - a.window)) {
                        asm volatile(""); // (a branch: few units are cut)
                        const int64_t base = t + 8 * hh;
                        const int to = (int)min(pos - base, (int64_t)64);
                        const int from = a.window > 0 ? (int)min(max(pos - a.window - base, (int64_t)-1), (int64_t)64) : -1;
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int at = 32 * y + 16 * (i >> 3) + (i & 7);
                                s[y][i] = (at <= to && at > from && !missing[y]) ? s[y][i] : -INFINITY;
                            }
                    }
                };
                scores();
                // references that no longer do
                float most, fk[2];
                bool grew = false;
                float top[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    fk[y] = fmaxf(factor * ks[y], 1e-30f); // (not 0: minus infinity stays that)
                    top[y] = s[y][0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) top[y] = fmaxf(top[y], s[y][i]);
                    top[y] *= fk[y];
                }
                most = fmaxf(top[0], top[1]);
                most = fmaxf(most, other_half(most));
                grew |= most > m + kRoom;
                const int vmost = max(vs[0], vs[1]); // (0 where there is no page)
                const bool move = vmost > 0 && !unit.is_near(vmost);
                const float to_unit = move ? unit.move_to(vmost) : 1.0f;
                if (__any(grew) || move) {
                    const float now = fmaxf(m, most), shrink = exp2_fast(m - now), by = shrink * to_unit;
                    m = now, l *= shrink;
                    far = __any(fabsf(m) >= kFarScore && m > kNothing);
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[v] *= by;
                }
                h16x8 p[4];
                // probabilities of a tile from the exponents of its scores; returns their sum
                const auto probabilities = [&](int y, auto exponent) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float e = exp2_fast(exponent(s[y][i]));
                        sum += e;
                        p[2 * y + (i >> 3)][i & 7] = (_Float16)e;
                    }
                    return sum;
                };
                const auto value = [&](int v, int k) { return *reinterpret_cast<const h16x8 *>(&s_v[buf][32 * v + c][16 * k + 8 * hh]); };
                const bool joined = !far && (missing[0] || unit.is_near(vs[0])) && (missing[1] || unit.is_near(vs[1])); // scales are part of p
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float ratio = joined && !missing[y] ? unit.of(vs[y]) : 1.0f;
                    const float off = joined ? __log2f(ratio) + kPromptHead - m : -INFINITY;
                    const float sum = probabilities(y, [&](float x) { return fmaf(x, fk[y], off); });
                    l = fmaf(sum, __builtin_amdgcn_rcpf(ratio), l); // (takes out of the sum what the scale has brought in)
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[v] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value(v, k), p[k], o[v], 0, 0, 0);
                if (!joined) { // nothing so far: each tile's product by itself, scores as they went into the maximum
                    asm volatile("" : "+v"(l)::"memory"); // (once more from the keys on: scores kept until here would take registers from every unit)
                    scores();
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        l += probabilities(y, [&](float x) {
                            float score = x * fk[y];
                            asm("" : "+v"(score)); // (rounded: not one operation with the difference)
                            return score - m + kPromptHead;
                        });
                        asm volatile("" : "+v"(l)); // (formed here: further down the sum would keep all of them)
                        const float scale = unit.of(vs[y]);
#pragma unroll
                        for (int v = 0; v < VT; ++v) {
                            f32x16 x;
#pragma unroll
                            for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
                            for (int k = 2 * y; k < 2 * y + 2; ++k) x = __builtin_amdgcn_mfma_f32_32x32x16_f16(value(v, k), p[k], x, 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[v][i] = fmaf(scale, x[i], o[v][i]);
                            __builtin_amdgcn_sched_barrier(0); // (one product's registers at a time)
                        }
                    }
                }
            }
            if (u + 1 < units) stage(buf ^ 1);
            __syncthreads();
        }

        l += other_half(l);
        if (wave_row + c >= rows) continue;
        if (chunks == 1) {
            const float inv = l != 0.0f ? unit.value() / l : 0.0f;
            uint16_t *out = a.out + row_id * D + 4 * hh;
#pragma unroll
            for (int v = 0; v < VT; ++v)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<w32x2 *>(out + 32 * v + 2 * i) = w32x2{narrow2<T>(o[v][i] * inv, o[v][i + 1] * inv), narrow2<T>(o[v][i + 2] * inv, o[v][i + 3] * inv)};
            if (a.lse && hh == 0) a.lse[row_id] = l != 0.0f ? (m - kPromptHead + log2f(l)) * 0.69314718056f : -INFINITY;
        } else {
            const bool large = unit.peak >= ValueUnit::exponent(__builtin_bit_cast(int, kLargeScale));
            const float own = ldexpf(unit.value(), large ? -kLargeUnit : 0);
            const int64_t part = part_row(a, r, h, rt + wave * 32 + c) * a.chunks + chunk;
#pragma unroll
            for (int v = 0; v < VT; ++v)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f32x4 *>(a.part_o + part * D + 32 * v + 2 * i + 4 * hh) =
                        f32x4{o[v][i], o[v][i + 1], o[v][i + 2], o[v][i + 3]} * own;
            if (hh == 0) a.part_ml[2 * part] = m - kPromptHead, a.part_ml[2 * part + 1] = large ? -l : l;
        }
    }
}

} // namespace qnn
