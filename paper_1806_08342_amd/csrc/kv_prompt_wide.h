// The kernel for many query rows, for large heads: accumulators and queries of 32 rows would leave no registers for two waves on
// a SIMD (heads of 256: 512 registers, most of them copied to and fro between the register file's halves, 5 us for 64 tokens by 128 rows).  Here a
// wave has 16 rows, on 16x16x32 tiles: twice the reads from LDS for each product, but eight waves.
// Five prompts up to 2047, 16 query heads of 256 over 4: 182 us (249 with 32 rows per wave), 485 TFLOP/s.  LDS is read in 33 % of the cycles,
// the vector unit works in 37 and the matrix units in 21; a wave waits for 44 % of its time: nearly every product for the fragment that is read
// from LDS right before it, with the next one's read behind it, and all waves at the barrier.  (Letting the second wave of each SIMD stage tokens before its products
// and the first after them changed nothing; uneven ends cost a tenth.)
#pragma once

#include "kv_prompt.h"

namespace qnn {

template <class T, int D> __global__ void __launch_bounds__(512, 2) attend_wide_kernel(const AttendArgs a)
{
    constexpr int WAVES = 8, BR = 16 * WAVES, KS = D / 32, VT = D / 16;
    constexpr int PIECES = (4 * D + 64 * WAVES - 1) / (64 * WAVES); // 16-byte pieces of 64 tokens' keys (or values) per thread
    constexpr bool EVEN = 4 * D % (64 * WAVES) == 0;
    // 16-byte pieces of a row are exchanged by its number.  A 16-byte read serves 16 lanes in a cycle: {0-3, 12-15, 20-27}, {4-11, 16-19,
    // 28-31} and the same + 32, here rows 0-3 and 12-15 of one piece with rows 4-11 of the next.  These meet 16 different places (of 16 bytes, in 256)
    // where a row is whole 256 bytes and the piece is turned by the row's number, or where two rows are and it is turned by half of that.
    constexpr int K_PIECES = D / 8, V_PIECES = 8;
    const auto k_place = [](int row, int piece) { return row * D + ((piece ^ (K_PIECES % 16 == 0 ? row & 15 : row >> 1 & 7)) * 8); };
    const auto v_place = [](int d, int piece) { return d * 64 + ((piece ^ (d >> 1 & 7)) * 8); };
    static_assert(K_PIECES % 8 == 0 && V_PIECES == 8, "rows of whole 128 bytes");
    __shared__ __attribute__((aligned(16))) _Float16 s_k[2][64 * D];
    __shared__ __attribute__((aligned(16))) _Float16 s_v[2][D * 64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
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
        const int wave_row = rt + wave * 16, row = wave_row + c;
        const int qi = min(row, rows - 1) / a.group, e = min(row, rows - 1) % a.group;
        const int64_t pos = row < rows ? pos0 + qi : -1, row_id = (rq.row0 + qi) * a.q_heads + h * a.group + e;
        h16x8 qf[KS];
        float factor;
        {
            const uint16_t *q = a.q + (rq.row0 + qi) * a.q_token_pitch + (int64_t)(h * a.group + e) * a.q_head_pitch + 8 * g;
            w32x4 raw[KS];
            float peak = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) raw[k] = load_any<w32x4>(q + 32 * k);
            if constexpr (!std::is_same_v<T, F16>)
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) peak = fmaxf(peak, fabsf(T::widen((uint16_t)(raw[k][i >> 1] >> (i & 1) * 16))));
            const int ex = std::is_same_v<T, F16> ? 0 : row_exponent(max_over_groups(peak));
            const float down = ldexpf(a.scale < 0.0f ? -1.0f : 1.0f, -ex); // (scores grow with the products: the sign goes to q)
            factor = fabsf(a.scale) * ldexpf(1.0f, ex);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) qf[k][i] = (_Float16)(T::widen((uint16_t)(raw[k][i >> 1] >> (i & 1) * 16)) * down);
        }
        const int64_t wave_first = pos0 + wave_row / a.group, wave_last = pos0 + min(wave_row + 15, rows - 1) / a.group;
        const bool idle = wave_row >= rows;

        f32x4 o[VT];
        float m = kNothing, l = 0.0f;
#pragma unroll
        for (int v = 0; v < VT; ++v) o[v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
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
                // token 32 * (s >> 1) + 8 * a + 4 * (s & 1) + b in row 16 * s + 4 * a + b
                const int row = (token & 32) | (token & 4) << 2 | (token & 24) >> 1 | (token & 3);
                *reinterpret_cast<h16x8 *>(&s_k[buf][k_place(row, 2 * d16)]) = codes_to_halves8(kr[x][0], kr[x][1]);
                *reinterpret_cast<h16x8 *>(&s_k[buf][k_place(row, 2 * d16 + 1)]) = codes_to_halves8(kr[x][2], kr[x][3]);
                const int d = piece >> 2, seg = piece & 3;
                *reinterpret_cast<h16x8 *>(&s_v[buf][v_place(d, 2 * seg)]) = codes_to_halves8(vr[x][0], vr[x][1]);
                *reinterpret_cast<h16x8 *>(&s_v[buf][v_place(d, 2 * seg + 1)]) = codes_to_halves8(vr[x][2], vr[x][3]);
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
                f32x4 s[4]; // (products of different tiles follow each other: one that waits for the last of its own takes twice as long)
                const auto scores = [&] {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < KS; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const h16x8 *>(&s_k[buf][k_place(16 * i + c, 4 * k + g)]), qf[k], s[i], 0, 0, 0);
                    if (missing[0] || missing[1] || t + 63 > wave_first || (a.window > 0 && t <= wave_last - a.window)) {
                        asm volatile(""); // (a branch: few units are cut)
                        const int64_t base = t + 8 * g;
                        const int to = (int)min(pos - base, (int64_t)64);
                        const int from = a.window > 0 ? (int)min(max(pos - a.window - base, (int64_t)-1), (int64_t)64) : -1;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const int at = 32 * (i >> 1) + 4 * (i & 1) + x;
                                s[i][x] = (at <= to && at > from && !missing[i >> 1]) ? s[i][x] : -INFINITY;
                            }
                    }
                };
                scores();
                // references that no longer do
                float fk[2], most = -INFINITY;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    fk[y] = fmaxf(factor * ks[y], 1e-30f); // (not 0: minus infinity stays that)
                    float top = s[2 * y][0];
#pragma unroll
                    for (int i = 1; i < 8; ++i) top = fmaxf(top, s[2 * y + (i >> 2)][i & 3]);
                    most = fmaxf(most, top * fk[y]);
                }
                most = max_over_groups(most);
                const int vmost = max(vs[0], vs[1]); // (0 where there is no page)
                const bool move = vmost > 0 && !unit.is_near(vmost);
                const float to_unit = move ? unit.move_to(vmost) : 1.0f;
                if (__any(most > m + kRoom) || move) {
                    const float now = fmaxf(m, most), shrink = exp2_fast(m - now), by = shrink * to_unit;
                    m = now, l *= shrink;
                    far = __any(fabsf(m) >= kFarScore && m > kNothing);
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[v] *= by;
                }
                h16x8 p[2];
                // probabilities of a tile from the exponents of its scores; returns their sum
                const auto probabilities = [&](int y, auto exponent) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = exp2_fast(exponent(s[2 * y + (i >> 2)][i & 3]));
                        sum += x;
                        p[y][i] = (_Float16)x;
                    }
                    return sum;
                };
                const auto value = [&](int v, int y) { return *reinterpret_cast<const h16x8 *>(&s_v[buf][v_place(16 * v + c, 4 * y + g)]); };
                const bool joined = !far && (missing[0] || unit.is_near(vs[0])) && (missing[1] || unit.is_near(vs[1])); // scales are part of p
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float ratio = joined && !missing[y] ? unit.of(vs[y]) : 1.0f;
                    const float off = joined ? __log2f(ratio) + kPromptHead - m : -INFINITY;
                    const float sum = probabilities(y, [&](float x) { return fmaf(x, fk[y], off); });
                    l = fmaf(sum, __builtin_amdgcn_rcpf(ratio), l); // (takes out of the sum what the scale has brought in)
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[v] = __builtin_amdgcn_mfma_f32_16x16x32_f16(value(v, y), p[y], o[v], 0, 0, 0);
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
                            const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_f16(value(v, y), p[y], f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[v][e] = fmaf(scale, x[e], o[v][e]);
                            __builtin_amdgcn_sched_barrier(0); // (one product's registers at a time)
                        }
                    }
                }
            }
            if (u + 1 < units) stage(buf ^ 1);
            __syncthreads();
        }

        l = sum_over_groups(l);
        if (row >= rows) continue;
        if (chunks == 1) {
            const float inv = l != 0.0f ? unit.value() / l : 0.0f;
            uint16_t *out = a.out + row_id * D + 4 * g;
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                const f32x4 x = o[v] * inv;
                *reinterpret_cast<w32x2 *>(out + 16 * v) = w32x2{narrow2<T>(x[0], x[1]), narrow2<T>(x[2], x[3])};
            }
            if (a.lse && g == 0) a.lse[row_id] = l != 0.0f ? (m - kPromptHead + log2f(l)) * 0.69314718056f : -INFINITY;
        } else {
            const bool large = unit.peak >= ValueUnit::exponent(__builtin_bit_cast(int, kLargeScale));
            const float own = ldexpf(unit.value(), large ? -kLargeUnit : 0);
            const int64_t part = part_row(a, r, h, row) * a.chunks + chunk;
#pragma unroll
            for (int v = 0; v < VT; ++v) *reinterpret_cast<f32x4 *>(a.part_o + part * D + 16 * v + 4 * g) = o[v] * own;
            if (g == 0) a.part_ml[2 * part] = m - kPromptHead, a.part_ml[2 * part + 1] = large ? -l : l;
        }
    }
}

} // namespace qnn
