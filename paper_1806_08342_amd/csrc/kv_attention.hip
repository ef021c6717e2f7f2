// Attention of query heads over a paged cache of 8-bit codes (qnn_kv_attention).
//
//   o = sum_t softmax_t(scale * ks[t] * q . ck[t]) * vs[t] * cv[t],  ks, vs: one scale per page and head
//
// One pass over the tokens with a running maximum m and sum l; a page's key scale multiplies its scores, its value scale the
// product of its probabilities with its codes, so that the codes themselves go through the matrix units, in binary16, where
// they are exact.
//
// The products are formed transposed, S^T = K q^T and O^T = V^T p^T on 16x16x32 tiles: a lane's column is one query row
// throughout, the maximum over tokens is a maximum over the lane's registers and four lanes, and which token a row
// of S^T stands for is free to choose.  It is chosen so that the four rows that a lane gets of each tile are tokens that lie one
// after the other in its part of the value product: the probabilities go from the first product into the second in the lane
// that holds them, without LDS or shuffles.  Keys and values come straight from memory into registers: each wave
// reads tokens of its own, so nothing would be shared through LDS.
//
// Bound by reading codes: 4 contexts of 131072 tokens, 40 query heads of 128 over 8: 190 us, 5.7 TB/s; 32 up to 8000, 64 heads over 8: 67 us, where
// the longest contexts end last; one of 777: 10 us, two launches (7 and 3) and a chain of loads.
#include "kv_attention.h"
#include "kv_prompt.h"
#include "kv_prompt_wide.h"

namespace qnn {

// One unit of U tokens per wave and step; four waves take units in turn.  NT tiles of 16 query rows (row = query * group + head of
// the group) share the cache's codes.
template <class T, int D, int U, int NT> __global__ void __launch_bounds__(256, D * NT <= 128 ? 2 : 1) attend_few_kernel(const AttendArgs a)
{
    constexpr int J = D / 64, TAIL = D % 64 != 0; // key pieces of 64 channels (16 bytes a lane), and one of 32
    constexpr int S = U / 16, VW = U / 16;        // score tiles; dwords of a value row that a lane takes
    constexpr int VT = D / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int h = blockIdx.y;
    const int chunk = blockIdx.x % a.chunks, rb = blockIdx.x / a.chunks % a.row_blocks, r = blockIdx.x / a.chunks / a.row_blocks;
    const Request rq = request_of<U>(a, r);
    const int rows = rq.n * a.group;
    if (rows <= a.rows_over || rows > a.rows_upto) return;
    const int chunks = chunks_of(a, rq);
    if (chunk >= chunks) return;
    const int64_t t0 = rq.low + (int64_t)chunk * a.chunk_tokens;
    const int block = a.cache.block, heads = a.cache.heads;

    __shared__ float s_m[4][16 * NT], s_l[4][16 * NT];
    __shared__ int s_large[4];
    __shared__ __attribute__((aligned(16))) float s_o[2][16 * NT][D + 4];

    for (int rt = rb * 16 * NT; rt < rows; rt += a.row_blocks * 16 * NT) {
        // queries: this lane's row of each tile, the channels that its key bytes have
        h16x8 qf[NT][J * 2 + TAIL];
        float factor[NT];
        int64_t pos[NT], row_id[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = rt + nt * 16 + c, qi = min(row, rows - 1) / a.group, e = min(row, rows - 1) % a.group;
            pos[nt] = row < rows ? rq.length - rq.n + qi : -1; // a row beyond the last sees nothing
            row_id[nt] = (rq.row0 + qi) * a.q_heads + h * a.group + e;
            const uint16_t *q = a.q + (rq.row0 + qi) * a.q_token_pitch + (int64_t)(h * a.group + e) * a.q_head_pitch;
            w32x4 raw[J * 2 + TAIL];
#pragma unroll
            for (int j = 0; j < J * 2 + TAIL; ++j)
                raw[j] = load_any<w32x4>(q + (j < 2 * J ? 64 * (j >> 1) + 16 * g + 8 * (j & 1) : 64 * J + 8 * g));
            float v[8 * (J * 2 + TAIL)], peak = 0.0f;
#pragma unroll
            for (int i = 0; i < 8 * (J * 2 + TAIL); ++i) {
                v[i] = T::widen((uint16_t)(raw[i >> 3][i >> 1 & 3] >> (i & 1) * 16));
                peak = fmaxf(peak, fabsf(v[i]));
            }
            const int ex = std::is_same_v<T, F16> ? 0 : row_exponent(max_over_groups(peak));
            const float down = ldexpf(1.0f, -ex);
            factor[nt] = a.scale * ldexpf(1.0f, ex);
#pragma unroll
            for (int j = 0; j < J * 2 + TAIL; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) qf[nt][j][i] = (_Float16)(v[j * 8 + i] * down);
        }
        // tokens beyond what the last row of this block sees are left out
        const int last_row = min(rt + 16 * NT, rows) - 1;
        const int64_t t1 = min(chunk + 1 < chunks ? min(rq.high, t0 + a.chunk_tokens) : rq.high, rq.length - rq.n + last_row / a.group + 1);
        const int64_t first_pos = rq.length - rq.n + rt / a.group, last_pos = rq.length - rq.n + last_row / a.group;
        const int units = t1 > t0 ? (int)((t1 - t0 + U - 1) / U) : 0;
        const int mine = (units - wave + 3) / 4; // units wave, wave + 4, ...

        f32x4 o[NT][VT];
        float m[NT], l[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt] = kNothing, l[nt] = 0.0f;
#pragma unroll
            for (int v = 0; v < VT; ++v) o[nt][v] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        // lane i holds page, place in the page and scales of the i-th of 64 units
        int32_t u_page = 0, u_at = 0;
        float u_ks = 0.0f, u_vs = 0.0f;
        auto look_up = [&](int from) {
            const int64_t t = t0 + (int64_t)(wave + 4 * (from + lane)) * U;
            u_page = -1, u_at = 0, u_ks = 0.0f, u_vs = 0.0f;
            if (from + lane < mine) {
                const int32_t p = a.table[(int64_t)r * a.table_width + t / block];
                u_at = (int32_t)(t % block);
                if ((uint32_t)p < (uint64_t)a.cache.pages) {
                    u_page = p;
                    u_ks = a.cache.k_scales[(int64_t)p * heads + h], u_vs = a.cache.v_scales[(int64_t)p * heads + h];
                }
            }
        };
        w32x4 kr[S][J];
        w32x2 kt[S];
        uint32_t vr[VT][VW];
        // (a unit without a page reads page 0 and is masked)
        auto load_keys = [&](int k) {
            const int p = max(__builtin_amdgcn_readlane(u_page, k & 63), 0), at = __builtin_amdgcn_readlane(u_at, k & 63);
            const int8_t *base = a.cache.k_codes + (((int64_t)p * heads + h) * block + at) * D;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int8_t *row = base + ((c >> 2) * (U / 4) + s * 4 + (c & 3)) * D;
#pragma unroll
                for (int j = 0; j < J; ++j) kr[s][j] = *reinterpret_cast<const w32x4 *>(row + 64 * j + 16 * g);
                if (TAIL) kt[s] = *reinterpret_cast<const w32x2 *>(row + 64 * J + 8 * g);
            }
        };
        auto load_values = [&](int k) {
            const int p = max(__builtin_amdgcn_readlane(u_page, k & 63), 0), at = __builtin_amdgcn_readlane(u_at, k & 63);
            const int8_t *base = a.cache.v_codes + ((int64_t)p * heads + h) * block * D + at + g * (U / 4);
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                const int8_t *row = base + (int64_t)(v * 16 + c) * block;
                if constexpr (VW == 4) {
                    const w32x4 w = *reinterpret_cast<const w32x4 *>(row);
                    vr[v][0] = w[0], vr[v][1] = w[1], vr[v][2] = w[2], vr[v][3] = w[3];
                } else {
                    const w32x2 w = *reinterpret_cast<const w32x2 *>(row);
                    vr[v][0] = w[0], vr[v][1] = w[1];
                }
            }
        };

        bool large = false; // o stands in units of 2^kLargeUnit
        for (int from = 64; from < mine; from += 64) {
            look_up(from);
            large |= (bool)__any(u_vs > kLargeScale);
        }
        if (mine > 0) {
            look_up(0);
            load_keys(0);
            load_values(0);
            large |= (bool)__any(u_vs > kLargeScale);
        }
        const float in_unit = ldexpf(1.0f, large ? -kLargeUnit : 0);
        u_vs *= in_unit;
        for (int k = 0; k < mine; ++k) {
            const int64_t t = t0 + (int64_t)(wave + 4 * k) * U;
            const bool missing = __builtin_amdgcn_readlane(u_page, k & 63) < 0;
            const float ks = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u_ks), k & 63));
            const float vs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, u_vs), k & 63));
            f32x4 s[NT][S];
#pragma unroll
            for (int i = 0; i < S; ++i) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[nt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const h16x8 kf = codes_to_halves8(kr[i][j][2 * half], kr[i][j][2 * half + 1]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            s[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[nt][2 * j + half], s[nt][i], 0, 0, 0);
                    }
                if constexpr (TAIL) {
                    const h16x8 kf = codes_to_halves8(kt[i][0], kt[i][1]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) s[nt][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[nt][2 * J], s[nt][i], 0, 0, 0);
                }
            }
            const bool more = k + 1 < mine, refill = ((k + 1) & 63) == 0;
            if (more && !refill) load_keys(k + 1);

            // probabilities, and what the accumulators are rescaled with where a maximum grew
            const bool masked = missing || t + U - 1 > first_pos || (a.window > 0 && t <= last_pos - a.window);
            h16x8 p[NT][U / 32];
            float shrink[NT];
            bool grew = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float f = factor[nt] * ks;
                float top = kNothing;
#pragma unroll
                for (int i = 0; i < S; ++i) s[nt][i] *= f;
                if (masked) {
                    // tokens of this lane that its row sees: base + (from, to]
                    const int64_t base = t + g * (U / 4);
                    const int to = missing ? -1 : (int)min(pos[nt] - base, (int64_t)U);
                    const int from = a.window > 0 ? (int)min(max(pos[nt] - a.window - base, (int64_t)-1), (int64_t)U) : -1;
#pragma unroll
                    for (int i = 0; i < S; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[nt][i][e] = (i * 4 + e <= to && i * 4 + e > from) ? s[nt][i][e] : -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, s[nt][i][e]);
                const float now = fmaxf(m[nt], max_over_groups(top)), against = reference_of(now);
                shrink[nt] = exp2_fast(reference_of(m[nt]) - against);
                grew |= now > m[nt];
                m[nt] = now;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < S; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = exp2_fast(s[nt][i][e] - against);
                        sum += x;
                        p[nt][i >> 1][(i & 1) * 4 + e] = (_Float16)x;
                    }
                l[nt] = l[nt] * shrink[nt] + sum;
            }
            if (__any(grew)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[nt][v] *= shrink[nt];
            }
#pragma unroll
            for (int v = 0; v < VT; ++v)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int half = 0; half < U / 32; ++half)
                        x = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_halves8(vr[v][2 * half], vr[v][2 * half + 1]), p[nt][half], x, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][v][e] = fmaf(vs, x[e], o[nt][v][e]);
                }
            if (more) {
                if (refill) {
                    look_up(k + 1);
                    u_vs *= in_unit;
                    load_keys(k + 1);
                }
                load_values(k + 1);
            }
        }

        // the four waves' parts, joined: two of them, then the other two, in a fixed order
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            l[nt] = sum_over_groups(l[nt]), m[nt] = reference_of(m[nt]); // (references from here on)
            if (g == 0) s_m[wave][nt * 16 + c] = m[nt], s_l[wave][nt * 16 + c] = l[nt];
        }
        if (lane == 0) s_large[wave] = large;
        __syncthreads();
        const bool any_large = s_large[0] | s_large[1] | s_large[2] | s_large[3];
        const float unit = ldexpf(1.0f, any_large && !large ? -kLargeUnit : 0), back = ldexpf(1.0f, any_large ? kLargeUnit : 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float top = s_m[0][nt * 16 + c], sum = 0.0f;
#pragma unroll
            for (int w = 1; w < 4; ++w) top = fmaxf(top, s_m[w][nt * 16 + c]);
#pragma unroll
            for (int w = 0; w < 4; ++w) sum += s_l[w][nt * 16 + c] * exp2_fast(s_m[w][nt * 16 + c] - top);
            const float by = exp2_fast(m[nt] - top) * unit;
            m[nt] = top, l[nt] = sum;
#pragma unroll
            for (int v = 0; v < VT; ++v) o[nt][v] *= by;
        }
#pragma unroll
        for (int half = 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int v = 0; v < VT; ++v) *reinterpret_cast<f32x4 *>(&s_o[wave - half][nt * 16 + c][v * 16 + g * 4]) = o[nt][v];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int v = 0; v < VT; ++v) o[nt][v] += *reinterpret_cast<const f32x4 *>(&s_o[wave][nt * 16 + c][v * 16 + g * 4]);
            __syncthreads();
        }
        if (wave == 0)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (rt + nt * 16 + c >= rows) continue;
                if (chunks == 1) {
                    const float inv = l[nt] != 0.0f ? 1.0f / l[nt] : 0.0f;
                    uint16_t *out = a.out + row_id[nt] * D;
#pragma unroll
                    for (int v = 0; v < VT; ++v) {
                        const f32x4 x = o[nt][v] * inv * back;
                        *reinterpret_cast<w32x2 *>(out + v * 16 + g * 4) = w32x2{narrow2<T>(x[0], x[1]), narrow2<T>(x[2], x[3])};
                    }
                    if (a.lse && g == 0) a.lse[row_id[nt]] = l[nt] != 0.0f ? (m[nt] + log2f(l[nt])) * 0.69314718056f : -INFINITY;
                } else {
                    const int64_t part = part_row(a, r, h, rt + nt * 16 + c) * a.chunks + chunk;
#pragma unroll
                    for (int v = 0; v < VT; ++v) *reinterpret_cast<f32x4 *>(a.part_o + part * D + v * 16 + g * 4) = o[nt][v];
                    if (g == 0) a.part_ml[2 * part] = m[nt], a.part_ml[2 * part + 1] = any_large ? -l[nt] : l[nt];
                }
            }
    }
}

// Joins the chunks of a row.  SHARED: one workgroup per row, whose four waves take chunks in turn (few rows of many chunks); else a
// wave per row.
template <class T, int D, int U, bool SHARED> __global__ void __launch_bounds__(256) attend_join_kernel(const AttendArgs a, int rows_at_once)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y;
    const int groups = SHARED ? rows_at_once : (rows_at_once + 3) / 4; // workgroups per request
    const int sub = SHARED ? blockIdx.x % groups : (blockIdx.x % groups) * 4 + wave, r = blockIdx.x / groups;
    const Request rq = request_of<U>(a, r);
    const int rows = rq.n * a.group;
    if (rows <= a.rows_over || rows > a.rows_upto) return;
    const int chunks = chunks_of(a, rq);
    if (chunks == 1) return;
    __shared__ float s_l[4], s_o[4][SHARED ? D : 1];
    for (int row = sub; row < rows; row += SHARED ? groups : 4 * groups) {
        const int64_t id = (rq.row0 + row / a.group) * a.q_heads + h * a.group + row % a.group;
        const int64_t part = part_row(a, r, h, row) * a.chunks;
        const float *ml = a.part_ml + part * 2, *po = a.part_o + part * D;
        float top = kNothing;
        bool large = false;
        for (int i = lane; i < chunks; i += 64) top = fmaxf(top, ml[2 * i]), large |= ml[2 * i + 1] < 0.0f;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
        large = __any(large);
        const float ordinary = ldexpf(1.0f, large ? -kLargeUnit : 0), back = ldexpf(1.0f, large ? kLargeUnit : 0);
        float o[(D + 63) / 64] = {}, l = 0.0f;
#pragma unroll 4
        for (int i = SHARED ? wave : 0; i < chunks; i += SHARED ? 4 : 1) {
            const float part_l = ml[2 * i + 1];
            float w = exp2_fast(ml[2 * i] - top);
            l += w * fabsf(part_l);
            w *= part_l < 0.0f ? 1.0f : ordinary;
#pragma unroll
            for (int d = 0; d < (D + 63) / 64; ++d)
                if (D % 64 == 0 || d * 64 + lane < D) o[d] = fmaf(w, po[(int64_t)i * D + d * 64 + lane], o[d]);
        }
        if (SHARED) {
            if (lane == 0) s_l[wave] = l;
#pragma unroll
            for (int d = 0; d < (D + 63) / 64; ++d)
                if (D % 64 == 0 || d * 64 + lane < D) s_o[wave][d * 64 + lane] = o[d];
            __syncthreads();
            l = (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]);
            const int d = threadIdx.x;
            if (d < D) {
                const float x = (s_o[0][d] + s_o[1][d]) + (s_o[2][d] + s_o[3][d]);
                a.out[id * D + d] = T::narrow(l != 0.0f ? x / l * back : 0.0f);
            }
        } else {
            const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
            for (int d = 0; d < (D + 63) / 64; ++d)
                if (D % 64 == 0 || d * 64 + lane < D) a.out[id * D + d * 64 + lane] = T::narrow(o[d] * inv * back);
        }
        if (a.lse && (SHARED ? threadIdx.x == 0 : lane == 0)) a.lse[id] = l != 0.0f ? (top + log2f(l)) * 0.69314718056f : -INFINITY;
        if (SHARED) __syncthreads();
    }
}

// One launch over a batch: the kernel for few rows, or that for many.
struct AttendLaunch {
    bool used = false;
    int tiles = 1, waves = 8, row_blocks = 1, chunks = 1, part_rows = 0, rows_over = 0, rows_upto = INT32_MAX;
    int64_t chunk_tokens = 256;
    size_t part_bytes(int64_t requests, const qnn_kv_cache &c) const
    {
        return used && chunks > 1 ? (size_t)requests * c.heads * part_rows * chunks * (c.dim + 2) * sizeof(float) : 0;
    }
};
struct AttendPlan {
    AttendLaunch few, many;
};

// Into how many chunks the context is divided: 1, 2, 4 ... 128, whichever is estimated to take least.  A workgroup takes 4 us to
// begin and to join its waves, and for each turn of its four waves 1 us per 4000 bytes of a wave's unit where a CU has one workgroup,
// per 3000 where it has two (what 4 contexts of 131072 tokens took in 8 and 16 chunks: 272 and 185 us); joining chunks is another
// launch, 5 us.  32 contexts up to 8000 took 64 us undivided, 65, 70 and 75 in 2, 4 and 8; 48 windows of 1024 16 undivided, 20 in 2.
static void divide_context(AttendLaunch &p, int64_t reach, int64_t groups, int64_t unit, int64_t unit_bytes, int per_cu)
{
    const int64_t turn = 4 * unit, turns = (reach + turn - 1) / turn;
    double best = 0.0;
    for (int64_t n = 1; n <= 128 && n <= (turns > 1 ? turns : 1); n *= 2) {
        const int64_t workgroups = groups * n, rounds = (workgroups + 256 * per_cu - 1) / (256 * per_cu);
        const double turn_us = (double)unit_bytes / (workgroups > 256 && per_cu > 1 ? 3000.0 : 4000.0);
        const double us = (double)rounds * (4.0 + (double)((turns + n - 1) / n) * turn_us) + (n > 1 ? 5.0 + 0.05 * (double)n : 0.0);
        if (n == 1 || us < best) best = us, p.chunk_tokens = (turns + n - 1) / n * turn;
    }
    if (p.chunk_tokens < turn) p.chunk_tokens = turn;
    p.chunks = (int)((reach + p.chunk_tokens - 1) / p.chunk_tokens);
    if (p.chunks < 1) p.chunks = 1;
}

// The same for requests with many rows, into at most 16.  A workgroup takes 4 us to begin and, for each 64 tokens, 2.5 us for heads up to 128,
// 3.8 for 192 and 5 for 256; the chip has 256 of 8 waves at a time, twice as many of 4; of a prompt's tokens a row sees half; parts are written
// and read at 6 TB/s, the latter in a launch of 5 us.  (Two prompts up to 1616, 8 query heads of 192: 86 us undivided, 84 in two chunks; five of 387, 2 of
// 128: 21 and 20.)
static void divide_prompts(AttendLaunch &p, int64_t reach, int64_t groups, int64_t blocks, int64_t rows, int dim, bool half)
{
    const int64_t units = (reach + 63) / 64;
    const double unit_us = dim > 128 ? dim / 51.0 : 2.5, share = (dim > 128 || p.waves == 8 ? 1.0 : 0.5) * (double)(groups * blocks) / 256.0;
    double best = 0.0;
    for (int64_t n = 1; n <= 16 && n <= (units > 1 ? units : 1); n *= 2) {
        const double one = 4.0 + (double)((units + n - 1) / n) * unit_us, all = share * ((double)units * (half ? 0.5 : 1.0) * unit_us + 4.0 * (double)n);
        const double us = (one > all ? one : all) + (n > 1 ? 5.0 + (double)(rows * groups * dim * n) * 8.0 / 6.0e6 : 0.0);
        if (n == 1 || us < best) best = us, p.chunk_tokens = (units + n - 1) / n * 64;
    }
    if (p.chunk_tokens < 64) p.chunk_tokens = 64;
    p.chunks = (int)((reach + p.chunk_tokens - 1) / p.chunk_tokens);
    if (p.chunks < 1) p.chunks = 1;
}

constexpr int kFewRows = 64;
// A launch has fewer than 2^32 threads along x (workgroups beyond them are left out without an error); workgroups loop over blocks of rows where there are more.
constexpr int64_t kMostGroups512 = (1 << 23) - 1, kMostGroups256 = (1 << 24) - 1;

static AttendPlan attend_plan(const qnn_kv_cache &cache, int q_heads, int64_t table_width, int64_t requests, int64_t tokens, int64_t window,
                              int64_t max_queries)
{
    AttendPlan p;
    if (max_queries <= 0 || max_queries > tokens) max_queries = tokens;
    const int64_t rows = max_queries * (q_heads / cache.heads), groups = requests * cache.heads;
    int64_t reach = table_width * cache.block;
    if (window > 0 && window < reach && window + max_queries + 127 < reach) reach = window + max_queries + 127;
    // Requests with few rows among others with many: a prompt's workgroups would walk along a long context for each of them
    p.few.used = rows <= kFewRows || requests > 1;
    p.many.used = rows > kFewRows;
    if (p.few.used) {
        const int64_t few = rows < kFewRows ? rows : kFewRows;
        const int most = cache.dim <= 64 ? 4 : cache.dim <= 128 ? 2 : 1; // (more do not fit the registers)
        p.few.tiles = few <= 16 || most == 1 ? 1 : few <= 32 || most == 2 ? 2 : 4;
        p.few.row_blocks = (int)((few + p.few.tiles * 16 - 1) / (p.few.tiles * 16));
        p.few.part_rows = (int)few;
        if (p.many.used) p.few.rows_upto = kFewRows;
        const int64_t unit = cache.block % 64 == 0 ? 64 : 32;
        divide_context(p.few, reach, groups * p.few.row_blocks, unit, unit * cache.dim * 2, p.few.tiles * cache.dim <= 128 ? 2 : 1);
        if (requests * p.few.row_blocks * p.few.chunks > kMostGroups256) p.few.chunks = 1; // (2^20 requests of 4 blocks are within it)
    }
    if (p.many.used) {
        if (p.few.used) p.many.rows_over = kFewRows;
        const int64_t wide = (rows + 255) / 256;
        p.many.waves = cache.dim > 128 || groups * wide < 256 ? 4 : 8;
        const int64_t blocks = (rows + 32 * p.many.waves - 1) / (32 * p.many.waves);
        p.many.part_rows = (int)rows;
        divide_prompts(p.many, reach, groups, blocks, rows, cache.dim, max_queries * 2 > reach);
        int64_t at_once = blocks < 4096 ? blocks : 4096;
        if (groups * p.many.chunks * at_once > kMostGroups512) at_once = kMostGroups512 / (groups * p.many.chunks);
        p.many.row_blocks = (int)(at_once > 1 ? at_once : 1);
    }
    return p;
}

template <class T, int D, int U> static void run_few(const AttendArgs &a, const AttendLaunch &p, hipStream_t s)
{
    constexpr int MOST = D <= 64 ? 4 : D <= 128 ? 2 : 1;
    const dim3 grid((unsigned)((int64_t)a.requests * p.row_blocks * p.chunks), (unsigned)a.cache.heads);
    if (p.tiles == 1) hipLaunchKernelGGL((attend_few_kernel<T, D, U, 1>), grid, dim3(256), 0, s, a);
    else if (p.tiles == 2) hipLaunchKernelGGL((attend_few_kernel<T, D, U, (MOST < 2 ? MOST : 2)>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attend_few_kernel<T, D, U, MOST>), grid, dim3(256), 0, s, a);
}

template <class T, int D> static void run_many(const AttendArgs &a, const AttendLaunch &p, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.requests * p.row_blocks * p.chunks * a.cache.heads));
    if constexpr (D > 128) hipLaunchKernelGGL((attend_wide_kernel<T, D>), grid, dim3(512), 0, s, a);
    else if (p.waves == 4) hipLaunchKernelGGL((attend_prompt_kernel<T, D, 4>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attend_prompt_kernel<T, D, 8>), grid, dim3(512), 0, s, a);
}

template <class T, int D, int U> static void run_join(const AttendArgs &a, hipStream_t s)
{
    int64_t per = a.part_rows < 4096 ? a.part_rows : 4096;
    if (a.requests * ((per + 3) / 4) > kMostGroups256) per = kMostGroups256 / a.requests * 4; // (at most 2^20 requests)
    const unsigned heads = (unsigned)a.cache.heads;
    // waves enough for the chip (or few chunks): one per row
    if (a.requests * per * heads >= 2048 || a.chunks <= 8)
        hipLaunchKernelGGL((attend_join_kernel<T, D, U, false>), dim3((unsigned)(a.requests * ((per + 3) / 4)), heads), dim3(256), 0, s, a, (int)per);
    else
        hipLaunchKernelGGL((attend_join_kernel<T, D, U, true>), dim3((unsigned)(a.requests * per), heads), dim3(256), 0, s, a, (int)per);
}

template <class T, int D> static qnn_status run_attend(AttendArgs a, const AttendPlan &p, char *workspace, hipStream_t s)
{
    const auto with = [&](const AttendLaunch &l) {
        a.chunk_tokens = (int32_t)l.chunk_tokens, a.chunks = l.chunks, a.row_blocks = l.row_blocks;
        a.part_rows = l.part_rows, a.rows_over = l.rows_over, a.rows_upto = l.rows_upto;
        a.part_o = reinterpret_cast<float *>(workspace);
        a.part_ml = a.part_o + (size_t)a.requests * a.cache.heads * l.part_rows * l.chunks * D;
        workspace += l.part_bytes(a.requests, a.cache);
    };
    if (p.many.used) {
        with(p.many);
        run_many<T, D>(a, p.many, s);
        if (p.many.chunks > 1) run_join<T, D, 64>(a, s);
    }
    if (p.few.used) {
        with(p.few);
        if (a.cache.block % 64 == 0) run_few<T, D, 64>(a, p.few, s);
        else run_few<T, D, 32>(a, p.few, s);
        if (p.few.chunks > 1 && a.cache.block % 64 == 0) run_join<T, D, 64>(a, s);
        else if (p.few.chunks > 1) run_join<T, D, 32>(a, s);
    }
    return launch_status(hipGetLastError());
}

template <class T> static qnn_status run_attend_dim(const AttendArgs &a, const AttendPlan &p, char *workspace, hipStream_t s)
{
    switch (a.cache.dim) {
    case 64: return run_attend<T, 64>(a, p, workspace, s);
    case 96: return run_attend<T, 96>(a, p, workspace, s);
    case 128: return run_attend<T, 128>(a, p, workspace, s);
    case 192: return run_attend<T, 192>(a, p, workspace, s);
    default: return run_attend<T, 256>(a, p, workspace, s);
    }
}

} // namespace qnn

using namespace qnn;

extern "C" {

static bool bad_attend_sizes(const qnn_kv_cache *cache, int32_t q_heads, int64_t table_width, int64_t requests, int64_t tokens, int64_t window)
{
    return bad_cache(cache) || q_heads <= 0 || q_heads % cache->heads != 0 || table_width < 0 || requests < 0 || requests > (1 << 20) || tokens < 0 ||
           tokens > INT32_MAX || table_width > INT32_MAX / cache->block || window < 0 || tokens * (q_heads / cache->heads) > INT32_MAX;
}

size_t qnn_kv_attention_workspace_bytes(const qnn_kv_cache *cache, int32_t q_heads, int64_t table_width, int64_t requests, int64_t tokens,
                                        int64_t window, int64_t max_queries)
{
    if (bad_attend_sizes(cache, q_heads, table_width, requests, tokens, window) || requests == 0 || tokens == 0) return 0;
    const AttendPlan p = attend_plan(*cache, q_heads, table_width, requests, tokens, window, max_queries);
    return p.few.part_bytes(requests, *cache) + p.many.part_bytes(requests, *cache);
}

qnn_status qnn_kv_attention(const qnn_kv_cache *cache, const void *q, int64_t q_token_pitch, int64_t q_head_pitch, int32_t q_heads, int type,
                            const int32_t *cu, const int32_t *lengths, const int32_t *table, int64_t table_width, int64_t requests, int64_t tokens,
                            float scale, int64_t window, int64_t max_queries, void *out, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_attend_sizes(cache, q_heads, table_width, requests, tokens, window) || bad_half_type(type) || !isfinite(scale)) return QNN_EINVAL;
    if (requests == 0 || tokens == 0) return QNN_OK;
    if (!q || !cu || !lengths || !out || (table_width > 0 && !table)) return QNN_EINVAL;
    if (bad_cache_arrays(cache) || ((uintptr_t)out & 15) != 0) return QNN_EINVAL;
    const AttendPlan p = attend_plan(*cache, q_heads, table_width, requests, tokens, window, max_queries);
    const size_t need = qnn_kv_attention_workspace_bytes(cache, q_heads, table_width, requests, tokens, window, max_queries);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < need)) return QNN_EINVAL;
    if (requests * p.many.row_blocks * p.many.chunks * cache->heads > kMostGroups512) return QNN_EUNSUPPORTED;
    AttendArgs a{};
    a.cache = *cache, a.q = static_cast<const uint16_t *>(q), a.q_token_pitch = q_token_pitch, a.q_head_pitch = q_head_pitch;
    a.cu = cu, a.lengths = lengths, a.table = table, a.out = static_cast<uint16_t *>(out), a.lse = lse;
    a.table_width = table_width, a.tokens = tokens, a.window = window, a.scale = scale * 1.44269504089f;
    a.q_heads = q_heads, a.group = q_heads / cache->heads, a.requests = (int32_t)requests;
    char *const scratch = static_cast<char *>(workspace);
    return type == QNN_BF16 ? run_attend_dim<Bf16>(a, p, scratch, as_stream(stream)) : run_attend_dim<F16>(a, p, scratch, as_stream(stream));
}

} // extern "C"
