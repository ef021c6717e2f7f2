// Products of e4m3 rows and weights with block scales, tens of rows and more: tiles of both operands through LDS.
#pragma once

#include "buffer_ops.h"
#include "f8.h"
#include "lds_ring.h"

namespace qnn {

// 32 x 32 outputs over 64 (NARROW) or 16 of K; operands and result as in f8_products, with rows of 32
__device__ __forceinline__ f32x16 f8_products32(const i32x8 a, const i32x8 b, const f32x16 c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

struct F8TileArgs {
    F8Args a;          // x, w: rows of whole 16-byte pieces
    float *parts;      // sums of parts of K: [splits][M][N], or null
    int32_t m_tiles, n_tiles, splits, band;
    uint32_t per_xcd;  // workgroups
};

// Workgroups are dealt to the 8 XCDs in turn.  Each XCD has a stretch of the tiles of its own, in bands of `band` tiles of rows, so that the tiles that
// it works on at a time share rows and weights in its L2.
__device__ __forceinline__ bool f8_tile_of(const F8TileArgs &t, int &tm, int &tn, int &part)
{
    const uint32_t id = blockIdx.x % 8 * t.per_xcd + blockIdx.x / 8, tiles = (uint32_t)t.m_tiles * t.n_tiles;
    part = (int)(id / tiles);
    if (part >= t.splits) return false;
    const uint32_t at = id % tiles, whole = (uint32_t)t.band * t.n_tiles, group = at / whole, rest = at % whole;
    const uint32_t high = min((uint32_t)t.band, t.m_tiles - group * t.band);
    tm = (int)(group * t.band + rest % high), tn = (int)(rest / high);
    return true;
}

// BM rows of x by BN rows of weights; WM x WN waves, each with BM / WM by BN / WN of them, in products of 32 x 32 formed transposed (weights are the
// left operand), so that a lane's outputs are of one row of x and its scale is one register.  K in steps of 128 through LDS,
// copied there directly, 16-byte pieces of a row exchanged by half its number, so that reads of 16 rows meet the 16 places of the 64 banks.
// Copies take longer than a step: those of weights are requested WB - 1 steps ahead, into WB buffers, those of x, which the waves read into
// registers as a step begins, nearly XB, into XB buffers behind a second barrier, and scales SETS (waits are in the order of requests: one step ahead
// they are also waits for copies that are needed later; but tiles of 256 x 256 have no registers for two sets).
// 8192 x 8192 x 8192 485 to 500 us (2250 TFLOP/s; the same with one scale for each operand, by a library, 424): matrix units 58 % of the cycles, vector
// unit 49 %, at 1.8 GHz, which is what power leaves of 2.4.  Tiles of 128 x 128 take 0.62 us for a step of 128 against 1.85 for four times as
// much; with binary32 results, whose codes are widened to bfloat16 first, 0.97.  Deeper rings, tiles of 64 x 128 and of 64 x 256 were no faster.
template <int BM, int BN, int WM, int WN, int XB, int WB, int SETS, bool NARROW, int PER_SIMD> __global__ void __launch_bounds__(64 * WM * WN, PER_SIMD) f8_tile_kernel(const F8TileArgs t)
{
    constexpr int WAVES = WM * WN, TJ = BM / WM / 32, TI = BN / WN / 32, X_BYTES = BM * 128, W_BYTES = BN * 128, X_COPIES = BM / 8 / WAVES,
                  W_COPIES = BN / 8 / WAVES, RING = XB * X_BYTES + WB * W_BYTES;
    static_assert(BN / WN <= 128 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "a wave's weights lie in one block; whole copies");
    __shared__ __attribute__((aligned(16))) uint8_t s_ring[RING];
    uint8_t *const s_w = s_ring + XB * X_BYTES;
    const F8Args &a = t.a;
    int tm, tn, part;
    if (!f8_tile_of(t, tm, tn, part)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, g = lane >> 5;
    const int wm = wave % WM, wn = wave / WM, m0 = tm * BM, n0 = tn * BN;
    const int blocks = (a.K + kF8Block - 1) / kF8Block;
    const int first = blocks * part / t.splits, last = blocks * (part + 1) / t.splits; // (up to 2^13 blocks by 16)

    const uint8_t *const x_tile = a.x + m0 * a.ldx, *const w_tile = a.w + (int64_t)n0 * a.K;
    const int x_bytes = (int)(min(a.M - m0, BM) * a.ldx), w_bytes = (int)(min(a.N - n0, BN) * a.K); // rows beyond the last read as zeros
    // Where a lane's 16 bytes of a block are in the rows that a copy of 8 begins with an even or odd multiple of 8; past the end of this part of K: beyond
    // the descriptors' sizes (which are below 2^31), where reads give zeros.
    const int k_end = min(a.K, last * kF8Block);
    // (Worked out from the lane's number each time where registers are short.)
    const auto offsets = [&](int b, int row, uint32_t pitch, uint32_t (&at)[2]) {
        int l = lane;
        if constexpr (SETS == 1) asm volatile("" : "+v"(l));
        const uint32_t begin = (uint32_t)(row + (l >> 3)) * pitch;
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const uint32_t k = (uint32_t)(b * kF8Block + ((l & 7) ^ (l >> 4) ^ 4 * odd) * 16);
            at[odd] = begin + ((int)k < k_end ? k : 0x80000000u);
        }
    };
    const auto copy_x = [&](int b, int buffer) {
        uint32_t at[2];
        offsets(b, wave * X_COPIES * 8, (uint32_t)a.ldx, at);
#pragma unroll
        for (int i = 0; i < X_COPIES; ++i)
            buffer_to_lds16(x_tile, x_bytes, at[(wave * X_COPIES + i) & 1] + (uint32_t)(i * 8) * (uint32_t)a.ldx, s_ring + buffer * X_BYTES + (wave * X_COPIES + i) * 1024);
    };
    const auto copy_w = [&](int b, int buffer) {
        uint32_t at[2];
        offsets(b, wave * W_COPIES * 8, (uint32_t)a.K, at);
#pragma unroll
        for (int i = 0; i < W_COPIES; ++i)
            buffer_to_lds16(w_tile, w_bytes, at[(wave * W_COPIES + i) & 1] + (uint32_t)(i * 8) * (uint32_t)a.K, s_w + buffer * W_BYTES + (wave * W_COPIES + i) * 1024);
    };
    const uint32_t x_at = 4u * (uint32_t)(wm * (BM / WM) + c); // (rows beyond the last: scales of 0)
    const float *const w_scale = a.ws + (int64_t)min((n0 + wn * (BN / WN)) / kF8Block, (a.N - 1) / kF8Block) * blocks;
    struct Scales {
        float x[TJ], w;
    };
    const auto load_scales = [&](Scales &s, int b) {
#pragma unroll
        for (int j = 0; j < TJ; ++j) s.x[j] = buffer_load_float(a.xs + b * a.ldxs + m0 + 32 * j, 4 * max(min(a.M - m0, BM) - 32 * j, 0), x_at);
        s.w = buffer_load_float(w_scale + b, 4, 0u); // (a vector load: the waits count it)
    };

    f32x16 acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    const auto fragment = [&](const uint8_t *rows, int h) { // 32 bytes of row c of 32
        const w32x4 p = *reinterpret_cast<const w32x4 *>(rows + c * 128 + ((4 * h + 2 * g) ^ (c >> 1 & 7)) * 16);
        const w32x4 q = *reinterpret_cast<const w32x4 *>(rows + c * 128 + ((4 * h + 2 * g + 1) ^ (c >> 1 & 7)) * 16);
        return i32x8{(int)p[0], (int)p[1], (int)p[2], (int)p[3], (int)q[0], (int)q[1], (int)q[2], (int)q[3]};
    };
    // The tiles of a step one after the other, the multiply-adds of a tile beside the products of the next one, and the pieces of the weights that the
    // tiles after that need read meanwhile; the last tile's are left for the next step.
    f32x16 p[2];
    float late = 0.0f; // the scale of the tile that is left
#pragma unroll
    for (int e = 0; e < 16; ++e) p[0][e] = p[1][e] = 0.0f;
    const auto join = [&](int tile, float by) {
        const int i = tile / TJ, j = tile % TJ;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = fmaf(p[tile & 1][e], by, acc[i][j][e]);
    };
    constexpr int TILES = TI * TJ;
    static_assert(TILES % 2 == 0 && TI % 2 == 0 && TJ >= 2, "sums and weights in two sets in turn");
    i32x8 x[TJ][2], w[2][2];
    const auto x_rows = [&](int buffer) { return s_ring + buffer * X_BYTES + wm * (BM / WM) * 128; };
    const auto w_rows = [&](int buffer) { return s_w + buffer * W_BYTES + wn * (BN / WN) * 128; };
    constexpr int STEP = TJ + 1 + X_COPIES + W_COPIES; // requests of a step: behind its first tiles scales and x, before its last tile weights
    // What is requested after the next step's x, and after its weights, when they are waited for:
    constexpr int ALLOWED = (XB - 1) * STEP < (WB - 1) * STEP - W_COPIES ? (XB - 1) * STEP : (WB - 1) * STEP - W_COPIES;
    static_assert(XB >= 2 && XB <= SETS + 1 && WB > XB, "the requests before the first step are those of a step from its second last on");
    Scales scales[SETS];
    const auto follow = [](int buffer, int many) { return buffer + 1 == many ? 0 : buffer + 1; };
#pragma unroll
    for (int v = -WB; v < 0; ++v) { // as the steps before the first would
        if (v >= -SETS) load_scales(scales[v & (SETS - 1)], min(first + v + SETS, last - 1));
        if (v >= -XB) copy_x(first + v + XB, v + XB);
        if (v == -1) {
            wait_vmcnt<ALLOWED>();
            lds_barrier();
        }
        copy_w(first + v + WB, v + WB);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) w[0][h] = fragment(w_rows(0), h), x[0][h] = fragment(x_rows(0), h);
    int w_buffer = 0, x_buffer = 0;
    const auto step = [&](int b, auto odd) {
        Scales &now = scales[decltype(odd)::value];
        const int w_next = follow(w_buffer, WB), x_next = follow(x_buffer, XB);
        float scale[TJ];
#pragma unroll
        for (int at = 0; at < TILES; ++at) {
            const int i = at / TJ, j = at % TJ;
            if (at == TILES - 1) {
                // The next step's copies have arrived (those requested after them may be on their way), and all waves have this step's weights in
                // registers.
                wait_vmcnt<ALLOWED>();
                lds_barrier();
                copy_w(b + WB, w_buffer);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (i == 0 && j + 1 < TJ) x[j + 1][h] = fragment(x_rows(x_buffer) + (j + 1) * 32 * 128, h);
                if (j == TJ - 1 && i + 1 < TI) w[(i + 1) & 1][h] = fragment(w_rows(w_buffer) + (i + 1) * 32 * 128, h);
                if (at == TILES - 1) w[0][h] = fragment(w_rows(w_next), h), x[0][h] = fragment(x_rows(x_next), h);
                if (h == 0)
#pragma unroll
                    for (int e = 0; e < 16; ++e) p[at & 1][e] = 0.0f;
                if constexpr (NARROW) {
                    p[at & 1] = f8_products32(w[i & 1][h], x[j][h], p[at & 1]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        p[at & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen_codes((uint32_t)w[i & 1][h][2 * q], (uint32_t)w[i & 1][h][2 * q + 1]),
                                                                            widen_codes((uint32_t)x[j][h][2 * q], (uint32_t)x[j][h][2 * q + 1]), p[at & 1], 0, 0, 0);
                }
                if (h == 1) { // (half a tile later than they might be: a wait for the products that they read would hold up all that follows)
                    if (at == 1)
#pragma unroll
                        for (int u = 0; u < TJ; ++u) scale[u] = now.x[u] * now.w;
                    join((at + TILES - 1) % TILES, at == 0 ? late : scale[(at - 1) % TJ]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (at == TJ - 1) {
                lds_barrier(); // all waves have this step's x in registers
                load_scales(now, min(b + SETS, last - 1));
                copy_x(b + XB, x_buffer);
            }
        }
        late = scale[TJ - 1], w_buffer = w_next, x_buffer = x_next;
    };
    for (int b = first; b < last; b += SETS) {
        step(b, std::integral_constant<int, 0>());
        if constexpr (SETS == 2)
            if (b + 1 < last) step(b + 1, std::integral_constant<int, 1>());
    }
    join(TILES - 1, late);

    // Outputs in binary32 through LDS, 32 rows of x by the wave's weights at a time, 16-byte pieces exchanged by the row's number
    constexpr int WIDE = BN / WN;
    static_assert(WAVES * 32 * WIDE * 4 <= RING, "outputs fit the ring");
    wait_vmcnt<0>();
    lds_barrier();
    float *const tile = reinterpret_cast<float *>(s_ring) + wave * 32 * WIDE;
    constexpr int EACH = 8, LANES = WIDE / EACH, ROWS = 64 / LANES; // outputs of a lane, lanes of a row, rows at a time
    const int n = n0 + wn * WIDE + lane % LANES * EACH;
    float bias[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) bias[e] = a.bias && !t.parts && n + e < a.N ? load_out(a.bias, n + e, a.type) : 0.0f;
#pragma unroll
    for (int j = 0; j < TJ; ++j) {
#pragma unroll
        for (int i = 0; i < TI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = (i * 8 + q * 2 + g) ^ (c & 15);
                *reinterpret_cast<f32x4 *>(tile + c * WIDE + at * 4) = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            }
        lds_barrier(); // (between waves nothing is exchanged; the compiler keeps the order of writes and reads)
#pragma unroll
        for (int r = 0; r < 32 / ROWS; ++r) {
            const int row = r * ROWS + lane / LANES, m = m0 + wm * (BM / WM) + j * 32 + row;
            float v[EACH];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const f32x4 u = *reinterpret_cast<const f32x4 *>(tile + row * WIDE + ((lane % LANES * 2 + p) ^ (row & 15)) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * p + e] = u[e] + bias[4 * p + e];
            }
            if (m >= a.M || n >= a.N) continue;
            if (t.parts) {
                float *const to = t.parts + ((int64_t)part * a.M + m) * a.N + n;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if (n + 4 * p + 4 <= a.N) store_any(to + 4 * p, f32x4{v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]});
                    else
                        for (int e = 0; e < 4; ++e)
                            if (n + 4 * p + e < a.N) to[4 * p + e] = v[4 * p + e];
                }
            } else if (n + EACH <= a.N) {
                if (a.type == QNN_F32) {
                    float *const to = static_cast<float *>(a.y) + m * a.ldy + n;
                    store_any(to, f32x4{v[0], v[1], v[2], v[3]}), store_any(to + 4, f32x4{v[4], v[5], v[6], v[7]});
                } else {
                    const w32x4 h = a.type == QNN_BF16 ? w32x4{narrow2<Bf16>(v[0], v[1]), narrow2<Bf16>(v[2], v[3]), narrow2<Bf16>(v[4], v[5]), narrow2<Bf16>(v[6], v[7])}
                                                       : w32x4{narrow2<F16>(v[0], v[1]), narrow2<F16>(v[2], v[3]), narrow2<F16>(v[4], v[5]), narrow2<F16>(v[6], v[7])};
                    store_any(static_cast<uint16_t *>(a.y) + m * a.ldy + n, h);
                }
            } else {
#pragma unroll
                for (int e = 0; e < EACH; ++e)
                    if (n + e < a.N) store_out(a.y, m * a.ldy + n + e, a.type, v[e]);
            }
        }
        lds_barrier();
    }
}

} // namespace qnn
