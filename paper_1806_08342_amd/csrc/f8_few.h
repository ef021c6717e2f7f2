// Products of e4m3 rows and weights with block scales, few rows: both operands straight into registers.
#pragma once

#include "f8.h"

namespace qnn {

// 16 bytes of a row, zeros behind its end
__device__ __forceinline__ w32x4 f8_load16(const uint8_t *row, int K, int k) { return k + 16 <= K ? load_any<w32x4>(row + k) : load_end(row, K, k); }

// the same of a row of whole pieces, without a branch
__device__ __forceinline__ w32x4 f8_load_piece(const uint8_t *row, int K, int k)
{
    const uint32_t there = k < K ? ~0u : 0u;
    return load_any<w32x4>(row + min(k, K - 16)) & w32x4{there, there, there, there};
}

// One wave takes 16 * NT rows of the weights and 16 * MT rows of x, the waves of a workgroup share K in turns of 128 and join their
// sums in LDS in their order.  The product is formed transposed (weights are the left operand): a lane has one row of x and four consecutive
// outputs.  The operands of the next DEPTH - 1 blocks are on their way while a wave works on one.
// Bound by reading the weights where x is short (24 x 28672 x 8192 51.6 us, 4.6 TB/s), and by x from the L2 for every 16 NT rows of them where it is not.
// 1 x 4096 x 4096: 4.7 us call behind call, a launch and a chain of loads.
// ANY: rows that begin within a word.  A lane has 32 bytes in a row then, loads the nine words that they lie in and moves them down: loads at any byte
// took longer (1 x 4096 x 4095 10.1 us, so 6.6; 16 rows 15 and 9, 64 rows 30 and 20).
template <int MT, int NT, int WAVES, int DEPTH, bool NARROW, bool ANY> __global__ void __launch_bounds__(64 * WAVES, 2) f8_rows_kernel(const F8Args a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int whole = a.K / kF8Block, blocks = (a.K + kF8Block - 1) / kF8Block;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *w_row[NT], *x_row[MT];
    const float *x_scale[MT], *const w_scale = a.ws + (int64_t)(n0 / kF8Block) * blocks;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w_row[nt] = a.w + (int64_t)min(n0 + nt * 16 + c, a.N - 1) * a.K;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int m = min(m0 + mt * 16 + c, a.M - 1); // (rows beyond the ends are the last one again, and dropped)
        x_row[mt] = a.x + m * a.ldx, x_scale[mt] = a.xs + m;
    }
    struct Step {
        w32x4 w[NT][2], x[MT][2];
        uint32_t w_more[ANY ? NT : 1], x_more[ANY ? MT : 1];
        float xs[MT], ws;
    };
    // (the ninth word is the eighth again where a row begins with a word: nothing behind the row's end is loaded)
    const auto within = [](const uint8_t *row) { return (uint32_t)(uintptr_t)row & 3; };
    const auto load_words = [&](const uint8_t *row, int k, w32x4 (&v)[2], uint32_t &more) {
        const uint8_t *const words = row - within(row) + k;
        v[0] = load_any<w32x4>(words), v[1] = load_any<w32x4>(words + 16), more = load_any<uint32_t>(words + (within(row) ? 32 : 28));
    };
    const auto move_down = [](const w32x4 (&v)[2], uint32_t more, uint32_t by, w32x4 (&to)[2]) {
        const uint32_t u[9] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3], more};
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i >> 2][i & 3] = __builtin_amdgcn_alignbyte(u[i + 1], u[i], by);
    };
    // (with 64 x 64 rows in binary32 the vector instructions are what bounds it: 1021 x 1001 x 1027 15.3 us with the exchange, 13.9 without)
    constexpr uint32_t HALF = !ANY && (NARROW || MT * NT < 16) ? 64 : 0, SECOND = ANY ? 16 : 64;
    constexpr int PIECE = ANY ? 32 : 16; // a lane's bytes in a row
    uint32_t w_first[NT], x_first[MT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w_first[nt] = HALF * half_first((uint32_t)(uintptr_t)w_row[nt], c);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x_first[mt] = HALF * half_first((uint32_t)(uintptr_t)x_row[mt], c);
    const auto load = [&](Step &s, int b) {
        const int k = b * kF8Block + PIECE * g;
        if constexpr (ANY) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) load_words(w_row[nt], k, s.w[nt], s.w_more[nt]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) load_words(x_row[mt], k, s.x[mt], s.x_more[mt]), s.xs[mt] = x_scale[mt][b * a.ldxs];
            s.ws = w_scale[b];
            return;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s.w[nt][0] = load_any<w32x4>(w_row[nt] + (k + w_first[nt])), s.w[nt][1] = load_any<w32x4>(w_row[nt] + (k + (w_first[nt] ^ 64)));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            s.x[mt][0] = load_any<w32x4>(x_row[mt] + (k + x_first[mt])), s.x[mt][1] = load_any<w32x4>(x_row[mt] + (k + (x_first[mt] ^ 64)));
            s.xs[mt] = x_scale[mt][b * a.ldxs];
        }
        s.ws = w_scale[b];
    };
    const auto compute = [&](const Step &t, bool moved) {
        Step s;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) ANY ? move_down(t.w[nt], t.w_more[ANY ? nt : 0], moved ? 0u : within(w_row[nt]), s.w[nt]) : in_order(t.w[nt], w_first[nt], s.w[nt]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            ANY ? move_down(t.x[mt], t.x_more[ANY ? mt : 0], moved ? 0u : within(x_row[mt]), s.x[mt]) : in_order(t.x[mt], x_first[mt], s.x[mt]);
            s.xs[mt] = t.xs[mt];
        }
        s.ws = t.ws;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                fma4(acc[mt][nt], f8_products<NARROW>(s.w[nt], s.x[mt]), s.xs[mt] * s.ws);
                asm volatile("" : "+v"(acc[mt][nt])); // (here, and not behind a branch, which the compiler's waits for the products do not reach over)
            }
    };
    const int mine = wave < whole ? (whole - wave + WAVES - 1) / WAVES : 0;
    // Each workgroup begins at another place of K: rows lie a power of two apart more often than not, and workgroups that
    // read the same columns of all rows at one time would keep to a part of the memory's channels.
    const int turned = mine > 0 ? (int)(blockIdx.x % (unsigned)mine) : 0;
    const auto block_at = [&](int i) { // (behind the last: that again, unused)
        const int at = min(i, mine - 1) + turned;
        return wave + WAVES * (at < mine ? at : at - mine);
    };
    Step f[DEPTH];
    if (mine > 0) {
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d) load(f[d], block_at(d));
    }
    if (whole < blocks && wave == whole % WAVES) { // the last, shorter block
        Step &s = f[DEPTH - 1];
        const int k = whole * kF8Block + PIECE * g;
        const auto load_last = [&](auto load) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s.w[nt][0] = load(w_row[nt], a.K, k + (int)w_first[nt]), s.w[nt][1] = load(w_row[nt], a.K, k + (int)(w_first[nt] ^ SECOND));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s.x[mt][0] = load(x_row[mt], a.K, k + (int)x_first[mt]), s.x[mt][1] = load(x_row[mt], a.K, k + (int)(x_first[mt] ^ SECOND));
        };
        // (one load waits for the other where branches lie between: 1021 x 1001 x 1027, whose copies have whole pieces, 14.1 us with f8_load16, 13.5 so)
        if (a.K % 16 == 0) load_last([](const uint8_t *row, int K, int at) { return f8_load_piece(row, K, at); });
        else load_last([](const uint8_t *row, int K, int at) { return f8_load16(row, K, at); });
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) s.xs[mt] = x_scale[mt][whole * a.ldxs];
        s.ws = w_scale[whole];
        if constexpr (ANY) { // (loaded to its place; of the ninth words nothing is used)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s.w_more[nt] = 0;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) s.x_more[mt] = 0;
        }
        compute(s, true);
    }
    int i = 0;
    for (; i + DEPTH <= mine; i += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            load(f[(d + DEPTH - 1) % DEPTH], block_at(i + d + DEPTH - 1));
            compute(f[d], false);
        }
    }
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (i + d < mine) compute(f[d], false);

    __shared__ float s_acc[WAVES][16 * MT][16 * NT + 4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4 *>(&s_acc[wave][mt * 16 + c][nt * 16 + g * 4]) = acc[mt][nt];
    __syncthreads();
    for (int j = threadIdx.x; j < 16 * MT * 16 * NT; j += 64 * WAVES) {
        const int m = j / (16 * NT), n = j % (16 * NT);
        if (m0 + m >= a.M || n0 + n >= a.N) continue;
        float v = s_acc[0][m][n];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_acc[w][m][n];
        if (a.bias) v += load_out(a.bias, n0 + n, a.type);
        store_out(a.y, (m0 + m) * a.ldy + n0 + n, a.type, v);
    }
}

} // namespace qnn
