// Products with 4-bit weights for tens of rows: weights are streamed once, x is shared through LDS.
//
// With the kernel for few rows every wave reads all of x for its rows of weights, from the L2: at 24 rows that is more
// bytes than the weights are (24 x 28672 x 8192: 49 us, as long as the L2 needs for them).  Here 16 waves are 4 times 32 rows of weights
// by 4 parts of K: the four waves of a part read one copy of x, which comes into LDS by itself, in a ring.  Arithmetic as
// in the kernel for many rows.
#include "buffer_ops.h"
#include "lds_ring.h"
#include "w4.h"

namespace qnn {

// A workgroup: 128 rows of weights, 32 * MT rows of x; part `part` of K takes 128s part, part + 4, ...: a turn is one of them.
// Requests are made two turns ahead, the same number in each turn (past the end the last one again), so that waiting for all
// but the youngest turn's is waiting for the copies of the one that begins.  GS: groups in 128 weights (1: of whole 128s, 2: of 64s,
// 4: any multiple of 32).
template <class T, int MT, int GS, bool ZEROS> __global__ void __launch_bounds__(1024, 4) w4_parts_kernel(const W4Args a, const W4Prepared p)
{
    constexpr int PARTS = 4, ROWS = 32 * MT, RING = 3;
    constexpr int X_BYTES = RING * PARTS * ROWS * 256, SUM_BYTES = PARTS * ROWS * (128 + 4) * 4;
    constexpr int REQUESTS = 2 * MT + 2 + GS * (ZEROS ? 2 : 1);
    __shared__ __attribute__((aligned(16))) uint8_t s_mem[X_BYTES > SUM_BYTES ? X_BYTES : SUM_BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, hh = lane >> 5;
    const int part = wave >> 2, nw = wave & 3;
    const int n0 = blockIdx.x * 128 + nw * 32, m0 = blockIdx.y * ROWS;
    const int row_bytes = a.K / 2, full = a.K / 128 / PARTS; // turns in which every part has a whole 128

    const uint32_t n_at = min(n0 + c, a.N - 1);
    const uint8_t *const w_row = a.codes + (int64_t)n_at * row_bytes;
    const uint8_t *const x_tile = reinterpret_cast<const uint8_t *>(p.x + (int64_t)m0 * p.pitch);
    const int x_bytes = min(a.M - m0, ROWS) * p.pitch * 2; // rows beyond the last read as zeros
    uint32_t x_from[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) {
        const int row = (nw * 2 * MT + i) * 4 + (lane >> 4);
        x_from[i] = (uint32_t)row * p.pitch * 2 + ((lane & 15) ^ (row & 15)) * 16;
    }
    auto copy_x = [&](int turn, int slot) {
        const int at = (turn * PARTS + part) * 256;
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i)
            buffer_to_lds16(x_tile, x_bytes, x_from[i] + at, s_mem + (slot * PARTS + part) * (ROWS * 256) + (nw * 2 * MT + i) * 1024);
    };
    struct Weights {
        w32x4 w[2];
        uint16_t s[GS];
        int8_t z[GS];
    };
    auto load_scales = [&](Weights &f, int step) {
#pragma unroll
        for (int q = 0; q < GS; ++q) {
            const uint32_t at = (uint32_t)group_of(a, min(step * 128 + q * (128 / GS), a.K - 1)) * a.N + n_at;
            f.s[q] = a.scales[at];
            f.z[q] = ZEROS ? a.zeros[at] : 0;
        }
    };
    auto load = [&](Weights &f, int turn) {
        const int step = turn * PARTS + part;
#pragma unroll
        for (int i = 0; i < 2; ++i) f.w[i] = load_any<w32x4>(w_row + step * 64 + 32 * hh + 16 * i);
        load_scales(f, step);
    };

    f32x16 acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[mt][i] = 0.0f;
    float unit = 0.0f;
    const uint32_t bits = kept(Nibbles<F16>::kBits);
    auto compute = [&](const Weights &f, int slot) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = f.w[i >> 2][i & 3];
        swap_halves<GS>(w);
        const uint8_t *const row = s_mem + (slot * PARTS + part) * (ROWS * 256) + c * 256;
        GroupUnit g;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i % (8 / GS) == 0) {
                g = enter_group(T::widen(f.s[i / (8 / GS)]), f.z[i / (8 / GS)], unit);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[mt] *= g.ratio;
            }
            const h16x8 wide = whole_weights(w[i], g, bits);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const h16x8 xf = *reinterpret_cast<const h16x8 *>(row + mt * (32 * 256) + (piece_of<GS>(i, hh) ^ (c & 15)) * 16);
                acc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xf, wide, acc[mt], 0, 0, 0);
            }
        }
    };

    Weights f[3];
    if (full > 0) {
        copy_x(0, 0);
        load(f[0], 0);
        copy_x(min(1, full - 1), 1);
        load(f[1], min(1, full - 1));
        for (int turn = 0; turn < full; turn += 3) {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (turn + k < full) {
                    wait_vmcnt<REQUESTS>();
                    lds_barrier(); // this turn's x is there, and all waves have left the slot that is filled next
                    copy_x(min(turn + k + 2, full - 1), (k + 2) % 3);
                    load(f[(k + 2) % 3], min(turn + k + 2, full - 1));
                    compute(f[k], k);
                }
        }
    }
    // what is left: less than a turn of all parts, the last 128 perhaps cut off
    if (full * PARTS * 128 < a.K) {
        wait_vmcnt<0>();
        lds_barrier();
        const int step = full * PARTS + part;
        if (step * 128 < a.K) {
            copy_x(full, 0);
#pragma unroll
            for (int i = 0; i < 2; ++i) f[0].w[i] = load_end(w_row, row_bytes, step * 64 + 32 * hh + 16 * i);
            load_scales(f[0], step);
        }
        wait_vmcnt<0>();
        lds_barrier();
        if (step * 128 < a.K) compute(f[0], 0);
    }

    // the parts' sums, added in their order
    wait_vmcnt<0>(); // (no copy may land on them)
    lds_barrier();
    float *const s_sum = reinterpret_cast<float *>(s_mem);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) s_sum[(part * ROWS + mt * 32 + 8 * (i >> 2) + 4 * hh + (i & 3)) * (128 + 4) + nw * 32 + c] = acc[mt][i] * unit;
    lds_barrier();
    for (int i = tid; i < ROWS * 128; i += 1024) {
        const int m = i / 128, n = blockIdx.x * 128 + i % 128;
        if (m0 + m >= a.M || n >= a.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) v += s_sum[(q * ROWS + m) * (128 + 4) + i % 128];
        v = ldexpf(v, p.row_exp[m0 + m]) + (a.bias ? T::widen(a.bias[n]) : 0.0f);
        a.y[(int64_t)(m0 + m) * a.ldy + n] = T::narrow(v);
    }
}

template <class T, int MT, int GS> static void launch_parts(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 127) / 128), (unsigned)((a.M + 32 * MT - 1) / (32 * MT)));
    if (a.zeros) hipLaunchKernelGGL((w4_parts_kernel<T, MT, GS, true>), grid, dim3(1024), 0, s, a, p);
    else hipLaunchKernelGGL((w4_parts_kernel<T, MT, GS, false>), grid, dim3(1024), 0, s, a, p);
}
template <class T> static void launch_groups(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    if (a.group % 128 == 0) launch_parts<T, 1, 1>(a, p, s);
    else if (a.group % 64 == 0) launch_parts<T, 1, 2>(a, p, s);
    else launch_parts<T, 1, 4>(a, p, s);
}
void launch_w4_parts(const W4Args &a, int type, const W4Prepared &p, hipStream_t s)
{
    if (type == QNN_BF16) launch_groups<Bf16>(a, p, s);
    else launch_groups<F16>(a, p, s);
}

} // namespace qnn
