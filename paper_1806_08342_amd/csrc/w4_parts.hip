// Products with 4-bit weights for tens of rows: weights are streamed once, x is shared through LDS.
//
// With the kernel for few rows every wave reads all of x for its rows of weights, from the L2: at 24 rows that is more
// bytes than the weights are (24 x 28672 x 8192: 49 us, as long as the L2 needs for them).  Here the waves of a workgroup are NW times 32 rows of weights
// by PARTS parts of K: the waves of a part read one copy of x, which comes into LDS by itself, in a ring.  Arithmetic as
// in the kernel for many rows.  24 x 28672 x 8192: 33 us, 3.7 TB/s of codes (224 workgroups leave 32 CUs without one, and each reads x, two
// thirds of the bytes of its codes, from the L2), and 5 us before it for the launch that writes x as binary16.
#include "buffer_ops.h"
#include "lds_ring.h"
#include "w4.h"

namespace qnn {

// A workgroup: 32 * NW rows of weights, 32 * MT rows of x; part `part` of K takes 128s part, part + PARTS, ...: a turn is one of them.
// Requests are made RING - 1 turns ahead, copies first, at least REQUESTS in each turn (past the end the last one again), so that
// waiting for all but so many for each younger turn is waiting for the copies of the one that begins.  GS: groups in 128 weights (1: of whole 128s, 2: of 64s,
// 4: any multiple of 32).
template <class T, int MT, int NW, int PARTS, int RING, int GS, bool ZEROS> __global__ void __launch_bounds__(64 * NW * PARTS, NW * PARTS == 16 ? 4 : 2) w4_parts_kernel(const W4Args a, const W4Prepared p)
{
    constexpr int ROWS = 32 * MT, BN = 32 * NW, COPIES = 8 * MT / NW; // copies of 1 KB per wave and turn
    constexpr int X_BYTES = RING * PARTS * ROWS * 256, SUM_BYTES = PARTS * ROWS * (BN + 4) * 4;
    constexpr int REQUESTS = COPIES + 2, AHEAD = RING - 1; // a turn's copies and codes (scales, or codes that the compiler moves, make it more: the wait is longer then, not shorter)
    __shared__ __attribute__((aligned(16))) uint8_t s_mem[X_BYTES > SUM_BYTES ? X_BYTES : SUM_BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 31, hh = lane >> 5;
    const int part = wave / NW, nw = wave % NW;
    const int n0 = blockIdx.x * BN + nw * 32, m0 = blockIdx.y * ROWS;
    const int row_bytes = a.K / 2, full = a.K / 128 / PARTS; // turns in which every part has a whole 128

    const uint32_t n_at = min(n0 + c, a.N - 1);
    const uint8_t *const w_row = a.codes + (int64_t)n_at * row_bytes;
    const uint8_t *const x_tile = reinterpret_cast<const uint8_t *>(p.x + (int64_t)m0 * p.pitch);
    const int x_bytes = min(a.M - m0, ROWS) * p.pitch * 2; // rows beyond the last read as zeros
    uint32_t x_from[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int row = (nw * COPIES + i) * 4 + (lane >> 4);
        x_from[i] = (uint32_t)row * p.pitch * 2 + ((lane & 15) ^ (row & 15)) * 16;
    }
    auto copy_x = [&](int turn, int slot) {
        const int at = (turn * PARTS + part) * 256;
#pragma unroll
        for (int i = 0; i < COPIES; ++i)
            buffer_to_lds16(x_tile, x_bytes, x_from[i] + at, s_mem + (slot * PARTS + part) * (ROWS * 256) + (nw * COPIES + i) * 1024);
    };
    struct Weights {
        Codes<8> w;
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
        f.w.load(w_row + step * 64 + 32 * hh, a.skewed);
        load_scales(f, step);
    };

    f32x16 acc[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[mt][i] = 0.0f;
    ScaleUnit unit;
    const uint32_t bits = kept(Nibbles<F16>::kBits);
    auto compute = [&](Weights &f, int slot) {
        f.w.place(w_row, a.skewed);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = f.w.w[i];
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

    Weights f[RING];
    if (full > 0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            copy_x(min(k, full - 1), k);
            load(f[k], min(k, full - 1));
        }
        for (int turn = 0; turn < full; turn += RING) {
#pragma unroll
            for (int k = 0; k < RING; ++k)
                if (turn + k < full) {
                    wait_vmcnt<REQUESTS *(AHEAD - 1)>();
                    lds_barrier(); // this turn's x is there, and all waves have left the slot that is filled next
                    copy_x(min(turn + k + AHEAD, full - 1), (k + AHEAD) % RING);
                    load(f[(k + AHEAD) % RING], min(turn + k + AHEAD, full - 1));
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
            f[0].w.load_tail(w_row, row_bytes, step * 64 + 32 * hh, a.skewed);
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
    const Result result(unit);
    using i32x4 = int32_t __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int m = mt * 32 + 2 * i + 4 * hh;
            const i32x4 exp = *reinterpret_cast<const i32x4 *>(p.row_exp + m0 + m); // (of whole tiles)
#pragma unroll
            for (int e = 0; e < 4; ++e) s_sum[(part * ROWS + m + e) * (BN + 4) + nw * 32 + c] = result.of(acc[mt][i + e], exp[e]);
        }
    lds_barrier();
    for (int i = tid; i < ROWS * BN; i += 64 * NW * PARTS) {
        const int m = i / BN, n = blockIdx.x * BN + i % BN;
        if (m0 + m >= a.M || n >= a.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) v += s_sum[(q * ROWS + m) * (BN + 4) + i % BN];
        if (a.bias) v += T::widen(a.bias[n]);
        a.y[(int64_t)(m0 + m) * a.ldy + n] = T::narrow(v);
    }
}

template <class T, int MT, int NW, int PARTS, int RING, int GS> static void launch_parts(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 32 * NW - 1) / (32 * NW)), (unsigned)((a.M + 32 * MT - 1) / (32 * MT)));
    if (a.zeros) hipLaunchKernelGGL((w4_parts_kernel<T, MT, NW, PARTS, RING, GS, true>), grid, dim3(64 * NW * PARTS), 0, s, a, p);
    else hipLaunchKernelGGL((w4_parts_kernel<T, MT, NW, PARTS, RING, GS, false>), grid, dim3(64 * NW * PARTS), 0, s, a, p);
}
template <class T, int MT, int NW, int PARTS, int RING> static void launch_groups(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    if (a.group % 128 == 0) launch_parts<T, MT, NW, PARTS, RING, 1>(a, p, s);
    else if (a.group % 64 == 0) launch_parts<T, MT, NW, PARTS, RING, 2>(a, p, s);
    else launch_parts<T, MT, NW, PARTS, RING, 4>(a, p, s);
}
// The forms: rows of x / 32, waves along the weights, parts of K, ring; and what a turn takes (us, at K = 4096 and 8192, with
// enough workgroups to load the memory).  A workgroup fills a CU, so that the time is that of ceil(workgroups / 256) rounds of
// K / 128 / parts turns, and 5 us of launches, first requests and the sums at the end: within 15 % of what was measured for 17 to 400
// rows with 4096 x 4096, 12288 x 4096 and 28672 x 8192 weights.
struct PartsForm {
    int mt, nw, parts;
    float turn_us;
    const char *name; // rows of x, x rows of weights, / parts of K
};
constexpr PartsForm kForms[] = {{1, 4, 4, 2.0f, "tens32x128/4"}, {1, 2, 4, 1.2f, "tens32x64/4"},   {1, 1, 8, 1.55f, "tens32x32/8"},
                                {2, 4, 4, 2.4f, "tens64x128/4"}, {2, 4, 2, 1.3f, "tens64x128/2"}, {2, 2, 4, 1.75f, "tens64x64/4"}};

static float form_us(const PartsForm &f, int64_t M, int64_t N, int64_t K)
{
    const int64_t groups = ((N + 32 * f.nw - 1) / (32 * f.nw)) * ((M + 32 * f.mt - 1) / (32 * f.mt));
    return (float)((groups + 255) / 256) * (float)((K + 128 * f.parts - 1) / (128 * f.parts)) * f.turn_us + 5.0f;
}
static int best_form(int64_t M, int64_t N, int64_t K)
{
    int best = 0;
    for (int i = 1; i < 6; ++i)
        if (form_us(kForms[i], M, N, K) < form_us(kForms[best], M, N, K)) best = i;
    return best;
}
const char *w4_parts_name(int64_t M, int64_t N, int64_t K) { return kForms[best_form(M, N, K)].name; }
float w4_parts_us(int64_t M, int64_t N, int64_t K) { return form_us(kForms[best_form(M, N, K)], M, N, K); }

template <class T> static void run_parts(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    switch (best_form(a.M, a.N, a.K)) {
    case 0: launch_groups<T, 1, 4, 4, 3>(a, p, s); break;
    case 1: launch_groups<T, 1, 2, 4, 3>(a, p, s); break;
    case 2: launch_groups<T, 1, 1, 8, 2>(a, p, s); break;
    case 3: launch_groups<T, 2, 4, 4, 2>(a, p, s); break;
    case 4: launch_groups<T, 2, 4, 2, 3>(a, p, s); break;
    default: launch_groups<T, 2, 2, 4, 2>(a, p, s); break;
    }
}
void launch_w4_parts(const W4Args &a, int type, const W4Prepared &p, hipStream_t s)
{
    if (type == QNN_BF16) run_parts<Bf16>(a, p, s);
    else run_parts<F16>(a, p, s);
}

} // namespace qnn
