// Products with 4-bit weights for many rows: x tiles through LDS, weights from memory into registers and from there, scaled, into
// the matrix units as binary16.
//
// Weights enter the matrix units as the whole numbers c - z, which binary16 holds exactly.  An accumulator stands in units of the
// scale of the group that it is at: at the next group it is multiplied by the ratio of the two scales.  That is
// one set of accumulators and one multiplication per output and group; as x is the left operand here, a lane's outputs are all of
// one row of weights, and the ratio is one number per lane.
// x has to fit binary16: a first launch writes it with each row scaled by a power of two, which is exact but for bfloat16 elements below
// 2^-32 of their row's largest, in the order of expand_nibbles, rows padded with zeros to whole 128s.
//
// Bound by the matrix units (50 % of the cycles) and the vector unit that turns codes into binary16 (49 %), which two waves on a SIMD overlap in part, and by the
// clock they leave: 2000 x 12288 x 4096 with zero-points 199-216 us with the first launch (6-12), 1000
// TFLOP/s; the library's product of the same size with 16-bit weights takes 180.  Tiles of 128 x 256 (64 x 256 with groups that are
// not whole 128s): 768 of them, three rounds of 256 CUs.
#include "buffer_ops.h"
#include "lds_ring.h"
#include "w4.h"

namespace qnn {

// One row per workgroup; rows of up to 16384 stay in registers between the two passes over them.
template <class T> __global__ void __launch_bounds__(1024) w4_prepare_kernel(const W4Args a, const W4Prepared p)
{
    const int tid = threadIdx.x;
    const uint8_t *const x = reinterpret_cast<const uint8_t *>(a.x + (int64_t)blockIdx.x * a.ldx);
    uint16_t *const out = p.x + (int64_t)blockIdx.x * p.pitch;
    __shared__ float s_peak[16];
    w32x4 first[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) first[i] = load_end(x, 2 * a.K, 16 * (tid + 1024 * i));
    float peak = 0.0f;
    const auto look = [&](const w32x4 &v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) peak = fmaxf(peak, fabsf(T::widen((uint16_t)(v[i >> 1] >> (i & 1) * 16))));
    };
    look(first[0]), look(first[1]);
    for (int k = 8 * (tid + 2048); k < a.K; k += 8 * 1024) look(load_end(x, 2 * a.K, 2 * k));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
    if ((tid & 63) == 0) s_peak[tid >> 6] = peak;
    __syncthreads();
    peak = s_peak[tid & 15];
#pragma unroll
    for (int d = 1; d < 16; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
    const int e = row_exponent(peak);
    if (tid == 0) p.row_exp[blockIdx.x] = e;
    const float down = ldexpf(1.0f, -e);
    const auto write = [&](const w32x4 &v, int k) {
        w32x4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = narrow2<F16>(T::widen((uint16_t)v[i]) * down, T::widen((uint16_t)(v[i] >> 16)) * down);
        *reinterpret_cast<w32x4 *>(out + k) = pair_order(h);
    };
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (8 * (tid + 1024 * i) < p.pitch) write(first[i], 8 * (tid + 1024 * i));
    for (int k = 8 * (tid + 2048); k < p.pitch; k += 8 * 1024) write(load_end(x, 2 * a.K, 2 * k), k);
}

// 256 rows of weights (64 per wave) times 32 * MT rows of x, K in steps of 128: x by LDS copies in two buffers, 16-byte pieces of a row exchanged
// by its number so that reads of 8 rows meet 8 different places; each lane loads 32 bytes of a row of codes, 64 weights, and
// the next 32 are on their way.
// GS: groups in 128 weights (1: groups of whole 128s, 2: of 64s, 4: any multiple of 32).  A product of 16 has to lie
// within a group: the two lanes of a row exchange dwords for GS > 1.
template <class T, int MT, int GS, bool ZEROS> __global__ void __launch_bounds__(256, 2) w4_tile_kernel(const W4Args a, const W4Prepared p, int m_tiles, int n_tiles)
{
    constexpr int BM = 32 * MT;
    __shared__ __attribute__((aligned(16))) uint8_t s_x[2][BM * 256];
    // workgroups are dealt to the 8 XCDs in turn: each XCD has weights of its own, for all rows of x
    const int xcd = blockIdx.x % 8, local = blockIdx.x / 8;
    const int tn = xcd + 8 * (local / m_tiles), tm = local % m_tiles;
    if (tn >= n_tiles) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 31, hh = lane >> 5;
    const int n0 = tn * 256 + wave * 64, m0 = tm * BM;
    const int row_bytes = a.K / 2, whole = a.K / 128, steps = (a.K + 127) / 128;

    const uint8_t *const x_tile = reinterpret_cast<const uint8_t *>(p.x + (int64_t)m0 * p.pitch);
    const int x_bytes = min(a.M - m0, BM) * p.pitch * 2; // rows beyond the last read as zeros
    auto copy_x = [&](int step, int buf) {
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) {
            const int row = (wave * 2 * MT + i) * 4 + (lane >> 4);
            const uint32_t piece = (lane & 15) ^ (row & 15);
            buffer_to_lds16(x_tile, x_bytes, (uint32_t)row * p.pitch * 2 + step * 256 + piece * 16, &s_x[buf][(wave * 2 * MT + i) * 1024]);
        }
    };

    const uint8_t *w_row[2];
    uint32_t n_at[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        n_at[t] = min(n0 + 32 * t + c, a.N - 1);
        w_row[t] = a.codes + (int64_t)n_at[t] * row_bytes + 32 * hh;
    }
    struct Weights {
        Codes<8> w[2];
        uint16_t s[2][GS];
        int8_t z[2][GS];
    };
    auto load_scales = [&](Weights &f, int step) {
#pragma unroll
        for (int q = 0; q < GS; ++q) {
            const uint32_t group = (uint32_t)group_of(a, min(step * 128 + q * (128 / GS), a.K - 1)) * a.N;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f.s[t][q] = a.scales[group + n_at[t]];
                f.z[t][q] = ZEROS ? a.zeros[group + n_at[t]] : 0;
            }
        }
    };
    auto load = [&](Weights &f, int step) {
#pragma unroll
        for (int t = 0; t < 2; ++t) f.w[t].load(w_row[t] + 64 * step, a.skewed);
        load_scales(f, step);
    };

    f32x16 acc[2][MT];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][mt][i] = 0.0f;
    ScaleUnit unit[2];
    const uint32_t bits = kept(Nibbles<F16>::kBits);

    auto compute = [&](Weights &f, int buf) {
        uint32_t w[2][8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f.w[t].place(w_row[t], a.skewed);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[t][i] = f.w[t].w[i];
            swap_halves<GS>(w[t]);
        }
        const uint8_t *const row = &s_x[buf][c * 256];
        GroupUnit unit_of[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i % (8 / GS) == 0) {
                const int q = i / (8 / GS);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    unit_of[t] = enter_group(T::widen(f.s[t][q]), f.z[t][q], unit[t]);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[t][mt] *= unit_of[t].ratio;
                }
            }
            const int piece = piece_of<GS>(i, hh);
            h16x8 xf[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) xf[mt] = *reinterpret_cast<const h16x8 *>(row + mt * 32 * 256 + (piece ^ (c & 15)) * 16);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const h16x8 wide = whole_weights(w[t][i], unit_of[t], bits);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[t][mt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xf[mt], wide, acc[t][mt], 0, 0, 0);
            }
        }
    };

    Weights f[2];
    copy_x(0, 0);
    if (whole > 0) load(f[0], 0);
    // This wave's copies have arrived, and all waves have what they read of the other buffer in registers: the compiler moves the last
    // products of a step, and the waits for their reads, past a barrier that does not wait itself, and copies into that buffer follow it.
    const auto next_buffer = [] {
        wait_vmcnt<0>();
        lds_barrier();
    };
    int step = 0;
    for (; step + 2 < whole; step += 2) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            next_buffer();
            copy_x(step + half + 1, 1 - half);
            load(f[1 - half], step + half + 1);
            compute(f[half], half);
        }
    }
    // up to two whole steps are left, and the part of one
    for (; step < steps; ++step) {
        next_buffer();
        if (step + 1 < steps) copy_x(step + 1, (step + 1) & 1);
        Weights last;
        if (step + 1 < whole) load(last, step + 1);
        if (step >= whole) {
#pragma unroll
            for (int t = 0; t < 2; ++t) f[0].w[t].load_tail(w_row[t] - 32 * hh, row_bytes, 64 * step + 32 * hh, a.skewed);
            load_scales(f[0], step);
        }
        compute(f[0], step & 1);
        if (step + 1 < whole) f[0] = last;
    }

    // outputs through LDS, rows of 64 per wave, 16-byte pieces exchanged as above
    lds_barrier(); // (the buffers' last reads are over)
    uint8_t *const tile = &s_x[0][0] + wave * (BM * 128);
    const Result result[2] = {Result(unit[0]), Result(unit[1])};
    float bias[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) bias[t] = a.bias ? T::widen(a.bias[n_at[t]]) : 0.0f;
    using i32x4 = int32_t __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int m = 32 * mt + 2 * i + 4 * hh;
            const i32x4 exp = *reinterpret_cast<const i32x4 *>(p.row_exp + m0 + m);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = result[t].of(acc[t][mt][i + e], exp[e]) + bias[t];
                    *reinterpret_cast<uint16_t *>(tile + (m + e) * 128 + ((4 * t + (c >> 3)) ^ ((m + e) & 7)) * 16 + (c & 7) * 2) = T::narrow(v);
                }
        }
    lds_barrier(); // (between waves nothing is exchanged; the compiler keeps the order of writes and reads)
#pragma unroll
    for (int i = 0; i < 4 * MT; ++i) {
        const int m = i * 8 + (lane >> 3), n = n0 + 8 * (lane & 7);
        if (m0 + m >= a.M || n >= a.N) continue;
        const w32x4 v = *reinterpret_cast<const w32x4 *>(tile + m * 128 + ((lane & 7) ^ (m & 7)) * 16);
        uint16_t *const y = a.y + (int64_t)(m0 + m) * a.ldy + n;
        if (n + 8 <= a.N) store_any(y, v);
        else
            for (int e = 0; e < a.N - n; ++e) y[e] = (uint16_t)(v[e >> 1] >> (e & 1) * 16);
    }
}

template <class T, int GS, bool ZEROS> static void launch_tiles(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    // (with groups of 64 and 32 the scales on their way and the sums of 128 rows would not fit the registers of two waves on a SIMD: 2000 x
    // 12288 x 4096 with zero-points 374 and 606 us, with 64 rows 280 and 337.  With whole 128s 11 to 15 registers are spilled, outside the loop.)
    constexpr int MT = GS == 1 ? 4 : 2;
    const int m_tiles = (a.M + 32 * MT - 1) / (32 * MT), n_tiles = (a.N + 255) / 256;
    hipLaunchKernelGGL((w4_tile_kernel<T, MT, GS, ZEROS>), dim3((unsigned)(((n_tiles + 7) / 8) * 8 * m_tiles)), dim3(256), 0, s, a, p, m_tiles, n_tiles);
}

template <class T> static void run_tiles(const W4Args &a, const W4Prepared &p, hipStream_t s)
{
    if (a.group % 128 == 0) a.zeros ? launch_tiles<T, 1, true>(a, p, s) : launch_tiles<T, 1, false>(a, p, s);
    else if (a.group % 64 == 0) a.zeros ? launch_tiles<T, 2, true>(a, p, s) : launch_tiles<T, 2, false>(a, p, s);
    else a.zeros ? launch_tiles<T, 4, true>(a, p, s) : launch_tiles<T, 4, false>(a, p, s);
}

void prepare_x(const W4Args &a, int type, const W4Prepared &p, hipStream_t s)
{
    if (type == QNN_BF16) hipLaunchKernelGGL(w4_prepare_kernel<Bf16>, dim3((unsigned)a.M), dim3(1024), 0, s, a, p);
    else hipLaunchKernelGGL(w4_prepare_kernel<F16>, dim3((unsigned)a.M), dim3(1024), 0, s, a, p);
}

void launch_w4_tile(const W4Args &a, int type, const W4Prepared &p, hipStream_t s)
{
    if (type == QNN_BF16) run_tiles<Bf16>(a, p, s);
    else run_tiles<F16>(a, p, s);
}

} // namespace qnn
