// Products of 16-bit float rows with 4-bit weights that have one scale per group of a row (qnn_w4_matmul).
//
//   y[m][n] = bias[n] + sum_g s[g][n] * (sum_{k in g} x[m][k] * (8 + c[n][k]) - (8 + z[g][n]) * sum_{k in g} x[m][k])
//
// A nibble u = 8 + c becomes a 16-bit float by setting the bits of a power of two above it: 128 + u in bfloat16, 1024 + u in
// binary16 (from which the 1024 is then taken off; bfloat16 has no packed subtraction, so there the 128 stays, as 2^-9 with all else in units
// of 2^16, and joins the 8 + z of the group's term).  No weight is rounded.  The group's sum of x comes from one more matrix product with ones.
//
// Few rows are bound by reading the codes, small products by the launch and one chain of loads: 1 x 4096 x 4096 4.6 us, 5 x 5001 x 2890 with
// zero-points 8.6 us (its rows of codes begin at any byte).  With more than about 16 rows x is shared through LDS (w4_parts.hip), with hundreds
// weights are as well used as in any dense product (w4_tile.hip).
#include "w4.h"

namespace qnn {

// dword j of lane group g <-> dword g of lane group j
__device__ __forceinline__ w32x4 transpose_groups(w32x4 a)
{
    const auto s02 = __builtin_amdgcn_permlane32_swap(a[0], a[2], false, false);
    const auto s13 = __builtin_amdgcn_permlane32_swap(a[1], a[3], false, false);
    const auto t01 = __builtin_amdgcn_permlane16_swap(s02[0], s13[0], false, false);
    const auto t23 = __builtin_amdgcn_permlane16_swap(s02[1], s13[1], false, false);
    return w32x4{t01[0], t01[1], t23[0], t23[1]};
}

// One wave takes 16 * NT rows of the weights and 16 * MT rows of x; the waves of a workgroup share K in turns of 128 and join
// their sums in LDS.  The product is formed transposed (weights are the left operand): a lane has one row of x and four
// consecutive outputs.  A lane loads 16 bytes of a row of codes, 32 weights.
// After an exchange of dwords among the four lanes of a row, dword j of each holds weights of the j-th 32 of the 128, so that every
// product of 32 lies within one group, and x is read in pieces of 64 consecutive bytes.
// GS: groups in 128 weights as far as the sums are concerned (1: groups of whole 128s, 2: 64, 4: any multiple of 32).
// TINY: fewer than four scales in all.
// The codes of a wave's next 128 are in flight while it works on these; x comes from the L2, which all workgroups read it from.  The loop has no branches (rows
// beyond the ends are the last one again, and dropped at the end); a last part of K below 128 goes before it.
template <class T, int MT, int NT, int WAVES, int GS, bool ZEROS, bool TINY> __global__ void __launch_bounds__(64 * WAVES, WAVES == 16 ? 4 : 2) w4_rows_kernel(const W4Args a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int whole = a.K / 128, row_bytes = a.K / 2;
    const uint32_t bits = kept(Nibbles<T>::kBits);
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *const w_base = a.codes + (int64_t)n0 * row_bytes;
    uint32_t w_row[NT]; // (at most 16 * NT rows of 2^23 bytes)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w_row[nt] = (uint32_t)(min(n0 + nt * 16 + c, a.N - 1) - n0) * row_bytes;
    const uint16_t *x_row[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x_row[mt] = a.x + (int64_t)min(m0 + mt * 16 + c, a.M - 1) * a.ldx;
    const uint32_t params = (uint32_t)a.groups * a.N; // scales, zero-points: less than 2^30

    // scales as they were loaded: four from (group, n) on or, where that is beyond the array, its last four, which have to be moved
    // down by `drop` when they are used
    struct Step {
        Codes<4> w[NT];
        uint64_t s[NT][GS];
        uint32_t z[NT][GS], drop[NT][GS];
    };
    auto load_scales = [&](Step &f, int step) {
#pragma unroll
        for (int q = 0; q < GS; ++q) {
            const uint32_t group = (uint32_t)group_of(a, min(step * 128 + q * (128 / GS), a.K - 1)) * a.N;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint32_t want = group + min(n0 + nt * 16 + 4 * g, a.N - 1);
                f.z[nt][q] = 0, f.drop[nt][q] = 0;
                if (TINY) {
                    f.s[nt][q] = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t at = min(want + e, params - 1);
                        f.s[nt][q] |= (uint64_t)a.scales[at] << 16 * e;
                        if (ZEROS) f.z[nt][q] |= (uint32_t)(uint8_t)a.zeros[at] << 8 * e;
                    }
                } else {
                    const uint32_t at = min(want, params - 4);
                    f.drop[nt][q] = want - at;
                    f.s[nt][q] = load_any<uint64_t>(a.scales + at);
                    if (ZEROS) f.z[nt][q] = load_any<uint32_t>(a.zeros + at);
                }
            }
        }
    };
    auto load = [&](Step &f, int step) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) f.w[nt].load(w_base + (w_row[nt] + (uint32_t)(64 * step + 16 * g)), a.skewed);
        load_scales(f, step);
    };
    auto row_at = [&](int step, int j) { return step * 128 + 32 * j + 8 * g; };
    auto compute = [&](Step &f, const w32x4 (&x)[MT][4]) {
        w32x4 w[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            f.w[nt].place(w_base + w_row[nt], a.skewed);
            w[nt] = transpose_groups(w32x4{f.w[nt].w[0], f.w[nt].w[1], f.w[nt].w[2], f.w[nt].w[3]});
        }
#pragma unroll
        for (int q = 0; q < GS; ++q) {
            f32x4 part[MT][NT], sums[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                sums[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) part[mt][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int j = q * (4 / GS); j < (q + 1) * (4 / GS); ++j) {
                w32x4 xp[MT];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    xp[mt] = pair_order(x[mt][j]);
                    const w32x4 ones = {Nibbles<T>::kOnes, Nibbles<T>::kOnes, Nibbles<T>::kOnes, Nibbles<T>::kOnes};
                    sums[mt] = Nibbles<T>::mfma(ones, xp[mt], sums[mt]);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const w32x4 wide = expand_nibbles<T>(w[nt][j], bits);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) part[mt][nt] = Nibbles<T>::mfma(wide, xp[mt], part[mt][nt]);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const u16x4 s4 = __builtin_bit_cast(u16x4, f.s[nt][q] >> (TINY ? 0 : 16 * f.drop[nt][q]));
                const uint32_t z4 = f.z[nt][q] >> (TINY ? 0 : 8 * f.drop[nt][q]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float s = T::widen(s4[e]);
                    const float z = Nibbles<T>::kOffset + (ZEROS ? (float)(int8_t)(z4 >> 8 * e) : 0.0f);
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) acc[mt][nt][e] = fmaf(s, fmaf(-z, sums[mt][e], part[mt][nt][e]), acc[mt][nt][e]);
                }
            }
        }
    };
    w32x4 x[MT][4];
    auto load_rows = [&](int step) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[mt][j] = load_any<w32x4>(x_row[mt] + row_at(step, j));
    };
    Step f[2];
    // Each workgroup begins at another place of K: rows lie a power of two apart more often than not, and workgroups that
    // read the same columns of all rows at one time would keep to a part of the memory's channels.
    const int mine = (whole - wave + WAVES - 1) / WAVES;
    int at = mine > 0 ? (int)(blockIdx.x % (uint32_t)mine) : 0;
    if (mine > 0) load(f[0], wave + WAVES * at);
    if (a.K % 128 != 0 && wave == whole % WAVES) { // the last, shorter part, while the first whole one is on its way
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) f[1].w[nt].load_tail(w_base + w_row[nt], row_bytes, 64 * whole + 16 * g, a.skewed);
        load_scales(f[1], whole);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[mt][j] = load_end(reinterpret_cast<const uint8_t *>(x_row[mt]), 2 * a.K, 2 * row_at(whole, j));
        compute(f[1], x);
    }
    if (mine > 0) {
        const auto next = [&] { at = at + 1 < mine ? at + 1 : 0; };
        for (int i = 0; i < mine / 2; ++i) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                load_rows(wave + WAVES * at);
                next();
                load(f[1 - half], wave + WAVES * at); // (after the last: once again, unused)
                compute(f[half], x);
            }
        }
        if (mine & 1) {
            load_rows(wave + WAVES * at);
            compute(f[0], x);
        }
    }

    // outputs [row of x][n], the waves' sums added in their order
    __shared__ float s_acc[WAVES][16 * MT][16 * NT + 4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4 *>(&s_acc[wave][mt * 16 + c][nt * 16 + g * 4]) = acc[mt][nt];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * MT * 16 * NT; i += 64 * WAVES) {
        const int m = i / (16 * NT), n = i % (16 * NT);
        if (m0 + m >= a.M || n0 + n >= a.N) continue;
        float v = s_acc[0][m][n];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s_acc[w][m][n];
        if constexpr (Nibbles<T>::kUnit != 0) v = ldexpf(v, Nibbles<T>::kUnit);
        if (a.bias) v += T::widen(a.bias[n0 + n]);
        a.y[(int64_t)(m0 + m) * a.ldy + n0 + n] = T::narrow(v);
    }
}

template <class T, int MT, int NT, int WAVES, int GS, bool TINY = false> static void launch_rows(const W4Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT)));
    if (a.zeros) hipLaunchKernelGGL((w4_rows_kernel<T, MT, NT, WAVES, GS, true, TINY>), grid, dim3(64 * WAVES), 0, s, a);
    else hipLaunchKernelGGL((w4_rows_kernel<T, MT, NT, WAVES, GS, false, TINY>), grid, dim3(64 * WAVES), 0, s, a);
}

// tiles of 16 rows of weights per wave
static int few_tiles(int64_t N) { return N > 16384 ? 2 : 1; }

// waves along K: fewer than four scales in all (no four to load at once); two tiles per wave; as a workgroup of 16 waves has a CU to
// itself, 16 only where there are no more workgroups than CUs (1 x 12288 x 4096 13.1 us with 16, 9.9 with 8).  (With groups that are not whole 64s
// 16 waves have too few registers: 21 to 29 are spilled, some of them inside the loop.)
static int few_form(int64_t N, int64_t groups) { return groups * N < 4 ? 0 : few_tiles(N) == 2 ? 1 : (N + 15) / 16 > 256 ? 2 : 3; }

template <class T, int GS> static void launch_w4(const W4Args &a, hipStream_t s)
{
    switch (few_form(a.N, a.groups)) {
    case 0: launch_rows<T, 1, 1, 4, GS, true>(a, s); break;
    case 1: launch_rows<T, 1, 2, 8, GS>(a, s); break;
    case 2: launch_rows<T, 1, 1, 8, GS>(a, s); break;
    default: launch_rows<T, 1, 1, 16, GS>(a, s); break;
    }
}

template <class T> static qnn_status run_w4(const W4Args &a, hipStream_t s)
{
    if (a.group % 128 == 0) launch_w4<T, 1>(a, s);
    else if (a.group % 64 == 0) launch_w4<T, 2>(a, s);
    else launch_w4<T, 4>(a, s);
    return launch_status(hipGetLastError());
}

} // namespace qnn

using namespace qnn;

extern "C" {

// (N: a launch has fewer than 2^32 threads along x, 16 for each row of weights)
static bool bad_w4_sizes(int64_t M, int64_t N, int64_t K, int64_t group)
{
    return M < 0 || N <= 0 || K <= 0 || K % 2 != 0 || group <= 0 || group % 32 != 0 || M > (1 << 20) || N > (1 << 28) - 32 || K > (1 << 24) || (K + group - 1) / group * N >= (1 << 30);
}

// Which kernel, by what each is estimated to take (us):
// few rows: weights at 4 TB/s and x, read again for every 16 or 32 rows of weights, at 9 TB/s from the L2 (measured / estimated at
// 16 rows: 4096 x 4096 7.5 / 8.3, 12288 x 4096 19.5 / 20, 28672 x 8192 51 / 58);
// tens: see w4_parts.hip;  many: for a round of tiles and 128 of K 2 us with groups of whole 128s (200 rows x 28672 x 8192 135 / 133, 1000: 471 /
// 453), else, for 64 rows, 1.3 with groups of 64s (1000: 586 / 587; 2000 x 12288 x 4096 271 / 255) and 1.65 with smaller ones (327 / 322).  With these
// groups the kernel for tens takes 1.35 and 1.75 times as long as with whole 128s (2000 x 12288 x 4096 330 / 315 and 416 / 408); up to 16 rows,
// where reading the codes takes most of its time (8 x 28672 x 8192 34, 38 and 47 us with groups of 128, 64 and 32), the choice does not look at the group.
enum class W4Kernel { Few, Tens, Many };
static W4Kernel w4_kernel(int64_t M, int64_t N, int64_t K, int64_t group)
{
    // (longer rows than the other kernels' offsets reach stay with that for few)
    if (K > (1 << 21)) return W4Kernel::Few;
    const float tens = w4_parts_us(M, N, K);
    if (M <= 16) {
        const float weights = (float)N * (float)K * 0.5e-6f;
        return 2.5f + weights * (0.25f + (float)M / (float)(36 * few_tiles(N))) <= tens ? W4Kernel::Few : W4Kernel::Tens;
    }
    const bool whole = group % 128 == 0 || group >= K;
    const int64_t tiles = (whole ? (M + 127) / 128 : (M + 63) / 64) * ((N + 255) / 256);
    const float rounds = tiles <= 256 ? 1.0f : (float)tiles / 256.0f;
    const float step_us = whole ? 2.0f : group % 64 == 0 ? 1.3f : 1.65f, longer = whole ? 1.0f : group % 64 == 0 ? 1.35f : 1.75f;
    return rounds * (float)((K + 127) / 128) * step_us < (tens - 5.0f) * longer ? W4Kernel::Many : W4Kernel::Tens; // (and 5 us for either)
}

size_t qnn_w4_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t group)
{
    if (bad_w4_sizes(M, N, K, group) || M == 0 || w4_kernel(M, N, K, group) == W4Kernel::Few) return 0;
    return w4_prepared_bytes(M, K);
}

const char *qnn_w4_matmul_plan(int64_t M, int64_t N, int64_t K, int64_t group)
{
    if (bad_w4_sizes(M, N, K, group) || M == 0) return "";
    switch (w4_kernel(M, N, K, group)) {
    case W4Kernel::Few: {
        static const char *const names[] = {"few16x16/4", "few16x32/8", "few16x16/8", "few16x16/16"};
        return names[few_form(N, (K + group - 1) / group)];
    }
    case W4Kernel::Tens: return w4_parts_name(M, N, K);
    default: return group % 128 == 0 || group >= K ? "many128x256" : "many64x256";
    }
}

qnn_status qnn_w4_matmul(const void *x, int64_t ldx, const uint8_t *codes, const void *scales, const int8_t *zeros, const void *bias, int64_t M,
                         int64_t N, int64_t K, int64_t group, int type, void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_w4_sizes(M, N, K, group) || bad_half_type(type)) return QNN_EINVAL;
    if (M == 0) return QNN_OK;
    if (!x || !codes || !scales || !y || ldx < K || ldy < N) return QNN_EINVAL;
    const size_t need = qnn_w4_matmul_workspace_bytes(M, N, K, group);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < need)) return QNN_EINVAL;
    W4Args a{static_cast<const uint16_t *>(x), codes, static_cast<const uint16_t *>(scales), zeros, static_cast<const uint16_t *>(bias),
                   static_cast<uint16_t *>(y), ldx, ldy, (int32_t)M, (int32_t)N, (int32_t)K, (int32_t)(group < K ? group : (K + 127) / 128 * 128), (int32_t)((K + group - 1) / group), 0, 0, (((uintptr_t)codes | (uintptr_t)(K / 2)) & 3) != 0};
    fast_division((uint32_t)a.group / 32, a.group_magic, a.group_shift);
    if (const W4Kernel kernel = w4_kernel(M, N, K, group); kernel != W4Kernel::Few) {
        const W4Prepared p = prepared(workspace, M, K);
        prepare_x(a, type, p, as_stream(stream));
        if (kernel == W4Kernel::Many) launch_w4_tile(a, type, p, as_stream(stream));
        else launch_w4_parts(a, type, p, as_stream(stream));
        return launch_status(hipGetLastError());
    }
    return type == QNN_BF16 ? run_w4<Bf16>(a, as_stream(stream)) : run_w4<F16>(a, as_stream(stream));
}

} // extern "C"
