// Products of 16-bit float rows with 4-bit weights that have one scale per group of a row (qnn_w4_matmul).
//
//   y[m][n] = bias[n] + sum_g s[g][n] * (sum_{k in g} x[m][k] * (8 + c[n][k]) - (8 + z[g][n]) * sum_{k in g} x[m][k])
//
// A nibble u = 8 + c becomes a 16-bit float by setting the bits of a power of two above it: 128 + u in bfloat16, 1024 + u in
// binary16 (from which the 1024 is then taken off; bfloat16 has no packed subtraction, so there the 128 stays and joins the
// 8 + z of the group's term).  No weight is rounded.  The group's sum of x comes from one more matrix product with ones.
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
    int32_t M, N, K, group;
};

// eight nibbles of a dword as 16-bit floats in the order 0 4 1 5 2 6 3 7: pairs (i, i + 4)
template <class T> struct Nibbles;
template <> struct Nibbles<Bf16> {
    static constexpr float kOffset = 128.0f + 8.0f;
    static __device__ __forceinline__ uint32_t two(uint32_t w) { return (w & 0x000f000fu) | 0x43004300u; }
    static __device__ __forceinline__ f32x4 mfma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
    static constexpr uint32_t kOnes = 0x3f803f80u;
};
template <> struct Nibbles<F16> {
    static constexpr float kOffset = 8.0f;
    static __device__ __forceinline__ uint32_t two(uint32_t w)
    {
        const h16x2 off = {(_Float16)1024.0f, (_Float16)1024.0f};
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(h16x2, (w & 0x000f000fu) | 0x64006400u) - off);
    }
    static __device__ __forceinline__ f32x4 mfma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
    }
    static constexpr uint32_t kOnes = 0x3c003c00u;
};
template <class T> __device__ __forceinline__ w32x4 expand_nibbles(uint32_t w)
{
    w ^= 0x88888888u;
    return w32x4{Nibbles<T>::two(w), Nibbles<T>::two(w >> 4), Nibbles<T>::two(w >> 8), Nibbles<T>::two(w >> 12)};
}
// eight consecutive 16-bit elements in the same order
__device__ __forceinline__ w32x4 pair_order(w32x4 v)
{
    return w32x4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                 __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}

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
// consecutive outputs.  A lane loads 16 bytes of a row of codes, 32 weights; after exchange among the four lanes of a
// row, dword j of each holds weights of the j-th 32 of the 128, so that every product of 32 lies within one group.
// GS: groups in 128 weights as far as the sums are concerned (1: groups of whole 128s, 2: 64, 4: any multiple of 32).
template <class T, int MT, int NT, int WAVES, int GS> __global__ void __launch_bounds__(64 * WAVES) w4_rows_kernel(const W4Args a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16 * NT, m0 = blockIdx.y * 16 * MT;
    const int steps = (a.K + 127) / 128;
    const int row_bytes = a.K / 2;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint8_t *w_row[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) w_row[nt] = a.codes + (int64_t)min(n0 + nt * 16 + c, a.N - 1) * row_bytes;
    const uint16_t *x_row[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) x_row[mt] = a.x + (int64_t)min(m0 + mt * 16 + c, a.M - 1) * a.ldx;

    for (int step = wave; step < steps; step += WAVES) {
        const int k0 = step * 128;
        const bool whole = k0 + 128 <= a.K;
        w32x4 w[NT], x[MT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int at = k0 / 2 + 16 * g;
            if (whole || at + 16 <= row_bytes) w[nt] = load_any<w32x4>(w_row[nt] + at);
            else {
                w[nt] = w32x4{0u, 0u, 0u, 0u};
                for (int b = 0; b < row_bytes - at; ++b) w[nt][b >> 2] |= (uint32_t)w_row[nt][at + b] << (b & 3) * 8;
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = k0 + 32 * j + 8 * g;
                x[mt][j] = w32x4{0u, 0u, 0u, 0u};
                if (m0 + mt * 16 + c < a.M) {
                    if (whole || at + 8 <= a.K) x[mt][j] = load_any<w32x4>(x_row[mt] + at);
                    else
                        for (int b = 0; b < a.K - at; ++b) x[mt][j][b >> 1] |= (uint32_t)x_row[mt][at + b] << (b & 1) * 16;
                }
            }
        float s[NT][GS][4], z[NT][GS][4];
#pragma unroll
        for (int q = 0; q < GS; ++q) {
            const int group = min((k0 + q * (128 / GS)), a.K - 1) / a.group;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int n = min(n0 + nt * 16 + 4 * g + e, a.N - 1);
                    s[nt][q][e] = T::widen(a.scales[(int64_t)group * a.N + n]);
                    z[nt][q][e] = Nibbles<T>::kOffset + (a.zeros ? (float)a.zeros[(int64_t)group * a.N + n] : 0.0f);
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) w[nt] = transpose_groups(w[nt]);
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
                w32x4 wide[NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) wide[nt] = expand_nibbles<T>(w[nt][j]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const w32x4 xp = pair_order(x[mt][j]);
                    const w32x4 ones = {Nibbles<T>::kOnes, Nibbles<T>::kOnes, Nibbles<T>::kOnes, Nibbles<T>::kOnes};
                    sums[mt] = Nibbles<T>::mfma(ones, xp, sums[mt]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) part[mt][nt] = Nibbles<T>::mfma(wide[nt], xp, part[mt][nt]);
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[mt][nt][e] = fmaf(s[nt][q][e], fmaf(-z[nt][q][e], sums[mt][e], part[mt][nt][e]), acc[mt][nt][e]);
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
        if (a.bias) v += T::widen(a.bias[n0 + n]);
        a.y[(int64_t)(m0 + m) * a.ldy + n0 + n] = T::narrow(v);
    }
}

template <class T, int GS> static void launch_w4(const W4Args &a, hipStream_t s)
{
    if (a.M <= 16) {
        const dim3 grid((unsigned)((a.N + 15) / 16), 1u);
        hipLaunchKernelGGL((w4_rows_kernel<T, 1, 1, 4, GS>), grid, dim3(256), 0, s, a);
    } else {
        const dim3 grid((unsigned)((a.N + 31) / 32), (unsigned)((a.M + 31) / 32));
        hipLaunchKernelGGL((w4_rows_kernel<T, 2, 2, 4, GS>), grid, dim3(256), 0, s, a);
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

static bool bad_w4_sizes(int64_t M, int64_t N, int64_t K, int64_t group)
{
    return M < 0 || N <= 0 || K <= 0 || K % 2 != 0 || group <= 0 || group % 32 != 0 || M > (1 << 20) || N > (1 << 28) || K > (1 << 28);
}

size_t qnn_w4_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t group)
{
    if (bad_w4_sizes(M, N, K, group)) return 0;
    return 0;
}

qnn_status qnn_w4_matmul(const void *x, int64_t ldx, const uint8_t *codes, const void *scales, const int8_t *zeros, const void *bias, int64_t M,
                         int64_t N, int64_t K, int64_t group, int type, void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_w4_sizes(M, N, K, group) || bad_half_type(type)) return QNN_EINVAL;
    if (M == 0) return QNN_OK;
    if (!x || !codes || !scales || !y || ldx < K || ldy < N) return QNN_EINVAL;
    const size_t need = qnn_w4_matmul_workspace_bytes(M, N, K, group);
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < need)) return QNN_EINVAL;
    const W4Args a{static_cast<const uint16_t *>(x), codes, static_cast<const uint16_t *>(scales), zeros, static_cast<const uint16_t *>(bias),
                   static_cast<uint16_t *>(y), ldx, ldy, (int32_t)M, (int32_t)N, (int32_t)K, (int32_t)(group < K ? group : (K + 127) / 128 * 128)};
    return type == QNN_BF16 ? run_w4<Bf16>(a, as_stream(stream)) : run_w4<F16>(a, as_stream(stream));
}

} // extern "C"
