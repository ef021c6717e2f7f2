// Products of rows and weights in e4m3 with a scale per 128 of a row and per 128 x 128 weights (qnn_f8_matmul).
//
//   y[m][n] = bias[n] + sum_b xs[b][m] ws[n / 128][b] * sum_{k in b} x[m][k] w[n][k]
//
// The sum over a block comes from the matrix unit; one multiply-add in binary32 for each output and block joins it to the others.
#include "f8_few.h"
#include "f8_matmul.h"

#include <cstdio>

namespace qnn {

template <int MT, int NT, int WAVES, int DEPTH> static void launch_rows(const F8Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), block(64 * WAVES);
    if (a.type == QNN_F32) hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, DEPTH, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, DEPTH, true>), grid, block, 0, s, a);
}

// 32 rows of weights per wave halve what x costs, where workgroups for all CUs are left: 16 x 28672 x 8192 54 us against 58, 64 rows 96 against 141; but
// one row 47 against 42, and 16 x 4096 x 4096 9.4 against 7.2.
static bool wide_rows(int64_t M, int64_t N) { return M > 8 && N >= 8192; }

static void launch_f8_rows(const F8Args &a, hipStream_t s)
{
    const bool wide = wide_rows(a.M, a.N);
    if (a.M <= 16) wide ? launch_rows<1, 2, 4, 3>(a, s) : launch_rows<1, 1, 8, 3>(a, s);
    else if (a.M <= 32) wide ? launch_rows<2, 2, 4, 3>(a, s) : launch_rows<2, 1, 8, 2>(a, s);
    else if (a.M <= 48) wide ? launch_rows<3, 2, 4, 3>(a, s) : launch_rows<3, 1, 8, 2>(a, s);
    else wide ? launch_rows<4, 2, 4, 3>(a, s) : launch_rows<4, 1, 8, 2>(a, s);
}

// By estimated time (us):
// rows: a launch, weights at 5.9 TB/s, and x from the L2 for every 16 rows of it and 16 or 32 of weights (measured / estimated: 16 x 4096 x 4096
// 7.2 / 8.5, 64 rows 15.1 / 15.0; 16 x 28672 x 8192 54 / 58, 64 rows 96 / 101; 32 x 12288 x 4096 18.6 / 18.1);
// 64 rows by 64 of weights per workgroup, whose 8 waves share K: 0.475 for a block of 128 on 256 CUs (1021 x 1001 x 1024 8.2 / 8.2, x 512 6.3 / 6.3);
// tiles: a CU does a step of 128 with a tile of 128 x 128 in 0.58 us, with binary32 results 0.9, of 256 x 256 in 1.93, or as fast as the weights come
// (24 x 28672 x 8192 52.5 / 52, 300 x 4096 x 4096 in two parts 16.6 and its sum / 17.6, 1000 x 12288 x 4096 67.5 / 59, 8192 x 8192 x 8192 495 / 499).
F8Plan f8_plan(int64_t M, int64_t N, int64_t K, int type)
{
    F8Plan best{F8Kernel::Rows, 1, 1e30f, false, 0, 0, 0};
    const float steps = (float)f8_blocks(K), weights = (float)N * (float)K * 1e-6f, outputs = (float)M * (float)N * 1e-6f; // (MB, if bytes)
    const bool wide = type == QNN_F32;
    const int64_t turns = (M + 63) / 64, tiles_of_16 = M < 64 ? (M + 15) / 16 : 4;
    best.us = (float)turns * (weights * (0.17f + (float)tiles_of_16 * (wide_rows(M, N) ? 0.061f : 0.13f)) * (wide ? 1.3f : 1.0f)) + 3.5f;
    if (K > (1 << 20) || M * N >= (int64_t)1 << 37) return best; // (beyond the tiles' offsets, and 2^32 threads)
    const bool padded = K % 16 != 0; // (loads from rows at any byte take twice as long)
    const float before = padded ? 3.0f + (weights + (float)M * (float)K * 1e-6f) * 0.45f : 0.0f;
    const float us64 = 4.4f + before + (float)((turns * ((N + 63) / 64) + 255) / 256) * steps * 0.475f;
    if (M > 64 && us64 < best.us) best.us = us64, best.kernel = F8Kernel::Rows64, best.padded = padded;
    const auto consider = [&](F8Kernel kernel, int64_t tile, float step) {
        const int64_t tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
        for (int splits = 1; splits <= 16; ++splits) {
            if (splits > 1 && (steps < 4.0f * (float)splits || tiles * (splits - 1) >= 512)) break;
            const float turn = (float)((tiles * splits + 255) / 256);
            float us = turn * ceilf(steps / (float)splits) * step;
            if (us < weights * 0.2f) us = weights * 0.2f;
            us += 5.0f + before + (splits > 1 ? 4.0f + (float)splits * outputs * 1.6f : 0.0f);
            if (us < best.us) best.us = us, best.kernel = kernel, best.splits = splits, best.padded = padded;
        }
    };
    consider(F8Kernel::Tile128, 128, wide ? 0.9f : 0.58f);
    if (!wide) consider(F8Kernel::Tile256, 256, 1.93f);
    const auto rounded = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    if (best.padded) best.x_bytes = rounded(M * f8_padded(K)), best.w_bytes = rounded(N * f8_padded(K));
    best.bytes = best.x_bytes + best.w_bytes + (best.splits > 1 ? rounded(4 * best.splits * M * N) : 0);
    return best;
}

} // namespace qnn

using namespace qnn;

extern "C" {

static bool bad_f8_sizes(int64_t M, int64_t N, int64_t K) { return M < 0 || N <= 0 || K <= 0 || M > (1 << 20) || N > (1 << 24) || K > (1 << 24); }

qnn_status qnn_f8_matmul(const uint8_t *x, int64_t ldx, const float *x_scales, int64_t ldxs, const uint8_t *w, const float *w_scales, const void *bias,
                         int64_t M, int64_t N, int64_t K, int type, void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_f8_sizes(M, N, K) || (bad_half_type(type) && type != QNN_F32)) return QNN_EINVAL;
    if (M == 0) return QNN_OK;
    if (!x || !x_scales || !w || !w_scales || !y || ldx < K || ldxs < M || ldy < N) return QNN_EINVAL;
    const F8Plan plan = f8_plan(M, N, K, type);
    if (plan.bytes > 0 && (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < plan.bytes)) return QNN_EINVAL;
    F8Args a{x, w, x_scales, w_scales, bias, y, ldx, ldxs, ldy, (int32_t)M, (int32_t)N, (int32_t)K, type};
    hipStream_t s = as_stream(stream);
    uint8_t *const space = static_cast<uint8_t *>(workspace);
    if (plan.padded) {
        launch_f8_pad(a, space, space + plan.x_bytes, s);
        a.x = space, a.w = space + plan.x_bytes, a.ldx = a.K = (int32_t)f8_padded(K);
    }
    const bool pieces = ((uintptr_t)a.x | (uintptr_t)a.ldx | (uintptr_t)a.w | (uintptr_t)a.K) % 16 == 0 && a.ldx < (1 << 22);
    if ((plan.kernel == F8Kernel::Tile128 || plan.kernel == F8Kernel::Tile256) && pieces) launch_f8_tiles(a, plan, reinterpret_cast<float *>(space + plan.x_bytes + plan.w_bytes), s);
    else if (plan.kernel == F8Kernel::Rows) launch_f8_rows(a, s);
    else launch_rows<4, 4, 8, 2>(a, s);
    return launch_status(hipGetLastError());
}

size_t qnn_f8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, int type)
{
    return bad_f8_sizes(M, N, K) || M == 0 || (bad_half_type(type) && type != QNN_F32) ? 0 : f8_plan(M, N, K, type).bytes;
}

const char *qnn_f8_matmul_plan(int64_t M, int64_t N, int64_t K, int type)
{
    if (bad_f8_sizes(M, N, K) || M == 0 || (bad_half_type(type) && type != QNN_F32)) return "";
    const F8Plan p = f8_plan(M, N, K, type);
    static thread_local char name[32];
    if (p.kernel == F8Kernel::Rows) std::snprintf(name, sizeof(name), "rows%dx%s", M < 64 ? (int)((M + 15) / 16 * 16) : 64, wide_rows(M, N) ? "32" : "16");
    else if (p.kernel == F8Kernel::Rows64) return "rows64x64";
    else std::snprintf(name, sizeof(name), "tile%s/%d", p.kernel == F8Kernel::Tile256 ? "256x256" : "128x128", p.splits);
    return name;
}

} // extern "C"
