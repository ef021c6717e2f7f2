// Products of rows and weights in e4m3 with a scale per 128 of a row and per 128 x 128 weights (qnn_f8_matmul).
//
//   y[m][n] = bias[n] + sum_b xs[b][m] ws[n / 128][b] * sum_{k in b} x[m][k] w[n][k]
//
// The sum over a block comes from the matrix unit; one multiply-add in binary32 for each output and block joins it to the others.
#include "f8_few.h"
#include "f8_matmul.h"

#include <cstdio>

namespace qnn {

// Rows that begin with a word each.  (Those that do not: one step ahead, and 16 rows of weights; 32 would not fit the registers.  64 by 64, which is
// what is left where that or tiles were planned for rows that begin with a word, spills 43 registers, with binary32 results 53.)
static bool words(const F8Args &a) { return ((uintptr_t)a.x | (uintptr_t)a.ldx | (uintptr_t)a.w | (uintptr_t)a.K) % 4 == 0; }

template <int MT, int NT, int WAVES, int DEPTH, bool ANY = false> static void launch_rows(const F8Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), block(64 * WAVES);
    if constexpr (!ANY && NT != 2)
        if (!words(a)) return launch_rows<MT, NT, WAVES, 2, true>(a, s);
    if (a.type == QNN_F32) hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, DEPTH, false, ANY>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, DEPTH, true, ANY>), grid, block, 0, s, a);
}

// 32 rows of weights per wave halve what x costs, where workgroups for all CUs are left: 24 x 28672 x 8192 51.5 us, 64 rows 74 (with 16: 55 and 104); but
// 8 rows 45 against 47, and 16 x 4096 x 4096 6.0 against 7.2.
static bool wide_rows(int64_t M, int64_t N) { return M > 8 && N >= 8192; }

static void launch_f8_rows(const F8Args &a, hipStream_t s)
{
    const bool wide = wide_rows(a.M, a.N) && words(a);
    if (a.M <= 16) wide ? launch_rows<1, 2, 4, 3>(a, s) : launch_rows<1, 1, 8, 3>(a, s);
    else if (a.M <= 32) wide ? launch_rows<2, 2, 4, 3>(a, s) : launch_rows<2, 1, 8, 2>(a, s);
    else if (a.M <= 48) wide ? launch_rows<3, 2, 4, 3>(a, s) : launch_rows<3, 1, 8, 2>(a, s);
    else wide ? launch_rows<4, 2, 4, 3>(a, s) : launch_rows<4, 1, 8, 2>(a, s);
}

// By estimated time (us), of a launch and what follows.  Measured / estimated, with bfloat16 results and weights that no cache holds:
// rows: 256 workgroups at a time, each a step of 128 in 0.045 and 0.0025 for each row (32 x 4096 x 4096 7.0 / 7.8,
// 64 rows 10.1 / 10.4, 1000 rows 121 / 121; without a bound by the weights' bytes: 1 x 28672 x 8192 51 / 29.9, 8 rows 50 / 37.7, where the others' are higher still), or wide by the weights' bytes (24 x 28672 x 8192 51.5 / 52, 64 x 12288 x 4096 21.6 / 20.3) while one turn
// takes all rows, then 512 at a time, 0.4 for a step (300 x 12288 x 4096 56 / 57).  Rows that begin within a
// word take 0.1 and 0.0065 (1 x 4096 x 4095 6.6 / 7.2, 64 rows 20.0 / 20.3), so that a copy with whole pieces comes first where that is less: 3, and 0.365 for
// a megabyte (64 x 4096 x 4095 19.3 / 20).
// 64 rows by 64 of weights per workgroup, whose 8 waves share K: 0.4 for a step on 256 CUs (1000 x 1024 x 1024 7.0 / 7.0, 500 x 2048 x 9216 32.3 / 32.6);
// tiles: a CU does a step of 128 with a tile of 128 x 128 in 0.62 us, with binary32 results 0.97, of 256 x 256 in 1.85, or as fast as the weights come
// (64 x 28672 x 8192 59 / 55, 300 x 4096 x 4096 in two parts 21.6 / 22.9, 1000 x 12288 x 4096 68.9 / 64.5 and 61.2 / 64.2, 8192 x 8192 x 8192 495 / 479).
F8Plan f8_plan(int64_t M, int64_t N, int64_t K, int type)
{
    F8Plan best{F8Kernel::Rows, 1, 1e30f, false, 0, 0, 0};
    const float steps = (float)f8_blocks(K), weights = (float)N * (float)K * 1e-6f, outputs = (float)M * (float)N * 1e-6f; // (MB, if bytes)
    const bool wide = type == QNN_F32, parts = K % 16 != 0, odd = K % 4 != 0;
    const int64_t turns = (M + 63) / 64;
    const float rows = M < 64 ? (float)M : 64.0f; // of a turn
    const auto rounds = [](int64_t groups, int64_t at_once) { return (float)((groups + at_once - 1) / at_once); };
    const auto rows_us = [&](bool any_byte) {
        if (any_byte || !wide_rows(M, N)) return 3.0f + rounds(turns * ((N + 15) / 16), 256) * (0.8f + steps * (any_byte ? 0.1f + 0.0065f * rows : 0.045f + 0.0025f * rows));
        const float wider = wide && M > 48 ? 1.5f : 1.0f;
        if (turns == 1) return 6.0f + weights * (0.142f + 0.00224f * rows) * wider;
        return 3.0f + rounds(turns * ((N + 31) / 32), 512) * (0.8f + steps * 0.4f * wider);
    };
    best.us = rows_us(odd);
    if (K > (1 << 20) || M * N >= (int64_t)1 << 37) return best; // (beyond the tiles' offsets, and 2^32 threads)
    const float before = parts ? 3.0f + (weights + (float)M * (float)K * 1e-6f) * 0.365f : 0.0f;
    if (odd && before + rows_us(false) < best.us) best.us = before + rows_us(false), best.padded = true;
    const float us64 = 3.0f + (odd ? before : 0.0f) + rounds(turns * ((N + 63) / 64), 256) * (0.8f + steps * (wide ? 0.51f : 0.4f));
    if (M > 64 && us64 < best.us) best.us = us64, best.kernel = F8Kernel::Rows64, best.padded = odd;
    const auto consider = [&](F8Kernel kernel, int64_t tile, float step) {
        const int64_t tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
        for (int splits = 1; splits <= 16; ++splits) {
            if (splits > 1 && (steps < 4.0f * (float)splits || tiles * (splits - 1) >= 512)) break;
            const float turn = (float)((tiles * splits + 255) / 256);
            float us = turn * ceilf(steps / (float)splits) * step;
            if (us < weights * (wide ? 0.25f : 0.215f)) us = weights * (wide ? 0.25f : 0.215f);
            us += 5.0f + before + (splits > 1 ? 4.0f + (float)splits * outputs * 1.6f : 0.0f);
            if (us < best.us) best.us = us, best.kernel = kernel, best.splits = splits, best.padded = parts;
        }
    };
    consider(F8Kernel::Tile128, 128, wide ? 0.97f : 0.62f);
    if (!wide) consider(F8Kernel::Tile256, 256, 1.85f);
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
    // (What is planned does not depend on addresses and pitches, and tiles need whole pieces: others, where K has them, go by 64 rows at a time.  4096 x
    // 4096 x 4096 67 us in tiles, 227 from rows that begin with a word, 460 from rows that do not.)
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
    if (p.kernel == F8Kernel::Rows) std::snprintf(name, sizeof(name), "rows%dx%s", M < 64 ? (int)((M + 15) / 16 * 16) : 64, wide_rows(M, N) && (p.padded || K % 4 == 0) ? "32" : "16");
    else if (p.kernel == F8Kernel::Rows64) return "rows64x64";
    else std::snprintf(name, sizeof(name), "tile%s/%d", p.kernel == F8Kernel::Tile256 ? "256x256" : "128x128", p.splits);
    return name;
}

} // extern "C"
