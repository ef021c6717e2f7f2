// Products of rows and weights in e4m3 with a scale per 128 of a row and per 128 x 128 weights (qnn_f8_matmul).
//
//   y[m][n] = bias[n] + sum_b xs[b][m] ws[n / 128][b] * sum_{k in b} x[m][k] w[n][k]
//
// The sum over a block comes from the matrix unit; one multiply-add in binary32 for each output and block joins it to the others.
#include "f8_matmul.h"

#include <cstdio>

namespace qnn {

// 16 bytes of a row, zeros behind its end
__device__ __forceinline__ w32x4 f8_load16(const uint8_t *row, int K, int k) { return k + 16 <= K ? load_any<w32x4>(row + k) : load_end(row, K, k); }

// One wave takes 16 * NT rows of the weights and 16 * MT rows of x, the waves of a workgroup share K in turns of 128 and join their
// sums in LDS in their order.  The product is formed transposed (weights are the left operand): a lane has one row of x and four consecutive
// outputs.  Both operands come straight into registers, DEPTH blocks ahead.
template <int MT, int NT, int WAVES, int DEPTH, bool NARROW> __global__ void __launch_bounds__(64 * WAVES) f8_rows_kernel(const F8Args a)
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
        float xs[MT], ws;
    };
    Step f[DEPTH];
    const auto load = [&](Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s.w[nt][0] = load_any<w32x4>(w_row[nt] + k), s.w[nt][1] = load_any<w32x4>(w_row[nt] + k + 64);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            s.x[mt][0] = load_any<w32x4>(x_row[mt] + k), s.x[mt][1] = load_any<w32x4>(x_row[mt] + k + 64);
            s.xs[mt] = x_scale[mt][b * a.ldxs];
        }
        s.ws = w_scale[b];
    };
    const auto load_last = [&](Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s.w[nt][0] = f8_load16(w_row[nt], a.K, k), s.w[nt][1] = f8_load16(w_row[nt], a.K, k + 64);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            s.x[mt][0] = f8_load16(x_row[mt], a.K, k), s.x[mt][1] = f8_load16(x_row[mt], a.K, k + 64);
            s.xs[mt] = x_scale[mt][b * a.ldxs];
        }
        s.ws = w_scale[b];
    };
    const auto compute = [&](const Step &s) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) fma4(acc[mt][nt], f8_products<NARROW>(s.w[nt], s.x[mt]), s.xs[mt] * s.ws);
    };
    const int mine = wave < whole ? (whole - wave + WAVES - 1) / WAVES : 0;
    if (whole < blocks && wave == whole % WAVES) { // the last, shorter block
        load_last(f[0], whole);
        compute(f[0]);
    }
    int i = 0;
    for (; i + DEPTH <= mine; i += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) load(f[d], wave + (i + d) * WAVES);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) compute(f[d]);
    }
    for (; i < mine; ++i) {
        load(f[0], wave + i * WAVES);
        compute(f[0]);
    }

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

template <int MT, int NT, int WAVES> static void launch_f8_rows(const F8Args &a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.N + 16 * NT - 1) / (16 * NT)), (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), block(64 * WAVES);
    if (a.type == QNN_F32) hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, 2, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((f8_rows_kernel<MT, NT, WAVES, 2, true>), grid, block, 0, s, a);
}

// By estimated time (us).
F8Plan f8_plan(int64_t M, int64_t N, int64_t K, int type)
{
    F8Plan best{F8Kernel::Rows, 1, 0.0f, false, 0, 0, 0};
    const float steps = (float)f8_blocks(K);
    if (M <= 64 || K > (1 << 20)) return best;
    const bool wide = type == QNN_F32, padded = K % 16 != 0;
    best.us = 1e30f;
    const auto consider = [&](F8Kernel kernel, int64_t tile, int64_t per_cu, float one, float full) {
        const int64_t tiles = ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
        for (int splits = 1; splits <= 16; ++splits) {
            if (splits > 1 && (steps / (float)splits < 4.0f || tiles * (splits - 1) >= 256 * per_cu)) break;
            const int64_t groups = tiles * splits;
            const float length = ceilf(steps / (float)splits) + 3.0f;
            const float us = (groups <= 256 ? one : full * (float)((groups + 256 * per_cu - 1) / (256 * per_cu))) * length +
                             (splits > 1 ? 3.0f + (float)splits * (float)(M * N) * 8.0f / 4e6f : 0.0f);
            if (us < best.us) best.us = us, best.kernel = kernel, best.splits = splits;
        }
    };
    consider(F8Kernel::Tile128, 128, 2, wide ? 1.2f : 0.9f, wide ? 1.9f : 1.2f);
    if (!wide) consider(F8Kernel::Tile256, 256, 1, 1.95f, 1.95f);
    best.padded = padded;
    const auto rounded = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    if (padded) best.x_bytes = rounded(M * f8_padded(K)), best.w_bytes = rounded(N * f8_padded(K));
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
    const bool pieces = ((uintptr_t)x | (uintptr_t)ldx | (uintptr_t)w | (uintptr_t)K) % 16 == 0 && ldx < (1 << 22);
    if (plan.kernel != F8Kernel::Rows && (plan.padded || pieces)) {
        uint8_t *const space = static_cast<uint8_t *>(workspace);
        if (plan.padded) {
            launch_f8_pad(a, space, space + plan.x_bytes, s);
            a.x = space, a.w = space + plan.x_bytes, a.ldx = f8_padded(K);
        }
        launch_f8_tiles(a, plan, plan.padded ? f8_padded(K) : K, reinterpret_cast<float *>(space + plan.x_bytes + plan.w_bytes), s);
    } else if (M <= 16) {
        launch_f8_rows<1, 1, 8>(a, s);
    } else {
        launch_f8_rows<4, 2, 4>(a, s);
    }
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
    if (p.kernel == F8Kernel::Rows) return M <= 16 ? "rows16x16/8" : "rows64x32/4";
    std::snprintf(name, sizeof(name), "tile%s/%d", p.kernel == F8Kernel::Tile256 ? "256x256" : "128x128", p.splits);
    return name;
}

} // extern "C"
