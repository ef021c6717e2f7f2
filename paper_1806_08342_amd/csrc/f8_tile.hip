// Products of e4m3 rows and weights for tens of rows and more: launches of the tiles (f8_tile.h), sums of parts of K, padded copies.
#include "f8_matmul.h"
#include "f8_tile.h"

namespace qnn {

// y = bias + the parts' sums in their order; 4 outputs per lane
__global__ void __launch_bounds__(256) f8_sum_kernel(const F8Args a, const float *parts, int splits)
{
    const int64_t n = (int64_t)a.M * a.N, at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int have = (int)min(n - at, (int64_t)4);
    if (have == 4)
        for (int s = 0; s < splits; ++s) {
            const f32x4 u = load_any<f32x4>(parts + s * n + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
    else
        for (int s = 0; s < splits; ++s)
            for (int e = 0; e < have; ++e) v[e] += parts[s * n + at + e];
    uint32_t m = (uint32_t)(at / a.N), c = (uint32_t)(at - (int64_t)m * a.N);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= have) break;
        store_out(a.y, m * a.ldy + c, a.type, v[e] + (a.bias ? load_out(a.bias, c, a.type) : 0.0f));
        if (++c == (uint32_t)a.N) c = 0, ++m;
    }
}

// rows of x and then of w as rows of whole 16-byte pieces, zeros behind their ends
__global__ void __launch_bounds__(128) f8_pad_kernel(const F8Args a, uint8_t *x, uint8_t *w, int pieces)
{
    const int row = blockIdx.x;
    const uint8_t *const from = row < a.M ? a.x + row * a.ldx : a.w + (int64_t)(row - a.M) * a.K;
    uint8_t *const to = row < a.M ? x + (int64_t)row * pieces * 16 : w + (int64_t)(row - a.M) * pieces * 16;
    for (int i = threadIdx.x; i < pieces; i += 128) *reinterpret_cast<w32x4 *>(to + i * 16) = load_end(from, a.K, i * 16);
}

template <int BM, int BN, int WM, int WN, int SETS, bool NARROW> static void launch_tiles(const F8Args &a, int splits, float *parts, hipStream_t s)
{
    F8TileArgs t{};
    t.a = a, t.parts = splits > 1 ? parts : nullptr, t.splits = splits;
    t.m_tiles = (a.M + BM - 1) / BM, t.n_tiles = (a.N + BN - 1) / BN;
    t.band = 8;
    t.per_xcd = (uint32_t)(((int64_t)t.m_tiles * t.n_tiles * splits + 7) / 8);
    hipLaunchKernelGGL((f8_tile_kernel<BM, BN, WM, WN, 2, 3, SETS, NARROW, 2>), dim3(8 * t.per_xcd), dim3(64 * WM * WN), 0, s, t);
}

void launch_f8_tiles(const F8Args &a, const F8Plan &plan, float *parts, hipStream_t s)
{
    if (a.type == QNN_F32) launch_tiles<128, 128, 2, 2, 1, false>(a, plan.splits, parts, s);
    else if (plan.kernel == F8Kernel::Tile256) launch_tiles<256, 256, 4, 2, 1, true>(a, plan.splits, parts, s);
    else launch_tiles<128, 128, 2, 2, 2, true>(a, plan.splits, parts, s);
    if (plan.splits > 1) {
        const int64_t n = (int64_t)a.M * a.N;
        hipLaunchKernelGGL(f8_sum_kernel, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, s, a, parts, plan.splits);
    }
}

void launch_f8_pad(const F8Args &a, uint8_t *x, uint8_t *w, hipStream_t s)
{
    hipLaunchKernelGGL(f8_pad_kernel, dim3((unsigned)(a.M + a.N)), dim3(128), 0, s, a, x, w, // (128 lanes: fewer than 2^32 threads)
                       (int)(f8_padded(a.K) / 16));
}

} // namespace qnn
