// Rows of 16-bit floats as e4m3 codes with a scale per 128 elements: plain, gated, and behind a root-mean-square norm
// (qnn_f8_quantize, qnn_f8_rmsnorm).
//
//   s = max(max|v| / 448, 2^-80), code = e4m3(v / s): the quotient is the correctly rounded one of binary32.  With r the rounded reciprocal of
//   s, q = v r and e = v - q s (one fma, exact), q + e r (one more) is that quotient.  (With the bound on s nothing underflows that a code shows.)
//   An infinity is cut off at the largest finite value's code, a NaN stays one.
//
// Bound by memory: each element is read once and written once, the row of a norm stays in registers.  A lane has 8 consecutive
// elements, sixteen lanes a block of 128.  16384 x 8192 with a residual 175 us (5.4 TB/s; a copy has 5.1), 9001 x 4100 to codes 23 us, gated 43;
// one row of 4096 2.9 us in a graph, a launch and one chain of loads.
#include "f8.h"

namespace qnn {

// over the 16 lanes of a block
template <class F> __device__ __forceinline__ float over16(float v, F f)
{
    const auto turned = [](float u, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, u), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = f(v, turned(v, std::integral_constant<int, 0x128>())); // row_ror:8 and so on
    v = f(v, turned(v, std::integral_constant<int, 0x124>()));
    v = f(v, turned(v, std::integral_constant<int, 0x122>()));
    return f(v, turned(v, std::integral_constant<int, 0x121>()));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

// the codes of a lane's 8 values, and of its block the scale and whether there is an infinity in it
__device__ __forceinline__ w32x2 encode8(const float (&v)[8], float &scale, bool &infinite)
{
    float peak = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) peak = fmaxf(peak, fabsf(v[i])); // (fmaxf passes over NaN)
    peak = over16(peak, larger);
    infinite = peak == INFINITY;
    if (infinite) {
        peak = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) peak = fmaxf(peak, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.0f);
        peak = over16(peak, larger);
    }
    scale = fmaxf(peak / kF8Largest, kF8LeastScale);
    const float r = 1.0f / scale, most = fmaxf(peak, kF8Largest * kF8LeastScale);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float c = __builtin_elementwise_minimum(__builtin_elementwise_maximum(v[i], -most), most); // (a NaN stays)
        const float t = c * r;
        q[i] = copysignf(fmaf(fmaf(-t, scale, c), r, t), c); // (that of -0 would be +0)
    }
    w32x2 codes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int low = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
        codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], low, true);
    }
    return codes;
}

// 8 elements from k on, zeros behind the row's end, in two steps: loads of several, which no branch holds up, and then, where the row ends within or before
// them, what was loaded before its end moved down (777 x 5003 with a residual 11.4 us in one step with a branch, 11.0 so, 20 x 5003 4.4 and 4.1).  WHOLE: K is a
// multiple of 8, and the first step is all.
template <bool WHOLE> __device__ __forceinline__ w32x4 load8(const uint16_t *row, int K, int k)
{
    if constexpr (WHOLE) {
        const w32x4 v = load_any<w32x4>(row + min(k, K - 8));
        const uint32_t there = k < K ? ~0u : 0u;
        return v & w32x4{there, there, there, there};
    }
    return K >= 8 ? load_any<w32x4>(row + min(k, K - 8)) : load_end(reinterpret_cast<const uint8_t *>(row), 2 * K, 2 * k);
}
template <bool WHOLE> __device__ __forceinline__ void settle8(w32x4 &v, int K, int k)
{
    if (WHOLE || K < 8 || k + 8 <= K) return;
    const int drop = min(k + 8 - K, 8);
    uint32_t u[5] = {v[0], v[1], v[2], v[3], 0u};
    if (drop & 2) u[0] = u[1], u[1] = u[2], u[2] = u[3], u[3] = 0u;
    if (drop & 4) u[0] = u[2], u[1] = u[3], u[2] = 0u, u[3] = 0u;
    if (drop & 8) u[0] = u[1] = u[2] = u[3] = 0u;
    const uint32_t by = 2 * (drop & 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(u[i + 1], u[i], by);
}
template <class T> __device__ __forceinline__ void widen8(const w32x4 w, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = T::widen((uint16_t)(w[i >> 1] >> (i & 1) * 16));
}
template <class T> __device__ __forceinline__ w32x4 narrow8(const float (&v)[8])
{
    return w32x4{narrow2<T>(v[0], v[1]), narrow2<T>(v[2], v[3]), narrow2<T>(v[4], v[5]), narrow2<T>(v[6], v[7])};
}
template <bool WHOLE> __device__ __forceinline__ void store8(uint16_t *row, int K, int k, const w32x4 v) // k < K
{
    if (WHOLE || k + 8 <= K) {
        store_any(row + k, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (k + i < K) row[k + i] = (uint16_t)(v[i >> 1] >> (i & 1) * 16);
}
template <bool WHOLE> __device__ __forceinline__ void store_codes(uint8_t *row, int K, int k, const w32x2 c) // k < K
{
    if (WHOLE || k + 8 <= K) {
        store_any(row + k, c);
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (k + i < K) row[k + i] = (uint8_t)(c[i >> 2] >> (i & 3) * 8);
}

// Consecutive rows' scales are consecutive in memory: each XCD takes a stretch of rows of its own, so that its L2 joins them.
__device__ __forceinline__ uint32_t of_xcd(uint32_t id, uint32_t groups) { return id % 8 * groups + id / 8; }

struct F8RowArgs {
    const uint16_t *x, *residual, *weight;
    uint16_t *total, *y;
    uint8_t *codes;
    float *scales;
    int64_t ldx, ldr, ldt, ldc, lds;
    int32_t M, K;
    float eps;
    uint32_t blocks, units, groups; // blocks of a row, of all rows; workgroups (or rows) of an XCD
    uint32_t magic, shift;          // of the division by blocks
};

// v / (1 + exp(-v)) by a reciprocal (off by 2^-23), but where that would leave the normal numbers: 9001 x 4100 gated 43 us, with divisions 49
__device__ __forceinline__ float silu(float v)
{
    const float q = 1.0f + expf(-v);
    return q < 0x1p100f ? v * __builtin_amdgcn_rcpf(q) : v / q;
}

// 16 lanes per block; kSlab blocks of the grid's first dimension.  (Several blocks after each other, their loads ahead, took longer at all sizes:
// with four 24 x 14336 gated 4.9 us for 2.6, 4096 x 4096 13.1 for 9.8, 9001 x 4100 24.2 for 24.3.)
constexpr uint32_t kSlab = 1u << 24;
template <class T, bool GATED, bool WHOLE> __global__ void __launch_bounds__(256) f8_quantize_kernel(const F8RowArgs a)
{
    const uint32_t unit = blockIdx.y * kSlab + of_xcd(blockIdx.x, a.groups) * 16 + (threadIdx.x >> 4);
    if (unit >= a.units) return; // (whole blocks)
    const int lane = threadIdx.x & 15;
    const uint32_t row = a.magic ? __umulhi(unit, a.magic) >> a.shift : unit, block = unit - row * a.blocks;
    const uint16_t *const x = a.x + (int64_t)row * a.ldx;
    const int k = (int)block * kF8Block + lane * 8;
    float v[8], scale;
    w32x4 in = load8<WHOLE>(x, a.K, k);
    if constexpr (GATED) {
        w32x4 in_up = load8<WHOLE>(x + a.K, a.K, k);
        settle8<WHOLE>(in, a.K, k), settle8<WHOLE>(in_up, a.K, k);
        float up[8];
        widen8<T>(in, v), widen8<T>(in_up, up);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = silu(v[e]) * up[e];
    } else {
        settle8<WHOLE>(in, a.K, k);
        widen8<T>(in, v);
    }
    bool infinite;
    const w32x2 codes = encode8(v, scale, infinite);
    if (k < a.K) store_codes<WHOLE>(a.codes + (int64_t)row * a.ldc, a.K, k, codes);
    if (lane == 0) a.scales[(int64_t)block * a.lds + row] = scale;
}

// One row per workgroup of up to 16 waves (4 rows per workgroup where one wave does).  CHUNKS: pieces of 8 elements that a lane keeps of a row; 0: rows
// that do not fit the registers are read a second time.
template <class T, int CHUNKS, bool SINGLE, bool WHOLE> __global__ void __launch_bounds__(SINGLE ? 256 : 1024) f8_rmsnorm_kernel(const F8RowArgs a)
{
    constexpr int ROWS = SINGLE ? 4 : 1, KEPT = CHUNKS ? CHUNKS : 1;
    __shared__ float s_part[2][16];
    const int lanes = SINGLE ? 64 : blockDim.x, tid = SINGLE ? threadIdx.x & 63 : threadIdx.x, waves = lanes >> 6;
    const uint32_t row = of_xcd(blockIdx.x, a.groups) * ROWS + (SINGLE ? threadIdx.x >> 6 : 0);
    if (row >= (uint32_t)a.M) return; // (whole waves, and where waves share a row the whole workgroup)
    const uint16_t *const x = a.x + row * a.ldx;
    const uint16_t *const residual = a.residual ? a.residual + row * a.ldr : nullptr;
    uint16_t *const total = a.total + row * a.ldt;
    const int turns = CHUNKS ? CHUNKS : (a.K + 8 * lanes - 1) / (8 * lanes);
    w32x4 h[KEPT], r[KEPT];

    const auto load = [&](int i, int k) {
        h[i] = load8<WHOLE>(x, a.K, k);
        if (residual) r[i] = load8<WHOLE>(residual, a.K, k);
    };
    const auto add = [&](int i, int k) {
        settle8<WHOLE>(h[i], a.K, k);
        if (!residual) return;
        settle8<WHOLE>(r[i], a.K, k);
        float u[8], v[8];
        widen8<T>(h[i], u), widen8<T>(r[i], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] += v[e];
        h[i] = narrow8<T>(u);
        if (k < a.K) store8<WHOLE>(total, a.K, k, h[i]);
    };
    // over the row
    int turn = 0;
    const auto over_row = [&](float v, auto f) {
        v = over16(v, f);
        v = f(v, __shfl_xor(v, 16));
        v = f(v, __shfl_xor(v, 32));
        if constexpr (!SINGLE) {
            turn ^= 1;
            if ((tid & 63) == 0) s_part[turn][tid >> 6] = v;
            __syncthreads();
            v = s_part[turn][0];
            for (int i = 1; i < waves; ++i) v = f(v, s_part[turn][i]);
        }
        return v;
    };
    // f(elements, k) for all pieces of the row as the norm sees it
    const auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < (CHUNKS ? CHUNKS : 0); ++i) {
            float v[8];
            widen8<T>(h[i], v);
            f(v, (i * lanes + tid) * 8);
        }
        if constexpr (CHUNKS == 0)
            for (int i = 0; i < turns; ++i) {
                const int k = (i * lanes + tid) * 8;
                float v[8];
                w32x4 in = load8<WHOLE>(residual ? total : x, a.K, k);
                settle8<WHOLE>(in, a.K, k);
                widen8<T>(in, v);
                f(v, k);
            }
    };

    if constexpr (CHUNKS > 0) {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) load(i, (i * lanes + tid) * 8);
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) add(i, (i * lanes + tid) * 8);
    } else if (residual) {
        for (int i = 0; i < turns; ++i) load(0, (i * lanes + tid) * 8), add(0, (i * lanes + tid) * 8);
    }
    const auto plus = [](float p, float q) { return p + q; };
    const float per = 1.0f / (float)a.K;
    const auto mean_square = [&](float c) {
        float sum = 0.0f;
        each([&](float (&v)[8], int) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(v[e] * c, v[e] * c, sum);
        });
        return over_row(sum, plus) * per;
    };
    float unit = 1.0f, mean = mean_square(1.0f), eps = a.eps;
    if (!(mean >= 0x1p-90f && mean <= 0x1p100f)) { // squares at the ends of binary32's range: once more in units of 2^e
        float peak = 0.0f;
        each([&](float (&v)[8], int) {
#pragma unroll
            for (int e = 0; e < 8; ++e) peak = fmaxf(peak, fabsf(v[e]));
        });
        peak = over_row(peak, larger);
        if (peak > 0.0f && peak < INFINITY) {
            unit = ldexpf(1.0f, -max(ilogbf(fmaxf(peak, sqrtf(eps))), -120));
            mean = mean_square(unit), eps = eps * unit * unit;
        }
    }
    const float by = mean + eps > 0.0f ? 1.0f / sqrtf(mean + eps) : mean + eps == 0.0f ? 0.0f : mean; // (zeros give zeros, NaN a NaN)
    // The codes do not depend on what a row is divided by: they are taken from its products with the weights, which are exact, so that only the scale and the
    // quotient are rounded, and the scale is multiplied afterwards.  (Of rows of 4096 bfloat16 33 % have a code that is another one than that
    // of 64 bits, where the products lie exactly between two; from v 42 %.)  Not so where the products, the factor or the scale come near the ends of the range.
    // Where v itself is asked for, codes are v's too: both ways in one took 777 x 5003 from 8.4 us to 8.9.
    const bool regular = !a.y && unit == 1.0f && by >= 0x1p-60f && by <= 0x1p60f;
    each([&](float (&v)[8], int k) {
        float g[8], scale;
        if (a.weight) {
            w32x4 weight = load8<WHOLE>(a.weight, a.K, k);
            settle8<WHOLE>(weight, a.K, k);
            widen8<T>(weight, g);
        }
        w32x2 codes;
        bool infinite, exact = false;
        if (regular) {
            float u[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = a.weight ? v[e] * g[e] : v[e];
            codes = encode8(u, scale, infinite);
            exact = !infinite && scale >= 0x1p-60f && scale <= 0x1p60f && scale * by >= kF8LeastScale && scale * by <= 0x1p118f;
            scale *= by;
        }
        if (!exact) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = a.weight ? v[e] * unit * by * g[e] : v[e] * unit * by;
            codes = encode8(v, scale, infinite);
        }
        if (k >= a.K) return;
        store_codes<WHOLE>(a.codes + row * a.ldc, a.K, k, codes);
        if (a.y) store8<WHOLE>(a.y + (int64_t)row * a.K, a.K, k, narrow8<T>(v));
        if ((threadIdx.x & 15) == 0) a.scales[(int64_t)(k / kF8Block) * a.lds + row] = scale;
    });
}

template <class T, int CHUNKS, bool SINGLE = false> static void launch_rmsnorm(F8RowArgs a, hipStream_t s)
{
    const uint32_t rows = SINGLE ? 4 : 1, need = (uint32_t)((a.M + rows - 1) / rows);
    a.groups = (need + 7) / 8;
    const int each = 512 * (CHUNKS ? CHUNKS : 4), waves = SINGLE ? 4 : CHUNKS ? (a.K + each - 1) / each : 16;
    if (a.K % 8 == 0) hipLaunchKernelGGL((f8_rmsnorm_kernel<T, CHUNKS, SINGLE, true>), dim3(8 * a.groups), dim3(64 * waves), 0, s, a);
    else hipLaunchKernelGGL((f8_rmsnorm_kernel<T, CHUNKS, SINGLE, false>), dim3(8 * a.groups), dim3(64 * waves), 0, s, a);
}

// Few rows: as many waves as they can use, up to 16.  Many: fewer with more each, for fewer waits on the others (between the two nothing jumps: 512 x
// 5000 4.2 us with a wave for every 512 elements, 516 rows 4.4 with one for 1024; 512 x 8192 6.1, 516 rows 6.7 with one for 2048).  With a residual, whose
// stores lie between the loads and the sum, more rows are few: 2048 x 4096 13.1 and 15.3, 2048 x 8192 27.0 and 29.7, but 777 x 5003 11.8 and 11.4.
template <class T> static void run_rmsnorm(const F8RowArgs &a, hipStream_t s)
{
    const bool few = a.M <= 512;
    if (a.K <= 512) launch_rmsnorm<T, 1, true>(a, s);
    else if ((few || (a.residual && a.K % 8 == 0 && a.M <= 4096)) && a.K <= 8192) launch_rmsnorm<T, 1>(a, s);
    else if (a.K <= 1024) launch_rmsnorm<T, 2, true>(a, s);
    else if (a.K <= (few ? 16384 : 6144)) launch_rmsnorm<T, 2>(a, s);
    else if (a.K <= 32768) launch_rmsnorm<T, 4>(a, s);
    else launch_rmsnorm<T, 0>(a, s);
}

template <class T, bool GATED> static void launch_quantize(F8RowArgs a, hipStream_t s)
{
    a.groups = ((a.units < kSlab ? a.units : kSlab) + 127) / 128;
    const dim3 grid(8 * a.groups, (a.units + kSlab - 1) / kSlab);
    if (a.K % 8 == 0) hipLaunchKernelGGL((f8_quantize_kernel<T, GATED, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((f8_quantize_kernel<T, GATED, false>), grid, dim3(256), 0, s, a);
}

} // namespace qnn

using namespace qnn;

extern "C" {

static bool bad_row_sizes(int64_t M, int64_t K) { return M < 0 || K <= 0 || M > (1 << 20) || K > (1 << 24) || M * f8_blocks(K) >= (int64_t)1 << 30; }

qnn_status qnn_f8_quantize(const void *x, int64_t ldx, int64_t M, int64_t K, int gated, int type, uint8_t *codes, int64_t ldc, float *scales,
                           int64_t lds, void *stream)
{
    if (bad_row_sizes(M, K) || bad_half_type(type)) return QNN_EINVAL;
    if (M == 0) return QNN_OK;
    if (!x || !codes || !scales || ldx < (gated ? 2 * K : K) || ldc < K || lds < M) return QNN_EINVAL;
    F8RowArgs a{};
    a.x = static_cast<const uint16_t *>(x), a.ldx = ldx, a.codes = codes, a.ldc = ldc, a.scales = scales, a.lds = lds;
    a.M = (int32_t)M, a.K = (int32_t)K, a.blocks = (uint32_t)f8_blocks(K), a.units = (uint32_t)(M * a.blocks);
    fast_division(a.blocks, a.magic, a.shift);
    hipStream_t s = as_stream(stream);
    if (type == QNN_BF16) gated ? launch_quantize<Bf16, true>(a, s) : launch_quantize<Bf16, false>(a, s);
    else gated ? launch_quantize<F16, true>(a, s) : launch_quantize<F16, false>(a, s);
    return launch_status(hipGetLastError());
}

qnn_status qnn_f8_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, float eps, int64_t M, int64_t K,
                          int type, void *total, int64_t ldt, void *y, uint8_t *codes, int64_t ldc, float *scales, int64_t lds, void *stream)
{
    if (bad_row_sizes(M, K) || bad_half_type(type) || !(eps >= 0.0f) || !(eps <= 0x1p100f)) return QNN_EINVAL;
    if (M == 0) return QNN_OK;
    if (!x || !codes || !scales || ldx < K || ldc < K || lds < M) return QNN_EINVAL;
    if (residual && (!total || ldr < K || ldt < K)) return QNN_EINVAL;
    F8RowArgs a{};
    a.x = static_cast<const uint16_t *>(x), a.ldx = ldx, a.residual = static_cast<const uint16_t *>(residual), a.ldr = ldr;
    a.weight = static_cast<const uint16_t *>(weight), a.total = static_cast<uint16_t *>(total), a.ldt = ldt, a.y = static_cast<uint16_t *>(y);
    a.codes = codes, a.ldc = ldc, a.scales = scales, a.lds = lds, a.M = (int32_t)M, a.K = (int32_t)K, a.eps = eps;
    if (type == QNN_BF16) run_rmsnorm<Bf16>(a, as_stream(stream));
    else run_rmsnorm<F16>(a, as_stream(stream));
    return launch_status(hipGetLastError());
}

} // extern "C"
