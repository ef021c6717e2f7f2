// Writing and reading the paged cache of 8-bit codes (qnn_kv_append, qnn_kv_gather).
//
//   s = max(s_old, max|x| / 127) over a page's new tokens,  codes held: round(c * (s_old / s)),  new ones: round(x / s)
//
// Bound by memory where there is much to move: 18.9 k tokens, 8 heads of 128, append 26 us (4.5 TB/s), gather 20 us (5.8).  Appending
// reads each element once: a page's part of a head stays in registers between its largest value and its codes.  One token for each of
// 64 requests takes 7 us for either, a launch and a chain of four loads (rows and lengths, the page's number, elements and scale, and
// where a scale grows the codes held).
#include "kv_attention.h"

namespace qnn {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

struct CacheArgs {
    qnn_kv_cache cache;
    const uint16_t *k, *v;
    int64_t k_token, k_head, v_token, v_head;
    uint16_t *k_out, *v_out;
    const int32_t *cu, *start, *table;
    int64_t table_width, tokens;
    int32_t requests;
};

// Workgroup `item` works on the item-th page that the call touches.  A request whose rows begin at cu and that has n of them
// touches at most n / block + 2 pages (rounded down), so that pages first / block + 2 r ... of request r are its own; the
// request is found by bisection with 64 lanes at a time, whose last step also brings what is needed of it.  (Rows are below 2^30, tokens below 2^31:
// 32 bits without a sign hold their sums, and their divisions take a fraction of 64 bits' time.)
__device__ __forceinline__ uint32_t row_of(const CacheArgs &a, int r) { return (uint32_t)min(max(a.cu[r], 0), (int)a.tokens); }

struct Piece {
    int64_t row;  // of k and v: the first new token's
    int64_t page; // -1: none
    int lo, hi;   // tokens of the page that are new, [lo, hi)
};
__device__ __forceinline__ Piece piece_of_item(const CacheArgs &a, uint32_t item)
{
    const int lane = threadIdx.x & 63;
    const uint32_t block = a.cache.block;
    int low = 0, n = a.requests; // in [low, low + n)
    while (n > 64) {
        const int step = (n + 63) / 64, r = low + min(lane * step, n - 1);
        const uint64_t reached = __ballot(lane * step < n && row_of(a, r) / block + 2u * r <= item);
        const int k = max(__popcll(reached) - 1, 0);
        low += k * step, n = min(step, n - k * step);
    }
    const int mine = low + min(lane, n - 1);
    const uint32_t from = row_of(a, mine), upto = row_of(a, mine + 1), held = max(a.start[mine], 0);
    const uint32_t base = from / block + 2u * mine;
    const int k = max(__popcll(__ballot(lane < n && base <= item)) - 1, 0);
    const auto of = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, k); };
    const uint32_t c0 = of(from), c1 = of(upto), at = of(held);
    const uint32_t j = at / block + (item - of(base)); // page of the request
    const uint32_t t0 = max(at, j * block), t1 = min(at + (max(c1, c0) - c0), (j + 1) * block);
    Piece p{(int64_t)c0 + (t0 - at), -1, (int)(t0 - j * block), (int)(t1 - j * block)};
    if (t1 <= t0) p.hi = p.lo;
    else if (j < a.table_width) {
        const int32_t page = a.table[(int64_t)(low + k) * a.table_width + j];
        if ((uint32_t)page < (uint64_t)a.cache.pages) p.page = page;
    }
    return p;
}

// round() with ties away from zero, as a code: 0.5 less its last bit added, then cut off.
__device__ __forceinline__ int rounded(float q) { return (int)(q + copysignf(0.49999997f, q)); }
__device__ __forceinline__ int code_of(float q)
{
    return rounded(__builtin_amdgcn_fmed3f(q, -127.0f, 127.0f)); // (infinities: the ends)
}
// The code of x at scale s is that of x / s rounded to binary32 once, which x * hi + x * lo (rounded once, but for a product that is
// 2^-24 of it) is within 3 * 2^-48 of before its rounding, where hi = 1 / s rounded and lo what it lacks.  The two codes differ only if the midpoint
// below some k + 1/2 lies between, and that close to x / s: with s = B * 2^.., 2^23 <= B < 2^24, and x of 11 bits at
// most, B would have to be within 6 of a multiple of 2^17 and not the multiple.  Scales within 8, and those whose reciprocals come near the
// ends of binary32's range, are divided by.
__device__ __forceinline__ bool divide_by(float s)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, s);
    return !(s > 0x1p-60f && s < 0x1p60f) || (((b + 8) & 0x1ffffu) <= 16 && (b & 0x1ffffu) != 0);
}
__device__ __forceinline__ uint32_t four_codes(int a, int b, int c, int d)
{
    const uint32_t lo = __builtin_amdgcn_perm((uint32_t)b, (uint32_t)a, 0x0c0c0400u), hi = __builtin_amdgcn_perm((uint32_t)d, (uint32_t)c, 0x04000c0cu);
    return lo | hi;
}
// the codes of a dword in another scale
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float ratio)
{
    int c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = code_of((float)(int8_t)(w >> 8 * i) * ratio);
    return four_codes(c[0], c[1], c[2], c[3]);
}

// WAVES waves take keys or values of one head in one page; blockIdx.y (times four and the wave's number if WAVES is 1) counts heads and, in its
// lowest bit, values.  Elements are loaded 8 at a time and stay in registers between the largest and the codes where they fit (64 x 128 in four
// waves do).
// Keys: piece i is row i / (D / 8), channels 8 * (i % (D / 8)).  Values, which are stored with consecutive tokens of a channel
// together: unit i is 4 tokens (aligned in the page) by 8 channels, turned in registers.
template <class T, int D, int WAVES> __global__ void __launch_bounds__(256) append_kernel(const CacheArgs a)
{
    constexpr int DG = D / 8, LANES = 64 * WAVES, HELD = 4; // HELD: pieces of 8 per lane
    const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x, hk = WAVES == 1 ? blockIdx.y * 4 + (threadIdx.x >> 6) : blockIdx.y, h = hk >> 1;
    const bool is_v = hk & 1;
    if (h >= a.cache.heads) return;
    const Piece p = piece_of_item(a, blockIdx.x);
    if (p.hi <= p.lo) return;
    const int block = a.cache.block;
    const int64_t token = is_v ? a.v_token : a.k_token;
    const uint16_t *const x = (is_v ? a.v : a.k) + p.row * token + (int64_t)h * (is_v ? a.v_head : a.k_head);
    const int groups0 = p.lo >> 2, groups = ((p.hi + 3) >> 2) - groups0; // of 4 tokens
    const int n = is_v ? groups * DG * 4 : (p.hi - p.lo) * DG, batches = (n + LANES * HELD - 1) / (LANES * HELD);

    if (p.page < 0) return;
    const int64_t slot = p.page * a.cache.heads + h;
    int8_t *const codes = (is_v ? a.cache.v_codes : a.cache.k_codes) + slot * block * D;
    float *const scale = (is_v ? a.cache.v_scales : a.cache.k_scales) + slot;
    const float before = p.lo > 0 ? *scale : 0.0f; // (on its way with the elements)

    w32x4 held[HELD];
    // piece k of a lane's 16 in a batch: keys by 64, values four of one unit after the other
    const auto past = [&](int batch, int k) { return is_v ? batch * LANES >= groups * DG : (batch * HELD + k) * LANES >= n; };
    const auto load = [&](int batch) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (past(batch, k)) break;
            const int i = is_v ? batch * LANES + lane : (batch * HELD + k) * LANES + lane;
            const int t = is_v ? (groups0 + i % groups) * 4 + k % 4 - p.lo : i / DG, d = is_v ? i / groups : i % DG;
            held[k] = w32x4{0u, 0u, 0u, 0u};
            if (is_v ? d < DG && t >= 0 && t < p.hi - p.lo : i < n) held[k] = load_any<w32x4>(x + t * token + d * 8);
        }
    };
    u16x2 peaks = {0, 0}; // of the absolute values' patterns, which are in the values' order
    for (int batch = 0; batch < batches; ++batch) {
        load(batch);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (past(batch, k)) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) peaks = __builtin_elementwise_max(peaks, __builtin_bit_cast(u16x2, held[k][e] & 0x7fff7fffu));
        }
    }
    uint32_t pattern = max(peaks[0], peaks[1]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) pattern = max(pattern, (uint32_t)__shfl_xor((int)pattern, d));
    __shared__ uint32_t s_most[WAVES];
    if constexpr (WAVES > 1) {
        if ((lane & 63) == 0) s_most[lane >> 6] = pattern;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) pattern = max(pattern, s_most[w]);
    }
    float peak = T::widen((uint16_t)pattern);
    const bool infinite = !(peak < INFINITY); // or NaN
    if (infinite) { // (rare: once more, by element)
        peak = 0.0f;
        for (int i = lane; i < (p.hi - p.lo) * D; i += LANES) {
            const float v = fabsf(T::widen(x[(i / D) * token + i % D]));
            peak = v < INFINITY ? fmaxf(peak, v) : peak;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
        if constexpr (WAVES > 1) {
            __syncthreads(); // (the patterns are read)
            if ((lane & 63) == 0) s_most[lane >> 6] = __builtin_bit_cast(uint32_t, peak);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) peak = fmaxf(peak, __builtin_bit_cast(float, s_most[w]));
        }
    }
    const float after = fmaxf(before, __fdiv_rn(peak, 127.0f)), by = after > 0.0f ? after : 1.0f;
    if (lane == 0) *scale = after;
    if (after > before && p.lo > 0) { // what is held, in the new scale
        const float ratio = __fdiv_rn(before, by);
        if (!is_v) {
            uint32_t *const w = reinterpret_cast<uint32_t *>(codes);
            for (int i = lane; i < p.lo * (D / 4); i += LANES) w[i] = rescaled(w[i], ratio);
        } else {
            for (int i = lane; i < groups0 * D; i += LANES) {
                uint32_t *const w = reinterpret_cast<uint32_t *>(codes + (i / groups0) * block) + i % groups0;
                *w = rescaled(*w, ratio);
            }
            const int rest = p.lo & 3; // of a group that new tokens share
            for (int i = lane; i < rest * D; i += LANES) {
                int8_t *const c = codes + (i / rest) * block + 4 * groups0 + i % rest;
                *c = (int8_t)code_of((float)*c * ratio);
            }
        }
    }
    if (infinite || divide_by(by)) {
        for (int i = lane; i < (p.hi - p.lo) * D; i += LANES) {
            const int t = i / D, d = i % D;
            const float v = T::widen(x[t * token + d]);
            codes[is_v ? d * block + p.lo + t : (p.lo + t) * D + d] = (int8_t)(v == v && after > 0.0f ? code_of(__fdiv_rn(v, by)) : 0); // (scale 0: nothing but infinities and zeros)
        }
        return;
    }
    const float hi = __fdiv_rn(1.0f, by), lo = hi * fmaf(-by, hi, 1.0f);
    for (int batch = 0; batch < batches; ++batch) {
        if (batches > 1) load(batch);
        int c[HELD][8];
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (past(batch, k)) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = T::widen((uint16_t)(held[k][e >> 1] >> (e & 1) * 16));
                c[k][e] = rounded(fmaf(v, hi, v * lo)); // (no value is over 127 steps of its own page's scale)
            }
            const int i = (batch * HELD + k) * LANES + lane;
            if (!is_v && i < n)
                *reinterpret_cast<w32x2 *>(codes + (int64_t)p.lo * D + i * 8) =
                    w32x2{four_codes(c[k][0], c[k][1], c[k][2], c[k][3]), four_codes(c[k][4], c[k][5], c[k][6], c[k][7])};
        }
        if (!is_v) continue;
        const int i = batch * LANES + lane, t = (groups0 + i % groups) * 4, d = i / groups;
        if (d >= DG) continue;
        int8_t *const to = codes + d * 8 * block + t;
        if (t >= p.lo && t + 4 <= p.hi) {
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<uint32_t *>(to + e * block) = four_codes(c[0][e], c[1][e], c[2][e], c[3][e]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t + j >= p.lo && t + j < p.hi)
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[e * block + j] = (int8_t)c[j][e];
        }
    }
}

// Each workgroup: keys or values (blockIdx.y odd) of one head in one page; 8 codes, or 4 tokens by 8 channels, per lane and step.
template <class T, int D> __global__ void __launch_bounds__(256) gather_kernel(const CacheArgs a)
{
    constexpr int DG = D / 8;
    const int tid = threadIdx.x, h = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const int heads = a.cache.heads;
    const Piece p = piece_of_item(a, blockIdx.x);
    if (p.hi <= p.lo) return;
    const int block = a.cache.block;
    uint16_t *const out = (is_v ? a.v_out : a.k_out) + (p.row * heads + h) * D;
    const bool none = p.page < 0; // zeros
    const int64_t slot = (none ? 0 : p.page) * heads + h;
    const float scale = none ? 0.0f : (is_v ? a.cache.v_scales : a.cache.k_scales)[slot];
    const int8_t *const codes = (is_v ? a.cache.v_codes : a.cache.k_codes) + slot * block * D;
    const auto value = [&](uint32_t w, int i) { return none ? 0.0f : (float)(int8_t)(w >> 8 * i) * scale; };
    if (!is_v) {
        const int n = (p.hi - p.lo) * DG;
#pragma unroll 4
        for (int i = tid; i < n; i += 256) {
            const w32x2 c = none ? w32x2{0u, 0u} : *reinterpret_cast<const w32x2 *>(codes + (int64_t)p.lo * D + i * 8);
            w32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = narrow2<T>(value(c[e >> 1], 2 * (e & 1)), value(c[e >> 1], 2 * (e & 1) + 1));
            *reinterpret_cast<w32x4 *>(out + (int64_t)(i / DG) * heads * D + i % DG * 8) = v;
        }
    } else {
        const int groups0 = p.lo >> 2, groups = ((p.hi + 3) >> 2) - groups0;
        for (int i = tid; i < groups * DG; i += 256) {
            const int t = (groups0 + i % groups) * 4, d = i / groups;
            uint32_t c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = none ? 0u : *reinterpret_cast<const uint32_t *>(codes + (d * 8 + e) * block + t);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (t + j < p.lo || t + j >= p.hi) continue;
                w32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = narrow2<T>(value(c[2 * e], j), value(c[2 * e + 1], j));
                *reinterpret_cast<w32x4 *>(out + (int64_t)(t + j - p.lo) * heads * D + d * 8) = v;
            }
        }
    }
}

template <class T, bool GATHER> static void launch_pieces(const CacheArgs &a, hipStream_t s)
{
    // from 8 new tokens per request on average a page's part is four waves' work
    const bool alone = a.tokens < 8 * (int64_t)a.requests;
    const dim3 grid((unsigned)(a.tokens / a.cache.block + 2 * (int64_t)a.requests), (unsigned)(GATHER || !alone ? 2 * a.cache.heads : (2 * a.cache.heads + 3) / 4));
    const auto with = [&](auto dim) {
        if constexpr (GATHER) hipLaunchKernelGGL((gather_kernel<T, dim>), grid, dim3(256), 0, s, a);
        else if (alone) hipLaunchKernelGGL((append_kernel<T, dim, 1>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((append_kernel<T, dim, 4>), grid, dim3(256), 0, s, a);
    };
    switch (a.cache.dim) {
    case 64: with(std::integral_constant<int, 64>{}); break;
    case 96: with(std::integral_constant<int, 96>{}); break;
    case 128: with(std::integral_constant<int, 128>{}); break;
    case 192: with(std::integral_constant<int, 192>{}); break;
    default: with(std::integral_constant<int, 256>{}); break;
    }
}

static bool bad_cache_call(const qnn_kv_cache *cache, int64_t table_width, int64_t requests, int64_t tokens, int type)
{
    return bad_cache(cache) || bad_half_type(type) || table_width < 0 || table_width > INT32_MAX / cache->block || requests < 0 || requests > (1 << 20) ||
           tokens < 0 || tokens > INT32_MAX / 2 || tokens / cache->block + 2 * requests >= (1 << 24); // (a launch has fewer than 2^32 threads along x)
}
} // namespace qnn

using namespace qnn;

extern "C" {

qnn_status qnn_kv_append(const qnn_kv_cache *cache, const void *k, int64_t k_token_pitch, int64_t k_head_pitch, const void *v, int64_t v_token_pitch,
                         int64_t v_head_pitch, int type, const int32_t *cu, const int32_t *start, const int32_t *table, int64_t table_width,
                         int64_t requests, int64_t tokens, void *stream)
{
    if (bad_cache_call(cache, table_width, requests, tokens, type)) return QNN_EINVAL;
    if (requests == 0 || tokens == 0) return QNN_OK;
    if (!k || !v || !cu || !start || (table_width > 0 && !table) || bad_cache_arrays(cache)) return QNN_EINVAL;
    const CacheArgs a{*cache, static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), k_token_pitch, k_head_pitch, v_token_pitch,
                      v_head_pitch, nullptr, nullptr, cu, start, table, table_width, tokens, (int32_t)requests};
    if (type == QNN_BF16) launch_pieces<Bf16, false>(a, as_stream(stream));
    else launch_pieces<F16, false>(a, as_stream(stream));
    return launch_status(hipGetLastError());
}

qnn_status qnn_kv_gather(const qnn_kv_cache *cache, const int32_t *cu, const int32_t *first, const int32_t *table, int64_t table_width,
                         int64_t requests, int64_t tokens, int type, void *k, void *v, void *stream)
{
    if (bad_cache_call(cache, table_width, requests, tokens, type)) return QNN_EINVAL;
    if (requests == 0 || tokens == 0) return QNN_OK;
    if (!k || !v || !cu || !first || (table_width > 0 && !table) || bad_cache_arrays(cache) || (((uintptr_t)k | (uintptr_t)v) & 15) != 0) return QNN_EINVAL;
    const CacheArgs a{*cache, nullptr, nullptr, 0, 0, 0, 0, static_cast<uint16_t *>(k), static_cast<uint16_t *>(v), cu, first, table, table_width,
                      tokens, (int32_t)requests};
    if (type == QNN_BF16) launch_pieces<Bf16, true>(a, as_stream(stream));
    else launch_pieces<F16, true>(a, as_stream(stream));
    return launch_status(hipGetLastError());
}

} // extern "C"
