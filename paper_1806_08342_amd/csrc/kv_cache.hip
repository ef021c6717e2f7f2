// Writing and reading the paged cache of 8-bit codes (qnn_kv_append, qnn_kv_gather).
#include "kv_attention.h"

namespace qnn {

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
// touches at most n / block + 2 pages (rounded down), so that pages item_base(r) ... item_base(r + 1) - 1 are its own; the
// request is found by bisection with 64 lanes at a time.
__device__ __forceinline__ int64_t first_row(const CacheArgs &a, int r) { return min(max((int64_t)a.cu[r], (int64_t)0), a.tokens); }
__device__ __forceinline__ int64_t item_base(const CacheArgs &a, int r) { return first_row(a, r) / a.cache.block + 2 * (int64_t)r; }
__device__ __forceinline__ int request_of_item(const CacheArgs &a, int64_t item)
{
    const int lane = threadIdx.x & 63;
    int low = 0, n = a.requests; // in [low, low + n)
    while (n > 1) {
        const int step = (n + 63) / 64, r = low + lane * step;
        const uint64_t reached = __ballot(lane * step < n && item_base(a, r) <= item);
        const int k = max(__popcll(reached) - 1, 0);
        low += k * step, n = min(step, n - k * step);
    }
    return low;
}

struct Piece {
    int64_t row;  // of k and v: the first new token's
    int64_t page; // -1: none
    int lo, hi;   // tokens of the page that are new, [lo, hi)
};
__device__ __forceinline__ Piece piece_of_item(const CacheArgs &a, int64_t item)
{
    const int r = request_of_item(a, item);
    const int64_t c0 = first_row(a, r), n = max(first_row(a, r + 1) - c0, (int64_t)0), at = max(a.start[r], 0);
    const int block = a.cache.block;
    const int64_t j = at / block + (item - item_base(a, r)); // page of the request
    const int64_t t0 = max(at, j * block), t1 = min(at + n, (j + 1) * block);
    Piece p{c0 + (t0 - at), -1, (int)(t0 - j * block), (int)(t1 - j * block)};
    if (t1 <= t0) p.hi = p.lo;
    else if (j < a.table_width) {
        const int32_t page = a.table[(int64_t)r * a.table_width + j];
        if ((uint32_t)page < (uint64_t)a.cache.pages) p.page = page;
    }
    return p;
}

// round(x / scale) of a finite or NaN quotient, as a code
__device__ __forceinline__ int code_of(float x)
{
    const float r = roundf(x); // ties away from zero
    return (int)fminf(fmaxf(r, -127.0f), 127.0f); // (NaN: the first comparison gives -127)
}

// One page and head of keys (blockIdx.y even) or values.
template <class T> __global__ void __launch_bounds__(256) append_kernel(const CacheArgs a)
{
    const int h = blockIdx.y >> 1, tid = threadIdx.x;
    const bool is_v = blockIdx.y & 1;
    const Piece p = piece_of_item(a, blockIdx.x);
    if (p.hi <= p.lo || p.page < 0) return;
    const int block = a.cache.block, D = a.cache.dim;
    const int64_t token = is_v ? a.v_token : a.k_token;
    const uint16_t *x = (is_v ? a.v : a.k) + p.row * token + (int64_t)h * (is_v ? a.v_head : a.k_head);
    const int64_t slot = p.page * a.cache.heads + h;
    int8_t *codes = (is_v ? a.cache.v_codes : a.cache.k_codes) + slot * block * D;
    float *scale = (is_v ? a.cache.v_scales : a.cache.k_scales) + slot;
    const int count = (p.hi - p.lo) * D;

    float peak = 0.0f;
    for (int i = tid; i < count; i += 256) {
        const float v = fabsf(T::widen(x[(int64_t)(i / D) * token + i % D]));
        peak = v < INFINITY ? fmaxf(peak, v) : peak;
    }
    __shared__ float s_peak[4];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) peak = fmaxf(peak, __shfl_xor(peak, d));
    if ((tid & 63) == 0) s_peak[tid >> 6] = peak;
    __syncthreads();
    peak = fmaxf(fmaxf(s_peak[0], s_peak[1]), fmaxf(s_peak[2], s_peak[3]));
    const float before = p.lo > 0 ? *scale : 0.0f;
    const float after = fmaxf(before, __fdiv_rn(peak, 127.0f)), by = after > 0.0f ? after : 1.0f;
    __syncthreads(); // the scale is read by all before one writes it
    if (tid == 0) *scale = after;
    if (after > before && p.lo > 0) { // what is held, in the new scale
        const float ratio = __fdiv_rn(before, by);
        for (int i = tid; i < p.lo * D; i += 256) {
            int8_t *c = is_v ? codes + (i / p.lo) * block + i % p.lo : codes + i;
            *c = (int8_t)code_of((float)*c * ratio);
        }
    }
    for (int i = tid; i < count; i += 256) {
        const int t = i / D, d = i % D;
        const float v = T::widen(x[(int64_t)t * token + d]);
        const int c = v == v ? code_of(__fdiv_rn(v, by)) : 0;
        codes[is_v ? d * block + p.lo + t : (p.lo + t) * D + d] = (int8_t)c;
    }
}

template <class T> __global__ void __launch_bounds__(256) gather_kernel(const CacheArgs a)
{
    const int h = blockIdx.y >> 1, tid = threadIdx.x;
    const bool is_v = blockIdx.y & 1;
    const Piece p = piece_of_item(a, blockIdx.x);
    if (p.hi <= p.lo) return;
    const int block = a.cache.block, D = a.cache.dim, heads = a.cache.heads;
    uint16_t *out = (is_v ? a.v_out : a.k_out) + (p.row * heads + h) * D;
    const int64_t slot = p.page * heads + h;
    const float scale = p.page < 0 ? 0.0f : (is_v ? a.cache.v_scales : a.cache.k_scales)[slot];
    const int8_t *codes = (is_v ? a.cache.v_codes : a.cache.k_codes) + slot * block * D;
    for (int i = tid; i < (p.hi - p.lo) * D; i += 256) {
        const int t = i / D, d = i % D;
        const float v = p.page < 0 ? 0.0f : (float)codes[is_v ? d * block + p.lo + t : (p.lo + t) * D + d] * scale;
        out[(int64_t)t * heads * D + d] = T::narrow(v);
    }
}

static bool bad_cache_call(const qnn_kv_cache *cache, int64_t table_width, int64_t requests, int64_t tokens, int type)
{
    return bad_cache(cache) || bad_half_type(type) || table_width < 0 || table_width > INT32_MAX / cache->block || requests < 0 || requests > (1 << 20) ||
           tokens < 0 || tokens > INT32_MAX / 2;
}
static dim3 piece_grid(const CacheArgs &a)
{
    return dim3((unsigned)(a.tokens / a.cache.block + 2 * (int64_t)a.requests), 2u * (unsigned)a.cache.heads);
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
    if (type == QNN_BF16) hipLaunchKernelGGL(append_kernel<Bf16>, piece_grid(a), dim3(256), 0, as_stream(stream), a);
    else hipLaunchKernelGGL(append_kernel<F16>, piece_grid(a), dim3(256), 0, as_stream(stream), a);
    return launch_status(hipGetLastError());
}

qnn_status qnn_kv_gather(const qnn_kv_cache *cache, const int32_t *cu, const int32_t *first, const int32_t *table, int64_t table_width,
                         int64_t requests, int64_t tokens, int type, void *k, void *v, void *stream)
{
    if (bad_cache_call(cache, table_width, requests, tokens, type)) return QNN_EINVAL;
    if (requests == 0 || tokens == 0) return QNN_OK;
    if (!k || !v || !cu || !first || (table_width > 0 && !table) || bad_cache_arrays(cache)) return QNN_EINVAL;
    const CacheArgs a{*cache, nullptr, nullptr, 0, 0, 0, 0, static_cast<uint16_t *>(k), static_cast<uint16_t *>(v), cu, first, table, table_width,
                      tokens, (int32_t)requests};
    if (type == QNN_BF16) hipLaunchKernelGGL(gather_kernel<Bf16>, piece_grid(a), dim3(256), 0, as_stream(stream), a);
    else hipLaunchKernelGGL(gather_kernel<F16>, piece_grid(a), dim3(256), 0, as_stream(stream), a);
    return launch_status(hipGetLastError());
}

} // extern "C"
