// Attention over a cache of 8-bit codes: what its kernels share.
#pragma once

#include "halves.h"

namespace qnn {

inline bool bad_cache(const qnn_kv_cache *c)
{
    if (!c || c->pages < 0 || c->pages > INT32_MAX || c->heads <= 0 || c->heads > 65535) return true;
    if (c->dim != 64 && c->dim != 96 && c->dim != 128 && c->dim != 192 && c->dim != 256) return true;
    return c->block <= 0 || c->block > 256 || c->block % 32 != 0;
}
inline bool bad_cache_arrays(const qnn_kv_cache *c)
{
    const void *const arrays[4] = {c->k_codes, c->k_scales, c->v_codes, c->v_scales};
    for (const void *p : arrays)
        if ((!p && c->pages > 0) || ((uintptr_t)p & 15) != 0) return true;
    return false;
}

struct AttendArgs {
    qnn_kv_cache cache;
    const uint16_t *q;
    int64_t q_token_pitch, q_head_pitch;
    const int32_t *cu, *lengths, *table;
    uint16_t *out;
    float *lse;
    float *part_o;  // [requests][heads][part_rows][chunks][dim]
    float *part_ml; // [requests][heads][part_rows][chunks][2]: reference and sum of a part; sum < 0: part_o in units of 2^kLargeUnit
    int64_t table_width, tokens, window;
    float scale; // times log2(e)
    int32_t q_heads, group, requests;
    int32_t chunk_tokens, chunks, row_blocks;
    int32_t part_rows;            // rows per request and head that there is scratch for
    int32_t rows_over, rows_upto; // requests with other numbers of rows (queries * group) are another launch's
};

constexpr float kNothing = -3.0e38f; // running maximum before the first token that is seen
// probabilities are held as 2^kHead times their value: what binary16 loses below its normal numbers starts that much lower
constexpr float kHead = 14.0f;
// Scores (times log2(e)) of this size are 2^-4 apart at least: a head room taken off them would be rounded away, or up to 2^16.
constexpr float kFarScore = 0x1p20f;
// what scores are taken against, below their maximum by the head room
__device__ __forceinline__ float reference_of(float most) { return most - (fabsf(most) < kFarScore ? kHead : 0.0f); }
// Sums of up to 2^31 probabilities of 2^14 with values of 127 steps stay within binary32 up to scales of 2^72.  Where a page's scale is
// larger, sums stand in units of 2^48 (parts of a context say so by the sign of l).
constexpr float kLargeScale = 0x1p72f;
constexpr int kLargeUnit = 48;

// one request's part of a call
struct Request {
    int64_t row0; // first query
    int32_t n;    // queries
    int64_t length, low, high; // tokens [low, high) are what any of its queries sees, low rounded down to whole units
};
template <int U> __device__ __forceinline__ Request request_of(const AttendArgs &a, int r)
{
    Request q;
    // (the same in all lanes: kept in scalar registers)
    const int32_t cu0 = __builtin_amdgcn_readfirstlane(a.cu[r]), cu1 = __builtin_amdgcn_readfirstlane(a.cu[r + 1]);
    const int64_t c0 = min(max((int64_t)cu0, (int64_t)0), a.tokens), c1 = min(max((int64_t)cu1, c0), a.tokens);
    q.row0 = c0, q.n = (int32_t)(c1 - c0);
    q.length = max(__builtin_amdgcn_readfirstlane(a.lengths[r]), 0);
    const int64_t held = min(q.length, a.table_width * a.cache.block); // (queries stand at the end of all tokens, the table's or not)
    int64_t low = a.window > 0 ? q.length - q.n + 1 - a.window : 0;
    low = max(low, (int64_t)0) / U * U;
    q.low = min(low, held / U * U), q.high = a.cache.pages > 0 ? held : q.low;
    return q;
}
__device__ __forceinline__ int chunks_of(const AttendArgs &a, const Request &q)
{
    if (q.n * a.group > a.part_rows) return 1; // (more queries than the host was told: no room for parts)
    // (a request with more queries than the host was told can reach back further under a window: its last chunk is longer)
    return (int)min(max((int64_t)1, (q.high - q.low + a.chunk_tokens - 1) / a.chunk_tokens), (int64_t)a.chunks);
}

__device__ __forceinline__ int64_t part_row(const AttendArgs &a, int r, int h, int row) { return ((int64_t)r * a.cache.heads + h) * a.part_rows + row; }

// Four codes of a dword to binary16, exactly: with the sign bit flipped a code is c + 128, which behind the byte 0x64 is the
// binary16 1024 + c + 128.
__device__ __forceinline__ void codes_to_halves(uint32_t w, h16x2 &lo, h16x2 &hi)
{
    w ^= 0x80808080u;
    const h16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(h16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off;
    hi = __builtin_bit_cast(h16x2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off;
}
__device__ __forceinline__ h16x8 codes_to_halves8(uint32_t w0, uint32_t w1)
{
    h16x2 a, b, c, d;
    codes_to_halves(w0, a, b);
    codes_to_halves(w1, c, d);
    return h16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

} // namespace qnn
