// A layer of experts for a few tokens, their weights in e4m3 (qnn_f8_moe): each token's top_k experts by its logits,
//
//   y[t] = sum_e weight[t][e] * down[e] (silu(gate[e] x[t]) * (up[e] x[t]))
//
// Bound by reading the weights of the experts that some token chose, each once.  Three launches for up to 64 tokens: the choice;
// gate and up, whose product h of each choice goes to the workspace, and beside them the list of the experts chosen with their tokens; down, which gathers
// a token's experts.  No atomics on memory: an output is the sum of its experts in the order of their numbers and of parts of K, whatever the order of workgroups.
//
// h keeps 16 significant bits, as two bfloat16 that are added up: in one it would cost the result as much as its own rounding.  Down's weights enter as
// bfloat16 beside it, exactly.
#include "buffer_ops.h"
#include "f8.h"
#include "lds_ring.h"

#include <algorithm>

namespace qnn {

constexpr int kTokens = 64;    // of one set of launches
constexpr int kMostExperts = 1024, kMostChosen = 32;

struct MoeArgs {
    const uint8_t *x, *up, *down; // [T][ldx], [E][2 I][H], [E][H][I]
    const float *xs, *ups, *downs;
    const void *logits;
    void *y;
    int32_t *experts;  // the caller's, or null
    float *weights;    // of a choice: the caller's or the workspace's
    int64_t ldx, ldxs, ldl, ldy;
    int32_t T, E, k, H, I, logit_type, type, renormalize;
    // workspace
    int32_t *chosen;   // [T][k]: a choice's expert, or -1
    uint64_t *bits;    // [T][words]: the experts that a token chose
    uint8_t *places;   // [T][E]: where among its choices, of those
    int32_t *list;     // how many stretches there are, then the stretches: heads (expert, how many), their choices (t * k + place) and their weights
    uint16_t *h; // [2][choices][I]: the two parts
    int32_t most, choices; // experts that can be chosen; choices
    float *sums;           // of parts of the blocks, [parts][T][H], or null
    int32_t parts;
};
// A stretch is up to 8 choices of one expert.
constexpr int kStretch = 8;
__host__ __device__ __forceinline__ int moe_most_stretches(int most, int choices) { return most + choices / kStretch; }
struct MoeHead {
    int32_t expert, count;
};
__device__ __forceinline__ MoeHead *moe_heads(const MoeArgs &a) { return reinterpret_cast<MoeHead *>(a.list + 2); }
__device__ __forceinline__ int32_t *moe_choices(const MoeArgs &a) { return a.list + 2 + 2 * moe_most_stretches(a.most, a.choices); }
__device__ __forceinline__ float *moe_shares(const MoeArgs &a) { return reinterpret_cast<float *>(a.list + 2 + 10 * moe_most_stretches(a.most, a.choices)); }

__host__ __device__ __forceinline__ int moe_words(int E) { return (E + 63) / 64; }

// larger key: larger logit; 0: never chosen (NaN and -inf)
__device__ __forceinline__ uint32_t logit_key(float v)
{
    if (!(v > -INFINITY)) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, fminf(v, 3.402823466e38f) + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k); }

// largest and smallest over a wave, the same in all lanes
__device__ __forceinline__ uint32_t wave_most(uint32_t v)
{
    const auto turned = [](uint32_t u, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, decltype(ctrl)::value, 0xf, 0xf, true); };
    v = max(v, turned(v, std::integral_constant<int, 0x128>())); // row_ror:8 and so on: over 16 lanes
    v = max(v, turned(v, std::integral_constant<int, 0x124>()));
    v = max(v, turned(v, std::integral_constant<int, 0x122>()));
    v = max(v, turned(v, std::integral_constant<int, 0x121>()));
    const auto of = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
    return max(max(of(0), of(16)), max(of(32), of(48)));
}
__device__ __forceinline__ float wave_sum(float v)
{
    const auto turned = [](float u, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, u), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += turned(v, std::integral_constant<int, 0x128>());
    v += turned(v, std::integral_constant<int, 0x124>());
    v += turned(v, std::integral_constant<int, 0x122>());
    v += turned(v, std::integral_constant<int, 0x121>());
    const auto of = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
    return (of(0) + of(16)) + (of(32) + of(48));
}

// A token's choice by a wave: lane j gets the expert at place j (-1 behind the last), and its weight.
template <int KEYS> __device__ __forceinline__ void choose(const MoeArgs &a, int t, int &expert, float &weight)
{
    const int lane = threadIdx.x & 63;
    uint32_t key[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
        const int e = i * 64 + lane;
        const float v = load_out(a.logits, t * a.ldl + min(e, a.E - 1), a.logit_type);
        key[i] = e < a.E ? logit_key(v) : 0u;
    }
    expert = -1;
    float sum = 0.0f, top = 0.0f;
    uint32_t mine = 0; // the key at place `lane`
    for (int j = 0; j < a.k; ++j) {
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) here = max(here, key[i]);
        const uint32_t best = wave_most(here);
        if (best == 0) break;
        if (j == 0) {
            top = key_logit(best);
            if (!a.renormalize)
#pragma unroll
                for (int i = 0; i < KEYS; ++i) sum += key[i] ? expf(key_logit(key[i]) - top) : 0.0f;
        }
        uint32_t first = 0; // the lowest index of those: the largest complement
#pragma unroll
        for (int i = KEYS - 1; i >= 0; --i)
            if (key[i] == best) first = ~(uint32_t)(i * 64 + lane);
        const uint64_t who = __ballot(here == best);
        const int e = (int)~(__popcll(who) == 1 ? (uint32_t)__builtin_amdgcn_readlane((int)first, __ffsll((unsigned long long)who) - 1) : wave_most(first));
#pragma unroll
        for (int i = 0; i < KEYS; ++i)
            if (i * 64 + lane == e) key[i] = 0;
        if (lane == j) mine = best, expert = e;
    }
    const float part = expert >= 0 ? expf(key_logit(mine) - top) : 0.0f;
    const float of = wave_sum(a.renormalize ? part : sum);
    weight = expert >= 0 ? part / of : 0.0f;
}

// One wave per token.  (One workgroup for all of them, which made the lists too, took 7 us for 63 tokens and 4 experts, 14 for 64 of which each chose 8.)
template <int KEYS> __global__ void __launch_bounds__(64) moe_choose_kernel(const MoeArgs a)
{
    const int t = blockIdx.x, lane = threadIdx.x;
    int expert;
    float weight;
    choose<KEYS>(a, t, expert, weight);
    if (lane < a.k) {
        a.chosen[t * a.k + lane] = expert;
        a.weights[t * a.k + lane] = weight;
        if (a.experts) a.experts[t * a.k + lane] = expert;
        if (expert >= 0) a.places[t * a.E + expert] = (uint8_t)lane;
    }
    // (all k of a wave's lanes, one after the other, into the word that lane w has)
    uint64_t word = 0;
    for (int j = 0; j < a.k; ++j) {
        const int e = __builtin_amdgcn_readlane(expert, j);
        if (e >= 0 && e / 64 == lane) word |= 1ull << (e & 63);
    }
    if (lane < moe_words(a.E)) a.bits[t * moe_words(a.E) + lane] = word;
}

// The stretches of all choices, experts in their order and an expert's tokens in theirs: by one workgroup of 256.
constexpr int kListBytes = kMostExperts * (8 + 4) + 16;
__device__ __forceinline__ void moe_list(const MoeArgs &a, uint8_t *shared)
{
    uint64_t *const s_tokens = reinterpret_cast<uint64_t *>(shared);             // who chose an expert
    int32_t *const s_at = reinterpret_cast<int32_t *>(shared + kMostExperts * 8); // an expert's first stretch
    int32_t *const s_sum = s_at + kMostExperts;
    constexpr int EACH = kMostExperts / 256;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int i = 0; i < EACH; ++i) s_tokens[tid + 256 * i] = 0;
    __syncthreads();
    for (int i = tid; i < a.choices; i += 256) {
        const int e = a.chosen[i];
        if (e >= 0) atomicOr(reinterpret_cast<unsigned long long *>(&s_tokens[e]), 1ull << i / a.k);
    }
    __syncthreads();
    int parts[EACH], before = 0; // (of the experts before this thread's, then)
#pragma unroll
    for (int i = 0; i < EACH; ++i) parts[i] = (__popcll(s_tokens[EACH * tid + i]) + kStretch - 1) / kStretch, before += parts[i];
    const int own = before;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(before, d);
        if (lane >= d) before += u;
    }
    if (lane == 63) s_sum[wave] = before;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += s_sum[w];
    if (tid == 255) a.list[0] = before;
    before -= own;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int e = EACH * tid + i, count = __popcll(s_tokens[e]);
        s_at[e] = before;
        for (int j = 0; j < parts[i]; ++j) moe_heads(a)[before + j] = MoeHead{e, min(count - j * kStretch, kStretch)};
        before += parts[i];
    }
    __syncthreads();
    for (int i = tid; i < a.choices; i += 256) {
        const int e = a.chosen[i];
        if (e < 0) continue;
        const int at = s_at[e] * kStretch + __popcll(s_tokens[e] & ((1ull << i / a.k) - 1));
        moe_choices(a)[at] = i, moe_shares(a)[at] = a.weights[i];
    }
}

constexpr int kSums = 20; // 16 sums of up, and what is between them
// Choices of the expert that group j of the workgroups has, in the order of their tokens, and how many (0: none).  Where there are
// no more experts than choices that is expert j, else the one of choice j, if none before chose it.
// (Found in the list of all choices, with two barriers more, 64 tokens that choose 8 of 64 experts took 75 us for what is 67 so.)
__device__ __forceinline__ int moe_choices_of(const MoeArgs &a, int j, int &expert, int32_t *s_choice)
{
    const int lane = threadIdx.x & 63, t = min(lane, a.T - 1), e = a.E <= a.choices ? j : a.chosen[j];
    if (e < 0) return 0;
    const uint64_t word = a.bits[t * moe_words(a.E) + e / 64];
    const int choice = t * a.k + a.places[t * a.E + e];
    const bool own = lane < a.T && (word >> (e & 63) & 1);
    const uint64_t who = __ballot(own);
    if (who == 0) return 0;
    if (a.E > a.choices && __builtin_amdgcn_readlane(choice, __ffsll((unsigned long long)who) - 1) != j) return 0;
    if (threadIdx.x < 64 && own) s_choice[kSums * __popcll(who & ((1ull << lane) - 1))] = choice;
    __syncthreads();
    expert = __builtin_amdgcn_readfirstlane(e);
    return __popcll(who);
}

// Up to 64 choices of up to 8 tokens, listed by every workgroup for itself (experts in the order in which they are first chosen): the choices of
// expert j, as bits.  The first workgroup writes the lists for what follows.  One launch less: a token's layer of 8 among 64 experts
// of 4096 x 1536 42 us with it, 39 without.
constexpr int kFewTokens = 8, kFewChoices = 64;
template <int KEYS> __device__ __forceinline__ uint64_t moe_route_few(const MoeArgs &a, int j, int &expert)
{
    __shared__ int16_t s_expert[kFewChoices];
    __shared__ float s_share[kFewChoices];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (threadIdx.x < kFewChoices) s_expert[threadIdx.x] = -1;
    __syncthreads();
    for (int t = wave; t < a.T; t += 4) {
        int e;
        float weight;
        choose<KEYS>(a, t, e, weight);
        if (lane < a.k) {
            s_expert[t * a.k + lane] = (int16_t)e, s_share[t * a.k + lane] = weight;
            if (blockIdx.x == 0) {
                a.weights[t * a.k + lane] = weight;
                if (a.experts) a.experts[t * a.k + lane] = e;
            }
        }
    }
    __syncthreads();
    const int e = s_expert[lane];
    uint64_t same = __ballot(e >= 0); // the choices of the same expert
#pragma unroll
    for (int bit = 0; bit < 10; ++bit) {
        const uint64_t set = __ballot(e >> bit & 1);
        same &= e >> bit & 1 ? set : ~set;
    }
    const uint64_t below = (1ull << lane) - 1;
    const bool first = e >= 0 && (same & below) == 0;
    const uint64_t firsts = __ballot(first);
    const int at = __popcll(firsts & below);
    if (blockIdx.x == 0 && wave == 0) {
        const int stretch = __shfl(at, same ? __ffsll((unsigned long long)same) - 1 : 0); // (of an expert chosen by up to 8 tokens there is one)
        if (e >= 0) {
            const int to = stretch * kStretch + __popcll(same & below);
            moe_choices(a)[to] = lane, moe_shares(a)[to] = s_share[lane];
        }
        if (first) moe_heads(a)[at] = MoeHead{e, (int)__popcll(same)};
        if (lane == 0) a.list[0] = __popcll(firsts);
    }
    const uint64_t who = __ballot(first && at == j);
    if (who == 0) return 0;
    const int l = __ffsll((unsigned long long)who) - 1;
    expert = __builtin_amdgcn_readlane(e, l);
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(same >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)same, l);
}

// h as two bfloat16 that are added up, its first 16 significant bits at least: the nearest, and what is left, rounded.  Finite numbers from
// 2^128 (1 - 2^-9) on, whose nearest is infinite, are the largest bfloat16 and what is left cut off (rounded, the two could add up to 2^128).  Of an infinity or a NaN the first
// part is all.
__device__ __forceinline__ void two_parts(float h, uint16_t &first, uint16_t &second)
{
    uint16_t high = Bf16::narrow(h), low = 0;
    if (fabsf(h) < INFINITY) {
        const bool past = (high & 0x7fff) == 0x7f80;
        high = (uint16_t)(high - past);
        const float rest = h - Bf16::widen(high);
        low = past ? (uint16_t)(__builtin_bit_cast(uint32_t, rest) >> 16) : Bf16::narrow(rest);
    }
    first = high, second = low;
}

// Workgroups: an expert by 16 columns of h; four waves share H and join their sums in LDS.
// Bound by the memory where H is long (64 tokens, 64 experts of 4096 x 2048 201 us, 5.3 TB/s; of 1024 x 2048 62 us, 4.3: a wave has two blocks).
// MORE: for experts of more than 16 MT tokens.  KEYS: 0: the choices are there, and the last workgroup lists them for what follows; else each workgroup chooses by itself, from so many times
// 64 logits.
template <int MT, int KEYS, bool MORE = false> __global__ void __launch_bounds__(256) moe_up_kernel(const MoeArgs a)
{
    constexpr int WAVES = 4, DEPTH = 2, SUMS = WAVES * 2 * 16 * MT * kSums * 4;
    __shared__ __attribute__((aligned(16))) uint8_t shared[KEYS == 0 && SUMS < kListBytes ? kListBytes : SUMS];
    int32_t *const choices = reinterpret_cast<int32_t *>(shared) + 16; // each behind 16 sums (in 40 KB, of which a CU holds four)
    const int columns = a.I / 16, j = blockIdx.x / columns, i0 = blockIdx.x % columns * 16;
    int e, count;
    if constexpr (KEYS == 0) {
        if (j == a.most) {
            moe_list(a, shared);
            return;
        }
        count = moe_choices_of(a, j, e, choices);
        if (count == 0) return;
    } else {
        const uint64_t mine = moe_route_few<KEYS>(a, j, e);
        if (mine == 0) return;
        count = __popcll(mine);
        if (threadIdx.x < 64 && (mine >> threadIdx.x & 1)) choices[kSums * __popcll(mine & ((1ull << threadIdx.x) - 1))] = threadIdx.x;
        __syncthreads();
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int blocks = (a.H + kF8Block - 1) / kF8Block, two = (2 * a.I + kF8Block - 1) / kF8Block;
    const uint8_t *const w_rows[2] = {a.up + ((int64_t)e * 2 * a.I + i0) * a.H, a.up + ((int64_t)e * 2 * a.I + a.I + i0) * a.H};
    const float *const w_scale[2] = {a.ups + ((int64_t)e * two + i0 / kF8Block) * blocks, a.ups + ((int64_t)e * two + (a.I + i0) / kF8Block) * blocks};
    const int x_bytes = (int)(a.T * a.ldx); // (below 2^30)
    for (int from = 0; from < (MORE ? count : 1); from += 16 * MT) { // (an expert's weights again, from the caches, for more)
        if (from > 0) __syncthreads();
        uint32_t x_row[MT];
        const float *x_scale[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int t = choices[kSums * min(from + mt * 16 + c, count - 1)] / a.k;
            x_row[mt] = (uint32_t)(t * a.ldx), x_scale[mt] = a.xs + t;
        }
        f32x4 acc[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt][0] = acc[mt][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        struct Step {
            w32x4 w[2][2];
            float ws[2];
        };
        // (H is a multiple of 16; what is behind a row's end lies beyond the buffers)
        const auto piece = [&](const uint8_t *rows, int bytes, uint32_t row, int k) { return buffer_load16(rows, bytes, k < a.H ? row + (uint32_t)k : 0x80000000u); };
        uint32_t w_first[2], x_first[MT]; // (with many tokens the exchange costs as much as it saves: 16 tokens, 8 experts of 4096 x 4096 91.9 us without, 94.3 with)
#pragma unroll
        for (int u = 0; u < 2; ++u) w_first[u] = KEYS == 0 ? 0 : half_first((uint32_t)(uintptr_t)w_rows[u] + (uint32_t)(c * a.H), c);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x_first[mt] = KEYS == 0 ? 0 : half_first((uint32_t)(uintptr_t)a.x + x_row[mt], c);
        const auto load = [&](Step &s, int b) {
            const int k = b * kF8Block + 16 * g;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                s.w[u][0] = piece(w_rows[u], 16 * a.H, (uint32_t)(c * a.H), k + 64 * (int)w_first[u]);
                s.w[u][1] = piece(w_rows[u], 16 * a.H, (uint32_t)(c * a.H), k + 64 * (int)(w_first[u] ^ 1));
                s.ws[u] = w_scale[u][b];
            }
        };
        const auto compute = [&](const Step &s, int b) {
            const int k = b * kF8Block + 16 * g;
            w32x4 w[2][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) in_order(s.w[u], w_first[u], w[u]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if (from + mt * 16 >= count) break;
                const w32x4 loaded[2] = {piece(a.x, x_bytes, x_row[mt], k + 64 * (int)x_first[mt]), piece(a.x, x_bytes, x_row[mt], k + 64 * (int)(x_first[mt] ^ 1))};
                w32x4 x[2];
                in_order(loaded, x_first[mt], x);
                const float xs = x_scale[mt][b * a.ldxs];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    fma4(acc[mt][u], f8_products<true>(w[u], x), xs * s.ws[u]);
                    asm volatile("" : "+v"(acc[mt][u])); // (before the branch: see the other kernel)
                }
            }
        };
        Step f[DEPTH];
        int b = wave;
        for (; b + (DEPTH - 1) * WAVES < blocks; b += DEPTH * WAVES) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) load(f[d], b + d * WAVES);
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) compute(f[d], b + d * WAVES);
        }
        for (; b < blocks; b += WAVES) {
            load(f[0], b);
            compute(f[0], b);
        }
        float(*const s_acc)[2][16 * MT][kSums] = reinterpret_cast<float(*)[2][16 * MT][kSums]>(shared);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int u = 0; u < 2; ++u) *reinterpret_cast<f32x4 *>(&s_acc[wave][u][mt * 16 + c][g * 4]) = acc[mt][u];
        __syncthreads();
        for (int i = threadIdx.x; i < min(count - from, 16 * MT) * 16; i += 64 * WAVES) {
            const int m = i / 16, n = i % 16;
            float gate = 0.0f, up = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) gate += s_acc[w][0][m][n], up += s_acc[w][1][m][n];
            const float h = gate / (1.0f + expf(-gate)) * up;
            const int64_t at = (int64_t)choices[kSums * (from + m)] * a.I + i0 + n;
            two_parts(h, a.h[at], a.h[(int64_t)a.choices * a.I + at]);
        }
    }
}

// A value at an address that is the same in the whole wave, which nothing writes while the kernel runs, over the scalar cache.
__device__ __forceinline__ float scalar_load(const float *p)
{
#if defined(__HIP_DEVICE_COMPILE__)
    return *(const __attribute__((address_space(4))) float *)(uintptr_t)p;
#else
    return *p;
#endif
}
__device__ __forceinline__ uint32_t lds_address(const uint8_t *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)p;
}
// A lane's two pieces of weights, and its four of h in two halves 2048 bytes apart.  (Written out, with their wait: as loads the compiler would have
// some of them wait for every copy into LDS that is on its way.)
__device__ __forceinline__ void read_pieces(uint32_t w0, uint32_t w1, uint32_t h0, uint32_t h1, w32x4 (&w)[2], w32x4 (&h)[4])
{
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("ds_read_b128 %0, %6\n\t"
                 "ds_read_b128 %1, %7\n\t"
                 "ds_read_b128 %2, %8\n\t"
                 "ds_read_b128 %3, %9\n\t"
                 "ds_read_b128 %4, %8 offset:2048\n\t"
                 "ds_read_b128 %5, %9 offset:2048\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0]), "=&v"(w[1]), "=&v"(h[0]), "=&v"(h[1]), "=&v"(h[2]), "=&v"(h[3])
                 : "v"(w0), "v"(w1), "v"(h0), "v"(h1)
                 : "memory");
#else
    (void)w0, (void)w1, (void)h0, (void)h1, (void)w, (void)h;
#endif
}

// Workgroups: 16 columns of y.  The blocks of 128 of all stretches of choices are shared out among the waves; a wave's sums of a stretch
// go to its own part of LDS, weighted, and the waves' parts are added up at the end.
// The two parts of the h of up to 8 choices are the 16 rows of one operand (an expert's weights are read again, from the caches, for more).  Weights and h
// are copied into rings in LDS, each wave's own, three blocks and one ahead: as fragments straight into registers, 64 bytes of a row at a time, the texture path took longer over h
// than the memory over the weights (64 tokens, 64 experts of 4096 x 2048: 93 us for the weights alone, 172 with h; so 123, 4.4 TB/s).
template <int TOKENS> __global__ void __launch_bounds__(512, 2) moe_down_kernel(const MoeArgs a)
{
    constexpr int WAVES = 8, W_SLOT = 2048, H_SLOT = 4096, RING = 4 * W_SLOT + 2 * H_SLOT;
    __shared__ __attribute__((aligned(128))) uint8_t s_ring[WAVES][RING];
    __shared__ float s_y[WAVES][TOKENS][16];
    const int n0 = blockIdx.x * 16, part = blockIdx.y;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    for (int i = lane; i < TOKENS * 16; i += 64) (&s_y[wave][0][0])[i] = 0.0f;
    uint8_t *const w_ring = s_ring[wave], *const h_ring = w_ring + 4 * W_SLOT;
    const int blocks = (a.I + kF8Block - 1) / kF8Block, row_blocks = (a.H + kF8Block - 1) / kF8Block;
    const int stretches = a.list[0], units = stretches * blocks;
    const int sharing = WAVES * a.parts, mine = part * WAVES + wave;
    const int first = units * mine / sharing, last = units * (mine + 1) / sharing; // (up to 1280 stretches of 1024 blocks, by 256)
    const uint8_t *const inner = reinterpret_cast<const uint8_t *>(a.h);
    const int inner_bytes = 4 * a.choices * a.I; // (up to 2^30)
    constexpr uint32_t kBeyond = 0x80000000u;    // of either buffer: zeros, without traffic
    // 16 rows of 128 bytes, 16-byte pieces exchanged by half the row's number, so that reads of 16 rows meet the 16 places of the 64 banks; a
    // copy's lanes have 8 rows, from `half` * 8 on
    const auto piece = [&](int half) { return (lane & 7) ^ (lane >> 4) ^ 4 * half; };
    // A lane's place among 16 rows of weights and in a row of h, and whether that is there in the last block
    const int tail = a.I - (blocks - 1) * kF8Block;
    const uint32_t w_lane[2] = {(uint32_t)((lane >> 3) * a.I + 16 * piece(0)), (uint32_t)((8 + (lane >> 3)) * a.I + 16 * piece(1))};
    const bool w_there[2] = {16 * piece(0) < tail, 16 * piece(1) < tail};
    const bool h_there[2][2] = {{8 * piece(0) < tail, 8 * piece(1) < tail}, {64 + 8 * piece(0) < tail, 64 + 8 * piece(1) < tail}};
    const uint32_t w_place = lds_address(w_ring) + c * 128 + (g ^ (c >> 1 & 7)) * 16, h_place = lds_address(h_ring) + c * 128 + (2 * g ^ (c >> 1 & 7)) * 16;
    // Each workgroup begins a stretch at another block: rows lie a power of two apart more often than not, and workgroups that read the same columns
    // of all rows at one time would keep to a part of the memory's channels.
    const int turn = (int)(blockIdx.x % (unsigned)blocks);
    // Up to 8 stretches at a time, whose lists lie in the lanes: lane l has choice l & 7 of stretch l >> 3.  What is on its way runs on from one
    // stretch into the next (with each stretch by itself 64 tokens, 64 experts of 4096 x 2048 took 132 us, so
    // 123).
    for (int from = first; from < last;) {
        const int j0 = from / blocks, to = min(last, (j0 + 8) * blocks), many = to - from;
        const int mine_j = min(j0 + (lane >> 3), stretches - 1);
        const MoeHead head = moe_heads(a)[mine_j];
        const int listed = moe_choices(a)[mine_j * kStretch + (lane & 7)]; // (anything behind the last)
        const float share = moe_shares(a)[mine_j * kStretch + (lane & 7)];
        const bool there = (lane & 7) < head.count;
        const int choice = there ? listed : 0, token = choice / a.k;
        const uint32_t copied = 2u * (uint32_t)(choice * a.I) | (there ? 0u : kBeyond);
        struct Cursor { // a place among these blocks
            int j, i, n, b0, turned; // stretch, block within what there is of it here, how many those are, the first, where it begins
        };
        const auto enter = [&](Cursor &at, int j) {
            const int begin = (j0 + j) * blocks, low = max(from, begin), high = min(to, begin + blocks);
            at.j = j, at.i = 0, at.n = high - low, at.b0 = low - begin, at.turned = turn < at.n ? turn : 0;
        };
        const auto advance = [&](Cursor &at) { // to another stretch? (behind the last block: n is 0 or less, and stays so)
            if (++at.i < at.n || at.n <= 0) return false;
            enter(at, at.j + 1);
            return true;
        };
        const auto block_of = [&](const Cursor &at) { return at.b0 + (at.i + at.turned < at.n ? at.i + at.turned : at.i + at.turned - at.n); };
        Cursor here, next, ahead;
        enter(here, 0), enter(next, 0), enter(ahead, 0);
        const uint8_t *w_rows;
        const float *scales;
        const auto enter_weights = [&](int j) { w_rows = a.down + ((int64_t)__builtin_amdgcn_readlane(head.expert, 8 * min(j, 7)) * a.H + n0) * a.I; };
        const auto enter_scales = [&](int j) {
            scales = a.downs + ((int64_t)__builtin_amdgcn_readlane(head.expert, 8 * min(j, 7)) * row_blocks + n0 / kF8Block) * blocks;
        };
        enter_weights(0), enter_scales(0);
        uint32_t row[2];
        const auto enter_rows = [&](int j) {
            const uint32_t first = (uint32_t)__shfl((int)copied, 8 * min(j, 7) + (lane >> 3));
            row[0] = first + 16 * piece(0), row[1] = first + 2 * a.choices * a.I + 16 * piece(1);
        };
        enter_rows(0);
        // (Without branches, so that the compiler's count of what is on its way holds: behind the last block the buffers have no bytes.)
        const auto load = [&](Cursor &at, int slot) {
            const int b = at.n > 0 ? block_of(at) : 0;
            const bool inside = b < blocks - 1;
            const int bytes = at.n > 0 ? 16 * a.I - b * kF8Block : 0;
#pragma unroll
            for (int half = 0; half < 2; ++half)
                buffer_to_lds16(w_rows + b * kF8Block, bytes, inside || w_there[half] ? w_lane[half] : kBeyond, w_ring + slot * W_SLOT + half * 1024);
            if (advance(at)) enter_weights(at.j);
        };
        const auto load_inner = [&](Cursor &at, int slot) {
            const int b = at.n > 0 ? block_of(at) : 0;
            const bool inside = b < blocks - 1;
            const int before = 2 * b * kF8Block, bytes = at.n > 0 ? inner_bytes - before : 0;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int part = 0; part < 2; ++part)
                    buffer_to_lds16(inner + before + 128 * p, bytes, inside || h_there[p][part] ? row[part] : kBeyond, h_ring + slot * H_SLOT + p * 2048 + part * 1024);
            if (advance(at)) enter_rows(at.j);
        };
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const auto compute = [&](int slot, float scale) {
            w32x4 w[2], v[4];
            const uint32_t w_at = w_place + slot * W_SLOT, h_at = h_place + (slot & 1) * H_SLOT;
            read_pieces(w_at, w_at ^ 64, h_at, h_at ^ 16, w, v);
            b16x8 wide[4];
#pragma unroll
            for (int p = 0; p < 2; ++p) wide[2 * p] = widen_codes(w[p][0], w[p][1]), wide[2 * p + 1] = widen_codes(w[p][2], w[p][3]);
            f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < 4; ++q) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[q], __builtin_bit_cast(b16x8, v[q]), part, 0, 0, 0);
            fma4(acc, part, scale);
            asm volatile("" : "+v"(acc)); // (here, and not behind a branch, which the compiler's waits for the products do not reach over)
        };
        const auto finish = [&]() { // a stretch's sums, weighted, to their tokens
            const int l = 8 * here.j + (c & 7), t = __shfl(token, l);
            const float weight = __shfl(share, l);
            const int count = __builtin_amdgcn_readlane(head.count, 8 * here.j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = acc[r] + __shfl_xor(acc[r], 8);
                if (c < 8 && c < count) s_y[wave][t][g * 4 + r] += weight * v;
            }
            acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        };
        wait_vmcnt<0>();
        load_inner(next, 0);
#pragma unroll 1
        for (int i = 0; i < 3; ++i) load(ahead, i);
#pragma unroll 1
        for (int i = 0; i < many; ++i) { // (not unrolled: the first passes over longer code would cost a small layer 1.5 us)
            const float scale = scalar_load(scales + block_of(here));
            load_inner(next, (i + 1) & 1);
            load(ahead, (i + 3) & 3);
            wait_vmcnt<2 + 4 + 2>(); // but the weights of the two blocks ahead and these
            compute(i & 3, scale);
            if (here.i + 1 == here.n) finish();
            if (advance(here)) enter_scales(here.j);
        }
        from = to;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += 64 * WAVES) {
        const int t = i / 16, n = i % 16;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += s_y[w][t][n];
        if (a.sums) a.sums[((int64_t)part * a.T + t) * a.H + n0 + n] = v;
        else store_out(a.y, t * a.ldy + n0 + n, a.type, v);
    }
}

// The same for more tokens: workgroups of 128 columns of y, 16 for each wave, which share the h of a stretch, two blocks at a time behind one barrier, in
// three slots; the weights' rings hold as much.  (With each wave's own copies of h, as above, the L2 delivers more of them than of weights: 64 tokens,
// 64 experts of 4096 x 2048 125 us, so 99, 5.4 TB/s of weights; 8 experts of 4096 x 4096 67 and 56.)
template <int TOKENS> __global__ void __launch_bounds__(512, 2) moe_down_wide_kernel(const MoeArgs a)
{
    constexpr int WAVES = 8, W_SLOT = 4096, H_SLOT = 8192, SLOTS = 3;
    __shared__ __attribute__((aligned(128))) uint8_t s_w[WAVES][SLOTS * W_SLOT], s_h[SLOTS * H_SLOT];
    __shared__ float s_y[WAVES][TOKENS][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 128 + wave * 16, part = blockIdx.y;
    const bool mine = n0 < a.H; // (a wave behind the last column copies its share of h all the same)
    for (int i = lane; i < TOKENS * 16; i += 64) (&s_y[wave][0][0])[i] = 0.0f;
    const int blocks = (a.I + kF8Block - 1) / kF8Block, pairs = (blocks + 1) / 2, row_blocks = (a.H + kF8Block - 1) / kF8Block;
    const int stretches = a.list[0], units = stretches * pairs;
    const int first = units * part / a.parts, last = units * (part + 1) / a.parts;
    const uint8_t *const inner = reinterpret_cast<const uint8_t *>(a.h);
    const int inner_bytes = 4 * a.choices * a.I;
    constexpr uint32_t kBeyond = 0x80000000u;
    const auto piece = [&](int half) { return (lane & 7) ^ (lane >> 4) ^ 4 * half; };
    const int tail = a.I - (blocks - 1) * kF8Block;
    const uint32_t w_lane[2] = {(uint32_t)((lane >> 3) * a.I + 16 * piece(0)), (uint32_t)((8 + (lane >> 3)) * a.I + 16 * piece(1))};
    const bool w_there[2] = {16 * piece(0) < tail, 16 * piece(1) < tail};
    // of two blocks' h a wave copies a block's half rows of one part
    const int own_block = wave >> 2, own_half = wave >> 1 & 1, own_part = wave & 1, own_piece = (lane & 7) ^ (lane >> 4) ^ 4 * own_part;
    const bool own_there = 64 * own_half + 8 * own_piece < tail;
    uint8_t *const own_slot = s_h + own_block * 4096 + own_half * 2048 + own_part * 1024;
    const uint32_t w_place = lds_address(s_w[wave]) + c * 128 + (g ^ (c >> 1 & 7)) * 16, h_place = lds_address(s_h) + c * 128 + (2 * g ^ (c >> 1 & 7)) * 16;
    const int turn = (int)(blockIdx.x % (unsigned)pairs);
    for (int from = first; from < last;) {
        const int j0 = from / pairs, to = min(last, (j0 + 8) * pairs), many = to - from;
        const int mine_j = min(j0 + (lane >> 3), stretches - 1);
        const MoeHead head = moe_heads(a)[mine_j];
        const int listed = moe_choices(a)[mine_j * kStretch + (lane & 7)];
        const float share = moe_shares(a)[mine_j * kStretch + (lane & 7)];
        const bool there = (lane & 7) < head.count;
        const int choice = there ? listed : 0, token = choice / a.k;
        const uint32_t copied = 2u * (uint32_t)(choice * a.I) | (there ? 0u : kBeyond);
        struct Cursor { // a place among these pairs of blocks
            int j, i, n, u0, turned;
        };
        const auto enter = [&](Cursor &at, int j) {
            const int begin = (j0 + j) * pairs, low = max(from, begin), high = min(to, begin + pairs);
            at.j = j, at.i = 0, at.n = high - low, at.u0 = low - begin, at.turned = turn < at.n ? turn : 0;
        };
        const auto advance = [&](Cursor &at) {
            if (++at.i < at.n || at.n <= 0) return false;
            enter(at, at.j + 1);
            return true;
        };
        const auto block_of = [&](const Cursor &at) { return 2 * (at.u0 + (at.i + at.turned < at.n ? at.i + at.turned : at.i + at.turned - at.n)); };
        Cursor here, ahead;
        enter(here, 0), enter(ahead, 0);
        const uint8_t *w_rows;
        const float *scales;
        uint32_t row;
        const auto enter_ahead = [&](int j) {
            w_rows = a.down + ((int64_t)__builtin_amdgcn_readlane(head.expert, 8 * min(j, 7)) * a.H + (mine ? n0 : 0)) * a.I;
            row = (uint32_t)__shfl((int)copied, 8 * min(j, 7) + (lane >> 3)) + (uint32_t)(own_part * 2 * a.choices * a.I) + 16 * own_piece;
        };
        const auto enter_scales = [&](int j) { scales = a.downs + ((int64_t)__builtin_amdgcn_readlane(head.expert, 8 * min(j, 7)) * row_blocks + blockIdx.x) * blocks; };
        enter_ahead(0), enter_scales(0);
        const auto load = [&](int slot) {
            const int b0 = ahead.n > 0 ? block_of(ahead) : blocks;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int b = b0 + q, bytes = b < blocks && mine ? 16 * a.I - b * kF8Block : 0;
                const bool inside = b < blocks - 1;
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    buffer_to_lds16(w_rows + b * kF8Block, bytes, inside || w_there[half] ? w_lane[half] : kBeyond, s_w[wave] + slot * W_SLOT + q * 2048 + half * 1024);
            }
            const int b = b0 + own_block, before = 2 * b * kF8Block, bytes = b < blocks ? inner_bytes - before : 0;
            buffer_to_lds16(inner + before + 128 * own_half, bytes, b < blocks - 1 || own_there ? row : kBeyond, own_slot + slot * H_SLOT);
            if (advance(ahead)) enter_ahead(ahead.j);
        };
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const auto compute = [&](int slot, int q, float scale) {
            w32x4 w[2], v[4];
            const uint32_t w_at = w_place + slot * W_SLOT + q * 2048, h_at = h_place + slot * H_SLOT + q * 4096;
            read_pieces(w_at, w_at ^ 64, h_at, h_at ^ 16, w, v);
            b16x8 wide[4];
#pragma unroll
            for (int p = 0; p < 2; ++p) wide[2 * p] = widen_codes(w[p][0], w[p][1]), wide[2 * p + 1] = widen_codes(w[p][2], w[p][3]);
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[i], __builtin_bit_cast(b16x8, v[i]), sum, 0, 0, 0);
            fma4(acc, sum, scale);
            asm volatile("" : "+v"(acc)); // (here, and not behind a branch, which the compiler's waits for the products do not reach over)
        };
        const auto finish = [&]() {
            const int l = 8 * here.j + (c & 7), t = __shfl(token, l);
            const float weight = __shfl(share, l);
            const int count = __builtin_amdgcn_readlane(head.count, 8 * here.j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = acc[r] + __shfl_xor(acc[r], 8);
                if (c < 8 && c < count) s_y[wave][t][g * 4 + r] += weight * v;
            }
            acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        };
        wait_vmcnt<0>();
        lds_barrier(); // (all waves are through with the stretches before, and nothing is on its way into the slots)
        load(0), load(1);
        int slot = 0;
#pragma unroll 1
        for (int i = 0; i < many; ++i) {
            const int b = block_of(here);
            const float scale = scalar_load(scales + b), second = b + 1 < blocks ? scalar_load(scales + b + 1) : 0.0f;
            wait_vmcnt<5>(); // but the next pair's copies
            lds_barrier();   // all waves' copies are here, and what the pair before was in is free
            load(slot == 0 ? 2 : slot - 1);
            compute(slot, 0, scale), compute(slot, 1, second);
            if (here.i + 1 == here.n) finish();
            if (advance(here)) enter_scales(here.j);
            slot = slot == 2 ? 0 : slot + 1;
        }
        from = to;
    }
    __syncthreads();
    for (int i = lane; mine && i < a.T * 16; i += 64) {
        const int t = i / 16, n = i % 16;
        const float v = s_y[wave][t][n];
        if (a.sums) a.sums[((int64_t)part * a.T + t) * a.H + n0 + n] = v;
        else store_out(a.y, t * a.ldy + n0 + n, a.type, v);
    }
}

// y = the parts' sums in their order
constexpr int kMostParts = 32;
__global__ void __launch_bounds__(256) moe_sum_kernel(const MoeArgs a)
{
    const int n = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (n >= a.H) return;
    float v = 0.0f;
    const auto add = [&](int begin, auto many) { // (all on their way at once: one after the other 8 took 4.8 us)
        constexpr int MANY = decltype(many)::value;
        float u[MANY];
#pragma unroll
        for (int p = 0; p < MANY; ++p) u[p] = a.sums[((int64_t)min(begin + p, a.parts - 1) * a.T + t) * a.H + n];
#pragma unroll
        for (int p = 0; p < MANY; ++p) v += begin + p < a.parts ? u[p] : 0.0f;
    };
    if (a.parts <= 4) add(0, std::integral_constant<int, 4>());
    else
        for (int begin = 0; begin < a.parts; begin += 16) add(begin, std::integral_constant<int, 16>());
    store_out(a.y, t * a.ldy + n, a.type, v);
}

struct MoeSpace {
    size_t chosen, bits, places, list, weights, inner, sums, bytes;
    int parts;
    bool wide; // down by 128 columns
};
static MoeSpace moe_space(int64_t T, int64_t E, int64_t k, int64_t H, int64_t I)
{
    const int64_t tokens = T < kTokens ? T : kTokens, choices = tokens * k, most = choices < E ? choices : E;
    const auto rounded = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    MoeSpace m;
    m.chosen = 0;
    m.bits = rounded(4 * choices);
    m.places = m.bits + rounded(8 * tokens * moe_words((int)E));
    m.list = m.places + rounded(tokens * E);
    m.weights = m.list + rounded(4 * (2 + (2 + 2 * kStretch) * moe_most_stretches((int)most, (int)choices)));
    m.inner = m.weights + rounded(4 * choices);
    m.sums = m.inner + rounded(4 * choices * I);
    // Where 16 columns each are too few workgroups of down for the CUs, the blocks are divided too, for a launch more (5 us): a block takes a wave 0.75 us
    // (41 tokens, 4 experts of 320 x 864, of which each token takes all: 20 workgroups 19 us).
    const int64_t groups = H / 16, parts = groups >= 256 ? 1 : 256 / groups;
    const float us = (float)(most + choices / 16) * (float)((I + kF8Block - 1) / kF8Block) * (0.75f / 8);
    m.parts = (int)(parts < kMostParts ? parts : kMostParts);
    if (us * (1.0f - 1.0f / (float)m.parts) < 5.0f) m.parts = 1;
    // By 128 columns (a launch more always, and a barrier for two blocks) where there are many tokens' h and weights to read: 64 tokens that choose 6 of 64 experts
    // of 4096 x 2048 306 us for the layer, by 16 columns 323, 48 that choose 2 of 4 of 4096 x 4096 83 and 88; but 16 that choose 2 of 8 of those 94 and
    // 90, 64 that choose 2 of 16 of 2048 x 1024 40 and 38.
    m.wide = tokens > 16 && H >= 1024 && (most + choices / 16) * H * I >= 100000000;
    if (m.wide) {
        const int64_t groups = (H + 127) / 128;
        m.parts = (int)(groups >= 256 ? 1 : std::min<int64_t>(kMostParts, 256 / groups));
    }
    m.bytes = m.sums + (m.parts > 1 ? rounded(4 * m.parts * tokens * H) : 0);
    return m;
}

static void launch_moe(const MoeArgs &a, bool wide, hipStream_t s)
{
    const dim3 up((unsigned)(a.most * (a.I / 16))), up_and_list((unsigned)(a.most * (a.I / 16) + 1)), down((unsigned)(a.H / 16), (unsigned)a.parts);
    if (a.T <= kFewTokens && a.choices <= kFewChoices && a.E <= 256) {
        if (a.E <= 64) hipLaunchKernelGGL((moe_up_kernel<1, 1>), up, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((moe_up_kernel<1, 4>), up, dim3(256), 0, s, a);
    } else {
        const dim3 tokens((unsigned)a.T);
        if (a.E <= 64) hipLaunchKernelGGL(moe_choose_kernel<1>, tokens, dim3(64), 0, s, a);
        else if (a.E <= 256) hipLaunchKernelGGL(moe_choose_kernel<4>, tokens, dim3(64), 0, s, a);
        else hipLaunchKernelGGL(moe_choose_kernel<kMostExperts / 64>, tokens, dim3(64), 0, s, a);
        if (a.T <= 16) hipLaunchKernelGGL((moe_up_kernel<1, 0>), up_and_list, dim3(256), 0, s, a);
        // With 16 tokens at a time a CU holds more workgroups than the four with 64 at a time, which counts where there are more of them, but weights are read again
        // for experts of more: 64 tokens that choose 8 of 64 experts of 1024 x 2048 113 us and 119, 40 that choose 4 of 64 of 1024 x 1024 55 and 58; but 64
        // that choose 2 of 16 of 2048 x 1024 39 and 38, of 8 of 4096 x 4096 147 and 133.
        else if (a.choices <= 8 * a.most && a.most * (a.I / 16) > 1024) hipLaunchKernelGGL((moe_up_kernel<1, 0, true>), up_and_list, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((moe_up_kernel<kTokens / 16, 0>), up_and_list, dim3(256), 0, s, a);
    }
    if (wide) hipLaunchKernelGGL(moe_down_wide_kernel<kTokens>, dim3((unsigned)((a.H + 127) / 128), (unsigned)a.parts), dim3(512), 0, s, a);
    else if (a.T <= 8) hipLaunchKernelGGL(moe_down_kernel<8>, down, dim3(512), 0, s, a);
    else hipLaunchKernelGGL(moe_down_kernel<kTokens>, down, dim3(512), 0, s, a);
    if (a.sums) hipLaunchKernelGGL(moe_sum_kernel, dim3((unsigned)((a.H + 255) / 256), (unsigned)a.T), dim3(256), 0, s, a);
}

} // namespace qnn

using namespace qnn;

extern "C" {

static bool bad_moe_sizes(int64_t T, int64_t E, int64_t k, int64_t H, int64_t I)
{
    return T < 0 || T > (1 << 20) || E <= 0 || E > kMostExperts || k <= 0 || k > E || k > kMostChosen || H <= 0 || H % 16 != 0 || I <= 0 || I % 16 != 0 || H > (1 << 20) ||
           I > (1 << 17);
}

size_t qnn_f8_moe_workspace_bytes(int64_t T, int64_t E, int64_t top_k, int64_t H, int64_t I)
{
    return bad_moe_sizes(T, E, top_k, H, I) || T == 0 ? 0 : moe_space(T, E, top_k, H, I).bytes;
}

qnn_status qnn_f8_moe(const uint8_t *x, int64_t ldx, const float *x_scales, int64_t ldxs, const void *logits, int64_t ldl, int logit_type, const uint8_t *up,
                      const float *up_scales, const uint8_t *down, const float *down_scales, int64_t T, int64_t E, int64_t top_k, int64_t H, int64_t I,
                      int renormalize, int type, void *y, int64_t ldy, int32_t *experts, float *weights, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_moe_sizes(T, E, top_k, H, I) || bad_half_type(type) || (bad_half_type(logit_type) && logit_type != QNN_F32)) return QNN_EINVAL;
    if (T == 0) return QNN_OK;
    if (!x || !x_scales || !logits || !up || !up_scales || !down || !down_scales || !y || ldx < H || ldx > (1 << 24) || ldxs < T || ldl < E || ldy < H) return QNN_EINVAL;
    if (((uintptr_t)up | (uintptr_t)down) % 16 != 0) return QNN_EINVAL;
    const MoeSpace m = moe_space(T, E, top_k, H, I);
    if (!workspace || ((uintptr_t)workspace & 15) != 0 || workspace_bytes < m.bytes) return QNN_EINVAL;
    uint8_t *const space = static_cast<uint8_t *>(workspace);
    for (int64_t t = 0; t < T; t += kTokens) {
        const int64_t n = T - t < kTokens ? T - t : kTokens;
        MoeArgs a{};
        a.x = x + t * ldx, a.xs = x_scales + t, a.up = up, a.ups = up_scales, a.down = down, a.downs = down_scales;
        a.logits = static_cast<const uint8_t *>(logits) + t * ldl * (logit_type == QNN_F32 ? 4 : 2);
        a.y = static_cast<uint8_t *>(y) + t * ldy * 2;
        a.experts = experts ? experts + t * top_k : nullptr;
        a.weights = weights ? weights + t * top_k : reinterpret_cast<float *>(space + m.weights);
        a.ldx = ldx, a.ldxs = ldxs, a.ldl = ldl, a.ldy = ldy;
        a.T = (int32_t)n, a.E = (int32_t)E, a.k = (int32_t)top_k, a.H = (int32_t)H, a.I = (int32_t)I;
        a.logit_type = logit_type, a.type = type, a.renormalize = renormalize;
        a.chosen = reinterpret_cast<int32_t *>(space + m.chosen), a.bits = reinterpret_cast<uint64_t *>(space + m.bits), a.places = space + m.places;
        a.list = reinterpret_cast<int32_t *>(space + m.list), a.h = reinterpret_cast<uint16_t *>(space + m.inner);
        a.choices = (int32_t)(n * top_k), a.most = a.choices < a.E ? a.choices : a.E;
        a.parts = m.parts, a.sums = m.parts > 1 ? reinterpret_cast<float *>(space + m.sums) : nullptr;
        launch_moe(a, m.wide, as_stream(stream));
    }
    return launch_status(hipGetLastError());
}

} // extern "C"
