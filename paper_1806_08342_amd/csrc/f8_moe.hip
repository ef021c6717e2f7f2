// A layer of experts for a few tokens, their weights in e4m3 (qnn_f8_moe): each token's top_k experts by its logits,
//
//   y[t] = sum_e weight[t][e] * down[e] (silu(gate[e] x[t]) * (up[e] x[t]))
//
// Bound by reading the weights of the experts that some token chose, each once.  Three launches for up to 64 tokens: the choice, as a list of the experts
// chosen with their tokens; gate and up, whose product h of each choice goes to the workspace; down, which gathers a token's experts.  No atomics on
// memory: an output is the sum of its experts in the order of their numbers and of parts of K, whatever the order of workgroups.
//
// h keeps 16 significant bits, as two bfloat16 that are added up: in one it would cost the result as much as its own rounding.  Down's weights enter as
// bfloat16 beside it, exactly.
#include "buffer_ops.h"
#include "f8.h"
#include "lds_ring.h"

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
    int32_t *list;     // number of experts chosen, number of stretches; each expert, and where its choices begin (one more); the stretches; the choices: t * k + place
    uint16_t *h; // [2][choices][I]: the two parts
    int32_t most, choices; // experts that can be chosen; choices
    float *sums;           // of parts of the blocks, [parts][T][H], or null
    int32_t parts;
};
__device__ __forceinline__ int32_t *moe_chosen(const MoeArgs &a) { return a.list + 2; }
__device__ __forceinline__ int32_t *moe_begins(const MoeArgs &a) { return a.list + 2 + a.most; }
// up to 8 choices of an expert: the expert, where they begin, how many
constexpr int kStretch = 8;
__device__ __forceinline__ int32_t *moe_stretches(const MoeArgs &a) { return a.list + 3 + 2 * a.most; }
__host__ __device__ __forceinline__ int moe_most_stretches(int most, int choices) { return most + choices / kStretch; }
__device__ __forceinline__ int32_t *moe_choices(const MoeArgs &a) { return moe_stretches(a) + 3 * moe_most_stretches(a.most, a.choices); }

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

// One workgroup: a wave per token and turn; then the list.
template <int KEYS> __global__ void __launch_bounds__(1024) moe_route_kernel(const MoeArgs a)
{
    __shared__ uint64_t s_tokens[kMostExperts]; // who chose an expert
    __shared__ int16_t s_place[kTokens][kMostChosen];
    __shared__ int32_t s_sum[3][16], s_begin[kMostExperts];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    s_tokens[tid] = 0;
    __syncthreads();
    for (int t = wave; t < a.T; t += 16) {
        int expert;
        float weight;
        choose<KEYS>(a, t, expert, weight);
        if (lane < a.k) {
            s_place[t][lane] = (int16_t)expert;
            if (expert >= 0) atomicOr(reinterpret_cast<unsigned long long *>(&s_tokens[expert]), 1ull << t);
            a.weights[t * a.k + lane] = weight;
            if (a.experts) a.experts[t * a.k + lane] = expert;
        }
    }
    __syncthreads();
    // thread e: how many experts before it were chosen, and how often
    const uint64_t tokens = s_tokens[tid];
    const int count = __popcll(tokens);
    const int parts = (count + kStretch - 1) / kStretch;
    int before = count > 0, times = count, stretch = parts;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(before, d), v = __shfl_up(times, d), w = __shfl_up(stretch, d);
        if (lane >= d) before += u, times += v, stretch += w;
    }
    if (lane == 63) s_sum[0][wave] = before, s_sum[1][wave] = times, s_sum[2][wave] = stretch;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += s_sum[0][w], times += s_sum[1][w], stretch += s_sum[2][w];
    int32_t *const begins = moe_begins(a);
    if (tid == 1023) a.list[0] = before, a.list[1] = stretch, begins[before] = times;
    s_begin[tid] = times - count;
    if (count > 0) {
        moe_chosen(a)[before - 1] = tid;
        begins[before - 1] = times - count;
        for (int i = 0; i < parts; ++i) {
            int32_t *const to = moe_stretches(a) + 3 * (stretch - parts + i);
            to[0] = tid, to[1] = times - count + i * kStretch, to[2] = min(count - i * kStretch, kStretch);
        }
    }
    __syncthreads();
    for (int i = tid; i < a.T * a.k; i += 1024) { // each choice behind those of the tokens before
        const int t = i / a.k, e = s_place[t][i - t * a.k];
        if (e >= 0) moe_choices(a)[s_begin[e] + __popcll(s_tokens[e] & ((1ull << t) - 1))] = i;
    }
}

// Up to 64 choices of up to 8 tokens, listed by every workgroup for itself (experts in the order in which they are first chosen): the choices of
// expert j, as bits.  The first workgroup writes the lists for what follows.  One launch less: a token's layer 42 -> 37 us.
constexpr int kFewTokens = 8, kFewChoices = 64;
template <int KEYS> __device__ __forceinline__ uint64_t moe_route_few(const MoeArgs &a, int j, int &expert)
{
    __shared__ int16_t s_expert[kFewChoices];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (threadIdx.x < kFewChoices) s_expert[threadIdx.x] = -1;
    __syncthreads();
    for (int t = wave; t < a.T; t += 4) {
        int e;
        float weight;
        choose<KEYS>(a, t, e, weight);
        if (lane < a.k) {
            s_expert[t * a.k + lane] = (int16_t)e;
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
        int before = 0; // choices of the experts before
        for (uint64_t rest = firsts; rest; rest &= rest - 1) {
            const int l = __ffsll((unsigned long long)rest) - 1;
            const uint64_t theirs = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(same >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)same, l);
            if (theirs >> lane & 1) moe_choices(a)[before + __popcll(theirs & below)] = lane;
            const int count = __popcll(theirs);
            if (lane < (count + kStretch - 1) / kStretch) {
                // (of an expert chosen by 8 tokens there is one stretch)
                int32_t *const to = moe_stretches(a) + 3 * __builtin_amdgcn_readlane(at, l);
                to[0] = __builtin_amdgcn_readlane(e, l), to[1] = before, to[2] = count;
            }
            before += count;
        }
        if (lane == 0) a.list[0] = a.list[1] = __popcll(firsts);
    }
    const uint64_t who = __ballot(first && at == j);
    if (who == 0) return 0;
    const int l = __ffsll((unsigned long long)who) - 1;
    expert = __builtin_amdgcn_readlane(e, l);
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(same >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)same, l);
}

// Workgroups: an expert by 16 columns of h; four waves share H and join their sums in LDS.
// KEYS: 0: the lists are there; else the workgroup chooses by itself, from so many times 64 logits.
template <int MT, int KEYS> __global__ void __launch_bounds__(256) moe_up_kernel(const MoeArgs a)
{
    constexpr int WAVES = 4, DEPTH = 2;
    __shared__ int32_t s_choice[KEYS ? kFewTokens : 1];
    const int columns = a.I / 16, j = blockIdx.x / columns, i0 = blockIdx.x % columns * 16;
    int e, count;
    const int32_t *choices = s_choice;
    if constexpr (KEYS == 0) {
        if (j >= a.list[0]) return;
        e = moe_chosen(a)[j];
        const int begin = moe_begins(a)[j];
        count = moe_begins(a)[j + 1] - begin, choices = moe_choices(a) + begin;
    } else {
        const uint64_t mine = moe_route_few<KEYS>(a, j, e);
        if (mine == 0) return;
        count = __popcll(mine);
        if (threadIdx.x < 64 && (mine >> threadIdx.x & 1)) s_choice[__popcll(mine & ((1ull << threadIdx.x) - 1))] = threadIdx.x;
        __syncthreads();
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int blocks = (a.H + kF8Block - 1) / kF8Block, two = (2 * a.I + kF8Block - 1) / kF8Block;
    const uint8_t *const w_rows[2] = {a.up + ((int64_t)e * 2 * a.I + i0) * a.H, a.up + ((int64_t)e * 2 * a.I + a.I + i0) * a.H};
    const float *const w_scale[2] = {a.ups + ((int64_t)e * two + i0 / kF8Block) * blocks, a.ups + ((int64_t)e * two + (a.I + i0) / kF8Block) * blocks};
    const int x_bytes = (int)(a.T * a.ldx); // (below 2^30)
    uint32_t x_row[MT];
    const float *x_scale[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int t = choices[min(mt * 16 + c, count - 1)] / a.k;
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
    const auto load = [&](Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s.w[u][0] = piece(w_rows[u], 16 * a.H, (uint32_t)(c * a.H), k), s.w[u][1] = piece(w_rows[u], 16 * a.H, (uint32_t)(c * a.H), k + 64);
            s.ws[u] = w_scale[u][b];
        }
    };
    const auto compute = [&](const Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt * 16 >= count) break;
            const w32x4 x[2] = {piece(a.x, x_bytes, x_row[mt], k), piece(a.x, x_bytes, x_row[mt], k + 64)};
            const float xs = x_scale[mt][b * a.ldxs];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                fma4(acc[mt][u], f8_products<true>(s.w[u], x), xs * s.ws[u]);
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
    __shared__ float s_acc[WAVES][2][16 * MT][20];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int u = 0; u < 2; ++u) *reinterpret_cast<f32x4 *>(&s_acc[wave][u][mt * 16 + c][g * 4]) = acc[mt][u];
    __syncthreads();
    for (int i = threadIdx.x; i < min(count, 16 * MT) * 16; i += 64 * WAVES) {
        const int m = i / 16, n = i % 16;
        float gate = 0.0f, up = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) gate += s_acc[w][0][m][n], up += s_acc[w][1][m][n];
        const float h = gate / (1.0f + expf(-gate)) * up;
        const uint16_t high = Bf16::narrow(h);
        const int64_t at = (int64_t)choices[m] * a.I + i0 + n;
        a.h[at] = high;
        a.h[(int64_t)a.choices * a.I + at] = fabsf(h) < INFINITY ? Bf16::narrow(h - Bf16::widen(high)) : 0; // (of an infinity the first part is all)
    }
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
// than the memory over the weights (64 tokens, 64 experts of 4096 x 2048: 93 us for the weights alone, 172 with h).
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
    const int units = a.list[1] * blocks;
    const int sharing = WAVES * a.parts, mine = part * WAVES + wave;
    const int first = (int)((int64_t)units * mine / sharing), last = (int)((int64_t)units * (mine + 1) / sharing);
    const uint8_t *const inner = reinterpret_cast<const uint8_t *>(a.h);
    const int inner_bytes = 4 * a.choices * a.I; // (up to 2^30)
    constexpr uint32_t kBeyond = 0x80000000u;    // of either buffer: zeros, without traffic
    // 16 rows of 128 bytes, 16-byte pieces exchanged by half the row's number, so that reads of 16 rows meet the 16 places of the 64 banks; a
    // copy's lanes have 8 rows, from `half` * 8 on
    const auto piece = [&](int half) { return (lane & 7) ^ (lane >> 4) ^ 4 * half; };
    const uint32_t w_place = lds_address(w_ring) + c * 128 + (g ^ (c >> 1 & 7)) * 16, h_place = lds_address(h_ring) + c * 128 + (2 * g ^ (c >> 1 & 7)) * 16;
    for (int u = first; u < last;) {
        const int j = u / blocks, b0 = u - j * blocks, many = min(last - j * blocks, blocks) - b0;
        const int32_t *const stretch = moe_stretches(a) + 3 * j;
        const int e = stretch[0], begin = stretch[1], count = stretch[2];
        const uint8_t *const w_rows = a.down + ((int64_t)e * a.H + n0) * a.I;
        const float *const w_scale = a.downs + ((int64_t)e * row_blocks + n0 / kF8Block) * blocks;
        // Each workgroup begins at another block: rows lie a power of two apart more often than not, and workgroups that read the same columns of
        // all rows at one time would keep to a part of the memory's channels.
        const int turned = (int)(blockIdx.x % (unsigned)many);
        const auto block_at = [&](int i) { return b0 + (i + turned < many ? i + turned : i + turned - many); };
        const uint32_t copied = 2u * (uint32_t)(moe_choices(a)[begin + min(lane >> 3, count - 1)] * a.I) | (lane >> 3 < count ? 0u : kBeyond);
        // (Without branches, so that the compiler's count of what is on its way holds: behind the last block nothing is below the end.)
        const auto end_of = [&](int i) { return a.I & ((i - many) >> 31); };
        const auto load = [&](float &scale, int i) {
            const int b = block_at(min(i, many - 1)), end = end_of(i);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int k = b * kF8Block + 16 * piece(half);
                buffer_to_lds16(w_rows, 16 * a.I, (uint32_t)((8 * half + (lane >> 3)) * a.I + k) | (k < end ? 0u : kBeyond), w_ring + (i & 3) * W_SLOT + half * 1024);
            }
            scale = w_scale[b];
        };
        const auto load_inner = [&](int i) {
            const int b = block_at(min(i, many - 1)), end = end_of(i);
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const int k = b * kF8Block + 64 * p + 8 * piece(part);
                    buffer_to_lds16(inner, inner_bytes, (copied + 2u * (uint32_t)(part * a.choices * a.I + k)) | (k < end ? 0u : kBeyond),
                                    h_ring + (i & 1) * H_SLOT + p * 2048 + part * 1024);
                }
        };
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const auto compute = [&](int i, float scale) {
            w32x4 w[2], v[4];
            const uint32_t w_at = w_place + (i & 3) * W_SLOT, h_at = h_place + (i & 1) * H_SLOT;
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
        float scale[4];
        wait_vmcnt<0>();
        load_inner(0);
#pragma unroll
        for (int d = 0; d < 3; ++d) load(scale[d], d);
        for (int i = 0; i < many; i += 4) {
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                if (i + d >= many) break;
                load_inner(i + d + 1);
                load(scale[(d + 3) & 3], i + d + 3);
                wait_vmcnt<3 + 4 + 3>(); // but the weights of the two blocks ahead and these
                compute(i + d, scale[d]);
            }
        }
        u = j * blocks + b0 + many;
        const int choice = moe_choices(a)[begin + min(c & 7, count - 1)];
        const float weight = a.weights[choice];
        const int t = choice / a.k;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float v = acc[r] + __shfl_xor(acc[r], 8);
            if (c < 8 && c < count) s_y[wave][t][g * 4 + r] += weight * v;
        }
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

// y = the parts' sums in their order
__global__ void __launch_bounds__(256) moe_sum_kernel(const MoeArgs a)
{
    const int n = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (n >= a.H) return;
    float v = 0.0f;
    for (int p = 0; p < a.parts; ++p) v += a.sums[((int64_t)p * a.T + t) * a.H + n];
    store_out(a.y, t * a.ldy + n, a.type, v);
}

struct MoeSpace {
    size_t list, weights, inner, sums, bytes;
    int64_t most;
    int parts;
};
static MoeSpace moe_space(int64_t T, int64_t E, int64_t k, int64_t H, int64_t I)
{
    const int64_t tokens = T < kTokens ? T : kTokens, choices = tokens * k, most = choices < E ? choices : E;
    const auto rounded = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    MoeSpace m;
    m.most = most, m.list = 0;
    m.weights = rounded(4 * (3 + 2 * most + 3 * moe_most_stretches((int)most, (int)choices) + choices));
    m.inner = m.weights + rounded(4 * choices);
    m.sums = m.inner + rounded(4 * choices * I);
    // A workgroup of down has 48 KB on its way, 20 KB/us; where 16 columns each are too few of them for the memory, the blocks are divided too, for a launch
    // more (4 us).
    const int64_t groups = H / 16, parts = groups >= 256 ? 1 : (256 + groups - 1) / groups;
    m.parts = (int)(parts < 8 ? parts : 8);
    const float us = (float)most * (float)H * (float)I / ((float)groups * 20e3f);
    if (us * (1.0f - 1.0f / (float)m.parts) < 4.0f) m.parts = 1;
    m.bytes = m.sums + (m.parts > 1 ? rounded(4 * m.parts * tokens * H) : 0);
    return m;
}

static void launch_moe(const MoeArgs &a, hipStream_t s)
{
    const dim3 up((unsigned)(a.most * (a.I / 16))), down((unsigned)(a.H / 16), (unsigned)a.parts);
    if (a.T <= kFewTokens && a.choices <= kFewChoices && a.E <= 256) {
        if (a.E <= 64) hipLaunchKernelGGL((moe_up_kernel<1, 1>), up, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((moe_up_kernel<1, 4>), up, dim3(256), 0, s, a);
    } else {
        if (a.E <= 64) hipLaunchKernelGGL(moe_route_kernel<1>, dim3(1), dim3(1024), 0, s, a);
        else if (a.E <= 256) hipLaunchKernelGGL(moe_route_kernel<4>, dim3(1), dim3(1024), 0, s, a);
        else hipLaunchKernelGGL(moe_route_kernel<kMostExperts / 64>, dim3(1), dim3(1024), 0, s, a);
        if (a.T <= 16) hipLaunchKernelGGL((moe_up_kernel<1, 0>), up, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((moe_up_kernel<kTokens / 16, 0>), up, dim3(256), 0, s, a);
    }
    if (a.T <= 8) hipLaunchKernelGGL(moe_down_kernel<8>, down, dim3(512), 0, s, a);
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
        a.list = reinterpret_cast<int32_t *>(space + m.list), a.h = reinterpret_cast<uint16_t *>(space + m.inner);
        a.most = (int32_t)m.most, a.choices = (int32_t)(n * top_k);
        a.parts = m.parts, a.sums = m.parts > 1 ? reinterpret_cast<float *>(space + m.sums) : nullptr;
        launch_moe(a, as_stream(stream));
    }
    return launch_status(hipGetLastError());
}

} // extern "C"
