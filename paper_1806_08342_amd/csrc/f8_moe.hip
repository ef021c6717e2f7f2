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
#include "f8.h"

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
    int32_t *list;     // number of experts chosen, then each one's number, then where each one's choices begin (one more), then the choices: t * k + place
    uint16_t *h_high, *h_low; // [choice][I]
    int32_t most; // experts that can be chosen
};
__device__ __forceinline__ int32_t *moe_chosen(const MoeArgs &a) { return a.list + 1; }
__device__ __forceinline__ int32_t *moe_begins(const MoeArgs &a) { return a.list + 1 + a.most; }
__device__ __forceinline__ int32_t *moe_choices(const MoeArgs &a) { return a.list + 2 + 2 * a.most; }

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
    float mine = 0.0f, sum = 0.0f, top = 0.0f; // (mine: exp of the logit at place `lane`, less the largest)
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
        if (lane == j) mine = expf(key_logit(best) - top), expert = e;
    }
    const float of = wave_sum(a.renormalize ? mine : sum);
    weight = expert >= 0 ? mine / of : 0.0f;
}

// One workgroup: a wave per token and turn; then the list.
template <int KEYS> __global__ void __launch_bounds__(1024) moe_route_kernel(const MoeArgs a)
{
    __shared__ uint64_t s_tokens[kMostExperts]; // who chose an expert
    __shared__ int16_t s_place[kTokens][kMostChosen];
    __shared__ int32_t s_sum[2][16];
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
    int before = count > 0, times = count;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(before, d), v = __shfl_up(times, d);
        if (lane >= d) before += u, times += v;
    }
    if (lane == 63) s_sum[0][wave] = before, s_sum[1][wave] = times;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before += s_sum[0][w], times += s_sum[1][w];
    int32_t *const begins = moe_begins(a);
    if (tid == 1023) a.list[0] = before, begins[before] = times;
    if (count > 0) {
        int at = times - count;
        moe_chosen(a)[before - 1] = tid;
        begins[before - 1] = at;
        for (int t = 0; t < a.T; ++t) {
            if (!(tokens >> t & 1)) continue;
            int j = 0;
            while (s_place[t][j] != tid) ++j;
            moe_choices(a)[at++] = t * a.k + j;
        }
    }
}

// Workgroups: an expert by 16 columns of h; four waves share H and join their sums in LDS.
template <int MT> __global__ void __launch_bounds__(256) moe_up_kernel(const MoeArgs a)
{
    constexpr int WAVES = 4, DEPTH = 2;
    const int columns = a.I / 16, j = blockIdx.x / columns, i0 = blockIdx.x % columns * 16;
    if (j >= a.list[0]) return;
    const int e = moe_chosen(a)[j], begin = moe_begins(a)[j], count = moe_begins(a)[j + 1] - begin;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int blocks = (a.H + kF8Block - 1) / kF8Block, two = (2 * a.I + kF8Block - 1) / kF8Block;
    const uint8_t *const w_row[2] = {a.up + ((int64_t)e * 2 * a.I + i0 + c) * a.H, a.up + ((int64_t)e * 2 * a.I + a.I + i0 + c) * a.H};
    const float *const w_scale[2] = {a.ups + ((int64_t)e * two + i0 / kF8Block) * blocks, a.ups + ((int64_t)e * two + (a.I + i0) / kF8Block) * blocks};
    const uint8_t *x_row[MT];
    const float *x_scale[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int t = moe_choices(a)[begin + min(mt * 16 + c, count - 1)] / a.k;
        x_row[mt] = a.x + t * a.ldx, x_scale[mt] = a.xs + t;
    }
    f32x4 acc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) acc[mt][0] = acc[mt][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    struct Step {
        w32x4 w[2][2];
        float ws[2];
    };
    const w32x4 zero = {0u, 0u, 0u, 0u};
    const auto piece = [&](const uint8_t *row, int k) { return k < a.H ? load_any<w32x4>(row + k) : zero; }; // (H is a multiple of 16)
    const auto load = [&](Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int u = 0; u < 2; ++u) s.w[u][0] = piece(w_row[u], k), s.w[u][1] = piece(w_row[u], k + 64), s.ws[u] = w_scale[u][b];
    };
    const auto compute = [&](const Step &s, int b) {
        const int k = b * kF8Block + 16 * g;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt * 16 >= count) break;
            const w32x4 x[2] = {piece(x_row[mt], k), piece(x_row[mt], k + 64)};
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
        const int64_t at = (int64_t)moe_choices(a)[begin + m] * a.I + i0 + n;
        a.h_high[at] = high;
        a.h_low[at] = Bf16::narrow(h - Bf16::widen(high));
    }
}

// Workgroups: 16 columns of y.  The blocks of 128 of all experts chosen are shared out among the waves, a stretch for each; a wave's sums of an
// expert go to its own part of LDS, weighted, and the waves' parts are added up at the end.
// Tiles of 8 tokens: the two parts of their h are the 16 columns of one product.  Weights, and h of the first tile, which another XCD may have written,
// are requested two or three blocks ahead (with h one block ahead 64 tokens x 64 experts x 4096 x 2048 took 197 us).
template <int MT> __global__ void __launch_bounds__(512) moe_down_kernel(const MoeArgs a)
{
    constexpr int WAVES = 8, DEPTH = MT == 8 ? 3 : 4;
    __shared__ float s_y[WAVES][8 * MT][17];
    const int n0 = blockIdx.x * 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    for (int i = lane; i < 8 * MT * 17; i += 64) (&s_y[wave][0][0])[i] = 0.0f;
    const int blocks = (a.I + kF8Block - 1) / kF8Block, row_blocks = (a.H + kF8Block - 1) / kF8Block;
    const int units = a.list[0] * blocks;
    const int first = (int)((int64_t)units * wave / WAVES), last = (int)((int64_t)units * (wave + 1) / WAVES);
    const w32x4 zero = {0u, 0u, 0u, 0u};
    const uint16_t *const part_of_h = c < 8 ? a.h_high : a.h_low;
    struct Weights {
        w32x4 w[2];
        float scale;
    };
    struct Inner {
        w32x4 h[4];
    };
    for (int u = first; u < last;) {
        const int j = u / blocks, b0 = u - j * blocks, b1 = min(last - j * blocks, blocks);
        const int e = moe_chosen(a)[j], begin = moe_begins(a)[j], count = moe_begins(a)[j + 1] - begin;
        const uint8_t *const w_row = a.down + ((int64_t)e * a.H + n0 + c) * a.I;
        const float *const w_scale = a.downs + ((int64_t)e * row_blocks + n0 / kF8Block) * blocks;
        f32x4 acc[MT];
        int choice[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            choice[mt] = moe_choices(a)[begin + min(mt * 8 + (c & 7), count - 1)];
            acc[mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const auto load = [&](Weights &f, int b) { // (behind the last: that again, unused)
            const int at = min(b, b1 - 1), k = at * kF8Block + 16 * g;
#pragma unroll
            for (int p = 0; p < 2; ++p) f.w[p] = k + 64 * p < a.I ? load_any<w32x4>(w_row + k + 64 * p) : zero;
            f.scale = w_scale[at];
        };
        const auto load_inner = [&](Inner &h, int b, int mt) {
            const uint16_t *const row = part_of_h + (int64_t)choice[mt] * a.I;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = min(b, b1 - 1) * kF8Block + 16 * g + 64 * (i >> 1) + 8 * (i & 1);
                h.h[i] = mt * 8 + (c & 7) < count && k < a.I ? load_any<w32x4>(row + k) : zero;
            }
        };
        const auto compute = [&](const Weights &f, const Inner &ahead, int b) {
            b16x8 wide[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) wide[i] = widen_codes(f.w[i >> 1][2 * (i & 1)], f.w[i >> 1][2 * (i & 1) + 1]);
            Inner h = ahead;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if (mt * 8 >= count) break;
                Inner next;
                if (mt + 1 < MT && (mt + 1) * 8 < count) load_inner(next, b, mt + 1);
                f32x4 part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 4; ++i) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[i], __builtin_bit_cast(b16x8, h.h[i]), part, 0, 0, 0);
                fma4(acc[mt], part, f.scale);
                // (Here, and not behind the branch: the compiler's waits for the products do not reach over it.)
                asm volatile("" : "+v"(acc[mt]));
                h = next;
            }
        };
        Weights f[DEPTH];
        Inner h[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d) load_inner(h[d], b0 + d, 0), load(f[d], b0 + d);
        for (int b = b0; b < b1; b += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (b + d >= b1) break;
                load_inner(h[(d + DEPTH - 1) % DEPTH], b + d + DEPTH - 1, 0);
                load(f[(d + DEPTH - 1) % DEPTH], b + d + DEPTH - 1);
                compute(f[d], h[d], b + d);
            }
        }
        u = j * blocks + b1;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            if (mt * 8 >= count) break;
            const float weight = a.weights[choice[mt]];
            const int t = choice[mt] / a.k;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = acc[mt][r] + __shfl_xor(acc[mt][r], 8);
                if (c < 8 && mt * 8 + c < count) s_y[wave][t][g * 4 + r] += weight * v;
            }
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < a.T * 16; i += 64 * WAVES) {
        const int t = i / 16, n = i % 16;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += s_y[w][t][n];
        store_out(a.y, t * a.ldy + n0 + n, a.type, v);
    }
}

struct MoeSpace {
    size_t list, weights, high, low, bytes;
    int64_t most;
};
static MoeSpace moe_space(int64_t T, int64_t E, int64_t k, int64_t I)
{
    const int64_t tokens = T < kTokens ? T : kTokens, choices = tokens * k, most = choices < E ? choices : E;
    const auto rounded = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    MoeSpace m;
    m.most = most, m.list = 0;
    m.weights = rounded(4 * (2 + 2 * most + choices));
    m.high = m.weights + rounded(4 * choices);
    m.low = m.high + rounded(2 * choices * I);
    m.bytes = m.low + rounded(2 * choices * I);
    return m;
}

static void launch_moe(const MoeArgs &a, hipStream_t s)
{
    if (a.E <= 64) hipLaunchKernelGGL(moe_route_kernel<1>, dim3(1), dim3(1024), 0, s, a);
    else if (a.E <= 256) hipLaunchKernelGGL(moe_route_kernel<4>, dim3(1), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL(moe_route_kernel<kMostExperts / 64>, dim3(1), dim3(1024), 0, s, a);
    const dim3 up((unsigned)(a.most * (a.I / 16))), down((unsigned)(a.H / 16));
    if (a.T <= 16) hipLaunchKernelGGL(moe_up_kernel<1>, up, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(moe_up_kernel<kTokens / 16>, up, dim3(256), 0, s, a);
    if (a.T <= 8) hipLaunchKernelGGL(moe_down_kernel<1>, down, dim3(512), 0, s, a);
    else if (a.T <= 16) hipLaunchKernelGGL(moe_down_kernel<2>, down, dim3(512), 0, s, a);
    else hipLaunchKernelGGL(moe_down_kernel<kTokens / 8>, down, dim3(512), 0, s, a);
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
    return bad_moe_sizes(T, E, top_k, H, I) || T == 0 ? 0 : moe_space(T, E, top_k, I).bytes;
}

qnn_status qnn_f8_moe(const uint8_t *x, int64_t ldx, const float *x_scales, int64_t ldxs, const void *logits, int64_t ldl, int logit_type, const uint8_t *up,
                      const float *up_scales, const uint8_t *down, const float *down_scales, int64_t T, int64_t E, int64_t top_k, int64_t H, int64_t I,
                      int renormalize, int type, void *y, int64_t ldy, int32_t *experts, float *weights, void *workspace, size_t workspace_bytes, void *stream)
{
    if (bad_moe_sizes(T, E, top_k, H, I) || bad_half_type(type) || (bad_half_type(logit_type) && logit_type != QNN_F32)) return QNN_EINVAL;
    if (T == 0) return QNN_OK;
    if (!x || !x_scales || !logits || !up || !up_scales || !down || !down_scales || !y || ldx < H || ldxs < T || ldl < E || ldy < H) return QNN_EINVAL;
    const MoeSpace m = moe_space(T, E, top_k, I);
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
        a.list = reinterpret_cast<int32_t *>(space + m.list), a.h_high = reinterpret_cast<uint16_t *>(space + m.high);
        a.h_low = reinterpret_cast<uint16_t *>(space + m.low), a.most = (int32_t)m.most;
        launch_moe(a, as_stream(stream));
    }
    return launch_status(hipGetLastError());
}

} // extern "C"
