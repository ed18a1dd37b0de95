// A router's choice: every token's experts by their scores, the weights that their results are added up with, and the gradient of
// the weights in the logits.
//
// Keys are compared as 64-bit numbers hold them: a score next to a border falls on the same side as in the definition.  A key travels
// as the 64-bit integer that has its order (a NaN above all), 0 for an expert that is not to be chosen.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

__device__ __forceinline__ uint64_t key_of(double v)
{
    if (v != v) return ~0ull;
    const uint64_t u = __builtin_bit_cast(uint64_t, v + 0.0);       // (one zero)
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double of_key(uint64_t k)
{
    return __builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
}

__device__ __forceinline__ double sigmoid(double x) { return 1.0 / (1.0 + exp(-x)); }

template <class T>
__device__ __forceinline__ float logit(const T *row, uint32_t e) { return (float)row[e]; }

__device__ __forceinline__ double wave_max(double v)
{
    return lanes_fold(v, [](double a, double b) { return a != a || a > b ? a : b; });
}
__device__ __forceinline__ double wave_sum(double v)
{
    return lanes_fold(v, [](double a, double b) { return a + b; });
}

// The weights of a wave's chosen experts, one to a lane: x the logit, in: whether the lane has one, all: what a softmax that is not
// renormalised divides by, with `most` taken off the logits.  Renormalised scores are divided by the largest of them first, so that none is lost
// for being small.
__device__ __forceinline__ double chosen_share(const seer_choice &how, float x, bool in, double most, double all)
{
    const double v = (double)x;
    if (!how.renormalise) return !in ? 0.0 : how.score == SEER_SIGMOID ? sigmoid(v) : exp(v - most) / all;
    double top = wave_max(in ? v : -INFINITY);
    double s = 0;
    if (how.score == SEER_SIGMOID) {
        if (!(top < 0)) top = 0;
        s = v > 0 ? 1.0 / (1.0 + exp(-v)) : exp(v - top) / (1.0 + exp(v));
    } else
        s = exp(v - top);
    if (!in) s = 0;
    const double sum = wave_sum(s);
    return in ? s / sum : 0.0;
}

// The choice of one token by a whole wave, in 64 bits; lane l has the experts l, 64 + l, ...  16 384 tokens of 1024 experts 102 us.  s_key: LDS of the wave, [experts], with groups.
template <class T, int PER>
__device__ __noinline__ void choose_exactly(const T *logits, int64_t ld, uint32_t t, uint32_t experts, const float *bias, const seer_choice &how, int32_t *expert,
                               float *weight, uint64_t *s_key)
{
    const uint32_t lane = threadIdx.x & 63;
    const bool grouped = how.best_groups < how.groups;
    const T *row = logits + (int64_t)t * ld;
    float x[PER];
    uint64_t key[PER];
    double most = -INFINITY, all = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t e = i * 64 + lane;
        x[i] = e < experts ? logit(row, e) : -INFINITY;
        most = x[i] != x[i] || x[i] > most ? (double)x[i] : most;
    }
    const bool scored = bias || (grouped && how.group_best == 2) || !how.renormalise;
    if (how.score == SEER_SOFTMAX && scored) {
        most = wave_max(most);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (x[i] != -INFINITY) all += exp((double)x[i] - most);
        all = wave_sum(all);
    }
    const auto score = [&](float v) { return how.score == SEER_SIGMOID ? sigmoid((double)v) : exp((double)v - most) / all; };
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t e = i * 64 + lane;
        const float b = bias && e < experts ? bias[e] : 0.0f;
        key[i] = x[i] == -INFINITY || b == -INFINITY ? 0 : key_of(bias ? score(x[i]) + (double)b : (double)x[i]);
    }
    if (grouped) {
        uint64_t *mine = s_key;
        const uint32_t length = experts / how.groups;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t e = i * 64 + lane;
            if (e < experts) mine[e] = key[i] == 0 || how.group_best == 1 || bias ? key[i] : key_of(score(x[i]));
        }
        __builtin_amdgcn_wave_barrier();
        uint64_t best = 0, second = 0;
        if (lane < (uint32_t)how.groups) {
            for (uint32_t j = 0; j < length; ++j) {
                const uint64_t k = mine[lane * length + j];
                second = max(second, min(best, k));
                best = max(best, k);
            }
            if (how.group_best == 2 && second) best = key_of((best == ~0ull ? NAN : of_key(best)) + (second == ~0ull ? NAN : of_key(second)));
        }
        uint32_t rank = 0;
        for (uint32_t g = 0; g < (uint32_t)how.groups; ++g) {
            const uint64_t other = __shfl(best, (int)g, 64);
            rank += other > best || (other == best && g < lane);
        }
        const uint64_t open = __ballot(lane < (uint32_t)how.groups && rank < (uint32_t)how.best_groups);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t e = i * 64 + lane;
            if (e < experts && !(open >> (e / length) & 1)) key[i] = 0;
        }
    }
    int32_t chosen = -1;                            // of the lane's number
    for (int k = 0; k < how.choices; ++k) {
        uint64_t best = 0;
        uint32_t at = ~0u;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (key[i] > best) {
                best = key[i];
                at = i * 64 + lane;
            }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t other = __shfl_xor(best, d, 64);
            const uint32_t there = __shfl_xor(at, d, 64);
            if (other > best || (other == best && there < at)) {
                best = other;
                at = there;
            }
        }
        if (best == 0) break;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (at == i * 64 + lane) key[i] = 0;
        if ((int)lane == k) chosen = (int32_t)at;
    }
    double share = chosen_share(how, chosen >= 0 ? logit(row, (uint32_t)chosen) : 0.0f, chosen >= 0, most, all);
    if (all != all && chosen >= 0) share = all;             // (what makes a softmax NaN need not be among the chosen)
    if ((int)lane < how.choices) {
        const size_t to = (size_t)t * how.choices + lane;
        expert[to] = chosen;
        weight[to] = (float)((double)how.factor * share);
    }
}

template <class T, int PER>
__global__ __launch_bounds__(kWG) void choose_kernel(const T *__restrict__ logits, int64_t ld, uint32_t tokens, uint32_t experts,
                                                     const float *__restrict__ bias, seer_choice how, int32_t *__restrict__ expert,
                                                     float *__restrict__ weight)
{
    extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];          // [waves][experts], with groups
    const uint32_t wave = threadIdx.x / 64;
    for (uint32_t t = blockIdx.x * (kWG / kWave) + wave; t < tokens; t += gridDim.x * (kWG / kWave))
        choose_exactly<T, PER>(logits, ld, t, experts, bias, how, expert, weight, s_key + (size_t)wave * experts);
}

// ------------------------------------------------------------------ four tokens to a wave
//
// 16 lanes to a token, a lane with PER consecutive experts; keys in 32 bits, with bounds on what they may be off by.  A token whose choice the
// bounds leave open is chosen again by the whole wave, in 64 bits.
//
// A key travels with its expert in one word: the 24 upper bits (23 with more than 256 experts) of the number that has the key's order, and 255 less
// the expert's number (511); the next best is the largest word below the last one.  Keys that are made of scores are taken less the largest of them, so
// that what is cut off is 2^-15 (2^-14) of the distance from the best.  The bounds on a score: of a sigmoid, 2^-21 (an exponential with an error
// of 2^-23 and 1.5 |x| 2^-24 of itself, times s (1 - s), where s (1 - s) |x| < 0.23; a sum and a reciprocal, 1.5 * 2^-23); of a softmax, 2^-18 of
// the largest (such exponentials, s |x - max| < 0.4 max s, a lane's sum by halves, in 64 bits from there, a reciprocal and a product).  A bias adds 2^-24 of the key.
// Without a bias keys are logits, and exact.
//
// Bound by instructions: 65 536 tokens of 256 experts, eight choices, fp32: sigmoids, bias and 8 groups 61 us (190 with a wave to a token in 64
// bits; the logits alone are read in 13), softmax without either 29, over all experts 35; 16 411 of 160 in bf16, 8 groups 11 (46).
//
// As many experts and choices as the form holds (9 bits of a word number an expert, a lane of 16 takes a choice, one shows what comes next); there
// it is still ahead.  16 384 tokens, softmax, this form and the other one: 64 experts, two choices 8.6 and 19, 15 choices 18 and 58; 256, 15 choices 21 and
// 58; 512, 10 choices 27 and 57, 15 choices 39 and 76; one token of 512, 15 choices 5.5 and 15.  Behind, 16 choices of 512 take 80, 10 of 513 112.
constexpr uint32_t kRowBlocks = 1024 /* as many as there is room for; a wave then goes on to other tokens */;
constexpr uint32_t kRowLanes = 16, kFastChoices = 15, kFastExperts = 512;
constexpr float kFar = 0x1p100f;    // above it sums of two keys, and distances from the best one, may be infinite in 32 bits
constexpr float kSigmoidError = 0x1p-21f, kSoftmaxError = 0x1p-18f;

// The other lanes of 16: fold with the same result in all of them.
template <int CTRL>
__device__ __forceinline__ uint32_t row_move(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
template <int CTRL>
__device__ __forceinline__ float row_move(float v) { return dpp_f<CTRL>(v); }
template <int CTRL>
__device__ __forceinline__ double row_move(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)row_move<CTRL>((uint32_t)(u >> 32)) << 32 | row_move<CTRL>((uint32_t)u));
}
template <class V, class F>
__device__ __forceinline__ V row_fold(V v, F f)
{
    v = f(v, row_move<0xB1>(v));
    v = f(v, row_move<0x4E>(v));
    v = f(v, row_move<0x141>(v));
    return f(v, row_move<0x140>(v));
}
template <class V>
__device__ __forceinline__ V row_sum(V v)
{
    return row_fold(v, [](V a, V b) { return a + b; });
}
__device__ __forceinline__ float row_max(float v)
{
    return row_fold(v, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ uint32_t word_of(float key)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, key + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_word(uint32_t w)
{
    return __builtin_bit_cast(float, w >> 31 ? w & 0x7fffffffu : ~w);
}

// f with the 15 other lanes' values in turn, and from which lane they are.
template <int N = 1, class F>
__device__ __forceinline__ void other_lanes(F f)
{
    if constexpr (N < (int)kRowLanes) {
        f(std::integral_constant<int, 0x120 + N>{}, (threadIdx.x - N) & (kRowLanes - 1));
        other_lanes<N + 1>(f);
    }
}

__device__ __forceinline__ float fast_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// e^x for x <= 0 to 2^-42 of itself: 2^n times the series of e^f up to f^10 / 10!, |f| <= ln(2) / 2.  (Numbers that are made where they are used: those of the
// library's exponential are kept in 22 registers from token to token.)
__device__ __forceinline__ double exp_below_0(double x)
{
    x = x < -1100.0 ? -1100.0 : x;
    const double n = rint(x * 0x1.71547652b82fep+0), f = fma(n, -0x1.62e42fefa39efp-1, x);
    const auto here = [](double c) {
        asm volatile("" : "+s"(c));
        return c;
    };
    double p = here(1.0 / 3628800);
    p = fma(p, f, here(1.0 / 362880));
    p = fma(p, f, here(1.0 / 40320));
    p = fma(p, f, here(1.0 / 5040));
    p = fma(p, f, here(1.0 / 720));
    p = fma(p, f, here(1.0 / 120));
    p = fma(p, f, here(1.0 / 24));
    p = fma(p, f, here(1.0 / 6));
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return x != x ? x : ldexp(p, (int)n);               // (a NaN is no int)
}

// The weights of the experts chosen for a token, one to a lane of 16: as chosen_share, and in 64 bits as there; only the sum that a softmax over all experts
// divides by has terms in 32.  (65 536 tokens of 256 experts, eight choices: 1.8 us longer than in 32 bits, which were off by up to 4e-7 of a weight.)
// rest: 1 less a sigmoid's score, for its gradient.
__device__ __forceinline__ double row_share(const seer_choice &how, float x, bool in, float most, double all, double *rest = nullptr)
{
    const double v = (double)x;
    const float top = how.renormalise ? row_max(in ? x : -INFINITY) : most;
    const bool sigmoid = how.score == SEER_SIGMOID && !(how.renormalise && top < -600.0f);      // (e^x: what 64 bits do not hold counts from the largest)
    const double z = exp_below_0(!in ? 0.0 : sigmoid ? -fabs(v) : v - (double)top);
    double s = in ? sigmoid && v > 0 ? 1.0 : z : 0.0;
    if (how.score == SEER_SIGMOID) {
        const double q = sigmoid ? 1.0 / (1.0 + z) : 1.0;
        s *= q;
        if (rest) *rest = sigmoid && v > 0 ? z * q : q;
    }
    const double sum = how.renormalise ? row_sum(s) : all;
    return (how.renormalise || how.score == SEER_SOFTMAX) && in ? s / sum : s;
}

// The sum of a lane's values by halves.
template <int N, class F>
__device__ __forceinline__ float sum_of(F f, int from = 0)
{
    if constexpr (N == 1) return f(from);
    else return sum_of<N / 2>(f, from) + sum_of<N - N / 2>(f, from + N / 2);
}

// per: the experts of a lane; VEC: rows are read 4 elements at a time.  group_lanes: lanes to a group, 0 without groups.
template <class T, int PER, bool VEC, bool BIAS>
__global__ __launch_bounds__(kWG, PER > 16 ? 2 : 4) void choose_rows_kernel(const T *__restrict__ logits, int64_t ld, uint32_t tokens, uint32_t experts, uint32_t per,
                                                          uint32_t group_lanes, const float *__restrict__ bias, seer_choice how,
                                                          int32_t *__restrict__ expert, float *__restrict__ weight)
{
    extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];          // [waves][experts], with groups
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, l = lane & (kRowLanes - 1);
    constexpr uint32_t NUMBERS = PER > 16 ? 512 : 256, NUMBER = NUMBERS - 1;       // of experts; the bits of a word that hold one
    constexpr float kCut = PER > 16 ? 0x1p-14f : 0x1p-15f;
    const bool two = group_lanes && how.group_best == 2;
    const auto bits = [](float v) { return __builtin_bit_cast(uint32_t, v); };
    float b[BIAS ? PER : 1];
    if constexpr (BIAS) {
#pragma unroll
        for (int i = 0; i < PER; ++i) b[i] = bias[min(l * per + i, experts - 1)];
    }
    for (uint32_t t0 = (blockIdx.x * (kWG / kWave) + wave) * 4; t0 < tokens; t0 += gridDim.x * kWG / kRowLanes) {
        const uint32_t t = t0 + lane / kRowLanes;
        const T *row = logits + (int64_t)min(t, tokens - 1) * ld;
        float x[PER];
        if constexpr (VEC) {
            typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
#pragma unroll
            for (int i = 0; i < PER; i += 4) {
                const uint32_t e = l * per + i;
                const bool in = e < experts && (uint32_t)i < per;
                four v = {};
                if (in) v = *reinterpret_cast<const four *>(row + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i + j] = in ? (float)v[j] : -INFINITY;
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) x[i] = l * per + i < experts && (uint32_t)i < per ? (float)row[l * per + i] : -INFINITY;
        }
        // keys: scores with the bias, or logits; -infinity is not to be chosen
        float key[PER], most = -INFINITY, score_error = kSigmoidError, by = 0;
        double all = 0;
        if (how.score == SEER_SOFTMAX && (BIAS || two || !how.renormalise)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) most = fmaxf(most, x[i]);
            most = row_max(most);
            most = most == -INFINITY ? 0 : most;
            all = row_sum((double)sum_of<PER>([&](int i) { return __expf(x[i] - most); }));
            by = all > 0 ? __builtin_amdgcn_rcpf((float)all) : 0;
            score_error = kSoftmaxError * by;
        }
        const auto score = [&](float v) { return how.score == SEER_SIGMOID ? fast_sigmoid(v) : __expf(v - most) * by; };
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = x[i] == -INFINITY ? x[i] : score(x[i]) + b[i];
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) key[i] = x[i];
        }
        // another number that is not finite leaves the token to 64 bits
        bool unsure = all != all, open = true;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) top = max(top, bits(key[i]) & 0x7fffffffu);
        if (__ballot(top >= 0x7f800000u)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) unsure = unsure || (bits(key[i]) != 0xff800000u && (bits(key[i]) & 0x7fffffffu) >= 0x7f800000u);
        }
        if (group_lanes) {
            float first = -INFINITY, second = -INFINITY;
            if (BIAS || !two) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    second = __builtin_amdgcn_fmed3f(first, second, key[i]);
                    first = fmaxf(first, key[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const float v = x[i] == -INFINITY ? x[i] : score(x[i]);
                    second = __builtin_amdgcn_fmed3f(first, second, v);
                    first = fmaxf(first, v);
                }
            }
            const auto meet = [&](float f, float sec) {
                second = fmaxf(fminf(first, f), fmaxf(second, sec));
                first = fmaxf(first, f);
            };
            if (group_lanes > 1) meet(row_move<0xB1>(first), row_move<0xB1>(second));
            if (group_lanes > 2) meet(row_move<0x4E>(first), row_move<0x4E>(second));
            if (group_lanes > 4) meet(row_move<0x141>(first), row_move<0x141>(second));
            const uint32_t room = (uint32_t)how.best_groups * group_lanes;          // in lanes, as the counts
            uint32_t above = 0;
            if (BIAS || two) {
                float worth = first;
                if (two && second != -INFINITY) worth += second;
                unsure = unsure || worth > kFar;
                // a group with none stays at -infinity, behind sums that are
                const bool there = first != -INFINITY;
                if (there) worth = fmaxf(worth, -0x1.fffffep127f);
                const float size = row_max(there ? fmaxf(fabsf(first), second == -INFINITY ? 0.0f : fabsf(second)) : 0.0f);
                const float near = 4 * score_error + size * 0x1p-21f;
                uint32_t not_below = 0;
                other_lanes([&](auto ctrl, uint32_t) {
                    const float gap = row_move<decltype(ctrl)::value>(worth) - worth;
                    above += gap > near;
                    not_below += gap >= -near;
                });
                open = above < room;
                // (the own group's other lanes are level with it; whether a group with none is open is nothing to the choice)
                unsure = unsure || (there && open && not_below - (group_lanes - 1) >= room);
            } else {
                // exact: a group with none is -infinity, behind the lowest number
                const uint32_t mine = l & ~(group_lanes - 1);
                other_lanes([&](auto ctrl, uint32_t from) {
                    const float other = row_move<decltype(ctrl)::value>(first);
                    above += other > first || (other == first && from < mine);
                });
                open = above < room;
            }
        }
        uint32_t word[PER], none;
        const uint32_t kept = open ? ~NUMBER : 0;
        float size = 0;
        if constexpr (BIAS) {
            float best = -INFINITY;
#pragma unroll
            for (int i = 0; i < PER; ++i) best = fmaxf(best, key[i]);
            best = row_max(open ? best : -INFINITY);
            best = best == -INFINITY ? 0 : best;
            unsure = unsure || best > kFar;
            // (what is below the best in an open group; what is above it is in a closed one)
#pragma unroll
            for (int i = 0; i < PER; ++i) word[i] = (~bits(fmaxf(best - key[i], 0.0f)) & kept) | (NUMBER - (l * per + i));
            size = fabsf(best) + 2;
            none = ~0x7f800000u | NUMBER;                            // an infinite distance, or less
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) word[i] = (word_of(key[i]) & kept) | (NUMBER - (l * per + i));
            none = ~0xff800000u | NUMBER;                            // -infinity
        }
        uint32_t last = 0, mine = 0;                        // lane k takes the k-th word
        for (int k = 0; k <= how.choices; ++k) {
            uint32_t next = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) next = max(next, word[i] - last);
            next = row_fold(next, [](uint32_t a, uint32_t c) { return max(a, c); }) + last;
            // (nothing below the last word: what comes out is that word or one above it)
            if (next <= none || (k > 0 && (last == 0 || next >= last))) next = 0;
            mine = (int)l == k ? next : mine;
            last = next;
        }
        const bool in = mine != 0 && (int)l < how.choices;
        const uint32_t at = min(NUMBER - (mine & NUMBER), experts - 1);
        const float xl = mine ? (float)row[at] : 0.0f;
        {
            const uint32_t after = row_move<0x101>(mine);   // of the next lane
            const float xa = row_move<0x101>(xl);
            const bool border = (int)l == how.choices - 1;
            bool sure;
            if constexpr (BIAS) {
                const float bl = mine ? bias[at] : 0.0f, ba = row_move<0x101>(bl);
                const float here = __builtin_bit_cast(float, ~mine & ~NUMBER), there = __builtin_bit_cast(float, ~after & ~NUMBER);      // distances from the best
                sure = there - here > 2 * score_error + size * 0x1p-22f + kCut * there || (!border && xl == xa && bl == ba);
            } else
                sure = mine / NUMBERS != after / NUMBERS || (border ? sizeof(T) == 2 : xl >= xa);
            unsure = unsure || (in && after && !sure);
        }
        const double share = row_share(how, xl, in, most, all);
        const uint64_t again = __ballot(unsure);
        if (t < tokens && (int)l < how.choices && !(again >> (lane & 48) & 0xffff)) {
            const size_t to = (size_t)t * how.choices + l;
            expert[to] = in ? (int32_t)at : -1;
            weight[to] = (float)((double)how.factor * share);
        }
        if (__builtin_expect(again != 0, 0))
            for (uint32_t i = 0; i < 4; ++i)
                if ((again >> (i * kRowLanes) & 0xffff) && t0 + i < tokens)
                    choose_exactly<T, (PER + 3) / 4>(logits, ld, t0 + i, experts, bias, how, expert, weight, s_key + (size_t)wave * experts);
    }
}

// One wave to a token.
template <class T>
__global__ __launch_bounds__(kWG) void choose_grad_kernel(const T *__restrict__ logits, int64_t ld, uint32_t tokens, uint32_t experts,
                                                          seer_choice how, const int32_t *__restrict__ expert, const float *__restrict__ dweight,
                                                          T *__restrict__ dlogits, int64_t ldd)
{
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const bool whole = how.score == SEER_SOFTMAX && !how.renormalise;
    for (uint32_t t = blockIdx.x * (kWG / kWave) + wave; t < tokens; t += gridDim.x * (kWG / kWave)) {
        const T *row = logits + (int64_t)t * ld;
        int32_t e = -1;
        float x = 0, dw = 0;
        if ((int)lane < how.choices) {
            const size_t at = (size_t)t * how.choices + lane;
            e = expert[at];
            if (e < 0 || e >= (int32_t)experts) e = -1;
            if (e >= 0) {
                x = logit(row, (uint32_t)e);
                dw = dweight[at];
                if (x == -INFINITY) e = -1;
            }
        }
        const bool in = e >= 0;
        double most = -INFINITY, all = 0;
        if (whole) {
            for (uint32_t i = lane; i < experts; i += 64) {
                const float v = logit(row, i);
                most = v != v || v > most ? (double)v : most;
            }
            most = wave_max(most);
            for (uint32_t i = lane; i < experts; i += 64) {
                const float v = logit(row, i);
                if (v != -INFINITY) all += exp((double)v - most);
            }
            all = wave_sum(all);
        }
        const double share = chosen_share(how, x, in, most, all), part = in ? share * (double)dw : 0.0, sum = wave_sum(part);
        double g = how.renormalise ? part - share * sum : part;
        if (how.score == SEER_SIGMOID) g *= 1.0 / (1.0 + exp((double)x));
        if (!in) g = 0;
        g *= (double)how.factor;
        const bool spread = whole && __ballot(in) != 0;         // to every logit
        const double off = (double)how.factor * sum;
        for (uint32_t i0 = 0; i0 < experts; i0 += 64) {
            const uint32_t i = i0 + lane;
            double d = 0;
            for (int k = 0; k < how.choices; ++k) {
                const double gk = __shfl(g, k, 64);
                if (__shfl(e, k, 64) == (int32_t)i) d += gk;
            }
            if (i < experts) {
                const float v = spread ? logit(row, i) : -INFINITY;
                if (v != -INFINITY) d -= exp((double)v - most) / all * off;
                dlogits[(int64_t)t * ldd + i] = (T)(float)d;
            }
        }
    }
}

// Four tokens to a wave: the chosen experts' gradients, one to a lane of 16, are put into a row of zeros in LDS, from where the row goes out
// whole, four elements at a time.  UNITS of these to a lane.  Bound by bytes: 65 536 x 256 fp32 in 17 us (67 MB written), 91
// with a wave to a token; WHOLE, which reads all logits, 27 (5.2 TB/s).  16 384 tokens, 16 choices of 512: 10 and 76, 10 choices of 513 57.
template <class T, int UNITS, bool WHOLE>
__global__ __launch_bounds__(kWG) void choose_grad_rows_kernel(const T *__restrict__ logits, int64_t ld, uint32_t tokens, uint32_t experts,
                                                               seer_choice how, const int32_t *__restrict__ expert,
                                                               const float *__restrict__ dweight, T *__restrict__ dlogits, int64_t ldd)
{
    constexpr uint32_t ROW = UNITS * kRowLanes * 4;
    __shared__ __attribute__((aligned(16))) float s_row[kWG / kRowLanes][ROW];
    const uint32_t lane = threadIdx.x & 63, l = lane & (kRowLanes - 1);
    float *mine = s_row[threadIdx.x / kRowLanes];
    for (uint32_t t0 = blockIdx.x * (kWG / kRowLanes); t0 < tokens; t0 += gridDim.x * (kWG / kRowLanes)) {
        const uint32_t t = min(t0 + threadIdx.x / kRowLanes, tokens - 1);
        const T *row = logits + (int64_t)t * ld;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) *reinterpret_cast<v4f *>(mine + (u * kRowLanes + l) * 4) = v4f{0, 0, 0, 0};
        float p[WHOLE ? UNITS * 4 : 1], most = -INFINITY;
        double all = 0;
        if constexpr (WHOLE) {
#pragma unroll
            for (int i = 0; i < UNITS * 4; ++i) {
                const uint32_t e = (i / 4 * kRowLanes + l) * 4 + i % 4;
                p[i] = e < experts ? (float)row[e] : -INFINITY;
                most = p[i] != p[i] ? p[i] : fmaxf(most, p[i]);
            }
            most = row_max(most);
#pragma unroll
            for (int i = 0; i < UNITS * 4; ++i) p[i] = p[i] == -INFINITY ? -0.0f : __expf(p[i] - most);       // (-0: masked)
            all = row_sum((double)sum_of<UNITS * 4>([&](int i) { return p[i]; }));
        }
        int32_t e = -1;
        float x = 0, dw = 0;
        if ((int)l < how.choices) {
            e = expert[(size_t)t * how.choices + l];
            if (e >= 0 && e < (int32_t)experts) {
                x = (float)row[e];
                dw = dweight[(size_t)t * how.choices + l];
            } else e = -1;
            if (x == -INFINITY) e = -1;
        }
        const bool in = e >= 0;
        double rest = 1;
        const double share = row_share(how, x, in, most, all, &rest), part = in ? share * (double)dw : 0.0, sum = row_sum(part);
        const double slope = (how.renormalise ? part - share * sum : part) * rest;
        const float g = in ? (float)((double)how.factor * slope) : 0.0f;
        // an expert that comes more than once: its first lane adds up
        float of_expert = g;
        bool first = in;
        other_lanes([&](auto ctrl, uint32_t from) {
            constexpr int CTRL = decltype(ctrl)::value;
            const bool same = (int32_t)row_move<CTRL>((uint32_t)e) == e;
            const float other = row_move<CTRL>(g);
            of_expert += same ? other : 0.0f;
            first = first && !(same && from < l);
        });
        __builtin_amdgcn_wave_barrier();            // (a wave's LDS accesses are served in order)
        if (first) mine[e] = of_expert;
        __builtin_amdgcn_wave_barrier();
        const float off = WHOLE ? (float)((double)how.factor * sum / all) : 0.0f;
        const bool any = (__ballot(in) >> (lane & 48) & 0xffff) != 0;
        if (t0 + threadIdx.x / kRowLanes < tokens) {
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const uint32_t at = (u * kRowLanes + l) * 4;
                if (at >= experts) continue;
                const v4f v = *reinterpret_cast<const v4f *>(mine + at);
                float d[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s = p[WHOLE ? u * 4 + j : 0];
                    d[j] = WHOLE && any && __builtin_bit_cast(uint32_t, s) != 1u << 31 ? v[j] - s * off : v[j];
                }
                T *to = dlogits + (int64_t)t * ldd + at;
                if (at + 4 <= experts) {
                    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
                    four o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = (T)d[j];
                    *reinterpret_cast<four *>(to) = o;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at + j < experts) to[j] = (T)d[j];
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ------------------------------------------------------------------ launches

static dim3 token_grid(uint32_t tokens) { return dim3(std::min((tokens + kWG / kWave - 1) / (kWG / kWave), 1u << 20)); }

// How a wave takes four tokens: the experts of a lane and the lanes of a group, which are whole and begin with a group's first.  per 0: it does not.
struct RowShape { uint32_t per, group_lanes; };

static RowShape row_shape(uint32_t experts, const seer_choice &how)
{
    if (experts > kFastExperts || how.choices > (int32_t)kFastChoices) return RowShape{0, 0};
    if (how.best_groups == how.groups) return RowShape{(experts + kRowLanes - 1) / kRowLanes, 0};
    const uint32_t groups = (uint32_t)how.groups, length = experts / groups;
    for (uint32_t lanes = 8; lanes; lanes /= 2)
        if (groups * lanes <= kRowLanes && length % lanes == 0 && length / lanes <= kFastExperts / kRowLanes) return RowShape{length / lanes, lanes};
    return RowShape{0, 0};
}

void launch_choose(const seer_dense &logits, const float *bias, const seer_choice &how, int32_t *expert, float *weight, hipStream_t st)
{
    const uint32_t tokens = (uint32_t)logits.rows, experts = (uint32_t)logits.cols;
    const size_t lds = how.best_groups < how.groups ? (size_t)(kWG / kWave) * experts * 8 : 0;
    by_type(logits.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        const auto launch = [&](auto per) {
            hipLaunchKernelGGL((choose_kernel<T, decltype(per)::value>), token_grid(tokens), dim3(kWG), lds, st, static_cast<const T *>(logits.data),
                               logits.ld, tokens, experts, bias, how, expert, weight);
        };
        using std::integral_constant;
        const RowShape r = row_shape(experts, how);
        if (r.per) {
            const bool vec = r.per % 4 == 0 && experts % 4 == 0;
            const auto rows = [&](auto per, auto vectors) {
                const auto go = [&](auto with_bias) {
                    hipLaunchKernelGGL((choose_rows_kernel<T, decltype(per)::value, decltype(vectors)::value, decltype(with_bias)::value>),
                                       dim3(std::min((tokens + kWG / kRowLanes - 1) / (kWG / kRowLanes), kRowBlocks)), dim3(kWG), lds, st,
                                       static_cast<const T *>(logits.data), logits.ld, tokens, experts, r.per, r.group_lanes, bias, how, expert, weight);
                };
                if (bias) go(std::true_type{});
                else go(std::false_type{});
            };
            const auto of_width = [&](auto per) { vec ? rows(per, std::true_type{}) : rows(per, std::false_type{}); };
            if (r.per == 1) rows(integral_constant<int, 1>{}, std::false_type{});
            else if (r.per <= 4) of_width(integral_constant<int, 4>{});
            else if (r.per <= 8) of_width(integral_constant<int, 8>{});
            else if (r.per <= 12) of_width(integral_constant<int, 12>{});
            else if (r.per <= 16) of_width(integral_constant<int, 16>{});
            else of_width(integral_constant<int, 32>{});
            return;
        }
        if (experts <= 64) launch(integral_constant<int, 1>{});
        else if (experts <= 128) launch(integral_constant<int, 2>{});
        else if (experts <= 256) launch(integral_constant<int, 4>{});
        else if (experts <= 512) launch(integral_constant<int, 8>{});
        else if (experts <= 1024) launch(integral_constant<int, 16>{});
        else launch(integral_constant<int, 64>{});
    });
}

void launch_choose_grad(const seer_dense &logits, const seer_choice &how, const int32_t *expert, const float *dweight, const seer_dense &dlogits,
                        hipStream_t st)
{
    by_type(logits.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        const uint32_t tokens = (uint32_t)logits.rows, experts = (uint32_t)logits.cols;
        if (experts <= kFastExperts && how.choices <= (int32_t)kRowLanes) {
            const bool whole = how.score == SEER_SOFTMAX && !how.renormalise;
            const auto rows = [&](auto units) {
                const auto go = [&](auto all) {
                    hipLaunchKernelGGL((choose_grad_rows_kernel<T, decltype(units)::value, decltype(all)::value>),
                                       dim3(std::min((tokens + kWG / kRowLanes - 1) / (kWG / kRowLanes), 1u << 20)), dim3(kWG), 0, st,
                                       static_cast<const T *>(logits.data), logits.ld, tokens, experts, how, expert, dweight,
                                       static_cast<T *>(dlogits.data), dlogits.ld);
                };
                if (whole) go(std::true_type{});
                else go(std::false_type{});
            };
            if (experts <= 64) rows(std::integral_constant<int, 1>{});
            else if (experts <= 128) rows(std::integral_constant<int, 2>{});
            else if (experts <= 256) rows(std::integral_constant<int, 4>{});
            else rows(std::integral_constant<int, 8>{});
            return;
        }
        hipLaunchKernelGGL((choose_grad_kernel<T>), token_grid((uint32_t)logits.rows), dim3(kWG), 0, st, static_cast<const T *>(logits.data), logits.ld,
                           (uint32_t)logits.rows, (uint32_t)logits.cols, how, expert, dweight, static_cast<T *>(dlogits.data), dlogits.ld);
    });
}

} // namespace seer
