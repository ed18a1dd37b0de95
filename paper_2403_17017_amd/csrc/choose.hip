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

// One wave to a token, lane l has the experts l, 64 + l, ...
template <class T, int PER>
__global__ __launch_bounds__(kWG) void choose_kernel(const T *__restrict__ logits, int64_t ld, uint32_t tokens, uint32_t experts,
                                                     const float *__restrict__ bias, seer_choice how, int32_t *__restrict__ expert,
                                                     float *__restrict__ weight)
{
    extern __shared__ __attribute__((aligned(16))) uint64_t s_key[];          // [waves][experts], with groups
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const bool grouped = how.best_groups < how.groups;
    for (uint32_t t = blockIdx.x * (kWG / kWave) + wave; t < tokens; t += gridDim.x * (kWG / kWave)) {
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
            uint64_t *mine = s_key + (size_t)wave * experts;
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

// ------------------------------------------------------------------ launches

static dim3 token_grid(uint32_t tokens) { return dim3(std::min((tokens + kWG / kWave - 1) / (kWG / kWave), 1u << 20)); }

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
        hipLaunchKernelGGL((choose_grad_kernel<T>), token_grid((uint32_t)logits.rows), dim3(kWG), 0, st, static_cast<const T *>(logits.data), logits.ld,
                           (uint32_t)logits.rows, (uint32_t)logits.cols, how, expert, dweight, static_cast<T *>(dlogits.data), dlogits.ld);
    });
}

} // namespace seer
