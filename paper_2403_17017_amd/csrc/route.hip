// A routed layer's rows: the choices sorted by expert, rows brought to the experts and back, and
// the gradients of both.  The choices are a sparse (experts x tokens) matrix: the sort writes its CSR
// form, `gather` multiplies by it and `combine` by its transpose, with dense rows as operands.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

// ------------------------------------------------------------------ sort
//
// A stable counting sort with one bucket per expert and one behind them for choices that are
// no expert's.  Each wave counts a run of consecutive choices, 64 at a time: the lanes with equal keys find
// each other with one ballot per key bit, a lane's rank among them is the set bits below it, and the run's
// counters lie in LDS.  A choice's slot is then
//   entries of lower keys + entries of its key in earlier workgroups + ... in earlier waves + its rank in the run
// where the rank is left in choice_slot between the two passes over the choices.  Bound by the latency of its few dependent
// steps: 8 choices of 128 experts 4.0 us (one launch), 98 304 of 160 in 12.7 us (two).
constexpr int kSortWaves = 16;
constexpr uint32_t kSortMaxGroups = 128;

template <class I>
__device__ __forceinline__ uint32_t key_of(const I *expert, uint32_t c, uint32_t experts)
{
    const I e = expert[c];
    return e >= 0 && e < (I)experts ? (uint32_t)e : experts;
}

// Ranks in the run [begin, end) of the calling wave; cnt [buckets] of this wave, zeroed before.
template <class I>
__device__ __forceinline__ void count_run(const I *expert, uint32_t begin, uint32_t end, uint32_t experts, int key_bits,
                                          uint32_t *cnt, int32_t *rank_out)
{
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t at = begin; at < end; at += 64) {
        const uint32_t c = at + lane;
        const bool in = c < end;
        const uint32_t key = in ? key_of(expert, c, experts) : 0;
        uint64_t peers = __ballot(in);
        for (int b = 0; b < key_bits; ++b) {
            const uint64_t set = __ballot(key >> b & 1);
            peers &= (key >> b & 1) ? set : ~set;
        }
        // the first lane of each key counts them all
        const int first = __ffsll((unsigned long long)peers) - 1;
        uint32_t before = 0;
        if (in && first == (int)lane) before = atomicAdd(&cnt[key], (uint32_t)__popcll(peers));
        before = __shfl(before, first, 64);
        if (in) rank_out[c] = (int32_t)(before + (uint32_t)__popcll(peers & ((1ull << lane) - 1)));
    }
}

// One workgroup's share of the sort: choices [begin, end) in `waves` runs.  base [buckets + 1] in LDS: where each key's
// entries of this workgroup begin.
template <class I>
__device__ void place_choices(const I *expert, uint32_t begin, uint32_t end, uint32_t per_wave, uint32_t experts,
                              const uint32_t *cnt, const uint32_t *base, int32_t *slot_choice, int32_t *choice_slot)
{
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63, buckets = experts + 1;
    const uint32_t from = begin + wave * per_wave, to = min(end, from + per_wave);
    for (uint32_t at = from; at < to; at += 64) {
        const uint32_t c = at + lane;
        if (c < to) {
            const uint32_t key = key_of(expert, c, experts);
            const uint32_t p = base[key] + cnt[wave * buckets + key] + (uint32_t)choice_slot[c];
            slot_choice[p] = (int32_t)c;
            choice_slot[c] = key < experts ? (int32_t)p : -1 - (int32_t)p;
        }
    }
}

// Exclusive prefix sum over v[0 .. n) in LDS by the whole workgroup, the total in v[n].
__device__ void scan_lds(uint32_t *v, uint32_t n, uint32_t *s_wave)
{
    const uint32_t threads = blockDim.x, lane = threadIdx.x & 63, wave = threadIdx.x / 64;
    uint32_t carry = 0;
    for (uint32_t at = 0; at < n; at += threads) {
        const uint32_t i = at + threadIdx.x;
        const uint32_t mine = i < n ? v[i] : 0;
        uint32_t sum = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = __shfl_up(sum, d, 64);
            if ((int)lane >= d) sum += other;
        }
        if (lane == 63) s_wave[wave] = sum;
        __syncthreads();
        uint32_t before = carry, all = 0;
        for (uint32_t w = 0; w < threads / 64; ++w) {
            if (w < wave) before += s_wave[w];
            all += s_wave[w];
        }
        if (i < n) v[i] = before + sum - mine;
        carry += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) v[n] = carry;
    __syncthreads();
}

struct SortArgs {
    const void *expert;
    uint32_t count, experts, per_wave, groups;
    uint32_t runs;          // waves that count (the others only add up)
    int key_bits;
    int32_t *expert_ptr, *slot_choice, *choice_slot;
    uint32_t *counts;       // [groups][buckets], in the workspace; null with one workgroup
};

// pass 0: everything in one workgroup; 1: counts of each workgroup's share; 2: the slots.
// LDS: cnt [waves][buckets], base [buckets + 1], in pass 2 before [buckets], too.
template <class I, int PASS>
__global__ __launch_bounds__(kSortWaves * 64) void route_kernel(SortArgs a)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ uint32_t s_wave[kSortWaves];
    const uint32_t waves = a.runs, wave = threadIdx.x / 64, buckets = a.experts + 1;
    uint32_t *cnt = lds, *base = lds + waves * buckets;
    const I *expert = static_cast<const I *>(a.expert);
    const uint32_t begin = blockIdx.x * waves * a.per_wave, end = min(a.count, begin + waves * a.per_wave);
    if constexpr (PASS == 0 || PASS == 1) {
        for (uint32_t i = threadIdx.x; i < waves * buckets; i += blockDim.x) cnt[i] = 0;
        __syncthreads();
        const uint32_t from = min(end, begin + wave * a.per_wave);
        if (wave < waves) count_run(expert, from, min(end, from + a.per_wave), a.experts, a.key_bits, cnt + wave * buckets, a.choice_slot);
        __syncthreads();
        // each wave's counters become the entries of the key in earlier waves, base the workgroup's
        for (uint32_t k = threadIdx.x; k < buckets; k += blockDim.x) {
            uint32_t sum = 0;
            for (uint32_t w = 0; w < waves; ++w) {
                const uint32_t n = cnt[w * buckets + k];
                if (PASS == 0) cnt[w * buckets + k] = sum;
                sum += n;
            }
            if (PASS == 0) base[k] = sum;
            else a.counts[(size_t)blockIdx.x * buckets + k] = sum;
        }
        if constexpr (PASS == 1) return;
        __syncthreads();
        scan_lds(base, buckets, s_wave);
    } else {
        // the counters of the waves again, without ranks, beside the counts of all workgroups and of those before this one
        uint32_t *before = base + buckets + 1;
        for (uint32_t i = threadIdx.x; i < (waves + 2) * buckets + 1; i += blockDim.x) lds[i] = 0;
        __syncthreads();
        const uint32_t from = min(end, begin + wave * a.per_wave), to = min(end, from + a.per_wave);
        for (uint32_t c = from + (threadIdx.x & 63); wave < waves && c < to; c += 64)
            atomicAdd(&cnt[wave * buckets + key_of(expert, c, a.experts)], 1u);
        for (uint32_t i = threadIdx.x, all = a.groups * buckets; i < all; i += blockDim.x) {
            const uint32_t n = a.counts[i], g = i / buckets, k = i - g * buckets;
            atomicAdd(&base[k], n);
            if (g < blockIdx.x) atomicAdd(&before[k], n);
        }
        __syncthreads();
        scan_lds(base, buckets, s_wave);
        if (blockIdx.x == 0)
            for (uint32_t k = threadIdx.x; k <= a.experts; k += blockDim.x) a.expert_ptr[k] = (int32_t)base[k];
        __syncthreads();
        for (uint32_t k = threadIdx.x; k < buckets; k += blockDim.x) {
            uint32_t sum = 0;
            for (uint32_t w = 0; w < waves; ++w) {
                const uint32_t n = cnt[w * buckets + k];
                cnt[w * buckets + k] = sum;
                sum += n;
            }
            base[k] += before[k];
        }
        __syncthreads();
    }
    if constexpr (PASS == 0)
        for (uint32_t k = threadIdx.x; k <= a.experts; k += blockDim.x) a.expert_ptr[k] = (int32_t)base[k];
    if (wave < waves) place_choices(expert, begin, end, a.per_wave, a.experts, cnt, base, a.slot_choice, a.choice_slot);
}

// Waves whose counters fit the LDS beside the workgroup's (16: up to 147 KB; 6: up to 131 KB).
static uint32_t sort_waves(uint32_t experts) { return experts <= 2048 ? kSortWaves : 6; }

// What one workgroup sorts on its own, and what each takes where there are more: the second launch of those reads the
// counts of all workgroups in each, so that shares grow with the number of experts.  Measured, us, one workgroup and
// two launches: 160 experts, 2048 choices 6.5 and 7.9, 4096 9.7 and 8.1; 4096 experts, 4096 choices 35 and 45.  98 304
// choices in shares of 1024, 2048 and 4096: 160 experts 12.9, 12.2, 14.5, 1024 experts 39, 27, 24.5.
static uint32_t sort_groups(uint32_t count, uint32_t experts, uint32_t *per_wave)
{
    const uint32_t waves = sort_waves(experts), most = std::max(1024u, 4 * experts);
    const uint32_t groups = count <= std::max(2048u, 2 * experts) ? 1 : std::min((count + most - 1) / most, kSortMaxGroups);
    const uint32_t share = (count + groups - 1) / groups;
    *per_wave = std::max(64u, ((share + waves - 1) / waves + 63) & ~63u);
    return (count + waves * *per_wave - 1) / (waves * *per_wave);
}

size_t route_workspace_bytes(uint32_t count, uint32_t experts)
{
    uint32_t per_wave;
    const uint32_t groups = sort_groups(count, experts, &per_wave);
    return groups > 1 ? (((size_t)groups * (experts + 1) * 4 + 255) & ~(size_t)255) : 0;
}

template <class I>
static void launch_route_of(SortArgs a, uint32_t waves, hipStream_t st)
{
    const size_t lds = ((size_t)(a.runs + 2) * (a.experts + 1) + 1) * 4;
    if (a.groups <= 1) {
        hipLaunchKernelGGL((route_kernel<I, 0>), dim3(1), dim3(waves * 64), lds, st, a);
        return;
    }
    hipLaunchKernelGGL((route_kernel<I, 1>), dim3(a.groups), dim3(waves * 64), lds, st, a);
    hipLaunchKernelGGL((route_kernel<I, 2>), dim3(a.groups), dim3(waves * 64), lds, st, a);
}

void launch_route(const void *expert, bool wide, uint32_t count, uint32_t experts, int32_t *expert_ptr, int32_t *slot_choice,
                  int32_t *choice_slot, void *workspace, hipStream_t st)
{
    SortArgs a{};
    a.expert = expert;
    a.count = count;
    a.experts = experts;
    a.groups = sort_groups(count, experts, &a.per_wave);
    a.runs = std::min(sort_waves(experts), std::max(1u, (count + a.per_wave - 1) / a.per_wave));
    for (a.key_bits = 1; (experts >> a.key_bits) != 0; ++a.key_bits) {}
    a.expert_ptr = expert_ptr;
    a.slot_choice = slot_choice;
    a.choice_slot = choice_slot;
    a.counts = static_cast<uint32_t *>(workspace);
    if (wide) launch_route_of<int64_t>(a, sort_waves(experts), st);
    else launch_route_of<int32_t>(a, sort_waves(experts), st);
}

// ------------------------------------------------------------------ rows to the experts and back
//
// All three kernels go by token: a token's row is read (or written) once, and its choices' rows, each contiguous, once.  Bound by
// bytes, and measured against a copy's 5.2 TB/s and a read's 6.2.

constexpr uint32_t kMaxGrid = 1u << 20;     // workgroups; more work is looped over

// LANES lanes to a row, kWG / LANES rows to a workgroup.  The token of a lane; uniform in a wave where it can be.
template <int LANES>
__device__ __forceinline__ uint32_t token_of(uint32_t block)
{
    const uint32_t t = block * (kWG / LANES) + threadIdx.x / LANES;
    return LANES >= kWave ? (uint32_t)__builtin_amdgcn_readfirstlane((int)t) : t;
}

// 16 411 tokens of 4096 bf16 to six experts each: 170 us, 5.5 TB/s; by slot, with the stores in order and every row read six times
// from the last-level cache, 230; with streaming stores 181; with two or four units a lane 178 and 174.
template <class T, int LANES>
__global__ __launch_bounds__(kWG) void gather_kernel(RouteRows r, const float *__restrict__ weight, const T *__restrict__ x,
                                                     int64_t ldx, T *__restrict__ out, int64_t ldo)
{
    constexpr int E = Unit<T>::kElems;
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < r.tokens; b += gridDim.y) {
        const uint32_t t = token_of<LANES>(b);
        if (t >= r.tokens) continue;
        for (uint32_t col = (blockIdx.x * LANES + threadIdx.x % LANES) * E; col < r.cols; col += gridDim.x * LANES * E) {
            const int n = (int)min((uint32_t)E, r.cols - col);
            const Unit<T> u = load_some(x + (int64_t)t * ldx + col, n);
            for (uint32_t k = 0; k < r.choices; ++k) {
                const uint32_t c = t * r.choices + k;
                const int32_t slot = r.choice_slot[c];
                Unit<T> v = u;
                if (weight) {
                    const float s = weight[c];
#pragma unroll
                    for (int j = 0; j < E; ++j) v.v[j] = (T)(s * (float)u.v[j]);
                }
                if (slot < 0) v = zero_unit<T>();
                store_some(out + (int64_t)(slot < 0 ? -1 - slot : slot) * ldo + col, v, n);
            }
        }
    }
}

// AT_ONCE choices are fetched together.
// 32 768 tokens of 4096 bf16 from four experts each: 224 us, 6.0 TB/s; 253 without the streaming hint on rows that are used once.
template <class T, bool STREAM, int LANES, int AT_ONCE>
__global__ __launch_bounds__(kWG) void combine_kernel(RouteRows r, const float *__restrict__ weight, const T *__restrict__ z,
                                                      int64_t ldz, T *__restrict__ y, int64_t ldy)
{
    constexpr int E = Unit<T>::kElems;
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < r.tokens; b += gridDim.y) {
        const uint32_t t = token_of<LANES>(b);
        if (t >= r.tokens) continue;
        for (uint32_t col = (blockIdx.x * LANES + threadIdx.x % LANES) * E; col < r.cols; col += gridDim.x * LANES * E) {
            const int n = (int)min((uint32_t)E, r.cols - col);
            float acc[E] = {};
            for (uint32_t k0 = 0; k0 < r.choices; k0 += AT_ONCE) {
                int32_t slot[AT_ONCE];
                float s[AT_ONCE];
                Unit<T> u[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    const uint32_t c = t * r.choices + min(k0 + i, r.choices - 1);
                    slot[i] = r.choice_slot[c];
                    s[i] = weight ? weight[c] : 1.0f;
                }
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (slot[i] >= 0 && k0 + i < r.choices) u[i] = load_row<STREAM>(z + (int64_t)slot[i] * ldz + col, n);
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (slot[i] >= 0 && k0 + i < r.choices) {
#pragma unroll
                        for (int j = 0; j < E; ++j) acc[j] += s[i] * (float)u[i].v[j];
                    }
            }
            Unit<T> v;
#pragma unroll
            for (int j = 0; j < E; ++j) v.v[j] = (T)acc[j];
            store_row<STREAM>(y + (int64_t)t * ldy + col, v, n);
        }
    }
}

// The dot products' lanes add up in a fixed order, and dy stays in the nearest caches from two choices to the next two (four at a time:
// the same; one: 1 % slower, 8 % where 1031 rows of 1023 floats wait for each other's ends).
// 16 384 tokens of 4096 bf16 with eight choices: 420 us, 5.4 TB/s; 465 without the streaming hint.
template <class T, bool STREAM, int LANES>
__global__ __launch_bounds__(kWG) void route_grad_kernel(RouteRows r, const float *__restrict__ weight, const T *__restrict__ dy,
                                                         int64_t lddy, const T *__restrict__ z, int64_t ldz, T *__restrict__ dz,
                                                         int64_t lddz, float *__restrict__ dweight)
{
    constexpr int E = Unit<T>::kElems, AT_ONCE = 2;   // choices
    __shared__ float s_dot[2][kWG / kWave][AT_ONCE];
    uint32_t turn = 0;
    for (uint32_t b = blockIdx.x; b * (kWG / LANES) < r.tokens; b += gridDim.x) {
        const uint32_t t = token_of<LANES>(b), lane = threadIdx.x % LANES;
        const bool mine = t < r.tokens;                 // (all lanes stay for the sums)
        for (uint32_t k0 = 0; k0 < r.choices; k0 += AT_ONCE) {
            int32_t slot[AT_ONCE];                      // (the last choice again behind it)
            float w[AT_ONCE], dot[AT_ONCE] = {};
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const uint32_t c = (mine ? t : 0) * r.choices + min(k0 + i, r.choices - 1);
                slot[i] = r.choice_slot[c];
                w[i] = weight ? weight[c] : 1.0f;
            }
            for (uint32_t col = lane * E; mine && col < r.cols; col += LANES * E) {
                const int n = (int)min((uint32_t)E, r.cols - col);
                const Unit<T> g = load_some(dy + (int64_t)t * lddy + col, n);
                Unit<T> u[AT_ONCE];
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (dweight && slot[i] >= 0 && k0 + i < r.choices) u[i] = load_row<STREAM>(z + slot[i] * ldz + col, n);
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i) {
                    if (k0 + i >= r.choices) break;
                    if (dweight && slot[i] >= 0) {
#pragma unroll
                        for (int j = 0; j < E; ++j) dot[i] += (float)g.v[j] * (float)u[i].v[j];
                    }
                    if (dz) {
                        Unit<T> v = zero_unit<T>();
                        if (slot[i] >= 0) {
#pragma unroll
                            for (int j = 0; j < E; ++j) v.v[j] = (T)(w[i] * (float)g.v[j]);
                        }
                        store_row<STREAM>(dz + (int64_t)(slot[i] < 0 ? -1 - slot[i] : slot[i]) * lddz + col, v, n);
                    }
                }
            }
            if (!dweight) continue;
            constexpr int FOLD = LANES < kWave ? LANES : kWave;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
                for (int d = 1; d < FOLD; d <<= 1) dot[i] += __shfl_xor(dot[i], d, kWave);
            if constexpr (LANES <= kWave) {
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if (mine && lane == 0 && k0 + i < r.choices) dweight[t * r.choices + k0 + i] = dot[i];
            } else {
#pragma unroll
                for (int i = 0; i < AT_ONCE; ++i)
                    if ((threadIdx.x & 63) == 0) s_dot[turn][threadIdx.x / 64][i] = dot[i];
                __syncthreads();                        // (two sets: one barrier is enough)
                const uint32_t i = threadIdx.x;
                if (i < AT_ONCE && k0 + i < r.choices)
                    dweight[t * r.choices + k0 + i] = (s_dot[turn][0][i] + s_dot[turn][1][i]) + (s_dot[turn][2][i] + s_dot[turn][3][i]);
                turn ^= 1;
            }
        }
    }
}

// q = x / scale to the nearest integer, the division rounded to fp32 first; |x| <= 127 scale.  0 for an infinite scale, too, where the
// quotients of infinite elements are no numbers.
__device__ __forceinline__ float quantised(float x, float scale)
{
    const float v = rintf(x / scale);
    return scale > 0 && scale < __builtin_inff() ? fminf(fmaxf(v, -127.0f), 127.0f) : 0.0f;
}

// Quantisation, of a row of x at a time; routed: its copies go to the slots of its choices.  A lane takes 16 elements at a
// time, whose 16 bytes of q go out in one store.
typedef uint32_t q_vec __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t q_whole __attribute__((ext_vector_type(4)));

// The scale of a row, and what its elements are multiplied by instead of being divided by it: off by at most 1.5 units in the
// last place, 2.3e-5 for quotients of up to 127, so that the nearest integer is the same unless the product is
// that close to the middle between two (kNearHalf leaves twice the room); then, and for scales that have no
// reciprocal (subnormal ones, 0, infinity, NaN: by = 0), the division itself is done.
struct RowScale { float scale, by; };
constexpr float kNearHalf = 0.49995f;
__device__ __forceinline__ RowScale row_scale(uint32_t top)
{
    RowScale s;
    s.scale = __uint_as_float(top) / 127.0f;
    s.by = s.scale >= 0x1p-100f && s.scale <= 0x1p120f ? 1.0f / s.scale : 0.0f;
    return s;
}

template <class T>
struct Sixteen {
    static constexpr int kElems = Unit<T>::kElems, kUnits = 16 / kElems;
    Unit<T> u[kUnits];
    __device__ __forceinline__ void load16(const T *p)
    {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) u[i] = load_unit(p + i * kElems);
    }
    __device__ __forceinline__ void load(const T *p, int n)         // n: elements that there are, more than 16 or none at all, too
    {
        if (n >= 16) {
            load16(p);
        } else {
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int have = n - i * kElems;
                u[i] = have > 0 ? load_some(p + i * kElems, have) : zero_unit<T>();
            }
        }
    }
    __device__ __forceinline__ float at(int j) const { return (float)u[j / kElems].v[j % kElems]; }
    // The largest magnitude as the bits of a float: they order as the magnitudes do, and a NaN's are above infinity's, so a
    // NaN anywhere is found.  16-bit types are compared two at a time before they are converted.
    __device__ __forceinline__ uint32_t largest() const
    {
        if constexpr (sizeof(T) == 2) {
            typedef unsigned short two __attribute__((ext_vector_type(2)));
            typedef uint32_t words __attribute__((ext_vector_type(4)));
            two top = {0, 0};
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const words w = __builtin_bit_cast(words, u[i].v) & 0x7fff7fffu;
#pragma unroll
                for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(two, (uint32_t)w[j]));
            }
            const unsigned short bits = top.x > top.y ? top.x : top.y;
            return __float_as_uint((float)__builtin_bit_cast(T, bits));
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(at(j)) & 0x7fffffffu);
            return top;
        }
    }
    __device__ __forceinline__ q_whole quantise(const RowScale &s) const
    {
        constexpr float kMagic = 0x1.8p23f;      // v + kMagic is rounded to an integer, whose last byte is that of the sum
        uint32_t b[16];
        float worst = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float v = at(j) * s.by, up = v + kMagic;
            worst = fmaxf(worst, fabsf(v - (up - kMagic)));
            b[j] = __float_as_uint(up);
        }
        if (!(worst < kNearHalf) || s.by == 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                b[j] = (uint32_t)(int)quantised(at(j), s.scale);
                asm volatile("" : "+v"(b[j]));       // (not to be done by everybody and thrown away, nor all 16 at a time)
            }
        }
        q_whole q;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t low = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400), high = __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x0c0c0400);
            q[i] = low | high << 16;
        }
        return q;
    }
};

// The largest of `top` over the WAVES waves of a row; s_max: two sets, taken in turn, so that one barrier a row is enough.
template <int WAVES>
__device__ __forceinline__ uint32_t row_largest(uint32_t top, uint32_t (*s_max)[WAVES], uint32_t *turn)
{
    top = lanes_fold(top, [](uint32_t a, uint32_t b) { return max(a, b); });
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) s_max[*turn][threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = max(top, s_max[*turn][w]);
        *turn ^= 1;
    }
    return top;
}

// Rows of whole sixteens, HELD of them to a lane of the WAVES waves of a row at most: each row stays in registers.  Bound by how many rows are
// under way, hence few registers: 3001 rows of 4112 in 10 us (3.6 TB/s), in a kernel that also knew the ends of other rows
// (106 registers) 24 us; 8192 rows of 4096 to four experts each 35 us (5.8 TB/s) and 49.
template <class T, bool ROUTED, int WAVES, int HELD>
__global__ __launch_bounds__(WAVES < 4 ? kWG : WAVES * kWave) void quantize_whole_kernel(RouteRows r, const T *__restrict__ x, int64_t ldx, int8_t *__restrict__ q,
                                                                                        int64_t ldq, float *__restrict__ scale)
{
    __shared__ uint32_t s_max[2][WAVES];
    constexpr uint32_t LANES = WAVES * kWave, ROWS = LANES < kWG ? kWG / LANES : 1;
    const uint32_t lane = threadIdx.x % LANES, sub = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / LANES));
    uint32_t turn = 0;
    for (uint32_t t = blockIdx.x * ROWS + sub; t < r.tokens; t += gridDim.x * ROWS) {
        const T *row = x + (int64_t)t * ldx;
        Sixteen<T> held[HELD];
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const uint32_t col = (h * LANES + lane) * 16;
            if (col < r.cols) held[h].load16(row + col);
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h)
            if ((h * LANES + lane) * 16 < r.cols) top = max(top, held[h].largest());
        const RowScale s = row_scale(row_largest<WAVES>(top, s_max, &turn));
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const uint32_t col = (h * LANES + lane) * 16;
            if (col >= r.cols) continue;
            const q_whole b = held[h].quantise(s);
            for (uint32_t k = 0; k < r.choices; ++k) {
                const int32_t slot = ROUTED ? r.choice_slot[t * r.choices + k] : (int32_t)t;
                *reinterpret_cast<q_vec *>(q + (int64_t)(slot < 0 ? -1 - slot : slot) * ldq + col) = slot < 0 ? (q_whole)0u : b;
            }
        }
        for (uint32_t k = lane; k < r.choices; k += LANES) {
            const int32_t slot = ROUTED ? r.choice_slot[t * r.choices + k] : (int32_t)t;
            scale[slot < 0 ? -1 - slot : slot] = slot < 0 ? 0.0f : s.scale;
        }
    }
}

// Any other row, one workgroup to each, read twice: 3001 rows of 4111 fp16 15 us (2.4 TB/s), 8192 of bf16 36 (2.8).
template <class T, bool ROUTED>
__global__ __launch_bounds__(kWG) void quantize_kernel(RouteRows r, const T *__restrict__ x, int64_t ldx, int8_t *__restrict__ q,
                                                       int64_t ldq, uint32_t padded, float *__restrict__ scale)
{
    constexpr int WAVES = kWG / kWave;
    __shared__ uint32_t s_max[2][WAVES];
    uint32_t turn = 0;
    for (uint32_t t = blockIdx.x; t < r.tokens; t += gridDim.x) {
        const T *row = x + (int64_t)t * ldx;
        uint32_t top = 0;
        for (uint32_t col = threadIdx.x * 16; col < r.cols; col += kWG * 16) {
            Sixteen<T> v;
            v.load(row + col, (int)(r.cols - col));
            top = max(top, v.largest());
        }
        const RowScale s = row_scale(row_largest<WAVES>(top, s_max, &turn));
        for (uint32_t col = threadIdx.x * 16; col < padded; col += kWG * 16) {
            Sixteen<T> v;
            v.load(row + col, (int)(r.cols - col));
            const q_whole b = v.quantise(s);            // (the zeros behind the row's end give 0)
            for (uint32_t k = 0; k < r.choices; ++k) {
                const int32_t slot = ROUTED ? r.choice_slot[t * r.choices + k] : (int32_t)t;
                int8_t *to = q + (int64_t)(slot < 0 ? -1 - slot : slot) * ldq + col;
                const q_whole out = slot < 0 ? (q_whole)0u : b;
                if (col + 16 <= padded) {
                    *reinterpret_cast<q_vec *>(to) = out;
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (col + j < padded) to[j] = (int8_t)(out[j / 4] >> (j % 4 * 8));
                }
            }
        }
        for (uint32_t k = threadIdx.x; k < r.choices; k += kWG) {
            const int32_t slot = ROUTED ? r.choice_slot[t * r.choices + k] : (int32_t)t;
            scale[slot < 0 ? -1 - slot : slot] = slot < 0 ? 0.0f : s.scale;
        }
    }
}

// ------------------------------------------------------------------ launches

template <class F>
static void by_type(int type, F f)
{
    if (type == SEER_F32) f((float *)nullptr);
    else if (type == SEER_BF16) f((bf16_t *)nullptr);
    else f((f16_t *)nullptr);
}

// Rows that begin on multiples of 16 bytes are streamed; the pieces of others share lines, which have to stay for the second one.
// (1031 rows of 1023 floats, two choices each, gradient: 6.9 us, 9.0 streamed.)
static bool streamed(const seer_dense &m, size_t size)
{
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (size_t)m.ld * size % 16 == 0;
}

// The lanes to a row, as a constant: the whole workgroup's, or fewer, so that a row of few 16-byte pieces does not leave most of them idle.
// Of 20 000 tokens of 120 bf16 with eight choices the gather takes 10.6 us with 16 lanes to a row and 16.3 with 256, the way back 9.3
// and 31.2, the gradient 26.6 and 135; of 100 tokens 256 lanes are 0.8 us faster, as they read the slots once a wave and fill more CUs.
// Rows of 72 to 128 pieces: the gradient 36 to 50 us with 64 lanes and 58 to 97 with 256, whose waves wait for each other's sums; the
// others have no sums and are 0 to 10 % faster with 256.
template <class F>
static void by_lanes(const RouteRows &r, uint32_t elems, bool sums, F f)
{
    const uint32_t pieces = (r.cols + elems - 1) / elems;
    if (pieces <= 32 && (sums || r.tokens >= 4096)) f(std::integral_constant<int, 16>{});
    else if (pieces <= 128 && sums) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 256>{});
}

// The same without the 64 lanes, which only sums gain from.
template <class F>
static void by_lanes_no_sums(const RouteRows &r, uint32_t elems, F f)
{
    by_lanes(r, elems, false, [&](auto lanes) {
        if constexpr (decltype(lanes)::value != 64) f(lanes);
    });
}

// A workgroup per kWG / lanes tokens and 16 bytes a lane; more of either is looped over.
static dim3 grid_of(const RouteRows &r, uint32_t elems, uint32_t lanes)
{
    const uint32_t rows = kWG / lanes;
    return dim3(lanes < kWG ? 1 : std::min(1024u, (r.cols + kWG * elems - 1) / (kWG * elems)), std::min((r.tokens + rows - 1) / rows, 65535u));
}

void launch_route_gather(const RouteRows &rows, const float *weight, const seer_dense &x, const seer_dense &out, hipStream_t st)
{
    by_type(x.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_lanes_no_sums(rows, Unit<T>::kElems, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            hipLaunchKernelGGL((gather_kernel<T, LANES>), grid_of(rows, Unit<T>::kElems, LANES), dim3(kWG), 0, st, rows, weight,
                               static_cast<const T *>(x.data), x.ld, static_cast<T *>(out.data), out.ld);
        });
    });
}

// Four choices at once for short rows (20 000 tokens of 120 bf16, eight choices: 9.3 us; one: 12.9), two for others (9295 x 5 x 576 bf16
// 15.0 and 16.2, 4000 x 4 x 1040 9.1 and 10.1), one where the rows do not fit the last-level cache, whose pages are then read in longer
// runs (32 768 x 4 x 4096: 224 us; two 227, four 228).
void launch_route_combine(const RouteRows &rows, const float *weight, const seer_dense &z, const seer_dense &y, hipStream_t st)
{
    by_type(z.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_lanes_no_sums(rows, Unit<T>::kElems, [&](auto lanes) {
            const auto launch = [&](auto stream, auto at_once) {
                constexpr int LANES = decltype(lanes)::value;
                hipLaunchKernelGGL((combine_kernel<T, decltype(stream)::value, LANES, decltype(at_once)::value>),
                                   grid_of(rows, Unit<T>::kElems, LANES), dim3(kWG), 0, st, rows, weight, static_cast<const T *>(z.data), z.ld,
                                   static_cast<T *>(y.data), y.ld);
            };
            const auto launch_at = [&](auto at_once) {
                if (streamed(z, sizeof(T)) && streamed(y, sizeof(T))) launch(std::true_type{}, at_once);
                else launch(std::false_type{}, at_once);
            };
            if constexpr (decltype(lanes)::value < kWave) launch_at(std::integral_constant<int, 4>{});
            else if ((uint64_t)z.rows * z.cols * sizeof(T) > 256u << 20) launch_at(std::integral_constant<int, 1>{});
            else launch_at(std::integral_constant<int, 2>{});
        });
    });
}

void launch_route_grad(const RouteRows &rows, const float *weight, const seer_dense &dy, const seer_dense *z,
                       const seer_dense *dz, float *dweight, hipStream_t st)
{
    by_type(dy.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_lanes(rows, Unit<T>::kElems, true, [&](auto lanes) {
            const auto launch = [&](auto stream) {
                constexpr int LANES = decltype(lanes)::value;
                constexpr uint32_t per = kWG / LANES;
                hipLaunchKernelGGL((route_grad_kernel<T, decltype(stream)::value, LANES>), dim3(std::min((rows.tokens + per - 1) / per, kMaxGrid)),
                                   dim3(kWG), 0, st, rows, weight, static_cast<const T *>(dy.data), dy.ld,
                                   z ? static_cast<const T *>(z->data) : (const T *)nullptr, z ? z->ld : 0,
                                   dz ? static_cast<T *>(dz->data) : (T *)nullptr, dz ? dz->ld : 0, dweight);
            };
            if ((!z || streamed(*z, sizeof(T))) && (!dz || streamed(*dz, sizeof(T)))) launch(std::true_type{});
            else launch(std::false_type{});
        });
    });
}

template <class T, int WAVES, int HELD>
static void launch_quantize_whole(const RouteRows &rows, const seer_dense &x, const seer_dense &q, float *scale, hipStream_t st)
{
    const uint32_t per = WAVES < 4 ? 4 / WAVES : 1;
    const dim3 grid(std::min((rows.tokens + per - 1) / per, kMaxGrid)), wg(WAVES < 4 ? kWG : WAVES * kWave);
    const T *xp = static_cast<const T *>(x.data);
    int8_t *qp = static_cast<int8_t *>(q.data);
    if (rows.choice_slot) hipLaunchKernelGGL((quantize_whole_kernel<T, true, WAVES, HELD>), grid, wg, 0, st, rows, xp, x.ld, qp, q.ld, scale);
    else hipLaunchKernelGGL((quantize_whole_kernel<T, false, WAVES, HELD>), grid, wg, 0, st, rows, xp, x.ld, qp, q.ld, scale);
}

void launch_quantize(const RouteRows &rows, const seer_dense &x, const seer_dense &q, float *scale, hipStream_t st)
{
    by_type(x.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        if (rows.cols % 16 == 0 && rows.cols <= 16384) {
            if (rows.cols <= 1024) launch_quantize_whole<T, 1, 1>(rows, x, q, scale, st);
            else if (rows.cols <= 4096) launch_quantize_whole<T, 4, 1>(rows, x, q, scale, st);
            else if (rows.cols <= 8192) launch_quantize_whole<T, 4, 2>(rows, x, q, scale, st);
            else launch_quantize_whole<T, 8, 2>(rows, x, q, scale, st);
            return;
        }
        const uint32_t padded = (uint32_t)std::min<int64_t>(q.ld, (x.cols + 15) & ~(int64_t)15);
        const dim3 grid(std::min(rows.tokens, kMaxGrid)), wg(kWG);
        const T *xp = static_cast<const T *>(x.data);
        int8_t *qp = static_cast<int8_t *>(q.data);
        if (rows.choice_slot) hipLaunchKernelGGL((quantize_kernel<T, true>), grid, wg, 0, st, rows, xp, x.ld, qp, q.ld, padded, scale);
        else hipLaunchKernelGGL((quantize_kernel<T, false>), grid, wg, 0, st, rows, xp, x.ld, qp, q.ld, padded, scale);
    });
}

} // namespace seer
