// Rows of a table by token, and the gradient in the table.  The tokens are a sparse (tokens x rows of the table) matrix with one
// entry a row: the lookup multiplies by it, with dense rows as the operand, and the gradient by its transpose, whose rows are as uneven
// as words are frequent.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

// The row of a token; `rows`: it has none.
template <class I>
__device__ __forceinline__ uint32_t row_of(const I *token, uint32_t t, uint32_t rows)
{
    const I v = token[t];
    return v >= 0 && v < (I)rows ? (uint32_t)v : rows;
}

// LANES lanes to a row, kWG / LANES rows to a workgroup: the row's number in the block, uniform in a wave where it can be.
template <int LANES>
__device__ __forceinline__ uint32_t row_in_block()
{
    const uint32_t r = threadIdx.x / LANES;
    return LANES >= kWave ? (uint32_t)__builtin_amdgcn_readfirstlane((int)r) : r;
}

// ------------------------------------------------------------------ lookup
//
// Bound by bytes: each row is read and written once.
template <class T, class I, int LANES>
__global__ __launch_bounds__(kWG) void embed_kernel(const I *__restrict__ token, uint32_t tokens, const T *__restrict__ table, int64_t ldt,
                                                    uint32_t rows, uint32_t cols, float scale, T *__restrict__ out, int64_t ldo)
{
    constexpr int E = Unit<T>::kElems;
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < tokens; b += gridDim.y) {
        const uint32_t t = b * (kWG / LANES) + row_in_block<LANES>();
        if (t >= tokens) continue;
        const uint32_t row = row_of(token, t, rows);
        for (uint32_t col = (blockIdx.x * LANES + threadIdx.x % LANES) * E; col < cols; col += gridDim.x * LANES * E) {
            const int n = (int)min((uint32_t)E, cols - col);
            Unit<T> u = zero_unit<T>();
            if (row < rows) {
                u = load_some(table + (int64_t)row * ldt + col, n);
                if (scale != 1.0f) {
#pragma unroll
                    for (int j = 0; j < E; ++j) u.v[j] = (T)(scale * (float)u.v[j]);
                }
            }
            store_some(out + (int64_t)t * ldo + col, u, n);
        }
    }
}

// ------------------------------------------------------------------ tokens sorted by row
//
// A stable sort of (row, token) pairs by digits of up to 10 bits, the lowest first, so the order is the same on every run.
// Each wave counts the digits of a run of pairs in LDS; a pair's place is then
//   pairs of lower digits + pairs of its digit in earlier workgroups + ... in earlier waves + ... before it in the run.
constexpr uint32_t kDigitWaves = 16;
constexpr int kDigitBits = 10;

struct Pairs { uint32_t *row, *token; };

struct DigitArgs {
    Pairs from, to;         // from.row null: the tokens themselves
    uint32_t count, rows, per_wave, groups;
    int shift, bits;
    uint32_t *counts;       // [groups][1 << bits], where there is more than one
};

template <class I>
__device__ __forceinline__ uint32_t pair_row(const DigitArgs &a, const I *token, uint32_t i)
{
    return a.from.row ? a.from.row[i] : row_of(token, i, a.rows);
}

// The calling workgroup's pairs to their places.  lds: kDigitWaves + 2 times (1 << bits) + 1 words.
template <class I>
__device__ __forceinline__ void place_digits(const DigitArgs &a, const I *token, uint32_t group, uint32_t *lds, uint32_t *s_wave)
{
    const uint32_t buckets = 1u << a.bits, mask = buckets - 1, wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    uint32_t *cnt = lds, *base = lds + kDigitWaves * buckets, *before = base + buckets + 1;
    for (uint32_t i = threadIdx.x; i < (kDigitWaves + 2) * buckets + 1; i += blockDim.x) lds[i] = 0;
    __syncthreads();
    const uint32_t from = min(a.count, (group * kDigitWaves + wave) * a.per_wave), to = min(a.count, from + a.per_wave);
    for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&cnt[wave * buckets + (pair_row(a, token, i) >> a.shift & mask)], 1u);
    if (a.groups > 1)
        for (uint32_t i = threadIdx.x, all = a.groups * buckets; i < all; i += blockDim.x) {
            const uint32_t n = a.counts[i];
            if (n == 0) continue;
            atomicAdd(&base[i & mask], n);
            if (i >> a.bits < group) atomicAdd(&before[i & mask], n);
        }
    __syncthreads();
    if (a.groups == 1) {
        for (uint32_t k = threadIdx.x; k < buckets; k += blockDim.x) {
            uint32_t sum = 0;
            for (uint32_t w = 0; w < kDigitWaves; ++w) sum += cnt[w * buckets + k];
            base[k] = sum;
        }
        __syncthreads();
    }
    scan_lds(base, buckets, s_wave);
    for (uint32_t k = threadIdx.x; k < buckets; k += blockDim.x) {
        uint32_t sum = base[k] + before[k];
        for (uint32_t w = 0; w < kDigitWaves; ++w) {
            const uint32_t n = cnt[w * buckets + k];
            cnt[w * buckets + k] = sum;
            sum += n;
        }
    }
    __syncthreads();
    for (uint32_t at = from; at < to; at += 64) {
        const uint32_t i = at + lane;
        const bool in = i < to;
        const uint32_t row = in ? pair_row(a, token, i) : 0, digit = row >> a.shift & mask;
        uint64_t peers = __ballot(in);
        for (int b = 0; b < a.bits; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            peers &= (digit >> b & 1) ? set : ~set;
        }
        const int first = __ffsll((unsigned long long)peers) - 1;      // of the pairs with this digit; it counts them all
        uint32_t place = 0;
        if (in && first == (int)lane) place = atomicAdd(&cnt[wave * buckets + digit], (uint32_t)__popcll(peers));
        place = __shfl(place, first, 64) + (uint32_t)__popcll(peers & ((1ull << lane) - 1));
        if (in) {
            a.to.row[place] = row;
            a.to.token[place] = a.from.row ? a.from.token[i] : i;
        }
    }
}

template <class I>
__global__ __launch_bounds__(kDigitWaves * 64) void count_digits_kernel(DigitArgs a, const I *__restrict__ token)
{
    __shared__ uint32_t s_cnt[1 << kDigitBits];
    const uint32_t buckets = 1u << a.bits;
    for (uint32_t i = threadIdx.x; i < buckets; i += blockDim.x) s_cnt[i] = 0;
    __syncthreads();
    const uint32_t per = kDigitWaves * a.per_wave, from = min(a.count, blockIdx.x * per), to = min(a.count, from + per);
    for (uint32_t i = from + threadIdx.x; i < to; i += blockDim.x) atomicAdd(&s_cnt[pair_row(a, token, i) >> a.shift & (buckets - 1)], 1u);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < buckets; i += blockDim.x) a.counts[(size_t)blockIdx.x * buckets + i] = s_cnt[i];
}

template <class I>
__global__ __launch_bounds__(kDigitWaves * 64) void place_digits_kernel(DigitArgs a, const I *__restrict__ token)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ uint32_t s_wave[kDigitWaves];
    place_digits(a, token, blockIdx.x, lds, s_wave);
}

// All digits in one workgroup; pass p leaves its pairs in pairs[p & 1].
struct PairBuffers { Pairs at[2]; };
template <class I>
__global__ __launch_bounds__(kDigitWaves * 64) void sort_pairs_kernel(DigitArgs a, const I *__restrict__ token, PairBuffers pairs, int passes)
{
    extern __shared__ __attribute__((aligned(16))) uint32_t lds[];
    __shared__ uint32_t s_wave[kDigitWaves];
    for (int p = 0; p < passes; ++p, a.shift += a.bits) {
        if (p) a.from = pairs.at[(p - 1) & 1];
        a.to = pairs.at[p & 1];
        place_digits(a, token, 0, lds, s_wave);
        __syncthreads();
    }
}

// ------------------------------------------------------------------ gradient
//
// Every row of the table adds up its tokens' rows of dy in the order of the tokens.  Where a row has many, sums of kRun
// consecutive places that are all its own are made beforehand, and of kRun such sums, each by a workgroup of its own; the row then
// takes the largest pieces that lie in its range.  Bound by bytes.
constexpr uint32_t kRun = 32;

// Where a row's places begin, plus one, and end; {0, ..} for rows that are no token's.
struct Places { uint32_t first, end; };

struct GradArgs {
    Pairs sorted;
    Places *places;         // [rows]
    float *run, *runs;      // sums of kRun places, and of kRun such sums, [count / kRun][cols] and [count / kRun^2][cols]
    uint32_t count, rows, cols;
    float scale;
};

__global__ __launch_bounds__(kWG) void clear_places_kernel(Places *places, uint32_t rows)
{
    for (uint32_t i = blockIdx.x * kWG + threadIdx.x; i < rows; i += gridDim.x * kWG) places[i] = Places{0, 0};
}

__global__ __launch_bounds__(kWG) void mark_places_kernel(GradArgs a)
{
    const uint32_t i = blockIdx.x * kWG + threadIdx.x;
    if (i >= a.count) return;
    const uint32_t row = a.sorted.row[i];
    if (row >= a.rows) return;
    if (i == 0 || a.sorted.row[i - 1] != row) a.places[row].first = i + 1;
    if (i + 1 == a.count || a.sorted.row[i + 1] != row) a.places[row].end = i + 1;
}

// acc += the rows of dy in places [from, to), columns col and further.
template <class T>
__device__ __forceinline__ void add_places(const GradArgs &a, const T *dy, int64_t ldy, uint32_t from, uint32_t to, uint32_t col, int n,
                                           float (&acc)[Unit<T>::kElems])
{
    constexpr int E = Unit<T>::kElems, AT_ONCE = 4;
    for (uint32_t at = from; at < to; at += AT_ONCE) {
        Unit<T> u[AT_ONCE];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
            if (at + i < to) u[i] = load_some(dy + (int64_t)a.sorted.token[at + i] * ldy + col, n);
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
            if (at + i < to) {
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] += (float)u[i].v[j];
            }
    }
}

// acc += sums [from, to) of those made beforehand.
template <int E>
__device__ __forceinline__ void add_sums(const float *sums, uint32_t cols, uint32_t from, uint32_t to, uint32_t col, int n, float (&acc)[E])
{
    for (uint32_t at = from; at < to; ++at)
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] += j < n ? sums[(size_t)at * cols + col + j] : 0.0f;
}

// LEVEL 1: sums of kRun places that are one row's; 2: of kRun such sums.
template <class T, int LANES, int LEVEL>
__global__ __launch_bounds__(kWG) void run_kernel(GradArgs a, const T *__restrict__ dy, int64_t ldy)
{
    constexpr int E = Unit<T>::kElems;
    constexpr uint32_t LENGTH = LEVEL == 1 ? kRun : kRun * kRun;
    const uint32_t runs = a.count / LENGTH;
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < runs; b += gridDim.y) {
        const uint32_t r = b * (kWG / LANES) + row_in_block<LANES>();
        if (r >= runs) continue;
        const uint32_t row = a.sorted.row[r * LENGTH];
        if (row >= a.rows || a.sorted.row[r * LENGTH + LENGTH - 1] != row) continue;
        for (uint32_t col = (blockIdx.x * LANES + threadIdx.x % LANES) * E; col < a.cols; col += gridDim.x * LANES * E) {
            const int n = (int)min((uint32_t)E, a.cols - col);
            float acc[E] = {};
            if constexpr (LEVEL == 1) add_places(a, dy, ldy, r * kRun, (r + 1) * kRun, col, n, acc);
            else add_sums<E>(a.run, a.cols, r * kRun, (r + 1) * kRun, col, n, acc);
            float *to = (LEVEL == 1 ? a.run : a.runs) + (size_t)r * a.cols + col;
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (j < n) to[j] = acc[j];
        }
    }
}

// E results, rounded to the type of the output.
template <class O, int E>
__device__ __forceinline__ void store_sums(O *p, const float (&v)[E], int n)
{
    constexpr int EO = Unit<O>::kElems;
#pragma unroll
    for (int at = 0; at < E; at += EO)
        if (at < n) {
            Unit<O> u;
#pragma unroll
            for (int j = 0; j < EO; ++j) u.v[j] = (O)v[at + j];
            store_some(p + at, u, n - at);
        }
}

// ADD: by place, the first of each row adds to it; else by row of the table.
template <class T, class O, int LANES, bool ADD>
__global__ __launch_bounds__(kWG) void embed_grad_kernel(GradArgs a, const T *__restrict__ dy, int64_t ldy, O *__restrict__ dtable, int64_t ldt)
{
    constexpr int E = Unit<T>::kElems;
    const uint32_t items = ADD ? a.count : a.rows;
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < items; b += gridDim.y) {
        const uint32_t item = b * (kWG / LANES) + row_in_block<LANES>();
        if (item >= items) continue;
        const uint32_t row = ADD ? a.sorted.row[item] : item;
        if (ADD && (row >= a.rows || (item > 0 && a.sorted.row[item - 1] == row))) continue;
        const Places p = a.places[row];
        const uint32_t first = p.first ? p.first - 1 : 0, end = p.first ? p.end : 0;
        // whole runs of kRun, and of kRun of these, in the row's range
        const uint32_t run0 = (first + kRun - 1) / kRun, run1 = end / kRun;
        const uint32_t runs0 = (run0 + kRun - 1) / kRun, runs1 = run1 / kRun;
        for (uint32_t col = (blockIdx.x * LANES + threadIdx.x % LANES) * E; col < a.cols; col += gridDim.x * LANES * E) {
            const int n = (int)min((uint32_t)E, a.cols - col);
            float acc[E] = {};
            if (run0 >= run1) add_places(a, dy, ldy, first, end, col, n, acc);
            else {
                add_places(a, dy, ldy, first, run0 * kRun, col, n, acc);
                if (runs0 >= runs1) add_sums<E>(a.run, a.cols, run0, run1, col, n, acc);
                else {
                    add_sums<E>(a.run, a.cols, run0, runs0 * kRun, col, n, acc);
                    add_sums<E>(a.runs, a.cols, runs0, runs1, col, n, acc);
                    add_sums<E>(a.run, a.cols, runs1 * kRun, run1, col, n, acc);
                }
                add_places(a, dy, ldy, run1 * kRun, end, col, n, acc);
            }
            O *to = dtable + (int64_t)row * ldt + col;
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] = !p.first ? 0.0f : a.scale * acc[j] + (ADD && j < n ? (float)to[j] : 0.0f);
            store_sums<O, E>(to, acc, n);
        }
    }
}

// ------------------------------------------------------------------ launches

// The lanes to a row, as a constant.
template <class F>
static void by_row_lanes(uint32_t cols, uint32_t elems, F f)
{
    const uint32_t pieces = (cols + elems - 1) / elems;
    if (pieces <= 32) f(std::integral_constant<int, 16>{});
    else if (pieces <= 128) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 256>{});
}
static dim3 row_grid(uint32_t rows, uint32_t cols, uint32_t elems, uint32_t lanes)
{
    const uint32_t per = kWG / lanes;
    return dim3(std::min(1024u, (cols + lanes * elems - 1) / (lanes * elems)), std::min((rows + per - 1) / per, 65535u));
}

void launch_embed(const void *token, bool wide, uint32_t tokens, const seer_dense &table, float scale, const seer_dense &out, hipStream_t st)
{
    by_type(table.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_row_lanes((uint32_t)table.cols, Unit<T>::kElems, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            const auto launch = [&](auto *ids) {
                using I = std::remove_pointer_t<decltype(ids)>;
                hipLaunchKernelGGL((embed_kernel<T, I, LANES>), row_grid(tokens, (uint32_t)table.cols, Unit<T>::kElems, LANES), dim3(kWG), 0, st,
                                   static_cast<const I *>(token), tokens, static_cast<const T *>(table.data), table.ld, (uint32_t)table.rows,
                                   (uint32_t)table.cols, scale, static_cast<T *>(out.data), out.ld);
            };
            if (wide) launch((int64_t *)nullptr);
            else launch((int32_t *)nullptr);
        });
    });
}

struct SortPlan { uint32_t per_wave, groups; int passes, bits; };

// One workgroup sorts few pairs in one launch; more take two launches for each digit.
static SortPlan sort_plan(uint32_t count, uint32_t rows)
{
    SortPlan p;
    int bits = 1;
    while (bits < 32 && rows >> bits) ++bits;           // `rows` is the largest key
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const uint32_t groups = count <= 8192 ? 1 : std::min((count + 4095) / 4096, 128u);
    const uint32_t share = (count + groups - 1) / groups;
    p.per_wave = std::max(64u, ((share + kDigitWaves - 1) / kDigitWaves + 63) & ~63u);
    p.groups = (count + kDigitWaves * p.per_wave - 1) / (kDigitWaves * p.per_wave);
    return p;
}

struct GradSpace { size_t pairs, counts, places, run, runs, bytes; };

static GradSpace grad_space(uint32_t count, uint32_t rows, uint32_t cols)
{
    const auto pad = [](size_t n) { return (n + 255) & ~(size_t)255; };
    const SortPlan p = sort_plan(count, rows);
    GradSpace s;
    s.pairs = 0;
    s.counts = 4 * pad((size_t)count * 4);
    s.places = s.counts + (p.groups > 1 ? pad(((size_t)p.groups << p.bits) * 4) : 0);
    s.run = s.places + pad((size_t)rows * sizeof(Places));
    s.runs = s.run + pad((size_t)(count / kRun) * cols * 4);
    s.bytes = s.runs + pad((size_t)(count / (kRun * kRun)) * cols * 4);
    return s;
}

size_t embed_grad_workspace_bytes(uint32_t count, uint32_t rows, uint32_t cols) { return grad_space(count, rows, cols).bytes; }

template <class I>
static Pairs launch_sort(const I *token, uint32_t count, uint32_t rows, char *ws, const GradSpace &s, hipStream_t st)
{
    const SortPlan p = sort_plan(count, rows);
    const size_t each = ((size_t)count * 4 + 255) & ~(size_t)255;
    const auto array = [&](int i) { return reinterpret_cast<uint32_t *>(ws + s.pairs + i * each); };
    const PairBuffers pairs{{Pairs{array(0), array(1)}, Pairs{array(2), array(3)}}};
    DigitArgs a{Pairs{nullptr, nullptr}, pairs.at[0], count, rows, p.per_wave, p.groups, 0, p.bits, reinterpret_cast<uint32_t *>(ws + s.counts)};
    const size_t lds = ((size_t)(kDigitWaves + 2) << p.bits) * 4 + 4;
    const dim3 wg(kDigitWaves * 64);
    if (p.groups == 1) {
        hipLaunchKernelGGL((sort_pairs_kernel<I>), dim3(1), wg, lds, st, a, token, pairs, p.passes);
        return pairs.at[(p.passes - 1) & 1];
    }
    for (int i = 0; i < p.passes; ++i, a.shift += a.bits) {
        if (i) a.from = pairs.at[(i - 1) & 1];
        a.to = pairs.at[i & 1];
        hipLaunchKernelGGL((count_digits_kernel<I>), dim3(p.groups), wg, 0, st, a, token);
        hipLaunchKernelGGL((place_digits_kernel<I>), dim3(p.groups), wg, lds, st, a, token);
    }
    return pairs.at[(p.passes - 1) & 1];
}

void launch_embed_grad(const void *token, bool wide, const seer_dense &dy, float scale, bool accumulate, const seer_dense &dtable, void *workspace,
                       hipStream_t st)
{
    const uint32_t count = (uint32_t)dy.rows, rows = (uint32_t)dtable.rows, cols = (uint32_t)dy.cols;
    char *ws = static_cast<char *>(workspace);
    const GradSpace s = grad_space(count, rows, cols);
    GradArgs a{Pairs{nullptr, nullptr}, reinterpret_cast<Places *>(ws + s.places), reinterpret_cast<float *>(ws + s.run),
               reinterpret_cast<float *>(ws + s.runs), count, rows, cols, scale};
    if (!accumulate) hipLaunchKernelGGL(clear_places_kernel, dim3(std::min((rows + kWG - 1) / kWG, 1024u)), dim3(kWG), 0, st, a.places, rows);
    if (count) {
        a.sorted = wide ? launch_sort(static_cast<const int64_t *>(token), count, rows, ws, s, st)
                        : launch_sort(static_cast<const int32_t *>(token), count, rows, ws, s, st);
        hipLaunchKernelGGL(mark_places_kernel, dim3((count + kWG - 1) / kWG), dim3(kWG), 0, st, a);
    }
    by_type(dy.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_row_lanes(cols, Unit<T>::kElems, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            const T *y = static_cast<const T *>(dy.data);
            const auto grid = [&](uint32_t n) { return row_grid(n, cols, Unit<T>::kElems, LANES); };
            if (count >= kRun) hipLaunchKernelGGL((run_kernel<T, LANES, 1>), grid(count / kRun), dim3(kWG), 0, st, a, y, dy.ld);
            if (count >= kRun * kRun) hipLaunchKernelGGL((run_kernel<T, LANES, 2>), grid(count / (kRun * kRun)), dim3(kWG), 0, st, a, y, dy.ld);
            const auto launch = [&](auto *to) {
                using O = std::remove_pointer_t<decltype(to)>;
                if (accumulate)
                    hipLaunchKernelGGL((embed_grad_kernel<T, O, LANES, true>), grid(count), dim3(kWG), 0, st, a, y, dy.ld,
                                       static_cast<O *>(dtable.data), dtable.ld);
                else
                    hipLaunchKernelGGL((embed_grad_kernel<T, O, LANES, false>), grid(rows), dim3(kWG), 0, st, a, y, dy.ld,
                                       static_cast<O *>(dtable.data), dtable.ld);
            };
            if (dtable.type == dy.type) launch((T *)nullptr);
            else if constexpr (!std::is_same<T, float>::value) launch((float *)nullptr);
        });
    });
}

} // namespace seer
