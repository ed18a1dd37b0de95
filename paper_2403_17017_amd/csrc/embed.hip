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
// Bound by bytes: each row is read and written once.  32 771 tokens, 131 072 x 4096 bf16: 87 us, 81 at least (268 MB written; of the rows, 11 000 different ones,
// 162 MB come from memory: 4.9 to 5.3 TB/s).
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
    uint32_t *counts;       // [groups][1 << bits]
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
    for (uint32_t i = threadIdx.x, all = a.groups * buckets; i < all; i += blockDim.x) {
        const uint32_t n = a.counts[i];
        if (n == 0) continue;
        atomicAdd(&base[i & mask], n);
        if (i >> a.bits < group) atomicAdd(&before[i & mask], n);
    }
    __syncthreads();
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

// Where a row's places begin, plus one, and end; {0, ..} for rows that are no token's.
struct Places { uint32_t first, end; };
// Beside the first launch of a sort other workgroups clear these (rows 0: they were not asked for).
struct Clear { Places *places; uint32_t rows; };
constexpr uint32_t kClearRows = 8192;               // of a workgroup

__device__ __forceinline__ void clear_places(const Clear &c, uint32_t block)
{
    for (uint32_t i = block * kClearRows + threadIdx.x, end = min(c.rows, (block + 1) * kClearRows); i < end; i += blockDim.x) c.places[i] = Places{0, 0};
}
__global__ __launch_bounds__(kDigitWaves * 64) void clear_places_kernel(Clear c) { clear_places(c, blockIdx.x); }

template <class I>
__global__ __launch_bounds__(kDigitWaves * 64) void count_digits_kernel(DigitArgs a, const I *__restrict__ token, Clear clear)
{
    __shared__ uint32_t s_cnt[1 << kDigitBits];
    if (blockIdx.x >= a.groups) return clear_places(clear, blockIdx.x - a.groups);
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

// Few tokens find their places by counting, 16 lanes to a token: the rows below its own, and its own row's tokens before it.  Every
// token looks at all, so this grows with their square, but it is one launch.  The whole gradient, us, so and with the sort: 8009 x 1023 fp32, 1024 tokens 27 and 35, 3000
// 40 and 42, 4096 47 and 45, 8192 66 and 49; 32 000 x 512 bf16, 1024 22 and 30, 4096 34 and 35, 6000 43 and 38; 131 072 x 64, 1024 18 and 28, 4096 33 and 35, 6000 39 and
// 36.  Of a table whose rows are one digit the sort is two launches: 100 x 256, 1024 tokens 16 and 17, 2048 22 and 21, 4096 30 and 23.
constexpr uint32_t kRankTokens = 4096, kRankLanes = 16;

template <class I>
__global__ __launch_bounds__(kWG) void rank_pairs_kernel(const I *__restrict__ token, uint32_t count, uint32_t rows, Pairs to, uint32_t blocks, Clear clear)
{
    __shared__ __attribute__((aligned(16))) uint32_t s_row[kRankTokens];
    if (blockIdx.x >= blocks) return clear_places(clear, blockIdx.x - blocks);
    const uint32_t padded = (count + 3) & ~3u;
    for (uint32_t i = threadIdx.x; i < padded; i += kWG) s_row[i] = i < count ? row_of(token, i, rows) : ~0u;     // (behind all rows)
    __syncthreads();
    const uint32_t t = blockIdx.x * (kWG / kRankLanes) + threadIdx.x / kRankLanes, lane = threadIdx.x % kRankLanes;
    const uint32_t row = s_row[min(t, count - 1)];
    uint32_t before = 0;
    for (uint32_t i = lane * 4; i < padded; i += kRankLanes * 4) {
        const v4i k = *reinterpret_cast<const v4i *>(s_row + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) before += (uint32_t)k[j] < row || ((uint32_t)k[j] == row && i + j < t);
    }
#pragma unroll
    for (uint32_t d = 1; d < kRankLanes; d <<= 1) before += (uint32_t)__shfl_xor((int)before, (int)d, kWave);
    if (t < count && lane == 0) {
        to.row[before] = row;
        to.token[before] = t;
    }
}

// ------------------------------------------------------------------ gradient
//
// Every row of the table adds up its tokens' rows of dy in the order of the tokens.  Where a row has many, sums of kRun
// consecutive places that are all its own are made beforehand, and of kRun such sums, each by a workgroup of its own; the row then
// takes the largest pieces that lie in its range.  1031 tokens by a power law, 8009 x 1023 fp32, the whole
// gradient: 26 us with runs of 16 (of which the sums made beforehand take 7.6 and the rows 13.4), 42 with runs of 32; 32 768 tokens, 131 072 x 4096 bf16, 287 and 290.
constexpr uint32_t kRun = 16;

struct GradArgs {
    Pairs sorted;
    Places *places;         // [rows]
    float *run, *runs;      // sums of kRun places, and of kRun such sums, [count / kRun][pitch] and [count / kRun^2][pitch]; runs may be null
    uint32_t count, rows, cols, pitch;
    float scale;
};

__device__ __forceinline__ void mark_places(const GradArgs &a, uint32_t i)
{
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
    constexpr int E = Unit<T>::kElems, AT_ONCE = 16;
    uint32_t at = from;
    for (; at + AT_ONCE <= to; at += AT_ONCE) {
        Unit<T> u[AT_ONCE];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i) u[i] = load_some(dy + (int64_t)a.sorted.token[at + i] * ldy + col, n);
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] += (float)u[i].v[j];
    }
    if (at < to) {                                      // (the last one again, and not added)
        Unit<T> u[AT_ONCE - 1];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE - 1; ++i)
            if (at + i < to) u[i] = load_some(dy + (int64_t)a.sorted.token[at + i] * ldy + col, n);
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE - 1; ++i)
            if (at + i < to) {
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] += (float)u[i].v[j];
            }
    }
}

// acc += sums [from, to) of those made beforehand.
template <int E>
__device__ __forceinline__ void add_sums(const float *sums, uint32_t pitch, uint32_t from, uint32_t to, uint32_t col, float (&acc)[E])
{
    constexpr uint32_t AT_ONCE = 8;
    for (uint32_t at = from; at < to; at += AT_ONCE) {
        v4f u[AT_ONCE][E / 4];
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
            if (at + i < to) {
#pragma unroll
                for (int j = 0; j < E / 4; ++j)
                    if (col + 4 * j < pitch) u[i][j] = *reinterpret_cast<const v4f *>(sums + (size_t)(at + i) * pitch + col + 4 * j);
            }
#pragma unroll
        for (uint32_t i = 0; i < AT_ONCE; ++i)
            if (at + i < to) {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (col + j / 4 * 4 < pitch) acc[j] += u[i][j / 4][j % 4];
            }
    }
}

// LEVEL 1: sums of kRun places that are one row's, and, in the first workgroups, where each row's places are; 2: of kRun such sums.
template <class T, int LANES, int LEVEL>
__global__ __launch_bounds__(kWG) void run_kernel(GradArgs a, const T *__restrict__ dy, int64_t ldy, uint32_t marking)
{
    constexpr int E = Unit<T>::kElems;
    constexpr uint32_t LENGTH = LEVEL == 1 ? kRun : kRun * kRun, ROWS = kWG / LANES;
    if (LEVEL == 1 && blockIdx.x < marking) return mark_places(a, blockIdx.x * kWG + threadIdx.x);
    const uint32_t runs = a.count / LENGTH, across = (a.cols + LANES * E - 1) / (LANES * E), block = blockIdx.x - marking;
    const uint32_t r = block / across * ROWS + row_in_block<LANES>(), col = (block % across * LANES + threadIdx.x % LANES) * E;
    if (r >= runs || col >= a.cols) return;
    const uint32_t row = a.sorted.row[r * LENGTH];
    if (row >= a.rows || a.sorted.row[r * LENGTH + LENGTH - 1] != row) return;
    const int n = (int)min((uint32_t)E, a.cols - col);
    float acc[E] = {};
    if constexpr (LEVEL == 1) add_places(a, dy, ldy, r * kRun, (r + 1) * kRun, col, n, acc);
    else add_sums<E>(a.run, a.pitch, r * kRun, (r + 1) * kRun, col, acc);
    float *to = (LEVEL == 1 ? a.run : a.runs) + (size_t)r * a.pitch + col;
#pragma unroll
    for (int j = 0; j < E; j += 4)
        if (j < n) *reinterpret_cast<v4f *>(to + j) = v4f{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
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

// The rows that are a token's: the first of a row's places is who adds up, LANES lanes to UNITS pieces of 16 bytes each (of dy), a row in as many
// parts as that takes; plus what is there, with ADD.  Its loads wait for one another four deep, so what counts is how many rows are
// under way, and how many of a row's places: 131 072 x 4096 bf16 with 28 000 rows of tokens, the whole call, 322 us with a workgroup to each row,
// 286 with four pieces and four places at a time, 275 with two and eight; 50 000 x 1024 84 and 67, 8000 x 512 54 and 44.
template <class T, class O, int LANES, int UNITS, bool ADD>
__device__ __forceinline__ void sum_row(const GradArgs &a, const T *__restrict__ dy, int64_t ldy, O *__restrict__ dtable, int64_t ldt, uint32_t i, uint32_t part)
{
    constexpr int E = Unit<T>::kElems;
    constexpr uint32_t AT_ONCE = 8;
    const uint32_t row = a.sorted.row[i];
    if (row >= a.rows || (i > 0 && a.sorted.row[i - 1] == row)) return;
    const uint32_t end = a.places[row].end, col0 = (part * UNITS * LANES + threadIdx.x % LANES) * E;
    O *to = dtable + (int64_t)row * ldt;
    float acc[UNITS][E] = {};
    Unit<O> held[ADD ? UNITS : 1][E / Unit<O>::kElems];
    const auto have = [&](int u) { return (int)a.cols - (int)(col0 + u * LANES * E); };         // columns from piece u's first on
    if constexpr (ADD) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int j = 0; j < E; j += Unit<O>::kElems)
                if (have(u) > j) held[u][j / Unit<O>::kElems] = load_some(to + col0 + u * LANES * E + j, have(u) - j);
    }
    const auto add = [&](uint32_t from, uint32_t upto) {
        for (uint32_t at = from; at < upto; at += AT_ONCE) {
            Unit<T> v[AT_ONCE][UNITS];
#pragma unroll
            for (uint32_t k = 0; k < AT_ONCE; ++k)
                if (at + k < upto) {
                    const T *y = dy + (int64_t)a.sorted.token[at + k] * ldy + col0;
#pragma unroll
                    for (int u = 0; u < UNITS; ++u)
                        if (have(u) > 0) v[k][u] = load_some(y + u * LANES * E, have(u));
                }
#pragma unroll
            for (uint32_t k = 0; k < AT_ONCE; ++k)
                if (at + k < upto) {
#pragma unroll
                    for (int u = 0; u < UNITS; ++u)
#pragma unroll
                        for (int j = 0; j < E; ++j) acc[u][j] += (float)v[k][u].v[j];
                }
        }
    };
    // whole runs of kRun, and of kRun of these, in the row's range
    const uint32_t run0 = (i + kRun - 1) / kRun, run1 = end / kRun;
    const uint32_t runs0 = (run0 + kRun - 1) / kRun, runs1 = a.runs ? run1 / kRun : 0;
    const auto sums = [&](const float *of, uint32_t from, uint32_t upto) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) add_sums<E>(of, a.pitch, from, upto, col0 + u * LANES * E, acc[u]);
    };
    if (run0 >= run1) add(i, end);
    else {
        add(i, run0 * kRun);
        if (runs0 >= runs1) sums(a.run, run0, run1);
        else {
            sums(a.run, run0, runs0 * kRun);
            sums(a.runs, runs0, runs1);
            sums(a.run, runs1 * kRun, run1);
        }
        add(run1 * kRun, end);
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
        if (have(u) <= 0) continue;
#pragma unroll
        for (int j = 0; j < E; ++j) acc[u][j] = a.scale * acc[u][j] + (ADD ? (float)held[ADD ? u : 0][j / Unit<O>::kElems].v[j % Unit<O>::kElems] : 0.0f);
        store_sums<O, E>(to + col0 + u * LANES * E, acc[u], have(u));
    }
}

// The first `summing` workgroups; the others write zeros to rows that are no token's, kAhead rows at a time.
// STREAM: whole rows lie at multiples of 16 bytes and leave the caches as they are written.
constexpr uint32_t kAhead = 2;

template <class T, class O, int LANES, int UNITS, bool ADD, bool STREAM>
__global__ __launch_bounds__(kWG) void rows_kernel(GradArgs a, const T *__restrict__ dy, int64_t ldy, O *__restrict__ dtable, int64_t ldt, uint32_t summing)
{
    constexpr uint32_t ROWS = kWG / LANES;
    if (blockIdx.x < summing) {
        const uint32_t parts = (a.cols + UNITS * LANES * Unit<T>::kElems - 1) / (UNITS * LANES * Unit<T>::kElems);
        const uint64_t items = (uint64_t)a.count * parts;
        for (uint64_t w = (uint64_t)blockIdx.x * ROWS + row_in_block<LANES>(); w < items; w += (uint64_t)summing * ROWS)
            sum_row<T, O, LANES, UNITS, ADD>(a, dy, ldy, dtable, ldt, (uint32_t)(w / parts), (uint32_t)(w % parts));
        return;
    }
    constexpr int E = Unit<O>::kElems;
    constexpr uint32_t ZLANES = LANES < kWave ? LANES : kWG, ZROWS = kWG / ZLANES;
    const uint32_t lane = threadIdx.x % ZLANES;
    for (uint32_t b = blockIdx.x - summing; b * ZROWS * kAhead < a.rows; b += gridDim.x - summing) {
        const uint32_t row0 = b * ZROWS * kAhead + row_in_block<ZLANES>();
        uint32_t first[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) first[i] = a.places[min(row0 + i * ZROWS, a.rows - 1)].first;
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) {
            const uint32_t row = row0 + i * ZROWS;
            if (row >= a.rows || first[i]) continue;
            O *to = dtable + (int64_t)row * ldt;
            for (uint32_t col = lane * E; col < a.cols; col += ZLANES * E) store_row<STREAM>(to + col, zero_unit<O>(), (int)min((uint32_t)E, a.cols - col));
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
static bool aligned_rows(const seer_dense &m, size_t size)
{
    return reinterpret_cast<uintptr_t>(m.data) % 16 == 0 && (size_t)m.ld * size % 16 == 0;
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

// Two launches for each digit.
static SortPlan sort_plan(uint32_t count, uint32_t rows)
{
    SortPlan p;
    int bits = 1;
    while (bits < 32 && rows >> bits) ++bits;           // `rows` is the largest key
    p.passes = (bits + kDigitBits - 1) / kDigitBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    const uint32_t groups = std::min(std::max((count + 1023) / 1024, 1u), 128u);
    const uint32_t share = (count + groups - 1) / groups;
    p.per_wave = std::max(64u, ((share + kDigitWaves - 1) / kDigitWaves + 63) & ~63u);
    p.groups = (count + kDigitWaves * p.per_wave - 1) / (kDigitWaves * p.per_wave);
    return p;
}

// Sums of sums are worth their launch from here on: one row's tokens may be all of them.  Without and with, us: all tokens of one row of 1024 bf16, 1024 tokens
// 26 and 16, 2040 45 and 25, 4096 79 and 29; where no row has that many, the launch alone: 32 000 x 512, 1024 tokens 22.2 and 23.5, 2048 25.3 and 26.8, 8192 36 and
// 39; 8009 x 1023 fp32 by a power law, 4096 42 and 47, 16 384 63 and 57.
constexpr uint32_t kManyTokens = 2048;

struct GradSpace { size_t pairs, counts, places, run, runs, bytes; };
static uint32_t sum_pitch(uint32_t cols) { return (cols + 3) & ~3u; }

static GradSpace grad_space(uint32_t count, uint32_t rows, uint32_t cols)
{
    const auto pad = [](size_t n) { return (n + 255) & ~(size_t)255; };
    const SortPlan p = sort_plan(count, rows);
    GradSpace s;
    s.pairs = 0;
    s.counts = 4 * pad((size_t)count * 4);
    s.places = s.counts + pad(((size_t)p.groups << p.bits) * 4);
    s.run = s.places + pad((size_t)rows * sizeof(Places));
    s.runs = s.run + pad((size_t)(count / kRun) * sum_pitch(cols) * 4);
    s.bytes = s.runs + (count < kManyTokens ? 0 : pad((size_t)(count / (kRun * kRun)) * sum_pitch(cols) * 4));
    return s;
}

size_t embed_grad_workspace_bytes(uint32_t count, uint32_t rows, uint32_t cols) { return grad_space(count, rows, cols).bytes; }

template <class I>
static Pairs launch_sort(const I *token, uint32_t count, uint32_t rows, char *ws, const GradSpace &s, const Clear &clear, hipStream_t st)
{
    const uint32_t clearing = (clear.rows + kClearRows - 1) / kClearRows;
    const size_t each = ((size_t)count * 4 + 255) & ~(size_t)255;
    const auto array = [&](int i) { return reinterpret_cast<uint32_t *>(ws + s.pairs + i * each); };
    const Pairs pairs[2] = {{array(0), array(1)}, {array(2), array(3)}};
    if (count <= kRankTokens) {
        const uint32_t blocks = (count + kWG / kRankLanes - 1) / (kWG / kRankLanes);
        hipLaunchKernelGGL((rank_pairs_kernel<I>), dim3(blocks + clearing), dim3(kWG), 0, st, token, count, rows, pairs[0], blocks, clear);
        return pairs[0];
    }
    const SortPlan p = sort_plan(count, rows);
    DigitArgs a{Pairs{nullptr, nullptr}, pairs[0], count, rows, p.per_wave, p.groups, 0, p.bits, reinterpret_cast<uint32_t *>(ws + s.counts)};
    const size_t lds = ((size_t)(kDigitWaves + 2) << p.bits) * 4 + 4;
    const dim3 wg(kDigitWaves * 64);
    for (int i = 0; i < p.passes; ++i, a.shift += a.bits) {
        if (i) a.from = pairs[(i - 1) & 1];
        a.to = pairs[i & 1];
        hipLaunchKernelGGL((count_digits_kernel<I>), dim3(p.groups + (i ? 0 : clearing)), wg, 0, st, a, token, clear);
        hipLaunchKernelGGL((place_digits_kernel<I>), dim3(p.groups), wg, lds, st, a, token);
    }
    return pairs[(p.passes - 1) & 1];
}

void launch_embed_grad(const void *token, bool wide, const seer_dense &dy, float scale, bool accumulate, const seer_dense &dtable, void *workspace,
                       hipStream_t st)
{
    const uint32_t count = (uint32_t)dy.rows, rows = (uint32_t)dtable.rows, cols = (uint32_t)dy.cols;
    char *ws = static_cast<char *>(workspace);
    const GradSpace s = grad_space(count, rows, cols);
    GradArgs a{Pairs{nullptr, nullptr}, reinterpret_cast<Places *>(ws + s.places), reinterpret_cast<float *>(ws + s.run),
               count < kManyTokens ? nullptr : reinterpret_cast<float *>(ws + s.runs), count, rows, cols, sum_pitch(cols), scale};
    const Clear clear{a.places, accumulate ? 0 : rows};
    if (count)
        a.sorted = wide ? launch_sort(static_cast<const int64_t *>(token), count, rows, ws, s, clear, st)
                        : launch_sort(static_cast<const int32_t *>(token), count, rows, ws, s, clear, st);
    else hipLaunchKernelGGL(clear_places_kernel, dim3((rows + kClearRows - 1) / kClearRows), dim3(kDigitWaves * 64), 0, st, clear);
    by_type(dy.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        by_row_lanes(cols, Unit<T>::kElems, [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            constexpr uint32_t ROWS = kWG / LANES, E = Unit<T>::kElems;
            const T *y = static_cast<const T *>(dy.data);
            const uint32_t across = (cols + LANES * E - 1) / (LANES * E), marking = (count + kWG - 1) / kWG;
            const auto runs = [&](uint32_t n) { return (n + ROWS - 1) / ROWS * across; };
            if (count) hipLaunchKernelGGL((run_kernel<T, LANES, 1>), dim3(marking + runs(count / kRun)), dim3(kWG), 0, st, a, y, dy.ld, marking);
            if (a.runs) hipLaunchKernelGGL((run_kernel<T, LANES, 2>), dim3(runs(count / (kRun * kRun))), dim3(kWG), 0, st, a, y, dy.ld, 0);
            const auto launch = [&](auto *out) {
                using O = std::remove_pointer_t<decltype(out)>;
                constexpr int L = LANES < kWave ? LANES : kWave, UNITS = LANES < kWave ? 1 : 2;
                constexpr uint32_t PART = L * UNITS * E, WAVES = kWG / L, ZROWS = LANES < kWave ? kWG / LANES : 1;
                O *to = static_cast<O *>(dtable.data);
                const uint64_t items = (uint64_t)count * ((cols + PART - 1) / PART);
                const uint32_t summing = (uint32_t)std::min<uint64_t>((items + WAVES - 1) / WAVES, 1u << 20);
                const uint32_t zeroing = std::min((rows + ZROWS * kAhead - 1) / (ZROWS * kAhead), 1u << 20);
                if (accumulate)
                    hipLaunchKernelGGL((rows_kernel<T, O, L, UNITS, true, false>), dim3(summing), dim3(kWG), 0, st, a, y, dy.ld, to, dtable.ld, summing);
                else if (aligned_rows(dtable, sizeof(O)))
                    hipLaunchKernelGGL((rows_kernel<T, O, L, UNITS, false, true>), dim3(summing + zeroing), dim3(kWG), 0, st, a, y, dy.ld, to, dtable.ld, summing);
                else
                    hipLaunchKernelGGL((rows_kernel<T, O, L, UNITS, false, false>), dim3(summing + zeroing), dim3(kWG), 0, st, a, y, dy.ld, to, dtable.ld, summing);
            };
            if (dtable.type == dy.type) launch((T *)nullptr);
            else if constexpr (!std::is_same<T, float>::value) launch((float *)nullptr);
        });
    });
}

} // namespace seer
