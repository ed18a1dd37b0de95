// Products of 8-bit integers with a scale for each token and channel, over ragged groups of rows:
//   out[i][n] = a_scale[i] * b_scale[g][n] * sum_k a[i][k] * b[g][n][k],  group_ptr[g] <= i < group_ptr[g + 1].
// The sums are 32-bit integers, exact whatever the order; one rounding to fp32 follows, two products there and
// the rounding to the type of the output.  The matrix instructions take channels for their rows and tokens for their
// columns, so that a lane's results are consecutive channels of one token.
#include "dense.hiph"
#include "dense_launch.h"
#include "i8_pieces.hiph"

namespace seer {

typedef int v4i32 __attribute__((ext_vector_type(4)));

// A tile: the rows of group `group` from `begin` to `end`, and which of the `across` tiles beside one another.  Group number
// `groups` stands for the rows behind the last one.
struct Tile { uint32_t group, begin, end, column; };

__device__ __forceinline__ uint32_t group_begin(const I8Args &a, uint32_t g)
{
    if (g > a.groups) return a.rows;
    if (!a.group_ptr) return g ? a.rows : 0;
    const int32_t p = a.group_ptr[g];
    return p < 0 ? 0 : min((uint32_t)p, a.rows);
}

// The last group that begins at or before a row; `groups`: none's.
__device__ __forceinline__ uint32_t group_of(const I8Args &a, uint32_t row)
{
    uint32_t low = 0, high = a.groups + 1;
    if (!a.group_ptr) return 0;
    while (low + 1 < high) {
        const uint32_t mid = (low + high) / 2;
        if (group_begin(a, mid) <= row) low = mid;
        else high = mid;
    }
    return low;
}

// What a lane knows of group g: its rows, and the tiles that they take.
struct GroupTiles { uint32_t from, to, tiles; };

__device__ __forceinline__ GroupTiles group_tiles(const I8Args &a, uint32_t g, uint32_t tokens)
{
    GroupTiles t;
    t.from = group_begin(a, min(g, a.groups + 1));
    t.to = group_begin(a, min(g + 1, a.groups + 1));
    t.tiles = t.to > t.from ? (t.to - t.from + tokens - 1) / tokens : 0;
    return t;
}

// Tiles lie in the order of the groups; in a group, kPanel rows of tiles make a panel that is gone through column by
// column, so that workgroups that run at the same time on an XCD share rows of both matrices in its L2, and every XCD has as
// many of the tiles that there are (of 32 groups and 32768 rows of 4096 x 4096: 780 us when they were dealt out by row
// of tiles among those that there may be, 685 us so).
constexpr uint32_t kPanel = 4;

__device__ __forceinline__ Tile tile_in_group(uint32_t group, uint32_t from, uint32_t to, uint32_t local, uint32_t tokens, uint32_t across)
{
    const uint32_t down = (to - from + tokens - 1) / tokens, panel = local / (kPanel * across), rest = local % (kPanel * across);
    const uint32_t height = min(kPanel, down - panel * kPanel), row = panel * kPanel + rest % height;
    Tile t;
    t.group = group;
    t.begin = from + row * tokens;
    t.end = min(to, t.begin + tokens);
    t.column = rest / height;
    return t;
}

// The tile of workgroup `block` among the tiles there are: as many for each XCD.  False: there is none.  All WAVES waves of the
// workgroup take part, a group to a lane; the result is uniform.  s: LDS of the workgroup, free again after the next barrier.
struct TileSearch { uint32_t sum[16], found[4]; };

template <uint32_t WAVES>
__device__ __forceinline__ bool find_tile(const I8Args &a, uint32_t block, uint32_t tokens, uint32_t across, TileSearch *s, Tile *t)
{
    if (!a.group_ptr) {
        const uint32_t all = (a.rows + tokens - 1) / tokens * across, w = tile_of_block(block, all, 1);
        if (w >= all) return false;
        *t = tile_in_group(0, 0, a.rows, w, tokens, across);
        return true;
    }
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    // tiles of the groups from `at` up to the lane's and with it; `all`: of all WAVES * 64 groups
    const auto prefix = [&](uint32_t tiles, uint32_t *all) {
        uint32_t sum = tiles;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = __shfl_up(sum, d, 64);
            if ((int)lane >= d) sum += other;
        }
        __syncthreads();
        if (lane == 63) s->sum[wave] = sum;
        __syncthreads();
        *all = 0;
#pragma unroll
        for (uint32_t w = 0; w < WAVES; ++w) {
            if (w < wave) sum += s->sum[w];
            *all += s->sum[w];
        }
        return sum;
    };
    constexpr uint32_t kAtOnce = WAVES * 64;
    uint32_t all = 0, before = 0, sum = 0, here = 0;
    GroupTiles g;
    for (uint32_t at = 0; at <= a.groups; at += kAtOnce) {
        g = group_tiles(a, at + threadIdx.x, tokens);
        sum = prefix(g.tiles, &here);
        all += here;
    }
    const uint32_t w = tile_of_block(block, all * across, 1);
    if (w >= all * across) return false;
    for (uint32_t at = 0; at <= a.groups; at += kAtOnce) {
        if (a.groups >= kAtOnce) {                  // (else they are known)
            g = group_tiles(a, at + threadIdx.x, tokens);
            sum = prefix(g.tiles, &here);
        }
        const uint32_t last = (before + sum) * across, first = last - g.tiles * across;
        if (first <= w && w < last) {               // one lane of the workgroup
            s->found[0] = at + threadIdx.x;
            s->found[1] = g.from;
            s->found[2] = g.to;
            s->found[3] = w - first;
        }
        before += here;
    }
    __syncthreads();
    const auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    *t = tile_in_group(uniform(s->found[0]), uniform(s->found[1]), uniform(s->found[2]), uniform(s->found[3]), tokens, across);
    return true;
}

// Rows of tiles of `tokens` rows that any division of the rows into groups needs.
static uint64_t most_tiles(const I8Args &a, uint32_t tokens)
{
    return a.group_ptr ? (uint64_t)a.rows / tokens + std::min(a.groups + 1, a.rows) : ((uint64_t)a.rows + tokens - 1) / tokens;
}

// Consecutive channels of one token, converted: 4 of them from channel n on, those below `channels`.
template <class T>
__device__ __forceinline__ void store_4(T *row, uint32_t n, uint32_t channels, const float (&v)[4])
{
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (n + 4 <= channels) {
        vec o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (T)v[j];
        *reinterpret_cast<vec *>(row + n) = o;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (n + j < channels) row[n + j] = (T)v[j];
    }
}

// ------------------------------------------------------------------ any size, any alignment
//
// For rows that do not lie at multiples of 16 bytes: 128 tokens x 128 channels, 128 columns at a time through registers and LDS, four
// waves of 64 x 64 each.  16 bytes of a row at a time, from any address; nothing is read behind the end of a row but the rest of its last
// word.  The next columns are fetched while these are multiplied: 3001 x 5001 x 4111 in 154 us, 800 TOP/s (66 in tiles, where rows lie
// at 4112; 278 with 64 x 64, nothing under way and loads from odd addresses).
constexpr uint32_t kAnyTokens = 128, kAnyChannels = 128, kAnyCols = 128, kAnyPitch = kAnyCols + 16;

// The first n bytes, and zeros behind them.
__device__ __forceinline__ v4i32 first_bytes(v4i32 v, int n)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int keep = min(max(n - 4 * j, 0), 4);
        v[j] = keep ? v[j] & (int)(~0u >> (32 - 8 * keep)) : 0;
    }
    return v;
}

// 16 bytes from any address, of which n are there (at least 1), out of whole words: loads that are not at multiples of 4 take four times as long.
// (A word of which a byte is there is in memory.)
__device__ __forceinline__ v4i32 load_16(const int8_t *p, int n)
{
    typedef int words __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t by = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const int8_t *from = p - by;
    int w[5];
    if (n >= 16) {
        const words v = *reinterpret_cast<const words *>(from);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = v[j];
        w[4] = *reinterpret_cast<const int *>(from + (by ? 16 : 12));
    } else {
        const int last = ((int)by + n - 1) / 4;
#pragma unroll
        for (int j = 0; j < 5; ++j) w[j] = *reinterpret_cast<const int *>(from + 4 * min(j, last));
    }
    v4i32 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (int)__builtin_amdgcn_alignbyte((uint32_t)w[j + 1], (uint32_t)w[j], by);
    return n >= 16 ? v : first_bytes(v, n);
}

template <class T>
__global__ __launch_bounds__(256) void i8_any_kernel(I8Args a, uint32_t blocks)
{
    __shared__ __attribute__((aligned(16))) int8_t s_a[kAnyTokens * kAnyPitch], s_b[kAnyChannels * kAnyPitch];
    __shared__ TileSearch s_search;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    for (uint32_t w = blockIdx.x; w < blocks; w += gridDim.x) {
        Tile t;
        if (!find_tile<4>(a, w, kAnyTokens, (a.channels + kAnyChannels - 1) / kAnyChannels, &s_search, &t)) continue;
        const uint32_t n0 = t.column * kAnyChannels;
        v4i32 acc[4][4] = {};
        if (t.group < a.groups) {
            const int8_t *b = a.b + (int64_t)t.group * a.channels * a.ldb;
            constexpr uint32_t kPieces = kAnyCols / 16, kEach = kAnyTokens * kPieces / 256;
            const uint32_t row = threadIdx.x / kPieces, col = threadIdx.x % kPieces * 16;     // and 256 / kPieces rows further on
            v4i32 va[kEach], vb[kEach];
            const int8_t *pa[kEach], *pb[kEach];                // (rows that are not there are taken as the last one: nobody stores them)
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) {
                const uint32_t at = row + i * (256 / kPieces);
                pa[i] = a.a + (int64_t)min(t.begin + at, t.end - 1) * a.lda;
                pb[i] = b + (int64_t)min(n0 + at, a.channels - 1) * a.ldb;
            }
            const auto fetch = [&](uint32_t k0) {
                if (k0 + kAnyCols <= a.columns) {
#pragma unroll
                    for (uint32_t i = 0; i < kEach; ++i) {
                        va[i] = load_16(pa[i] + (k0 + col), 16);
                        vb[i] = load_16(pb[i] + (k0 + col), 16);
                    }
                } else if (k0 < a.columns) {
                    const RowPiece p = row_piece(k0, col, a.columns);       // (b's columns behind the end meet zeros)
#pragma unroll
                    for (uint32_t i = 0; i < kEach; ++i) {
                        va[i] = first_bytes(load_16(pa[i] + p.from, p.have), p.keep);
                        vb[i] = load_16(pb[i] + p.from, p.have);
                    }
                }
            };
            fetch(0);
            for (uint32_t k0 = 0; k0 < a.columns; k0 += kAnyCols) {
                __syncthreads();
#pragma unroll
                for (uint32_t i = 0; i < kEach; ++i) {
                    const uint32_t at = (row + i * (256 / kPieces)) * kAnyPitch + col;
                    *reinterpret_cast<v4i32 *>(s_a + at) = va[i];
                    *reinterpret_cast<v4i32 *>(s_b + at) = vb[i];
                }
                __syncthreads();
                fetch(k0 + kAnyCols);
#pragma unroll
                for (uint32_t k = 0; k < kAnyCols; k += 64) {
                    v4i32 fb[4], fa[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        fb[i] = *reinterpret_cast<const v4i32 *>(s_b + ((wave & 1) * 64 + i * 16 + (lane & 15)) * kAnyPitch + k + lane / 16 * 16);
                        fa[i] = *reinterpret_cast<const v4i32 *>(s_a + ((wave >> 1) * 64 + i * 16 + (lane & 15)) * kAnyPitch + k + lane / 16 * 16);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[i], fa[j], acc[i][j], 0, 0, 0);
                }
            }
        }
        // (every scale is fetched before the first store: a wait for a load is one for all stores before it, too)
        const bool zero = t.group >= a.groups;
        const float *sb = a.b_scale + (int64_t)(zero ? 0 : t.group) * a.channels;
        const uint32_t row1 = t.begin + (wave >> 1) * 64 + (lane & 15), n1 = n0 + (wave & 1) * 64 + lane / 16 * 4;
        float of_row[4], of_channel[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) of_row[j] = a.a_scale[min(row1 + j * 16, t.end - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) of_channel[i][v] = sb[min(n1 + i * 16 + v, a.channels - 1)];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t row = row1 + j * 16, n = n1 + i * 16;
                if (row >= t.end || n >= a.channels) continue;
                float v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = zero ? 0.0f : (float)acc[i][j][u] * (of_row[j] * of_channel[i][u]);
                store_4(static_cast<T *>(a.out) + (int64_t)row * a.ldo, n, a.channels, v);
            }
    }
}

// ------------------------------------------------------------------ tiles
//
// 256 channels x 64, 128 or 256 tokens per workgroup.  Whole lines of 128 columns come straight from memory into one of two or three
// LDS buffers, and from there, 64 columns at a time, into registers while the 64 columns before them are multiplied; so the matrix
// instructions wait for neither, but for one barrier every second step.  What a CU has on its way is counted in requests, so that half
// lines (64 columns to each of four buffers) bring half as much: with weights from memory 14 x 6240 x 4896, mean 148, took 202 us
// instead of 172, 32 x 4096 x 4096, mean 1013, 661 instead of 615.  A row's eight pieces of 16 bytes lie in LDS in the order of
// their number xor row % 8 xor row / 8 % 2, so that lanes that read together use all banks.
// 8192 x 8192 x 8192: 420 us, 2.6 POP/s (the library: 2.38).  Bound by the card's power: all-zero operands take
// three quarters of the time, and instructions of 32 x 32 x 32, as fast with zeros, are a tenth slower with values.
// Slower, too: wave tiles of 128 x 128 in 512 registers, two workgroups of four waves with 128 tokens each on a CU, workgroups that
// go on to their next tile (the registers for that spill).
constexpr uint32_t kTileChannels = 256, kTileCols = 64, kLineCols = 2 * kTileCols;

typedef __attribute__((address_space(3))) int8_t lds_byte;

// WC x WAVES / WC waves, each of CI * 16 channels x TJ * 16 tokens; `BUFFERS` of two steps each.
template <int WAVES, int WC, int CI, int TJ, int BUFFERS>
struct TileShape {
    static constexpr int kWT = WAVES / WC;
    static constexpr uint32_t kThreads = WAVES * 64, kTokens = kWT * TJ * 16;
    // loads of a lane for each buffer: a wave's load brings 8 rows
    static constexpr uint32_t kLoadsA = kTokens / (WAVES * 8), kLoadsB = kTileChannels / (WAVES * 8);
    static constexpr uint32_t kBytes = (kTokens + kTileChannels) * kLineCols;
    static_assert(WC * CI * 16 == (int)kTileChannels, "waves cover the channels");
};

// The columns shared out: workgroups of share `s` multiply columns s * share ... and leave sums of 32-bit integers,
// [shares][rows][pitch], which i8_join_kernel adds up and scales.
struct SharedColumns { int32_t *sums; uint32_t blocks, share, pitch; };

// Waits until all but the last `LOADS` of the wave's loads have arrived and its LDS reads are through, then for the other waves.
template <uint32_t LOADS>
__device__ __forceinline__ void step_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
}

template <class T, int WAVES, int WC, int CI, int TJ, int BUFFERS>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 || BUFFERS == 2 ? 2 : 1) void i8_tile_kernel(I8Args a, SharedColumns shared)
{
    // (T = int32_t: sums of one share of the columns, as they are)
    constexpr bool kShared = std::is_same<T, int32_t>::value;
    using Shape = TileShape<WAVES, WC, CI, TJ, BUFFERS>;
    constexpr uint32_t TOKENS = Shape::kTokens, LA = Shape::kLoadsA, LB = Shape::kLoadsB;
    // (arrays of their own: the compiler knows that loads into one are nothing to reads from another)
    static_assert(BUFFERS == 2 || BUFFERS == 3, "");
    __shared__ __attribute__((aligned(1024))) int8_t s_0[Shape::kBytes], s_1[Shape::kBytes], s_2[BUFFERS > 2 ? Shape::kBytes : 16];
    int8_t *const buffer[3] = {s_0, s_1, BUFFERS > 2 ? s_2 : s_0};
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), lane = threadIdx.x & 63;
    const uint32_t across = (a.channels + kTileChannels - 1) / kTileChannels;
    Tile t;
    const uint32_t part = kShared ? blockIdx.x / shared.blocks : 0;
    if constexpr (kShared) {
        a.a += part * shared.share;
        a.b += part * shared.share;
        a.columns = min(shared.share, a.columns - part * shared.share);
    }
    if (!find_tile<WAVES>(a, kShared ? blockIdx.x % shared.blocks : blockIdx.x, TOKENS, across, reinterpret_cast<TileSearch *>(s_0), &t)) return;
    __syncthreads();                                // (s_0 is filled from now on)
    const uint32_t n0 = t.column * kTileChannels;
    const uint32_t wc = wave % WC, wt = wave / WC;
    T *out = static_cast<T *>(a.out);
    v4i32 acc[CI][TJ];
#pragma unroll
    for (int i = 0; i < CI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = v4i32{0, 0, 0, 0};

    if (t.group < a.groups) {
        const uint32_t rows = t.end - t.begin, chans = min(kTileChannels, a.channels - n0);
        const uint32_t lda = (uint32_t)a.lda, ldb = (uint32_t)a.ldb;
        const uint32_t readable = (a.columns + 15) & ~15u;      // (rows lie at multiples of 16: the last piece is theirs to its end)
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.a + (int64_t)t.begin * a.lda), 0,
                                                          (int)((rows - 1) * lda + readable), 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.b + ((int64_t)t.group * a.channels + n0) * a.ldb), 0,
                                                          (int)((chans - 1) * ldb + readable), 0x00020000);
        // A wave's load brings eight rows, 128 columns of each: whole lines of memory.  Piece c of row r lies in place c ^ order(r).
        // What is not there, rows and pieces, has an offset out of the buffer's range and costs nothing.
        const auto order = [](uint32_t row) { return (row & 7) ^ (row >> 3 & 1); };
        constexpr uint32_t kNowhere = 1u << 31;
        const uint32_t piece = ((lane & 7) ^ order(wave * 8 + lane / 8)) * 16;
        uint32_t at_a[LA], at_b[LB];
#pragma unroll
        for (uint32_t i = 0; i < LA; ++i) {
            const uint32_t row = (i * WAVES + wave) * 8 + lane / 8;
            at_a[i] = row < rows ? row * lda + piece : kNowhere;
        }
#pragma unroll
        for (uint32_t i = 0; i < LB; ++i) {
            const uint32_t row = (i * WAVES + wave) * 8 + lane / 8;
            at_b[i] = row < chans ? row * ldb + piece : kNowhere;
        }
        const uint32_t steps = (a.columns + kTileCols - 1) / kTileCols;
        const auto fetch = [&](uint32_t line, int8_t *lds) {
            const uint32_t k0 = line * kLineCols, nowhere = k0 + piece < a.columns ? 0 : kNowhere;
#pragma unroll
            for (uint32_t i = 0; i < LA; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_byte *)(lds + (i * WAVES + wave) * 1024), 16, (int)(at_a[i] | nowhere), (int)k0, 0, 0);
#pragma unroll
            for (uint32_t i = 0; i < LB; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_byte *)(lds + TOKENS * kLineCols + (i * WAVES + wave) * 1024), 16, (int)(at_b[i] | nowhere), (int)k0, 0, 0);
        };
        // a lane's place in the first and the second 64 columns
        const uint32_t own = (lane & 15) * kLineCols;
        const uint32_t from[2] = {own + ((lane >> 4) ^ order(lane & 15)) * 16, own + ((4 + (lane >> 4)) ^ order(lane & 15)) * 16};
        const uint32_t from_a = wt * TJ * 16 * kLineCols, from_b = (TOKENS + wc * CI * 16) * kLineCols;
        const bool busy = wt * TJ * 16 < rows;          // (waves without tokens only fetch)
        struct Frags { v4i32 b[CI], a[TJ]; };
        const auto read = [&](const int8_t *lds, uint32_t half, Frags &f) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) f.a[j] = *reinterpret_cast<const v4i32 *>(lds + from[half] + from_a + j * 16 * kLineCols);
#pragma unroll
            for (int i = 0; i < CI; ++i) f.b[i] = *reinterpret_cast<const v4i32 *>(lds + from[half] + from_b + i * 16 * kLineCols);
        };
        const auto multiply = [&](const Frags &f) {
#pragma unroll
            for (int i = 0; i < CI; ++i)
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.b[i], f.a[j], acc[i][j], 0, 0, 0);
        };
        // Step s multiplies what step s - 1 has read and reads the columns of step s + 1.  Odd steps find the next buffer filled and
        // nobody reading their own one any more, and send for the columns that come into it next.
        Frags frags[2];
        const auto turn = [&](uint32_t s, int i) {          // (s a multiple of 2 BUFFERS)
            if (i % 2 == 0) return;
            step_barrier<(BUFFERS - 2) * (LA + LB)>();
            fetch((s + i) / 2 + BUFFERS, buffer[i / 2 % BUFFERS]);
        };
        // zeros for the tokens' columns behind the last one
        const uint32_t whole = a.columns / kTileCols;
        const auto clear_end = [&](int8_t *lds, uint32_t half) {
            step_barrier<0>();
            for (uint32_t i = threadIdx.x; i < TOKENS * 4; i += Shape::kThreads) {
                v4i32 *const at = reinterpret_cast<v4i32 *>(lds + i / 4 * kLineCols + ((half * 4 + (i & 3)) ^ order(i / 4 & 15)) * 16);
                const int n = (int)a.columns - (int)(whole * kTileCols + (i & 3) * 16);
                if (n < 16) *at = first_bytes(*at, n);
            }
            step_barrier<0>();
        };
#pragma unroll
        for (int i = 0; i < BUFFERS; ++i) fetch(i, buffer[i]);
        step_barrier<(BUFFERS - 1) * (LA + LB)>();
        if (whole == 0) clear_end(s_0, 0);
        read(s_0, 0, frags[0]);
        constexpr int ROUND = 2 * BUFFERS;
        uint32_t s = 0;
        for (; s + ROUND < whole; s += ROUND)
#pragma unroll
            for (int i = 0; i < ROUND; ++i) {
                turn(s, i);
                if (!busy) continue;
                read(buffer[(i + 1) / 2 % BUFFERS], (i + 1) % 2, frags[(i + 1) % 2]);
                multiply(frags[i % 2]);
#pragma unroll
                for (int k = 0; k < CI + TJ; ++k) { // a read behind every few multiplications: the first ones wait for nothing
                    __builtin_amdgcn_sched_group_barrier(0x008, CI * TJ / (CI + TJ), 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
        // up to ROUND + 1 steps are left, the last of them perhaps not whole
#pragma unroll
        for (int i = 0; i <= ROUND; ++i) {
            if (s + i >= steps) break;
            turn(s, i);
            if (s + i + 1 < steps) {
                if (s + i + 1 == whole) clear_end(buffer[(i + 1) / 2 % BUFFERS], (i + 1) % 2);
                read(buffer[(i + 1) / 2 % BUFFERS], (i + 1) % 2, frags[(i + 1) % 2]);
            }
            if (busy) multiply(frags[i % 2]);
        }
    }
    if constexpr (kShared) {
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int i = 0; i < CI; ++i) {
                const uint32_t row = t.begin + (wt * TJ + j) * 16 + (lane & 15), n = n0 + (wc * CI + i) * 16 + (lane >> 4) * 4;
                if (row < t.end && n < shared.pitch)
                    *reinterpret_cast<v4i32 *>(shared.sums + ((size_t)part * a.rows + row) * shared.pitch + n) = acc[i][j];
            }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // nothing is on its way to LDS when the workgroup ends
        return;
    } else {
        // every scale is fetched before the first store: a wait for a load is one for all stores before it, too
        const bool zero = t.group >= a.groups;
        const float *sb = a.b_scale + (int64_t)(zero ? 0 : t.group) * a.channels;
        const uint32_t n1 = n0 + wc * CI * 16 + (lane >> 4) * 4, row1 = t.begin + wt * TJ * 16 + (lane & 15);
        float of_row[TJ], of_channel[CI][4];
#pragma unroll
        for (int j = 0; j < TJ; ++j) of_row[j] = a.a_scale[min(row1 + j * 16, t.end - 1)];
#pragma unroll
        for (int i = 0; i < CI; ++i)
#pragma unroll
            for (int v = 0; v < 4; ++v) of_channel[i][v] = sb[min(n1 + i * 16 + v, a.channels - 1)];
        // A lane's results are four channels each of TJ * CI tokens.  They change places in LDS, in a region of the wave's own, so
        // that stores are of 16 bytes and lines are written whole (4096 x 4096 x 256, where the stores are most of the
        // time: 15.4 us, and 18.3 with 8-byte stores, 16 rows at a time).  A row's pieces lie in the order of their number xor the row.
        constexpr int CIP = CI * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : CI;      // channels go by up to 256 bytes of a row
        constexpr uint32_t PIECES = CIP * sizeof(T), ROW = PIECES * 16, E = Unit<T>::kElems;
        constexpr uint32_t kPer = (WAVES + BUFFERS - 1) / BUFFERS;      // waves to a buffer
        static_assert(kPer * TJ * 16 * ROW <= Shape::kBytes && CI % CIP == 0, "the waves' regions fit");
        step_barrier<0>();                              // nothing is on its way to LDS, and nobody reads the last columns any more
        const uint32_t turn = wave / kPer;
        int8_t *mine = (turn == 0 ? buffer[0] : turn == 1 ? buffer[1] : buffer[2]) + (wave % kPer) * (TJ * 16 * ROW);
#pragma unroll
        for (int first = 0; first < CI; first += CIP) {
#pragma unroll
            for (int j = 0; j < TJ; ++j)
#pragma unroll
                for (int i = 0; i < CIP; ++i) {
                    typedef T four __attribute__((ext_vector_type(4)));
                    four v;
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = zero ? (T)0.0f : (T)((float)acc[first + i][j][u] * (of_row[j] * of_channel[first + i][u]));
                    const uint32_t row = j * 16 + (lane & 15), at = (i * 16 + (lane >> 4) * 4) * (uint32_t)sizeof(T);
                    *reinterpret_cast<four *>(mine + row * ROW + ((at / 16) ^ (row % PIECES)) * 16 + at % 16) = v;
                }
            __builtin_amdgcn_wave_barrier();            // (a wave's LDS accesses are served in order)
#pragma unroll
            for (uint32_t part = 0; part < TJ * 16 * PIECES / 64; ++part) {
                const uint32_t row = part * (64 / PIECES) + lane / PIECES, piece16 = lane % PIECES;
                const uint32_t to = t.begin + wt * TJ * 16 + row, n = n0 + (wc * CI + first) * 16 + piece16 * E;
                if (to < t.end && n < a.channels) {
                    Unit<T> u;
                    u.v = *reinterpret_cast<const typename Unit<T>::whole *>(mine + row * ROW + (piece16 ^ (row % PIECES)) * 16);
                    store_some(out + (int64_t)to * a.ldo + n, u, (int)min(E, a.channels - n));
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// The sums of all shares, scaled: four channels to a lane.
template <class T>
__global__ __launch_bounds__(kWG) void i8_join_kernel(I8Args a, SharedColumns shared, uint32_t shares)
{
    const uint32_t quads = shared.pitch / 4;
    for (uint64_t w = (uint64_t)blockIdx.x * kWG + threadIdx.x; w < (uint64_t)a.rows * quads; w += (uint64_t)gridDim.x * kWG) {
        const uint32_t row = (uint32_t)(w / quads), n = (uint32_t)(w % quads) * 4;
        v4i32 sum = {0, 0, 0, 0};
        for (uint32_t s = 0; s < shares; ++s)
            sum += *reinterpret_cast<const v4i32 *>(shared.sums + ((size_t)s * a.rows + row) * shared.pitch + n);
        const uint32_t g = group_of(a, row);
        const float sa = a.a_scale[row], *sb = a.b_scale + (int64_t)min(g, a.groups - 1) * a.channels;
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = g < a.groups ? (float)sum[u] * (sa * sb[min(n + u, a.channels - 1)]) : 0.0f;
        store_4(static_cast<T *>(a.out) + (int64_t)row * a.ldo, n, a.channels, v);
    }
}

// ------------------------------------------------------------------ few rows to a group
//
// CI * 16 channels of one group per workgroup, whose waves each take a share of the columns; both operands come straight from memory, the
// weights once per 64 rows, and the waves' sums meet in LDS.  Bound by the bytes of b: 8192 x 8192, one row, in 12.4 us
// (5.4 TB/s), 64 groups of 2048 x 4096 with four rows each on average in 84 (6.3 TB/s).  Plain loads: an instruction takes half
// of 16 lines, and with the streaming hint the other half comes from memory again (96 and 110 us).  Rows that do not lie at multiples of 16 bytes: 8192 x 8191, one row, 25 us (14 where they do).
constexpr uint32_t kFewRows = 64;

template <bool PIECES>
__device__ __forceinline__ v4i32 load_piece(const int8_t *p)
{
    if constexpr (PIECES) return *reinterpret_cast<const v4i32 *>(p);
    else return load_16(p, 16);
}

// 16 TJ rows from `at` on: the calling wave's columns [k_begin, k_end), U pieces of each row at a time.  PIECES: rows lie at multiples
// of 16 bytes, and their last piece is read whole.
template <bool PIECES, int CI, int TJ, int U>
__device__ __forceinline__ void few_sums(const int8_t *const (&pb)[CI], const int8_t *const (&pa)[TJ], uint32_t k_begin, uint32_t k_end, uint32_t q,
                                         v4i32 (&acc)[CI][TJ])
{
#pragma unroll
    for (int i = 0; i < CI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = v4i32{0, 0, 0, 0};
    uint32_t k = k_begin;
    for (; k + U * 64 <= k_end; k += U * 64) {
        v4i32 fb[U][CI], fa[U][TJ];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < CI; ++i) fb[u][i] = load_piece<PIECES>(pb[i] + k + u * 64);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < TJ; ++j) fa[u][j] = load_piece<PIECES>(pa[j] + k + u * 64);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < CI; ++i)
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][i], fa[u][j], acc[i][j], 0, 0, 0);
    }
    for (; k < k_end; k += 64) {
        const bool in = k + q < k_end;
        const int have = (int)k_end - (int)(k + q);     // columns of the piece (b's others meet zeros)
        const auto last = [&](const int8_t *p) { return PIECES ? *reinterpret_cast<const v4i32 *>(p) : load_16(p, have); };
        v4i32 fb[CI], fa[TJ];
#pragma unroll
        for (int i = 0; i < CI; ++i) fb[i] = in ? last(pb[i] + k) : v4i32{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < TJ; ++j) fa[j] = in ? first_bytes(last(pa[j] + k), have) : v4i32{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < CI; ++i)
#pragma unroll
            for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[i], fa[j], acc[i][j], 0, 0, 0);
    }
}

template <class T, int CI, int WAVES, bool PIECES>
__global__ __launch_bounds__(WAVES * 64) void i8_few_kernel(I8Args a, uint32_t share)
{
    __shared__ __attribute__((aligned(16))) v4i32 s_acc[2][WAVES][CI][64];
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), lane = threadIdx.x & 63;
    const uint32_t n0 = blockIdx.x * (CI * 16), g = blockIdx.y;
    const uint32_t begin = group_begin(a, g), end = group_begin(a, g + 1);
    T *out = static_cast<T *>(a.out);
    if (g == a.groups) {                            // the rows behind the groups
        constexpr uint32_t kChannels = CI * 16;
        const uint32_t n = n0 + threadIdx.x % kChannels;
        for (uint32_t row = begin + threadIdx.x / kChannels; row < end; row += WAVES * 64 / kChannels)
            if (n < a.channels) out[(int64_t)row * a.ldo + n] = (T)0.0f;
        return;
    }
    const uint32_t k_begin = min(a.columns, wave * share), k_end = min(a.columns, k_begin + share);
    const uint32_t q = (lane >> 4) * 16;
    const int8_t *pb[CI];
#pragma unroll
    for (int i = 0; i < CI; ++i) pb[i] = a.b + ((int64_t)g * a.channels + min(n0 + i * 16 + (lane & 15), a.channels - 1)) * a.ldb + q;
    const float *sb = a.b_scale + (int64_t)g * a.channels;

    const auto rows = [&](uint32_t at, auto count, auto pieces) {
        constexpr int TJ = decltype(count)::value;
        const int8_t *pa[TJ];
#pragma unroll
        for (int j = 0; j < TJ; ++j) pa[j] = a.a + (int64_t)min(at + j * 16 + (lane & 15), end - 1) * a.lda + q;
        v4i32 acc[CI][TJ];
        few_sums<PIECES, CI, TJ, decltype(pieces)::value>(pb, pa, k_begin, k_end, q, acc);
        // 16 rows at a time the waves' sums meet; wave i adds up and stores channels i * 16 ...
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
#pragma unroll
            for (int i = 0; i < CI; ++i) s_acc[j & 1][wave][i][lane] = acc[i][j];
            __syncthreads();
            if (wave < CI) {
                v4i32 sum = s_acc[j & 1][0][wave][lane];
#pragma unroll
                for (int o = 1; o < WAVES; ++o) sum += s_acc[j & 1][o][wave][lane];
                const uint32_t row = at + j * 16 + (lane & 15), n = n0 + wave * 16 + (lane >> 4) * 4;
                if (row < end && n < a.channels) {
                    const float sa = a.a_scale[row];
                    float v[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[u] = (float)sum[u] * (sa * sb[min(n + u, a.channels - 1)]);
                    store_4(out + (int64_t)row * a.ldo, n, a.channels, v);
                }
            }
        }
        __syncthreads();
    };
    using std::integral_constant;
    for (uint32_t at = begin; at < end; at += kFewRows) {
        const uint32_t left = end - at;
        if (left <= 16) rows(at, integral_constant<int, 1>{}, integral_constant<int, 8>{});
        else if (left <= 32) rows(at, integral_constant<int, 2>{}, integral_constant<int, 4>{});
        else rows(at, integral_constant<int, 4>{}, integral_constant<int, 4>{});
    }
}

// ------------------------------------------------------------------ launches

// Rows at multiples of 16 bytes: what the kernels for tiles and for few rows load in pieces of 16.  The last piece of a row may
// end before its 16 bytes do; it is loaded whole all the same (an aligned piece of which a byte is there is in memory), and what
// lies behind the last column of a is taken as zero.
static bool in_pieces(const I8Args &a)
{
    const auto whole = [](uintptr_t v) { return v % 16 == 0; };
    return whole(reinterpret_cast<uintptr_t>(a.a)) && whole(reinterpret_cast<uintptr_t>(a.b)) && whole((uintptr_t)a.lda) &&
           whole((uintptr_t)a.ldb);
}

constexpr uint32_t kCUs = 256;

// Workgroups for the tiles that there may be.
static uint64_t most_blocks(const I8Args &a, uint32_t tokens, uint32_t channels)
{
    return (most_tiles(a, tokens) * ((a.channels + channels - 1) / channels) + kXCD - 1) / kXCD * kXCD;
}

// The arithmetic on tiles is 32-bit; of the tiles for any address, which no other kernel's launches outnumber (i8_plan), there are the most.
bool i8_product_fits(const I8Args &a) { return a.groups <= SEER_MAX_EXPERTS && most_blocks(a, kAnyTokens, kAnyChannels) < (1u << 30); }

template <class T, int WAVES, int WC, int CI, int TJ, int BUFFERS>
static void launch_tiles(const I8Args &a, hipStream_t st)
{
    using Shape = TileShape<WAVES, WC, CI, TJ, BUFFERS>;
    const uint32_t blocks = (uint32_t)most_blocks(a, Shape::kTokens, kTileChannels);
    hipLaunchKernelGGL((i8_tile_kernel<T, WAVES, WC, CI, TJ, BUFFERS>), dim3(blocks), dim3(Shape::kThreads), 0, st, a, SharedColumns{});
}

// Tiles of 64 tokens have two buffers, which leaves room for two workgroups on a CU (32 x 4096 x 4096, mean 1013: 785 us; three, and one
// workgroup: 894), or, where there is only one, three (8192 x 8192, 384 rows: 41 us; two: 52; up to 2048 columns two are 0 to 5 % faster).
static bool three_buffers(const I8Args &a, uint64_t blocks) { return blocks <= kCUs && a.columns > 2048; }

template <class T>
static void launch_tiles_64(const I8Args &a, hipStream_t st)
{
    if (three_buffers(a, most_blocks(a, 64, kTileChannels))) launch_tiles<T, 4, 4, 4, 4, 3>(a, st);
    else launch_tiles<T, 4, 4, 4, 4, 2>(a, st);
}

static_assert(SEER_MAX_EXPERTS < 65535, "groups are a dimension of the grid of the kernel for few rows");
template <class T, int CI, int WAVES, bool PIECES>
static void launch_few(const I8Args &a, hipStream_t st)
{
    const uint32_t groups = a.groups + (a.group_ptr ? 1 : 0), share = ((a.columns + WAVES - 1) / WAVES + 63) & ~63u;
    const uint32_t across = (a.channels + CI * 16 - 1) / (CI * 16);
    hipLaunchKernelGGL((i8_few_kernel<T, CI, WAVES, PIECES>), dim3(across, groups), dim3(WAVES * 64), 0, st, a, share);
}

// Which kernel, and for how many shares of the columns: the one whose time by the following lines is the least.  They are fitted to 256
// draws (one matrix, or 3 to 64 with rows to a group 1, 1 / sqrt(rank) or 1 / rank; 4 to 6000 rows to a group; 128 to 16 384 channels; 256 to
// 11 000 columns; weights from memory, not from a cache), of which each kernel was timed.  Of 256 other draws, whose times are
// kept in profiles/i8_kernel_times.csv, what is chosen takes 3 % longer than the best one on average, 1.6 times at most.
//
// Few rows: a workgroup reads its group's rows and its channels at some 24 GB/s, and so does a CU that has several.  Where lengths
// differ, a group may be four times as long as the mean.  (1 x 2960 x 1424, 88 rows: few rows 9.5 us, tiles 16;
// 9 x 1576 x 3856, mean 34: 27 and 44; 41 x 784 x 3520, mean 63: 72 and 47; 49 x 144 x 672, mean 126, longest 1356: 102 and 11.)
// 16 channels to a workgroup where 32 are fewer than half of the CUs (2048 x 2048, one row: 3.8 and 4.7); eight waves to share the columns
// where each has 512 or more and there is more than one row (8192 x 8192, 64 rows: 25.6 and 27.8; one row: 14.0 and 13.1;
// 2048 columns, 64 groups of 8: 29 and 26).
static uint32_t few_channels(const I8Args &a) { return (uint64_t)((a.channels + 31) / 32) * a.groups < 128 ? 16 : 32; }

struct FewCost { double start, batch, each /* 64 rows of a workgroup, where a CU has several */, rate /* thousand bytes a us */, read /* million */; };
constexpr FewCost kFewPieces = {4, 1.2, 0, 24, 5.8}, kFewWords = {3.5, 1.6, 1.2, 16, 2.1};

static double few_cost(const I8Args &a, const FewCost &c)
{
    const double mean = a.rows / a.groups, channels = few_channels(a);
    const double workgroups = (double)((a.channels + few_channels(a) - 1) / few_channels(a)) * a.groups;
    const double rows = std::max((mean + channels) * workgroups / kCUs, (a.group_ptr ? 4 : 1) * mean + channels);
    const double batches = a.rows / a.groups / kFewRows;        // (behind the first)
    return std::max(c.start + c.batch * batches + c.each * (batches + 1) * workgroups / kCUs + rows * a.columns / (1e3 * c.rate), (double)a.groups * a.channels * a.columns / (1e6 * c.read));
}

// Tiles: rounds of as many as there is room for, `round` each and `least` to `least + more` for a step of 64 columns by how many are at
// work.  Measured (1 x 8192 channels, 16 | 64 | 128 steps): tiles of 64 tokens
// 128: 10 | 24 | 39, 256: 11 | 26 | 44, 384: 15 | 36 | 64, 512: 17 | 41 | 74, 768: 24 | 65 | 122, 1024: 30 | 80 | 144; of 128 tokens
// 64: 13 | 30 | 52, 192: 15 | 34 | 62, 256: 16 | 40 | 67, 384: 26 | 67 | 119, 1024: 57 | 147 | 261; of 256 tokens 32: 18 | 45 | 81,
// 128: 21 | 48 | 85, 192: 22 | 52 | 96, 256: 24 | 59 | 107, 416: 40 | 104 | 192, 1024: 89 | 235 | 422.
// Weights that come from memory cost the smaller tiles more (`cold`), and several groups, which end in the middle of a tile each and
// share theirs between fewer, a quarter more again.
struct TileCost { uint32_t tokens, room; double least, more, above /* share of the room */, round, cold; };
constexpr TileCost kCost64 = {64, 2 * kCUs, 0.12, 0.42, 0, 5.5, 1.25}, kCost64Alone = {64, kCUs, 0.26, 0.04, 0, 6, 1.25},
                   kCost128 = {128, kCUs, 0.34, 0.115, 0.3, 8, 1.05}, kCost256 = {256, kCUs, 0.565, 0.195, 0.5, 10, 1};

static double tile_cost(const I8Args &a, const TileCost &c, uint32_t shares)
{
    const uint64_t down = a.group_ptr ? (uint64_t)a.rows / c.tokens + (a.groups + 1) / 2 : ((uint64_t)a.rows + c.tokens - 1) / c.tokens;
    const uint64_t tiles = down * ((a.channels + kTileChannels - 1) / kTileChannels) * shares;
    if (c.room > kCUs && tiles <= kCUs) return tile_cost(a, kCost64Alone, shares);
    const double steps = ((double)a.columns / kTileCols) / shares;
    const auto round = [&](double full) {
        return steps * (c.least + c.more * std::max(0.0, (full - c.above) / (1 - c.above))) + c.round;
    };
    const uint64_t rest = tiles % c.room;
    const double t = (double)(tiles / c.room) * round(1) + (rest ? round((double)rest / c.room) : 0);
    return std::max(t * c.cold * (a.group_ptr ? 1.25 : 1), (double)a.groups * a.channels * a.columns / 4.2e6);
}

// Tiles of 64 tokens that leave CUs idle may have the columns shared out, at 1 us for every 3 MB of sums written and read and 8 us for the
// second launch.  Measured, us, one and several shares (channels x columns, rows 128, 256, 512, 1024):
//   512 x 8192:  34 34 34 36 and 15 17 18 20      2048 x 8192: 34 35 45 46 and 19 20 24 33
//   8192 x 8192: 46 46 55 74 and 24 33 43 64      2048 x 2048: 12.5 12.7 13 14 and 13 16 25 27 (hence one)
// and of groups (mean 66, 100, 160, 256): 10 x 256 x 6656: 37 39 41 41 and 17 18 20 21, 32 x 256 x 4096: 26 28 29 30 and 20 22 24 25.
struct Choice { uint32_t tokens /* 0: few rows */, shares /* 0: tiles for any address */; };

static Choice choose(const I8Args &a)
{
    Choice best{0, 1};
    double least = few_cost(a, kFewPieces);
    const auto consider = [&](uint32_t tokens, uint32_t shares, double cost) {
        if (cost >= least) return;
        least = cost;
        best = Choice{tokens, shares};
    };
    consider(256, 1, tile_cost(a, kCost256, 1));
    consider(128, 1, tile_cost(a, kCost128, 1));
    consider(64, 1, tile_cost(a, kCost64, 1));
    const uint64_t tiles = most_blocks(a, 64, kTileChannels);
    if (tiles > kCUs * 2 / 3) return best;
    const uint32_t most = (uint32_t)std::min<uint64_t>({kCUs * 2 / tiles, (uint64_t)a.columns / kTileCols / 6, 16});
    for (uint32_t n = 2; n <= most; ++n) consider(64, n, tile_cost(a, kCost64, n) + n * (8.0 * a.rows * a.channels) / 3e6 + 8);
    return best;
}

// Rows off multiples of 16 bytes: few rows, in realigned words, or the tiles for any address, two workgroups of which are on a CU.  Fitted
// to 373 draws like those above with rows at odd addresses, both kernels timed (the same file): what is chosen takes 1.4 % longer than the better
// one on average, 1.6 times at most.  Measured, us, any and few: 97 x 16 x 3089 40 and 23, 100 x 512 x 8190 105 and 62, 47 x 656 x 8946 140 and 36;
// 500 x 130 x 4111 57 and 113, 3001 x 5001 x 4111 152 and 875, 17 x 186 x 2278, mean 85, longest 682 9.9 and 28, 39 x 2168 x 123,
// mean 165, 33 and 89.
static bool few_words(const I8Args &a)
{
    const double steps = (a.columns + kAnyCols - 1) / kAnyCols;
    const uint64_t across = (a.channels + kAnyChannels - 1) / kAnyChannels,
                   down = a.group_ptr ? (uint64_t)a.rows / kAnyTokens + (a.groups + 1) / 2 : ((uint64_t)a.rows + kAnyTokens - 1) / kAnyTokens;
    const uint64_t room = 2 * kCUs, rest = down * across % room;
    const auto round = [&](double full) { return 6.6 + steps * (1.6 + 1.36 * full); };
    const double any = (double)(down * across / room) * round(1) + (rest ? round((double)rest / room) : 0);
    return few_cost(a, kFewWords) < std::max(any, (double)a.groups * a.channels * a.columns / 2.6e6);
}

static SharedColumns shared_columns(const I8Args &a, uint32_t shares, void *workspace)
{
    const uint32_t steps = (a.columns + kTileCols - 1) / kTileCols;
    return SharedColumns{static_cast<int32_t *>(workspace), (uint32_t)most_blocks(a, 64, kTileChannels), ((steps + 1) / 2 + shares - 1) / shares * kLineCols,
                         (a.channels + 3) & ~3u};
}

size_t i8_workspace_bytes(uint32_t rows, uint32_t channels, uint32_t columns, uint32_t groups)
{
    I8Args a{};
    a.rows = rows;
    a.channels = channels;
    a.columns = columns;
    a.groups = groups;
    if (rows == 0 || channels == 0) return 0;
    static const int32_t some = 0;                  // one group may come with its group_ptr or without
    uint32_t shares = groups == 1 ? choose(a).shares : 1;
    a.group_ptr = &some;
    shares = std::max(shares, choose(a).shares);
    return shares > 1 ? (size_t)shares * rows * ((channels + 3) & ~3u) * 4 : 0;
}

template <class T>
static void launch_shared(const I8Args &a, uint32_t shares, void *workspace, hipStream_t st)
{
    const SharedColumns c = shared_columns(a, shares, workspace);
    shares = (a.columns + c.share - 1) / c.share;
    if (three_buffers(a, (uint64_t)c.blocks * shares))
        hipLaunchKernelGGL((i8_tile_kernel<int32_t, 4, 4, 4, 4, 3>), dim3(c.blocks * shares), dim3(256), 0, st, a, c);
    else
        hipLaunchKernelGGL((i8_tile_kernel<int32_t, 4, 4, 4, 4, 2>), dim3(c.blocks * shares), dim3(256), 0, st, a, c);
    const uint64_t lanes = (uint64_t)a.rows * (c.pitch / 4);
    hipLaunchKernelGGL((i8_join_kernel<T>), dim3((uint32_t)std::min<uint64_t>((lanes + kWG - 1) / kWG, 8 * kCUs)), dim3(kWG), 0, st, a, c, shares);
}

static bool few_in_eights(const I8Args &a) { return few_channels(a) == 32 && a.rows / a.groups > 1 && a.columns >= 4096; }

template <class T, bool PIECES>
static void launch_few_rows(const I8Args &a, hipStream_t st)
{
    if (few_channels(a) == 16) launch_few<T, 1, 4, PIECES>(a, st);
    else if (few_in_eights(a)) launch_few<T, 2, 8, PIECES>(a, st);
    else launch_few<T, 2, 4, PIECES>(a, st);
}

// The kernel for a product: what takes least, where the operands and a launch (fewer than 2^32 lanes) allow it.
I8Plan i8_plan(const I8Args &a)
{
    const I8Plan any{SEER_I8_ANY, 0, 1};
    if (a.columns == 0) return any;
    // (rows further apart than that: offsets into a tile are 32-bit)
    const Choice c = in_pieces(a) && a.lda < (1 << 23) && a.ldb < (1 << 23) ? choose(a) : Choice{few_words(a) ? 0u : kAnyTokens, 0};
    if (c.tokens == 0) {
        const uint64_t across = (a.channels + few_channels(a) - 1) / few_channels(a);
        return across * (few_in_eights(a) ? 512 : 256) < 1ull << 32 ? I8Plan{SEER_I8_FEW, 0, 1} : any;
    }
    if (c.shares == 0) return any;
    if (c.shares > 1) return I8Plan{SEER_I8_SHARED, c.tokens, c.shares};
    const uint64_t lanes = most_blocks(a, c.tokens, kTileChannels) * (c.tokens == 64 ? 256 : 512);
    return lanes < 1ull << 32 ? I8Plan{SEER_I8_TILES, c.tokens, 1} : any;
}

template <class T>
static void launch_product(const I8Args &a, const I8Plan &p, void *workspace, hipStream_t st)
{
    switch (p.kernel) {
    case SEER_I8_FEW:
        if (in_pieces(a)) launch_few_rows<T, true>(a, st);
        else launch_few_rows<T, false>(a, st);
        return;
    case SEER_I8_TILES:
        if (p.tokens == 256) launch_tiles<T, 8, 2, 8, 4, 2>(a, st);
        else if (p.tokens == 128) launch_tiles<T, 8, 2, 8, 2, 3>(a, st);
        else launch_tiles_64<T>(a, st);
        return;
    case SEER_I8_SHARED:
        launch_shared<T>(a, p.shares, workspace, st);
        return;
    default:
        const uint32_t blocks = (uint32_t)most_blocks(a, kAnyTokens, kAnyChannels);
        hipLaunchKernelGGL((i8_any_kernel<T>), dim3(std::min(blocks, 1u << 22)), dim3(256), 0, st, a, blocks);
    }
}

void launch_i8_product(const I8Args &a, const I8Plan &p, void *workspace, hipStream_t st)
{
    if (a.type == SEER_F32) launch_product<float>(a, p, workspace, st);
    else if (a.type == SEER_BF16) launch_product<bf16_t>(a, p, workspace, st);
    else launch_product<f16_t>(a, p, workspace, st);
}

} // namespace seer
