// Products of 8-bit integers with a scale for each token and channel, over ragged groups of rows:
//   out[i][n] = a_scale[i] * b_scale[g][n] * sum_k a[i][k] * b[g][n][k],  group_ptr[g] <= i < group_ptr[g + 1].
// The sums are 32-bit integers, exact whatever the order; one rounding to fp32 follows, two products there and
// the rounding to the type of the output.  The matrix instructions take channels for their rows and tokens for their
// columns, so that a lane's results are consecutive channels of one token.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

typedef int v4i32 __attribute__((ext_vector_type(4)));

// The rows of tile `tile` of `tokens` rows: those of group g from `begin` to `end`.  Group number `groups` stands for
// the rows behind the last one.  All lanes of a wave take part.
struct TileRows { uint32_t group, begin, end; };

__device__ __forceinline__ uint32_t group_begin(const I8Args &a, uint32_t g)
{
    if (g > a.groups) return a.rows;
    if (!a.group_ptr) return g ? a.rows : 0;
    const int32_t p = a.group_ptr[g];
    return p < 0 ? 0 : min((uint32_t)p, a.rows);
}

__device__ __forceinline__ bool find_tile(const I8Args &a, uint32_t tile, uint32_t tokens, TileRows *t)
{
    if (!a.group_ptr) {
        t->group = 0;
        t->begin = tile * tokens;
        t->end = min(a.rows, t->begin + tokens);
        return t->begin < a.rows;
    }
    const uint32_t lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (uint32_t at = 0; at <= a.groups; at += 64) {
        const uint32_t g = at + lane;
        const uint32_t from = group_begin(a, min(g, a.groups + 1)), to = group_begin(a, min(g + 1, a.groups + 1));
        const uint32_t tiles = to > from ? (to - from + tokens - 1) / tokens : 0;
        uint32_t sum = tiles;
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = __shfl_up(sum, d, 64);
            if ((int)lane >= d) sum += other;
        }
        const uint64_t past = __ballot(before + sum > tile);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            const uint32_t first = before + (uint32_t)__builtin_amdgcn_readlane((int)(sum - tiles), l);
            t->group = at + (uint32_t)l;
            t->begin = (uint32_t)__builtin_amdgcn_readlane((int)from, l) + (tile - first) * tokens;
            t->end = min((uint32_t)__builtin_amdgcn_readlane((int)to, l), t->begin + tokens);
            return true;
        }
        before += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    }
    return false;
}

// Tiles of `tokens` rows that any division of the rows into groups needs.
static uint32_t most_tiles(const I8Args &a, uint32_t tokens)
{
    return a.group_ptr ? a.rows / tokens + std::min(a.groups + 1, a.rows) : (a.rows + tokens - 1) / tokens;
}

__device__ __forceinline__ void store_1(const I8Args &a, uint32_t row, uint32_t channel, float v)
{
    const int64_t at = (int64_t)row * a.ldo + channel;
    if (a.type == SEER_F32) static_cast<float *>(a.out)[at] = v;
    else if (a.type == SEER_BF16) static_cast<bf16_t *>(a.out)[at] = (bf16_t)v;
    else static_cast<f16_t *>(a.out)[at] = (f16_t)v;
}

// ------------------------------------------------------------------ any size, any alignment
//
// 64 tokens x 64 channels, 128 columns at a time through LDS, four waves of 32 x 32 each.  16 bytes of
// a row at a time, from any address; the end of a row byte by byte, and zeros behind it.
constexpr uint32_t kAnyTokens = 64, kAnyChannels = 64, kAnyCols = 128, kAnyPitch = kAnyCols + 16;

__device__ __forceinline__ v4i32 load_16(const int8_t *p, int n)
{
    if (n >= 16) {
        typedef int v4i_a1 __attribute__((ext_vector_type(4), aligned(1)));
        return *reinterpret_cast<const v4i_a1 *>(p);
    }
    v4i32 v = {0, 0, 0, 0};
    for (int j = 0; j < 16; ++j)
        if (j < n) v[j / 4] |= (int)(uint8_t)p[j] << (j % 4 * 8);
    return v;
}

__global__ __launch_bounds__(256) void i8_any_kernel(I8Args a, uint32_t tiles)
{
    __shared__ __attribute__((aligned(16))) int8_t s_a[kAnyTokens * kAnyPitch], s_b[kAnyChannels * kAnyPitch];
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const uint32_t across = (a.channels + kAnyChannels - 1) / kAnyChannels;
    for (uint64_t w = blockIdx.x; w < (uint64_t)across * tiles; w += gridDim.x) {
    TileRows t;
    if (!find_tile(a, (uint32_t)(w / across), kAnyTokens, &t)) return;
    const uint32_t n0 = (uint32_t)(w % across) * kAnyChannels;
    v4i32 acc[2][2] = {};
    if (t.group < a.groups) {
        const int8_t *b = a.b + (int64_t)t.group * a.channels * a.ldb;
        for (uint32_t k0 = 0; k0 < a.columns; k0 += kAnyCols) {
            for (uint32_t i = threadIdx.x; i < kAnyTokens * (kAnyCols / 16); i += 256) {
                const uint32_t row = i / (kAnyCols / 16), col = k0 + i % (kAnyCols / 16) * 16;
                const int left = (int)a.columns - (int)col;
                const v4i32 va = t.begin + row < t.end ? load_16(a.a + (int64_t)(t.begin + row) * a.lda + col, left) : v4i32{0, 0, 0, 0};
                *reinterpret_cast<v4i32 *>(s_a + row * kAnyPitch + (col - k0)) = va;
                const v4i32 vb = n0 + row < a.channels ? load_16(b + (int64_t)(n0 + row) * a.ldb + col, left) : v4i32{0, 0, 0, 0};
                *reinterpret_cast<v4i32 *>(s_b + row * kAnyPitch + (col - k0)) = vb;
            }
            __syncthreads();
            for (uint32_t k = 0; k < kAnyCols; k += 64) {
                v4i32 fb[2], fa[2];
                for (int i = 0; i < 2; ++i) {
                    fb[i] = *reinterpret_cast<const v4i32 *>(s_b + ((wave & 1) * 32 + i * 16 + (lane & 15)) * kAnyPitch + k + lane / 16 * 16);
                    fa[i] = *reinterpret_cast<const v4i32 *>(s_a + ((wave >> 1) * 32 + i * 16 + (lane & 15)) * kAnyPitch + k + lane / 16 * 16);
                }
                for (int i = 0; i < 2; ++i)
                    for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[i], fa[j], acc[i][j], 0, 0, 0);
            }
            __syncthreads();
        }
    }
    for (int j = 0; j < 2; ++j) {
        const uint32_t row = t.begin + (wave >> 1) * 32 + j * 16 + (lane & 15);
        if (row >= t.end) continue;
        const float sa = t.group < a.groups ? a.a_scale[row] : 0.0f;
        for (int i = 0; i < 2; ++i)
            for (int v = 0; v < 4; ++v) {
                const uint32_t n = n0 + (wave & 1) * 32 + i * 16 + lane / 16 * 4 + v;
                if (n >= a.channels) continue;
                const float sb = t.group < a.groups ? a.b_scale[(int64_t)t.group * a.channels + n] : 0.0f;
                store_1(a, row, n, t.group < a.groups ? (float)acc[i][j][v] * (sa * sb) : 0.0f);
            }
    }
    }
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

// ------------------------------------------------------------------ tiles
//
// kTileChannels channels x TOKENS tokens per workgroup of eight waves, 128 columns at a time, straight from memory into one of
// two LDS buffers while the other is multiplied.  A row's eight pieces of 16 bytes lie in the order of their number
// xor the row's last three bits, so that the eight lanes that read at a time use all banks.
constexpr uint32_t kTileChannels = 256, kTileCols = 128, kTileThreads = 512;

typedef __attribute__((address_space(3))) int8_t lds_byte;

// TOKENS x CHANNELS: WC x WT waves of CI * 16 channels x TJ * 16 tokens.
template <int WC, int CI, int TJ>
struct TileShape {
    static constexpr int kWT = 8 / WC;
    static constexpr uint32_t kTokens = kWT * TJ * 16;
    static_assert(WC * CI * 16 == (int)kTileChannels, "waves cover the channels");
};

// ROWS rows of kTileCols columns to LDS: at[i] is where the calling lane's piece of rows i * 64 + wave * 8 ... lies, `col` is uniform.
template <uint32_t ROWS>
__device__ __forceinline__ void fetch_tile(__amdgpu_buffer_rsrc_t rows, const uint32_t (&at)[ROWS / 64], uint32_t back, uint32_t col,
                                           uint32_t wave, int8_t *lds)
{
#pragma unroll
    for (uint32_t i = 0; i < ROWS / 64; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_byte *)(lds + (i * 8 + wave) * 1024), 16, (int)(at[i] - back), (int)col, 0, 0);
}

template <class T, int WC, int CI, int TJ>
__global__ __launch_bounds__(kTileThreads, 2) void i8_tile_kernel(I8Args a, uint32_t tiles)
{
    using Shape = TileShape<WC, CI, TJ>;
    constexpr uint32_t TOKENS = Shape::kTokens;
    __shared__ __attribute__((aligned(1024))) int8_t s_a0[TOKENS * kTileCols], s_b0[kTileChannels * kTileCols];
    __shared__ __attribute__((aligned(1024))) int8_t s_a1[TOKENS * kTileCols], s_b1[kTileChannels * kTileCols];
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), lane = threadIdx.x & 63;
    const uint32_t across = (a.channels + kTileChannels - 1) / kTileChannels;
    const uint32_t w = tile_of_block(blockIdx.x, across * tiles, 1);
    if (w >= across * tiles) return;
    TileRows t;
    if (!find_tile(a, w / across, TOKENS, &t)) return;
    const uint32_t n0 = (w % across) * kTileChannels;
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
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.a + (int64_t)t.begin * a.lda), 0,
                                                          (int)((rows - 1) * lda + a.columns), 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(a.b + ((int64_t)t.group * a.channels + n0) * a.ldb), 0,
                                                          (int)((chans - 1) * ldb + a.columns), 0x00020000);
        // a wave's load brings eight rows, eight pieces each; rows that are not there are taken as the last one
        const uint32_t piece = ((lane & 7) ^ (lane >> 3)) * 16;
        uint32_t at_a[TOKENS / 64], at_b[kTileChannels / 64];
#pragma unroll
        for (uint32_t i = 0; i < TOKENS / 64; ++i) at_a[i] = min((i * 8 + wave) * 8 + lane / 8, rows - 1) * lda + piece;
#pragma unroll
        for (uint32_t i = 0; i < kTileChannels / 64; ++i) at_b[i] = min((i * 8 + wave) * 8 + lane / 8, chans - 1) * ldb + piece;
        const auto fetch = [&](uint32_t k0, int8_t *la, int8_t *lb) {
            // pieces behind the last column are not loaded: the first one of the 128 columns is
            const uint32_t back = k0 + piece < a.columns ? 0 : piece;
            fetch_tile<TOKENS>(ra, at_a, back, k0, wave, la);
            fetch_tile<kTileChannels>(rb, at_b, back, k0, wave, lb);
        };
        const uint32_t from = (lane & 15) * kTileCols + (((lane >> 4) ^ (lane & 7)) * 16);
        const uint32_t from_b = wc * CI * 16 * kTileCols + from, from_a = wt * TJ * 16 * kTileCols + from;
        const auto multiply = [&](const int8_t *la, const int8_t *lb) {
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) {
                const int8_t *pa = la + (from_a ^ (h * 64)), *pb = lb + (from_b ^ (h * 64));
                v4i32 fb[CI], fa[TJ];
#pragma unroll
                for (int j = 0; j < TJ; ++j) fa[j] = *reinterpret_cast<const v4i32 *>(pa + j * 16 * kTileCols);
#pragma unroll
                for (int i = 0; i < CI; ++i) fb[i] = *reinterpret_cast<const v4i32 *>(pb + i * 16 * kTileCols);
#pragma unroll
                for (int i = 0; i < CI; ++i)
#pragma unroll
                    for (int j = 0; j < TJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[i], fa[j], acc[i][j], 0, 0, 0);
            }
        };
        // zeros for the tokens' pieces behind the last column
        const auto clear_end = [&](uint32_t k0, int8_t *la) {
            for (uint32_t i = threadIdx.x; i < TOKENS * 8; i += kTileThreads)
                if (k0 + ((i ^ (i >> 3)) & 7) * 16 >= a.columns) *reinterpret_cast<v4i32 *>(la + i * 16) = v4i32{0, 0, 0, 0};
            __syncthreads();
        };
        fetch(0, s_a0, s_b0);
        uint32_t k0 = 0;
        for (; k0 + 2 * kTileCols <= a.columns; k0 += 2 * kTileCols) {
            __syncthreads();                         // the first buffer is there, the second no longer read
            fetch(k0 + kTileCols, s_a1, s_b1);
            multiply(s_a0, s_b0);
            __syncthreads();
            if (k0 + 2 * kTileCols < a.columns) fetch(k0 + 2 * kTileCols, s_a0, s_b0);
            multiply(s_a1, s_b1);
        }
        if (k0 < a.columns) {                        // up to 255 columns are left, the first 128 of them on their way
            const bool more = k0 + kTileCols < a.columns;
            __syncthreads();
            if (more) fetch(k0 + kTileCols, s_a1, s_b1);
            else clear_end(k0, s_a0);
            multiply(s_a0, s_b0);
            if (more) {
                __syncthreads();
                clear_end(k0 + kTileCols, s_a1);
                multiply(s_a1, s_b1);
            }
        }
    }
    const bool zero = t.group >= a.groups;
    const float *sb = a.b_scale + (int64_t)(zero ? 0 : t.group) * a.channels;
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const uint32_t n = n0 + (wc * CI + i) * 16 + (lane >> 4) * 4;
        if (n >= a.channels) continue;
        float scale[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) scale[v] = sb[min(n + v, a.channels - 1)];
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const uint32_t row = t.begin + (wt * TJ + j) * 16 + (lane & 15);
            if (row >= t.end) continue;
            const float sa = a.a_scale[row];
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = zero ? 0.0f : (float)acc[i][j][u] * (sa * scale[u]);
            store_4(out + (int64_t)row * a.ldo, n, a.channels, v);
        }
    }
}

// ------------------------------------------------------------------ few rows to a group
//
// 16 channels of one group per workgroup, whose waves each take a share of the columns; weights come straight from memory, once per 32
// rows, and the waves' sums meet in LDS.  Bound by the bytes of b.
constexpr uint32_t kFewWaves = 4, kFewUnroll = 8;

template <class T>
__global__ __launch_bounds__(kFewWaves * 64) void i8_few_kernel(I8Args a, uint32_t share)
{
    __shared__ __attribute__((aligned(16))) v4i32 s_acc[2][kFewWaves][64];
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), lane = threadIdx.x & 63;
    const uint32_t n0 = blockIdx.x * 16, g = blockIdx.y;
    const uint32_t begin = group_begin(a, g), end = group_begin(a, g + 1);
    T *out = static_cast<T *>(a.out);
    if (g == a.groups) {                            // the rows behind the groups
        for (uint32_t row = begin + threadIdx.x / 16; row < end; row += kFewWaves * 4)
            if (n0 + (threadIdx.x & 15) < a.channels) out[(int64_t)row * a.ldo + n0 + (threadIdx.x & 15)] = (T)0.0f;
        return;
    }
    const uint32_t k_begin = min(a.columns, wave * share), k_end = min(a.columns, k_begin + share);
    const uint32_t q = (lane >> 4) * 16;
    const int8_t *pb = a.b + ((int64_t)g * a.channels + min(n0 + (lane & 15), a.channels - 1)) * a.ldb + q;
    for (uint32_t at = begin; at < end; at += 32) {
        const bool two = end - at > 16;
        const int8_t *pa0 = a.a + (int64_t)min(at + (lane & 15), end - 1) * a.lda + q;
        const int8_t *pa1 = a.a + (int64_t)min(at + 16 + (lane & 15), end - 1) * a.lda + q;
        v4i32 acc0 = {0, 0, 0, 0}, acc1 = {0, 0, 0, 0};
        uint32_t k = k_begin;
        for (; k + kFewUnroll * 64 <= k_end; k += kFewUnroll * 64) {
            v4i32 fb[kFewUnroll], fa[kFewUnroll];
#pragma unroll
            for (uint32_t u = 0; u < kFewUnroll; ++u) fb[u] = __builtin_nontemporal_load(reinterpret_cast<const v4i32 *>(pb + k + u * 64));
#pragma unroll
            for (uint32_t u = 0; u < kFewUnroll; ++u) fa[u] = *reinterpret_cast<const v4i32 *>(pa0 + k + u * 64);
#pragma unroll
            for (uint32_t u = 0; u < kFewUnroll; ++u) acc0 = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u], fa[u], acc0, 0, 0, 0);
            if (two) {
#pragma unroll
                for (uint32_t u = 0; u < kFewUnroll; ++u) fa[u] = *reinterpret_cast<const v4i32 *>(pa1 + k + u * 64);
#pragma unroll
                for (uint32_t u = 0; u < kFewUnroll; ++u) acc1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u], fa[u], acc1, 0, 0, 0);
            }
        }
        for (; k < k_end; k += 64) {
            v4i32 fb = {0, 0, 0, 0}, f0 = fb, f1 = fb;
            if (k + q < k_end) {
                fb = *reinterpret_cast<const v4i32 *>(pb + k);
                f0 = *reinterpret_cast<const v4i32 *>(pa0 + k);
                f1 = *reinterpret_cast<const v4i32 *>(pa1 + k);
            }
            acc0 = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, f0, acc0, 0, 0, 0);
            acc1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb, f1, acc1, 0, 0, 0);
        }
        s_acc[0][wave][lane] = acc0;
        s_acc[1][wave][lane] = acc1;
        __syncthreads();
        if (wave < 2 && (wave == 0 || two)) {
            v4i32 sum = s_acc[wave][0][lane];
            for (uint32_t o = 1; o < kFewWaves; ++o) sum += s_acc[wave][o][lane];
            const uint32_t row = at + wave * 16 + (lane & 15), n = n0 + (lane >> 4) * 4;
            if (row < end && n < a.channels) {
                const float *sb = a.b_scale + (int64_t)g * a.channels;
                const float sa = a.a_scale[row];
                float v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = (float)sum[u] * (sa * sb[min(n + u, a.channels - 1)]);
                store_4(out + (int64_t)row * a.ldo, n, a.channels, v);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ launches

size_t i8_workspace_bytes(uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

// Whole pieces of 16 bytes at multiples of 16: what the kernels for tiles and for few rows load.
static bool in_pieces(const I8Args &a)
{
    const auto whole = [](uintptr_t v) { return v % 16 == 0; };
    return whole(reinterpret_cast<uintptr_t>(a.a)) && whole(reinterpret_cast<uintptr_t>(a.b)) && whole((uintptr_t)a.lda) &&
           whole((uintptr_t)a.ldb) && a.columns % 16 == 0 && a.columns > 0;
}

template <class T, int WC, int CI, int TJ>
static void launch_tiles(const I8Args &a, hipStream_t st)
{
    constexpr uint32_t tokens = TileShape<WC, CI, TJ>::kTokens;
    const uint32_t across = (a.channels + kTileChannels - 1) / kTileChannels, tiles = most_tiles(a, tokens);
    hipLaunchKernelGGL((i8_tile_kernel<T, WC, CI, TJ>), dim3(8 * tiles_per_xcd(across * tiles)), dim3(kTileThreads), 0, st, a, tiles);
}

template <class T>
static bool launch_pieces(const I8Args &a, hipStream_t st)
{
    const uint32_t mean = a.rows / a.groups;
    if (mean <= 32) {
        if (a.groups >= 65535) return false;
        const uint32_t share = ((a.columns + kFewWaves - 1) / kFewWaves + 63) & ~63u;
        hipLaunchKernelGGL((i8_few_kernel<T>), dim3((a.channels + 15) / 16, a.groups + (a.group_ptr ? 1 : 0)), dim3(kFewWaves * 64), 0, st, a, share);
        return true;
    }
    // (offsets into a tile are 32-bit, and so is the number of workgroups' lanes)
    const uint64_t across = (a.channels + kTileChannels - 1) / kTileChannels;
    if (a.lda >= (1 << 23) || a.ldb >= (1 << 23) || across * most_tiles(a, 64) >= (1u << 22)) return false;
    if (mean > 160) launch_tiles<T, 2, 8, 4>(a, st);
    else if (mean > 80) launch_tiles<T, 2, 8, 2>(a, st);
    else launch_tiles<T, 4, 4, 2>(a, st);
    return true;
}

void launch_i8_product(const I8Args &a, void *, hipStream_t st)
{
    if (in_pieces(a)) {
        if (a.type == SEER_F32 ? launch_pieces<float>(a, st) : a.type == SEER_BF16 ? launch_pieces<bf16_t>(a, st) : launch_pieces<f16_t>(a, st)) return;
    }
    const uint32_t across = (a.channels + kAnyChannels - 1) / kAnyChannels, tiles = most_tiles(a, kAnyTokens);
    const uint32_t grid = (uint32_t)std::min<uint64_t>((uint64_t)across * tiles, 1u << 22);
    hipLaunchKernelGGL(i8_any_kernel, dim3(grid), dim3(256), 0, st, a, tiles);
}

} // namespace seer
