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
            const uint32_t first = before + __shfl(sum - tiles, l, 64);
            t->group = at + (uint32_t)l;
            t->begin = __shfl(from, l, 64) + (tile - first) * tokens;
            t->end = min(__shfl(to, l, 64), t->begin + tokens);
            return true;
        }
        before += __shfl(sum, 63, 64);
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

size_t i8_workspace_bytes(uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

void launch_i8_product(const I8Args &a, void *, hipStream_t st)
{
    const uint32_t across = (a.channels + kAnyChannels - 1) / kAnyChannels, tiles = most_tiles(a, kAnyTokens);
    const uint32_t grid = (uint32_t)std::min<uint64_t>((uint64_t)across * tiles, 1u << 22);
    hipLaunchKernelGGL(i8_any_kernel, dim3(grid), dim3(256), 0, st, a, tiles);
}

} // namespace seer
