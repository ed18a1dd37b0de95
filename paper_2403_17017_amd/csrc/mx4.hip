// Rows in 4-bit floating point (a sign, two bits of exponent and one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with a power of two as the scale
// of every 32 values, and products of such rows over ragged groups of them:
//   out[i][n] = sum over k of a[i][k] * b[g][n][k],  group_ptr[g] <= i < group_ptr[g + 1].
// A block's 32 values are 16 bytes, two values to a byte, the first in the lower half; its scale is a byte e that stands for 2^(e - 127), 255 for
// a NaN.  The matrix instructions take the 16 bytes and the scale byte of a block from each lane, multiply exactly and add up in fp32; as in the
// products of 8-bit integers they take channels for their rows and tokens for their columns.
#include "dense_launch.h"
#include "ragged.hiph"

namespace seer {

typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef int v8i32 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ quantisation
//
// Four lanes to a block, eight values each; the largest of a block decides its scale.  Bound by bytes: 8192 rows of 4096 bf16 to four experts each
// 28 us (138 MB, 4.9 TB/s).
constexpr uint32_t kMxBlock = 32, kMxEach = 8;

// Eight values as floats, of which n are there, zeros behind them.
template <class T>
__device__ __forceinline__ void load_eight(const T *p, int n, float (&v)[kMxEach])
{
    constexpr int E = Unit<T>::kElems;
#pragma unroll
    for (int at = 0; at < (int)kMxEach; at += E) {
        const Unit<T> u = n > at ? load_some(p + at, n - at) : zero_unit<T>();
#pragma unroll
        for (int j = 0; j < E; ++j) v[at + j] = (float)u.v[j];
    }
}

// The scale's exponent: floor(log2(largest)) - 2, so that the largest value comes to lie in 4 .. 8; `top` is the largest's bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top)
{
    return top >= 0x7f800000u ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}

// Four bytes of codes: to the nearest, ties to the even code, at most 6 in magnitude.
__device__ __forceinline__ uint32_t codes_of(const float (&v)[kMxEach], uint32_t byte)
{
    const float scale = __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
    return byte == 255 ? 0 : q;
}

template <class T, bool ROUTED, int LANES>
__global__ __launch_bounds__(kWG) void mx4_quantize_kernel(RouteRows r, const T *__restrict__ x, int64_t ldx, uint8_t *__restrict__ q, int64_t ldq,
                                                           uint8_t *__restrict__ scale, int64_t lds)
{
    const uint32_t units = (r.cols + kMxBlock - 1) / kMxBlock * (kMxBlock / kMxEach);
    for (uint32_t b = blockIdx.y; b * (kWG / LANES) < r.tokens; b += gridDim.y) {
        uint32_t t = b * (kWG / LANES) + threadIdx.x / LANES;
        if (LANES >= kWave) t = (uint32_t)__builtin_amdgcn_readfirstlane((int)t);
        if (t >= r.tokens) continue;
        for (uint32_t u = blockIdx.x * LANES + threadIdx.x % LANES; u < units; u += gridDim.x * LANES) {
            float v[kMxEach];
            load_eight(x + (int64_t)t * ldx + u * kMxEach, (int)min(r.cols - min(u * kMxEach, r.cols), kMxEach), v);
            uint32_t top = 0;
#pragma unroll
            for (uint32_t j = 0; j < kMxEach; ++j) top = max(top, __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu);
            top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
            top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
            const uint32_t byte = scale_byte(top), code = codes_of(v, byte);
            for (uint32_t k = 0; k < r.choices; ++k) {
                const int32_t slot = ROUTED ? r.choice_slot[t * r.choices + k] : (int32_t)t;
                const int64_t to = slot < 0 ? -1 - slot : slot;
                *reinterpret_cast<uint32_t *>(q + to * ldq + u * 4) = slot < 0 ? 0 : code;
                if (u % 4 == 0) scale[to * lds + u / 4] = slot < 0 ? 0 : (uint8_t)byte;
            }
        }
    }
}

// ------------------------------------------------------------------ products
//
// For rows further apart than 32-bit offsets into a tile reach: 128 tokens x 128 channels, 8 blocks of columns at a time through registers and
// LDS, four waves of 64 x 64 each, scales straight from memory.  8192 x 4 rows through 32 matrices of 4096 x 4096: 1500 us (tiles: 410).
constexpr uint32_t kMxTile = 128, kMxLine = 128 /* bytes */, kMxPitch = kMxLine + 16;

// 16 channels x 16 tokens x 128 columns: byte S of each scale word is the lane's.
template <int S>
__device__ __forceinline__ v4f32 mx4_step(v4i32 b, v4i32 a, v4f32 acc, uint32_t sb, uint32_t sa)
{
    const v8i32 wb = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1), wa = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc, 4, 4, S, (int)sb, S, (int)sa);     // (4: 4 bits, of which four registers are read)
}

template <class T>
__global__ __launch_bounds__(256) void mx4_any_kernel(Mx4Args a, uint32_t blocks)
{
    __shared__ __attribute__((aligned(16))) uint8_t s_a[kMxTile * kMxPitch], s_b[kMxTile * kMxPitch];
    __shared__ TileSearch s_search;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    for (uint32_t w = blockIdx.x; w < blocks; w += gridDim.x) {
        Tile t;
        if (!find_tile<4>(a, w, kMxTile, (a.channels + kMxTile - 1) / kMxTile, &s_search, &t)) continue;
        const uint32_t n0 = t.column * kMxTile;
        const bool zero = t.group >= a.groups;
        const int64_t group = zero ? 0 : (int64_t)t.group * a.channels;
        const uint32_t row1 = t.begin + (wave >> 1) * 64 + (lane & 15), n1 = n0 + (wave & 1) * 64;
        v4f32 acc[4][4] = {};
        for (uint32_t k0 = 0; k0 < a.blocks && !zero; k0 += 8) {
            __syncthreads();
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t row = i * 32 + threadIdx.x / 8, piece = threadIdx.x % 8;
                const v4i32 nothing = {0, 0, 0, 0};
                const bool in = k0 + piece < a.blocks;
                // (rows that are not there are taken as the last one: nobody stores them)
                *reinterpret_cast<v4i32 *>(s_a + row * kMxPitch + piece * 16) =
                    in ? *reinterpret_cast<const v4i32 *>(a.a + (int64_t)min(t.begin + row, t.end - 1) * a.lda + (k0 + piece) * 16) : nothing;
                *reinterpret_cast<v4i32 *>(s_b + row * kMxPitch + piece * 16) =
                    in ? *reinterpret_cast<const v4i32 *>(a.b + (group + min(n0 + row, a.channels - 1)) * a.ldb + (k0 + piece) * 16) : nothing;
            }
            __syncthreads();
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                v4i32 fb[4], fa[4];
                uint32_t sb[4], sa[4];
                const uint32_t block = k0 + k * 4 + lane / 16;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    fb[i] = *reinterpret_cast<const v4i32 *>(s_b + ((wave & 1) * 64 + i * 16 + (lane & 15)) * kMxPitch + k * 64 + lane / 16 * 16);
                    fa[i] = *reinterpret_cast<const v4i32 *>(s_a + ((wave >> 1) * 64 + i * 16 + (lane & 15)) * kMxPitch + k * 64 + lane / 16 * 16);
                    sb[i] = block < a.blocks ? a.b_scale[(group + min(n1 + i * 16 + (lane & 15), a.channels - 1)) * a.ldsb + block] : 0;
                    sa[i] = block < a.blocks ? a.a_scale[(int64_t)min(row1 + i * 16, t.end - 1) * a.ldsa + block] : 0;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = mx4_step<0>(fb[i], fa[j], acc[i][j], sb[i], sa[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t row = row1 + j * 16, n = n1 + i * 16 + lane / 16 * 4;
                if (row >= t.end || n >= a.channels) continue;
                float v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = acc[i][j][u];
                store_4(static_cast<T *>(a.out) + (int64_t)row * a.ldo, n, a.channels, v);
            }
    }
}

// ------------------------------------------------------------------ tiles
//
// 256 channels x 64, 128 or 256 tokens per workgroup, the codes on the same way as those of 8-bit integers: lines of 128 bytes (8 blocks) come
// straight from memory into one of two LDS buffers, and from there, 4 blocks (a step) at a time, into registers while those before
// are multiplied.  Scales come 16 blocks (a round of four steps) at a time through registers, a row to a thread, which puts the bytes in
// the order that the matrix instructions take them in: one word of a lane has the bytes of its block in each of the four steps.
// 8192 x 8192 x 8192: 281 to 300 us, 3.9 PFLOP/s at best (zeros 234; matrix instructions alone 6.4 on random codes, at the card's power).  A step takes
// 0.96 us where they would take 0.67; without its loads 0.79.  A tile's first loads and last stores add some 12 us, which nothing
// hides: 32 groups of 4096 x 4096, mean 1013, 410 us (391 at least).  Slower: wave tiles of 128 x 128 in 512 registers (the same product 420 against 390
// then, 448 before scales were realigned late), registers for the next channels' codes besides (spilled).
constexpr uint32_t kTileChannels = 256, kStepBlocks = 4, kRoundSteps = 4, kLineBytes = 128;

// WC x WAVES / WC waves, each of CI * 16 channels x TJ * 16 tokens.
template <int WAVES, int WC, int CI, int TJ>
struct Mx4Shape {
    static constexpr int kWT = WAVES / WC;
    static constexpr uint32_t kThreads = WAVES * 64, kTokens = kWT * TJ * 16, kRows = kTokens + kTileChannels;
    // loads of a lane for each buffer: a wave's load brings 8 rows
    static constexpr uint32_t kLoadsA = kTokens / (WAVES * 8), kLoadsB = kTileChannels / (WAVES * 8);
    static constexpr uint32_t kBytes = kRows * kLineBytes, kScaleRows = (kRows + kThreads - 1) / kThreads;
    static_assert(WC * CI * 16 == (int)kTileChannels, "waves cover the channels");
};

// The columns shared out: workgroups of share `s` multiply blocks s * share ... and leave their sums, [shares][rows][pitch], which
// mx4_join_kernel adds up in the order of the shares.
struct Mx4Shared { float *sums; uint32_t blocks, share /* a multiple of a round's blocks */, pitch; };

template <class T, int WAVES, int WC, int CI, int TJ, bool SHARED>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : 1) void mx4_tile_kernel(Mx4Args a, Mx4Shared shared)
{
    using Shape = Mx4Shape<WAVES, WC, CI, TJ>;
    constexpr uint32_t TOKENS = Shape::kTokens, LA = Shape::kLoadsA, LB = Shape::kLoadsB, ROWS = Shape::kRows;
    // (arrays of their own: the compiler knows that loads into one are nothing to reads from another)
    __shared__ __attribute__((aligned(1024))) int8_t s_0[Shape::kBytes], s_1[Shape::kBytes];
    __shared__ __attribute__((aligned(16))) v4i32 s_scale[2][ROWS];
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64)), lane = threadIdx.x & 63;
    const uint32_t across = (a.channels + kTileChannels - 1) / kTileChannels;
    Tile t;
    const uint32_t part = SHARED ? blockIdx.x / shared.blocks : 0;
    if constexpr (SHARED) {
        const uint32_t first = part * shared.share;
        a.a += (size_t)first * 16;
        a.b += (size_t)first * 16;
        a.a_scale += first;
        a.b_scale += first;
        a.blocks = min(shared.share, a.blocks - first);
    }
    if (!find_tile<WAVES>(a, SHARED ? blockIdx.x % shared.blocks : blockIdx.x, TOKENS, across, reinterpret_cast<TileSearch *>(s_0), &t)) return;
    __syncthreads();                                // (s_0 is filled from now on)
    const uint32_t n0 = t.column * kTileChannels;
    const uint32_t wc = wave % WC, wt = wave / WC;
    T *out = static_cast<T *>(a.out);
    v4f32 acc[CI][TJ];
#pragma unroll
    for (int i = 0; i < CI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = v4f32{0, 0, 0, 0};

    if (t.group < a.groups && a.blocks) {
        const uint32_t rows = t.end - t.begin, chans = min(kTileChannels, a.channels - n0), bytes = a.blocks * 16;
        const uint32_t lda = (uint32_t)a.lda, ldb = (uint32_t)a.ldb;
        const int64_t channel0 = (int64_t)t.group * a.channels + n0;
        const auto ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.a + (int64_t)t.begin * a.lda), 0,
                                                          (int)((rows - 1) * lda + bytes), 0x00020000);
        const auto rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.b + channel0 * a.ldb), 0, (int)((chans - 1) * ldb + bytes), 0x00020000);
        // A wave's load brings eight rows, 128 bytes of each.  Piece c of row r lies in place c ^ order(r).  What is not
        // there, rows and pieces, has an offset out of the buffer's range, costs nothing and leaves zeros.
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
        // (an offset is held against the range less the line's, which lines fetched behind the last one must not turn below zero)
        const auto fetch = [&](uint32_t line, int8_t *lds) {
            const uint32_t k0 = line * kLineBytes, nowhere = k0 + piece < bytes ? 0 : kNowhere, at = min(k0, bytes);
#pragma unroll
            for (uint32_t i = 0; i < LA; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_byte *)(lds + (i * WAVES + wave) * 1024), 16, (int)(at_a[i] | nowhere), (int)at, 0, 0);
#pragma unroll
            for (uint32_t i = 0; i < LB; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_byte *)(lds + TOKENS * kLineBytes + (i * WAVES + wave) * 1024), 16, (int)(at_b[i] | nowhere), (int)at, 0, 0);
        };
        // the scales of a thread's rows (those that are not there: the last one's), 16 blocks of round r
        const int8_t *from_scale[Shape::kScaleRows];
#pragma unroll
        for (uint32_t i = 0; i < Shape::kScaleRows; ++i) {
            const uint32_t row = threadIdx.x + i * Shape::kThreads;
            from_scale[i] = reinterpret_cast<const int8_t *>(row < TOKENS ? a.a_scale + (int64_t)(t.begin + min(row, rows - 1)) * a.ldsa
                                                                          : a.b_scale + (channel0 + min(row - TOKENS, chans - 1)) * a.ldsb);
        }
        // as words that the bytes lie in; they are realigned when they are put, not while they are on their way
        int held[Shape::kScaleRows][5];
        const auto get_scales = [&](uint32_t r) {
            const int n = (int)a.blocks - (int)(r * 16);
            if (n <= 0) return;
#pragma unroll
            for (uint32_t i = 0; i < Shape::kScaleRows; ++i) load_words(from_scale[i] + r * 16, n, held[i]);
        };
        const auto put_scales = [&](uint32_t r) {
            const int n = (int)a.blocks - (int)(r * 16);
#pragma unroll
            for (uint32_t i = 0; i < Shape::kScaleRows; ++i) {
                const uint32_t row = threadIdx.x + i * Shape::kThreads;
                // word s has the blocks of step s; word q is to have block q of every step
                const auto mix = [](int high, int low, uint32_t sel) { return (int)__builtin_amdgcn_perm((uint32_t)high, (uint32_t)low, sel); };
                v4i32 w = realigned(held[i], from_scale[i]);
                if (n < 16) w = first_bytes(w, n);
                const int a0 = mix(w[1], w[0], 0x05010400), a1 = mix(w[1], w[0], 0x07030602), b0 = mix(w[3], w[2], 0x05010400),
                          b1 = mix(w[3], w[2], 0x07030602);
                if (ROWS % Shape::kThreads == 0 || row < ROWS)
                    s_scale[r & 1][row] = v4i32{mix(b0, a0, 0x05040100), mix(b0, a0, 0x07060302), mix(b1, a1, 0x05040100), mix(b1, a1, 0x07060302)};
            }
        };
        uint32_t scale_b[CI], scale_a[TJ];
        const auto lane_scales = [&](uint32_t r) { return reinterpret_cast<const uint32_t *>(s_scale[r & 1]) + (lane & 15) * 4 + (lane >> 4); };
        const auto read_scale_a = [&](uint32_t r) {
#pragma unroll
            for (int j = 0; j < TJ; ++j) scale_a[j] = lane_scales(r)[(wt * TJ + j) * 64];
        };
        const auto read_scale_b = [&](uint32_t r, int i) { scale_b[i] = lane_scales(r)[(TOKENS / 16 + wc * CI + i) * 64]; };
        // a lane's place in the first and the second 64 bytes
        const uint32_t own = (lane & 15) * kLineBytes;
        const uint32_t from[2] = {own + ((lane >> 4) ^ order(lane & 15)) * 16, own + ((4 + (lane >> 4)) ^ order(lane & 15)) * 16};
        const uint32_t from_a = wt * TJ * 16 * kLineBytes, from_b = (TOKENS + wc * CI * 16) * kLineBytes;
        const bool busy = wt * TJ * 16 < rows;          // (waves without tokens only fetch)
        // Channels' codes are read for the next step where the last of this one has been multiplied by them, tokens' into a second set.
        v4i32 fb[CI], fa[2][TJ];
        const auto read_a = [&](const int8_t *lds, uint32_t half, v4i32 (&f)[TJ], int j) {
            f[j] = *reinterpret_cast<const v4i32 *>(lds + from[half] + from_a + j * 16 * kLineBytes);
        };
        const auto read_b = [&](const int8_t *lds, uint32_t half, int i) {
            fb[i] = *reinterpret_cast<const v4i32 *>(lds + from[half] + from_b + i * 16 * kLineBytes);
        };
        const auto multiply = [&](auto step, bool more, uint32_t next_round) __attribute__((always_inline)) {
            constexpr int S = decltype(step)::value;
            const int8_t *next = (S + 1) / 2 % 2 ? s_1 : s_0;
#pragma unroll
            for (int i = 0; i < CI; ++i) {
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = mx4_step<S>(fb[i], fa[S % 2][j], acc[i][j], scale_b[i], scale_a[j]);
                if (!more) continue;
                read_b(next, (S + 1) % 2, i);
                if (i < TJ) read_a(next, (S + 1) % 2, fa[(S + 1) % 2], i);
                if (S == kRoundSteps - 1) read_scale_b(next_round, i);
            }
            if (S == kRoundSteps - 1 && more) read_scale_a(next_round);
        };
        const uint32_t steps = (a.blocks + kStepBlocks - 1) / kStepBlocks;
        // Step s multiplies what step s - 1 has read and reads the codes of step s + 1, and in a round's last step the scales of the next one.  Odd
        // steps find the next buffer filled and nobody reading their own one any more, and send for what comes into it next.  So do, once a
        // round, the scales of the round after the next: fetched in its step 1 and put in step 3 where this round's were.
        const auto turn = [&](uint32_t s, auto step, bool scales) __attribute__((always_inline)) {
            constexpr int i = decltype(step)::value;
            if constexpr (i % 2 == 1) {
                step_barrier<0>();
                if (i == 3 && scales) put_scales(s / kRoundSteps + 2);
                fetch((s + i) / 2 + 2, i == 1 ? s_0 : s_1);
                if (i == 1 && scales) get_scales(s / kRoundSteps + 2);
            }
        };
        get_scales(0);
        put_scales(0);
        get_scales(1);
        put_scales(1);
        fetch(0, s_0);
        fetch(1, s_1);
        step_barrier<LA + LB>();
#pragma unroll
        for (int j = 0; j < TJ; ++j) read_a(s_0, 0, fa[0], j);
#pragma unroll
        for (int i = 0; i < CI; ++i) {
            read_b(s_0, 0, i);
            read_scale_b(0, i);
        }
        read_scale_a(0);
        using std::integral_constant;
        uint32_t s = 0;
        const auto work = [&](auto step) __attribute__((always_inline)) {
            constexpr int i = decltype(step)::value;
            turn(s, step, true);
            if (!busy) return;
            multiply(step, true, s / kRoundSteps + 1);
#pragma unroll
            for (int k = 0; k < CI; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, TJ, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (k < TJ) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (i == kRoundSteps - 1 && k % 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // (two scales a read)
            }
        };
        for (; s + kRoundSteps < steps; s += kRoundSteps) {
            work(integral_constant<int, 0>{});
            work(integral_constant<int, 1>{});
            work(integral_constant<int, 2>{});
            work(integral_constant<int, 3>{});
        }
        // up to four steps are left
        const auto rest = [&](auto step) __attribute__((always_inline)) {
            constexpr int i = decltype(step)::value;
            if (s + i >= steps) return;
            turn(s, step, false);
            if (busy) multiply(step, s + i + 1 < steps, s / kRoundSteps + 1);
        };
        rest(integral_constant<int, 0>{});
        rest(integral_constant<int, 1>{});
        rest(integral_constant<int, 2>{});
        rest(integral_constant<int, 3>{});
    }
    if constexpr (SHARED) {
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int i = 0; i < CI; ++i) {
                const uint32_t row = t.begin + (wt * TJ + j) * 16 + (lane & 15), n = n0 + (wc * CI + i) * 16 + (lane >> 4) * 4;
                if (row < t.end && n < shared.pitch)
                    *reinterpret_cast<v4f32 *>(shared.sums + ((size_t)part * a.rows + row) * shared.pitch + n) = acc[i][j];
            }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // nothing is on its way to LDS when the workgroup ends
        return;
    }
    // A lane's results are four channels each of TJ * CI tokens.  They change places in LDS, in a region of the wave's own, so that
    // stores are of 16 bytes and lines are written whole.  A row's pieces lie in the order of their number xor the row.
    const bool zero = t.group >= a.groups;
    constexpr int CIP = CI * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : CI;      // channels go by up to 256 bytes of a row
    constexpr uint32_t PIECES = CIP * sizeof(T), ROW = PIECES * 16, E = Unit<T>::kElems;
    constexpr uint32_t kPer = WAVES / 2;            // waves to a buffer
    static_assert(kPer * TJ * 16 * ROW <= Shape::kBytes && CI % CIP == 0, "the waves' regions fit");
    step_barrier<0>();                              // nothing is on its way to LDS, and nobody reads the last codes any more
    int8_t *mine = (wave / kPer == 0 ? s_0 : s_1) + (wave % kPer) * (TJ * 16 * ROW);
#pragma unroll
    for (int first = 0; first < CI; first += CIP) {
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
            for (int i = 0; i < CIP; ++i) {
                typedef T four __attribute__((ext_vector_type(4)));
                four v;
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = zero ? (T)0.0f : (T)acc[first + i][j][u];
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

// The sums of all shares: four channels to a lane.
template <class T>
__global__ __launch_bounds__(kWG) void mx4_join_kernel(Mx4Args a, Mx4Shared shared, uint32_t shares)
{
    const uint32_t quads = shared.pitch / 4;
    for (uint64_t w = (uint64_t)blockIdx.x * kWG + threadIdx.x; w < (uint64_t)a.rows * quads; w += (uint64_t)gridDim.x * kWG) {
        const uint32_t row = (uint32_t)(w / quads), n = (uint32_t)(w % quads) * 4;
        v4f32 sum = *reinterpret_cast<const v4f32 *>(shared.sums + (size_t)row * shared.pitch + n);
        for (uint32_t s = 1; s < shares; ++s) sum += *reinterpret_cast<const v4f32 *>(shared.sums + ((size_t)s * a.rows + row) * shared.pitch + n);
        const bool in = group_of(a, row) < a.groups;
        const float v[4] = {in ? sum[0] : 0.0f, in ? sum[1] : 0.0f, in ? sum[2] : 0.0f, in ? sum[3] : 0.0f};
        store_4(static_cast<T *>(a.out) + (int64_t)row * a.ldo, n, a.channels, v);
    }
}

// ------------------------------------------------------------------ few rows to a group
//
// CI * 16 channels of one group per workgroup, whose waves each take a share of the columns; both operands come straight from memory, the
// weights once per 64 rows, and the waves' sums meet in LDS.  Bound by the bytes of b: 8192 x 8192, one row, 10.3 us (3.5 TB/s), 64 groups of
// 2048 x 4096 with four rows each on average 63 (4.5 TB/s).  32 channels to a workgroup: 14.8 us for the one row with its quantisation
// (16: 15.7), 61.8 for the groups (67.2), but 2 % slower over 300 draws; eight waves 15.0 and 99.9.
constexpr uint32_t kMxFewRows = 64, kRoundBlocks = kRoundSteps * kStepBlocks;

// 16 TJ rows: the calling wave's blocks [k, k_end), R rounds of 16 at a time.  Pointers are those of the lane's rows, of codes with the lane's
// block added.
template <int CI, int TJ, int R>
__device__ __forceinline__ void mx4_few_sums(const uint8_t *const (&pb)[CI], const uint8_t *const (&pa)[TJ], const int8_t *const (&sb)[CI],
                                             const int8_t *const (&sa)[TJ], uint32_t k, uint32_t k_end, uint32_t q, v4f32 (&acc)[CI][TJ])
{
#pragma unroll
    for (int i = 0; i < CI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j) acc[i][j] = v4f32{0, 0, 0, 0};
    const auto rounds = [&](auto count, auto whole) {
        constexpr int N = decltype(count)::value;
        constexpr bool WHOLE = decltype(whole)::value;
        v4i32 fb[4 * N][CI], fa[4 * N][TJ], wb[N][CI], wa[N][TJ];
        const int n = WHOLE ? 16 : (int)(k_end - k);
#pragma unroll
        for (int r = 0; r < N; ++r) {
#pragma unroll
            for (int i = 0; i < CI; ++i) wb[r][i] = load_16(sb[i] + k + r * 16, n);
#pragma unroll
            for (int j = 0; j < TJ; ++j) wa[r][j] = load_16(sa[j] + k + r * 16, n);
        }
        const auto piece = [&](const uint8_t *p, int u) {
            if (WHOLE || k + u * 4 + q < k_end) return *reinterpret_cast<const v4i32 *>(p + (size_t)(k + u * 4) * 16);
            return v4i32{0, 0, 0, 0};
        };
#pragma unroll
        for (int u = 0; u < 4 * N; ++u)
#pragma unroll
            for (int i = 0; i < CI; ++i) fb[u][i] = piece(pb[i], u);
#pragma unroll
        for (int u = 0; u < 4 * N; ++u)
#pragma unroll
            for (int j = 0; j < TJ; ++j) fa[u][j] = piece(pa[j], u);
#pragma unroll
        for (int u = 0; u < 4 * N; ++u) {
            uint32_t a_byte[TJ];
#pragma unroll
            for (int j = 0; j < TJ; ++j) a_byte[j] = (uint32_t)wa[u / 4][j][u % 4] >> (8 * q);
#pragma unroll
            for (int i = 0; i < CI; ++i) {
                const uint32_t b_byte = (uint32_t)wb[u / 4][i][u % 4] >> (8 * q);
#pragma unroll
                for (int j = 0; j < TJ; ++j) acc[i][j] = mx4_step<0>(fb[u][i], fa[u][j], acc[i][j], b_byte, a_byte[j]);
            }
        }
        k += 16 * N;
    };
    using std::integral_constant;
    while (k + 16 * R <= k_end) rounds(integral_constant<int, R>{}, std::true_type{});
    if constexpr (R > 1)
        while (k + 16 <= k_end) rounds(integral_constant<int, 1>{}, std::true_type{});
    if (k < k_end) rounds(integral_constant<int, 1>{}, std::false_type{});
}

template <class T, int CI, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void mx4_few_kernel(Mx4Args a, uint32_t share)
{
    __shared__ __attribute__((aligned(16))) v4f32 s_acc[2][WAVES][CI][64];
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
    const uint32_t k_begin = min(a.blocks, wave * share), k_end = min(a.blocks, k_begin + share);
    const uint32_t q = lane >> 4;
    const uint8_t *pb[CI];
    const int8_t *sb[CI];
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const int64_t row = (int64_t)g * a.channels + min(n0 + i * 16 + (lane & 15), a.channels - 1);
        pb[i] = a.b + row * a.ldb + q * 16;
        sb[i] = reinterpret_cast<const int8_t *>(a.b_scale + row * a.ldsb);
    }
    const auto rows = [&](uint32_t at, auto count, auto at_once) {
        constexpr int TJ = decltype(count)::value;
        const uint8_t *pa[TJ];
        const int8_t *sa[TJ];
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
            const int64_t row = min(at + j * 16 + (lane & 15), end - 1);
            pa[j] = a.a + row * a.lda + q * 16;
            sa[j] = reinterpret_cast<const int8_t *>(a.a_scale + row * a.ldsa);
        }
        v4f32 acc[CI][TJ];
        mx4_few_sums<CI, TJ, decltype(at_once)::value>(pb, pa, sb, sa, k_begin, k_end, q, acc);
        // 16 rows at a time the waves' sums meet; wave i adds up and stores channels i * 16 ...
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
#pragma unroll
            for (int i = 0; i < CI; ++i) s_acc[j & 1][wave][i][lane] = acc[i][j];
            __syncthreads();
            if (wave < CI) {
                v4f32 sum = s_acc[j & 1][0][wave][lane];
#pragma unroll
                for (int o = 1; o < WAVES; ++o) sum += s_acc[j & 1][o][wave][lane];
                const uint32_t row = at + j * 16 + (lane & 15), n = n0 + wave * 16 + (lane >> 4) * 4;
                if (row < end && n < a.channels) {
                    const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
                    store_4(out + (int64_t)row * a.ldo, n, a.channels, v);
                }
            }
        }
        __syncthreads();
    };
    using std::integral_constant;
    for (uint32_t at = begin; at < end; at += kMxFewRows) {
        const uint32_t left = end - at;
        if (left <= 16) rows(at, integral_constant<int, 1>{}, integral_constant<int, 2>{});
        else if (left <= 32) rows(at, integral_constant<int, 2>{}, integral_constant<int, 1>{});
        else rows(at, integral_constant<int, 4>{}, integral_constant<int, 1>{});
    }
}

// ------------------------------------------------------------------ launches

void launch_mx4_quantize(const RouteRows &rows, const seer_dense &x, const seer_mx4 &q, hipStream_t st)
{
    by_type(x.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        const uint32_t units = (rows.cols + kMxBlock - 1) / kMxBlock * (kMxBlock / kMxEach);
        const auto launch = [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            constexpr uint32_t per = kWG / LANES;
            const dim3 grid(std::min(1024u, (units + LANES - 1) / LANES), std::min((rows.tokens + per - 1) / per, 65535u));
            const T *xp = static_cast<const T *>(x.data);
            uint8_t *qp = static_cast<uint8_t *>(q.data), *sp = static_cast<uint8_t *>(q.scale);
            if (rows.choice_slot)
                hipLaunchKernelGGL((mx4_quantize_kernel<T, true, LANES>), grid, dim3(kWG), 0, st, rows, xp, x.ld, qp, q.ld, sp, q.scale_ld);
            else hipLaunchKernelGGL((mx4_quantize_kernel<T, false, LANES>), grid, dim3(kWG), 0, st, rows, xp, x.ld, qp, q.ld, sp, q.scale_ld);
        };
        if (units <= 32) launch(std::integral_constant<int, 16>{});
        else if (units <= 128) launch(std::integral_constant<int, 64>{});
        else launch(std::integral_constant<int, 256>{});
    });
}

// The arithmetic on tiles is 32-bit.  Of the tiles of 64 rows there may be twice as many as of these (up to 128 channels), so below 2^31, and a launch has
// fewer than 2^24 of them (mx4_plan).
bool mx4_product_fits(const Mx4Args &a) { return a.groups <= SEER_MAX_EXPERTS && most_blocks(a, kMxTile, kMxTile) < (1u << 30); }

template <class T, int WAVES, int WC, int CI, int TJ>
static void launch_tiles(const Mx4Args &a, hipStream_t st)
{
    using Shape = Mx4Shape<WAVES, WC, CI, TJ>;
    hipLaunchKernelGGL((mx4_tile_kernel<T, WAVES, WC, CI, TJ, false>), dim3((uint32_t)most_blocks(a, Shape::kTokens, kTileChannels)), dim3(Shape::kThreads),
                       0, st, a, Mx4Shared{});
}

// Which kernel: the one whose time by the following lines (us) is the least.  They are fitted to 300 draws (one matrix, or 2 to 64 with rows to a group
// 1, 1 / sqrt(rank) or 1 / rank; 128 to 12 288 channels and 256 to 12 288 columns; weights from memory) of which each kernel was
// timed.  Of 220 other draws, whose times are kept in profiles/mx4_kernel_times.csv, what is chosen takes 2.4 % longer than the best one on average,
// 1.47 times at most.  Measured, us, few rows, tiles of 64, of 128 and of 256 tokens: 1848 x 1856, 41 rows 5.4, 11, 11 and 14; 11 976 x 7872,
// 16 rows 20, 61, 56 and 59; 8944 x 1536, 82 rows 13, 11, 12 and 14; 46 groups of 456 x 10 912, mean 142, 239, 152, 86 and 110; 43 of
// 6088 x 1792, mean 168, 516, 175, 146 and 113.  Columns shared between two and four workgroups (tiles of 64, one share): 6520 x 6304,
// 19 rows 32 and 22 (48), 2936 x 3296, 44 rows 17 and 13 (20).
constexpr double kJoinCost = 5;     // the second launch; and 1 us for every 3 MB of sums written and read

static double few_cost(const Mx4Args &a)
{
    const double mean = a.rows / a.groups, bytes = 17.0 * a.blocks, workgroups = (double)((a.channels + 15) / 16) * a.groups;
    const double rows = std::max((mean + 16) * workgroups / kCUs, (a.group_ptr ? 4 : 1) * mean + 16);
    const double batches = a.rows / a.groups / kMxFewRows;      // (behind the first)
    return std::max(2.9 + 1.55 * batches + 0.56 * (batches + 1) * workgroups / kCUs + rows * bytes / 30.6e3, 2.9 + a.groups * (double)a.channels * bytes / 3.9e6);
}

struct Mx4TileCost { uint32_t tokens; double least, more /* a step, by how many CUs are at work */, round, read, groups; };
constexpr Mx4TileCost kMx64 = {64, 0.513, 0.251, 4.4, 2.6, 1.10}, kMx128 = {128, 0.564, 0.284, 5.5, 2.5, 1.08}, kMx256 = {256, 0.695, 0.389, 7.9, 2.7, 1.07};

static double tile_cost(const Mx4Args &a, const Mx4TileCost &c, uint32_t shares)
{
    const uint64_t down = a.group_ptr ? (uint64_t)a.rows / c.tokens + (a.groups + 1) / 2 : ((uint64_t)a.rows + c.tokens - 1) / c.tokens;
    const uint64_t tiles = down * ((a.channels + kTileChannels - 1) / kTileChannels) * shares, rest = tiles % kCUs;
    const double steps = (double)((a.blocks + kStepBlocks - 1) / kStepBlocks) / shares;
    const auto round = [&](double full) { return steps * (c.least + c.more * full) + c.round; };
    const double t = (double)(tiles / kCUs) * round(1) + (rest ? round((double)rest / kCUs) : 0);
    return std::max(t * (a.group_ptr ? c.groups : 1), (double)a.groups * a.channels * (17.0 * a.blocks) / (c.read * 1e6) + 3);
}

static Mx4Shared shared_columns(const Mx4Args &a, uint32_t shares, void *workspace)
{
    const uint32_t rounds = (a.blocks + kRoundBlocks - 1) / kRoundBlocks;
    return Mx4Shared{static_cast<float *>(workspace), (uint32_t)most_blocks(a, 64, kTileChannels), (rounds + shares - 1) / shares * kRoundBlocks, (a.channels + 3) & ~3u};
}

// How many of `shares` are left when each is whole rounds.
static uint32_t whole_shares(uint32_t blocks, uint32_t shares)
{
    const uint32_t rounds = (blocks + kRoundBlocks - 1) / kRoundBlocks, each = (rounds + shares - 1) / shares;
    return (rounds + each - 1) / each;
}

struct Mx4Choice { uint32_t tokens /* 0: few rows */, shares; };

static Mx4Choice choose(const Mx4Args &a)
{
    Mx4Choice best{0, 1};
    double least = few_cost(a);
    const auto consider = [&](uint32_t tokens, uint32_t shares, double cost) {
        if (cost >= least) return;
        least = cost;
        best = Mx4Choice{tokens, shares};
    };
    consider(256, 1, tile_cost(a, kMx256, 1));
    consider(128, 1, tile_cost(a, kMx128, 1));
    consider(64, 1, tile_cost(a, kMx64, 1));
    const uint64_t tiles = most_blocks(a, 64, kTileChannels);
    if (tiles > kCUs / 2) return best;
    const uint32_t most = (uint32_t)std::min<uint64_t>({kCUs / tiles, (uint64_t)a.blocks / kRoundBlocks / 2, 16});
    for (uint32_t n = 2; n <= most; ++n) consider(64, n, tile_cost(a, kMx64, n) + n * (8.0 * a.rows * a.channels) / 3e6 + kJoinCost);
    return best;
}

size_t mx4_workspace_bytes(uint32_t rows, uint32_t channels, uint32_t blocks, uint32_t groups)
{
    Mx4Args a{};
    a.rows = rows;
    a.channels = channels;
    a.blocks = blocks;
    a.groups = groups;
    if (rows == 0 || channels == 0) return 0;
    static const int32_t some = 0;                  // one group may come with its group_ptr or without
    uint32_t shares = groups == 1 ? choose(a).shares : 1;
    a.group_ptr = &some;
    shares = std::max(shares, choose(a).shares);
    return shares > 1 ? (size_t)shares * rows * ((channels + 3) & ~3u) * 4 : 0;
}

// The kernel for a product: what takes least, where rows are near enough (offsets into a tile are 32-bit) and a launch has fewer than 2^32 lanes.
Mx4Plan mx4_plan(const Mx4Args &a)
{
    const Mx4Plan any{SEER_MX4_ANY, 0, 1};
    if (a.lda >= (1 << 23) || a.ldb >= (1 << 23)) return any;
    const Mx4Choice c = choose(a);
    if (c.tokens == 0) return (uint64_t)((a.channels + 15) / 16) * 256 < 1ull << 32 ? Mx4Plan{SEER_MX4_FEW, 0, 1} : any;
    if (c.shares > 1) return Mx4Plan{SEER_MX4_SHARED, c.tokens, whole_shares(a.blocks, c.shares)};
    return most_blocks(a, c.tokens, kTileChannels) * (c.tokens == 64 ? 256 : 512) < 1ull << 32 ? Mx4Plan{SEER_MX4_TILES, c.tokens, 1} : any;
}

static_assert(SEER_MAX_EXPERTS < 65535, "groups are a dimension of the grid of the kernel for few rows");

void launch_mx4_product(const Mx4Args &a, const Mx4Plan &p, void *workspace, hipStream_t st)
{
    by_type(a.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        switch (p.kernel) {
        case SEER_MX4_FEW: {
            const uint32_t groups = a.groups + (a.group_ptr ? 1 : 0), share = ((a.blocks + 3) / 4 + kRoundBlocks - 1) / kRoundBlocks * kRoundBlocks;
            hipLaunchKernelGGL((mx4_few_kernel<T, 1, 4>), dim3((a.channels + 15) / 16, groups), dim3(256), 0, st, a, share);
            return;
        }
        case SEER_MX4_TILES:
            if (p.tokens == 256) launch_tiles<T, 8, 2, 8, 4>(a, st);
            else if (p.tokens == 128) launch_tiles<T, 8, 2, 8, 2>(a, st);
            else launch_tiles<T, 4, 4, 4, 4>(a, st);
            return;
        case SEER_MX4_SHARED: {
            const Mx4Shared c = shared_columns(a, p.shares, workspace);
            hipLaunchKernelGGL((mx4_tile_kernel<float, 4, 4, 4, 4, true>), dim3(c.blocks * p.shares), dim3(256), 0, st, a, c);
            const uint64_t lanes = (uint64_t)a.rows * (c.pitch / 4);
            hipLaunchKernelGGL((mx4_join_kernel<T>), dim3((uint32_t)std::min<uint64_t>((lanes + kWG - 1) / kWG, 8 * kCUs)), dim3(kWG), 0, st, a, c, p.shares);
            return;
        }
        default: {
            const uint32_t blocks = (uint32_t)most_blocks(a, kMxTile, kMxTile);
            hipLaunchKernelGGL((mx4_any_kernel<T>), dim3(std::min(blocks, 1u << 22)), dim3(256), 0, st, a, blocks);
        }
        }
    });
}

} // namespace seer
