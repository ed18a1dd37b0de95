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
// Four lanes to a block, eight values each; the largest of a block decides its scale.
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
// 128 tokens x 128 channels, 8 blocks of columns at a time through registers and LDS, four waves of 64 x 64 each.
constexpr uint32_t kMxTile = 128, kMxLine = 128 /* bytes */, kMxPitch = kMxLine + 16;

__device__ __forceinline__ v4f32 mx4_multiply(v4i32 b, v4i32 a, v4f32 acc, uint32_t sb, uint32_t sa)
{
    v8i32 wb, wa;
#pragma unroll
    for (int j = 0; j < 4; ++j) wb[j] = b[j], wa[j] = a[j];     // (the instruction reads four registers of 4-bit operands)
    wb[4] = wb[5] = wb[6] = wb[7] = wa[4] = wa[5] = wa[6] = wa[7] = 0;
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, wa, acc, 4, 4, 0, (int)sb, 0, (int)sa);
}

template <class T>
__global__ __launch_bounds__(256) void mx4_plain_kernel(Mx4Args a, uint32_t blocks)
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
                    for (int j = 0; j < 4; ++j) acc[i][j] = mx4_multiply(fb[i], fa[j], acc[i][j], sb[i], sa[j]);
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

bool mx4_product_fits(const Mx4Args &a) { return a.groups <= SEER_MAX_EXPERTS && most_blocks(a, kMxTile, kMxTile) < (1u << 30); }

size_t mx4_workspace_bytes(uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }

void launch_mx4_product(const Mx4Args &a, void *, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)most_blocks(a, kMxTile, kMxTile);
    by_type(a.type, [&](auto *of) {
        using T = std::remove_pointer_t<decltype(of)>;
        hipLaunchKernelGGL((mx4_plain_kernel<T>), dim3(std::min(blocks, 1u << 22)), dim3(256), 0, st, a, blocks);
    });
}

} // namespace seer
