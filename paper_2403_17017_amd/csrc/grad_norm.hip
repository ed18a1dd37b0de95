// The norm over many gradient tensors, and the gradients clipped by it.  A list of tensors is a matrix of ragged
// rows; the work is cut into chunks of equal size whatever tensor they belong to.  Where the tensors lie travels in
// the kernel arguments, as many as fit at a time.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

constexpr uint32_t kGradUnits = 16;                 // units of 16 bytes per lane and chunk
constexpr int kGradList = 128;
constexpr uint32_t kGradChunk = kWG * kGradUnits;   // units per chunk

struct GradList {
    const void *grad[kGradList];
    int64_t n[kGradList];
    uint32_t end[kGradList];                        // chunks up to and with this tensor's
    uint32_t count;
    int add;                                        // sums are added to what an earlier launch left
};
struct ClipList {
    GradList g;
    void *out[kGradList];
};

// The tensor that chunk c belongs to (uniform).
__device__ __forceinline__ uint32_t tensor_of(const GradList &l, uint32_t c)
{
    uint32_t lo = 0, hi = l.count - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (l.end[mid] > c) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Sums of squares in fp64: no gradient is too large or too small to be squared, and a billion terms lose nothing.
template <class T>
__global__ __launch_bounds__(kWG) void grad_square_kernel(GradList l, double *__restrict__ part)
{
    constexpr int E = Unit<T>::kElems;
    __shared__ double s_sum[kWG / kWave];
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < l.end[l.count - 1]; c += gridDim.x) {
        const uint32_t i = tensor_of(l, c);
        const T *g = static_cast<const T *>(l.grad[i]);
        const int64_t n = l.n[i], begin = (int64_t)(c - (i ? l.end[i - 1] : 0)) * kGradChunk * E;
#pragma unroll
        for (uint32_t k = 0; k < kGradUnits; ++k) {
            const int64_t at = begin + (int64_t)(k * kWG + threadIdx.x) * E;
            if (at >= n) break;
            const Unit<T> u = load_some(g + at, (int)min((int64_t)E, n - at));
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const double v = (double)(float)u.v[j];
                sum = fma(v, v, sum);
            }
        }
    }
    sum = lanes_fold(sum, [](double a, double b) { return a + b; });
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
        part[blockIdx.x] = l.add ? part[blockIdx.x] + sum : sum;
    }
}

__global__ __launch_bounds__(kWG) void grad_fold_kernel(const double *__restrict__ part, uint32_t n, float *__restrict__ norm)
{
    __shared__ double s_sum[kWG / kWave];
    double sum = 0;
    for (uint32_t i = threadIdx.x; i < n; i += kWG) sum += part[i];
    sum = lanes_fold(sum, [](double a, double b) { return a + b; });
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) norm[0] = (float)sqrt((s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]));
}

template <class T>
__global__ __launch_bounds__(kWG) void grad_scale_kernel(ClipList l, const float *__restrict__ norm, float max_norm)
{
    constexpr int E = Unit<T>::kElems;
    float by = max_norm / (norm[0] + 1e-6f);
    if (by >= 1.0f) by = 1.0f;
    for (uint32_t c = blockIdx.x; c < l.g.end[l.g.count - 1]; c += gridDim.x) {
        const uint32_t i = tensor_of(l.g, c);
        const T *g = static_cast<const T *>(l.g.grad[i]);
        T *out = static_cast<T *>(l.out[i]);
        if (by == 1.0f && g == out) continue;           // nothing changes
        const int64_t n = l.g.n[i], begin = (int64_t)(c - (i ? l.g.end[i - 1] : 0)) * kGradChunk * E;
#pragma unroll
        for (uint32_t k = 0; k < kGradUnits; ++k) {
            const int64_t at = begin + (int64_t)(k * kWG + threadIdx.x) * E;
            if (at >= n) break;
            const int have = (int)min((int64_t)E, n - at);
            Unit<T> u = load_some(g + at, have);
#pragma unroll
            for (int j = 0; j < E; ++j) u.v[j] = (T)(by * (float)u.v[j]);
            store_some(out + at, u, have);
        }
    }
}

// The tensors of one type from number `from` on that fit one launch; `from` is where the next list begins.
template <class T>
static bool next_list(const seer_grad *tensors, int32_t count, int type, int32_t *from, GradList *l, void **out)
{
    constexpr uint64_t per = (uint64_t)kGradChunk * Unit<T>::kElems;
    l->count = 0;
    uint64_t chunks = 0;
    for (; *from < count && l->count < kGradList; ++*from) {
        const seer_grad &t = tensors[*from];
        if (t.type != type || t.n == 0) continue;
        const uint64_t more = ((uint64_t)t.n + per - 1) / per;
        if (l->count && chunks + more > 0x7fffffffu) break;
        l->grad[l->count] = t.grad;
        l->n[l->count] = t.n;
        if (out) out[l->count] = t.out;
        chunks += more;
        l->end[l->count++] = (uint32_t)chunks;
    }
    return l->count != 0;
}

template <class F>
static void each_type(F f)
{
    f((float *)nullptr, SEER_F32);
    f((bf16_t *)nullptr, SEER_BF16);
    f((f16_t *)nullptr, SEER_F16);
}

void launch_grad_norm(const seer_grad *tensors, int32_t count, float *norm, void *workspace, hipStream_t st)
{
    double *part = static_cast<double *>(workspace);
    uint32_t parts = 0;
    bool first = true;
    // the partials of the launch with the most workgroups; the first launch writes all of them
    each_type([&](auto *of, int type) {
        using T = std::remove_pointer_t<decltype(of)>;
        GradList l;
        for (int32_t from = 0; next_list<T>(tensors, count, type, &from, &l, nullptr);) {
            l.add = !first;
            parts = kGradParts;
            hipLaunchKernelGGL((grad_square_kernel<T>), dim3(kGradParts), dim3(kWG), 0, st, l, part);
            first = false;
        }
    });
    hipLaunchKernelGGL(grad_fold_kernel, dim3(1), dim3(kWG), 0, st, part, parts, norm);
}

void launch_grad_clip(const seer_grad *tensors, int32_t count, float max_norm, const float *norm, hipStream_t st)
{
    each_type([&](auto *of, int type) {
        using T = std::remove_pointer_t<decltype(of)>;
        ClipList l;
        for (int32_t from = 0; next_list<T>(tensors, count, type, &from, &l.g, l.out);)
            hipLaunchKernelGGL((grad_scale_kernel<T>), dim3(std::min(l.g.end[l.g.count - 1], 4096u)), dim3(kWG), 0, st, l, norm, max_norm);
    });
}

} // namespace seer
