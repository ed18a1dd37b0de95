// The norm over many gradient tensors, and the gradients clipped by it.  A list of tensors is a matrix of ragged
// rows; the work is cut into chunks of equal size whatever tensor they belong to.  Where the tensors lie travels in
// the kernel arguments, as many as fit 4 KB at a time.  Bound by bytes: every gradient is read for the norm and, since that has to be
// known first, once more; the second pass goes backwards, so that it begins with what the first has left in the last-level cache.
// A billion bf16 in 291 tensors: 335 us for the norm (6.0 TB/s, near a read's rate), 717 for the scaling into a bucket (5.6 TB/s), 735 in place,
// two launches each; in place with nothing to scale 90, for a walk over the chunks that reads the first of each workgroup.
#include "dense.hiph"
#include "dense_launch.h"

namespace seer {

constexpr uint32_t kGradUnits = 4;                  // units of 16 bytes per lane and chunk
constexpr uint32_t kGradChunk = kWG * kGradUnits;   // units per chunk (16 KB; 8 and 32 KB: 2 % slower, 2 and 8 KB: 10 %)
constexpr int kSquareList = 288, kScaleList = 180;

// Tensors of one type: `end` chunks up to and with each, `rest` elements in the last chunk of each less one.
template <int N>
struct GradList {
    const void *grad[N];
    uint32_t end[N];
    uint16_t rest[N];
    uint32_t count;
};
template <int N>
struct OutList {
    void *out[N];
};
static_assert(sizeof(GradList<kSquareList>) + 24 <= 4096 && sizeof(GradList<kScaleList>) + sizeof(OutList<kScaleList>) + 32 <= 4096,
              "the lists fit the kernel arguments");

// A chunk: `have` elements from element `begin` on of tensor i.
struct Chunk {
    uint32_t i, have;
    int64_t begin;
};

// Chunk c of the list, of E elements a unit; `back`: a tensor's chunks are counted from its end.  The lanes of a wave look for the
// tensor together; the result is uniform.
template <int E, int N>
__device__ __forceinline__ Chunk chunk_of(const GradList<N> &l, uint32_t c, bool back)
{
    uint32_t i = 0;
    for (uint32_t at = 0; at < l.count; at += kWave) {
        const uint32_t mine = at + (threadIdx.x & 63);
        const uint64_t past = __ballot(mine < l.count && l.end[min(mine, (uint32_t)N - 1)] <= c);
        i += (uint32_t)__popcll(past);
        if (past != ~0ull) break;
    }
    const uint32_t first = i ? l.end[i - 1] : 0, last = l.end[i] - 1 - first;
    const uint32_t k = back ? last - (c - first) : c - first;
    return Chunk{i, k == last ? (uint32_t)l.rest[i] + 1 : kGradChunk * E, (int64_t)k * (kGradChunk * E)};
}

// Sum over a workgroup in a fixed order, in every lane.
__device__ __forceinline__ double workgroup_sum(double v, double *s_sum)
{
    v = lanes_fold(v, [](double a, double b) { return a + b; });
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x / 64] = v;
    __syncthreads();
    return (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}

// Sums of squares in fp64: no gradient is too large or too small to be squared, and a billion terms lose nothing.
// part[b] is added to where an earlier launch has left something there (b < left).
template <class T>
__global__ __launch_bounds__(kWG) void grad_square_kernel(GradList<kSquareList> l, double *__restrict__ part, uint32_t left)
{
    constexpr int E = Unit<T>::kElems;
    __shared__ double s_sum[kWG / kWave];
    double sum[2] = {0, 0};
    const auto add = [&](const Unit<T> &u) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const double v = (double)(float)u.v[j];
            sum[j & 1] = fma(v, v, sum[j & 1]);
        }
    };
    for (uint32_t c = blockIdx.x; c < l.end[l.count - 1]; c += gridDim.x) {
        const Chunk k = chunk_of<E>(l, c, false);
        const T *g = static_cast<const T *>(l.grad[k.i]) + k.begin + threadIdx.x * E;
        if (k.have == kGradChunk * E) {
            Unit<T> u[kGradUnits];
#pragma unroll
            for (uint32_t h = 0; h < kGradUnits; ++h) u[h] = load_unit(g + h * kWG * E);
#pragma unroll
            for (uint32_t h = 0; h < kGradUnits; ++h) add(u[h]);
        } else {
            for (uint32_t at = threadIdx.x * E; at < k.have; at += kWG * E, g += kWG * E)
                add(load_some(g, (int)min((uint32_t)E, k.have - at)));
        }
    }
    const double all = workgroup_sum(sum[0] + sum[1], s_sum);
    if (threadIdx.x == 0) part[blockIdx.x] = blockIdx.x < left ? part[blockIdx.x] + all : all;
}

// The partial sums, as each lane of a workgroup adds them up; fetched before, folded when the rest of a kernel's loads are on their way.
struct Partial {
    double v[kGradParts / kWG];
    __device__ __forceinline__ void fetch(const double *part, uint32_t parts)
    {
#pragma unroll
        for (uint32_t i = 0; i < kGradParts / kWG; ++i) v[i] = i * kWG + threadIdx.x < parts ? part[i * kWG + threadIdx.x] : 0.0;
    }
    __device__ __forceinline__ float norm(double *s_sum) const
    {
        double sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kGradParts / kWG; ++i) sum += v[i];
        return (float)sqrt(workgroup_sum(sum, s_sum));
    }
};

__global__ __launch_bounds__(kWG) void grad_norm_kernel(const double *__restrict__ part, uint32_t parts, float *__restrict__ norm)
{
    __shared__ double s_sum[kWG / kWave];
    Partial p;
    p.fetch(part, parts);
    const float n = p.norm(s_sum);
    if (threadIdx.x == 0) norm[0] = n;
}

// Every workgroup folds the partial sums for itself (16 KB at most, from L2): quicker than a launch of one workgroup between
// the two passes.  Its first chunk is fetched meanwhile
// (61 tensors of 24 MB, both passes: 18.0 us, 19.3 without).
template <class T>
__global__ __launch_bounds__(kWG) void grad_scale_kernel(GradList<kScaleList> l, OutList<kScaleList> o, const double *__restrict__ part,
                                                         uint32_t parts, float max_norm, float *__restrict__ norm)
{
    constexpr int E = Unit<T>::kElems;
    constexpr uint32_t kWhole = kGradChunk * E;
    __shared__ double s_sum[kWG / kWave];
    const uint32_t chunks = l.end[l.count - 1];
    Unit<T> u[kGradUnits];
    const auto fetch = [&](const Chunk &k) {
        const T *g = static_cast<const T *>(l.grad[k.i]) + k.begin + threadIdx.x * E;
        if (k.have == kWhole) {
#pragma unroll
            for (uint32_t h = 0; h < kGradUnits; ++h) u[h] = stream_unit(g + h * kWG * E);
        }
    };
    Partial p;
    p.fetch(part, parts);
    Chunk k = chunk_of<E>(l, blockIdx.x, true);         // (there are no more workgroups than chunks)
    fetch(k);
    const float n = p.norm(s_sum);
    if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = n;
    float by = max_norm / (n + 1e-6f);
    if (by >= 1.0f) by = 1.0f;
    const auto scaled = [by](Unit<T> v) {
#pragma unroll
        for (int j = 0; j < E; ++j) v.v[j] = (T)(by * (float)v.v[j]);
        return v;
    };
    for (uint32_t c = blockIdx.x;;) {
        T *out = static_cast<T *>(o.out[k.i]) + k.begin + threadIdx.x * E;
        if (by == 1.0f && l.grad[k.i] == o.out[k.i]) {
            // nothing changes
        } else if (k.have == kWhole) {
#pragma unroll
            for (uint32_t h = 0; h < kGradUnits; ++h) stream_unit(out + h * kWG * E, scaled(u[h]));
        } else {
            const T *g = static_cast<const T *>(l.grad[k.i]) + k.begin + threadIdx.x * E;
            for (uint32_t at = threadIdx.x * E; at < k.have; at += kWG * E, g += kWG * E, out += kWG * E) {
                const int have = (int)min((uint32_t)E, k.have - at);
                store_some(out, scaled(load_some(g, have)), have);
            }
        }
        if ((c += gridDim.x) >= chunks) return;
        k = chunk_of<E>(l, c, true);
        if (by != 1.0f || l.grad[k.i] != o.out[k.i]) fetch(k);
    }
}

// The tensors of one type from number *from on (step 1: upwards, -1: downwards) that fit one launch; *from is where the next
// list begins.
template <class T, int N>
static bool next_list(const seer_grad *tensors, int32_t count, int type, int32_t *from, int32_t step, GradList<N> *l, OutList<N> *o)
{
    constexpr uint64_t per = (uint64_t)kGradChunk * Unit<T>::kElems;
    static_assert(per <= 65536, "the rest of a chunk has 16 bits");
    l->count = 0;
    uint64_t chunks = 0;
    for (; *from >= 0 && *from < count && l->count < (uint32_t)N; *from += step) {
        const seer_grad &t = tensors[*from];
        if (t.type != type || t.n == 0) continue;
        const uint64_t more = ((uint64_t)t.n + per - 1) / per;
        if (l->count && chunks + more > 0x7fffffffu) break;
        l->grad[l->count] = t.grad;
        l->rest[l->count] = (uint16_t)(((uint64_t)t.n - 1) % per);
        if (o) o->out[l->count] = t.out;
        chunks += more;
        l->end[l->count++] = (uint32_t)chunks;
    }
    return l->count != 0;
}

template <int N>
static uint32_t grid_of(const GradList<N> &l) { return std::min(l.end[l.count - 1], kGradParts); }

template <class T>
static void launch_squares(const seer_grad *tensors, int32_t count, int type, double *part, uint32_t *parts, hipStream_t st)
{
    GradList<kSquareList> l;
    for (int32_t from = 0; next_list<T>(tensors, count, type, &from, 1, &l, (OutList<kSquareList> *)nullptr);) {
        const uint32_t grid = grid_of(l);
        hipLaunchKernelGGL((grad_square_kernel<T>), dim3(grid), dim3(kWG), 0, st, l, part, *parts);
        *parts = std::max(*parts, grid);
    }
}

template <class T>
static bool launch_scales(const seer_grad *tensors, int32_t count, int type, const double *part, uint32_t parts, float max_norm, float *norm,
                          hipStream_t st)
{
    GradList<kScaleList> l;
    OutList<kScaleList> o;
    bool any = false;
    for (int32_t from = count - 1; next_list<T>(tensors, count, type, &from, -1, &l, &o); any = true)
        hipLaunchKernelGGL((grad_scale_kernel<T>), dim3(grid_of(l)), dim3(kWG), 0, st, l, o, part, parts, max_norm, norm);
    return any;
}

static uint32_t launch_all_squares(const seer_grad *tensors, int32_t count, double *part, hipStream_t st)
{
    uint32_t parts = 0;
    launch_squares<float>(tensors, count, SEER_F32, part, &parts, st);
    launch_squares<f16_t>(tensors, count, SEER_F16, part, &parts, st);
    launch_squares<bf16_t>(tensors, count, SEER_BF16, part, &parts, st);
    return parts;
}

void launch_grad_norm(const seer_grad *tensors, int32_t count, float *norm, void *workspace, hipStream_t st)
{
    double *part = static_cast<double *>(workspace);
    const uint32_t parts = launch_all_squares(tensors, count, part, st);
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kWG), 0, st, part, parts, norm);
}

void launch_grad_clip(const seer_grad *tensors, int32_t count, float max_norm, float *norm, void *workspace, hipStream_t st)
{
    double *part = static_cast<double *>(workspace);
    const uint32_t parts = launch_all_squares(tensors, count, part, st);
    const bool b = launch_scales<bf16_t>(tensors, count, SEER_BF16, part, parts, max_norm, norm, st);
    const bool h = launch_scales<f16_t>(tensors, count, SEER_F16, part, parts, max_norm, norm, st);
    const bool f = launch_scales<float>(tensors, count, SEER_F32, part, parts, max_norm, norm, st);
    if (!b && !h && !f) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kWG), 0, st, part, parts, norm);
}

} // namespace seer
