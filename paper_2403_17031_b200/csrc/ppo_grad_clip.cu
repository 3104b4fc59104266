// Norm over many gradients and their clipping (ppo_grad_clip):
//     norm = |scale| * sqrt(sum over all tensors and elements of x^2),   coef = min(1, max_norm / norm),
//     out  = x * (scale * coef)
// Bound by memory: every tensor is read for the norm and again for the result, which cannot start before the norm is known.
// 50 tensors, 1.22 G elements, bf16 to fp32: 1610 us = 370 for the norm (6.6 TB/s) and 1240 for the results (5.9 TB/s; stores of fp32
// in two halves of 16 bytes, which write every sector twice, took 1650).
//
// Two launches. Both walk the tensors in chunks of 32 K elements, chunk c by block c mod grid, so that a list of a few large
// and many small tensors is shared out evenly. Pass 1 leaves one fp64 sum per block; every block of pass 2 adds those up in
// the same order (no atomics: the norm does not depend on timing) and scales its chunks in reverse order, the last ones of
// pass 1 first, which are still in L2. Where nothing changes (in place, scale * coef = 1) pass 2 ends there.
//
// Squares are fp32 and summed eight at a time before they go to fp64 (a conversion per element would bound the pass: 16 per
// clock and SM). Eight squares that overflow, or that are small enough to lose digits, are taken again in fp64.
#include "ppo_packs.cuh"

#include <algorithm>
#include <cstdlib>

namespace ppo {
namespace clip {

constexpr int kThreads = 512, kBlocksPerSm = 4;
constexpr int kChunk = 32768;                     // elements
constexpr int kMaxBlocks = kBlocksPerSm * 256;    // partial sums of one launch

// The tensors of one launch travel as kernel arguments: nothing has to be copied to the device before it, and a captured
// launch keeps them.
template <int N>
struct Table {
    const void *in[N];
    void *out[N];
    int64_t numel[N];
    int32_t first[N];                             // first chunk
    uint8_t type[N];                              // bit 0: bf16 in, bit 1: bf16 out, bit 2: packs of 8, bit 3: in place
};

struct Args {
    int n, chunks;                                // of this launch
    double *part;                                 // [launches][kMaxBlocks]
    int launch, launches, blocks;                 // partial sums: `blocks` of each launch
    float scale, max_norm;
    float *norm;                                  // [2] norm, coef
    int *status;
};

template <int COUNT>
__device__ __forceinline__ double squares(const float *x)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < COUNT; ++j) s = fmaf(x[j], x[j], s);
    // (2^-100 is far enough above fp32's smallest values)
    if (s < 7.9e-31f || s > 1e38f) {
        double d = 0.0;
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) any |= __float_as_uint(x[j]) << 1;
        if (!any) return d;
#pragma unroll
        for (int j = 0; j < COUNT; ++j) d = fma((double)x[j], (double)x[j], d);
        return d;
    }
    return (double)s;                             // (NaN comes through)
}

template <int N>
__device__ __forceinline__ int tensor_of(const Table<N> &t, int n, int chunk)
{
    int lo = 0, hi = n - 1;                       // last tensor whose first chunk is at or before this one
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// elements [e0, e1) of one tensor
template <typename TI>
__device__ __forceinline__ double sum_chunk(const TI *in, int64_t e0, int64_t e1, bool packs)
{
    double sum = 0.0;
    const int64_t whole = packs ? e0 + ((e1 - e0) & ~7ll) : e0;
#pragma unroll 4
    for (int64_t j = e0 + threadIdx.x * 8; j < whole; j += kThreads * 8) {
        Pack<TI, 8> p;
        p.load(in + j);
        float x[8];
        p.get(x);
        sum += squares<8>(x);
    }
#pragma unroll 4
    for (int64_t j = whole + threadIdx.x; j < e1; j += kThreads) {
        Pack<TI, 1> p;
        p.load(in + j);
        float x[1];
        p.get(x);
        sum += squares<1>(x);
    }
    return sum;
}

template <typename TI, typename TO>
__device__ __forceinline__ void scale_chunk(const TI *in, TO *out, float f, int64_t e0, int64_t e1, bool packs)
{
    const int64_t whole = packs ? e0 + ((e1 - e0) & ~7ll) : e0;
#pragma unroll 4
    for (int64_t j = e0 + threadIdx.x * 8; j < whole; j += kThreads * 8) {
        Pack<TI, 8> p;
        p.load(in + j);
        float x[8];
        p.get(x);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] *= f;
        Pack<TO, 8>::store(out + j, x);
    }
#pragma unroll 4
    for (int64_t j = whole + threadIdx.x; j < e1; j += kThreads) {
        Pack<TI, 1> p;
        p.load(in + j);
        float x[1];
        p.get(x);
        x[0] *= f;
        Pack<TO, 1>::store(out + j, x);
    }
}

// A factor below fp32's normal numbers has lost digits as an fp32 number, or is 0, while the results may well be normal (values of 3e38
// and a small max_norm): products in fp64.
constexpr float kLeastFactor = 1.17549435e-38f;
template <typename TI>
__device__ __forceinline__ void scale_chunk_wide(const TI *in, void *out, bool out16, double f, int64_t e0, int64_t e1)
{
    for (int64_t j = e0 + threadIdx.x; j < e1; j += kThreads) {
        Pack<TI, 1> p;
        p.load(in + j);
        float x[1];
        p.get(x);
        x[0] = (float)((double)x[0] * f);
        if (out16) Pack<__nv_bfloat16, 1>::store(reinterpret_cast<__nv_bfloat16 *>(out) + j, x);
        else Pack<float, 1>::store(reinterpret_cast<float *>(out) + j, x);
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const __grid_constant__ Table<N> t, const Args a)
{
    __shared__ double red[32];
    grid_dependents_may_launch();
    grid_dependency_wait();
    double sum = 0.0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(t, a.n, c), type = t.type[i];
        const int64_t e0 = (int64_t)(c - t.first[i]) * kChunk, e1 = min(e0 + (int64_t)kChunk, t.numel[i]);
        sum += type & 1 ? sum_chunk(reinterpret_cast<const __nv_bfloat16 *>(t.in[i]), e0, e1, type & 4)
                        : sum_chunk(reinterpret_cast<const float *>(t.in[i]), e0, e1, type & 4);
    }
    sum = block_sum<kThreads>(sum, red);
    if (threadIdx.x == 0) a.part[(size_t)a.launch * kMaxBlocks + blockIdx.x] = sum;
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
scale_kernel(const __grid_constant__ Table<N> t, const Args a)
{
    __shared__ double red[32];
    grid_dependents_may_launch();
    grid_dependency_wait();
    double sum = 0.0;
    for (int j = threadIdx.x; j < a.launches * kMaxBlocks; j += kThreads)
        if (j % kMaxBlocks < a.blocks) sum += a.part[j];
    sum = block_sum<kThreads>(sum, red);
    const double norm = sqrt(sum) * fabs((double)a.scale);
    double coef = norm > (double)a.max_norm ? (double)a.max_norm / norm : 1.0;
    const bool bad = !isfinite(norm);
    if (bad) coef = __longlong_as_double(0x7ff8000000000000ll);
    if (a.launch == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        a.norm[0] = (float)norm;
        a.norm[1] = (float)coef;
        if (bad && a.status) atomicOr(a.status, PPO_DEV_BAD_GRAD);
    }
    // (one more number in the threads' registers would cost a quarter of the blocks on an SM: 1667 us for 1632)
    __shared__ double factor;
    if (threadIdx.x == 0) factor = coef * (double)a.scale;
    __syncthreads();
    const float f = (float)factor;
    for (int c0 = blockIdx.x; c0 < a.chunks; c0 += gridDim.x) {
        const int c = a.chunks - 1 - c0;
        const int i = tensor_of(t, a.n, c);
        const int type = t.type[i];
        if ((type & 8) && f == 1.f) continue;
        const int64_t e0 = (int64_t)(c - t.first[i]) * kChunk, e1 = min(e0 + (int64_t)kChunk, t.numel[i]);
        const float *in32 = reinterpret_cast<const float *>(t.in[i]);
        const __nv_bfloat16 *in16 = reinterpret_cast<const __nv_bfloat16 *>(t.in[i]);
        float *out32 = reinterpret_cast<float *>(t.out[i]);
        __nv_bfloat16 *out16 = reinterpret_cast<__nv_bfloat16 *>(t.out[i]);
        if (fabsf(f) < kLeastFactor) {
            if (type & 1) scale_chunk_wide(in16, t.out[i], type & 2, factor, e0, e1);
            else scale_chunk_wide(in32, t.out[i], type & 2, factor, e0, e1);
            continue;
        }
        switch (type & 3) {
        case 0: scale_chunk(in32, out32, f, e0, e1, type & 4); break;
        case 1: scale_chunk(in16, out32, f, e0, e1, type & 4); break;
        case 2: scale_chunk(in32, out16, f, e0, e1, type & 4); break;
        default: scale_chunk(in16, out16, f, e0, e1, type & 4);
        }
    }
}

// ---------------------------------------------------------------- host side
constexpr int kSmall = 64, kLarge = 900;          // tensors of one launch

template <int N>
static int launch_group(bool scale, const void *const *in, void *const *out, const int64_t *numel, const int32_t *in_dtype,
                        const int32_t *out_dtype, int n, Args a, cudaStream_t s)
{
    Table<N> t = {};
    int64_t chunks = 0;
    a.n = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const int k = a.n++;
        t.in[k] = in[i];
        t.out[k] = out ? out[i] : const_cast<void *>(in[i]);
        t.numel[k] = numel[i];
        t.first[k] = (int32_t)chunks;
        const int32_t od = out ? out_dtype[i] : in_dtype[i];
        t.type[k] = (in_dtype[i] == PPO_BF16) | (od == PPO_BF16) << 1 |
                    (packs_fit(t.in[k], 8, in_dtype[i], 8) && packs_fit(t.out[k], 8, od, 8)) << 2 |
                    (t.in[k] == t.out[k]) << 3;
        chunks += (numel[i] + kChunk - 1) / kChunk;
        if (chunks >= ((int64_t)1 << 30)) return PPO_ERR_SHAPE;
    }
    a.chunks = (int)chunks;
    // (the first launch waits for all work before the call)
    if (scale || a.launch > 0) {
        PPO_RETURN_IF_CUDA(launch_dependent(scale ? scale_kernel<N> : norm_kernel<N>, dim3(a.blocks), dim3(kThreads), 0, s, t, a));
        return PPO_OK;
    }
    norm_kernel<N><<<a.blocks, kThreads, 0, s>>>(t, a);
    return launch_status();
}

struct Range {
    uintptr_t from, to;
    bool written;
};

// Whether a tensor that is written shares memory with another one, read or written: blocks of pass 2 would read what others have
// scaled. (Tensors that are only read may share theirs.) `ranges` holds 2 n.
static bool clash(int32_t n, const void *const *in, void *const *out, const int64_t *numel, const int32_t *in_dtype,
                  const int32_t *out_dtype, Range *ranges)
{
    int64_t count = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const uintptr_t from = reinterpret_cast<uintptr_t>(in[i]);
        const bool in_place = !out || out[i] == in[i];
        ranges[count++] = {from, from + (uintptr_t)numel[i] * (in_dtype[i] == PPO_F32 ? 4 : 2), in_place};
        if (in_place) continue;
        const uintptr_t to = reinterpret_cast<uintptr_t>(out[i]);
        ranges[count++] = {to, to + (uintptr_t)numel[i] * (out_dtype[i] == PPO_F32 ? 4 : 2), true};
    }
    std::sort(ranges, ranges + count, [](const Range &a, const Range &b) { return a.from < b.from; });
    uintptr_t end = 0, end_written = 0;                        // of the ranges so far, and of those that are written
    for (int64_t i = 0; i < count; ++i) {
        const Range r = ranges[i];
        if (r.from < (r.written ? end : end_written)) return true;
        end = std::max(end, r.to);
        if (r.written) end_written = std::max(end_written, r.to);
    }
    return false;
}

static int groups_of(int32_t n) { return n <= kSmall ? 1 : (n + kLarge - 1) / kLarge; }

}   // namespace clip
}   // namespace ppo

using namespace ppo;

extern "C" size_t ppo_grad_clip_scratch_bytes(int32_t n)
{
    return n <= 0 ? 0 : align256((size_t)clip::groups_of(n) * clip::kMaxBlocks * sizeof(double));
}

extern "C" int ppo_grad_clip(int32_t n, const void *const *in, const int64_t *numel, const int32_t *in_dtype,
                             void *const *out, const int32_t *out_dtype, float scale, float max_norm, float *norm,
                             void *workspace, void *scratch, void *stream)
{
    using namespace clip;
    if (n <= 0 || n > 1000000) return PPO_ERR_SHAPE;
    if (!finite_f(scale) || scale == 0.f || !(max_norm > 0.f)) return PPO_ERR_PARAM;
    if (!in || !numel || !in_dtype || !norm || !scratch || (out && !out_dtype)) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(scratch) % 256 || reinterpret_cast<uintptr_t>(workspace) % 256)
        return PPO_ERR_ALIGN;
    int64_t chunks = 0;
    for (int i = 0; i < n; ++i) {
        const int32_t od = out ? out_dtype[i] : in_dtype[i];
        if ((in_dtype[i] != PPO_F32 && in_dtype[i] != PPO_BF16) || (od != PPO_F32 && od != PPO_BF16)) return PPO_ERR_DTYPE;
        if (numel[i] < 0 || numel[i] >= ((int64_t)1 << 44)) return PPO_ERR_SHAPE;
        if (numel[i] == 0) continue;
        if (!in[i] || (out && !out[i])) return PPO_ERR_NULL;
        if (reinterpret_cast<uintptr_t>(in[i]) % (in_dtype[i] == PPO_F32 ? 4 : 2) ||
            (out && reinterpret_cast<uintptr_t>(out[i]) % (od == PPO_F32 ? 4 : 2)))
            return PPO_ERR_ALIGN;
        if (out && out[i] == in[i] && od != in_dtype[i]) return PPO_ERR_PARAM;
        chunks += (numel[i] + kChunk - 1) / kChunk;
    }
    {
        Range few[2 * kSmall], *many = n <= kSmall ? few : static_cast<Range *>(std::malloc((size_t)n * 2 * sizeof(Range)));
        if (!many) return (int)cudaErrorMemoryAllocation;
        const bool bad = clash(n, in, out, numel, in_dtype, out_dtype, many);
        if (many != few) std::free(many);
        if (bad) return PPO_ERR_PARAM;
    }
    int dev = 0, sms = 148;
    PPO_RETURN_IF_CUDA(cudaGetDevice(&dev));
    PPO_RETURN_IF_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    Args a = {};
    a.part = reinterpret_cast<double *>(scratch);
    a.launches = groups_of(n);
    a.scale = scale;
    a.max_norm = max_norm;
    a.norm = norm;
    a.status = workspace ? &ws_header(workspace)->status : nullptr;
    const int most = sms * kBlocksPerSm < kMaxBlocks ? sms * kBlocksPerSm : kMaxBlocks;
    a.blocks = chunks < 1 ? 1 : chunks < most ? (int)chunks : most;
    const int step = n <= kSmall ? kSmall : kLarge;
    for (int pass = 0; pass < 2; ++pass) {
        for (int g = 0; g < a.launches; ++g) {
            // the groups, too, in reverse order in the second pass
            a.launch = pass ? a.launches - 1 - g : g;
            const int i0 = a.launch * step, count = n - i0 < step ? n - i0 : step;
            const auto go = n <= kSmall ? launch_group<kSmall> : launch_group<kLarge>;
            const int rc = go(pass == 1, in + i0, out ? out + i0 : nullptr, numel + i0, in_dtype + i0, out_dtype ? out_dtype + i0 : nullptr,
                              count, a, s);
            if (rc) return rc;
        }
    }
    return PPO_OK;
}
