// Norm over many gradients and their clipping (ppo_grad_clip):
//     norm = |scale| * sqrt(sum over all tensors and elements of x^2),   coef = min(1, max_norm / norm),
//     out  = x * (scale * coef)
// Bound by memory: every tensor is read for the norm and again for the result, which cannot start before the norm is known.
//
// Two launches. Both walk the tensors in chunks of 32 K elements, chunk c by block c mod grid, so that a list of a few large
// and many small tensors is shared out evenly. Pass 1 leaves one fp64 sum per block; every block of pass 2 adds those up in
// the same order (no atomics: the norm does not depend on timing) and scales its chunks in reverse order, the last ones of
// pass 1 first, which are still in L2. Where nothing changes (in place, scale * coef = 1) pass 2 ends there.
//
// Squares are fp32 and summed eight at a time before they go to fp64 (a conversion per element would bound the pass: 16 per
// clock and SM). Eight squares that overflow, or that are small enough to lose digits, are taken again in fp64.
#include "ppo_common.cuh"

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
    uint8_t type[N];                              // bit 0: bf16 in, bit 1: bf16 out, bit 2: 16-byte accesses, bit 3: in place
};

struct Args {
    int n, chunks;                                // of this launch
    double *part;                                 // [launches][kMaxBlocks]
    int launch, launches, blocks;                 // partial sums: `blocks` of each launch
    float scale, max_norm;
    float *norm;                                  // [2] norm, coef
    int *status;
};

__device__ __forceinline__ float up(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xffff0000u : w << 16); }

__device__ __forceinline__ void load8(const void *p, bool bf16, float *x)
{
    if (bf16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = up(w[j >> 1], j & 1);
    } else {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

__device__ __forceinline__ float load1(const void *p, bool bf16, int64_t i)
{
    return bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i]) : reinterpret_cast<const float *>(p)[i];
}

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

template <int N>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const __grid_constant__ Table<N> t, const Args a)
{
    __shared__ double red[32];
    double sum = 0.0;
    for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(t, a.n, c);
        const bool bf16 = t.type[i] & 1;
        const int64_t e0 = (int64_t)(c - t.first[i]) * kChunk, e1 = min(e0 + (int64_t)kChunk, t.numel[i]);
        const unsigned char *in = reinterpret_cast<const unsigned char *>(t.in[i]);
        int64_t e = e0;
        if (t.type[i] & 4) {
            const int64_t whole = e0 + ((e1 - e0) & ~7ll);
#pragma unroll 4
            for (int64_t j = e0 + threadIdx.x * 8; j < whole; j += kThreads * 8) {
                float x[8];
                load8(in + j * (bf16 ? 2 : 4), bf16, x);
                sum += squares<8>(x);
            }
            e = whole;
        }
#pragma unroll 4
        for (int64_t j = e + threadIdx.x; j < e1; j += kThreads) {
            const float x = load1(in, bf16, j);
            sum += squares<1>(&x);
        }
    }
    sum = block_sum<kThreads>(sum, red);
    if (threadIdx.x == 0) a.part[(size_t)a.launch * kMaxBlocks + blockIdx.x] = sum;
}

template <int N>
__global__ void __launch_bounds__(kThreads)
scale_kernel(const __grid_constant__ Table<N> t, const Args a)
{
    __shared__ double red[32];
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
    const float f = (float)(coef * (double)a.scale);
    for (int c0 = blockIdx.x; c0 < a.chunks; c0 += gridDim.x) {
        const int c = a.chunks - 1 - c0;
        const int i = tensor_of(t, a.n, c);
        const int type = t.type[i];
        if ((type & 8) && f == 1.f) continue;
        const bool in16 = type & 1, out16 = type & 2;
        const int64_t e0 = (int64_t)(c - t.first[i]) * kChunk, e1 = min(e0 + (int64_t)kChunk, t.numel[i]);
        const unsigned char *in = reinterpret_cast<const unsigned char *>(t.in[i]);
        unsigned char *out = reinterpret_cast<unsigned char *>(t.out[i]);
        int64_t e = e0;
        if (type & 4) {
            const int64_t whole = e0 + ((e1 - e0) & ~7ll);
#pragma unroll 2
            for (int64_t j = e0 + threadIdx.x * 8; j < whole; j += kThreads * 8) {
                float x[8];
                load8(in + j * (in16 ? 2 : 4), in16, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] *= f;
                if (out16) {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
                        w[k] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                    __stcs(reinterpret_cast<uint4 *>(out + j * 2), make_uint4(w[0], w[1], w[2], w[3]));
                } else {
                    __stcs(reinterpret_cast<float4 *>(out + j * 4), make_float4(x[0], x[1], x[2], x[3]));
                    __stcs(reinterpret_cast<float4 *>(out + j * 4) + 1, make_float4(x[4], x[5], x[6], x[7]));
                }
            }
            e = whole;
        }
        for (int64_t j = e + threadIdx.x; j < e1; j += kThreads) {
            const float x = load1(in, in16, j) * f;
            if (out16) reinterpret_cast<__nv_bfloat16 *>(out)[j] = __float2bfloat16_rn(x);
            else reinterpret_cast<float *>(out)[j] = x;
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
                    ((reinterpret_cast<uintptr_t>(t.in[k]) | reinterpret_cast<uintptr_t>(t.out[k])) % 16 == 0) << 2 |
                    (t.in[k] == t.out[k]) << 3;
        chunks += (numel[i] + kChunk - 1) / kChunk;
        if (chunks >= ((int64_t)1 << 30)) return PPO_ERR_SHAPE;
    }
    a.chunks = (int)chunks;
    if (scale) scale_kernel<N><<<a.blocks, kThreads, 0, s>>>(t, a);
    else norm_kernel<N><<<a.blocks, kThreads, 0, s>>>(t, a);
    return launch_status();
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
    if (reinterpret_cast<uintptr_t>(norm) % 4 || reinterpret_cast<uintptr_t>(scratch) % 256) return PPO_ERR_ALIGN;
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
