// Quantisation of a matrix to e4m3 with one fp32 scale per 1 x 128 or 128 x 128 block (ppo_fp8_quantize):
//     a = max(|x| over the block, 2^-100),  scale = a / 448,  q = e4m3(x * (448 / a))   (ties to even)
// y [R, C] is x or its transpose, blocks run along C. One read and one write of the matrix: bound by HBM bytes.
// A thread always owns 8 consecutive elements of x (16 bytes of bf16, 32 of fp32), so that 16 threads span a block's
// 128 columns, and every row of q it writes goes out in runs of 128 bytes.
//   rows kernel  1 x 128 blocks of x itself: the maximum is a shuffle over 16 lanes.
//   tile kernel  128 x 128 tile per block of 256 threads, each holding 8 x 8 elements in registers: 128 x 128
//                blocks, and every transposed case (q is turned in shared memory, 8 bytes at a time, XOR-placed so
//                that neither side has bank conflicts).
// A block with a NaN or an infinity has scale NaN and q NaN throughout.
// [4096, 50304] bf16, transposed, 128 x 128: 102 us = 6.0 TB/s; 27136 x 4096 rows: 55 us = 6.1 TB/s. Magnitudes are compared in the
// storage type, two to an instruction, and a warp divides once for all its rows: with integer maxima of widened values and
// two divisions per 8 elements the arithmetic took twice as long as the bytes (219 and 101 us).
#include <cuda_fp8.h>
#include <string.h>

#include "ppo_rows.cuh"

namespace ppo {
namespace quant {

constexpr int kThreads = 256;
constexpr float kMax = 448.f;
constexpr float kMinAmax = 7.8886090522101181e-31f;   // 2^-100: keeps 448 / a finite

// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// Eight consecutive elements as they lie in memory, and maxima of their magnitudes: in the storage type for bf16 (two per
// instruction), column by column or over all.
template <typename T> struct Eight;

template <> struct Eight<float> {
    uint4 w[2];
    struct Max {
        float m;
        __device__ __forceinline__ void init() { m = 0.f; }
        __device__ __forceinline__ void add(const Eight &x)
        {
            float y[8];
            x.get(y);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(y[e]));
        }
        __device__ __forceinline__ float value() const { return m; }
    };
    struct MaxByColumn {
        float m[8];
        __device__ __forceinline__ void init()
        {
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = 0.f;
        }
        __device__ __forceinline__ void add(const Eight &x)
        {
            float y[8];
            x.get(y);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = max_nan(m[e], fabsf(y[e]));
        }
        __device__ __forceinline__ float value(int e) const { return m[e]; }
    };
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const float *f = reinterpret_cast<const float *>(w);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = f[e];
    }
};

template <> struct Eight<__nv_bfloat16> {
    uint4 w[1];
    static __device__ __forceinline__ __nv_bfloat162 as2(uint32_t v) { return *reinterpret_cast<__nv_bfloat162 *>(&v); }
    struct MaxByColumn {
        __nv_bfloat162 m[4];
        __device__ __forceinline__ void init()
        {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = as2(0u);
        }
        __device__ __forceinline__ void add(const Eight &x)
        {
            m[0] = __hmax2_nan(m[0], __habs2(as2(x.w[0].x)));
            m[1] = __hmax2_nan(m[1], __habs2(as2(x.w[0].y)));
            m[2] = __hmax2_nan(m[2], __habs2(as2(x.w[0].z)));
            m[3] = __hmax2_nan(m[3], __habs2(as2(x.w[0].w)));
        }
        __device__ __forceinline__ float value(int e) const
        {
            const uint32_t bits = *reinterpret_cast<const uint32_t *>(&m[e >> 1]);
            return __uint_as_float((e & 1) ? bits & 0xffff0000u : bits << 16);
        }
    };
    struct Max {
        __nv_bfloat162 m;
        __device__ __forceinline__ void init() { m = as2(0u); }
        __device__ __forceinline__ void add(const Eight &x)
        {
            const __nv_bfloat162 a = __hmax2_nan(__habs2(as2(x.w[0].x)), __habs2(as2(x.w[0].y)));
            const __nv_bfloat162 b = __hmax2_nan(__habs2(as2(x.w[0].z)), __habs2(as2(x.w[0].w)));
            m = __hmax2_nan(m, __hmax2_nan(a, b));
        }
        __device__ __forceinline__ float value() const
        {
            const uint32_t bits = *reinterpret_cast<const uint32_t *>(&m);
            return max_nan(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u));
        }
    };
    __device__ __forceinline__ void get(float (&x)[8]) const { Pack<__nv_bfloat16>::unpack_raw(w[0], x); }
};

template <typename T>
__device__ __forceinline__ void load8(const T *src, int valid, bool vec, Eight<T> &x)
{
    if (vec && valid >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / Pack<T>::N; ++h) x.w[h] = ld_stream(reinterpret_cast<const uint4 *>(src) + h);
    } else {
        T y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = e < valid ? src[e] : T(0.f);
        memcpy(x.w, y, sizeof(y));
    }
}

struct Scale {
    float s, r;     // scale, and what x is multiplied with
};

__device__ __forceinline__ Scale scale_of(float amax /* NaN when one was among the magnitudes */)
{
    Scale o;
    const float a = fmaxf(amax, kMinAmax);
    o.s = __fdiv_rn(a, kMax);
    o.r = __fdiv_rn(kMax, a);
    if (!(amax <= 3.4028234664e38f)) o.s = o.r = __uint_as_float(0x7fffffffu);
    return o;
}

__device__ __forceinline__ uint32_t q2(float lo, float hi)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
template <typename T>
__device__ __forceinline__ uint2 q8(const Eight<T> &v, float r)
{
    float x[8];
    v.get(x);
    return make_uint2(q2(x[0] * r, x[1] * r) | (q2(x[2] * r, x[3] * r) << 16),
                      q2(x[4] * r, x[5] * r) | (q2(x[6] * r, x[7] * r) << 16));
}

__device__ __forceinline__ void store8(uint8_t *dst, uint2 v, int valid)
{
    if (valid >= 8) {
        *reinterpret_cast<uint2 *>(dst) = v;
    } else {
        for (int e = 0; e < valid; ++e) dst[e] = (uint8_t)((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
    }
}

struct Args {
    const void *x;
    int R, C;               // of y
    int64_t x_stride, q_stride;
    uint8_t *q;
    float *scales;
    int vec;                // 16-byte loads of x are aligned
    int tiles_r, tiles_c;
};

// 32 rows x 256 columns per block: a warp takes 4 rows, a lane 8 columns
template <typename T>
__global__ void __launch_bounds__(kThreads)
rows_kernel(const Args a)
{
    __shared__ float sc[2][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tc = blockIdx.x % a.tiles_c, tr = blockIdx.x / a.tiles_c;
    const int c = tc * 256 + lane * 8, r0 = tr * 32;
    const T *x = reinterpret_cast<const T *>(a.x);
    const int valid = min(8, a.C - c);
    Eight<T> v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + i * 8 + warp;
        load8<T>(x + (int64_t)r * a.x_stride + c, r < a.R ? valid : 0, a.vec, v[i]);
    }
    // the maximum over the block's 16 lanes, of four rows; lane i then divides for row i
    float mine = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        typename Eight<T>::Max mx;
        mx.init();
        mx.add(v[i]);
        float m = mx.value();
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, off));
        if ((lane & 3) == i) mine = m;
    }
    const Scale s = scale_of(mine);
    if ((lane & 15) < 4) sc[lane >> 4][(lane & 3) * 8 + warp] = s.s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + i * 8 + warp;
        const float ri = __shfl_sync(0xffffffffu, s.r, (lane & 16) + i);
        if (r < a.R) store8(a.q + (int64_t)r * a.q_stride + c, q8(v[i], ri), valid);
    }
    __syncthreads();
    const int kb = tc * 2 + warp, r = r0 + lane;       // scales [ceil(C/128), R]
    if (warp < 2 && kb * 128 < a.C && r < a.R) a.scales[(int64_t)kb * a.R + r] = sc[warp][lane];
}

// BLOCK: one scale per 128 x 128; else one per row of y and 128 columns (transposed inputs only)
template <typename T, bool TRANS, bool BLOCK>
__global__ void __launch_bounds__(kThreads)
tile_kernel(const Args a)
{
    static_assert(TRANS || BLOCK, "the rows kernel does the rest");
    __shared__ uint2 turn[TRANS ? 128 * 16 : 1];
    __shared__ float red[BLOCK ? 8 : 16 * 128];
    const int tid = threadIdx.x;
    // neighbouring blocks take neighbouring tiles along the contiguous direction of x
    const int tr = TRANS ? blockIdx.x % a.tiles_r : blockIdx.x / a.tiles_c;
    const int tc = TRANS ? blockIdx.x / a.tiles_r : blockIdx.x % a.tiles_c;
    const int r0 = tr * 128, c0 = tc * 128;
    const T *x = reinterpret_cast<const T *>(a.x);
    const int g = tid & 15, h = tid >> 4;
    // TRANS: x rows c0 + 8 h + i, columns (= rows of y) r0 + 8 g ..; else x rows r0 + 16 i + h, columns c0 + 8 g ..
    Eight<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int xr = TRANS ? c0 + h * 8 + i : r0 + i * 16 + h, xc = (TRANS ? r0 : c0) + g * 8;
        const int rows = TRANS ? a.C : a.R, cols = TRANS ? a.R : a.C;
        load8<T>(x + (int64_t)xr * a.x_stride + xc, xr < rows ? min(8, cols - xc) : 0, a.vec, v[i]);
    }
    float r8[8];
    if (BLOCK) {
        typename Eight<T>::Max mx;
        mx.init();
#pragma unroll
        for (int i = 0; i < 8; ++i) mx.add(v[i]);
        float m = mx.value();
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, off));
        if ((tid & 31) == 0) red[tid >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) m = max_nan(m, red[w]);
        const Scale s = scale_of(m);
        if (tid == 0) a.scales[(int64_t)tr * a.tiles_c + tc] = s.s;
#pragma unroll
        for (int e = 0; e < 8; ++e) r8[e] = s.r;
    } else {
        typename Eight<T>::MaxByColumn mx;
        mx.init();
#pragma unroll
        for (int i = 0; i < 8; ++i) mx.add(v[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) red[h * 128 + g * 8 + e] = mx.value(e);
        __syncthreads();
        if (tid < 128) {
            float m = 0.f;
#pragma unroll
            for (int w = 0; w < 16; ++w) m = max_nan(m, red[w * 128 + tid]);
            const Scale s = scale_of(m);
            red[tid] = s.r;                                 // (row 0 of this column has been read by this thread only)
            if (r0 + tid < a.R) a.scales[(int64_t)tc * a.R + r0 + tid] = s.s;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) r8[e] = red[g * 8 + e];
    }
    if (TRANS) {
        // two rows of x at a time: their columns' values go into two neighbouring bytes of a row of q
        uint32_t out[8][4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float x0[8], x1[8];
            v[i].get(x0);
            v[i + 1].get(x1);
#pragma unroll
            for (int e = 0; e < 8; ++e) out[e][i >> 1] = q2(x0[e] * r8[e], x1[e] * r8[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            turn[(g * 8 + e) * 16 + (h ^ g)] = make_uint2(out[e][0] | (out[e][1] << 16), out[e][2] | (out[e][3] << 16));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 16 + h, c = c0 + g * 8;
            if (r0 + r < a.R) store8(a.q + (int64_t)(r0 + r) * a.q_stride + c, turn[r * 16 + (g ^ (r >> 3))], min(8, a.C - c));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + i * 16 + h, c = c0 + g * 8;
            if (r < a.R) store8(a.q + (int64_t)r * a.q_stride + c, q8(v[i], r8[0]), min(8, a.C - c));
        }
    }
}

template <typename T>
static int launch(Args a, int block_rows, bool trans, cudaStream_t s)
{
    a.vec = aligned16(a.x) && (a.x_stride * (int64_t)sizeof(T)) % 16 == 0;
    const bool rows = block_rows == 1 && !trans;
    a.tiles_r = rows ? (a.R + 31) / 32 : (a.R + 127) / 128;
    a.tiles_c = rows ? (a.C + 255) / 256 : (a.C + 127) / 128;
    const int64_t blocks = (int64_t)a.tiles_r * a.tiles_c;
    if (blocks >= ((int64_t)1 << 31)) return PPO_ERR_SHAPE;
    const unsigned grid = (unsigned)blocks;
    if (rows) rows_kernel<T><<<grid, kThreads, 0, s>>>(a);
    else if (!trans) tile_kernel<T, false, true><<<grid, kThreads, 0, s>>>(a);
    else if (block_rows == 1) tile_kernel<T, true, false><<<grid, kThreads, 0, s>>>(a);
    else tile_kernel<T, true, true><<<grid, kThreads, 0, s>>>(a);
    return launch_status();
}

}   // namespace quant
}   // namespace ppo

using namespace ppo;

extern "C" int ppo_fp8_quantize(const void *x, int dtype, int64_t R, int64_t C, int64_t x_stride, int transpose,
                                int block_rows, void *q, int64_t q_stride, float *scales, void *stream)
{
    if (dtype != PPO_F32 && dtype != PPO_BF16) return PPO_ERR_DTYPE;
    const int64_t limit = ((int64_t)1 << 31) - 512;
    if (R < 0 || C <= 0 || R >= limit || C >= limit || x_stride < (transpose ? R : C) || q_stride < C || q_stride % 16)
        return PPO_ERR_SHAPE;
    if (block_rows != 1 && block_rows != 128) return PPO_ERR_PARAM;
    if (R == 0) return PPO_OK;
    if (!x || !q || !scales) return PPO_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(x) % (dtype == PPO_F32 ? 4 : 2) || !aligned16(q)) return PPO_ERR_ALIGN;
    quant::Args a = {};
    a.x = x;
    a.R = (int)R;
    a.C = (int)C;
    a.x_stride = x_stride;
    a.q = reinterpret_cast<uint8_t *>(q);
    a.q_stride = q_stride;
    a.scales = scales;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return dtype == PPO_F32 ? quant::launch<float>(a, block_rows, transpose != 0, s)
                            : quant::launch<__nv_bfloat16>(a, block_rows, transpose != 0, s);
}
