// Neighbouring elements as fp32: loads and stores of VEC of them, one access each (8: 16 bytes of bf16, 32 of fp32; 4: half of
// that; 1: single elements). An fp32 store in two halves would write every 32-byte sector twice.
#pragma once

#include "ppo_common.cuh"

namespace ppo {

__device__ __forceinline__ void unpack2(uint32_t w, float *x)
{
    x[0] = __uint_as_float(w << 16);
    x[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// load() keeps the bits as they came, so that loads in flight take no more registers than they bring; get() widens them.
// load_once(): of data that is not read again soon.
template <typename T, int VEC> struct Pack;

template <> struct Pack<float, 1> {
    float r;
    __device__ __forceinline__ void load(const float *p) { r = *p; }
    __device__ __forceinline__ void load_once(const float *p) { r = __ldcs(p); }
    __device__ __forceinline__ void zero() { r = 0.f; }
    __device__ __forceinline__ void get(float *x) const { x[0] = r; }
    __device__ __forceinline__ static void store(float *p, const float *x) { __stcs(p, x[0]); }
};
template <> struct Pack<float, 4> {
    float4 r;
    __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void load_once(const float *p) { r = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float *x) const { x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w; }
    __device__ __forceinline__ static void store(float *p, const float *x)
    {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(x[0], x[1], x[2], x[3]));
    }
};
template <> struct Pack<float, 8> {
    float r[8];
    __device__ __forceinline__ void load(const float *p)
    {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
                     : "l"(p) : "memory");
    }
    __device__ __forceinline__ void load_once(const float *p) { load(p); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = 0.f;
    }
    __device__ __forceinline__ void get(float *x) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r[e];
    }
    __device__ __forceinline__ static void store(float *p, const float *x)
    {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
    }
};
template <> struct Pack<__nv_bfloat16, 1> {
    __nv_bfloat16 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *p; }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { r = *p; }
    __device__ __forceinline__ void zero() { r = __ushort_as_bfloat16(0); }
    __device__ __forceinline__ void get(float *x) const { x[0] = __bfloat162float(r); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x) { *p = __float2bfloat16_rn(x[0]); }
};
template <> struct Pack<__nv_bfloat16, 4> {
    uint2 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { r = __ldcs(reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void zero() { r = make_uint2(0u, 0u); }
    __device__ __forceinline__ void get(float *x) const { unpack2(r.x, x); unpack2(r.y, x + 2); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x)
    {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])));
    }
};
template <> struct Pack<__nv_bfloat16, 8> {
    uint4 r;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { r = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { r = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void zero() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float *x) const { unpack2(r.x, x); unpack2(r.y, x + 2); unpack2(r.z, x + 4); unpack2(r.w, x + 6); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x)
    {
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])));
    }
};

// zeros over [p, p + bytes), any address and size that are multiples of 2, by a warp
__device__ __forceinline__ void zero_bytes(unsigned char *p, int64_t bytes)
{
    const int lane = threadIdx.x & 31;
    const int64_t head = min(bytes, (int64_t)(-reinterpret_cast<uintptr_t>(p) & 15u)), body = (bytes - head) & ~(int64_t)15;
    unsigned char *q = p + head;
#pragma unroll 4
    for (int64_t i = lane * 16; i < body; i += 512) __stcs(reinterpret_cast<uint4 *>(q + i), make_uint4(0u, 0u, 0u, 0u));
    if (lane * 2 < head) *reinterpret_cast<uint16_t *>(p + lane * 2) = 0;
    if (lane * 2 < bytes - head - body) *reinterpret_cast<uint16_t *>(q + body + lane * 2) = 0;
}

// whether packs of `vec` elements may be accessed at p and at every multiple of `pitch` elements from there
inline bool packs_fit(const void *p, int64_t pitch, int dtype, int vec)
{
    const int size = dtype == PPO_F32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(p) % (vec * size) == 0 && pitch % vec == 0;
}

}   // namespace ppo
