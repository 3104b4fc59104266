// Neighbouring elements as fp32: loads and stores of VEC of them, one access each (8: 16 bytes of bf16, 32 of fp32; 4: half of
// that; 1: single elements). An fp32 store in two halves would write every 32-byte sector twice.
#pragma once

#include "ppo_common.cuh"

namespace ppo {

template <typename T, int VEC> struct Pack;

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

template <> struct Pack<float, 1> {
    float v[1];
    __device__ __forceinline__ void load(const float *p) { v[0] = *p; }
    __device__ __forceinline__ void load_once(const float *p) { v[0] = __ldcs(p); }
    __device__ __forceinline__ static void store(float *p, const float *x) { __stcs(p, x[0]); }
};
template <> struct Pack<float, 4> {
    float v[4];
    __device__ __forceinline__ void set(const float4 &a) { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
    __device__ __forceinline__ void load(const float *p) { set(*reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void load_once(const float *p) { set(__ldcs(reinterpret_cast<const float4 *>(p))); }
    __device__ __forceinline__ static void store(float *p, const float *x)
    {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(x[0], x[1], x[2], x[3]));
    }
};
template <> struct Pack<float, 8> {
    float v[8];
    __device__ __forceinline__ void load(const float *p)
    {
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "l"(p) : "memory");
    }
    __device__ __forceinline__ void load_once(const float *p) { load(p); }
    __device__ __forceinline__ static void store(float *p, const float *x)
    {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
    }
};
template <> struct Pack<__nv_bfloat16, 1> {
    float v[1];
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v[0] = __bfloat162float(*p); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { v[0] = __bfloat162float(*p); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x) { *p = __float2bfloat16_rn(x[0]); }
};
template <> struct Pack<__nv_bfloat16, 4> {
    float v[4];
    __device__ __forceinline__ void set(const uint2 &a) { unpack2(a.x, v); unpack2(a.y, v + 2); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { set(*reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { set(__ldcs(reinterpret_cast<const uint2 *>(p))); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x)
    {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])));
    }
};
template <> struct Pack<__nv_bfloat16, 8> {
    float v[8];
    __device__ __forceinline__ void set(const uint4 &a) { unpack2(a.x, v); unpack2(a.y, v + 2); unpack2(a.z, v + 4); unpack2(a.w, v + 6); }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { set(*reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16 *p) { set(__ldcs(reinterpret_cast<const uint4 *>(p))); }
    __device__ __forceinline__ static void store(__nv_bfloat16 *p, const float *x)
    {
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])));
    }
};

// whether packs of `vec` elements may be accessed at p and at every multiple of `pitch` elements from there
inline bool packs_fit(const void *p, int64_t pitch, int dtype, int vec)
{
    const int size = dtype == PPO_F32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(p) % (vec * size) == 0 && pitch % vec == 0;
}

}   // namespace ppo
