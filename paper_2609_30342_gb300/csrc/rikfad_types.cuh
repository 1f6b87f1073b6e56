// rikfad_types.cuh -- float32, bfloat16 and float16 elements as float32, alone
// and eight at a time, for the operators beside the optimiser step.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace rikfad {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// Rounds to nearest even; a float16 beyond its range becomes infinite.
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Eight elements as loaded: 16 bytes of a 16-bit type, 32 of float32.
template <typename T> struct Raw8 {
    uint4 w;
};
template <> struct Raw8<float> {
    float4 a, b;
};

// The two elements of a 32-bit word.
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);          // exact: a bfloat16 is a float32's high half
    hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

template <typename T> __device__ __forceinline__ void unpack8(const Raw8<T> &r, float (&v)[8])
{
    unpack2(r.w.x, v[0], v[1], T());
    unpack2(r.w.y, v[2], v[3], T());
    unpack2(r.w.z, v[4], v[5], T());
    unpack2(r.w.w, v[6], v[7], T());
}
__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&v)[8])
{
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}

template <typename T> __device__ __forceinline__ Raw8<T> pack8(const float (&v)[8], T)
{
    Raw8<T> r;
    r.w = make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
    return r;
}
__device__ __forceinline__ Raw8<float> pack8(const float (&v)[8], float)
{
    return {make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7])};
}

// Loads and stores of eight elements from 16-byte aligned addresses: plain,
// and streaming (touched once).
template <typename T> __device__ __forceinline__ Raw8<T> load_raw8(const T *p)
{
    return {*reinterpret_cast<const uint4 *>(p)};
}
template <> __device__ __forceinline__ Raw8<float> load_raw8<float>(const float *p)
{
    return {reinterpret_cast<const float4 *>(p)[0], reinterpret_cast<const float4 *>(p)[1]};
}
template <typename T> __device__ __forceinline__ Raw8<T> load_raw8_cs(const T *p)
{
    return {__ldcs(reinterpret_cast<const uint4 *>(p))};
}
template <> __device__ __forceinline__ Raw8<float> load_raw8_cs<float>(const float *p)
{
    return {__ldcs(reinterpret_cast<const float4 *>(p)), __ldcs(reinterpret_cast<const float4 *>(p) + 1)};
}
template <typename T> __device__ __forceinline__ void store_raw8_cs(T *p, const Raw8<T> &r)
{
    __stcs(reinterpret_cast<uint4 *>(p), r.w);
}
template <> __device__ __forceinline__ void store_raw8_cs<float>(float *p, const Raw8<float> &r)
{
    __stcs(reinterpret_cast<float4 *>(p), r.a);
    __stcs(reinterpret_cast<float4 *>(p) + 1, r.b);
}

}  // namespace rikfad
