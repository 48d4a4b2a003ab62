// Element types of the operators beside the attention (16-bit and fp32 rows, fp32 arithmetic): loads and stores of one
// element and of eight neighbouring ones with 16-byte accesses.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"

namespace regenvc {

enum { kTypeBf16 = 0, kTypeF16 = 1, kTypeF32 = 2 };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f32(float v, float& o) { o = v; }
__device__ __forceinline__ void from_f32(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f32(float v, __half& o) { o = __float2half_rn(v); }

// Eight elements as they lie in memory: one 16-byte word of a 16-bit type, two of fp32.
template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = reinterpret_cast<const uint4*>(p)[i];
    return r;
}
template <typename T>
__device__ __forceinline__ void store_raw8(T* p, const Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) reinterpret_cast<uint4*>(p)[i] = r.w[i];
}
// The same for data that a kernel touches once (first to leave the caches).
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8_once(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.w[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
__device__ __forceinline__ void widen2(uint32_t w, float& a, float& b, const __nv_bfloat16*) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void widen2(uint32_t w, float& a, float& b, const __half*) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[4 * i + 0] = __uint_as_float(r.w[i].x);
            v[4 * i + 1] = __uint_as_float(r.w[i].y);
            v[4 * i + 2] = __uint_as_float(r.w[i].z);
            v[4 * i + 3] = __uint_as_float(r.w[i].w);
        }
    } else {
        const T* tag = nullptr;
        widen2(r.w[0].x, v[0], v[1], tag);
        widen2(r.w[0].y, v[2], v[3], tag);
        widen2(r.w[0].z, v[4], v[5], tag);
        widen2(r.w[0].w, v[6], v[7], tag);
    }
}
__device__ __forceinline__ uint32_t narrow2(float a, float b, const __nv_bfloat16*) { return pack_bf16x2(a, b); }
__device__ __forceinline__ uint32_t narrow2(float a, float b, const __half*) { return pack_f16x2(a, b); }
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            reinterpret_cast<float4*>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    } else {
        const T* tag = nullptr;
        *reinterpret_cast<uint4*>(p) = make_uint4(narrow2(v[0], v[1], tag), narrow2(v[2], v[3], tag),
                                                  narrow2(v[4], v[5], tag), narrow2(v[6], v[7], tag));
    }
}

template <typename T>
__device__ __forceinline__ void store8_once(T* p, const float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            __stcs(reinterpret_cast<float4*>(p) + i, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
    } else {
        const T* tag = nullptr;
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(narrow2(v[0], v[1], tag), narrow2(v[2], v[3], tag),
                                                       narrow2(v[4], v[5], tag), narrow2(v[6], v[7], tag)));
    }
}

}  // namespace regenvc
