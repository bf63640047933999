// Eight consecutive values at a time, in 16-byte accesses: widened to fp32 when read, rounded once (nearest, ties to even) when written.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace zq {

template <typename T> struct Pack8;             // eight values rounded into one or two 16-byte stores
template <> struct Pack8<float> {
    static __device__ __forceinline__ void store(float* d, const float (&v)[8]) {
        reinterpret_cast<float4*>(d)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(d)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
};
template <> struct Pack8<__nv_bfloat16> {
    static __device__ __forceinline__ void store(__nv_bfloat16* d, const float (&v)[8]) {
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(d) = *reinterpret_cast<const uint4*>(h);
    }
};
template <> struct Pack8<__half> {
    static __device__ __forceinline__ void store(__half* d, const float (&v)[8]) {
        __half2 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(d) = *reinterpret_cast<const uint4*>(h);
    }
};

// the eight values as they lie in memory, and widened
template <typename T> struct Raw8 {
    uint4 w;
    __device__ __forceinline__ void load(const T* s) { w = __ldg(reinterpret_cast<const uint4*>(s)); }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
        const T* x = reinterpret_cast<const T*>(&w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(x[e]);
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* s) { a = __ldg(reinterpret_cast<const float4*>(s)); b = __ldg(reinterpret_cast<const float4*>(s) + 1); }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};

}  // namespace zq
