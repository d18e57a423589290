// Elements of the three types (fp32, bf16, fp16) in 16-byte vectors: loads, conversions to and from fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace adacomp {

__host__ __device__ __forceinline__ uint32_t type_size(int type) { return type == ADACOMP_F32 ? 4u : 2u; }
inline bool known_type(int type) { return type == ADACOMP_F32 || type == ADACOMP_BF16 || type == ADACOMP_F16; }

template <int TYPE> struct ElemOf;
template <> struct ElemOf<ADACOMP_F32> { using T = float; };
template <> struct ElemOf<ADACOMP_BF16> { using T = __nv_bfloat16; };
template <> struct ElemOf<ADACOMP_F16> { using T = __half; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// The two halves of a 32-bit word as fp32.
template <typename T> __device__ __forceinline__ float2 halves(uint32_t w);
template <> __device__ __forceinline__ float2 halves<__nv_bfloat16>(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 halves<__half>(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Read-only streaming load of an aligned 16-byte vector.
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// N elements (N * size a multiple of 16 bytes) between their packed form and fp32.
template <typename T, int N> struct Packed {
    static constexpr int kVecs = N * static_cast<int>(sizeof(T)) / 16;
    static_assert(kVecs * 16 == N * static_cast<int>(sizeof(T)), "whole 16-byte vectors");
    uint4 v[kVecs];

    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) v[i] = load16(reinterpret_cast<const char*>(p) + 16 * i);
    }
    __device__ __forceinline__ void store(T* p) const {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) reinterpret_cast<uint4*>(p)[i] = v[i];
    }
    __device__ __forceinline__ void unpack(float (&f)[N]) const {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) {
                    f[4 * i + j] = __uint_as_float(w[j]);
                } else {
                    const float2 h = halves<T>(w[j]);
                    f[8 * i + 2 * j] = h.x;
                    f[8 * i + 2 * j + 1] = h.y;
                }
            }
        }
    }
    __device__ __forceinline__ void pack(const float (&f)[N]) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(f[4 * i + j]);
                else w[j] = pack2<T>(f[8 * i + 2 * j], f[8 * i + 2 * j + 1]);
            }
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// Entries per vectorised item: 16 bytes of the narrower of the two types.
template <typename A, typename B> constexpr int kItemElems = sizeof(A) == 4 && sizeof(B) == 4 ? 4 : 8;

}  // namespace adacomp
