// Elements of the three types (fp32, bf16, fp16) in 16-byte vectors: loads, conversions to and from fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace adacomp {

__host__ __device__ __forceinline__ uint32_t type_size(int type) { return type == ADACOMP_F32 ? 4u : 2u; }
inline bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool known_type(int type) { return type == ADACOMP_F32 || type == ADACOMP_BF16 || type == ADACOMP_F16; }

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

// How a kernel's loads and stores want to be kept in L2: as usual, or given up first.
__device__ __forceinline__ uint64_t l2_policy(bool give_up_first) {
    uint64_t p;
    if (give_up_first) asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    else asm("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
}

__device__ __forceinline__ uint4 load16(const void* p, uint64_t policy) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p), "l"(policy));
    return v;
}
__device__ __forceinline__ void store16(void* p, const uint4& v, uint64_t policy) {
    asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;"
                 :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "l"(policy) : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
// 32-byte vectors, one instruction each (32-byte aligned).
__device__ __forceinline__ void load32(const void* p, uint4& a, uint4& b, uint64_t policy) {
    asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8], %9;"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p), "l"(policy));
}
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b, uint64_t policy) {
    asm volatile("st.global.L2::cache_hint.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8}, %9;"
                 :: "l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w), "l"(policy) : "memory");
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
    // The same for items on their own grid: 32-byte ones in one instruction.
    __device__ __forceinline__ void load_whole(const T* p, uint64_t policy) {
        if constexpr (kVecs == 2) load32(p, v[0], v[1], policy);
        else v[0] = load16(p, policy);
    }
    __device__ __forceinline__ void store_whole(T* p, uint64_t policy) const {
        if constexpr (kVecs == 2) store32(p, v[0], v[1], policy);
        else store16(p, v[0], policy);
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

// A single entry, with the same interface.
template <typename T> struct Packed<T, 1> {
    static constexpr int kVecs = 1;
    uint4 v[1];                     // unused
    T x;
    __device__ __forceinline__ void load(const T* p) { x = __ldg(p); }
    __device__ __forceinline__ void store(T* p) const { *p = x; }
    __device__ __forceinline__ void unpack(float (&f)[1]) const { f[0] = to_float(x); }
    __device__ __forceinline__ void pack(const float (&f)[1]) { x = from_float<T>(f[0]); }
};

// Entries [e, e + N) of a tensor of n entries at `in` that does not sit on the 16-byte grid there: the vectors around them,
// shifted into place, if all of those lie inside the tensor.
template <typename A, int N>
__device__ __forceinline__ Packed<A, N> load_shifted(const A* in, int64_t e, uint64_t n) {
    constexpr int kVecs = Packed<A, N>::kVecs, kWords = 4 * (kVecs + 1);
    const uintptr_t a = reinterpret_cast<uintptr_t>(in + e), lo = a & ~static_cast<uintptr_t>(15);
    const uintptr_t first = reinterpret_cast<uintptr_t>(in), end = first + n * sizeof(A);
    Packed<A, N> p;
    if (lo >= first && lo + 16 * (kVecs + 1) <= end) {
        uint32_t w[kWords];
#pragma unroll
        for (int i = 0; i <= kVecs; ++i) {
            const uint4 q = __ldg(reinterpret_cast<const uint4*>(lo + 16 * i));     // the neighbour reads it too
            w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
        }
        if (a & 8)
#pragma unroll
            for (int i = 0; i + 2 < kWords; ++i) w[i] = w[i + 2];
        if (a & 4)
#pragma unroll
            for (int i = 0; i + 1 < kWords; ++i) w[i] = w[i + 1];
        if (a & 2)
#pragma unroll
            for (int i = 0; i + 1 < kWords; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
#pragma unroll
        for (int i = 0; i < kVecs; ++i) p.v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    } else {
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = to_float(in[e + j]);
        p.pack(f);
    }
    return p;
}

// Entries per vectorised item: 16 bytes of the narrower of the two types.
template <typename A, typename B> constexpr int kItemElems = sizeof(A) == 4 && sizeof(B) == 4 ? 4 : 8;

}  // namespace adacomp
