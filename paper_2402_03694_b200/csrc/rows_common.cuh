// Pieces shared by the kernels that work on rows of bf16, fp16 or fp32 (mx4.cu, experts.cu): element types, 16-byte
// vectors of elements, a host-side guard of the current device.
#pragma once
#include <cuda_fp16.h>
#include "common.cuh"

namespace sfrow {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N consecutive elements of T: 16-byte accesses where ALIGNED, else one access per element
template <typename T, int N, bool ALIGNED>
__device__ __forceinline__ void load_f32(const T* __restrict__ p, float (&x)[N]) {
    if constexpr (ALIGNED) {
        static_assert((N * sizeof(T)) % 16 == 0, "whole 16-byte pieces");
        union { uint4 q[N * sizeof(T) / 16]; T e[N]; } u;
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); i++) u.q[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = to_f32(u.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = to_f32(p[i]);
    }
}
template <typename T, int N, bool ALIGNED>
__device__ __forceinline__ void store_f32(T* __restrict__ p, const float (&x)[N]) {
    if constexpr (ALIGNED) {
        union { uint4 q[N * sizeof(T) / 16]; T e[N]; } u;
#pragma unroll
        for (int i = 0; i < N; i++) u.e[i] = from_f32<T>(x[i]);
#pragma unroll
        for (int i = 0; i < (int)(N * sizeof(T) / 16); i++) reinterpret_cast<uint4*>(p)[i] = u.q[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) p[i] = from_f32<T>(x[i]);
    }
}

// N elements as one access of N * sizeof(T) = 2, 4 or 16 bytes (p on a boundary of as many)
template <int BYTES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<16> { typedef uint4 type; };
template <typename T, int N> __device__ __forceinline__ void load_word(const T* __restrict__ p, float (&x)[N]) {
    typedef typename Word<N * sizeof(T)>::type W;
    union { W w; T e[N]; } u;
    u.w = __ldg(reinterpret_cast<const W*>(p));
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = to_f32(u.e[i]);
}
template <typename T, int N> __device__ __forceinline__ void store_word(T* __restrict__ p, const float (&x)[N]) {
    typedef typename Word<N * sizeof(T)>::type W;
    union { W w; T e[N]; } u;
#pragma unroll
    for (int i = 0; i < N; i++) u.e[i] = from_f32<T>(x[i]);
    *reinterpret_cast<W*>(p) = u.w;
}

// N elements as whole 32-byte accesses (p on a 32-byte boundary): a lane that has 32 bytes or more of a row to itself then moves whole
// sectors, where 16-byte stores would send every sector twice
template <typename T, int N>
__device__ __forceinline__ void load_sectors(const T* __restrict__ p, float (&x)[N]) {
    static_assert((N * sizeof(T)) % 32 == 0, "whole sectors");
    union { uint32_t w[N * sizeof(T) / 4]; T e[N]; } u;
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 32); i++)
        asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(u.w[8 * i]), "=r"(u.w[8 * i + 1]), "=r"(u.w[8 * i + 2]), "=r"(u.w[8 * i + 3]), "=r"(u.w[8 * i + 4]), "=r"(u.w[8 * i + 5]),
                       "=r"(u.w[8 * i + 6]), "=r"(u.w[8 * i + 7]) : "l"(reinterpret_cast<const char*>(p) + 32 * i));
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = to_f32(u.e[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_sectors(T* __restrict__ p, const float (&x)[N]) {
    static_assert((N * sizeof(T)) % 32 == 0, "whole sectors");
    union { uint32_t w[N * sizeof(T) / 4]; T e[N]; } u;
#pragma unroll
    for (int i = 0; i < N; i++) u.e[i] = from_f32<T>(x[i]);
#pragma unroll
    for (int i = 0; i < (int)(N * sizeof(T) / 32); i++)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(reinterpret_cast<char*>(p) + 32 * i), "r"(u.w[8 * i]), "r"(u.w[8 * i + 1]), "r"(u.w[8 * i + 2]), "r"(u.w[8 * i + 3]), "r"(u.w[8 * i + 4]),
                       "r"(u.w[8 * i + 5]), "r"(u.w[8 * i + 6]), "r"(u.w[8 * i + 7]) : "memory");
}

// ---- host ---------------------------------------------------------------------
inline uint32_t type_bytes(int dtype) { return dtype == SF_F32 ? 4u : 2u; }
inline bool type_ok(int dtype) { return dtype == SF_F32 || dtype == SF_BF16 || dtype == SF_F16; }
inline bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// The calling thread's current device is the context's inside a call and what it was before after it.
struct DeviceGuard {
    int before = -1;
    cudaError_t e;
    explicit DeviceGuard(int device) {
        e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != device) e = cudaSetDevice(device); else before = -1;
    }
    ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
};
#define SF_ON_DEVICE(ctx) sfrow::DeviceGuard guard__((ctx)->device); if (guard__.e != cudaSuccess) return sf_set_cuda_error(guard__.e, "cudaSetDevice")

// call f with a value of the element type
template <typename F> inline int by_type(int dtype, F f) {
    if (dtype == SF_F32) return f(float());
    if (dtype == SF_BF16) return f(__nv_bfloat16());
    return f(__half());
}

}  // namespace sfrow
