// Value types of the operators on model tensors (fp32, fp64, fp16, bf16) and loads and stores of several values at once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "nups_internal.cuh"

static inline bool type_known(int t) { return t == NUPS_F32 || t == NUPS_F64 || t == NUPS_F16 || t == NUPS_BF16; }
static inline size_t type_bytes(int t) { return t == NUPS_F64 ? 8 : t == NUPS_F32 ? 4 : 2; }

// Does the call's current device hold the store?  Kernels are launched on the current device, on a stream of it.
static inline nups_status on_own_device(const nups_store* s)
{
    int dev = -1;
    CK(cudaGetDevice(&dev));
    return dev == s->device ? NUPS_OK : NUPS_ESTATE;
}

#ifdef __CUDACC__
template <class A> __device__ __forceinline__ A widen(float x) { return (A)x; }
template <class A> __device__ __forceinline__ A widen(double x) { return (A)x; }
template <class A> __device__ __forceinline__ A widen(__half x) { return (A)__half2float(x); }
template <class A> __device__ __forceinline__ A widen(__nv_bfloat16 x) { return (A)__bfloat162float(x); }

template <class T, class A> struct Narrow;
template <> struct Narrow<float, float> { static __device__ __forceinline__ float of(float x) { return x; } };
template <> struct Narrow<double, double> { static __device__ __forceinline__ double of(double x) { return x; } };
template <> struct Narrow<float, double> { static __device__ __forceinline__ float of(double x) { return (float)x; } };
template <> struct Narrow<__half, float> { static __device__ __forceinline__ __half of(float x) { return __float2half_rn(x); } };
template <> struct Narrow<__nv_bfloat16, float> { static __device__ __forceinline__ __nv_bfloat16 of(float x) { return __float2bfloat16_rn(x); } };
template <class T, class A> __device__ __forceinline__ T narrow(A x) { return Narrow<T, A>::of(x); }

// An aligned run of N values, moved by one instruction of up to 16 bytes (two for 32).
template <class T, int N> struct __align__(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack { T v[N]; };

template <class T, int N> __device__ __forceinline__ Pack<T, N> load_pack(const T* p)
{
    constexpr int B = sizeof(T) * N;
    Pack<T, N> r;
    if constexpr (B == 32) {
        const uint4 a = *(const uint4*)p, b = *((const uint4*)p + 1);
        *(uint4*)&r = a;
        *((uint4*)&r + 1) = b;
    } else if constexpr (B == 16) {
        *(uint4*)&r = *(const uint4*)p;
    } else if constexpr (B == 8) {
        *(uint2*)&r = *(const uint2*)p;
    } else if constexpr (B == 4) {
        *(unsigned*)&r = *(const unsigned*)p;
    } else {
        static_assert(B == 2, "2 to 32 bytes");
        *(unsigned short*)&r = *(const unsigned short*)p;
    }
    return r;
}
template <class T, int N> __device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r)
{
    constexpr int B = sizeof(T) * N;
    if constexpr (B == 32) {
        *(uint4*)p = *(const uint4*)&r;
        *((uint4*)p + 1) = *((const uint4*)&r + 1);
    } else if constexpr (B == 16) {
        *(uint4*)p = *(const uint4*)&r;
    } else if constexpr (B == 8) {
        *(uint2*)p = *(const uint2*)&r;
    } else if constexpr (B == 4) {
        *(unsigned*)p = *(const unsigned*)&r;
    } else {
        static_assert(B == 2, "2 to 32 bytes");
        *(unsigned short*)p = *(const unsigned short*)&r;
    }
}
template <class A, class T, int N> __device__ __forceinline__ void unpack(const Pack<T, N>& r, A* out)
{
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = widen<A>(r.v[i]);
}
template <class T, int N, class A> __device__ __forceinline__ void store_values(T* p, const A* x)
{
    Pack<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = narrow<T>(x[i]);
    store_pack<T, N>(p, r);
}
#endif
