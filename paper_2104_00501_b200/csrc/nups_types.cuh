// Value types of the operators on model tensors (fp32, fp64, fp16, bf16) and loads and stores of several values at once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "nups_internal.cuh"

static inline bool type_known(int t) { return t == NUPS_F32 || t == NUPS_F64 || t == NUPS_F16 || t == NUPS_BF16; }
static inline size_t type_bytes(int t) { return t == NUPS_F64 ? 8 : t == NUPS_F32 ? 4 : 2; }

// Are these addresses (NULL included) multiples of `bytes`, a power of two?  Kernels read and write whole values.
template <class... P> static inline bool suits(size_t bytes, const P*... p) { return ((... | (uintptr_t)p) & (bytes - 1)) == 0; }

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
    if constexpr (sizeof(T) == 2 && N >= 2) {
        const uint32_t* u = (const uint32_t*)&r;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {       // a bf16 is a float's upper half
                out[2 * i] = __uint_as_float(u[i] << 16);
                out[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
            } else {
                const float2 f = __half22float2(*(const __half2*)(u + i));
                out[2 * i] = f.x;
                out[2 * i + 1] = f.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = widen<A>(r.v[i]);
    }
}
template <class T, int N, class A> __device__ __forceinline__ void store_values(T* p, const A* x)
{
    Pack<T, N> r;
    if constexpr (sizeof(T) == 2 && N >= 2) {
        uint32_t* u = (uint32_t*)&r;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                const __nv_bfloat162 h = __floats2bfloat162_rn((float)x[2 * i], (float)x[2 * i + 1]);
                u[i] = *(const uint32_t*)&h;
            } else {
                const __half2 h = __floats2half2_rn((float)x[2 * i], (float)x[2 * i + 1]);
                u[i] = *(const uint32_t*)&h;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = narrow<T>(x[i]);
    }
    store_pack<T, N>(p, r);
}

// Arithmetic on runs of N values; two floats go through one instruction (sm_100's f32x2 forms, each half rounded on its own).
__device__ __forceinline__ unsigned long long two(const float* x) { unsigned long long r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x[0]), "f"(x[1])); return r; }
__device__ __forceinline__ void untwo(unsigned long long r, float* x) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x[0]), "=f"(x[1]) : "l"(r)); }
__device__ __forceinline__ unsigned long long both(float x) { unsigned long long r; asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x)); return r; }
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) { unsigned long long r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) { unsigned long long r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) { unsigned long long r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

__device__ __forceinline__ float mul_add(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double mul_add(double a, double b, double c) { return fma(a, b, c); }

// out = a b + c, elementwise; SA, SB, SC: that operand is one value
template <int N, bool SA, bool SB, bool SC, class A> __device__ __forceinline__ void run_fma(A* out, const A* a, const A* b, const A* c)
{
    if constexpr (std::is_same<A, float>::value && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            untwo(fma2(SA ? both(a[0]) : two(a + i), SB ? both(b[0]) : two(b + i), SC ? both(c[0]) : two(c + i)), out + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = mul_add(a[SA ? 0 : i], b[SB ? 0 : i], c[SC ? 0 : i]);
    }
}
template <int N, bool SB, class A> __device__ __forceinline__ void run_add(A* out, const A* a, const A* b)
{
    if constexpr (std::is_same<A, float>::value && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) untwo(add2(two(a + i), SB ? both(b[0]) : two(b + i)), out + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = a[i] + b[SB ? 0 : i];
    }
}
template <int N, class A> __device__ __forceinline__ void run_mul(A* out, const A* a, const A* b)
{
    if constexpr (std::is_same<A, float>::value && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) untwo(mul2(two(a + i), two(b + i)), out + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = a[i] * b[i];
    }
}
template <int N, class A> __device__ __forceinline__ void run_scale(A* out, const A* a, A f)
{
    if constexpr (std::is_same<A, float>::value && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) untwo(mul2(two(a + i), both(f)), out + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = a[i] * f;
    }
}
// Two running sums over runs of N values (an even and an odd one; VEC = 1 uses the first alone): acc += a, or acc += a b.
template <int N, class A> __device__ __forceinline__ void sum_run(A (&acc)[2], const A* a)
{
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) run_add<2, false, A>(acc, acc, a + i);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) acc[0] += a[i];
    }
}
template <int N, class A> __device__ __forceinline__ void sum_run_of_products(A (&acc)[2], const A* a, const A* b)
{
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) run_fma<2, false, false, false, A>(acc, a + i, b + i, acc);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) acc[0] = mul_add(a[i], b[i], acc[0]);
    }
}
#endif
