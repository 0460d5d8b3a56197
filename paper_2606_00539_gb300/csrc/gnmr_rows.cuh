// 16 bytes of a row at a time, widened to fp32 and rounded back: what the row kernels of the
// gated blocks, the layer norm and the clipping share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <type_traits>

#include "gnmr.h"

namespace gnmr_rows {

template <typename T> __device__ __forceinline__ float to_f32(T v) { return static_cast<float>(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v) { return static_cast<T>(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }

// Elements of 16 bytes.
template <typename T> constexpr int kIn16 = 16 / static_cast<int>(sizeof(T));

template <typename T> __device__ __forceinline__ void widen(const uint4 &v, float (&f)[kIn16<T>])
{
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            f[i] = __uint_as_float(w[i]);
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 p = __half22float2(reinterpret_cast<const __half2 &>(w[i]));
            f[2 * i] = p.x;
            f[2 * i + 1] = p.y;
        }
    }
}

template <typename T> __device__ __forceinline__ uint4 narrow(const float (&f)[kIn16<T>])
{
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(f[i]);
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = reinterpret_cast<const unsigned &>(p);
        } else {
            const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
            w[i] = reinterpret_cast<const unsigned &>(p);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Two fp32 numbers in a pair of registers, and their operations in one instruction.
using Pair = unsigned long long;

__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}

__device__ __forceinline__ Pair both(float v) { return pair(v, v); }

__device__ __forceinline__ float2 apart(Pair p)
{
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}

__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// 16 bytes as pairs of neighbours, and back.
template <typename T> __device__ __forceinline__ void widen2(const uint4 &v, Pair (&f)[kIn16<T> / 2])
{
    float e[kIn16<T>];
    widen<T>(v, e);
#pragma unroll
    for (int i = 0; i < kIn16<T> / 2; ++i)
        f[i] = pair(e[2 * i], e[2 * i + 1]);
}

template <typename T> __device__ __forceinline__ uint4 narrow2(const Pair (&f)[kIn16<T> / 2])
{
    float e[kIn16<T>];
#pragma unroll
    for (int i = 0; i < kIn16<T> / 2; ++i) {
        const float2 v = apart(f[i]);
        e[2 * i] = v.x, e[2 * i + 1] = v.y;
    }
    return narrow<T>(e);
}

// Copies of 16 bytes to shared memory that their thread waits for, by the groups that it begins.
__device__ __forceinline__ void copy16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

__device__ __forceinline__ void copies_begun() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

__device__ __forceinline__ uint4 load_shared(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

__device__ __forceinline__ void store_shared(uint32_t at, const uint4 &v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint32_t shared_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// Loads and stores of what is used once.  Volatile: none moves up over griddepcontrol.wait.
__device__ __forceinline__ uint4 load_once(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ void store_once(void *p, const uint4 &v)
{
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

// ---- host ---------------------------------------------------------------------

inline bool misaligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

inline size_t element_bytes(int32_t dtype) { return dtype == GNMR_DTYPE_F32 ? 4 : 2; }

inline bool known(int32_t dtype) { return dtype == GNMR_DTYPE_F32 || dtype == GNMR_DTYPE_BF16 || dtype == GNMR_DTYPE_F16; }

// Whether rows of `stride` elements from p on all start at multiples of 16 bytes.
inline bool rows_of_16(const void *p, int64_t rows, int64_t stride, size_t bytes)
{
    return !misaligned(p, 16) && (rows <= 1 || stride * bytes % 16 == 0);
}

// The current device's SMs, or what hides them.
inline cudaError_t current_sms(int *sms)
{
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    return e == cudaSuccess ? cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) : e;
}

// Lets a kernel have all of an SM's shared memory on the current device, asking the driver once for each kernel and device
// (every call would cost a small launch a quarter of its time).
constexpr int kSharedMost = 226 << 10;

template <auto kKernel> cudaError_t allow_shared()
{
    static std::atomic<unsigned long long> asked{0};   // a bit for each device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (asked.load(std::memory_order_relaxed) & bit)
        return cudaSuccess;
    e = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
    if (e == cudaSuccess)
        asked.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Calls f with a value of the type that `dtype` names.
template <typename F> cudaError_t by_type(int32_t dtype, F f)
{
    if (dtype == GNMR_DTYPE_F32)
        return f(0.0f);
    if (dtype == GNMR_DTYPE_BF16)
        return f(__nv_bfloat16());
    return f(__half());
}

template <typename F> cudaError_t by_16_bit_type(int32_t dtype, F f)
{
    return dtype == GNMR_DTYPE_BF16 ? f(__nv_bfloat16()) : f(__half());
}

}  // namespace gnmr_rows
