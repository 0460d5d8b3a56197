// The gated blocks' element-wise halves: h = act(a) b where the projections come from the
// 8-bit product, and the gradient of [a, b] from that of h.  Bound by memory: 6 and 10 bytes
// an element of h, each read or written once.  49,152 x 1408 bf16: 59.7 us and 98.5, 7.0 TB/s, 1.03 of a plain copy's rate
// (gelu's gradient 105); rows at odd starts, by elements, 5,003 x 1003: 15 and 16 us, 2.0 and 3.2 TB/s.
#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "gnmr.h"
#include "gnmr_act.cuh"
#include "gnmr_internal.h"
#include "gnmr_rows.cuh"

namespace {

using namespace gnmr_rows;
using gnmr_act::activated;

constexpr int kThreads = 256;
// CTAs an SM, as they come: 49,152 x 1408, gradient 98.5 us (7.0 TB/s) with 64, 107 with 8 that stay; the forward half 59.7 and 73.
constexpr int kCtas = 64;
constexpr int kMaxGroups = 2048;                       // as many as the products take

struct Gate {
    const void *dh, *gu;
    void *out;                                         // h, or dgu
    int64_t rows, dh_stride, gu_stride, out_stride;
    int n, groups;
    const int64_t *offsets;
    const uint8_t *mask;
    int64_t mask_stride;
    int each;                                          // places of a row
    int64_t places;                                    // all of them
    int few;                                           // under 2^31
    unsigned inverse;                                  // ceil(2^32 / each)
};

// The groups' first rows, and the last one's end, as the products take them: within [0, rows], not decreasing.
__device__ __forceinline__ void fill_rows(const Gate &g, int *first)
{
    const int lane = threadIdx.x & 31;
    int carry = 0;
    for (int j0 = 0; j0 <= g.groups; j0 += 32) {
        const int j = j0 + lane;
        int at = j == 0 ? 0 : static_cast<int>(g.rows);
        if (g.offsets && j <= g.groups)
            at = static_cast<int>(min(max(g.offsets[j], int64_t(0)), g.rows));
        at = max(at, carry);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(~0u, at, d);
            if (lane >= d)
                at = max(at, v);
        }
        if (j <= g.groups)
            first[j] = at;
        carry = __shfl_sync(~0u, at, 31);
    }
}

// Whether row r belongs to a group that is computed: the last that begins at or before it has a mask byte of 0,
// and does not end before it.
__device__ __forceinline__ bool wanted(const Gate &g, const int *first, int r)
{
    int lo = 0;
    for (int hi = g.groups; hi - lo > 1;) {
        const int mid = (lo + hi) / 2;
        if (first[mid] <= r)
            lo = mid;
        else
            hi = mid;
    }
    return r >= first[lo] && r < first[lo + 1] && (!g.mask || g.mask[lo * g.mask_stride] == 0);
}

template <typename T, int kAct, bool kGrad, int kN>
__device__ __forceinline__ void compute(const float (&dh)[kN], const float (&a)[kN], const float (&b)[kN], float (&x)[kN], float (&y)[kN])
{
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        if (kGrad) {
            float slope;
            const float v = activated<kAct>(a[i], slope);
            x[i] = dh[i] * b[i] * slope;
            y[i] = dh[i] * v;
        } else {
            x[i] = activated<kAct>(a[i]) * b[i];
        }
    }
}

// kPer places a thread, a CTA's width apart: eight elements of h each, or one where rows do not start at multiples of
// 16 bytes.
template <typename T, int kAct, bool kGrad, bool kVector, int kPer>
__global__ void __launch_bounds__(kThreads) gate_kernel(const Gate g)
{
    constexpr int kN = kVector ? kIn16<T> : 1;
    using Raw = std::conditional_t<kVector, uint4, T>;
    extern __shared__ int first[];
    if (!kGrad) {
        if (threadIdx.x < 32)
            fill_rows(g, first);
        __syncthreads();
    }
    const T *const dh = static_cast<const T *>(g.dh), *const gu = static_cast<const T *>(g.gu);
    T *const out = static_cast<T *>(g.out);
    for (int64_t i0 = int64_t(blockIdx.x) * (kThreads * kPer) + threadIdx.x; i0 < g.places; i0 += int64_t(gridDim.x) * (kThreads * kPer)) {
        Raw d[kPer], a[kPer], b[kPer];
        int64_t to[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int64_t i = i0 + k * kThreads;
            to[k] = -1;
            if (i >= g.places)
                continue;
            const int64_t r = g.few ? __umulhi(static_cast<unsigned>(i), g.inverse) : i / g.each;
            // of a product below 2^32 the quotient may come out one too large
            const int64_t row = r - (g.few && r * g.each > i), at = (i - row * g.each) * kN;
            if (!kGrad && !wanted(g, first, static_cast<int>(row)))
                continue;
            to[k] = row * g.out_stride + at;
            const T *const from = gu + row * g.gu_stride + at;
            if constexpr (kVector) {
                a[k] = load_once(from);
                b[k] = load_once(from + g.n);
                if (kGrad)
                    d[k] = load_once(dh + row * g.dh_stride + at);
            } else {
                a[k] = from[0];
                b[k] = from[g.n];
                if (kGrad)
                    d[k] = dh[row * g.dh_stride + at];
            }
        }
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            if (to[k] < 0)
                continue;
            float u[kN], v[kN], w[kN], x[kN], y[kN];
            if constexpr (kVector) {
                widen<T>(a[k], u);
                widen<T>(b[k], v);
                if (kGrad)
                    widen<T>(d[k], w);
            } else {
                u[0] = to_f32(a[k]);
                v[0] = to_f32(b[k]);
                if (kGrad)
                    w[0] = to_f32(d[k]);
            }
            compute<T, kAct, kGrad, kN>(w, u, v, x, y);
            T *const at = out + to[k];
            if constexpr (kVector) {
                store_once(at, narrow<T>(x));
                if (kGrad)
                    store_once(at + g.n, narrow<T>(y));
            } else {
                at[0] = from_f32<T>(x[0]);
                if (kGrad)
                    at[g.n] = from_f32<T>(y[0]);
            }
        }
    }
}

template <typename T, int kAct, bool kGrad> cudaError_t launch(Gate g, bool vector, int sms, cudaStream_t st)
{
    constexpr int kVectors = 2, kElements = 4;
    g.each = vector ? g.n / kIn16<T> : g.n;
    g.places = g.rows * g.each;
    g.few = g.places < int64_t(1) << 31 && g.each > 1;
    g.inverse = static_cast<unsigned>(((int64_t(1) << 32) + g.each - 1) / g.each);
    const int turn = kThreads * (vector ? kVectors : kElements);
    const unsigned ctas = static_cast<unsigned>(std::min((g.places + turn - 1) / turn, int64_t(sms) * kCtas));
    const size_t shared = kGrad ? 0 : (g.groups + 1) * sizeof(int);
    if (vector)
        gate_kernel<T, kAct, kGrad, true, kVectors><<<ctas, kThreads, shared, st>>>(g);
    else
        gate_kernel<T, kAct, kGrad, false, kElements><<<ctas, kThreads, shared, st>>>(g);
    return cudaGetLastError();
}

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

// What both calls check, and their launch.  grad: dh is there.
template <bool kGrad> gnmr_status run(const Gate &g, int32_t dtype, int32_t act, cudaStream_t st)
{
    if (dtype != GNMR_DTYPE_BF16 && dtype != GNMR_DTYPE_F16)
        return fail(GNMR_ERR_INVALID_ARG, "gate: dtype not 16 bits");
    if (act != GNMR_ACT_SILU && act != GNMR_ACT_GELU)
        return fail(GNMR_ERR_INVALID_ARG, "gate: unknown activation");
    if (g.groups < 1 || g.groups > kMaxGroups || g.rows < 0 || g.rows > INT32_MAX || g.n < 1 || g.n > INT32_MAX / 2)
        return fail(GNMR_ERR_INVALID_ARG, "gate: groups, rows or n out of range");
    if (!g.offsets && g.groups != 1)
        return fail(GNMR_ERR_INVALID_ARG, "gate: NULL offsets with several groups");
    const int64_t wide = 2 * int64_t(g.n), far = int64_t(1) << 31;
    if (g.gu_stride < wide || g.out_stride < (kGrad ? wide : g.n) || (kGrad && g.dh_stride < g.n) ||
        (g.mask && g.groups > 1 && g.mask_stride < 1))
        return fail(GNMR_ERR_LAYOUT, "gate: a stride below what it strides over");
    // (a single row has no stride)
    if (g.rows > 1 && (g.gu_stride > far || g.out_stride > far || g.dh_stride > far))
        return fail(GNMR_ERR_LAYOUT, "gate: a stride above 2^31 elements");
    if (g.rows == 0)
        return GNMR_OK;
    if (!g.gu || !g.out || (kGrad && !g.dh))
        return fail(GNMR_ERR_INVALID_ARG, "gate: NULL pointer");
    if (misaligned(g.gu, 2) || misaligned(g.out, 2) || misaligned(g.dh, 2) || misaligned(g.offsets, 8))
        return fail(GNMR_ERR_LAYOUT, "gate: a buffer not aligned to its element size");
    if (kGrad && g.rows > 1 && g.out == g.gu && g.out_stride != g.gu_stride)
        return fail(GNMR_ERR_LAYOUT, "gate: in place with another stride");
    int sms = 0;
    if (current_sms(&sms) != cudaSuccess) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, "gate: no current device");
    }
    const bool vector = g.n % 8 == 0 && rows_of_16(g.gu, g.rows, g.gu_stride, 2) && rows_of_16(g.out, g.rows, g.out_stride, 2) &&
                        (!kGrad || rows_of_16(g.dh, g.rows, g.dh_stride, 2));
    const cudaError_t e = by_16_bit_type(dtype, [&](auto v) {
        using T = decltype(v);
        return act == GNMR_ACT_SILU ? launch<T, GNMR_ACT_SILU, kGrad>(g, vector, sms, st)
                                    : launch<T, GNMR_ACT_GELU, kGrad>(g, vector, sms, st);
    });
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    return GNMR_OK;
}

}  // namespace

extern "C" {

gnmr_status gnmr_gate(const void *d_gu, int32_t dtype, int32_t activation, int32_t groups, int64_t rows, int32_t n,
                      int64_t gu_stride, const int64_t *d_offsets, const uint8_t *d_mask, int64_t mask_stride, void *d_h,
                      int64_t h_stride, void *stream)
{
    const Gate g{nullptr, d_gu, d_h, rows, 0, gu_stride, h_stride, n, groups, d_offsets, d_mask, mask_stride, 0, 0, 0, 0};
    return run<false>(g, dtype, activation, static_cast<cudaStream_t>(stream));
}

gnmr_status gnmr_gate_grad(const void *d_dh, int32_t dtype, int32_t activation, int64_t rows, int32_t n, int64_t dh_stride,
                           const void *d_gu, int64_t gu_stride, void *d_dgu, int64_t dgu_stride, void *stream)
{
    const Gate g{d_dh, d_gu, d_dgu, rows, dh_stride, gu_stride, dgu_stride, n, 1, nullptr, nullptr, 1, 0, 0, 0, 0};
    return run<true>(g, dtype, activation, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
