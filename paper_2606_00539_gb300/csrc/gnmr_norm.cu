// Layer norm by row, and its backward pass with the reduction of the parameters' gradients.
//
//   forward   mean, rstd = 1 / sqrt(mean of (x - mean)^2 + eps); y = (x - mean) rstd w + b
//   backward  xh = (x - mean) rstd, t = dy w; dx = rstd (t - mean of t - xh mean of t xh);
//             dw = sum over rows of dy xh, db = sum over rows of dy
//
// Bound by memory: x read and y written; x and dy read and dx written.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "gnmr.h"
#include "gnmr_internal.h"
#include "gnmr_rows.cuh"

namespace {

using namespace gnmr_rows;

struct Norm {
    int64_t rows;
    int cols;
    float inverse;                                     // 1 / cols
    float eps;
    const void *x, *w, *b, *dy;
    int64_t x_stride, y_stride, dy_stride;
    const float *mean_in, *rstd_in;
    float *mean, *rstd;
    void *y;                                           // or dx
    float *part_w, *part_b;                            // [parts][cols] each
    int parts;
    void *dw, *db;
    int add;
    int aligned;                                       // the parameters start at multiples of 16 bytes
};

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// The sum over a CTA, the same bits in every thread.  `shared`: a float for each warp, which no other call within the
// same two barriers uses.
__device__ __forceinline__ float cta_sum(float v, float *shared)
{
    const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    v = warp_sum(v);
    if (warps == 1)
        return v;
    if (lane == 0)
        shared[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < warps ? shared[lane] : 0.0f);
}

template <int kN> __device__ __forceinline__ float tree_sum(const float (&f)[kN])
{
    if constexpr (kN == 1)
        return f[0];
    else if constexpr (kN == 4)
        return (f[0] + f[1]) + (f[2] + f[3]);
    else
        return ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
}

// What a thread holds of a row: kUnits times 16 bytes, or single elements.
template <typename T, int kUnits, bool kVector> struct Held {
    static constexpr int kN = kVector ? kIn16<T> : 1;
    std::conditional_t<kVector, uint4, T> v[kUnits];

    // Units at, at + step, ... of the row, as far as they are below `units`.
    __device__ __forceinline__ void load(const T *row, int at, int step, int units)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (at + u * step < units) {
                if constexpr (kVector)
                    v[u] = load_once(row + int64_t(at + u * step) * kN);
                else
                    v[u] = row[at + u * step];
            }
    }
    __device__ __forceinline__ void get(int u, float (&f)[kN]) const
    {
        if constexpr (kVector)
            widen<T>(v[u], f);
        else
            f[0] = to_f32(v[u]);
    }
    __device__ __forceinline__ float sum(int at, int step, int units) const
    {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (at + u * step < units) {
                float f[kN];
                get(u, f);
                s += tree_sum<kN>(f);
            }
        return s;
    }
    // Of (x - mean)^2.
    __device__ __forceinline__ float squares(int at, int step, int units, float mean) const
    {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (at + u * step < units) {
                float f[kN];
                get(u, f);
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    f[j] = (f[j] - mean) * (f[j] - mean);
                s += tree_sum<kN>(f);
            }
        return s;
    }
};

// kN parameters from element `at` on, or `none` where there are none.  aligned: whole 16 bytes may be read.
template <typename P, int kN> __device__ __forceinline__ void params(const void *from, int64_t at, float none, bool aligned, float (&f)[kN])
{
    const P *p = static_cast<const P *>(from) + at;
    if (!from) {
#pragma unroll
        for (int j = 0; j < kN; ++j)
            f[j] = none;
        return;
    }
    if constexpr (kN % kIn16<P> == 0) {
        if (aligned) {
#pragma unroll
            for (int j = 0; j < kN; j += kIn16<P>) {
                float part[kIn16<P>];
                widen<P>(__ldg(reinterpret_cast<const uint4 *>(p + j)), part);
#pragma unroll
                for (int k = 0; k < kIn16<P>; ++k)
                    f[j + k] = part[k];
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < kN; ++j)
        f[j] = to_f32(p[j]);
}

template <typename T, int kN> __device__ __forceinline__ void store_unit(T *to, const float (&f)[kN])
{
    if constexpr (kN == 1)
        *to = from_f32<T>(f[0]);
    else
        store_once(to, narrow<T>(f));
}

__device__ __forceinline__ float rstd_of(float squares, const Norm &n) { return 1.0f / sqrtf(squares / n.cols + n.eps); }

// A warp a row, which it holds in registers: no barrier, sums by shuffles.  The parameters are in shared
// memory, as fp32, in groups of four of which a warp reads contiguous ones.
template <typename T, typename P, int kUnits>
__global__ void __launch_bounds__(kThreads, kUnits > 12 ? 2 : kUnits > 6 ? 3 : 4) norm_warp_kernel(const Norm n)
{
    constexpr int kN = kIn16<T>, kQuads = kN / 4;
    extern __shared__ float4 quads[];                  // weight: [kQuads][units], then bias
    const int units = n.cols / kN, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < units; i += kThreads) {
        float w[kN], b[kN];
        params<P, kN>(n.w, int64_t(i) * kN, 1.0f, n.aligned, w);
        params<P, kN>(n.b, int64_t(i) * kN, 0.0f, n.aligned, b);
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            quads[q * units + i] = make_float4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            quads[(kQuads + q) * units + i] = make_float4(b[4 * q], b[4 * q + 1], b[4 * q + 2], b[4 * q + 3]);
        }
    }
    __syncthreads();
    for (int64_t r = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); r < n.rows; r += int64_t(gridDim.x) * kWarps) {
        Held<T, kUnits, true> x;
        x.load(static_cast<const T *>(n.x) + r * n.x_stride, lane, 32, units);
        const float mean = warp_sum(x.sum(lane, 32, units)) / n.cols;
        const float rstd = rstd_of(warp_sum(x.squares(lane, 32, units, mean)), n);
        if (lane == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = lane + u * 32;
            if (at < units) {
                float f[kN];
                x.get(u, f);
#pragma unroll
                for (int q = 0; q < kQuads; ++q) {
                    const float4 w = quads[q * units + at], b = quads[(kQuads + q) * units + at];
                    f[4 * q] = fmaf((f[4 * q] - mean) * rstd, w.x, b.x);
                    f[4 * q + 1] = fmaf((f[4 * q + 1] - mean) * rstd, w.y, b.y);
                    f[4 * q + 2] = fmaf((f[4 * q + 2] - mean) * rstd, w.z, b.z);
                    f[4 * q + 3] = fmaf((f[4 * q + 3] - mean) * rstd, w.w, b.w);
                }
                store_unit<T, kN>(y + int64_t(at) * kN, f);
            }
        }
    }
}

// A CTA a row, which it holds in registers: few rows, wide ones, and those that do not start at multiples of 16 bytes.
template <typename T, typename P, int kUnits, bool kVector>
__global__ void __launch_bounds__(1024) norm_cta_kernel(const Norm n)
{
    using H = Held<T, kUnits, kVector>;
    constexpr int kN = H::kN;
    __shared__ float shared[2][2][32];                 // by turns: a row's sums are read while the next one's are formed
    const int units = n.cols / kN, at = threadIdx.x, step = blockDim.x;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x, turn ^= 1) {
        H x;
        x.load(static_cast<const T *>(n.x) + r * n.x_stride, at, step, units);
        const float mean = cta_sum(x.sum(at, step, units), shared[turn][0]) / n.cols;
        const float rstd = rstd_of(cta_sum(x.squares(at, step, units, mean), shared[turn][1]), n);
        if (threadIdx.x == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (at + u * step < units) {
                const int64_t e = int64_t(at + u * step) * kN;
                float f[kN], w[kN], b[kN];
                params<P, kN>(n.w, e, 1.0f, n.aligned, w);
                params<P, kN>(n.b, e, 0.0f, n.aligned, b);
                x.get(u, f);
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    f[j] = fmaf((f[j] - mean) * rstd, w[j], b[j]);
                store_unit<T, kN>(y + e, f);
            }
    }
}

// ---- backward -------------------------------------------------------------------

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

// kV sums (2 or 4) over a warp at once: in the end lanes of 32 / kV have one each, lane l the (l kV / 32)-th.
template <int kV> __device__ __forceinline__ float warp_sums(const float (&v)[kV])
{
    const int lane = threadIdx.x & 31;
    float s;
    if constexpr (kV == 4) {
        const bool high = lane & 16;
        const float a = (high ? v[2] : v[0]) + __shfl_xor_sync(~0u, high ? v[0] : v[2], 16);
        const float b = (high ? v[3] : v[1]) + __shfl_xor_sync(~0u, high ? v[1] : v[3], 16);
        const bool second = lane & 8;
        s = (second ? b : a) + __shfl_xor_sync(~0u, second ? a : b, 8);
    } else {
        const bool high = lane & 16;
        s = (high ? v[1] : v[0]) + __shfl_xor_sync(~0u, high ? v[0] : v[1], 16);
        s += __shfl_xor_sync(~0u, s, 8);
    }
    s += __shfl_xor_sync(~0u, s, 4);
    s += __shfl_xor_sync(~0u, s, 2);
    return s + __shfl_xor_sync(~0u, s, 1);
}

// How the backward kernel takes rows: a group of `span` threads has kRows of them a turn, as many groups as there are
// threads for.  A thread has the same columns of every row, kUnits times 16 bytes (or single elements), so that the sums over the rows
// stay in its registers; rows on their way are in shared memory, where each thread copies its own bytes (no barrier for
// that), kTurns turns ahead.  One barrier a turn, for the row sums.
template <typename T_, typename P_, int kUnits_, int kRows_, int kTurns_, int kMost_, bool kVector_> struct Shape {
    using T = T_;
    using P = P_;
    static constexpr int kUnits = kUnits_, kRows = kRows_, kTurns = kTurns_, kMost = kMost_;
    static constexpr bool kVector = kVector_;
    static constexpr int kN = kVector ? kIn16<T> : 1;
    static constexpr int kV = 2 * kRows;               // row sums a turn
    static constexpr int kTurnBytes = kVector ? kRows * kUnits * 2 * 16 : 0;       // of a thread
    static constexpr int kShared = kMost * kTurnBytes * kTurns;
};

template <typename S> __global__ void __launch_bounds__(S::kMost, 1) norm_grad_kernel(const Norm n, int span)
{
    using T = typename S::T;
    using P = typename S::P;
    constexpr int kN = S::kN, kUnits = S::kUnits, kRows = S::kRows, kV = S::kV, kMost = S::kMost;
    extern __shared__ __align__(16) uint8_t bytes[];
    __shared__ float sums[2][kMost / 32][kV];
    const int units = n.cols / kN, groups = blockDim.x / span, group = threadIdx.x / span, at = threadIdx.x - group * span;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = span >> 5, warp0 = group * warps;
    const T *const x = static_cast<const T *>(n.x), *const dy = static_cast<const T *>(n.dy);
    T *const dx = static_cast<T *>(n.y);
    const int64_t turns = (n.rows + groups * kRows - 1) / (groups * kRows);
    // 16-byte places of this thread: turn, row, unit, x or dy; those of a warp side by side
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(bytes)) + threadIdx.x * 16;
    const auto place = [&](int slot, int row, int u, int which) {
        return mine + (((slot * kRows + row) * kUnits + u) * 2 + which) * (blockDim.x * 16);
    };
    const auto row_of = [&](int64_t turn, int row) { return (turn * groups + group) * kRows + row; };
    const auto fetch = [&](int64_t turn, int slot) {
        if (S::kVector && turn < turns)
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int64_t r = row_of(turn, i);
                if (r < n.rows)
#pragma unroll
                    for (int u = 0; u < kUnits; ++u)
                        if (at + u * span < units) {
                            copy16(place(slot, i, u, 0), x + r * n.x_stride + int64_t(at + u * span) * kN);
                            copy16(place(slot, i, u, 1), dy + r * n.dy_stride + int64_t(at + u * span) * kN);
                        }
            }
        copies_begun();
    };
    float w[kUnits][kN], dw[kUnits][kN], db[kUnits][kN];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
#pragma unroll
        for (int j = 0; j < kN; ++j)
            w[u][j] = dw[u][j] = db[u][j] = 0.0f;
        if (at + u * span < units)
            params<P, kN>(n.w, int64_t(at + u * span) * kN, 1.0f, n.aligned, w[u]);
    }
    float mean[kRows], rstd[kRows];                    // of the turn to come
    const auto statistics = [&](int64_t turn) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t r = row_of(turn, i);
            mean[i] = r < n.rows ? n.mean_in[r] : 0.0f;
            rstd[i] = r < n.rows ? n.rstd_in[r] : 0.0f;
        }
    };
    int64_t turn = blockIdx.x;
#pragma unroll
    for (int s = 0; s < S::kTurns; ++s)
        fetch(turn + int64_t(s) * gridDim.x, s);
    statistics(turn);
    int slot = 0, parity = 0;
    for (; turn < turns; turn += gridDim.x) {
        copies_done<S::kTurns - 1>();
        float xh[kRows][kUnits][kN], t[kRows][kUnits][kN], v[kV], scale[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t r = row_of(turn, i);
            const bool there = r < n.rows;
            scale[i] = rstd[i];
            v[2 * i] = v[2 * i + 1] = 0.0f;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                float d[kN], q[kN];
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    xh[i][u][j] = t[i][u][j] = d[j] = q[j] = 0.0f;
                if (there && at + u * span < units) {
                    float f[kN];
                    if constexpr (S::kVector) {
                        widen<T>(load_shared(place(slot, i, u, 0)), f);
                        widen<T>(load_shared(place(slot, i, u, 1)), d);
                    } else {
                        f[0] = to_f32(x[r * n.x_stride + at + u * span]);
                        d[0] = to_f32(dy[r * n.dy_stride + at + u * span]);
                    }
#pragma unroll
                    for (int j = 0; j < kN; ++j) {
                        xh[i][u][j] = (f[j] - mean[i]) * rstd[i];
                        t[i][u][j] = d[j] * w[u][j];
                        q[j] = t[i][u][j] * xh[i][u][j];
                        dw[u][j] = fmaf(d[j], xh[i][u][j], dw[u][j]);
                        db[u][j] += d[j];
                    }
                }
                v[2 * i] += tree_sum<kN>(t[i][u]);
                v[2 * i + 1] += tree_sum<kN>(q);
            }
        }
        fetch(turn + int64_t(S::kTurns) * gridDim.x, slot);
        if (++slot == S::kTurns)
            slot = 0;
        statistics(turn + gridDim.x);
        if (!dx)
            continue;
        // the sums of every warp, and then of the group's warps in their order
        const float s = warp_sums<kV>(v);
        constexpr int kLanes = 32 / kV;
        float of_group = s;
        if (warps > 1) {
            if (lane % kLanes == 0)
                sums[parity][warp][lane / kLanes] = s;
            __syncthreads();
            of_group = 0.0f;
            for (int i = lane % kLanes; i < warps; i += kLanes)
                of_group += sums[parity][warp0 + i][lane / kLanes];
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1)
                of_group += __shfl_xor_sync(~0u, of_group, o);
            parity ^= 1;
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float m1 = __shfl_sync(~0u, of_group, 2 * i * kLanes) / n.cols, m2 = __shfl_sync(~0u, of_group, (2 * i + 1) * kLanes) / n.cols;
            const int64_t r = row_of(turn, i);
            if (r < n.rows)
#pragma unroll
                for (int u = 0; u < kUnits; ++u)
                    if (at + u * span < units) {
                        float f[kN];
#pragma unroll
                        for (int j = 0; j < kN; ++j)
                            f[j] = scale[i] * (t[i][u][j] - m1 - xh[i][u][j] * m2);
                        store_unit<T, kN>(dx + r * n.y_stride + int64_t(at + u * span) * kN, f);
                    }
        }
    }
    if (!n.dw && !n.db)
        return;
    // the groups' sums over their rows, added up in their order
    copies_done<0>();
    float *const all = reinterpret_cast<float *>(bytes);           // [2][unit's element][thread]
    if (groups > 1) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                all[(u * kN + j) * blockDim.x + threadIdx.x] = dw[u][j];
                all[((kUnits + u) * kN + j) * blockDim.x + threadIdx.x] = db[u][j];
            }
        __syncthreads();
        if (group)
            return;
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
            for (int j = 0; j < kN; ++j)
                for (int g = 1; g < groups; ++g) {
                    dw[u][j] += all[(u * kN + j) * blockDim.x + g * span + at];
                    db[u][j] += all[((kUnits + u) * kN + j) * blockDim.x + g * span + at];
                }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
        if (at + u * span < units) {
            const int64_t e = int64_t(blockIdx.x) * n.cols + int64_t(at + u * span) * kN;
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                n.part_w[e + j] = dw[u][j];
                n.part_b[e + j] = db[u][j];
            }
        }
}

// Any width and alignment: a CTA a row, which it reads three times.
template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_any_kernel(const Norm n)
{
    __shared__ float shared[2][2][32];
    const P *const w = static_cast<const P *>(n.w), *const b = static_cast<const P *>(n.b);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x, turn ^= 1) {
        const T *const x = static_cast<const T *>(n.x) + r * n.x_stride;
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
        float s = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads)
            s += to_f32(x[i]);
        const float mean = cta_sum(s, shared[turn][0]) / n.cols;
        s = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            const float d = to_f32(x[i]) - mean;
            s += d * d;
        }
        const float rstd = rstd_of(cta_sum(s, shared[turn][1]), n);
        if (threadIdx.x == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            float v = (to_f32(x[i]) - mean) * rstd;
            v = n.w ? v * to_f32(w[i]) : v;
            y[i] = from_f32<T>(n.b ? v + to_f32(b[i]) : v);
        }
    }
}

template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_grad_any_kernel(const Norm n)
{
    __shared__ float shared[2][2][32];
    const P *const w = static_cast<const P *>(n.w);
    int turn = 0;
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x, turn ^= 1) {
        const T *const x = static_cast<const T *>(n.x) + r * n.x_stride, *const dy = static_cast<const T *>(n.dy) + r * n.dy_stride;
        T *const dx = static_cast<T *>(n.y) + r * n.y_stride;
        const float mean = n.mean_in[r], rstd = n.rstd_in[r];
        float s = 0.0f, q = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            const float t = to_f32(dy[i]) * (n.w ? to_f32(w[i]) : 1.0f);
            s += t;
            q += t * ((to_f32(x[i]) - mean) * rstd);
        }
        s = cta_sum(s, shared[turn][0]) / n.cols;
        q = cta_sum(q, shared[turn][1]) / n.cols;
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            const float t = to_f32(dy[i]) * (n.w ? to_f32(w[i]) : 1.0f);
            dx[i] = from_f32<T>(rstd * (t - s - (to_f32(x[i]) - mean) * rstd * q));
        }
    }
}

// Part blockIdx.y of the rows, a column a thread.
template <typename T>
__global__ void __launch_bounds__(kThreads) columns_any_kernel(const Norm n)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= n.cols)
        return;
    const int64_t r0 = n.rows * blockIdx.y / n.parts, r1 = n.rows * (blockIdx.y + 1) / n.parts;
    float s = 0.0f, q = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        const float d = to_f32(static_cast<const T *>(n.dy)[r * n.dy_stride + i]);
        const float xh = (to_f32(static_cast<const T *>(n.x)[r * n.x_stride + i]) - n.mean_in[r]) * n.rstd_in[r];
        s += d;
        q += d * xh;
    }
    n.part_b[int64_t(blockIdx.y) * n.cols + i] = s;
    n.part_w[int64_t(blockIdx.y) * n.cols + i] = q;
}

// The parts' sums: 32 columns a CTA, its warps a share of the parts each, joined in their order.
template <typename G>
__global__ void __launch_bounds__(kThreads) join_kernel(const Norm n)
{
    __shared__ float shared[kWarps][32];
    G *const to = static_cast<G *>(blockIdx.y ? n.db : n.dw);
    if (!to)
        return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (i < n.cols) {
        const float *const part = (blockIdx.y ? n.part_b : n.part_w) + i;
#pragma unroll 8
        for (int p = warp; p < n.parts; p += kWarps)
            s += part[int64_t(p) * n.cols];
    }
    shared[warp][lane] = s;
    __syncthreads();
    if (warp || i >= n.cols)
        return;
#pragma unroll
    for (int k = 1; k < kWarps; ++k)
        s += shared[k][lane];
    to[i] = from_f32<G>(n.add ? to_f32(to[i]) + s : s);
}

// ---- host -----------------------------------------------------------------------

constexpr int kMostParts = 512;

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

int64_t parts_bytes(const gnmr_norm *p)
{
    return p->d_dweight || p->d_dbias ? (2 * int64_t(kMostParts) * p->cols * 4 + 255) / 256 * 256 : 0;
}

gnmr_status check(const gnmr_norm *p, bool grad)
{
    if (!p)
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: NULL argument");
    if (!known(p->dtype) || (p->param_dtype != p->dtype && p->param_dtype != GNMR_DTYPE_F32) || (grad && !known(p->grad_dtype)))
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: a dtype that is not taken");
    if (p->rows < 0 || p->rows > INT32_MAX || p->cols < 1 || p->cols > int64_t(1) << 30)
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: rows or cols out of range");
    if (!grad && !(p->eps >= 0 && std::isfinite(p->eps)))
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: eps has to be finite and not negative");
    const int64_t far = int64_t(1) << 31;
    if (p->x_stride < p->cols || (!grad && p->y_stride < p->cols) || (grad && p->dy_stride < p->cols) ||
        (grad && p->d_dx && p->dx_stride < p->cols))
        return fail(GNMR_ERR_LAYOUT, "layer norm: a row stride below the row's length");
    if (p->x_stride > far || (!grad && p->y_stride > far) || (grad && (p->dy_stride > far || (p->d_dx && p->dx_stride > far))))
        return fail(GNMR_ERR_LAYOUT, "layer norm: a row stride above 2^31 elements");
    const size_t eb = element_bytes(p->dtype), pb = element_bytes(p->param_dtype), gb = element_bytes(p->grad_dtype);
    if (p->rows > 0 && (!p->d_x || (grad ? !p->d_dy || !p->d_mean || !p->d_rstd : !p->d_y)))
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: NULL pointer");
    if (misaligned(p->d_x, eb) || (!grad && misaligned(p->d_y, eb)) || (grad && (misaligned(p->d_dy, eb) || misaligned(p->d_dx, eb))) ||
        misaligned(p->d_weight, pb) || (!grad && misaligned(p->d_bias, pb)) || misaligned(p->d_mean, 4) || misaligned(p->d_rstd, 4) ||
        (grad && (misaligned(p->d_dweight, gb) || misaligned(p->d_dbias, gb))))
        return fail(GNMR_ERR_LAYOUT, "layer norm: a buffer not aligned to its element size");
    if ((!grad && p->d_y == p->d_x && p->y_stride != p->x_stride) || (grad && p->d_dx && p->d_dx == p->d_dy && p->dx_stride != p->dy_stride))
        return fail(GNMR_ERR_LAYOUT, "layer norm: in place with another stride");
    if (grad && p->rows > 0) {
        const int64_t need = parts_bytes(p);
        if (need && (!p->d_scratch || p->scratch_bytes < need || misaligned(p->d_scratch, 256)))
            return fail(GNMR_ERR_LAYOUT, "layer norm: scratch missing, too small or misaligned");
    }
    return GNMR_OK;
}

Norm norm_of(const gnmr_norm *p)
{
    Norm n = {};
    n.rows = p->rows;
    n.cols = static_cast<int>(p->cols);
    n.inverse = 1.0f / static_cast<float>(p->cols);
    n.eps = static_cast<float>(p->eps);
    n.x = p->d_x;
    n.x_stride = p->x_stride;
    n.w = p->d_weight;
    n.aligned = !misaligned(p->d_weight, 16) && !misaligned(p->d_bias, 16);
    return n;
}

gnmr_status said(cudaError_t e)
{
    if (e == cudaSuccess)
        return GNMR_OK;
    cudaGetLastError();
    return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
}

template <typename T, typename P, int kUnits> cudaError_t launch_warps(const Norm &n, int sms, cudaStream_t st)
{
    const int shared = 8 * n.cols, most = kUnits > 12 ? 2 : kUnits > 6 ? 3 : 4;
    const cudaError_t e = cudaFuncSetAttribute(norm_warp_kernel<T, P, kUnits>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e != cudaSuccess)
        return e;
    const int64_t ctas = std::min<int64_t>((n.rows + kWarps - 1) / kWarps, int64_t(sms) * most);
    norm_warp_kernel<T, P, kUnits><<<static_cast<unsigned>(ctas), kThreads, shared, st>>>(n);
    return cudaGetLastError();
}

template <typename T, typename P, int kUnits, bool kVector> cudaError_t launch_ctas(const Norm &n, int units, int sms, cudaStream_t st)
{
    const int threads = ((units + kUnits - 1) / kUnits + 31) / 32 * 32;
    const int64_t ctas = std::min<int64_t>(n.rows, int64_t(sms) * std::min(2048 / threads, 16));
    norm_cta_kernel<T, P, kUnits, kVector><<<static_cast<unsigned>(ctas), threads, 0, st>>>(n);
    return cudaGetLastError();
}

constexpr int64_t kFewRows = 600;

template <typename T, typename P> cudaError_t forward(const Norm &n, int sms, cudaStream_t st)
{
    constexpr int kN = kIn16<T>;
    const bool vector = n.cols % kN == 0 && rows_of_16(n.x, n.rows, n.x_stride, sizeof(T)) && rows_of_16(n.y, n.rows, n.y_stride, sizeof(T));
    const int units = vector ? n.cols / kN : n.cols;
    if (vector && units <= 24 * 32 && (n.rows > kFewRows || units <= 64)) {
        if (units <= 2 * 32)
            return launch_warps<T, P, 2>(n, sms, st);
        if (units <= 4 * 32)
            return launch_warps<T, P, 4>(n, sms, st);
        if (units <= 8 * 32)
            return launch_warps<T, P, 8>(n, sms, st);
        if (units <= 12 * 32)
            return launch_warps<T, P, 12>(n, sms, st);
        if (units <= 16 * 32)
            return launch_warps<T, P, 16>(n, sms, st);
        if (units <= 20 * 32)
            return launch_warps<T, P, 20>(n, sms, st);
        return launch_warps<T, P, 24>(n, sms, st);
    }
    if (vector && units <= 8 * 1024) {
        if (units <= 1024)
            return launch_ctas<T, P, 1, true>(n, units, sms, st);
        if (units <= 2 * 1024)
            return launch_ctas<T, P, 2, true>(n, units, sms, st);
        if (units <= 4 * 1024)
            return launch_ctas<T, P, 4, true>(n, units, sms, st);
        return launch_ctas<T, P, 8, true>(n, units, sms, st);
    }
    if (!vector && units <= 32 * 1024) {
        if (units <= 4 * 1024)
            return launch_ctas<T, P, 4, false>(n, units, sms, st);
        if (units <= 12 * 1024)
            return launch_ctas<T, P, 12, false>(n, units, sms, st);
        return launch_ctas<T, P, 32, false>(n, units, sms, st);
    }
    norm_any_kernel<T, P><<<static_cast<unsigned>(std::min(n.rows, int64_t(sms) * 8)), kThreads, 0, st>>>(n);
    return cudaGetLastError();
}

template <typename S> cudaError_t launch_grad(Norm &n, int units, int sms, cudaStream_t st)
{
    const int span = ((units + S::kUnits - 1) / S::kUnits + 31) / 32 * 32, groups = S::kMost / span;
    // the groups' sums over the rows pass through the same memory
    const int sums = groups > 1 ? S::kMost * S::kUnits * S::kN * 8 : 0;
    const int shared = std::max(S::kShared / S::kMost * (groups * span), sums);
    const cudaError_t e = cudaFuncSetAttribute(norm_grad_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
    if (e != cudaSuccess)
        return e;
    const int64_t turns = (n.rows + groups * S::kRows - 1) / (groups * S::kRows);
    n.parts = static_cast<int>(std::min<int64_t>(turns, std::min(sms * (S::kVector ? 1 : 2), kMostParts)));
    norm_grad_kernel<S><<<n.parts, groups * span, shared, st>>>(n, span);
    return cudaGetLastError();
}

template <typename T, typename P> cudaError_t backward(Norm &n, int sms, cudaStream_t st)
{
    constexpr int kN = kIn16<T>;
    const bool vector = n.cols % kN == 0 && rows_of_16(n.x, n.rows, n.x_stride, sizeof(T)) && rows_of_16(n.dy, n.rows, n.dy_stride, sizeof(T)) &&
                        (!n.y || rows_of_16(n.y, n.rows, n.y_stride, sizeof(T)));
    if (vector && n.cols <= 640 * 8)
        return launch_grad<Shape<T, P, 8 / kN, kN / 4, 4, 640, true>>(n, n.cols / kN, sms, st);
    if (vector && n.cols <= 512 * 16)
        return launch_grad<Shape<T, P, 16 / kN, 1, kN == 8 ? 6 : 3, 512, true>>(n, n.cols / kN, sms, st);
    if (!vector && n.cols <= 256 * 8)
        return launch_grad<Shape<T, P, 8, 1, 1, 256, false>>(n, n.cols, sms, st);
    if (!vector && n.cols <= 512 * 16)
        return launch_grad<Shape<T, P, 16, 1, 1, 512, false>>(n, n.cols, sms, st);
    if (n.dw || n.db) {
        n.parts = static_cast<int>(std::min<int64_t>(n.rows, std::min(kMostParts, 2 * sms)));
        columns_any_kernel<T><<<dim3((n.cols + kThreads - 1) / kThreads, n.parts), kThreads, 0, st>>>(n);
    }
    if (n.y)                                           // last: it may write over dy
        norm_grad_any_kernel<T, P><<<static_cast<unsigned>(std::min(n.rows, int64_t(sms) * 8)), kThreads, 0, st>>>(n);
    return cudaGetLastError();
}

template <typename T> cudaError_t by_params(const gnmr_norm *p, Norm &n, bool grad, int sms, cudaStream_t st)
{
    if (p->param_dtype == p->dtype)
        return grad ? backward<T, T>(n, sms, st) : forward<T, T>(n, sms, st);
    return grad ? backward<T, float>(n, sms, st) : forward<T, float>(n, sms, st);
}

}  // namespace

extern "C" {

gnmr_status gnmr_layer_norm(const gnmr_norm *p, void *stream)
{
    if (const gnmr_status s = check(p, false))
        return s;
    if (p->rows == 0)
        return GNMR_OK;
    int sms = 0;
    if (const cudaError_t e = current_sms(&sms))
        return said(e);
    Norm n = norm_of(p);
    n.b = p->d_bias;
    n.y = p->d_y;
    n.y_stride = p->y_stride;
    n.mean = p->d_mean;
    n.rstd = p->d_rstd;
    return said(by_type(p->dtype, [&](auto v) { return by_params<decltype(v)>(p, n, false, sms, static_cast<cudaStream_t>(stream)); }));
}

gnmr_status gnmr_layer_norm_scratch_bytes(const gnmr_norm *p, int64_t *bytes)
{
    if (!bytes || !p)
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: NULL argument");
    *bytes = 0;
    if (p->cols < 1 || p->cols > int64_t(1) << 30)
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: cols out of range");
    *bytes = parts_bytes(p);
    return GNMR_OK;
}

gnmr_status gnmr_layer_norm_grad(const gnmr_norm *p, void *stream)
{
    if (const gnmr_status s = check(p, true))
        return s;
    int sms = 0;
    if (const cudaError_t e = current_sms(&sms))
        return said(e);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Norm n = norm_of(p);
    n.dy = p->d_dy;
    n.dy_stride = p->dy_stride;
    n.mean_in = p->d_mean;
    n.rstd_in = p->d_rstd;
    n.y = p->d_dx;
    n.y_stride = p->dx_stride;
    n.dw = p->d_dweight;
    n.db = p->d_dbias;
    n.add = p->add;
    n.part_w = static_cast<float *>(p->d_scratch);
    n.part_b = n.part_w + int64_t(kMostParts) * n.cols;
    cudaError_t e = cudaSuccess;
    if (n.rows > 0)
        e = by_type(p->dtype, [&](auto v) { return by_params<decltype(v)>(p, n, true, sms, st); });
    if (e == cudaSuccess && (n.dw || n.db) && (n.rows > 0 || !n.add))
        e = by_type(p->grad_dtype, [&](auto v) {
            join_kernel<decltype(v)><<<dim3((n.cols + 31) / 32, 2), kThreads, 0, st>>>(n);
            return cudaGetLastError();
        });
    return said(e);
}

}  // extern "C"
