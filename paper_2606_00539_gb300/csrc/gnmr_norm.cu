// Layer norm by row, and its backward pass with the reduction of the parameters' gradients.
//
//   forward   mean, rstd = 1 / sqrt(mean of (x - mean)^2 + eps); y = (x - mean) rstd w + b
//   backward  xh = (x - mean) rstd, t = dy w; dx = rstd (t - mean of t - xh mean of t xh);
//             dw = sum over rows of dy xh, db = sum over rows of dy
//
// Bound by memory: x read and y written; x and dy read and dx written.  A row's sums need all of it before its first
// output, so rows are held on the SM between the two: in registers, the next ones on their way to shared memory (cp.async, each thread
// its own bytes, no wait but its own).  Which threads hold a row goes by its width and alignment:
//
//   forward   up to 4 KB a warp a row; wider ones 2 to 16 warps; odd starts by pairs of elements; few rows a CTA each
//   backward  a CTA has the same columns of every row it takes, so that the sums over the rows stay in its registers; each CTA's go
//             to memory, and a second kernel adds them up in their order.  Rows past 16 KB (32 KB in fp32): these sums by strips
//             of columns, which need no sums over a row, and dx by a kernel like the forward's, up to 64 KB (16-bit rows with
//             an fp32 weight, which lies in shared memory too: 25,088 columns)
//
// What is beyond is read three times, and from memory or L2: backward, wider rows and odd starts past 8,190 columns; forward, rows past 128 KB
// and odd starts past 32,768 columns.  Forward, odd starts past 12,286 columns are read once, by single elements.
//
// Measured (one GB300, bf16 unless said; us, and TB/s of what is read and written once): 16384 x 5120 forward 56 (6.0), backward
// 92 (5.4); 16384 x 2048 20.5 (6.5) and 45; 4096 x 8192 27 (5.0) and 48; 8192 x 5120 fp32 61 (5.5) and 86 (5.8);
// 16384 x 1371, odd starts, 32 (2.8) and 64; 2000 x 16384 29 (4.5) and 80; one row of 5120 2.7 and 8; 2000 x 20001, odd starts, 230 and
// 191; 2048 x 32768, an fp32 weight, 96 and 383.  The backward kernel
// is bound by its threads' latency: 10 warps of 168 registers, instructions issued 42 % of the time.  Two turns in flight at
// once, twice the warps with half the registers, and a scalar in place of the paired arithmetic were slower.
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
    int strip;                                         // columns that a CTA of the backward kernel takes
    int pairs, split;                                  // elements are read two at a time; rows that start alike: every one, or every second
    void *dw, *db;
    int add;
    int aligned;                                       // the parameters start at multiples of 16 bytes
};

constexpr int kThreads = 256;

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

__device__ __forceinline__ float sum_of(Pair p)
{
    const float2 v = apart(p);
    return v.x + v.y;
}

__device__ __forceinline__ float rstd_of(float squares, const Norm &n) { return 1.0f / sqrtf(squares / n.cols + n.eps); }

// A warp a row, which it holds in registers: no barrier, sums by shuffles.  The next row is on its way to
// shared memory meanwhile, where each lane copies its own bytes.  The parameters are there too, as fp32, in groups of
// four of which a warp reads contiguous ones.
template <int kUnits> struct Warps {
    static constexpr int kEach = 8, kCtas = kUnits > 4 ? 2 : 4;    // of a CTA; an SM
};

template <typename T, typename P, int kUnits>
__global__ void __launch_bounds__(32 * Warps<kUnits>::kEach, Warps<kUnits>::kCtas) norm_warp_kernel(const Norm n)
{
    constexpr int kN = kIn16<T>, kQuads = kN / 4, kPairs = kN / 2, kEach = Warps<kUnits>::kEach;
    extern __shared__ float4 quads[];                  // weight: [kQuads][units], then bias; then [kEach][kUnits][32] of 16 bytes
    const int units = n.cols / kN, lane = threadIdx.x & 31;
    const uint32_t mine = shared_address(quads + 2 * kQuads * units) + ((threadIdx.x >> 5) * kUnits * 32 + lane) * 16;
    const auto fetch = [&](int64_t r) {
        if (r < n.rows) {
            const T *const x = static_cast<const T *>(n.x) + r * n.x_stride;
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
                if (lane + u * 32 < units)
                    copy16(mine + u * 512, x + (lane + u * 32) * kN);
        }
        copies_begun();
    };
    int64_t r = int64_t(blockIdx.x) * kEach + (threadIdx.x >> 5);
    fetch(r);
    for (int i = threadIdx.x; i < units; i += 32 * kEach) {
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
    for (; r < n.rows; r += int64_t(gridDim.x) * kEach) {
        copies_done<0>();
        uint4 x[kUnits];
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (lane + u * 32 < units)
                x[u] = load_shared(mine + u * 512);
        fetch(r + int64_t(gridDim.x) * kEach);
        Pair s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (lane + u * 32 < units) {
                Pair f[kPairs];
                widen2<T>(x[u], f);
                s = add2(s, kPairs == 4 ? add2(add2(f[0], f[1]), add2(f[2], f[kPairs - 1])) : add2(f[0], f[1]));
            }
        const float mean = warp_sum(sum_of(s)) / n.cols;
        const Pair minus = both(-mean);
        s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (lane + u * 32 < units) {
                Pair f[kPairs], q = both(0.0f);
                widen2<T>(x[u], f);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    f[j] = add2(f[j], minus);
                    q = fma2(f[j], f[j], q);
                }
                s = add2(s, q);
            }
        const float rstd = rstd_of(warp_sum(sum_of(s)), n);
        if (lane == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
        const Pair by = both(rstd);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = lane + u * 32;
            if (at < units) {
                Pair f[kPairs];
                widen2<T>(x[u], f);
#pragma unroll
                for (int q = 0; q < kQuads; ++q) {
                    const float4 w = quads[q * units + at], b = quads[(kQuads + q) * units + at];
                    f[2 * q] = fma2(mul2(add2(f[2 * q], minus), by), pair(w.x, w.y), pair(b.x, b.y));
                    f[2 * q + 1] = fma2(mul2(add2(f[2 * q + 1], minus), by), pair(w.z, w.w), pair(b.z, b.w));
                }
                store_once(y + at * kN, narrow2<T>(f));
            }
        }
    }
    copies_done<0>();
}

// ---- rows by groups of warps --------------------------------------------------------

// Wider rows: `each` warps of a CTA share one, kUnits times 16 bytes a lane, so that 32 warps are under way with 64
// registers a thread; sums by shuffles, and between the group's warps through shared memory and a barrier of their
// own.  The next row is on its way to shared memory meanwhile, where each lane copies its own bytes.  The
// parameters are there too, as they are, since a CTA takes many rows.
struct Group {
    int each, base, at, step;                          // warps; this group's first; this thread's first unit, and from one to the next
    __device__ __forceinline__ Group(int warps)
        : each(warps), base((threadIdx.x >> 5) / warps * warps), at(threadIdx.x - base * 32), step(32 * warps)
    {
    }
    // The sum of v over the group, the same bits in every thread.  shared: [32] floats that no other sum between two
    // barriers uses.
    __device__ __forceinline__ float sum(float v, float *shared) const
    {
        v = warp_sum(v);
        if (each == 1)
            return v;
        if ((threadIdx.x & 31) == 0)
            shared[threadIdx.x >> 5] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(base / each), "r"(step) : "memory");
        v = shared[base];
        for (int i = 1; i < each; ++i)
            v += shared[base + i];
        return v;
    }
};

// The parameters in shared memory, filled by the CTA: those of unit u in place u, and, where they are wider than the
// rows' elements, the second half of them `units` places behind, so that a warp reads contiguous places.
template <typename T, typename P> __device__ __forceinline__ void fill_params(uint4 *to, const void *from, float none, const Norm &n)
{
    constexpr int kN = kIn16<P>, kEach = static_cast<int>(sizeof(P) / sizeof(T));
    const int places = n.cols / kN, units = places / kEach;
    for (int i = threadIdx.x; i < places; i += blockDim.x) {
        float f[kN];
        params<P, kN>(from, int64_t(i) * kN, none, n.aligned, f);
        to[i / kEach + i % kEach * units] = narrow<P>(f);
    }
}

template <typename T, typename P> __device__ __forceinline__ void params_of(const uint4 *from, int u, int units, Pair (&f)[kIn16<T> / 2])
{
    if constexpr (sizeof(T) == sizeof(P)) {
        widen2<P>(from[u], f);
    } else {
        Pair half[2];
        widen2<P>(from[u], half);
        f[0] = half[0], f[1] = half[1];
        widen2<P>(from[units + u], half);
        f[2] = half[0], f[3] = half[1];
    }
}

// Bytes of shared memory beside the rows.
template <typename P> __host__ __device__ constexpr int params_bytes(int cols, int how_many) { return how_many * cols * static_cast<int>(sizeof(P)); }

template <typename T, typename P, int kUnits, int kThreadsMost>
__global__ void __launch_bounds__(kThreadsMost, 1) norm_group_kernel(const Norm n, int each)
{
    constexpr int kN = kIn16<T>, kPairs = kN / 2;
    extern __shared__ uint4 held[];                    // the weight, the bias; the rows on their way: [warps][kUnits][32]
    __shared__ float shared[2][2][32];                 // by turns: a row's sums are read while the next one's are formed
    const int units = n.cols / kN, of_params = params_bytes<P>(n.cols, 1) / 16;
    const Group g(each);
    const uint4 *const weight = held, *const bias = held + of_params;
    const uint32_t mine = shared_address(held + 2 * of_params) + ((threadIdx.x >> 5) * kUnits * 32 + (threadIdx.x & 31)) * 16;
    const int rows = (blockDim.x >> 5) / each;         // at a time
    const auto fetch = [&](int64_t r) {
        if (r < n.rows) {
            const T *const x = static_cast<const T *>(n.x) + r * n.x_stride;
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
                if (g.at + u * g.step < units)
                    copy16(mine + u * 512, x + (g.at + u * g.step) * kN);
        }
        copies_begun();
    };
    int64_t r = int64_t(blockIdx.x) * rows + g.base / each;
    fetch(r);
    fill_params<T, P>(held, n.w, 1.0f, n);
    fill_params<T, P>(held + of_params, n.b, 0.0f, n);
    __syncthreads();
    int turn = 0;
    for (; r < n.rows; r += int64_t(gridDim.x) * rows, turn ^= 1) {
        copies_done<0>();
        uint4 x[kUnits];
        Pair s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (g.at + u * g.step < units) {
                x[u] = load_shared(mine + u * 512);
                Pair f[kPairs];
                widen2<T>(x[u], f);
                s = add2(s, kPairs == 4 ? add2(add2(f[0], f[1]), add2(f[2], f[kPairs - 1])) : add2(f[0], f[1]));
            }
        fetch(r + int64_t(gridDim.x) * rows);
        const float mean = g.sum(sum_of(s), shared[turn][0]) * n.inverse;
        const Pair minus = both(-mean);
        s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (g.at + u * g.step < units) {
                Pair f[kPairs], q = both(0.0f);
                widen2<T>(x[u], f);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    f[j] = add2(f[j], minus);
                    q = fma2(f[j], f[j], q);
                }
                s = add2(s, q);
            }
        const float rstd = rstd_of(g.sum(sum_of(s), shared[turn][1]), n);
        if (g.at == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
        const Pair by = both(rstd);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = g.at + u * g.step;
            if (at < units) {
                Pair f[kPairs], w[kPairs], b[kPairs];
                widen2<T>(x[u], f);
                params_of<T, P>(weight, at, units, w);
                params_of<T, P>(bias, at, units, b);
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
                    f[j] = fma2(mul2(add2(f[j], minus), by), w[j], b[j]);
                store_once(y + at * kN, narrow2<T>(f));
            }
        }
    }
    copies_done<0>();
}

// Two neighbouring elements of a row, as they are in memory.
template <typename T> using Two = std::conditional_t<sizeof(T) == 2, unsigned, unsigned long long>;

template <typename T> __device__ __forceinline__ Two<T> two_of(T lo, T hi)
{
    struct alignas(2 * sizeof(T)) { T lo, hi; } v{lo, hi};
    return reinterpret_cast<const Two<T> &>(v);
}

template <typename T> __device__ __forceinline__ Pair widen_two(Two<T> v)
{
    if constexpr (sizeof(T) == 4) {
        return v;
    } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        return pair(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    } else {
        const float2 f = __half22float2(reinterpret_cast<const __half2 &>(v));
        return pair(f.x, f.y);
    }
}

// Columns c and c + 1 of a row of `cols`, c from -1 on: which of them there are.
template <typename T> __device__ __forceinline__ Two<T> mask_of(int c, int cols)
{
    constexpr int kBits = 8 * sizeof(T);
    const Two<T> all = ~Two<T>(0);
    return (c >= 0 && c < cols ? all >> kBits : 0) | (c + 1 < cols ? all << kBits : 0);
}

// Both at once.  One of them may be a neighbour outside the row, whose value means nothing: not in the first row or the last,
// beyond which there may be no memory.
template <typename T> __device__ __forceinline__ Two<T> load_two(const T *row, int c, int cols)
{
    return c < cols ? *reinterpret_cast<const Two<T> *>(row + c) : Two<T>(0);
}

template <typename T> __device__ __forceinline__ Two<T> load_each(const T *row, int c, int cols)
{
    const T none = from_f32<T>(0.0f);
    return two_of<T>(c >= 0 && c < cols ? row[c] : none, c + 1 < cols ? row[c + 1] : none);
}

template <typename T> __device__ __forceinline__ void store_two(T *row, int c, int cols, bool together, float2 v)
{
    const T lo = from_f32<T>(v.x), hi = from_f32<T>(v.y);
    if (together && c >= 0 && c + 1 < cols) {
        *reinterpret_cast<Two<T> *>(row + c) = two_of<T>(lo, hi);
        return;
    }
    if (c >= 0 && c < cols)
        row[c] = lo;
    if (c + 1 < cols)
        row[c + 1] = hi;
}

// Whether a row starts at an odd element, seen from places where pairs may be read.
template <typename T> __device__ __forceinline__ int odd_start(const T *row) { return reinterpret_cast<uintptr_t>(row) / sizeof(T) & 1; }

// The same for rows that do not start at multiples of 16 bytes: kTwos pairs a lane, straight to registers.  The parameters are
// there twice, for rows that start at even and at odd elements.
template <typename T, typename P, int kTwos>
__global__ void __launch_bounds__(1024, 1) norm_pairs_kernel(const Norm n, int each)
{
    extern __shared__ uint4 held[];
    __shared__ float shared[2][2][32];
    const int twos = n.cols / 2 + 1;                   // of a row, one that begins early among them
    float2 *const weight = reinterpret_cast<float2 *>(held), *const bias = weight + 2 * twos;
    for (int i = threadIdx.x; i < 2 * twos; i += blockDim.x) {
        const int c = 2 * (i % twos) - i / twos;
        const auto of = [&](const void *p, int c, float none) { return c < 0 || c >= n.cols ? 0.0f : p ? to_f32(static_cast<const P *>(p)[c]) : none; };
        weight[i] = make_float2(of(n.w, c, 1.0f), of(n.w, c + 1, 1.0f));
        bias[i] = make_float2(of(n.b, c, 0.0f), of(n.b, c + 1, 0.0f));
    }
    __syncthreads();
    const Group g(each);
    const int rows = (blockDim.x >> 5) / each;
    int turn = 0;
    for (int64_t r = int64_t(blockIdx.x) * rows + g.base / each; r < n.rows; r += int64_t(gridDim.x) * rows, turn ^= 1) {
        const T *const from = static_cast<const T *>(n.x) + r * n.x_stride;
        const int odd = odd_start(from);
        Two<T> raw[kTwos];
        if (r > 0 && r + 1 < n.rows) {
#pragma unroll
            for (int u = 0; u < kTwos; ++u)
                raw[u] = load_two(from, 2 * (g.at + u * g.step) - odd, n.cols);
        } else {
#pragma unroll
            for (int u = 0; u < kTwos; ++u)
                raw[u] = load_each(from, 2 * (g.at + u * g.step) - odd, n.cols);
        }
        Pair x[kTwos], s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kTwos; ++u) {
            x[u] = widen_two<T>(raw[u] & mask_of<T>(2 * (g.at + u * g.step) - odd, n.cols));
            s = add2(s, x[u]);
        }
        const float mean = g.sum(sum_of(s), shared[turn][0]) * n.inverse;
        s = both(0.0f);
#pragma unroll
        for (int u = 0; u < kTwos; ++u) {
            const int c = 2 * (g.at + u * g.step) - odd;
            x[u] = add2(x[u], both(-mean));
            if (c >= 0 && c + 1 < n.cols) {
                s = fma2(x[u], x[u], s);
            } else {
                const float2 v = apart(x[u]);
                const Pair there = pair(c >= 0 && c < n.cols ? v.x : 0.0f, c + 1 < n.cols ? v.y : 0.0f);
                s = fma2(there, there, s);
            }
        }
        const float rstd = rstd_of(g.sum(sum_of(s), shared[turn][1]), n);
        if (g.at == 0) {
            if (n.mean)
                n.mean[r] = mean;
            if (n.rstd)
                n.rstd[r] = rstd;
        }
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
        const Pair by = both(rstd);
#pragma unroll
        for (int u = 0; u < kTwos; ++u) {
            const int i = g.at + u * g.step;
            if (2 * i - odd < n.cols) {
                const float2 w = weight[odd * twos + i], b = bias[odd * twos + i];
                store_two(y, 2 * i - odd, n.cols, true, apart(fma2(mul2(x[u], by), pair(w.x, w.y), pair(b.x, b.y))));
            }
        }
    }
}

// dx alone, likewise: rows too wide for one CTA to hold their columns' sums.
template <typename T, typename P, int kUnits, int kThreadsMost>
__global__ void __launch_bounds__(kThreadsMost, 1) norm_dx_kernel(const Norm n, int each)
{
    constexpr int kN = kIn16<T>, kPairs = kN / 2;
    extern __shared__ uint4 held[];                    // the weight; the rows of x and dy: [warps][2][kUnits][32]
    __shared__ float shared[2][2][32];
    const int units = n.cols / kN, of_params = params_bytes<P>(n.cols, 1) / 16;
    const Group g(each);
    const uint32_t mine = shared_address(held + of_params) + ((threadIdx.x >> 5) * 2 * kUnits * 32 + (threadIdx.x & 31)) * 16;
    const int rows = (blockDim.x >> 5) / each;
    const auto fetch = [&](int64_t r) {
        if (r < n.rows) {
            const T *const x = static_cast<const T *>(n.x) + r * n.x_stride, *const dy = static_cast<const T *>(n.dy) + r * n.dy_stride;
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
                if (g.at + u * g.step < units) {
                    copy16(mine + u * 512, x + (g.at + u * g.step) * kN);
                    copy16(mine + (kUnits + u) * 512, dy + (g.at + u * g.step) * kN);
                }
        }
        copies_begun();
    };
    int64_t r = int64_t(blockIdx.x) * rows + g.base / each;
    fetch(r);
    fill_params<T, P>(held, n.w, 1.0f, n);
    __syncthreads();
    int turn = 0;
    for (; r < n.rows; r += int64_t(gridDim.x) * rows, turn ^= 1) {
        const float mean = n.mean_in[r], by = n.rstd_in[r];
        copies_done<0>();
        const Pair minus = both(-mean), rstd = both(by);
        uint4 x[kUnits], dy[kUnits];
        Pair s = both(0.0f), q = both(0.0f);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            if (g.at + u * g.step < units) {
                x[u] = load_shared(mine + u * 512);
                dy[u] = load_shared(mine + (kUnits + u) * 512);
                Pair f[kPairs], d[kPairs], w[kPairs];
                widen2<T>(x[u], f);
                widen2<T>(dy[u], d);
                params_of<T, P>(held, g.at + u * g.step, units, w);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    const Pair t = mul2(d[j], w[j]);
                    s = add2(s, t);
                    q = fma2(t, mul2(add2(f[j], minus), rstd), q);
                }
            }
        fetch(r + int64_t(gridDim.x) * rows);
        const Pair minus_m1 = both(-(g.sum(sum_of(s), shared[turn][0]) * n.inverse) * by), minus_m2 = both(-(g.sum(sum_of(q), shared[turn][1]) * n.inverse));
        T *const dx = static_cast<T *>(n.y) + r * n.y_stride;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = g.at + u * g.step;
            if (at < units) {
                Pair f[kPairs], d[kPairs], w[kPairs];
                widen2<T>(x[u], f);
                widen2<T>(dy[u], d);
                params_of<T, P>(held, at, units, w);
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
                    f[j] = fma2(fma2(mul2(add2(f[j], minus), rstd), minus_m2, mul2(d[j], w[j])), rstd, minus_m1);
                store_once(dx + at * kN, narrow2<T>(f));
            }
        }
    }
    copies_done<0>();
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

// kV sums (2, 4 or 8) over a warp at once: in the end lanes of 32 / kV have one each, lane l the (l kV / 32)-th.
template <int kV> __device__ __forceinline__ float warp_sums(const float (&v)[kV])
{
    const int lane = threadIdx.x & 31;
    const bool high = lane & 16;
    float s;
    if constexpr (kV == 2) {
        s = (high ? v[1] : v[0]) + __shfl_xor_sync(~0u, high ? v[0] : v[1], 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
            s += __shfl_xor_sync(~0u, s, o);
        return s;
    } else {
        float half[kV / 2];
#pragma unroll
        for (int i = 0; i < kV / 2; ++i)
            half[i] = (high ? v[kV / 2 + i] : v[i]) + __shfl_xor_sync(~0u, high ? v[i] : v[kV / 2 + i], 16);
        const bool second = lane & 8;
        if constexpr (kV == 4) {
            s = (second ? half[1] : half[0]) + __shfl_xor_sync(~0u, second ? half[0] : half[1], 8);
            s += __shfl_xor_sync(~0u, s, 4);
        } else {
            const float a = (second ? half[2] : half[0]) + __shfl_xor_sync(~0u, second ? half[0] : half[2], 8);
            const float b = (second ? half[3] : half[1]) + __shfl_xor_sync(~0u, second ? half[1] : half[3], 8);
            const bool third = lane & 4;
            s = (third ? b : a) + __shfl_xor_sync(~0u, third ? a : b, 4);
        }
    }
    s += __shfl_xor_sync(~0u, s, 2);
    return s + __shfl_xor_sync(~0u, s, 1);
}

// How the backward kernel takes rows: a group of `span` threads has kRows of them a turn, as many groups as there are
// threads for.  A thread has the same columns of every row, in kPairs pairs: kUnits times 16 bytes, or, where rows do not start at
// multiples of 16 bytes, pairs of elements `span` apart (a CTA then takes rows that start alike, at even elements or at odd ones:
// its pairs are the same columns of each).  So the sums over the rows stay in its registers; rows on their way
// are in shared memory, where each thread copies its own bytes (no barrier for that), kTurns turns ahead.  One barrier a
// turn, for the row sums; across it a thread holds what it read as it was, and widens it twice: several rows a turn
// share what a turn costs besides.
template <typename T_, typename P_, int kColumns, int kRows_, int kTurns_, int kMost_, int kCtas_, bool kVector_> struct Shape {
    using T = T_;
    using P = P_;
    static constexpr int kRows = kRows_, kTurns = kTurns_, kMost = kMost_, kCtas = kCtas_;
    static constexpr bool kVector = kVector_;
    static constexpr int kN = kVector ? kIn16<T> : 2;  // elements of a unit
    static constexpr int kUnits = kColumns / kN, kPairs = kColumns / 2, kHalf = kN / 2;
    static constexpr int kV = 2 * kRows;               // row sums a turn
    static constexpr int kTurnBytes = kVector ? kRows * kUnits * 2 * 16 : 0;       // of a thread
    using Raw = std::conditional_t<kVector, uint4, Two<T>>;
};

// The first column of pair k of a thread at `at` of `span`; odd: rows start at odd elements.
template <typename S> __device__ __forceinline__ int column(int k, int at, int span, int odd)
{
    if (S::kVector)
        return (at + (2 * k / S::kN) * span) * S::kN + 2 * k % S::kN;
    return 2 * (at + k * span) - odd;
}

template <typename S> __device__ __forceinline__ void pairs_of(const typename S::Raw &raw, Pair (&f)[S::kHalf])
{
    if constexpr (S::kVector)
        widen2<typename S::T>(raw, f);
    else
        f[0] = widen_two<typename S::T>(raw);
}

template <typename S> __global__ void __launch_bounds__(S::kMost, S::kCtas) norm_grad_kernel(const Norm n, int span)
{
    using T = typename S::T;
    using P = typename S::P;
    constexpr int kN = S::kN, kUnits = S::kUnits, kPairs = S::kPairs, kHalf = S::kHalf, kRows = S::kRows, kV = S::kV, kMost = S::kMost;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    extern __shared__ __align__(16) uint8_t bytes[];
    __shared__ float sums[2][kMost / 32][kV];
    const int col0 = blockIdx.y * n.strip, cols = min(n.strip, n.cols - col0);
    const int groups = blockDim.x / span, group = threadIdx.x / span, at = threadIdx.x - group * span;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = span >> 5, warp0 = group * warps;
    // of rows that start alike (all of them, or every second) the first, how many, and the CTAs that share them
    const int first = blockIdx.x % n.split, ctas = gridDim.x / n.split;
    const int64_t rows = (n.rows - first + n.split - 1) / n.split;
    const int64_t x_stride = n.x_stride * n.split, dy_stride = n.dy_stride * n.split, y_stride = n.y_stride * n.split;
    const int turns = static_cast<int>((rows + groups * kRows - 1) / (groups * kRows));
    int turn = blockIdx.x / n.split;
    // the first row of this group's next turn, of its next copies, and where these lie
    int64_t row = (int64_t(turn) * groups + group) * kRows, ahead = row;
    const int64_t step = int64_t(ctas) * groups * kRows;
    const T *x = static_cast<const T *>(n.x) + first * n.x_stride + row * x_stride + col0 + (S::kVector ? at * kN : 0);
    const T *dy = static_cast<const T *>(n.dy) + first * n.dy_stride + row * dy_stride + col0 + (S::kVector ? at * kN : 0);
    T *dx = n.y ? static_cast<T *>(n.y) + first * n.y_stride + row * y_stride + col0 + (S::kVector ? at * kN : 0) : nullptr;
    const int odd = !S::kVector && n.pairs ? odd_start(static_cast<const T *>(n.x) + first * n.x_stride + col0) : 0;
    // 16-byte places of this thread: turn, row, unit, x or dy; those of a warp side by side
    const uint32_t mine = shared_address(bytes) + threadIdx.x * 16, next = blockDim.x * 16;
    const auto place = [&](int slot, int i, int u) { return mine + ((slot * kRows + i) * kUnits + u) * 2 * next; };
    const auto fetch = [&](int slot) {
        if (S::kVector) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (ahead + i < rows)
#pragma unroll
                    for (int u = 0; u < kUnits; ++u)
                        if ((at + u * span) * kN < cols) {
                            copy16(place(slot, i, u), x + i * x_stride + u * span * kN);
                            copy16(place(slot, i, u) + next, dy + i * dy_stride + u * span * kN);
                        }
            ahead += step;
            x += step * x_stride;
            dy += step * dy_stride;
        }
        copies_begun();
    };
#pragma unroll
    for (int s = 0; s < S::kTurns; ++s) {
        if (S::kVector)                                // columns that there are not: zeros
#pragma unroll
            for (int u = 0; u < kUnits; ++u)
                if ((at + u * span) * kN >= cols)
                    for (int i = 0; i < kRows; ++i) {
                        store_shared(place(s, i, u), make_uint4(0, 0, 0, 0));
                        store_shared(place(s, i, u) + next, make_uint4(0, 0, 0, 0));
                    }
        fetch(s);
    }
    Pair w[kPairs], dw[kPairs], db[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const int c = column<S>(k, at, span, odd);
        const P *const p = n.w ? static_cast<const P *>(n.w) + col0 : nullptr;
        const auto weight = [&](int c) { return c < 0 || c >= cols ? 0.0f : p ? to_f32(p[c]) : 1.0f; };
        w[k] = pair(weight(c), weight(c + 1));
        dw[k] = db[k] = both(0.0f);
    }
    // lane l has the statistics of row l % kRows of the (l / kRows)-th turn from here, reloaded when they are used up
    constexpr int kStored = 32 / kRows;
    float minus_of = 0.0f, rstd_of = 0.0f;
    int slot = 0, parity = 0, stored = 0;
    typename S::Raw a[kRows][kUnits], d[kRows][kUnits];
    const auto elements = [&](auto &a, auto &d, int64_t r) {
#pragma unroll
        for (int i = 0; i < kRows; ++i)
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int c = column<S>(u, at, span, odd);
                if (r + i >= rows)
                    continue;
                if (n.pairs && r + i > 0 && r + i + 1 < rows) {
                    a[i][u] = load_two(x + i * x_stride, c, cols);
                    d[i][u] = load_two(dy + i * dy_stride, c, cols);
                } else {
                    a[i][u] = load_each(x + i * x_stride, c, cols);
                    d[i][u] = load_each(dy + i * dy_stride, c, cols);
                }
            }
    };
    typename S::Raw there[S::kVector ? 1 : kUnits];
    if constexpr (!S::kVector) {
        elements(a, d, row);
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
            there[u] = mask_of<T>(column<S>(u, at, span, odd), cols);
    }
    for (; turn < turns; turn += ctas, row += step, stored = (stored + 1) % kStored) {
        if (stored == 0) {
            const int64_t r = row + lane / kRows * step + lane % kRows;
            if (r < rows)
                minus_of = -n.mean_in[r * n.split + first], rstd_of = n.rstd_in[r * n.split + first];
        }
        Pair minus[kRows], rstd[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            minus[i] = both(__shfl_sync(~0u, minus_of, stored * kRows + i));
            rstd[i] = both(__shfl_sync(~0u, rstd_of, stored * kRows + i));
        }
        copies_done<S::kTurns - 1>();
        float v[kV];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            Pair s = both(0.0f), q = both(0.0f);
            if (row + i < rows)
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                    if constexpr (S::kVector) {
                        a[i][u] = load_shared(place(slot, i, u));
                        d[i][u] = load_shared(place(slot, i, u) + next);
                    } else {
                        a[i][u] &= there[u];
                        d[i][u] &= there[u];
                    }
                    Pair f[kHalf], g[kHalf];
                    pairs_of<S>(a[i][u], f);
                    pairs_of<S>(d[i][u], g);
#pragma unroll
                    for (int j = 0; j < kHalf; ++j) {
                        const Pair t = mul2(g[j], w[u * kHalf + j]);
                        s = add2(s, t);
                        q = fma2(t, mul2(add2(f[j], minus[i]), rstd[i]), q);
                    }
                }
            v[2 * i] = sum_of(s);
            v[2 * i + 1] = sum_of(q);
        }
        typename S::Raw a2[S::kVector ? 1 : kRows][kUnits], d2[S::kVector ? 1 : kRows][kUnits];
        if constexpr (!S::kVector) {                   // a turn ahead too, in registers
            x += step * x_stride;
            dy += step * dy_stride;
            elements(a2, d2, row + step);
        }
        fetch(slot);
        if (++slot == S::kTurns)
            slot = 0;
        // the sums of every warp, and then of the group's warps in their order
        constexpr int kLanes = 32 / kV;
        float of_group = warp_sums<kV>(v);
        if (warps > 1 && dx) {
            if (lane % kLanes == 0)
                sums[parity][warp][lane / kLanes] = of_group;
            __syncthreads();
            of_group = 0.0f;
            for (int i = lane % kLanes; i < warps; i += kLanes)
                of_group += sums[parity][warp0 + i][lane / kLanes];
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1)
                of_group += __shfl_xor_sync(~0u, of_group, o);
            parity ^= 1;
        }
        of_group *= n.inverse;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const float m1 = __shfl_sync(~0u, of_group, 2 * i * kLanes), m2 = __shfl_sync(~0u, of_group, (2 * i + 1) * kLanes);
            if (row + i >= rows)
                continue;
            const Pair minus_m2 = both(-m2), minus_m1 = mul2(both(-m1), rstd[i]);
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                Pair f[kHalf], g[kHalf];
                pairs_of<S>(a[i][u], f);
                pairs_of<S>(d[i][u], g);
#pragma unroll
                for (int j = 0; j < kHalf; ++j) {
                    const int k = u * kHalf + j;
                    const Pair xh = mul2(add2(f[j], minus[i]), rstd[i]);
                    dw[k] = fma2(g[j], xh, dw[k]);
                    db[k] = add2(db[k], g[j]);
                    f[j] = fma2(fma2(xh, minus_m2, mul2(g[j], w[k])), rstd[i], minus_m1);
                }
                if (!dx)
                    continue;
                if constexpr (S::kVector) {
                    if ((at + u * span) * kN < cols)
                        store_once(dx + i * y_stride + u * span * kN, narrow2<T>(f));
                } else {
                    store_two(dx + i * y_stride, column<S>(u, at, span, odd), cols, n.pairs, apart(f[0]));
                }
            }
        }
        if (dx)
            dx += step * y_stride;
        if constexpr (!S::kVector)
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int u = 0; u < kUnits; ++u)
                    a[i][u] = a2[i][u], d[i][u] = d2[i][u];
    }
    copies_done<0>();
    if (!n.dw && !n.db)
        return;
    // the groups' sums over their rows, added up in their order
    if (groups > 1) {
        ulonglong2 *const all = reinterpret_cast<ulonglong2 *>(bytes);       // [pair][thread]
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
            all[k * blockDim.x + threadIdx.x] = make_ulonglong2(dw[k], db[k]);
        __syncthreads();
        if (group)
            return;
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
            for (int g = 1; g < groups; ++g) {
                const ulonglong2 o = all[k * blockDim.x + g * span + at];
                dw[k] = add2(dw[k], o.x);
                db[k] = add2(db[k], o.y);
            }
    }
    float *const part_w = n.part_w + int64_t(blockIdx.x) * n.cols + col0, *const part_b = n.part_b + int64_t(blockIdx.x) * n.cols + col0;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const int c = column<S>(k, at, span, odd);
        if (S::kVector) {                              // pairs of neighbours, an even number of columns
            if (c < cols) {
                *reinterpret_cast<Pair *>(part_w + c) = dw[k];
                *reinterpret_cast<Pair *>(part_b + c) = db[k];
            }
        } else {
            store_two(part_w, c, cols, false, apart(dw[k]));
            store_two(part_b, c, cols, false, apart(db[k]));
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
constexpr int kJoinWarps = 16;

template <typename G>
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const Norm n)
{
    __shared__ float shared[kJoinWarps][32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    G *const to = static_cast<G *>(blockIdx.y ? n.db : n.dw);
    if (!to)
        return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (i < n.cols) {
        const float *const part = (blockIdx.y ? n.part_b : n.part_w) + i;
        constexpr int kBatch = 10;                     // loads on their way
        for (int p0 = warp; p0 < n.parts; p0 += kBatch * kJoinWarps) {
            float v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int p = p0 + k * kJoinWarps;
                v[k] = p < n.parts ? __ldcg(part + int64_t(p) * n.cols) : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                s += v[k];
        }
    }
    shared[warp][lane] = s;
    __syncthreads();
    if (warp || i >= n.cols)
        return;
#pragma unroll
    for (int k = 1; k < kJoinWarps; ++k)
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

// The parts that any kernel makes of so many rows: a row each at most, and where every second row starts alike the odd and the
// even ones' parts are as many, one more than the rows where these are odd.
int64_t most_parts(int64_t rows) { return rows ? std::min<int64_t>(rows + 1, kMostParts) : 0; }

int64_t parts_bytes(const gnmr_norm *p)
{
    return p->d_dweight || p->d_dbias ? (2 * most_parts(p->rows) * p->cols * 4 + 255) / 256 * 256 : 0;
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

// How many warps share a row of `units`, at most kMost units a lane: a power of two, or 0 where 16 do not hold it.
int warps_for(int units, int most)
{
    int each = 1;
    while (each <= 16 && (units + 32 * each - 1) / (32 * each) > most)
        each *= 2;
    return each <= 16 ? each : 0;
}

template <typename T, typename P, int kUnits> cudaError_t launch_warps(const Norm &n, int sms, cudaStream_t st)
{
    using W = Warps<kUnits>;
    const int shared = 8 * n.cols + W::kEach * kUnits * 512;
    const cudaError_t e = allow_shared<norm_warp_kernel<T, P, kUnits>>();
    if (e != cudaSuccess)
        return e;
    const int64_t ctas = std::min<int64_t>((n.rows + W::kEach - 1) / W::kEach, int64_t(sms) * W::kCtas);
    norm_warp_kernel<T, P, kUnits><<<static_cast<unsigned>(ctas), 32 * W::kEach, shared, st>>>(n);
    return cudaGetLastError();
}

// kKernel in CTAs of up to `threads`, as many as have shared memory beside the parameters, and as few as give every SM rows.
template <auto kKernel>
cudaError_t launch_groups(const Norm &n, int each, int threads, int params, int held, int sms, cudaStream_t st)
{
    while (threads > 32 * each && (params + threads * held > kSharedMost || n.rows * 32 * each <= int64_t(threads) / 2 * sms))
        threads /= 2;
    const int shared = params + threads * held;
    const cudaError_t e = allow_shared<kKernel>();
    if (e != cudaSuccess)
        return e;
    const int rows = threads / (32 * each);
    const int64_t ctas = std::min<int64_t>((n.rows + rows - 1) / rows, int64_t(sms));
    kKernel<<<static_cast<unsigned>(ctas), threads, shared, st>>>(n, each);
    return cudaGetLastError();
}

// 16-byte units a lane of the forward kernel, by 1,024 threads with 64 registers each.  16384 x 5120: four warps a row, 5 units, 56 us; one
// warp, 20 units, 16 warps with 128 registers 58.
constexpr int kMostUnits = 5;

template <typename T, typename P> cudaError_t launch_forward(const Norm &n, int units, int sms, cudaStream_t st)
{
    const int each = warps_for(units, kMostUnits), lane = (units + 32 * each - 1) / (32 * each);
    const auto go = [&](auto k) {
        constexpr int kUnits = decltype(k)::value;
        return launch_groups<norm_group_kernel<T, P, kUnits, 1024>>(n, each, 1024, params_bytes<P>(n.cols, 2), kUnits * 16, sms, st);
    };
    if (lane <= 3)
        return go(std::integral_constant<int, 3>());
    if (lane <= 4)
        return go(std::integral_constant<int, 4>());
    return go(std::integral_constant<int, 5>());
}

template <typename T, typename P> cudaError_t launch_dx(const Norm &n, int units, int sms, cudaStream_t st)
{
    const int each = warps_for(units, 8);
    return launch_groups<norm_dx_kernel<T, P, 8, 512>>(n, each, 512, params_bytes<P>(n.cols, 1), 2 * 8 * 16, sms, st);
}

template <typename T, typename P, int kUnits, bool kVector> cudaError_t launch_ctas(const Norm &n, int units, int sms, cudaStream_t st)
{
    const int threads = ((units + kUnits - 1) / kUnits + 31) / 32 * 32;
    const int64_t ctas = std::min<int64_t>(n.rows, int64_t(sms) * std::min(2048 / threads, 32));
    norm_cta_kernel<T, P, kUnits, kVector><<<static_cast<unsigned>(ctas), threads, 0, st>>>(n);
    return cudaGetLastError();
}

// Up to here a CTA a row, without laying the parameters down first.  5120 columns: 200 rows 3.5 us so, 600 5.9 and by groups of warps 5.2,
// 1200 10.9 and 7.0; 2048: 600 3.2 and 3.7, 1200 5.2 and 3.9; 1371 at odd starts: 600 5.5 and 5.2.
constexpr int64_t kFewRows = 400;

// Whether the rows of two matrices begin at odd elements alike, and all elements where their size says.
bool alike(const void *a, int64_t a_stride, const void *b, int64_t b_stride, size_t bytes)
{
    return ((reinterpret_cast<uintptr_t>(a) ^ reinterpret_cast<uintptr_t>(b)) / bytes & 1) == 0 && ((a_stride ^ b_stride) & 1) == 0;
}

template <typename T, typename P> cudaError_t forward(const Norm &n, int sms, cudaStream_t st)
{
    constexpr int kN = kIn16<T>;
    const bool vector = n.cols % kN == 0 && rows_of_16(n.x, n.rows, n.x_stride, sizeof(T)) && rows_of_16(n.y, n.rows, n.y_stride, sizeof(T));
    const int units = vector ? n.cols / kN : n.cols;
    if (vector && units <= 8 * 32 && (n.rows > kFewRows || units <= 64)) {
        if (units <= 2 * 32)
            return launch_warps<T, P, 2>(n, sms, st);
        if (units <= 4 * 32)
            return launch_warps<T, P, 4>(n, sms, st);
        return launch_warps<T, P, 8>(n, sms, st);
    }
    const int each = vector ? warps_for(units, kMostUnits) : 0;
    // a row's CTA of its own where there are few rows: no parameters to be laid down first
    if (each && params_bytes<P>(n.cols, 2) + 32 * each * kMostUnits * 16 <= kSharedMost && n.rows > kFewRows)
        return launch_forward<T, P>(n, units, sms, st);
    if (vector && units <= 8 * 1024) {
        if (units <= 1024)
            return launch_ctas<T, P, 1, true>(n, units, sms, st);
        if (units <= 2 * 1024)
            return launch_ctas<T, P, 2, true>(n, units, sms, st);
        if (units <= 4 * 1024)
            return launch_ctas<T, P, 4, true>(n, units, sms, st);
        return launch_ctas<T, P, 8, true>(n, units, sms, st);
    }
    constexpr int kTwos = 12;
    const int twos = units / 2 + 1, of_row = vector ? 0 : warps_for(twos, kTwos);
    if (of_row && alike(n.x, n.x_stride, n.y, n.y_stride, sizeof(T)) && 32 * twos <= kSharedMost && n.rows > kFewRows) {
        const int bytes = 32 * twos;
        return twos <= 2 * 32   ? launch_groups<norm_pairs_kernel<T, P, 2>>(n, of_row, 1024, bytes, 0, sms, st)
               : twos <= 6 * 32 ? launch_groups<norm_pairs_kernel<T, P, 6>>(n, of_row, 1024, bytes, 0, sms, st)
                                : launch_groups<norm_pairs_kernel<T, P, kTwos>>(n, of_row, 1024, bytes, 0, sms, st);
    }
    if (!vector && units <= 32 * 1024) {
        if (n.rows <= kFewRows && units <= 4 * 1024)
            return launch_ctas<T, P, 4, false>(n, units, sms, st);
        if (units <= 8 * 1024)
            return launch_ctas<T, P, 8, false>(n, units, sms, st);
        if (units <= 12 * 1024)
            return launch_ctas<T, P, 12, false>(n, units, sms, st);
        return launch_ctas<T, P, 32, false>(n, units, sms, st);
    }
    norm_any_kernel<T, P><<<static_cast<unsigned>(std::min(n.rows, int64_t(sms) * 8)), kThreads, 0, st>>>(n);
    return cudaGetLastError();
}

// strip: columns that a CTA takes, all of them unless n.y is NULL.
template <typename S> cudaError_t launch_grad(Norm &n, int strip, int sms, cudaStream_t st)
{
    // (a row at odd elements has one more pair)
    const int units = S::kVector ? strip / S::kN : strip / 2 + 1, span = ((units + S::kUnits - 1) / S::kUnits + 31) / 32 * 32, groups = S::kMost / span;
    // the groups' sums over the rows pass through the same memory
    const int sums = groups > 1 ? groups * span * S::kPairs * 16 : 0;
    const int shared = std::max(S::kTurnBytes * S::kTurns * groups * span, sums);
    const cudaError_t e = allow_shared<norm_grad_kernel<S>>();
    if (e != cudaSuccess)
        return e;
    n.pairs = !S::kVector && alike(n.x, n.x_stride, n.dy, n.dy_stride, sizeof(typename S::T)) &&
              (!n.y || alike(n.x, n.x_stride, n.y, n.y_stride, sizeof(typename S::T)));
    n.split = n.pairs && n.x_stride % 2 && n.rows > 1 ? 2 : 1;
    const int64_t turns = ((n.rows + n.split - 1) / n.split + groups * S::kRows - 1) / (groups * S::kRows);
    const int strips = (n.cols + strip - 1) / strip;
    n.parts = n.split * static_cast<int>(std::min<int64_t>(turns, std::max(std::min(sms * S::kCtas / strips, kMostParts) / n.split, 1)));
    n.strip = strip;
    norm_grad_kernel<S><<<dim3(n.parts, strips), groups * span, shared, st>>>(n, span);
    return cudaGetLastError();
}

template <typename T, typename P> cudaError_t backward(Norm &n, int sms, cudaStream_t st)
{
    constexpr int kN = kIn16<T>;
    const bool vector = n.cols % kN == 0 && rows_of_16(n.x, n.rows, n.x_stride, sizeof(T)) && rows_of_16(n.dy, n.rows, n.dy_stride, sizeof(T)) &&
                        (!n.y || rows_of_16(n.y, n.rows, n.y_stride, sizeof(T)));
    // columns a thread, rows a turn, turns ahead, threads: 16384 x 5120 bf16 8, 2, 4, 640 98 us; 16, 2, 4, 320 99.5; 16, 4, 2, 320 92.  Narrow
    // rows with 16 columns a thread leave lanes idle: 60,000 x 64 32 us, with 8 20.
    if (vector && n.cols <= 256)
        return launch_grad<Shape<T, P, 8, kN / 4, 4, 640, 1, true>>(n, n.cols, sms, st);
    if (vector && n.cols <= 320 * 16)
        return launch_grad<Shape<T, P, 16, kN / 2, 2, 320, 1, true>>(n, n.cols, sms, st);
    if (vector && n.cols <= 512 * 16)
        return launch_grad<Shape<T, P, 16, kN / 4, 3, 512, 1, true>>(n, n.cols, sms, st);
    if (!vector && n.cols <= 256 * 8 - 2)
        return launch_grad<Shape<T, P, 8, 1, 1, 256, 2, false>>(n, n.cols, sms, st);
    if (!vector && n.cols <= 512 * 16 - 2)
        return launch_grad<Shape<T, P, 16, 1, 1, 512, 1, false>>(n, n.cols, sms, st);
    const int units = n.cols / kN, each = vector ? warps_for(units, 8) : 0;
    if (each && params_bytes<P>(n.cols, 1) + 32 * each * 2 * 8 * 16 <= kSharedMost) {
        cudaError_t e = cudaSuccess;
        void *const dx = n.y;
        if (n.dw || n.db) {                            // strips of columns need no sums over rows
            n.y = nullptr;
            const int strips = (n.cols + 5119) / 5120;
            e = launch_grad<Shape<T, P, 16, kN / 2, 2, 320, 1, true>>(n, (n.cols / kN + strips - 1) / strips * kN, sms, st);
            n.y = dx;
        }
        return e == cudaSuccess && dx ? launch_dx<T, P>(n, units, sms, st) : e;      // last: it may write over dy
    }
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
    if (p->rows < 0 || p->rows > INT32_MAX || p->cols < 1 || p->cols > int64_t(1) << 30)
        return fail(GNMR_ERR_INVALID_ARG, "layer norm: rows or cols out of range");
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
    n.part_b = n.part_w + most_parts(n.rows) * n.cols;
    cudaError_t e = cudaSuccess;
    if (n.rows > 0)
        e = by_type(p->dtype, [&](auto v) { return by_params<decltype(v)>(p, n, true, sms, st); });
    if (e == cudaSuccess && (n.dw || n.db) && (n.rows > 0 || !n.add))
        e = by_type(p->grad_dtype, [&](auto v) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((n.cols + 31) / 32, 2);
            cfg.blockDim = dim3(32 * kJoinWarps);
            cfg.stream = st;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr.val.programmaticStreamSerializationAllowed = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            return cudaLaunchKernelEx(&cfg, join_kernel<decltype(v)>, n);
        });
    return said(e);
}

}  // extern "C"
