// 8-bit codes with one scale for every row, or for every column and then
// transposed: the operands of the low-cost path's products.
//
//   amax = max |x|, up = 127 * (1 / amax), scale = amax / 127, q = rint(x * up)
//
// in fp32, by row or by column, each operation rounded.  Both are bound by memory: 3 bytes an element
// from 16-bit inputs.  Measured on 64 x 1408 x 2048 bf16 (553 MB): by row 85 us, 6.5 TB/s; by column
// 93 us, 5.9 TB/s.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "gnmr.h"
#include "gnmr_internal.h"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr unsigned kInfBits = 0x7f800000u;

template <typename T> __device__ __forceinline__ float to_f32(T v) { return static_cast<float>(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

// |v|'s bits order as its value does, infinities and then NaNs last.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct Scale {
    float up, down;
    unsigned keep;                                   // 0 where the codes are 0 whatever the values
};

__device__ __forceinline__ Scale scale_of(unsigned amax_bits)
{
    if (amax_bits >= kInfBits)
        return {0.0f, __uint_as_float(0x7fc00000u), 0u};
    const float amax = __uint_as_float(amax_bits);
    const float up = __fmul_rn(127.0f, __frcp_rn(amax));
    if (!(magnitude(up) < kInfBits))                 // amax is 0, or 127 / amax is past fp32
        return {0.0f, 0.0f, 0u};
    return {up, __fdiv_rn(amax, 127.0f), ~0u};
}

// v * up, rounded, plus 1.5 * 2^23, rounded: halves to even at whole numbers, which are
// then the low bits of the sum.  (Conversions to integers run at an eighth of the rate.
// Products two at a time; sums are left single: a packed product and a packed sum came out
// of the assembler as one operation with one rounding: values just below 63.5 as 63 for 64.)
constexpr float kWhole = 12582912.0f;

__device__ __forceinline__ unsigned whole(float v) { return __float_as_uint(__fadd_rn(v, kWhole)); }

__device__ __forceinline__ void whole2(float a, float b, float up_a, float up_b, unsigned &wa, unsigned &wb)
{
    float pa, pb;
    asm("{\n.reg .b64 v, u;\nmov.b64 v, {%2, %3};\nmov.b64 u, {%4, %5};\n"
        "mul.rn.f32x2 v, v, u;\nmov.b64 {%0, %1}, v;\n}"
        : "=f"(pa), "=f"(pb)
        : "f"(a), "f"(b), "f"(up_a), "f"(up_b));
    wa = whole(pa);
    wb = whole(pb);
}

__device__ __forceinline__ unsigned low_bytes(unsigned a, unsigned b, unsigned c, unsigned d)
{
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

__device__ __forceinline__ int8_t code_of(float v, const Scale &s)
{
    return static_cast<int8_t>(whole(__fmul_rn(v, s.up)) & s.keep);
}

// 16 bytes of a row, and how many elements they are.
template <typename T> struct Vec {
    static constexpr int kN = 16 / sizeof(T);
    uint4 w;
};

template <typename T> __device__ __forceinline__ void widen(const Vec<T> &v, float (&f)[Vec<T>::kN])
{
    const unsigned w[4] = {v.w.x, v.w.y, v.w.z, v.w.w};
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

// The running maximum of magnitudes in the inputs' own bits, 16-bit types two at a time.
template <typename T> __device__ __forceinline__ void add_max(unsigned &m, const Vec<T> &v)
{
    if constexpr (sizeof(T) == 4) {
        m = __vimax3_u32(m, v.w.x & 0x7fffffffu, v.w.y & 0x7fffffffu);
        m = __vimax3_u32(m, v.w.z & 0x7fffffffu, v.w.w & 0x7fffffffu);
    } else {
        m = __vimax3_u16x2(m, v.w.x & 0x7fff7fffu, v.w.y & 0x7fff7fffu);
        m = __vimax3_u16x2(m, v.w.z & 0x7fff7fffu, v.w.w & 0x7fff7fffu);
    }
}

// The same as fp32 bits; of the larger half.
template <typename T> __device__ __forceinline__ unsigned half_bits(unsigned half)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>)
        return half << 16;
    else
        return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(half))));
}

template <typename T> __device__ __forceinline__ unsigned max_bits(unsigned m)
{
    if constexpr (sizeof(T) == 4)
        return m;
    else
        return half_bits<T>(max(m & 0xffffu, m >> 16));
}

struct Matrix {
    const void *x;
    int64_t rows, cols, stride, group_stride;
    int8_t *q;
    int64_t q_stride, q_group_stride;
    float *scale;
    int groups;
    const uint8_t *mask;                             // groups whose byte is not 0 are left out; NULL: none
    int64_t mask_stride;
};

__device__ __forceinline__ bool left_out(const Matrix &m, int64_t g) { return m.mask && m.mask[g * m.mask_stride] != 0; }

// ---- by row ---------------------------------------------------------------
// kTeam threads hold a row in registers, kHeld 16-byte vectors each, so that it
// is read once, and load the next one while they work on it.  A row that they cannot hold
// is read twice, the second time mostly from L2.
template <int kTeam>
__device__ __forceinline__ unsigned team_max(unsigned m, unsigned *shared)
{
    m = __reduce_max_sync(~0u, m);
    if (kTeam > 32) {
        __syncthreads();                             // the last row's maxima have been read
        if ((threadIdx.x & 31) == 0)
            shared[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kTeam / 32; ++w)
            m = max(m, shared[w]);
    }
    return m;
}

template <typename T>
__device__ __forceinline__ void store_codes(int8_t *to, const Vec<T> &v, const Scale &s)
{
    constexpr int kN = Vec<T>::kN;
    float f[kN];
    widen<T>(v, f);
    unsigned w[kN];
#pragma unroll
    for (int i = 0; i < kN; i += 2)
        whole2(f[i], f[i + 1], s.up, s.up, w[i], w[i + 1]);
    if constexpr (kN == 8)
        *reinterpret_cast<uint2 *>(to) =
            make_uint2(low_bytes(w[0], w[1], w[2], w[3]) & s.keep, low_bytes(w[4], w[5], w[6], w[7]) & s.keep);
    else
        *reinterpret_cast<unsigned *>(to) = low_bytes(w[0], w[1], w[2], w[3]) & s.keep;
}

// Blocks of kTeam threads, or of 256 where a team is a warp.
template <int kTeam> constexpr int kBlockOf = kTeam == 32 ? 256 : kTeam;

template <typename T, int kTeam, int kHeld>
__global__ void __launch_bounds__(kBlockOf<kTeam>) rows_kernel(Matrix m)
{
    constexpr int kN = Vec<T>::kN, kTeams = kBlockOf<kTeam> / kTeam;
    __shared__ unsigned s_max[kTeam / 32];
    const int lane = threadIdx.x % kTeam;
    const int64_t total = m.rows * m.groups, step = int64_t(gridDim.x) * kTeams;
    const int64_t vecs = m.cols / kN;                // whole vectors; the rest one by one
    const auto row_of = [&](int64_t r) {
        const int64_t g = m.groups == 1 ? 0 : r / m.rows;
        return static_cast<const T *>(m.x) + g * m.group_stride + (r - g * m.rows) * m.stride;
    };
    const auto load = [&](Vec<T> (&v)[kHeld], const T *x) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
                v[k].w = __ldcs(reinterpret_cast<const uint4 *>(x) + lane + k * kTeam);
    };
    // the team's next row that is wanted, r itself or one after it
    const auto wanted = [&](int64_t r) {
        while (m.mask && r < total && left_out(m, r / m.rows))
            r += step;
        return r;
    };
    int64_t r = wanted(int64_t(blockIdx.x) * kTeams + threadIdx.x / kTeam);
    if (r >= total)
        return;
    Vec<T> held[kHeld], next[kHeld];
    load(held, row_of(r));
    for (;;) {
        const T *x = row_of(r);
        const int64_t after = wanted(r + step);
        if (after < total)
            load(next, row_of(after));
        unsigned own = 0;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
                add_max<T>(own, held[k]);
        for (int64_t at = lane + int64_t(kHeld) * kTeam; at < vecs; at += kTeam)
            add_max<T>(own, Vec<T>{*(reinterpret_cast<const uint4 *>(x) + at)});
        unsigned amax = max_bits<T>(own);
        for (int64_t c = vecs * kN + lane; c < m.cols; c += kTeam)
            amax = max(amax, magnitude(to_f32(x[c])));
        const Scale s = scale_of(team_max<kTeam>(amax, s_max));
        if (lane == 0)
            m.scale[r] = s.down;
        const int64_t g = m.groups == 1 ? 0 : r / m.rows;
        int8_t *q = m.q + g * m.q_group_stride + (r - g * m.rows) * m.q_stride;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
                store_codes<T>(q + int64_t(lane + k * kTeam) * kN, held[k], s);
        for (int64_t at = lane + int64_t(kHeld) * kTeam; at < vecs; at += kTeam)
            store_codes<T>(q + at * kN, Vec<T>{*(reinterpret_cast<const uint4 *>(x) + at)}, s);
        for (int64_t c = vecs * kN + lane; c < m.cols; c += kTeam)
            q[c] = code_of(to_f32(x[c]), s);
        r = after;
        if (r >= total)
            return;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            held[k] = next[k];
    }
}

// Rows that 16-byte loads cannot take: element by element, read twice.
template <typename T>
__global__ void __launch_bounds__(kThreads) rows_by_element_kernel(Matrix m)
{
    const int lane = threadIdx.x & 31;
    const int64_t total = m.rows * m.groups, step = int64_t(gridDim.x) * (kThreads / 32);
    for (int64_t r = int64_t(blockIdx.x) * (kThreads / 32) + threadIdx.x / 32; r < total; r += step) {
        const int64_t g = r / m.rows, i = r - g * m.rows;
        if (left_out(m, g))
            continue;
        const T *x = static_cast<const T *>(m.x) + g * m.group_stride + i * m.stride;
        int8_t *q = m.q + g * m.q_group_stride + i * m.q_stride;
        unsigned amax = 0;
#pragma unroll 8
        for (int64_t c = lane; c < m.cols; c += 32)
            amax = max(amax, magnitude(to_f32(x[c])));
        const Scale s = scale_of(team_max<32>(amax, nullptr));
        if (lane == 0)
            m.scale[r] = s.down;
#pragma unroll 8
        for (int64_t c = lane; c < m.cols; c += 32)
            q[c] = code_of(to_f32(x[c]), s);
    }
}

// ---- by column --------------------------------------------------------------
// A cluster takes a strip of 64 columns, its CTAs an equal part of the rows each, a
// warp 8 of the columns.  Chunks of 128 rows come through shared memory, three in
// flight; a lane has 4 rows of a chunk, so that a warp's 4-byte words of codes are 128
// contiguous bytes of a transposed row, with no exchange between warps (through tiles
// that the CTA transposed together, with two barriers each, 64 x 1408 x 2048 took 132 us).
// Maxima first, written to every CTA of the cluster through distributed shared memory (read there
// instead, no CTA might end before all had read: a second barrier, 98 us for 95 below), then
// the codes, last chunks first: parts of up to three chunks are still there, others are
// read again, from L2.  16-byte vectors lie swizzled by their rows: lanes that read 4 rows
// apart meet no conflict.
constexpr int kStrip = 64, kChunkRows = 128, kChunks = 3, kMostParts = 8;
static_assert(kThreads / 32 * 8 == kStrip && 32 * 4 == kChunkRows, "a warp's columns, a lane's rows");

template <typename T> constexpr int kVecs = 8 / Vec<T>::kN;              // vectors of 8 columns
template <typename T> constexpr int kChunkVecs = kChunkRows * 8 * kVecs<T>;

__device__ __forceinline__ void copy16(void *to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<unsigned>(__cvta_generic_to_shared(to))),
                 "l"(from)
                 : "memory");
}

// `rows` rows of a strip, x its first element; zeros past the rows and the columns.
template <typename T, bool kVector>
__device__ __forceinline__ void load_chunk(uint4 *chunk, const T *x, int64_t stride, int rows, int64_t cols)
{
    constexpr int kN = Vec<T>::kN, kAcross = 8 * kVecs<T>, kDown = kThreads / kAcross;
    static_assert(kDown % 4 == 0, "a thread's rows are swizzled alike, or in turn");
    const int c = threadIdx.x % kAcross, r0 = threadIdx.x / kAcross;     // a thread's column stays
    const int64_t left = cols - c * kN;
    const T *from = x + r0 * stride + c * kN;
    if (kVector && rows == kChunkRows && left >= kN) {
#pragma unroll
        for (int k = 0; k < kChunkRows / kDown; ++k, from += kDown * stride) {
            const int r = r0 + k * kDown;
            copy16(chunk + r * kAcross + (c ^ ((r >> 2) & 7)), from);
        }
        return;
    }
    for (int r = r0; r < kChunkRows; r += kDown, from += kDown * stride) {
        uint4 *to = chunk + r * kAcross + (c ^ ((r >> 2) & 7));
        if (kVector && r < rows && left >= kN) {
            copy16(to, from);
            continue;
        }
        union {
            T e[kN];
            uint4 w;
        } u;
        u.w = make_uint4(0, 0, 0, 0);
        if (r < rows)
#pragma unroll
            for (int e = 0; e < kN; ++e)
                if (e < left)
                    u.e[e] = from[e];
        *to = u.w;
    }
}

__device__ __forceinline__ void end_load() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// The load before the last two has arrived, for the whole CTA.
__device__ __forceinline__ void await_load()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kChunks - 1) : "memory");
    __syncthreads();
}

template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads) columns_kernel(Matrix m, unsigned parts, int64_t each)
{
    constexpr int kV = kVecs<T>, kN = Vec<T>::kN;
    extern __shared__ uint4 s_chunks[];
    __shared__ unsigned s_max[kMostParts][kStrip];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // fewer CTAs than 2^31, so strips too
    const unsigned strips = static_cast<unsigned>((m.cols + kStrip - 1) / kStrip);
    const unsigned at = blockIdx.x / parts, part = blockIdx.x - at * parts, g = at / strips;
    if (left_out(m, g))
        return;                                                  // and so do the cluster's other CTAs
    if (parts > 1)
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // this CTA has begun
    const int64_t c0 = int64_t(at - g * strips) * kStrip;
    const int64_t r0 = min(m.rows, part * each), r1 = min(m.rows, r0 + each);
    const int chunks = static_cast<int>((r1 - r0 + kChunkRows - 1) / kChunkRows);
    const int64_t cols = m.cols - c0, col = 8 * warp;            // columns of the strip that there are; this warp's first
    const T *x = static_cast<const T *>(m.x) + g * m.group_stride + r0 * m.stride + c0;
    const auto load = [&](int k) {
        if (k >= 0 && k < chunks)
            load_chunk<T, kVector>(s_chunks + k % kChunks * kChunkVecs<T>, x + int64_t(k) * kChunkRows * m.stride, m.stride,
                                   min(kChunkRows, static_cast<int>(r1 - r0) - k * kChunkRows), cols);
        end_load();
    };
    const auto row = [&](int k, int i, Vec<T> (&v)[kV]) {
        const uint4 *from = s_chunks + k % kChunks * kChunkVecs<T> + (4 * lane + i) * 8 * kV;
#pragma unroll
        for (int h = 0; h < kV; ++h)
            v[h].w = from[(warp * kV + h) ^ (lane & 7)];
    };

    for (int k = 0; k < kChunks; ++k)
        load(k);
    unsigned own[4 * kV] = {};                                   // of 8 columns: fp32 bits, or pairs of 16-bit magnitudes
    for (int k = 0; k < chunks; ++k) {
        await_load();
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            Vec<T> v[kV], w[kV];
            row(k, i, v);
            row(k, i + 1, w);
#pragma unroll
            for (int h = 0; h < kV; ++h) {
                const unsigned a[4] = {v[h].w.x, v[h].w.y, v[h].w.z, v[h].w.w}, b[4] = {w[h].w.x, w[h].w.y, w[h].w.z, w[h].w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    own[4 * h + j] = sizeof(T) == 4 ? __vimax3_u32(own[4 * h + j], a[j] & 0x7fffffffu, b[j] & 0x7fffffffu)
                                                    : __vimax3_u16x2(own[4 * h + j], a[j] & 0x7fff7fffu, b[j] & 0x7fff7fffu);
            }
        }
        if (chunks > kChunks)
            __syncthreads();                                     // the chunk makes room for another
        load(k + kChunks);
    }
    // lane e: the maximum of the warp's column e
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned bits = sizeof(T) == 4 ? own[e % (4 * kV)] : half_bits<T>(e % 2 ? own[e / 2] >> 16 : own[e / 2] & 0xffffu);
        const unsigned most = __reduce_max_sync(~0u, bits);
        top = lane == e ? most : top;
    }
    if (parts > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // all have begun
        if (lane < 8)
            for (unsigned k = 0; k < parts; ++k)
                cluster.map_shared_rank(&s_max[part][col + lane], k)[0] = top;
        cluster.sync();                                          // nothing of another CTA's is touched after this
        if (lane < 8)
            for (unsigned k = 0; k < parts; ++k)
                top = max(top, s_max[k][col + lane]);
    }
    const Scale mine = scale_of(top);
    if (part == 0 && lane < 8 && col + lane < cols)
        m.scale[g * m.cols + c0 + col + lane] = mine.down;
    float up[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        up[e] = __shfl_sync(~0u, mine.up, e);
    const bool any_dead = __any_sync(~0u, lane < 8 && top >= kInfBits);     // a column with a NaN or an infinity

    int8_t *q = m.q + g * m.q_group_stride + (c0 + col) * m.q_stride + r0 + 4 * lane;
    const bool words = ((reinterpret_cast<uintptr_t>(m.q) | m.q_stride | m.q_group_stride) & 3) == 0;
    for (int k = chunks - 1; k >= 0; --k) {
        if (chunks > kChunks)
            await_load();
        if (col < cols) {
            unsigned w[4][8];                                    // a row's 8 codes, each a word's low byte
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Vec<T> v[kV];
                row(k, i, v);
                float f[8];
#pragma unroll
                for (int h = 0; h < kV; ++h) {
                    float some[kN];
                    widen<T>(v[h], some);
#pragma unroll
                    for (int e = 0; e < kN; ++e)
                        f[h * kN + e] = some[e];
                }
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    whole2(f[e], f[e + 1], up[e], up[e + 1], w[i][e], w[i][e + 1]);
            }
            const int rows = static_cast<int>(r1 - r0) - k * kChunkRows, left = rows - 4 * lane;     // from this lane's first on
            int8_t *to = q + int64_t(k) * kChunkRows;
            if (words && rows >= kChunkRows && col + 8 <= cols && !any_dead) {
#pragma unroll
                for (int e = 0; e < 8; ++e, to += m.q_stride)
                    *reinterpret_cast<unsigned *>(to) = low_bytes(w[0][e], w[1][e], w[2][e], w[3][e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e, to += m.q_stride) {
                    const unsigned four = low_bytes(w[0][e], w[1][e], w[2][e], w[3][e]) & __shfl_sync(~0u, mine.keep, e);
                    if (col + e >= cols)
                        break;
                    if (words && left >= 4)
                        *reinterpret_cast<unsigned *>(to) = four;
                    else
                        for (int i = 0; i < 4 && i < left; ++i)
                            to[i] = static_cast<int8_t>(four >> (8 * i));
                }
            }
        }
        if (chunks > kChunks) {
            __syncthreads();
            load(k - kChunks);
        }
    }
}

// ---- launches -----------------------------------------------------------------

struct Device {
    int sms = 0;
    cudaError_t status = cudaSuccess;
};

Device current_device()
{
    int dev = 0;
    Device d;
    d.status = cudaGetDevice(&dev);
    if (d.status == cudaSuccess)
        d.status = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
    return d;
}

template <typename T>
cudaError_t launch_rows(const Matrix &m, int sms, cudaStream_t st)
{
    constexpr int kN = Vec<T>::kN;
    const bool vector = ((reinterpret_cast<uintptr_t>(m.x) | (m.stride * sizeof(T)) | (m.group_stride * sizeof(T))) & 15) == 0 &&
                        ((reinterpret_cast<uintptr_t>(m.q) | m.q_stride | m.q_group_stride) % kN) == 0;
    const int64_t total = m.rows * m.groups;
    const auto launch = [&](auto kernel, int threads, int rows, int ctas) {
        kernel<<<static_cast<unsigned>(std::min((total + rows - 1) / rows, int64_t(sms) * ctas)), threads, 0, st>>>(m);
        return cudaGetLastError();
    };
    const int64_t vecs = m.cols / kN;
    if (!vector)
        return launch(rows_by_element_kernel<T>, kThreads, kThreads / 32, 8);
    if (vecs <= 32 * 4)
        return launch(rows_kernel<T, 32, 4>, 256, 8, 4);
    if (vecs <= 32 * 8)
        return launch(rows_kernel<T, 32, 8>, 256, 8, 2);
    if (vecs <= 128 * 4)
        return launch(rows_kernel<T, 128, 4>, 128, 1, 6);
    if (vecs <= 128 * 8)
        return launch(rows_kernel<T, 128, 8>, 128, 1, 4);
    return launch(rows_kernel<T, 256, 8>, 256, 1, 2);
}

template <typename T>
cudaError_t launch_columns(const Matrix &m, int sms, cudaStream_t st)
{
    const bool vector = ((reinterpret_cast<uintptr_t>(m.x) | (m.stride * sizeof(T)) | (m.group_stride * sizeof(T))) & 15) == 0;
    const int64_t strips = (m.cols + kStrip - 1) / kStrip * m.groups;
    const int64_t chunks = std::max<int64_t>((m.rows + kChunkRows - 1) / kChunkRows, 1);
    // Parts of up to six chunks; fewer, to fill the SMs; more, where a cluster's eight CTAs have to
    // take all.  64 x 1408 x 2048: parts of three 122 us, of six 109, of all eleven 115.
    const int64_t fill = chunks * strips / (4 * int64_t(sms)) + 1;
    const int64_t per = std::max(std::min<int64_t>(6, fill), (chunks + kMostParts - 1) / kMostParts), each = per * kChunkRows;
    const int parts = static_cast<int>((chunks + per - 1) / per);
    if (strips * parts > INT32_MAX)
        return cudaErrorInvalidValue;
    const auto kernel = vector ? columns_kernel<T, true> : columns_kernel<T, false>;
    constexpr int kShared = kChunks * kChunkVecs<T> * 16;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(strips * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kShared;
    cfg.stream = st;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
    if (e != cudaSuccess)
        return e;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, m, static_cast<unsigned>(parts), each);
}

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

// Elements that `groups` matrices span, or -1 where that is past 2^60.
int64_t span(int64_t groups, int64_t rows, int64_t stride, int64_t group_stride)
{
    const __int128 n = static_cast<__int128>(groups - 1) * group_stride + static_cast<__int128>(rows) * stride;
    return n > (int64_t(1) << 60) ? -1 : static_cast<int64_t>(n);
}

gnmr_status quantize(bool columns, const void *d_x, int32_t dtype, int32_t groups, int64_t rows, int64_t cols,
                     int64_t x_stride, int64_t x_group_stride, const uint8_t *d_mask, int64_t mask_stride, int8_t *d_q,
                     int64_t q_stride, int64_t q_group_stride, float *d_scale, void *stream)
{
    if (dtype != GNMR_DTYPE_F32 && dtype != GNMR_DTYPE_BF16 && dtype != GNMR_DTYPE_F16)
        return fail(GNMR_ERR_INVALID_ARG, "quantize: unknown dtype");
    if (groups < 1 || rows < 0 || cols < 0)
        return fail(GNMR_ERR_INVALID_ARG, "quantize: groups < 1, or a negative size");
    const int64_t high = columns ? cols : rows, wide = columns ? rows : cols;    // of the codes
    if (x_stride < cols || q_stride < wide || x_group_stride < 0 || q_group_stride < 0 || (d_mask && groups > 1 && mask_stride < 1))
        return fail(GNMR_ERR_LAYOUT, "quantize: a row stride below the row's length, or a negative stride");
    if (rows > INT32_MAX || cols > INT32_MAX || span(groups, rows, x_stride, x_group_stride) < 0 || span(groups, high, q_stride, q_group_stride) < 0)
        return fail(GNMR_ERR_LAYOUT, "quantize: matrices too large");
    if (high == 0)
        return GNMR_OK;
    if (!d_scale || (wide > 0 && (!d_x || !d_q)))
        return fail(GNMR_ERR_INVALID_ARG, "quantize: NULL pointer");
    const size_t eb = dtype == GNMR_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(d_x) % eb || reinterpret_cast<uintptr_t>(d_scale) % 4)
        return fail(GNMR_ERR_LAYOUT, "quantize: buffers not aligned to the element size");
    const Device d = current_device();
    if (d.status != cudaSuccess) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, "quantize: no current device");
    }
    const Matrix m{d_x, rows, cols, x_stride, x_group_stride, d_q, q_stride, q_group_stride, d_scale, groups, d_mask, mask_stride};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (columns)
        e = dtype == GNMR_DTYPE_F32    ? launch_columns<float>(m, d.sms, st)
            : dtype == GNMR_DTYPE_BF16 ? launch_columns<__nv_bfloat16>(m, d.sms, st)
                                       : launch_columns<__half>(m, d.sms, st);
    else
        e = dtype == GNMR_DTYPE_F32    ? launch_rows<float>(m, d.sms, st)
            : dtype == GNMR_DTYPE_BF16 ? launch_rows<__nv_bfloat16>(m, d.sms, st)
                                       : launch_rows<__half>(m, d.sms, st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    return GNMR_OK;
}

}  // namespace

extern "C" {

gnmr_status gnmr_quantize_rows(const void *d_x, int32_t dtype, int32_t groups, int64_t rows, int64_t cols,
                               int64_t x_stride, int64_t x_group_stride, const uint8_t *d_mask, int64_t mask_stride,
                               int8_t *d_q, int64_t q_stride, int64_t q_group_stride, float *d_scale, void *stream)
{
    return quantize(false, d_x, dtype, groups, rows, cols, x_stride, x_group_stride, d_mask, mask_stride, d_q, q_stride,
                    q_group_stride, d_scale, stream);
}

gnmr_status gnmr_quantize_columns(const void *d_x, int32_t dtype, int32_t groups, int64_t rows, int64_t cols,
                                  int64_t x_stride, int64_t x_group_stride, const uint8_t *d_mask, int64_t mask_stride,
                                  int8_t *d_q, int64_t q_stride, int64_t q_group_stride, float *d_scale, void *stream)
{
    return quantize(true, d_x, dtype, groups, rows, cols, x_stride, x_group_stride, d_mask, mask_stride, d_q, q_stride,
                    q_group_stride, d_scale, stream);
}

}  // extern "C"
