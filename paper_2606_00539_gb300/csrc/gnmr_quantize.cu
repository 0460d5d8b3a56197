// 8-bit codes with one scale for every row, or for every column and then
// transposed: the operands of the low-cost path's products.
//
//   amax = max |x|, up = 127 * (1 / amax), scale = amax / 127, q = rint(x * up)
//
// in fp32, by row or by column, each operation rounded.  Both are bound by memory: 3 bytes an element
// from 16-bit inputs.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

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
};

__device__ __forceinline__ Scale scale_of(unsigned amax_bits)
{
    if (amax_bits >= kInfBits)
        return {0.0f, __uint_as_float(0x7fc00000u)};
    const float amax = __uint_as_float(amax_bits);
    const float up = __fmul_rn(127.0f, __frcp_rn(amax));
    if (!(magnitude(up) < kInfBits))                 // amax is 0, or 127 / amax is past fp32
        return {0.0f, 0.0f};
    return {up, __fdiv_rn(amax, 127.0f)};
}

// A row that holds a NaN or an infinity has up = 0: its codes are 0, not NaN * 0.
__device__ __forceinline__ int code_of(float v, const Scale &s)
{
    return s.up == 0.0f ? 0 : __float2int_rn(__fmul_rn(v, s.up));
}

__device__ __forceinline__ unsigned pack4(int a, int b, int c, int d)
{
    return (a & 255u) | (b & 255u) << 8 | (c & 255u) << 16 | static_cast<unsigned>(d) << 24;
}

// 16 bytes of a row, and how many elements they are.
template <typename T> struct Vec {
    static constexpr int kN = 16 / sizeof(T);
    alignas(16) T v[kN];
};

struct Matrix {
    const void *x;
    int64_t rows, cols, stride, group_stride;
    int8_t *q;
    int64_t q_stride, q_group_stride;
    float *scale;
    int groups;
};

// ---- by row ---------------------------------------------------------------
// kTeam threads hold a row in registers, kHeld 16-byte vectors each, so that it
// is read once.  A row that they cannot hold is read twice, the second time
// mostly from L2.
template <int kTeam>
__device__ __forceinline__ unsigned team_max(unsigned m, unsigned *shared)
{
#pragma unroll
    for (int d = 16; d; d >>= 1)
        m = max(m, __shfl_xor_sync(~0u, m, d));
    if (kTeam > 32) {
        __syncthreads();                             // the last row's maxima have been read
        if ((threadIdx.x & 31) == 0)
            shared[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w)
            m = max(m, shared[w]);
    }
    return m;
}

template <typename T>
__device__ __forceinline__ void store_codes(int8_t *to, const Vec<T> &v, const Scale &s)
{
    constexpr int kN = Vec<T>::kN;
    unsigned w[kN / 4];
#pragma unroll
    for (int i = 0; i < kN; i += 4)
        w[i / 4] = pack4(code_of(to_f32(v.v[i]), s), code_of(to_f32(v.v[i + 1]), s), code_of(to_f32(v.v[i + 2]), s),
                         code_of(to_f32(v.v[i + 3]), s));
    if (kN == 8)
        *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[kN / 4 - 1]);
    else
        *reinterpret_cast<unsigned *>(to) = w[0];
}

template <typename T, int kTeam, int kHeld>
__global__ void __launch_bounds__(kThreads) rows_kernel(Matrix m)
{
    constexpr int kN = Vec<T>::kN;
    __shared__ unsigned s_max[kThreads / 32];
    const int lane = threadIdx.x % kTeam;
    const int64_t total = m.rows * m.groups, step = int64_t(gridDim.x) * (kThreads / kTeam);
    const int64_t vecs = m.cols / kN;                // whole vectors; the rest one by one
    for (int64_t r = int64_t(blockIdx.x) * (kThreads / kTeam) + threadIdx.x / kTeam; r < total; r += step) {
        const int64_t g = r / m.rows, i = r - g * m.rows;
        const T *x = static_cast<const T *>(m.x) + g * m.group_stride + i * m.stride;
        int8_t *q = m.q + g * m.q_group_stride + i * m.q_stride;
        Vec<T> held[kHeld];
        unsigned amax = 0;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
                *reinterpret_cast<uint4 *>(held[k].v) =
                    __ldcs(reinterpret_cast<const uint4 *>(x) + lane + k * kTeam);
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
#pragma unroll
                for (int e = 0; e < kN; ++e)
                    amax = max(amax, magnitude(to_f32(held[k].v[e])));
        for (int64_t at = lane + int64_t(kHeld) * kTeam; at < vecs; at += kTeam) {
            Vec<T> v;
            *reinterpret_cast<uint4 *>(v.v) = *(reinterpret_cast<const uint4 *>(x) + at);
#pragma unroll
            for (int e = 0; e < kN; ++e)
                amax = max(amax, magnitude(to_f32(v.v[e])));
        }
        for (int64_t c = vecs * kN + lane; c < m.cols; c += kTeam)
            amax = max(amax, magnitude(to_f32(x[c])));
        const Scale s = scale_of(team_max<kTeam>(amax, s_max));
        if (lane == 0)
            m.scale[r] = s.down;
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (lane + k * kTeam < vecs)
                store_codes(q + int64_t(lane + k * kTeam) * kN, held[k], s);
        for (int64_t at = lane + int64_t(kHeld) * kTeam; at < vecs; at += kTeam) {
            Vec<T> v;
            *reinterpret_cast<uint4 *>(v.v) = *(reinterpret_cast<const uint4 *>(x) + at);
            store_codes(q + at * kN, v, s);
        }
        for (int64_t c = vecs * kN + lane; c < m.cols; c += kTeam)
            q[c] = static_cast<int8_t>(code_of(to_f32(x[c]), s));
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
            q[c] = static_cast<int8_t>(code_of(to_f32(x[c]), s));
    }
}

// ---- by column --------------------------------------------------------------
// A cluster takes a strip of 64 columns, its CTAs an equal part of the rows
// each: maxima first, joined over the cluster through distributed shared
// memory, then the same rows again (from L2) as codes, transposed by shared
// memory in tiles of 64 columns and 128 rows, 128-byte lines of codes going out.
constexpr int kStrip = 64;
constexpr int kTileRows = 128;
constexpr int kPitch = kTileRows / 4 + 1;            // words a column: lanes that read along rows meet no conflict

template <typename T, bool kVector>
__device__ __forceinline__ void load8(const T *x, int64_t cols_left, float (&v)[8])
{
    if (kVector && cols_left >= 8) {
#pragma unroll
        for (int h = 0; h < 8 / Vec<T>::kN; ++h) {
            Vec<T> t;
            *reinterpret_cast<uint4 *>(t.v) = *(reinterpret_cast<const uint4 *>(x) + h);
#pragma unroll
            for (int e = 0; e < Vec<T>::kN; ++e)
                v[h * Vec<T>::kN + e] = to_f32(t.v[e]);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = e < cols_left ? to_f32(x[e]) : 0.0f;
}

template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads) columns_kernel(Matrix m, int parts)
{
    __shared__ unsigned s_max[kStrip];
    __shared__ unsigned s_tile[kStrip * kPitch];
    const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;       // 8 columns; a row of 32
    const int64_t strips = (m.cols + kStrip - 1) / kStrip;
    const int64_t at = blockIdx.x / parts, part = blockIdx.x % parts;
    const int64_t g = at / strips, c0 = (at - g * strips) * kStrip;
    const int64_t each = (m.rows + int64_t(parts) * kTileRows - 1) / (int64_t(parts) * kTileRows) * kTileRows;
    const int64_t r0 = min(m.rows, part * each), r1 = min(m.rows, r0 + each);
    const int64_t left = m.cols - c0 - 8 * tx;
    const T *x = static_cast<const T *>(m.x) + g * m.group_stride + c0 + 8 * tx;

    if (threadIdx.x < kStrip)
        s_max[threadIdx.x] = 0;
    __syncthreads();
    unsigned amax[8] = {};
    if (left > 0) {
#pragma unroll 4
        for (int64_t r = r0 + ty; r < r1; r += kThreads / 8) {
            float v[8];
            load8<T, kVector>(x + r * m.stride, left, v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                amax[e] = max(amax[e], magnitude(v[e]));
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        amax[e] = max(amax[e], __shfl_xor_sync(~0u, amax[e], 8));
        amax[e] = max(amax[e], __shfl_xor_sync(~0u, amax[e], 16));
        if ((threadIdx.x & 31) < 8)
            atomicMax(&s_max[8 * tx + e], amax[e]);              // a maximum: order does not matter
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    unsigned mine = 0;
    if (threadIdx.x < kStrip)
        for (int k = 0; k < parts; ++k)
            mine = max(mine, cluster.map_shared_rank(s_max, k)[threadIdx.x]);
    cluster.sync();                                              // every CTA has read every other's
    if (threadIdx.x < kStrip) {
        s_max[threadIdx.x] = mine;
        if (part == 0 && c0 + threadIdx.x < m.cols)
            m.scale[g * m.cols + c0 + threadIdx.x] = scale_of(mine).down;
    }
    __syncthreads();
    Scale s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        s[e] = scale_of(s_max[8 * tx + e]);

    int8_t *q = m.q + g * m.q_group_stride + c0 * m.q_stride;
    const bool words = ((reinterpret_cast<uintptr_t>(m.q) | m.q_stride | m.q_group_stride) & 3) == 0;
    for (int64_t t0 = r0; t0 < r1; t0 += kTileRows) {
        if (left > 0) {
            float v[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t r = t0 + 4 * ty + i;
                if (r < r1)
                    load8<T, kVector>(x + r * m.stride, left, v[i]);
                else
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[i][e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s_tile[(8 * tx + e) * kPitch + ty] = pack4(code_of(v[0][e], s[e]), code_of(v[1][e], s[e]),
                                                           code_of(v[2][e], s[e]), code_of(v[3][e], s[e]));
        }
        __syncthreads();
        const int lane = threadIdx.x & 31;
        const int64_t r = t0 + 4 * lane;
        for (int c = threadIdx.x >> 5; c < kStrip && c0 + c < m.cols; c += kThreads / 32) {
            const unsigned w = s_tile[c * kPitch + lane];
            int8_t *to = q + c * m.q_stride + r;
            if (words && r + 4 <= r1)
                *reinterpret_cast<unsigned *>(to) = w;
            else
                for (int i = 0; i < 4 && r + i < r1; ++i)
                    to[i] = static_cast<int8_t>(w >> (8 * i));
        }
        __syncthreads();
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
    const auto grid = [&](int64_t per, int ctas) {
        return static_cast<unsigned>(std::min<int64_t>((total + per - 1) / per, int64_t(sms) * ctas));
    };
    if (!vector)
        rows_by_element_kernel<T><<<grid(kThreads / 32, 8), kThreads, 0, st>>>(m);
    else if (m.cols <= 32 * kN * 4)
        rows_kernel<T, 32, 4><<<grid(kThreads / 32, 8), kThreads, 0, st>>>(m);
    else if (m.cols <= kThreads * kN * 4)
        rows_kernel<T, kThreads, 4><<<grid(1, 8), kThreads, 0, st>>>(m);
    else
        rows_kernel<T, kThreads, 8><<<grid(1, 5), kThreads, 0, st>>>(m);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_columns(const Matrix &m, int sms, cudaStream_t st)
{
    const bool vector = ((reinterpret_cast<uintptr_t>(m.x) | (m.stride * sizeof(T)) | (m.group_stride * sizeof(T))) & 15) == 0;
    const int64_t strips = (m.cols + kStrip - 1) / kStrip * m.groups;
    int parts = 1;
    while (parts < 8 && m.rows > int64_t(parts) * kTileRows && strips * parts < 8 * int64_t(sms))
        parts *= 2;
    if (strips * parts > INT32_MAX)
        return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(strips * parts));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = parts;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return vector ? cudaLaunchKernelEx(&cfg, columns_kernel<T, true>, m, parts)
                  : cudaLaunchKernelEx(&cfg, columns_kernel<T, false>, m, parts);
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
                     int64_t x_stride, int64_t x_group_stride, int8_t *d_q, int64_t q_stride, int64_t q_group_stride,
                     float *d_scale, void *stream)
{
    if (dtype != GNMR_DTYPE_F32 && dtype != GNMR_DTYPE_BF16 && dtype != GNMR_DTYPE_F16)
        return fail(GNMR_ERR_INVALID_ARG, "quantize: unknown dtype");
    if (groups < 1 || rows < 0 || cols < 0)
        return fail(GNMR_ERR_INVALID_ARG, "quantize: groups < 1, or a negative size");
    const int64_t high = columns ? cols : rows, wide = columns ? rows : cols;    // of the codes
    if (x_stride < cols || q_stride < wide || x_group_stride < 0 || q_group_stride < 0)
        return fail(GNMR_ERR_LAYOUT, "quantize: a row stride below the row's length, or a negative stride");
    if (span(groups, rows, x_stride, x_group_stride) < 0 || span(groups, high, q_stride, q_group_stride) < 0)
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
    const Matrix m{d_x, rows, cols, x_stride, x_group_stride, d_q, q_stride, q_group_stride, d_scale, groups};
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
                               int64_t x_stride, int64_t x_group_stride, int8_t *d_q, int64_t q_stride,
                               int64_t q_group_stride, float *d_scale, void *stream)
{
    return quantize(false, d_x, dtype, groups, rows, cols, x_stride, x_group_stride, d_q, q_stride, q_group_stride,
                    d_scale, stream);
}

gnmr_status gnmr_quantize_columns(const void *d_x, int32_t dtype, int32_t groups, int64_t rows, int64_t cols,
                                  int64_t x_stride, int64_t x_group_stride, int8_t *d_q, int64_t q_stride,
                                  int64_t q_group_stride, float *d_scale, void *stream)
{
    return quantize(true, d_x, dtype, groups, rows, cols, x_stride, x_group_stride, d_q, q_stride, q_group_stride,
                    d_scale, stream);
}

}  // extern "C"
