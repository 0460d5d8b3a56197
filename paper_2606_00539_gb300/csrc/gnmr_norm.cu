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

// The sum over a CTA, the same bits in every thread.  `shared`: kWarps floats that nothing else uses; every
// call begins with a barrier.
__device__ __forceinline__ float cta_sum(float v, float *shared)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        shared[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i)
        s += shared[i];
    return s;
}

// Any width and alignment: a CTA a row, which it reads three times.
template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_any_kernel(const Norm n)
{
    __shared__ float shared[kWarps];
    const P *const w = static_cast<const P *>(n.w), *const b = static_cast<const P *>(n.b);
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x) {
        const T *const x = static_cast<const T *>(n.x) + r * n.x_stride;
        T *const y = static_cast<T *>(n.y) + r * n.y_stride;
        float s = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads)
            s += to_f32(x[i]);
        const float mean = cta_sum(s, shared) / n.cols;
        s = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            const float d = to_f32(x[i]) - mean;
            s += d * d;
        }
        const float rstd = 1.0f / sqrtf(cta_sum(s, shared) / n.cols + n.eps);
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
    __shared__ float shared[kWarps];
    const P *const w = static_cast<const P *>(n.w);
    for (int64_t r = blockIdx.x; r < n.rows; r += gridDim.x) {
        const T *const x = static_cast<const T *>(n.x) + r * n.x_stride, *const dy = static_cast<const T *>(n.dy) + r * n.dy_stride;
        T *const dx = static_cast<T *>(n.y) + r * n.y_stride;
        const float mean = n.mean_in[r], rstd = n.rstd_in[r];
        float s = 0.0f, q = 0.0f;
        for (int i = threadIdx.x; i < n.cols; i += kThreads) {
            const float t = to_f32(dy[i]) * (n.w ? to_f32(w[i]) : 1.0f);
            s += t;
            q += t * ((to_f32(x[i]) - mean) * rstd);
        }
        s = cta_sum(s, shared) / n.cols;
        q = cta_sum(q, shared) / n.cols;
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

// The parts' sums, in their order.
template <typename G>
__global__ void __launch_bounds__(kThreads) join_kernel(const Norm n)
{
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= n.cols)
        return;
    G *const to = static_cast<G *>(blockIdx.y ? n.db : n.dw);
    if (!to)
        return;
    const float *const part = (blockIdx.y ? n.part_b : n.part_w) + i;
    float s = 0.0f;
    for (int p = 0; p < n.parts; ++p)
        s += part[int64_t(p) * n.cols];
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
    return n;
}

gnmr_status said(cudaError_t e)
{
    if (e == cudaSuccess)
        return GNMR_OK;
    cudaGetLastError();
    return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
}

template <typename T, typename P> cudaError_t forward(const Norm &n, int sms, cudaStream_t st)
{
    norm_any_kernel<T, P><<<static_cast<unsigned>(std::min(n.rows, int64_t(sms) * 8)), kThreads, 0, st>>>(n);
    return cudaGetLastError();
}

template <typename T, typename P> cudaError_t backward(Norm n, int sms, cudaStream_t st)
{
    if (n.rows > 0 && (n.dw || n.db)) {
        n.parts = static_cast<int>(std::min<int64_t>(n.rows, std::min(kMostParts, 2 * sms)));
        columns_any_kernel<T><<<dim3((n.cols + kThreads - 1) / kThreads, n.parts), kThreads, 0, st>>>(n);
    }
    if (n.rows > 0 && n.y)                             // last: it may write over dy
        norm_grad_any_kernel<T, P><<<static_cast<unsigned>(std::min(n.rows, int64_t(sms) * 8)), kThreads, 0, st>>>(n);
    return cudaGetLastError();
}

template <typename T> cudaError_t by_params(const gnmr_norm *p, const Norm &n, bool grad, int sms, cudaStream_t st)
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
    n.parts = static_cast<int>(std::min<int64_t>(n.rows, std::min(kMostParts, 2 * sms)));
    n.part_w = static_cast<float *>(p->d_scratch);
    n.part_b = n.part_w + int64_t(kMostParts) * n.cols;
    cudaError_t e = cudaSuccess;
    if (n.rows > 0)
        e = by_type(p->dtype, [&](auto v) { return by_params<decltype(v)>(p, n, true, sms, st); });
    if (e == cudaSuccess && (n.dw || n.db) && (n.rows > 0 || !n.add))
        e = by_type(p->grad_dtype, [&](auto v) {
            join_kernel<decltype(v)><<<dim3((n.cols + kThreads - 1) / kThreads, 2), kThreads, 0, st>>>(n);
            return cudaGetLastError();
        });
    return said(e);
}

}  // extern "C"
