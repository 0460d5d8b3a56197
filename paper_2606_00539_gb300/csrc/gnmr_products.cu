// Expert products: the linear units of both paths, grouped by expert.
//
// Every product is out[col][lane] = sum over c of A[lane][c] B[col][c]:
//   forward      A = W_g           B = x's rows     c runs over n_in
//   input grad   A = W_g^T         B = dy's rows    c runs over n_out
//   weight grad  A = x^T           B = dy^T         c runs over the group's rows
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>

#include "gnmr.h"
#include "gnmr_internal.h"

struct gnmr_products {
    int device = 0;
    int sms = 1;
};

namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

struct Product {
    const void *a, *b;
    int64_t a_lane, a_c, a_group, b_col, b_c;      // strides in elements
    int64_t lanes, cols, depth;                    // cols or depth are a group's rows where ragged
    bool ragged_cols;
    const int64_t *offsets;
    int64_t rows;
    int groups;
    const uint8_t *mask;
    int64_t mask_stride;
    int want;                                      // groups computed: mask byte != 0 (1), == 0 (0)
    void *out;
    int64_t out_col, out_group;
    const float *lane_scale, *col_scale;           // 8-bit codes
    int add;
};

template <typename T> __device__ __forceinline__ float wide(T v) { return static_cast<float>(v); }
template <> __device__ __forceinline__ float wide(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float wide(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v) { return static_cast<T>(v); }
template <> __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }

template <typename T> struct Sum { using type = float; };
template <> struct Sum<int8_t> { using type = int; };

// One 64 x 64 tile of outputs a block, 4 x 4 a thread.
template <typename T, typename O>
__global__ void __launch_bounds__(kThreads) product_kernel(Product p)
{
    using S = typename Sum<T>::type;
    __shared__ S s_a[kStep][kTile + 1], s_b[kStep][kTile + 1];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int64_t first = 0, begin = 0;
    for (int g = 0; g < p.groups; ++g) {
        int64_t end = p.rows;
        if (p.offsets) {
            begin = min(max(p.offsets[g], begin), p.rows);
            end = min(max(p.offsets[g + 1], begin), p.rows);
        }
        const int64_t lo = begin;
        begin = end;
        if (p.mask && (p.mask[g * p.mask_stride] != 0) != p.want)
            continue;
        const int64_t cols = p.ragged_cols ? end - lo : p.cols, depth = p.ragged_cols ? p.depth : end - lo;
        const int64_t lane_tiles = (p.lanes + kTile - 1) / kTile;
        const int64_t tiles = lane_tiles * ((cols + kTile - 1) / kTile);
        const int64_t skip = (blockIdx.x + gridDim.x - first % gridDim.x) % gridDim.x;
        first += tiles;
        const T *a = static_cast<const T *>(p.a) + (p.ragged_cols ? g * p.a_group : lo * p.a_c);
        const T *b = static_cast<const T *>(p.b) + lo * (p.ragged_cols ? p.b_col : p.b_c);
        for (int64_t t = skip; t < tiles; t += gridDim.x) {
            const int64_t l0 = t % lane_tiles * kTile, c0 = t / lane_tiles * kTile;
            S sum[4][4] = {};
            for (int64_t d = 0; d < depth; d += kStep) {
                for (int i = threadIdx.x; i < kTile * kStep; i += kThreads) {
                    const int k = i % kStep, r = i / kStep;
                    s_a[k][r] = l0 + r < p.lanes && d + k < depth ? S(wide(a[(l0 + r) * p.a_lane + (d + k) * p.a_c])) : S(0);
                    s_b[k][r] = c0 + r < cols && d + k < depth ? S(wide(b[(c0 + r) * p.b_col + (d + k) * p.b_c])) : S(0);
                }
                __syncthreads();
                for (int k = 0; k < kStep; ++k)
                    for (int i = 0; i < 4; ++i)
                        for (int j = 0; j < 4; ++j)
                            sum[i][j] += s_b[k][ty * 4 + i] * s_a[k][tx + 16 * j];
                __syncthreads();
            }
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) {
                    const int64_t c = c0 + ty * 4 + i, l = l0 + tx + 16 * j;
                    if (c >= cols || l >= p.lanes)
                        continue;
                    O *out = static_cast<O *>(p.out) + (p.ragged_cols ? (lo + c) * p.out_col : g * p.out_group + c * p.out_col) + l;
                    float v = static_cast<float>(sum[i][j]);
                    if (p.lane_scale)
                        v = v * p.col_scale[lo + c] * p.lane_scale[g * p.lanes + l];
                    *out = narrow<O>(p.add ? wide(*out) + v : v);
                }
        }
    }
}

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

bool sixteen(int32_t dtype) { return dtype == GNMR_DTYPE_BF16 || dtype == GNMR_DTYPE_F16; }

bool misaligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

gnmr_status check(const gnmr_product *p)
{
    if (!p)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    if (p->op < GNMR_PRODUCT_FORWARD || p->op > GNMR_PRODUCT_FORWARD_I8)
        return fail(GNMR_ERR_INVALID_ARG, "products: unknown op");
    if (p->groups < 1 || p->groups > 2048)
        return fail(GNMR_ERR_INVALID_ARG, "products: groups outside 1 .. 2048");
    if (p->rows < 0 || p->rows > INT32_MAX || p->n_out < 1 || p->n_in < 1)
        return fail(GNMR_ERR_INVALID_ARG, "products: rows, n_out or n_in out of range");
    const bool codes = p->op == GNMR_PRODUCT_FORWARD_I8, wgrad = p->op == GNMR_PRODUCT_WEIGHT_GRAD;
    if (codes ? !sixteen(p->out_dtype) && p->out_dtype != GNMR_DTYPE_F32
              : !sixteen(p->dtype) || (p->out_dtype != p->dtype && p->out_dtype != GNMR_DTYPE_F32))
        return fail(GNMR_ERR_INVALID_ARG, "products: dtype or out_dtype not of this product");
    if (codes && p->n_in > 131071)
        return fail(GNMR_ERR_INVALID_ARG, "products: n_in above 131071 for 8-bit codes");
    if (!p->d_offsets && p->groups != 1)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL offsets with several groups");
    const bool x = p->op != GNMR_PRODUCT_INPUT_GRAD, w = !wgrad;
    const bool dy = wgrad || p->op == GNMR_PRODUCT_INPUT_GRAD, any = p->rows > 0;
    if ((any && ((x && !p->d_x) || (dy && !p->d_dy) || (codes && !p->d_x_scale))) || (w && !p->d_w) ||
        (codes && !p->d_w_scale) || (!p->d_out && (any || wgrad)))
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL operand");
    const int64_t wide_out = p->op == GNMR_PRODUCT_FORWARD || codes ? p->n_out : p->n_in;
    if ((x && p->x_stride < p->n_in) || (dy && p->dy_stride < p->n_out) ||
        (w && (p->w_stride < p->n_in || p->w_group_stride < 0)) || p->out_stride < wide_out ||
        (wgrad && p->groups > 1 && p->out_group_stride < (p->n_out - 1) * p->out_stride + p->n_in) ||
        (p->d_mask && p->groups > 1 && p->mask_stride < 1))
        return fail(GNMR_ERR_LAYOUT, "products: a stride below what it strides over");
    const size_t eb = codes ? 1 : 2, ob = p->out_dtype == GNMR_DTYPE_F32 ? 4 : 2;
    if ((x && misaligned(p->d_x, eb)) || (dy && misaligned(p->d_dy, eb)) || (w && misaligned(p->d_w, eb)) ||
        misaligned(p->d_out, ob) || misaligned(p->d_offsets, 8) ||
        (codes && (misaligned(p->d_x_scale, 4) || misaligned(p->d_w_scale, 4))))
        return fail(GNMR_ERR_LAYOUT, "products: an operand not aligned to its element size");
    return GNMR_OK;
}

template <typename T>
cudaError_t launch(const Product &q, int out_dtype, int sms, cudaStream_t st)
{
    if (out_dtype == GNMR_DTYPE_BF16)
        product_kernel<T, __nv_bfloat16><<<sms * 4, kThreads, 0, st>>>(q);
    else if (out_dtype == GNMR_DTYPE_F16)
        product_kernel<T, __half><<<sms * 4, kThreads, 0, st>>>(q);
    else
        product_kernel<T, float><<<sms * 4, kThreads, 0, st>>>(q);
    return cudaGetLastError();
}

}  // namespace

extern "C" {

gnmr_status gnmr_products_create(int32_t device, gnmr_products **out)
{
    if (out)
        *out = nullptr;
    if (!out)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || device < 0 || device >= ndev) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, "products: device not available");
    }
    gnmr_products *h = new (std::nothrow) gnmr_products;
    if (!h)
        return fail(GNMR_ERR_OOM, "products: host allocation failed");
    h->device = device;
    cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, device);
    *out = h;
    return GNMR_OK;
}

gnmr_status gnmr_products_scratch_bytes(const gnmr_product *p, int64_t *bytes)
{
    if (!bytes)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    *bytes = 0;
    return check(p);
}

gnmr_status gnmr_products_run(gnmr_products *h, const gnmr_product *p, void *stream)
{
    if (!h)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL handle");
    if (const gnmr_status s = check(p))
        return s;
    const bool codes = p->op == GNMR_PRODUCT_FORWARD_I8, wgrad = p->op == GNMR_PRODUCT_WEIGHT_GRAD;
    if (p->rows == 0 && !wgrad)
        return GNMR_OK;
    Product q = {};
    q.offsets = p->d_offsets;
    q.rows = p->rows;
    q.groups = p->groups;
    q.mask = p->d_mask;
    q.mask_stride = p->mask_stride;
    q.want = codes ? 0 : 1;
    q.out = p->d_out;
    q.out_col = p->out_stride;
    q.out_group = p->out_group_stride;
    q.ragged_cols = !wgrad;
    if (wgrad) {
        q.a = p->d_x, q.a_lane = 1, q.a_c = p->x_stride;
        q.b = p->d_dy, q.b_col = 1, q.b_c = p->dy_stride;
        q.lanes = p->n_in, q.cols = p->n_out;
        q.add = p->add != 0;
    } else {
        const bool back = p->op == GNMR_PRODUCT_INPUT_GRAD;
        q.a = p->d_w, q.a_group = p->w_group_stride;
        q.a_lane = back ? 1 : p->w_stride, q.a_c = back ? p->w_stride : 1;
        q.b = back ? p->d_dy : p->d_x, q.b_col = back ? p->dy_stride : p->x_stride, q.b_c = 1;
        q.lanes = back ? p->n_in : p->n_out, q.depth = back ? p->n_out : p->n_in;
    }
    if (codes)
        q.lane_scale = p->d_w_scale, q.col_scale = p->d_x_scale;
    int prev = h->device;
    cudaGetDevice(&prev);
    if (prev != h->device)
        cudaSetDevice(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = codes                           ? launch<int8_t>(q, p->out_dtype, h->sms, st)
                          : p->dtype == GNMR_DTYPE_BF16 ? launch<__nv_bfloat16>(q, p->out_dtype, h->sms, st)
                                                        : launch<__half>(q, p->out_dtype, h->sms, st);
    if (prev != h->device)
        cudaSetDevice(prev);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    return GNMR_OK;
}

gnmr_status gnmr_products_destroy(gnmr_products *h)
{
    if (!h)
        return GNMR_OK;
    delete h;
    return GNMR_OK;
}

}  // extern "C"
