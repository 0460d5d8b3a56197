// The norm over many tensors, and the tensors scaled down to a limit.
//
//   norm = sqrt(sum of x^2), scale = min(1, max_norm / norm), out = x scale
//
// Two kernels: sums of squares, a partial sum from each CTA; then every CTA of the second one adds the
// partial sums up in the same order, which takes it a microsecond, and scales its share.  Both are bound by
// memory: the gradients are read twice (once where nothing is written: in place, below the limit) and
// written once.  Where the tensors lie comes with each call, as kernel parameters, so that a captured
// call keeps its own; how they are cut into chunks is in the plan.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "gnmr.h"
#include "gnmr_internal.h"
#include "gnmr_rows.cuh"
#include "gnmr_stream.cuh"

struct gnmr_clip {
    int device = 0, sms = 1;
    int tensors = 0;
    int64_t chunks = 0;
    std::vector<int64_t> lengths, first;               // first[i]: chunks before tensor i
    std::vector<int32_t> dtypes;
    int64_t chunk = 0;                                 // bytes
    void *dmem = nullptr;
    const int64_t *d_lengths = nullptr, *d_first = nullptr;
    const int32_t *d_dtypes = nullptr;
};

namespace {

using namespace gnmr_rows;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 8;
constexpr int kCtas = 4;                               // an SM
constexpr int kMostCtas = 1024;                        // of the first kernel: the partial sums


// Tensors first .. first + count - 1 of the plan, those that one launch takes.
struct Plan {
    const int64_t *lengths, *first;                    // [tensors], [tensors + 1]
    const int32_t *dtypes;
    int64_t chunk;
    int tensor0, tensors;
    int64_t chunk0, chunks;
};

template <int kN> struct Places {
    const char *in[kN];
    char *out[kN];
};

struct Part {
    int tensor;                                        // among the launch's
    int64_t at, n;                                     // elements
};

__device__ __forceinline__ int bytes_of(int dtype) { return dtype == GNMR_DTYPE_F32 ? 4 : 2; }

// Chunk c: the last tensor that begins at or before it.  t: that of an earlier chunk.
__device__ __forceinline__ Part part_of(const Plan &p, int64_t c, int &t)
{
    int hi = p.tensors;
    if (t + 1 < hi && __ldg(p.first + p.tensor0 + t + 1) > c)
        hi = t + 1;
    for (; hi - t > 1;) {
        const int mid = (t + hi) / 2;
        if (__ldg(p.first + p.tensor0 + mid) <= c)
            t = mid;
        else
            hi = mid;
    }
    const int i = p.tensor0 + t;
    const int64_t each = p.chunk / bytes_of(__ldg(p.dtypes + i));
    Part part;
    part.tensor = t;
    part.at = (c - __ldg(p.first + i)) * each;
    part.n = min(each, __ldg(p.lengths + i) - part.at);
    return part;
}

template <int DT> __device__ __forceinline__ double squares(const char *at, int64_t n, int lane)
{
    bool suspect;
    const double s = gnmr::warp_segment_sumsq<DT, kUnroll>(at, n, lane, suspect);
    return suspect ? gnmr::warp_segment_sumsq_f64<DT>(at, n, lane) : s;
}

// This CTA's partial sum.
template <int kN>
__global__ void __launch_bounds__(kThreads) squares_kernel(const __grid_constant__ Plan p, const __grid_constant__ Places<kN> places, double *partial)
{
    __shared__ double sums[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + warp, all = int64_t(gridDim.x) * kWarps;
    const int64_t c0 = p.chunk0 + p.chunks * w / all, c1 = p.chunk0 + p.chunks * (w + 1) / all;
    double sum = 0.0;
    int t = 0;
    for (int64_t c = c0; c < c1; ++c) {
        const Part part = part_of(p, c, t);
        const int dtype = __ldg(p.dtypes + p.tensor0 + part.tensor);
        const char *at = places.in[part.tensor] + part.at * bytes_of(dtype);
        if (dtype == GNMR_DTYPE_F32)
            sum += squares<GNMR_DTYPE_F32>(at, part.n, lane);
        else if (dtype == GNMR_DTYPE_BF16)
            sum += squares<GNMR_DTYPE_BF16>(at, part.n, lane);
        else
            sum += squares<GNMR_DTYPE_F16>(at, part.n, lane);
    }
    if (lane == 0)
        sums[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kWarps; ++i)
            sum += sums[i];
        partial[blockIdx.x] = sum;
    }
}

// The same from norms.
__global__ void __launch_bounds__(kThreads) norms_kernel(const double *norms, int64_t n, double *partial)
{
    __shared__ double sums[kWarps];
    double sum = 0.0;
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads)
        sum = fma(norms[i], norms[i], sum);
    sum = gnmr::warp_allreduce_sum(sum);
    if ((threadIdx.x & 31) == 0)
        sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kWarps; ++i)
            sum += sums[i];
        partial[blockIdx.x] = sum;
    }
}

// n elements scaled, by a warp.
template <typename T> __device__ __forceinline__ void scale_part(const T *in, T *out, int64_t n, float scale, int lane)
{
    constexpr int kV = kIn16<T>;
    const int64_t head = min(n, int64_t((16 - (reinterpret_cast<uintptr_t>(in) & 15)) & 15) / int64_t(sizeof(T)));
    const bool alike = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int64_t vecs = alike ? (n - head) / kV : 0;
    for (int64_t i = lane; i < vecs; i += 32) {
        float f[kV];
        widen<T>(load_once(in + head + i * kV), f);
#pragma unroll
        for (int j = 0; j < kV; ++j)
            f[j] *= scale;
        store_once(out + head + i * kV, narrow<T>(f));
    }
    // what lies around the vectors
    const int64_t rest = n - vecs * kV;
    for (int64_t i = lane; i < rest; i += 32) {
        const int64_t at = i < head ? i : i + vecs * kV;
        out[at] = from_f32<T>(to_f32(in[at]) * scale);
    }
}

template <int kN>
__global__ void __launch_bounds__(kThreads)
scale_kernel(const __grid_constant__ Plan p, const __grid_constant__ Places<kN> places, const double *partial, int partials, double max_norm,
             float *norm_out, int in_place)
{
    __shared__ double sums[kWarps];
    __shared__ float scale_of_all;
    double sum = 0.0;
    for (int i = threadIdx.x; i < partials; i += kThreads)
        sum += partial[i];
    sum = gnmr::warp_allreduce_sum(sum);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0)
        sums[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kWarps; ++i)
            sum += sums[i];
        const double norm = sqrt(sum);
        // a norm that is not finite compares as not above the limit, or as infinite
        scale_of_all = norm > max_norm && isfinite(norm) ? static_cast<float>(max_norm / norm) : 1.0f;
        if (blockIdx.x == 0 && norm_out)
            *norm_out = static_cast<float>(norm);
    }
    __syncthreads();
    const float scale = scale_of_all;
    if (in_place && scale == 1.0f)
        return;
    const int64_t w = int64_t(blockIdx.x) * kWarps + warp, all = int64_t(gridDim.x) * kWarps;
    const int64_t c0 = p.chunk0 + p.chunks * w / all, c1 = p.chunk0 + p.chunks * (w + 1) / all;
    int t = 0;
    for (int64_t c = c0; c < c1; ++c) {
        const Part part = part_of(p, c, t);
        const int dtype = __ldg(p.dtypes + p.tensor0 + part.tensor);
        const int64_t at = part.at * bytes_of(dtype);
        const char *in = places.in[part.tensor] + at;
        char *out = places.out[part.tensor] + at;
        if (dtype == GNMR_DTYPE_F32)
            scale_part(reinterpret_cast<const float *>(in), reinterpret_cast<float *>(out), part.n, scale, lane);
        else if (dtype == GNMR_DTYPE_BF16)
            scale_part(reinterpret_cast<const __nv_bfloat16 *>(in), reinterpret_cast<__nv_bfloat16 *>(out), part.n, scale, lane);
        else
            scale_part(reinterpret_cast<const __half *>(in), reinterpret_cast<__half *>(out), part.n, scale, lane);
    }
}

// ---- host -----------------------------------------------------------------------

constexpr int kMost = 1900;                            // tensors of one launch: places in 32,764 bytes of parameters

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

int ctas_for(const gnmr_clip *c, int64_t chunks)
{
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((chunks + kWarps - 1) / kWarps, std::min(c->sms * kCtas, kMostCtas))));
}

template <int kN> Places<kN> places_of(int from, int count, const void *const *in, void *const *out)
{
    Places<kN> p;
    for (int i = 0; i < count; ++i) {
        p.in[i] = static_cast<const char *>(in[from + i]);
        p.out[i] = static_cast<char *>(out ? out[from + i] : const_cast<void *>(in[from + i]));
    }
    return p;
}

int launches_of(const gnmr_clip *c) { return std::max(1, (c->tensors + kMost - 1) / kMost); }

// Calls f(plan, places) for every launch's tensors.
template <typename F> cudaError_t by_launch(const gnmr_clip *c, const void *const *in, void *const *out, F f)
{
    for (int from = 0; from < std::max(c->tensors, 1); from += kMost) {
        const int count = std::min(kMost, c->tensors - from);
        const Plan p{c->d_lengths, c->d_first, c->d_dtypes, c->chunk, from, count, c->first[from], c->first[from + count] - c->first[from]};
        const cudaError_t e = count <= 64    ? f(p, places_of<64>(from, count, in, out))
                              : count <= 400 ? f(p, places_of<400>(from, count, in, out))
                                             : f(p, places_of<kMost>(from, count, in, out));
        if (e != cudaSuccess)
            return e;
    }
    return cudaSuccess;
}

template <int kN>
cudaError_t launch_squares(const gnmr_clip *c, const Plan &p, const Places<kN> &places, double *partial, int *count, cudaStream_t st)
{
    const int ctas = ctas_for(c, p.chunks);
    squares_kernel<kN><<<ctas, kThreads, 0, st>>>(p, places, partial + *count);
    *count += ctas;
    return cudaGetLastError();
}

}  // namespace

extern "C" {

gnmr_status gnmr_clip_create(int32_t num_tensors, const int64_t *lengths, const int32_t *dtypes, int32_t device, gnmr_clip **out)
{
    if (out)
        *out = nullptr;
    if (!out || num_tensors < 0 || (num_tensors > 0 && (!lengths || !dtypes)))
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument, or a negative number of tensors");
    __int128 bytes = 0;
    for (int i = 0; i < num_tensors; ++i) {
        if (lengths[i] < 0 || lengths[i] > int64_t(1) << 48 || !known(dtypes[i]))
            return fail(GNMR_ERR_INVALID_ARG, "clip: a length out of range, or an unknown dtype");
        bytes += static_cast<__int128>(lengths[i]) * element_bytes(dtypes[i]);
    }
    if (bytes > int64_t(1) << 50)
        return fail(GNMR_ERR_INVALID_ARG, "clip: more bytes than any device has");
    int ndev = 0;
    if (cudaGetDeviceCount(&ndev) != cudaSuccess || device < 0 || device >= ndev) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, "clip: device not available");
    }
    gnmr_clip *c = nullptr;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaError_t e = cudaSuccess;
    try {
        c = new gnmr_clip;
        c->device = device;
        c->tensors = num_tensors;
        c->lengths.assign(lengths, lengths + num_tensors);
        c->dtypes.assign(dtypes, dtypes + num_tensors);
        e = cudaDeviceGetAttribute(&c->sms, cudaDevAttrMultiProcessorCount, device);
        // chunks of 4 KB that give every warp one, 64 KB at most
        const int64_t warps = int64_t(c->sms) * kCtas * kWarps;
        c->chunk = std::min<int64_t>(65536, std::max<int64_t>(1, (static_cast<int64_t>(bytes) / warps + 4095) / 4096) * 4096);
        c->first.resize(num_tensors + 1);
        for (int i = 0; i < num_tensors; ++i)
            c->first[i + 1] = c->first[i] + (lengths[i] * int64_t(element_bytes(dtypes[i])) + c->chunk - 1) / c->chunk;
        c->chunks = c->first[num_tensors];
    } catch (const std::bad_alloc &) {
        delete c;
        return fail(GNMR_ERR_OOM, "clip: host allocation failed");
    }
    const size_t wide = num_tensors * sizeof(int64_t), all = 2 * wide + sizeof(int64_t) + num_tensors * sizeof(int32_t);
    cudaSetDevice(device);
    if (e == cudaSuccess)
        e = cudaMalloc(&c->dmem, all);
    char *at = static_cast<char *>(c->dmem);
    if (e == cudaSuccess) {
        c->d_first = reinterpret_cast<const int64_t *>(at);
        c->d_lengths = c->d_first + num_tensors + 1;
        c->d_dtypes = reinterpret_cast<const int32_t *>(c->d_lengths + num_tensors);
        e = cudaMemcpy(at, c->first.data(), wide + sizeof(int64_t), cudaMemcpyHostToDevice);
    }
    if (e == cudaSuccess && num_tensors) {
        e = cudaMemcpy(at + wide + sizeof(int64_t), lengths, wide, cudaMemcpyHostToDevice);
        if (e == cudaSuccess)
            e = cudaMemcpy(at + 2 * wide + sizeof(int64_t), dtypes, num_tensors * sizeof(int32_t), cudaMemcpyHostToDevice);
    }
    if (e == cudaSuccess)
        e = cudaStreamSynchronize(nullptr);            // the tables are in place whatever stream reads them
    cudaSetDevice(prev);
    if (e != cudaSuccess) {
        cudaGetLastError();
        gnmr_clip_destroy(c);
        return fail(e == cudaErrorMemoryAllocation ? GNMR_ERR_OOM : GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    *out = c;
    return GNMR_OK;
}

gnmr_status gnmr_clip_scratch_bytes(const gnmr_clip *c, int64_t *bytes)
{
    if (!c || !bytes)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument");
    *bytes = int64_t(launches_of(c)) * kMostCtas * sizeof(double);
    return GNMR_OK;
}

gnmr_status gnmr_clip_run(const gnmr_clip *c, const void *const *d_in, void *const *d_out, double max_norm, const double *d_unit_norms,
                          int64_t num_norms, float *d_norm, void *d_scratch, int64_t scratch_bytes, void *stream)
{
    if (!c || !d_norm || (c->tensors > 0 && !d_in) || num_norms < 0)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument, or a negative number of norms");
    if (!(max_norm >= 0))
        return fail(GNMR_ERR_INVALID_ARG, "clip: max_norm has to be 0 or more");
    int64_t need = 0;
    gnmr_clip_scratch_bytes(c, &need);
    if (!d_scratch || scratch_bytes < need || misaligned(d_scratch, 256))
        return fail(GNMR_ERR_LAYOUT, "clip: scratch missing, too small or misaligned");
    if (misaligned(d_unit_norms, 8) || misaligned(d_norm, 4))
        return fail(GNMR_ERR_LAYOUT, "clip: a buffer not aligned to its element size");
    for (int i = 0; i < c->tensors; ++i) {
        const size_t eb = element_bytes(c->dtypes[i]);
        if (c->lengths[i] > 0 && (!d_in[i] || (d_out && !d_out[i])))
            return fail(GNMR_ERR_INVALID_ARG, "clip: NULL tensor");
        if (misaligned(d_in[i], eb) || (d_out && misaligned(d_out[i], eb)))
            return fail(GNMR_ERR_LAYOUT, "clip: a tensor not aligned to its element size");
    }
    int prev = c->device;
    cudaGetDevice(&prev);
    if (prev != c->device)
        cudaSetDevice(c->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    double *partial = static_cast<double *>(d_scratch);
    int partials = 0;
    cudaError_t e = cudaSuccess;
    if (d_unit_norms) {
        partials = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((num_norms + kThreads - 1) / kThreads, c->sms)));
        norms_kernel<<<partials, kThreads, 0, st>>>(d_unit_norms, num_norms, partial);
        e = cudaGetLastError();
    } else {
        e = by_launch(c, d_in, d_out, [&](const Plan &p, const auto &places) {
            return launch_squares(c, p, places, partial, &partials, st);
        });
    }
    float *norm = d_norm;
    if (e == cudaSuccess)
        e = by_launch(c, d_in, d_out, [&](const Plan &p, const auto &places) {
            scale_kernel<<<ctas_for(c, p.chunks), kThreads, 0, st>>>(p, places, partial, partials, max_norm, norm, !d_out);
            norm = nullptr;
            return cudaGetLastError();
        });
    if (e != cudaSuccess)
        cudaGetLastError();
    if (prev != c->device)
        cudaSetDevice(prev);
    return e == cudaSuccess ? GNMR_OK : fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
}

gnmr_status gnmr_clip_destroy(gnmr_clip *c)
{
    if (!c)
        return GNMR_OK;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaSetDevice(c->device);
    const cudaError_t e = c->dmem ? cudaFree(c->dmem) : cudaSuccess;
    cudaSetDevice(prev);
    delete c;
    return e == cudaSuccess ? GNMR_OK : GNMR_ERR_CUDA;
}

}  // extern "C"
