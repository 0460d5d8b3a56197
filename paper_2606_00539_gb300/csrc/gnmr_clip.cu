// The norm over many tensors, and the tensors scaled down to a limit.
//
//   norm = sqrt(sum of x^2), scale = min(1, max_norm / norm), out = x scale
//
// Two kernels: sums of squares, a partial sum from each CTA; then every CTA of the second one adds the
// partial sums up in the same order, which takes it a microsecond, and scales its share.  Both are bound by
// memory: the gradients are read twice (once where nothing is written: in place, below the limit) and
// written once.  Where the tensors lie comes with each call, as kernel parameters, so that a captured
// call keeps its own; who takes what is in the plan: every warp an equal share of all tensors, laid end to end.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "gnmr.h"
#include "gnmr_internal.h"
#include "gnmr_rows.cuh"
#include "gnmr_stream.cuh"

namespace {

// A tensor of a plan: its length, and where its share of the tensors laid end to end begins.
struct alignas(16) Entry {
    int64_t length, first;                             // elements; units
    int32_t dtype;
};

// A kernel's CTAs, and where the table of its warps' first tensors begins (of its CTAs', where outputs are in other memory: many
// with little each), one more than there are.
struct Grid {
    int ctas;
    size_t start;
};

// The tensors of one launch.
struct Launch {
    int from, tensors;
    int64_t unit0, units;
    Grid squares, both, in_place;                      // both: outputs in other memory
};

}  // namespace

struct gnmr_clip {
    int device = 0;
    std::vector<Entry> entries;                        // and one behind the last
    std::vector<Launch> launches;
    std::vector<int32_t> start;                        // the launches' tables of their warps' first tensors

    size_t entries_bytes() const { return entries.size() * sizeof(Entry); }
};

namespace {

using namespace gnmr_rows;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// Few warps with many loads each on their way: 2.4 GB of bf16 took the first kernel 340 us so (7.1 TB/s), with 8
// loads a lane and four CTAs an SM 377, with two 569.
constexpr int kUnroll = 16, kSquaresCtas = 2;          // 16-byte loads a lane; CTAs an SM
// The second kernel, into other memory: CTAs of 64 KB, as they come, with 8 loads a lane: 2.4 GB 720 us (6.7 TB/s moved), 8 CTAs an
// SM that stay 763; 256 MB 83.  In place most calls end with the limit not reached, and then the CTAs are what they cost: 64 an
// SM 85 us, 4 4 us more than 2.  Calls that do scale in place pay for so few: 2.4 GB 1025 us by given norms (4.7 TB/s moved), 1381 with
// the norm's reading; 268 MB 107 and 137.  Three types' loops in one kernel spill: 384 bytes a thread stored into other memory, 508 in place.
constexpr int kBothCtas = 256, kBothLeast = 4, kInPlaceCtas = 2;
constexpr int64_t kBothUnits = 128;                    // of a CTA, beyond kBothLeast an SM
constexpr int kMostSquares = 512;                      // the first kernel's CTAs, each with a partial sum

// Shares are counted in units of 512 bytes, and four for beginning a tensor: a microsecond's latency,
// in which a warp's part of the memory's rate is 1.4 KB.
constexpr int64_t kUnit = 512, kBegin = 4;
// A warp takes 4 KB at least.
constexpr int64_t kLeastUnits = 8;

struct Plan {
    const Entry *entries;                              // [tensors + 1], those of the launch
    const int32_t *start;                              // each warp's, or CTA's, first tensor, and one more
    int tensors;
    int64_t unit0, units;
};

template <int kN> struct Places {
    const char *in[kN];
};

template <int kN, bool kBoth> struct Outs {
    char *out[kBoth ? kN : 1];
};

struct Share {
    int64_t u0, u1;                                    // units
};

__device__ __forceinline__ Share share_of(const Plan &p, int64_t w, int64_t all) { return {p.unit0 + p.units * w / all, p.unit0 + p.units * (w + 1) / all}; }

// The elements of an entry that lie in a share.
__device__ __forceinline__ void part_of(const Entry &e, const Share &s, int64_t &from, int64_t &to)
{
    const int64_t each = e.dtype == GNMR_DTYPE_F32 ? kUnit / 4 : kUnit / 2;
    from = min(max(s.u0 - e.first - kBegin, int64_t(0)) * each, e.length);
    to = min(max(s.u1 - e.first - kBegin, int64_t(0)) * each, e.length);
}

template <int DT> __device__ __forceinline__ double squares(const char *at, int64_t n, int lane)
{
    bool suspect;
    const double s = gnmr::warp_segment_sumsq<DT, kUnroll>(at, n, lane, suspect);
    return suspect ? gnmr::warp_segment_sumsq_f64<DT>(at, n, lane) : s;
}

// A CTA's sum from its warps', in their order; in thread 0.
__device__ __forceinline__ double cta_total(double sum, double *shared)
{
    if ((threadIdx.x & 31) == 0)
        shared[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < kWarps; ++i)
            sum += shared[i];
    return sum;
}

// This CTA's partial sum.
template <int kN>
__global__ void __launch_bounds__(kThreads, kSquaresCtas) squares_kernel(const __grid_constant__ Plan p, const __grid_constant__ Places<kN> places, double *partial)
{
    __shared__ double sums[kWarps];
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const Share share = share_of(p, w, int64_t(gridDim.x) * kWarps);
    double sum = 0.0;
    int t = __ldg(p.start + w);
    Entry e = p.entries[t];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    while (t < p.tensors && e.first < share.u1) {
        int64_t from, to;
        part_of(e, share, from, to);
        const int dtype = e.dtype;
        const char *const at = places.in[t] + from * (dtype == GNMR_DTYPE_F32 ? 4 : 2);
        e = p.entries[++t];
        if (from >= to)
            continue;
        if (dtype == GNMR_DTYPE_F32)
            sum += squares<GNMR_DTYPE_F32>(at, to - from, lane);
        else if (dtype == GNMR_DTYPE_BF16)
            sum += squares<GNMR_DTYPE_BF16>(at, to - from, lane);
        else
            sum += squares<GNMR_DTYPE_F16>(at, to - from, lane);
    }
    sum = cta_total(sum, sums);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = sum;
}

// The same from norms.
__global__ void __launch_bounds__(kThreads) norms_kernel(const double *norms, int64_t n, double *partial)
{
    __shared__ double sums[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    double sum = 0.0;
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads)
        sum = fma(norms[i], norms[i], sum);
    sum = cta_total(gnmr::warp_allreduce_sum(sum), sums);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = sum;
}

// Vectors 0, 32, ... from here on, as far as they are below `there`: kBatch of them at most.
template <typename T, int kBatch> __device__ __forceinline__ void scale_batch(const uint4 *in, uint4 *out, int there, float scale)
{
    uint4 v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
        if (32 * j < there)
            v[j] = load_once(in + 32 * j);
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
        if (32 * j < there) {
            float f[kIn16<T>];
            widen<T>(v[j], f);
#pragma unroll
            for (int k = 0; k < kIn16<T>; ++k)
                f[k] *= scale;
            store_once(out + 32 * j, narrow<T>(f));
        }
}

// n elements scaled, by a warp, the last ones first: those that the first kernel read last are still in L2.  An output that starts otherwise
// than its gradient, seen from multiples of 16 bytes, is written by elements, one a lane: 2.4 GB 3.8 ms with the norm, where alike starts
// take 1.06; 268 MB 0.43 and 0.13.
template <typename T, int kBatch> __device__ __forceinline__ void scale_part(const T *in, T *out, int64_t n, float scale, int lane)
{
    constexpr int kV = kIn16<T>;
    const int64_t head = min(n, int64_t((16 - (reinterpret_cast<uintptr_t>(in) & 15)) & 15) / int64_t(sizeof(T)));
    const bool alike = ((reinterpret_cast<uintptr_t>(in) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
    const int64_t vecs = alike ? (n - head) / kV : 0;
    // what lies around the vectors
    const int64_t rest = n - vecs * kV;
    for (int64_t i = lane; i < rest; i += 32) {
        const int64_t at = i < head ? i : i + vecs * kV;
        out[at] = from_f32<T>(to_f32(in[at]) * scale);
    }
    const uint4 *const from = reinterpret_cast<const uint4 *>(in + head) + lane;
    uint4 *const to = reinterpret_cast<uint4 *>(out + head) + lane;
    int64_t end = vecs;
    for (; end >= 32 * kBatch; end -= 32 * kBatch)
        scale_batch<T, kBatch>(from + (end - 32 * kBatch), to + (end - 32 * kBatch), 32 * kBatch, scale);
    if (end > 0)
        scale_batch<T, kBatch>(from, to, static_cast<int>(end) - lane, scale);
}

template <int kN, bool kBoth>
__global__ void __launch_bounds__(kThreads, kBoth ? 4 : 2)
scale_kernel(const __grid_constant__ Plan p, const __grid_constant__ Places<kN> places, const __grid_constant__ Outs<kN, kBoth> outs,
             const double *partial, int partials, double max_norm, float *norm_out)
{
    __shared__ float scale_of_all;
    constexpr int kBatch = kBoth ? 8 : 16;             // loads a lane
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const Share share = share_of(p, w, int64_t(gridDim.x) * kWarps);
    int t = __ldg(p.start + (kBoth ? int64_t(blockIdx.x) : w) + 1);         // at or behind the last one
    Entry e = p.entries[t];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // by one warp: the SM's 64-bit unit takes 20 cycles an instruction, whoever they come from
    if (threadIdx.x < 32) {
        double sum = 0.0;
#pragma unroll 4
        for (int i = lane; i < partials; i += 32)
            sum += __ldcg(partial + i);
        sum = gnmr::warp_allreduce_sum(sum);
        if (lane == 0) {
            float scale = 1.0f;
            if (blockIdx.x == 0 || sum > 0.999999 * max_norm * max_norm) {       // else surely below the limit
                const double norm = sqrt(sum);
                // a norm that is not finite compares as not above the limit, or as infinite
                if (norm > max_norm && isfinite(norm))
                    scale = static_cast<float>(max_norm / norm);
                if (blockIdx.x == 0 && norm_out)
                    *norm_out = static_cast<float>(norm);
            }
            scale_of_all = scale;
        }
    }
    __syncthreads();
    const float scale = scale_of_all;
    if (!kBoth && scale == 1.0f)
        return;
    for (;;) {
        int64_t from, to;
        part_of(e, share, from, to);
        if (t < p.tensors && from < to) {
            const int64_t at = from * (e.dtype == GNMR_DTYPE_F32 ? 4 : 2);
            const char *const in = places.in[t] + at;
            char *const out = kBoth ? outs.out[t] + at : const_cast<char *>(in);
            if (e.dtype == GNMR_DTYPE_F32)
                scale_part<float, kBatch>(reinterpret_cast<const float *>(in), reinterpret_cast<float *>(out), to - from, scale, lane);
            else if (e.dtype == GNMR_DTYPE_BF16)
                scale_part<__nv_bfloat16, kBatch>(reinterpret_cast<const __nv_bfloat16 *>(in), reinterpret_cast<__nv_bfloat16 *>(out), to - from, scale, lane);
            else
                scale_part<__half, kBatch>(reinterpret_cast<const __half *>(in), reinterpret_cast<__half *>(out), to - from, scale, lane);
        }
        if (t == 0 || e.first <= share.u0)
            return;
        e = p.entries[--t];
    }
}

// ---- host -----------------------------------------------------------------------

constexpr int kMost = 2000;                            // tensors of one launch: places in 32,764 bytes of parameters

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

cudaLaunchConfig_t config(int ctas, cudaStream_t st, cudaLaunchAttribute *attr)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    attr->id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr->val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

template <int kN> Places<kN> places_of(const Launch &l, const void *const *in)
{
    Places<kN> p;
    std::copy(in + l.from, in + l.from + l.tensors, reinterpret_cast<const void **>(p.in));
    return p;
}

Plan plan_of(const gnmr_clip *c, const void *table, const Launch &l, const Grid &g)
{
    const char *const at = static_cast<const char *>(table);
    return {reinterpret_cast<const Entry *>(at) + l.from, reinterpret_cast<const int32_t *>(at + c->entries_bytes()) + g.start, l.tensors, l.unit0,
            l.units};
}

template <int kN> cudaError_t launch_squares(const gnmr_clip *c, const void *table, const Launch &l, const void *const *in, double *partial, cudaStream_t st)
{
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = config(l.squares.ctas, st, &attr);
    return cudaLaunchKernelEx(&cfg, squares_kernel<kN>, plan_of(c, table, l, l.squares), places_of<kN>(l, in), partial);
}

template <int kN, bool kBoth>
cudaError_t launch_scale(const gnmr_clip *c, const void *table, const Launch &l, const void *const *in, void *const *out, const double *partial, int partials,
                         double max_norm, float *norm, cudaStream_t st)
{
    Outs<kN, kBoth> outs;
    if (kBoth)
        std::copy(out + l.from, out + l.from + l.tensors, reinterpret_cast<void **>(outs.out));
    const Grid &g = kBoth ? l.both : l.in_place;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = config(g.ctas, st, &attr);
    return cudaLaunchKernelEx(&cfg, scale_kernel<kN, kBoth>, plan_of(c, table, l, g), places_of<kN>(l, in), outs, partial, partials, max_norm, norm);
}

// Calls f with the capacity that a launch's parameters take, as a constant.
template <typename F> cudaError_t by_capacity(const Launch &l, F f)
{
    if (l.tensors <= 64)
        return f(std::integral_constant<int, 64>());
    if (l.tensors <= 400)
        return f(std::integral_constant<int, 400>());
    return f(std::integral_constant<int, kMost>());
}

// The launches and each one's table of where its warps begin, for tensors laid end to end.
void cut(gnmr_clip *c, int sms)
{
    std::vector<int32_t> &start = c->start;
    const int all = static_cast<int>(c->entries.size()) - 1;
    for (int from = 0; from < std::max(all, 1); from += kMost) {
        Launch l = {};
        l.from = from;
        l.tensors = std::min(kMost, all - from);
        l.unit0 = c->entries[from].first;
        l.units = c->entries[from + l.tensors].first - l.unit0;
        const int64_t most = std::max<int64_t>(1, l.units / (kLeastUnits * kWarps));
        l.squares.ctas = static_cast<int>(std::min<int64_t>(most, std::min(sms * kSquaresCtas, kMostSquares)));
        l.both.ctas = static_cast<int>(std::min<int64_t>(std::max<int64_t>(std::min<int64_t>(most, sms * kBothLeast), l.units / kBothUnits), sms * kBothCtas));
        l.in_place.ctas = static_cast<int>(std::min<int64_t>(most, sms * kInPlaceCtas));
        for (Grid *g : {&l.squares, &l.both, &l.in_place}) {
            const int64_t shares = int64_t(g->ctas) * (g == &l.both ? 1 : kWarps);
            g->start = start.size();
            int t = 0;
            for (int64_t w = 0; w <= shares; ++w) {
                while (t < l.tensors && c->entries[from + t + 1].first <= l.unit0 + l.units * w / shares)
                    ++t;
                start.push_back(t);
            }
        }
        c->launches.push_back(l);
    }
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
    int sms = 1;
    if (const cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)) {
        cudaGetLastError();
        return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    gnmr_clip *c = nullptr;
    try {
        c = new gnmr_clip;
        c->device = device;
        c->entries.resize(num_tensors + 1);
        int64_t units = 0;
        for (int i = 0; i < num_tensors; ++i) {
            c->entries[i] = Entry{lengths[i], units, dtypes[i]};
            if (lengths[i])
                units += kBegin + (lengths[i] * int64_t(element_bytes(dtypes[i])) + kUnit - 1) / kUnit;
        }
        c->entries[num_tensors] = Entry{0, units, 0};
        cut(c, sms);
    } catch (const std::bad_alloc &) {
        delete c;
        return fail(GNMR_ERR_OOM, "clip: host allocation failed");
    }
    *out = c;
    return GNMR_OK;
}

gnmr_status gnmr_clip_table_bytes(const gnmr_clip *c, int64_t *bytes)
{
    if (!c || !bytes)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument");
    *bytes = static_cast<int64_t>(c->entries_bytes() + c->start.size() * sizeof(int32_t));
    return GNMR_OK;
}

gnmr_status gnmr_clip_write_table(const gnmr_clip *c, void *table)
{
    if (!c || !table)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument");
    memcpy(table, c->entries.data(), c->entries_bytes());
    memcpy(static_cast<char *>(table) + c->entries_bytes(), c->start.data(), c->start.size() * sizeof(int32_t));
    return GNMR_OK;
}

gnmr_status gnmr_clip_scratch_bytes(const gnmr_clip *c, int64_t *bytes)
{
    if (!c || !bytes)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument");
    *bytes = int64_t(c->launches.size()) * kMostSquares * sizeof(double);
    return GNMR_OK;
}

gnmr_status gnmr_clip_run(const gnmr_clip *c, const void *d_table, const void *const *d_in, void *const *d_out, double max_norm,
                          const double *d_unit_norms, int64_t num_norms, float *d_norm, void *d_scratch, int64_t scratch_bytes, void *stream)
{
    const int tensors = c ? static_cast<int>(c->entries.size()) - 1 : 0;
    if (!c || !d_table || !d_norm || (tensors > 0 && !d_in) || num_norms < 0)
        return fail(GNMR_ERR_INVALID_ARG, "clip: NULL argument, or a negative number of norms");
    if (!(max_norm >= 0))
        return fail(GNMR_ERR_INVALID_ARG, "clip: max_norm has to be 0 or more");
    int64_t need = 0;
    gnmr_clip_scratch_bytes(c, &need);
    if (!d_scratch || scratch_bytes < need || misaligned(d_scratch, 256))
        return fail(GNMR_ERR_LAYOUT, "clip: scratch missing, too small or misaligned");
    if (misaligned(d_table, 16) || misaligned(d_unit_norms, 8) || misaligned(d_norm, 4))
        return fail(GNMR_ERR_LAYOUT, "clip: a buffer not aligned to its element size");
    for (int i = 0; i < tensors; ++i) {
        const size_t eb = element_bytes(c->entries[i].dtype);
        if (c->entries[i].length > 0 && (!d_in[i] || (d_out && !d_out[i])))
            return fail(GNMR_ERR_INVALID_ARG, "clip: NULL tensor");
        if (misaligned(d_in[i], eb) || (d_out && misaligned(d_out[i], eb)))
            return fail(GNMR_ERR_LAYOUT, "clip: a tensor not aligned to its element size");
    }
    int prev = c->device;
    cudaGetDevice(&prev);
    if (prev != c->device)
        cudaSetDevice(c->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    double *const partial = static_cast<double *>(d_scratch);
    int partials = 0;
    cudaError_t e = cudaSuccess;
    if (d_unit_norms) {
        partials = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((num_norms + kThreads - 1) / kThreads, 128)));
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = config(partials, st, &attr);
        e = cudaLaunchKernelEx(&cfg, norms_kernel, d_unit_norms, num_norms, partial);
    } else {
        for (const Launch &l : c->launches)
            if (e == cudaSuccess) {
                e = by_capacity(l, [&](auto n) { return launch_squares<n.value>(c, d_table, l, d_in, partial + partials, st); });
                partials += l.squares.ctas;
            }
    }
    float *norm = d_norm;
    for (const Launch &l : c->launches)
        if (e == cudaSuccess) {
            e = by_capacity(l, [&](auto n) {
                return d_out ? launch_scale<n.value, true>(c, d_table, l, d_in, d_out, partial, partials, max_norm, norm, st)
                             : launch_scale<n.value, false>(c, d_table, l, d_in, nullptr, partial, partials, max_norm, norm, st);
            });
            norm = nullptr;
        }
    if (e != cudaSuccess)
        cudaGetLastError();
    if (prev != c->device)
        cudaSetDevice(prev);
    return e == cudaSuccess ? GNMR_OK : fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
}

gnmr_status gnmr_clip_destroy(gnmr_clip *c)
{
    delete c;
    return GNMR_OK;
}

}  // extern "C"
