// Expert products: the linear units of both paths, grouped by expert.
//
// Every product is out[col][lane] = sum over c of A[lane][c] B[col][c]:
//   forward      A = W_g      [n_out lanes], c along its rows     B = x's rows    c < n_in
//   input grad   A = W_g^T    [n_in lanes], lanes along its rows  B = dy's rows   c < n_out
//   weight grad  A = x^T      [n_in lanes], lanes along its rows  B = dy^T        c < the group's rows
// so that the tensor cores' 128 lanes lie along the output's contiguous axis and a
// group's ragged rows are columns, of which a tile has any multiple of 32 up to 256.
//
// A pair of CTAs computes 256 lanes by up to 256 columns (two SMs share an operand
// tile: 32 KB of operands an SM for 64 steps of the contraction, where one SM alone
// would need 48).  Per CTA: one warp has the TMA unit load tiles of 64 steps into a
// ring of stages, one (of the first CTA) issues the multiplies, eight add up the
// finished pieces and write the outputs, and one clears what the last tile of a
// group's rows holds past their end (weight gradient).
//
// A piece is at most 1,024 steps (512 for fp32 outputs).  The tensor cores cut
// sums that they hold rather than rounding them: 2,047 steps in one piece were
// 1.5e-6 of the result off, in fp32 arithmetic 3.9e-7.  Pieces are added in registers,
// rounded, while the next one is multiplied into the other half of tensor memory.  For
// 8-bit codes a piece's sum is below 2^24, an exact integer in fp32, and pieces
// are added as integers.
//
// Where there are fewer tiles than pairs, a tile's contraction is split over
// several pairs; each writes its part, and the last one to finish adds them up
// in their order.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <new>

#include "gnmr.h"
#include "gnmr_internal.h"
#include "gnmr_mma.cuh"

namespace {

constexpr int kMaxGroups = 2048;
constexpr int kMaxPairs = 80;
constexpr int kMaxParts = 2 * kMaxPairs;               // split tiles' parts in one call
constexpr int64_t kPartFloats = 256 * 256;             // one part: both CTAs' lanes by the columns

}  // namespace

struct gnmr_products {
    int device = 0;
    int pairs = 1;
    float *parts = nullptr;            // [kMaxParts][kPartFloats]
    unsigned *tickets = nullptr;       // [kMaxParts][2], 0 between calls
    int *gave_up = nullptr;            // host memory that the kernels can write
    void *dmem = nullptr;
    CUresult (*encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                       const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                       CUtensorMapL2promotion, CUtensorMapFloatOOBfill) = nullptr;
};

namespace {

using namespace gnmr_mma;

constexpr int kLanes = 256;                            // of a pair's tile
constexpr int kStep = 64;                              // contraction steps of a stage: 128-byte rows of 16 bits
constexpr int kEpilogueWarps = 8;
constexpr int kProducerWarp = 0, kMultiplyWarp = 1, kFirstEpilogueWarp = 2, kTailWarp = kFirstEpilogueWarp + kEpilogueWarps;
constexpr int kThreads = 32 * (kTailWarp + 1);
constexpr int kAStage = 128 * 128;                     // bytes of A's tile in one CTA
constexpr int kBlock = 64 * 128;                       // bytes of a tile of 64 lanes or columns lying along rows

// kColumns columns at most; a CTA loads half of B's tile, in boxes of kBox rows.
template <int kColumns> struct Shape {
    static constexpr int kBStage = kColumns / 2 * 128;
    static constexpr int kStage = kAStage + (kBStage < kBlock ? kBlock : kBStage);
    static constexpr int kStages = kColumns == 256 ? 6 : 8;
    static constexpr int kBox = kColumns == 256 ? 64 : 16;
    static constexpr int kTmem = 2 * kColumns;
    static constexpr int kPieces = kColumns / 2 / 16;  // 16-column pieces of an epilogue warp
};

struct Product {
    int lanes, depth, cols;            // depth, or cols, is 0 where it is a group's rows
    int rows, groups;
    const int64_t *offsets;
    const uint8_t *mask;
    int64_t mask_stride;
    int want;                          // groups computed: mask byte != 0 (1), == 0 (0)
    int a_along_lanes, b_along_columns;
    int a_by_group;                    // A's third coordinate is the group
    int bf16;
    int chunk;                         // stages of a piece
    void *out;
    int out_type;
    int pairs_aligned;                 // two outputs of a row may be stored as one
    int add;
    int64_t out_col, out_group;
    const float *lane_scale, *col_scale;
    float *parts;
    unsigned *tickets;
    int *gave_up;
};

// ---- work: tiles of every group, and their parts --------------------------------

struct Tables {
    int first[kMaxGroups + 1];         // tiles before group g; in the end all of them
    int row[kMaxGroups + 1];           // first row of group g; in the end the last group's end
    int split;                         // parts of every tile's contraction
};

struct Item {
    int g, lane0, col0, cols;          // the tile: the pair's lanes, and its columns
    int row0;                          // the group's first row
    int depth, k0, k1;                 // the whole contraction; the stages of this part
    int tile, part;
};

__device__ __forceinline__ int parts_of(int n, int each) { return (n + each - 1) / each; }

// Filled by one warp.  Offsets are clamped to [0, rows] and made not decreasing.
__device__ __forceinline__ void fill_tables(const Product &p, Tables &t, int most, int lane_tiles, int pairs)
{
    const int lane = threadIdx.x & 31;
    int carry = 0;
    for (int j0 = 0; j0 <= p.groups; j0 += 32) {
        const int j = j0 + lane;
        int at = j == 0 ? 0 : p.rows;
        if (p.offsets && j <= p.groups)
            at = static_cast<int>(min(max(p.offsets[j], int64_t(0)), int64_t(p.rows)));
        at = max(at, carry);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(~0u, at, d);
            if (lane >= d)
                at = max(at, v);
        }
        if (j <= p.groups)
            t.row[j] = at;
        carry = __shfl_sync(~0u, at, 31);
    }
    __syncwarp();
    int tiles = 0, deepest = 0;
    for (int g0 = 0; g0 < p.groups; g0 += 32) {
        const int g = g0 + lane;
        int n = 0;
        if (g < p.groups && (!p.mask || (p.mask[g * p.mask_stride] != 0) == (p.want != 0))) {
            const int rows = t.row[g + 1] - t.row[g];
            n = lane_tiles * parts_of(p.cols ? p.cols : rows, most);
            deepest = max(deepest, p.depth ? p.depth : rows);
        }
        int sum = n;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(~0u, sum, d);
            if (lane >= d)
                sum += v;
        }
        if (g < p.groups)
            t.first[g] = tiles + sum - n;
        tiles += __shfl_sync(~0u, sum, 31);
    }
    // Few tiles: the number of parts that takes the fewest rounds of stages, a
    // part costing about six stages more for its beginning and its joining.
    int best = 1;
    if (tiles > 0 && tiles < pairs) {
        const int stages = parts_of(__reduce_max_sync(~0u, deepest), kStep), parts = lane + 1;
        const bool fits = parts == 1 || (tiles * parts <= min(2 * pairs, kMaxParts) && 2 * parts <= stages);
        const int cost = fits ? parts_of(tiles * parts, pairs) * (parts_of(stages, parts) + (parts > 1 ? 6 : 0)) : INT32_MAX;
        const int least = __reduce_min_sync(~0u, cost);
        best = __ffs(__ballot_sync(~0u, cost == least));
    }
    if (lane == 0) {
        t.first[p.groups] = tiles;
        t.split = best;
    }
}

template <int kColumns>
__device__ __forceinline__ Item item_of(const Product &p, const Tables &t, int lane_tiles, int i)
{
    Item it;
    it.tile = i / t.split;
    it.part = i - it.tile * t.split;
    int lo = 0, hi = p.groups;                       // the last group that begins at or before the tile
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= it.tile)
            lo = mid;
        else
            hi = mid;
    }
    it.g = lo;
    it.row0 = t.row[lo];
    const int rows = t.row[lo + 1] - it.row0, at = it.tile - t.first[lo];
    const int cols = p.cols ? p.cols : rows;
    // a group's columns are shared out evenly, in multiples of 32
    const int each = (parts_of(cols, parts_of(cols, kColumns)) + 31) / 32 * 32;
    const int c = at / lane_tiles;
    it.lane0 = (at - c * lane_tiles) * kLanes;
    it.col0 = c * each;
    it.cols = min(each, cols - it.col0);
    it.depth = p.depth ? p.depth : rows;
    const int stages = parts_of(it.depth, kStep);
    it.k0 = static_cast<int>(int64_t(stages) * it.part / t.split);
    it.k1 = static_cast<int>(int64_t(stages) * (it.part + 1) / t.split);
    return it;
}

// ---- outputs --------------------------------------------------------------------

__device__ __forceinline__ unsigned pack(float lo, float hi, int type)
{
    if (type == GNMR_DTYPE_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return reinterpret_cast<const unsigned &>(v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const unsigned &>(v);
}

__device__ __forceinline__ float load_out(const void *at, int type)
{
    return type == GNMR_DTYPE_F32    ? *static_cast<const float *>(at)
           : type == GNMR_DTYPE_BF16 ? __bfloat162float(*static_cast<const __nv_bfloat16 *>(at))
                                     : __half2float(*static_cast<const __half *>(at));
}

// 16 columns of this thread's lane.  Two lanes' values of a column go out as one
// where they can: 64 contiguous bytes a column from a warp.
__device__ __forceinline__ void store16(const Product &p, const Item &it, int lane, int col, float (&v)[16])
{
    const int64_t base = p.cols ? it.g * p.out_group + int64_t(it.col0 + col) * p.out_col
                                : int64_t(it.row0 + it.col0 + col) * p.out_col;
    const int left = it.cols - col;
    const bool mine = lane < p.lanes;
    if (p.out_type == GNMR_DTYPE_F32) {
        float *out = static_cast<float *>(p.out) + base + lane;
        if (p.add)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (mine && j < left)
                    v[j] += out[j * p.out_col];
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (mine && j < left)
                out[j * p.out_col] = v[j];
        return;
    }
    uint16_t *out = static_cast<uint16_t *>(p.out) + base + lane;
    if (p.add)
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (mine && j < left)
                v[j] += load_out(out + j * p.out_col, p.out_type);
    const int odd = lane & 1;
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
        const float other = __shfl_xor_sync(~0u, odd ? v[j] : v[j + 1], 1);
        const unsigned w = odd ? pack(other, v[j + 1], p.out_type) : pack(v[j], other, p.out_type);
        const int k = j + odd;                       // the column that this thread writes, lanes lane & ~1 and the next
        uint16_t *to = out - odd + k * p.out_col;
        if (k < left) {
            if (p.pairs_aligned && (lane | 1) < p.lanes) {
                *reinterpret_cast<unsigned *>(to) = w;
            } else {
                if ((lane & ~1) < p.lanes)
                    to[0] = static_cast<uint16_t>(w);
                if ((lane | 1) < p.lanes)
                    to[1] = static_cast<uint16_t>(w >> 16);
            }
        }
    }
}

template <bool kCodes>
__device__ __forceinline__ void finish16(const Product &p, const Item &it, int lane, int col, uint32_t (&acc)[16])
{
    float v[16];
    if (kCodes) {
        const float by_lane = lane < p.lanes ? p.lane_scale[int64_t(it.g) * p.lanes + lane] : 0.0f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float by_col = col + j < it.cols ? p.col_scale[it.row0 + it.col0 + col + j] : 0.0f;
            v[j] = static_cast<float>(static_cast<int>(acc[j])) * by_col * by_lane;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            v[j] = __uint_as_float(acc[j]);
    }
    store16(p, it, lane, col, v);
}

template <bool kCodes>
__device__ __forceinline__ void add_piece(uint32_t (&acc)[16], const uint32_t (&v)[16], bool first)
{
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        if (kCodes) {
            const int whole = __float2int_rn(__uint_as_float(v[j]));
            acc[j] = first ? whole : static_cast<int>(acc[j]) + whole;
        } else {
            acc[j] = first ? v[j] : __float_as_uint(__uint_as_float(acc[j]) + __uint_as_float(v[j]));
        }
    }
}

// ---- the kernel -------------------------------------------------------------------

struct Barriers {
    uint64_t full[8], empty[8];        // stages; `full` counts in the first CTA of the pair
    uint64_t tail[8];                  // a stage that the tail warp looks at first
    uint64_t done[2], drained[2];      // halves of tensor memory; `drained` counts in the first CTA
    uint64_t written, counted;         // of a split tile's part: by its warps, and its ticket
    uint32_t tmem;
    unsigned last;                     // whether this CTA is a split tile's last
};

template <int kColumns, bool kCodes>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Product p)
{
    using S = Shape<kColumns>;
    extern __shared__ uint8_t dynamic[];
    uint8_t *stages = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    Tables &tables = *reinterpret_cast<Tables *>(stages + S::kStages * S::kStage);
    __shared__ Barriers bars;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int lane_tiles = parts_of(p.lanes, kLanes);

    if (warp == kProducerWarp && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < S::kStages; ++s) {
            barrier_init(smem_addr(&bars.full[s]), 2);
            barrier_init(smem_addr(&bars.empty[s]), 1);
            barrier_init(smem_addr(&bars.tail[s]), 1);
        }
        for (int h = 0; h < 2; ++h) {
            barrier_init(smem_addr(&bars.done[h]), 1);
            barrier_init(smem_addr(&bars.drained[h]), 2 * kEpilogueWarps);
        }
        barrier_init(smem_addr(&bars.written), kEpilogueWarps);
        barrier_init(smem_addr(&bars.counted), 1);
        barrier_init_fence();
    }
    if (warp == kMultiplyWarp)
        tmem_alloc(smem_addr(&bars.tmem), S::kTmem);
    if (warp == kTailWarp)
        fill_tables(p, tables, kColumns, lane_tiles, pairs);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = bars.tmem;
    const int items = tables.first[p.groups] * tables.split;
    const bool rows_deep = p.depth == 0;               // the contraction is a group's rows
    bool fine = true;

    if (warp == kProducerWarp) {
        if (lane == 0) {
            const uint32_t first = in_cta(smem_addr(&bars.full[0]), 0);
            int stage = 0;
            uint32_t phase = 0;
            for (int i = pair; fine && i < items; i += pairs) {
                const Item it = item_of<kColumns>(p, tables, lane_tiles, i);
                const int half = (it.cols + 31) / 32 * 16;                 // B's columns in this CTA
                const int a_lane = it.lane0 + rank * 128, b_col = it.col0 + rank * half;
                const int box_b = p.b_along_columns ? 64 : S::kBox, boxes = parts_of(half, box_b);
                const uint32_t bytes = kAStage + boxes * box_b * 128;
                for (int k = it.k0; k < it.k1; ++k) {
                    if (!(fine = wait(smem_addr(&bars.empty[stage]), phase ^ 1)))
                        break;
                    const bool tail = rows_deep && (k + 1) * kStep > it.depth;
                    const uint32_t bar = tail ? smem_addr(&bars.tail[stage]) : first + stage * 8;
                    arrive_expect(tail ? in_cta(bar, rank) : bar, bytes);
                    const uint32_t a = smem_addr(stages + stage * S::kStage), b = a + kAStage;
                    const int c = k * kStep + (rows_deep ? it.row0 : 0);
                    const int za = p.a_by_group ? it.g : 0;
                    if (p.a_along_lanes) {
                        load_tile(a, &map_a, a_lane, c, za, bar);
                        load_tile(a + kBlock, &map_a, a_lane + 64, c, za, bar);
                    } else {
                        load_tile(a, &map_a, c, a_lane, za, bar);
                    }
                    for (int q = 0; q < boxes; ++q)
                        if (p.b_along_columns)
                            load_tile(b + q * kBlock, &map_b, b_col + q * 64, c, 0, bar);
                        else
                            load_tile(b + q * S::kBox * 128, &map_b, c, it.row0 + b_col + q * S::kBox, 0, bar);
                    if (++stage == S::kStages)
                        stage = 0, phase ^= 1;
                }
            }
        }
    } else if (warp == kMultiplyWarp) {
        if (lane == 0 && rank == 0) {
            int stage = 0, half = 0;
            uint32_t phase = 0, drained = 0;
            const uint32_t a_lead = p.a_along_lanes ? kBlock : 16, b_lead = p.b_along_columns ? kBlock : 16;
            const uint32_t a_next = (p.a_along_lanes ? 16 * 128 : 32) >> 4, b_next = (p.b_along_columns ? 16 * 128 : 32) >> 4;
            for (int i = pair; fine && i < items; i += pairs) {
                const Item it = item_of<kColumns>(p, tables, lane_tiles, i);
                const uint32_t idesc = shape(p.bf16, p.a_along_lanes, p.b_along_columns, (it.cols + 31) / 32 * 32);
                for (int k = it.k0; fine && k < it.k1;) {
                    if (!(fine = wait(smem_addr(&bars.drained[half]), ((drained >> half) & 1) ^ 1)))
                        break;
                    drained ^= 1u << half;
                    fence_after();
                    const int stop = min(it.k1, k + p.chunk);
                    for (bool add = false; k < stop; ++k) {
                        if (!(fine = wait(smem_addr(&bars.full[stage]), phase)))
                            break;
                        fence_after();
                        const uint32_t a = smem_addr(stages + stage * S::kStage), b = a + kAStage;
                        const uint64_t da = operand(a, a_lead, 1024), db = operand(b, b_lead, 1024);
                        const int steps = parts_of(min(kStep, it.depth - k * kStep), 16);
                        for (int q = 0; q < steps; ++q, add = true)
                            multiply(tmem + half * kColumns, da + q * a_next, db + q * b_next, idesc, add);
                        commit(smem_addr(&bars.empty[stage]));
                        if (++stage == S::kStages)
                            stage = 0, phase ^= 1;
                    }
                    commit(smem_addr(&bars.done[half]));
                    half ^= 1;
                }
            }
        }
    } else if (warp == kTailWarp) {
        // The last stage of a group's rows holds rows of the next group: cleared up to
        // the next multiple of 16, beyond which nothing is multiplied.
        if (rows_deep) {
            const uint32_t full = in_cta(smem_addr(&bars.full[0]), 0);
            int stage = 0;
            uint32_t phase = 0;
            for (int i = pair; fine && i < items; i += pairs) {
                const Item it = item_of<kColumns>(p, tables, lane_tiles, i);
                const int left = it.depth % kStep, stages_of = it.k1 - it.k0;
                if (left && it.k1 * kStep > it.depth && stages_of > 0) {
                    const int at = (stage + stages_of - 1) % S::kStages;
                    if (!(fine = __all_sync(~0u, wait(smem_addr(&bars.tail[at]), (phase >> at) & 1))))
                        break;
                    phase ^= 1u << at;
                    const int blocks = 2 + parts_of((it.cols + 31) / 32 * 16, 64), stop = (left + 15) / 16 * 16;
                    uint4 *to = reinterpret_cast<uint4 *>(stages + at * S::kStage);
                    for (int q = 0; q < blocks; ++q)
                        for (int v = left * 8 + lane; v < stop * 8; v += 32)
                            to[q * (kBlock / 16) + v] = make_uint4(0, 0, 0, 0);
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0)
                        arrive(full + at * 8);
                }
                stage = (stage + stages_of) % S::kStages;
            }
        }
    } else {
        const int quarter = warp & 3, side = (warp - kFirstEpilogueWarp) >> 2;
        const uint32_t drained = in_cta(smem_addr(&bars.drained[0]), 0);
        int half = 0;
        uint32_t phase = 0, joins = 0;
        for (int i = pair; fine && i < items; i += pairs) {
            const Item it = item_of<kColumns>(p, tables, lane_tiles, i);
            const int span = (it.cols + 31) / 32 * 16;                      // columns of this warp
            const int at = it.lane0 + rank * 128 + quarter * 32 + lane, col = side * span;
            uint32_t acc[S::kPieces][16];
#pragma unroll
            for (int q = 0; q < S::kPieces; ++q)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    acc[q][j] = 0;
            for (int k = it.k0; k < it.k1; k += p.chunk) {
                if (!(fine = __all_sync(~0u, wait(smem_addr(&bars.done[half]), (phase >> half) & 1))))
                    break;
                phase ^= 1u << half;
                fence_after();
                const uint32_t from = tmem + half * kColumns + (uint32_t(quarter * 32) << 16) + col;
#pragma unroll
                for (int q = 0; q < S::kPieces; ++q)
                    if (q * 16 < span) {
                        uint32_t v[16];
                        load16(from + q * 16, v);
                        load_wait(v);
                        add_piece<kCodes>(acc[q], v, k == it.k0);
                    }
                fence_before();
                __syncwarp();
                if (lane == 0)
                    arrive(drained + half * 8);
                half ^= 1;
            }
            if (!fine)
                break;
            if (tables.split > 1) {
                // this part to memory; the last CTA of its rank to get here adds them all
                uint32_t *part = reinterpret_cast<uint32_t *>(p.parts) +
                                 (int64_t(it.tile) * tables.split) * kPartFloats + rank * (kPartFloats / 2) + quarter * 32 + lane;
#pragma unroll
                for (int q = 0; q < S::kPieces; ++q)
                    if (q * 16 < span)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            part[it.part * kPartFloats + (col + q * 16 + j) * 128] = acc[q][j];
                __threadfence();
                __syncwarp();
                if (lane == 0)
                    arrive(in_cta(smem_addr(&bars.written), rank));
                if (warp == kFirstEpilogueWarp) {
                    if (!(fine = __all_sync(~0u, wait(smem_addr(&bars.written), joins & 1))))
                        break;
                    if (lane == 0) {
                        const unsigned n = atomicAdd(&p.tickets[2 * it.tile + rank], 1u);
                        bars.last = n + 1 == static_cast<unsigned>(tables.split);
                        if (bars.last)
                            p.tickets[2 * it.tile + rank] = 0;
                        __threadfence();
                        arrive(in_cta(smem_addr(&bars.counted), rank));
                    }
                    __syncwarp();
                }
                if (!(fine = __all_sync(~0u, wait(smem_addr(&bars.counted), joins & 1))))
                    break;
                ++joins;
                const bool last = bars.last;
                if (!last)
                    continue;
#pragma unroll
                for (int q = 0; q < S::kPieces; ++q)
                    if (q * 16 < span) {
                        for (int s = 0; s < tables.split; ++s)
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const uint32_t v = __ldcg(part + s * kPartFloats + (col + q * 16 + j) * 128);
                                if (kCodes)
                                    acc[q][j] = s ? acc[q][j] + v : v;
                                else
                                    acc[q][j] = s ? __float_as_uint(__uint_as_float(acc[q][j]) + __uint_as_float(v)) : v;
                            }
                    }
            }
            if (p.add && it.depth == 0)
                continue;                              // nothing to add
#pragma unroll
            for (int q = 0; q < S::kPieces; ++q)
                if (q * 16 < span && col + q * 16 < it.cols)
                    finish16<kCodes>(p, it, at, col + q * 16, acc[q]);
        }
    }
    __syncwarp();
    if (!fine) {
        // Loads that a role left behind are in long before this ends.
        if (lane == 0)
            *p.gave_up = 1;
        for (int i = 0; i < 1000; ++i)
            __nanosleep(1000);
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    if (warp == kMultiplyWarp)
        tmem_free(tmem, S::kTmem);
}

// ---- operands that the TMA unit cannot read, and codes as 16-bit numbers ------------
// [groups][rows][cols] with any strides to rows of `held` 16-bit elements (a multiple of
// eight), the rest of each row 0.  Bound by memory.
struct Copy {
    const void *from;
    uint16_t *to;
    int64_t rows, cols, stride, group_stride, held, total;   // total: vectors of 8
};

template <typename T>
__global__ void __launch_bounds__(256) copy_kernel(Copy c)
{
    const int64_t across = c.held / 8;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < c.total; i += int64_t(gridDim.x) * 256) {
        const int64_t r = i / across, at = (i - r * across) * 8, g = r / c.rows;
        const T *from = static_cast<const T *>(c.from) + g * c.group_stride + (r - g * c.rows) * c.stride + at;
        uint16_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0;
            if (at + j < c.cols) {
                if (sizeof(T) == 1)
                    v[j] = __half_as_ushort(__int2half_rn(static_cast<int>(from[j])));
                else
                    v[j] = static_cast<uint16_t>(from[j]);
            }
        }
        uint4 w;
        memcpy(&w, v, 16);
        *reinterpret_cast<uint4 *>(c.to + i * 8) = w;
    }
}

// ---- host -----------------------------------------------------------------------

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
    if (p->groups < 1 || p->groups > kMaxGroups)
        return fail(GNMR_ERR_INVALID_ARG, "products: groups outside 1 .. 2048");
    const int64_t most = INT32_MAX / 2;                  // row and column numbers stay within 31 bits in tiles
    if (p->rows < 0 || p->rows > most || p->n_out < 1 || p->n_in < 1 || p->n_out > most || p->n_in > most)
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
    const int64_t far = int64_t(1) << 36;                // strides stay within what a tensor map takes
    if ((x && p->x_stride < p->n_in) || (dy && p->dy_stride < p->n_out) ||
        (w && (p->w_stride < p->n_in || p->w_group_stride < 0)) || p->out_stride < wide_out ||
        (wgrad && p->groups > 1 && p->out_group_stride < (p->n_out - 1) * p->out_stride + p->n_in) ||
        (p->d_mask && p->groups > 1 && p->mask_stride < 1))
        return fail(GNMR_ERR_LAYOUT, "products: a stride below what it strides over");
    if ((x && p->x_stride > far) || (dy && p->dy_stride > far) || (w && (p->w_stride > far || p->w_group_stride > far)) ||
        p->out_stride > far || (wgrad && p->out_group_stride > far))
        return fail(GNMR_ERR_LAYOUT, "products: a stride above 2^36 elements");
    const size_t eb = codes ? 1 : 2, ob = p->out_dtype == GNMR_DTYPE_F32 ? 4 : 2;
    if ((x && misaligned(p->d_x, eb)) || (dy && misaligned(p->d_dy, eb)) || (w && misaligned(p->d_w, eb)) ||
        misaligned(p->d_out, ob) || misaligned(p->d_offsets, 8) ||
        (codes && (misaligned(p->d_x_scale, 4) || misaligned(p->d_w_scale, 4))))
        return fail(GNMR_ERR_LAYOUT, "products: an operand not aligned to its element size");
    return GNMR_OK;
}

// A matrix operand, and whether (and how large) a copy of it has to be made.
struct Operand {
    const void *at;
    int64_t rows, cols, stride, group_stride;
    int groups;
    bool codes;
    int64_t held() const { return (cols + 7) / 8 * 8; }
    bool in_place() const
    {
        return !codes && !misaligned(at, 16) && stride % 8 == 0 && (groups == 1 || group_stride % 8 == 0);
    }
    int64_t copy_bytes() const
    {
        return in_place() || rows == 0 ? 0 : (groups * rows * held() * 2 + 255) / 256 * 256;
    }
};

struct Operands {
    Operand a, b;
};

Operands operands(const gnmr_product *p)
{
    const bool codes = p->op == GNMR_PRODUCT_FORWARD_I8;
    const Operand x{p->d_x, p->rows, p->n_in, p->x_stride, 0, 1, codes};
    const Operand dy{p->d_dy, p->rows, p->n_out, p->dy_stride, 0, 1, false};
    const bool shared = p->w_group_stride == 0;          // one weight for all groups
    const Operand w{p->d_w, p->n_out, p->n_in, p->w_stride, p->w_group_stride, shared ? 1 : p->groups, codes};
    if (p->op == GNMR_PRODUCT_WEIGHT_GRAD)
        return {x, dy};
    return {w, p->op == GNMR_PRODUCT_INPUT_GRAD ? dy : x};
}

cudaError_t copy(const Operand &o, uint16_t *to, int sms, cudaStream_t st)
{
    const Copy c{o.at, to, o.rows, o.cols, o.stride, o.group_stride, o.held(), o.groups * o.rows * (o.held() / 8)};
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((c.total + 255) / 256, int64_t(sms) * 8));
    if (o.codes)
        copy_kernel<int8_t><<<grid, 256, 0, st>>>(c);
    else
        copy_kernel<uint16_t><<<grid, 256, 0, st>>>(c);
    return cudaGetLastError();
}

// Tiles of `high` rows by 64 columns of an operand.
bool tile_map(const gnmr_products *h, CUtensorMap *map, const Operand &o, bool bf16, int high)
{
    if (o.rows == 0) {                                   // nothing will be loaded
        memset(map, 0, sizeof(*map));
        return true;
    }
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(o.cols), static_cast<cuuint64_t>(o.rows), static_cast<cuuint64_t>(o.groups)};
    const cuuint64_t row = static_cast<cuuint64_t>(o.stride) * 2;
    const cuuint64_t strides[2] = {row, o.groups > 1 ? static_cast<cuuint64_t>(o.group_stride) * 2 : row};
    const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(high), 1}, one[3] = {1, 1, 1};
    const auto encode = [&] {
        return h->encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                         const_cast<void *>(o.at), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = encode();
    if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
        cudaSetDevice(h->device);                        // a host thread's first CUDA call: it has no context yet
        r = encode();
    }
    return r == CUDA_SUCCESS;
}

template <int kColumns> constexpr int shared_bytes()
{
    return Shape<kColumns>::kStages * Shape<kColumns>::kStage + static_cast<int>(sizeof(Tables)) + 1024;
}

template <int kColumns, bool kCodes>
cudaError_t launch(const gnmr_products *h, const Operands &o, const Product &p, cudaStream_t st, bool *mapped)
{
    CUtensorMap a, b;
    *mapped = tile_map(h, &a, o.a, p.bf16, p.a_along_lanes ? 64 : 128) &&
              tile_map(h, &b, o.b, p.bf16, p.b_along_columns ? 64 : Shape<kColumns>::kBox);
    if (!*mapped)
        return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * h->pairs);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared_bytes<kColumns>();
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, product_kernel<kColumns, kCodes>, a, b, p);
}

template <int kColumns, bool kCodes> cudaError_t allow_shared()
{
    return cudaFuncSetAttribute(product_kernel<kColumns, kCodes>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                shared_bytes<kColumns>());
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
    int prev = 0, sms = 2;
    cudaGetDevice(&prev);
    cudaSetDevice(device);
    h->device = device;
    const size_t parts = size_t(kMaxParts) * kPartFloats * 4, tickets = size_t(kMaxParts) * 2 * 4;
    cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    h->pairs = std::min(std::max(sms / 2, 1), kMaxPairs);
    if (e == cudaSuccess)
        e = cudaMalloc(&h->dmem, parts + tickets);
    if (e == cudaSuccess) {
        h->parts = static_cast<float *>(h->dmem);
        h->tickets = reinterpret_cast<unsigned *>(static_cast<char *>(h->dmem) + parts);
        e = cudaMemset(h->tickets, 0, tickets);
    }
    if (e == cudaSuccess)
        e = cudaStreamSynchronize(nullptr);              // the tickets are in place whatever stream reads them
    if (e == cudaSuccess)
        e = cudaHostAlloc(reinterpret_cast<void **>(&h->gave_up), sizeof(int), cudaHostAllocMapped | cudaHostAllocPortable);
    if (e == cudaSuccess)
        *h->gave_up = 0;
    cudaDriverEntryPointQueryResult found;
    void *encode = nullptr;
    if (e == cudaSuccess)
        e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &encode, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !encode))
        e = cudaErrorNotSupported;
    h->encode = reinterpret_cast<decltype(h->encode)>(encode);
    if (e == cudaSuccess)
        e = allow_shared<256, false>();
    if (e == cudaSuccess)
        e = allow_shared<256, true>();
    if (e == cudaSuccess)
        e = allow_shared<64, false>();
    if (e == cudaSuccess)
        e = allow_shared<64, true>();
    cudaSetDevice(prev);
    if (e != cudaSuccess) {
        cudaGetLastError();
        gnmr_products_destroy(h);
        return fail(e == cudaErrorMemoryAllocation ? GNMR_ERR_OOM : GNMR_ERR_CUDA, cudaGetErrorString(e));
    }
    *out = h;
    return GNMR_OK;
}

gnmr_status gnmr_products_scratch_bytes(const gnmr_product *p, int64_t *bytes)
{
    if (!bytes)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    *bytes = 0;
    if (const gnmr_status s = check(p))
        return s;
    const Operands o = operands(p);
    *bytes = o.a.copy_bytes() + o.b.copy_bytes();
    return GNMR_OK;
}

gnmr_status gnmr_products_run(gnmr_products *h, const gnmr_product *p, void *stream)
{
    if (!h)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL handle");
    if (const gnmr_status s = check(p))
        return s;
    if (*static_cast<volatile int *>(h->gave_up))
        return fail(GNMR_ERR_STATE, "products: an earlier product gave up waiting inside the GPU");
    const bool codes = p->op == GNMR_PRODUCT_FORWARD_I8, wgrad = p->op == GNMR_PRODUCT_WEIGHT_GRAD;
    if (p->rows == 0 && (!wgrad || p->add))
        return GNMR_OK;
    Operands o = operands(p);
    const int64_t need = o.a.copy_bytes() + o.b.copy_bytes();
    if (need && (!p->d_scratch || p->scratch_bytes < need || misaligned(p->d_scratch, 256)))
        return fail(GNMR_ERR_LAYOUT, "products: operands that cannot be read in place, and no scratch for them");

    Product q = {};
    const bool back = p->op == GNMR_PRODUCT_INPUT_GRAD;
    q.lanes = wgrad || back ? p->n_in : p->n_out;
    q.depth = wgrad ? 0 : back ? p->n_out : p->n_in;
    q.cols = wgrad ? p->n_out : 0;
    q.rows = static_cast<int>(p->rows);
    q.groups = p->groups;
    q.offsets = p->d_offsets;
    q.mask = p->d_mask;
    q.mask_stride = p->mask_stride;
    q.want = codes ? 0 : 1;
    q.a_along_lanes = wgrad || back;
    q.b_along_columns = wgrad;
    q.a_by_group = o.a.groups > 1;
    q.bf16 = !codes && p->dtype == GNMR_DTYPE_BF16;
    q.chunk = !codes && p->out_dtype == GNMR_DTYPE_F32 ? 8 : 16;
    q.out = p->d_out;
    q.out_type = p->out_dtype;
    q.add = wgrad && p->add;
    q.out_col = p->out_stride;
    q.out_group = p->out_group_stride;
    q.pairs_aligned = !misaligned(p->d_out, 4) && p->out_stride % 2 == 0 && (!wgrad || p->groups == 1 || p->out_group_stride % 2 == 0);
    if (codes)
        q.lane_scale = p->d_w_scale, q.col_scale = p->d_x_scale;
    q.parts = h->parts;
    q.tickets = h->tickets;
    q.gave_up = h->gave_up;

    int prev = h->device;
    cudaGetDevice(&prev);
    if (prev != h->device)
        cudaSetDevice(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    char *scratch = static_cast<char *>(p->d_scratch);
    for (Operand *m : {&o.a, &o.b})
        if (const int64_t n = m->copy_bytes(); n && e == cudaSuccess) {
            e = copy(*m, reinterpret_cast<uint16_t *>(scratch), 2 * h->pairs, st);
            *m = Operand{scratch, m->rows, m->cols, m->held(), m->rows * m->held(), m->groups, false};
            scratch += n;
        }
    // few rows to a group: smaller tiles, more of them in flight
    const bool few = !wgrad && p->rows <= 32 * int64_t(p->groups);
    bool mapped = true;
    if (e == cudaSuccess)
        e = codes ? (few ? launch<64, true>(h, o, q, st, &mapped) : launch<256, true>(h, o, q, st, &mapped))
                  : (few ? launch<64, false>(h, o, q, st, &mapped) : launch<256, false>(h, o, q, st, &mapped));
    if (e != cudaSuccess)
        cudaGetLastError();                              // reported here, not by the caller's next call
    if (prev != h->device)
        cudaSetDevice(prev);
    if (!mapped)
        return fail(GNMR_ERR_LAYOUT, "products: the strides of an operand have no tensor map");
    if (e != cudaSuccess)
        return fail(GNMR_ERR_CUDA, cudaGetErrorString(e));
    return GNMR_OK;
}

gnmr_status gnmr_products_destroy(gnmr_products *h)
{
    if (!h)
        return GNMR_OK;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaSetDevice(h->device);
    cudaError_t e = h->dmem ? cudaFree(h->dmem) : cudaSuccess;
    if (h->gave_up) {
        const cudaError_t f = cudaFreeHost(h->gave_up);
        e = e == cudaSuccess ? f : e;
    }
    cudaSetDevice(prev);
    delete h;
    return e == cudaSuccess ? GNMR_OK : GNMR_ERR_CUDA;
}

}  // extern "C"
