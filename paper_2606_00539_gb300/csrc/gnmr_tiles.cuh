// What the kernels of the expert products share: the work of a call as tiles of every
// group, sums that several pairs of CTAs share, and the epilogue.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "gnmr.h"
#include "gnmr_act.cuh"
#include "gnmr_mma.cuh"

namespace gnmr_tiles {

using namespace gnmr_mma;

constexpr int kMaxGroups = 2048;
constexpr int kMaxPairs = 80;
constexpr int kMaxParts = 2 * kMaxPairs;               // split tiles' parts in one call
constexpr int64_t kPartFloats = 256 * 256;             // one part: both CTAs' lanes by the columns
constexpr int kLanes = 256;                            // of a pair's tile
constexpr int kMostEpilogueWarps = 16;
constexpr int kFirstEpilogueWarp = 4;

struct Product {
    int lanes, depth, cols;            // depth, or cols, is 0 where it is a group's rows
    int rows, groups;
    const int64_t *offsets;
    const uint8_t *mask;
    int64_t mask_stride;
    int want;                          // groups computed: mask byte != 0 (1), == 0 (0)
    unsigned lane_tiles_inverse;       // ceil(2^32 / tiles of 256 lanes)
    int a_by_group;                    // A's tiles are those of the group
    int a_blocks, b_blocks;            // two blocks of 64 lanes or columns in one load
    int granule;                       // a tile's columns are multiples of it: 32 or 128
    int bf16;
    int piece;                         // contraction steps of a piece
    int ring;                          // stages of operands in shared memory
    void *out;
    int out_type;
    int pairs_aligned;                 // two outputs of a row may be stored as one
    int add;
    int64_t out_col, out_group;
    const float *lane_scale, *col_scale;
    int act;                           // gated: lanes are the two projections' in turn
    void *keep;
    int64_t keep_col;
    int keep_aligned;
    float *parts;
    unsigned *tickets;
    int *gave_up;
    uint64_t most_ns;                  // of every wait; 0: nothing is loaded, so that they run out
};

// ---- work: tiles of every group, and their parts --------------------------------

// In shared memory, [groups + 1] each, after the barriers.
struct Tables {
    int *first;                        // tiles before group g; in the end all of them
    int *row;                          // first row of group g; in the end the last group's end
    uint16_t *each;                    // columns of group g's tiles; in the end the parts of every tile's contraction
};

__host__ __device__ constexpr int table_bytes(int groups) { return (groups + 1) * (4 + 4 + 2); }

struct Item {
    int g, lane0, col0, cols;          // the tile: the pair's lanes, and its columns
    int wide;                          // the columns multiplied, half of them from each CTA's B
    int row0;                          // the group's first row
    int depth, k0, k1;                 // the whole contraction; the stages of this part
    int tile, part;
    bool tail;                         // the last stage holds rows past the group's end
};

__device__ __forceinline__ int parts_of(int n, int each) { return (n + each - 1) / each; }

// Filled by one warp; kStep: contraction steps of a stage; kJoin: stages that reading one
// part of a tile back takes as long as.  Offsets are clamped to [0, rows] and made not decreasing.
template <int kStep, int kJoin>
__device__ __forceinline__ void fill_tables(const Product &p, const Tables &t, int most, int lane_tiles, int pairs)
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
    // One group, all tiles alike: narrower ones where they make the last round fuller.
    // 4096^3: 256 tiles of 256 columns are 4 rounds of 76 pairs, as are 304 of 224 (80 and 76 us).
    // A tile costs its columns and about 128 more; of many groups' tiles, of many widths, the choice
    // gained nothing.
    int width = most;
    if (p.groups == 1 && most > 128) {
        const int cols = p.cols ? p.cols : t.row[1] - t.row[0];
        int64_t least = INT64_MAX;
        for (int m = most; m > most / 2; m -= p.granule) {
            const int64_t rounds = (int64_t(lane_tiles) * parts_of(cols, m) + pairs - 1) / pairs;
            if (rounds * (m + 128) < least)
                least = rounds * (m + 128), width = m;
        }
    }
    int tiles = 0, deepest = 0;
    for (int g0 = 0; g0 < p.groups; g0 += 32) {
        const int g = g0 + lane;
        int n = 0;
        if (g < p.groups && (!p.mask || (p.mask[g * p.mask_stride] != 0) == (p.want != 0))) {
            const int rows = t.row[g + 1] - t.row[g];
            const int cols = p.cols ? p.cols : rows, across = parts_of(cols, width);
            n = lane_tiles * across;
            // a group's columns are shared out evenly, in multiples of the granule
            t.each[g] = static_cast<uint16_t>(across ? parts_of(parts_of(cols, across), p.granule) * p.granule : 0);
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
    // Few tiles: the number of parts that takes the fewest stages, those included that
    // beginning parts (six) and reading them back (kJoin each) take as long as.  With reading
    // left out, 50,000 rows into a gradient of 136 x 200 took 32 parts and 70 us.
    int best = 1;
    if (tiles > 0 && tiles < pairs) {
        const int stages = parts_of(__reduce_max_sync(~0u, deepest), kStep), parts = lane + 1;
        const bool fits = parts == 1 || (tiles * parts <= min(2 * pairs, kMaxParts) && 2 * parts <= stages);
        const int cost = fits ? parts_of(tiles * parts, pairs) * parts_of(stages, parts) + (parts > 1 ? 6 + kJoin * parts : 0) : INT32_MAX;
        const int least = __reduce_min_sync(~0u, cost);
        best = __ffs(__ballot_sync(~0u, cost == least));
    }
    if (lane == 0) {
        t.first[p.groups] = tiles;
        t.each[p.groups] = static_cast<uint16_t>(best);
    }
}

// Item i of the call, by a whole warp that comes with growing i.  g: the group of the one
// before, 0 at first.
template <int kStep>
__device__ __forceinline__ Item item_of(const Product &p, const Tables &t, int split, int lane_tiles, int i, int &g)
{
    Item it;
    it.tile = split == 1 ? i : i / split;
    it.part = i - it.tile * split;
    for (;;) {                                       // the last group that begins at or before the tile
        const int next = g + 1 + (threadIdx.x & 31);
        const unsigned past = __ballot_sync(~0u, next >= p.groups || t.first[next] > it.tile);
        if (past) {
            g += __ffs(past) - 1;
            break;
        }
        g += 32;
    }
    it.g = g;
    it.row0 = t.row[g];
    const int rows = t.row[g + 1] - it.row0, at = it.tile - t.first[g], each = t.each[g];
    int c = at;                                      // at / lane_tiles
    if (lane_tiles > 1) {
        c = __umulhi(at, p.lane_tiles_inverse);      // that, or one more
        c -= c * lane_tiles > at;
    }
    it.lane0 = (at - c * lane_tiles) * kLanes;
    it.col0 = c * each;
    it.cols = min(each, (p.cols ? p.cols : rows) - it.col0);
    it.wide = (it.cols + p.granule - 1) & -p.granule;
    it.depth = p.depth ? p.depth : rows;
    const int stages = parts_of(it.depth, kStep);
    it.k0 = 0;
    it.k1 = stages;
    if (split > 1) {
        it.k0 = stages * it.part / split;
        it.k1 = stages * (it.part + 1) / split;
    }
    it.tail = !p.depth && it.depth % kStep && it.k0 < it.k1 && it.k1 == stages;
    return it;
}

// ---- a CTA ------------------------------------------------------------------------

constexpr int kMostStages = 11;

struct Barriers {
    uint64_t full[kMostStages], empty[kMostStages];      // stages of operands
    uint64_t tail[kMostStages];        // a stage that the tail warp looks at first
    uint64_t ready[4], used[4];        // operands widened from 8 bits
    uint64_t done[2], drained[2];      // halves of tensor memory; in a pair `drained` counts in the first CTA
    uint32_t tmem;
};

// What the roles of a CTA share.
struct Cta {
    uint8_t *stages;                   // operands, in dynamic shared memory
    int ring;                          // how many stages there are
    Barriers *bars;
    Tables tables;
    uint32_t rank, tmem;
    int pair, pairs, lane_tiles, items, split;
};

// Dynamic shared memory: `bytes` of operands, whole kilobytes, then barriers and tables.
// None is static, so that it begins at a multiple of 1,024, as swizzled tiles have to.
__device__ __forceinline__ Cta cta_of(const Product &p, uint8_t *shared, int bytes)
{
    Cta c;
    c.stages = shared;
    c.ring = p.ring;
    c.bars = reinterpret_cast<Barriers *>(shared + bytes);
    c.tables.first = reinterpret_cast<int *>(c.bars + 1);
    c.tables.row = c.tables.first + p.groups + 1;
    c.tables.each = reinterpret_cast<uint16_t *>(c.tables.row + p.groups + 1);
    c.rank = cta_rank();
    c.pair = blockIdx.x >> 1;
    c.pairs = gridDim.x >> 1;
    c.lane_tiles = parts_of(p.lanes, kLanes);
    return c;
}

// As many stages as fit beside `more` bytes of operands, barriers and tables.
constexpr int kSharedMost = 227 << 10;

constexpr int ring_of(int groups, int stage, int more)
{
    const int n = (kSharedMost - more - static_cast<int>(sizeof(Barriers)) - table_bytes(groups)) / stage;
    return n < kMostStages ? n : kMostStages;
}

constexpr int shared_bytes(int groups, int stage, int more)
{
    return ring_of(groups, stage, more) * stage + more + static_cast<int>(sizeof(Barriers)) + table_bytes(groups);
}

// ---- outputs --------------------------------------------------------------------

template <int kOut> __device__ __forceinline__ unsigned pack(float lo, float hi)
{
    if (kOut == GNMR_DTYPE_BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return reinterpret_cast<const unsigned &>(v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const unsigned &>(v);
}

template <int kOut> __device__ __forceinline__ float load_out(const char *at)
{
    return kOut == GNMR_DTYPE_F32    ? *reinterpret_cast<const float *>(at)
           : kOut == GNMR_DTYPE_BF16 ? __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(at))
                                     : __half2float(*reinterpret_cast<const __half *>(at));
}

// Two columns of this thread's lane become one column of two lanes: the even lane gets
// the first column's, the odd lane the second's.
template <int kOut> __device__ __forceinline__ unsigned exchange(float first, float second, unsigned which)
{
    const unsigned w = pack<kOut>(first, second);
    return __byte_perm(w, __shfl_xor_sync(~0u, w, 1), which);
}

// The outputs that a tile will be added to, to L2 while it is multiplied: read as they are
// needed, 16 at a time, they took longer than the multiplies.
__device__ __forceinline__ void fetch_outputs(const Product &p, const Cta &c, const Item &it, int warp, int warps)
{
    const int bytes = p.out_type == GNMR_DTYPE_F32 ? 4 : 2, lines = 128 * bytes / 128;     // of a column, a CTA's lanes
    const int lane = threadIdx.x & 31, first = it.lane0 + c.rank * 128;
    const int64_t row = p.cols ? it.col0 : int64_t(it.row0) + it.col0;
    const char *out = static_cast<const char *>(p.out) + ((p.cols ? it.g * p.out_group : 0) + row * p.out_col + first) * bytes;
    for (int i = warp * 32 + lane; i < it.cols * lines; i += warps * 32) {
        const int col = i / lines, line = i - col * lines;
        if (first + line * (128 / bytes) < p.lanes)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(out + col * p.out_col * bytes + line * 128));
    }
}

// This warp's sums to the outputs: lane `lane` of columns col .. col + span - 1 of the
// tile.  Two lanes' 16-bit values of a column go out as one where they can: 64
// contiguous bytes a column from a warp.
template <int kPieces, bool kCodes, int kOut>
__device__ __forceinline__ void finish(const Product &p, const Item &it, uint32_t (&acc)[kPieces][16], int lane, int col, int span)
{
    constexpr int kBytes = kOut == GNMR_DTYPE_F32 ? 4 : 2;
    const int64_t step = p.out_col * kBytes;
    const int64_t row = p.cols ? it.col0 + col : int64_t(it.row0) + it.col0 + col;
    char *out = static_cast<char *>(p.out) + (p.cols ? it.g * p.out_group * kBytes : 0) + row * step + int64_t(lane) * kBytes;
    const int left = it.cols - col, odd = lane & 1;
    const bool mine = lane < p.lanes;
    // every lane there, and 16 columns' offsets that one multiplication each gives (a chain of
    // additions held up stores)
    const bool whole = (lane | 31) < p.lanes && (kBytes == 4 || (p.pairs_aligned && !p.add)) && step < (int64_t(1) << 28);
    const unsigned near = static_cast<unsigned>(step);
    const unsigned which = odd ? 0x3276 : 0x5410;
    float by_lane = 0.0f;
    const float *by_col = nullptr;
    if (kCodes) {
        by_lane = mine ? p.lane_scale[int64_t(it.g) * p.lanes + lane] : 0.0f;
        by_col = p.col_scale + it.row0 + it.col0 + col;
    }
    if (whole && kBytes == 2)
        out += odd ? step - 2 : 0;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
        const int n = min(span, left) - q * 16;          // columns of this piece that there are
        if (n <= 0)
            break;
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j)
            v[j] = kCodes ? (j < n ? by_col[q * 16 + j] : 0.0f) : __uint_as_float(acc[q][j]);
        if (kCodes)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                v[j] = static_cast<float>(static_cast<int>(acc[q][j])) * v[j] * by_lane;
        if (whole && n >= 16) {
            if (kBytes == 4) {
                if (p.add) {
                    float old[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        old[j] = *reinterpret_cast<const float *>(out + j * near);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        v[j] += old[j];
                }
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    *reinterpret_cast<float *>(out + j * near) = v[j];
            } else {
#pragma unroll
                for (int h = 0; h < 16; h += 8) {
                    unsigned w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        w[j] = exchange<kOut>(v[h + 2 * j], v[h + 2 * j + 1], which);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<unsigned *>(out + (h + 2 * j) * near) = w[j];
                }
            }
            out += 16 * step;
            continue;
        }
        if (whole && kBytes == 2)                        // back to this lane's own place in the first column
            out -= odd ? step - 2 : 0;
        if (p.add)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (mine && j < n)
                    v[j] += load_out<kOut>(out + j * step);
        if (kBytes == 4) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (mine && j < n)
                    *reinterpret_cast<float *>(out + j * step) = v[j];
        } else {
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
                const unsigned w = exchange<kOut>(v[j], v[j + 1], which);
                char *to = out - 2 * odd + (j + odd) * step;     // the column that this thread writes, two lanes of it
                if (j + odd < n) {
                    if (p.pairs_aligned && (lane | 1) < p.lanes) {
                        *reinterpret_cast<unsigned *>(to) = w;
                    } else {
                        if ((lane & ~1) < p.lanes)
                            *reinterpret_cast<uint16_t *>(to) = static_cast<uint16_t>(w);
                        if ((lane | 1) < p.lanes)
                            *reinterpret_cast<uint16_t *>(to + 2) = static_cast<uint16_t>(w >> 16);
                    }
                }
            }
        }
        out += 16 * step;
    }
}

// The same for a gated block: lanes 2 i and 2 i + 1 are output i's two projections.  Two
// columns of a lane pair are exchanged, so that the even lane forms the first column's h and the odd
// lane the second's; then two lane pairs exchange h's of four columns, so that each thread stores
// two outputs of one column.  A warp's outputs of a column are 32 contiguous bytes: whole sectors, which L2 puts together.
// h costs an exchange and an activation (two special-function operations) for each of 64 sums a thread, hidden
// behind the next tile's multiplies: 49,152 rows of 64 x 1408 x 2048 take 347 us in a burst of 20 (1.6 PFLOP/s) where the plain product of
// both projections takes 345 to 385, and 393 over seconds, at the power limit; the projections kept as well, 277 MB more, 366 and
// 416.  With a predicate at every store they took 438.
template <int kPieces, int kType, int kAct>
__device__ __forceinline__ void finish_gated(const Product &p, const Item &it, uint32_t (&acc)[kPieces][16], int lane, int col, int span)
{
    const int odd = lane & 1, second = (lane >> 1) & 1, half = p.lanes >> 1;
    const int first = (lane >> 1) & ~1;                  // the first of the two outputs that this lane stores
    const int64_t row = int64_t(it.row0) + it.col0 + col, out_step = p.out_col * 2, keep_step = p.keep_col * 2;
    char *out = static_cast<char *>(p.out) + row * out_step + int64_t(first) * 2;
    char *keep = static_cast<char *>(p.keep) + row * keep_step + int64_t((odd ? half : 0) + first) * 2;
    const int left = it.cols - col;
    const int there = min(half - first, 2);              // of the two outputs: 0 or less, 1, 2
    const unsigned which = second ? 0x3276 : 0x5410;
    // both outputs of every lane there, stored as one, 16 columns' offsets within 32 bits
    const bool whole = (lane | 31) < p.lanes && p.pairs_aligned && (!p.keep || p.keep_aligned) && (out_step | keep_step) < (int64_t(1) << 27);
    const unsigned out_near = static_cast<unsigned>(out_step), keep_near = static_cast<unsigned>(keep_step);
    const auto store = [&](char *to, unsigned two) {
        if (there == 2 && (reinterpret_cast<uintptr_t>(to) & 3) == 0) {
            *reinterpret_cast<unsigned *>(to) = two;
        } else {
            if (there > 0)
                *reinterpret_cast<uint16_t *>(to) = static_cast<uint16_t>(two);
            if (there > 1)
                *reinterpret_cast<uint16_t *>(to + 2) = static_cast<uint16_t>(two >> 16);
        }
    };
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
        const int n = min(span, left) - q * 16;          // columns of this piece that there are
        if (n <= 0)
            break;
        if (p.keep) {
            unsigned two[8];                             // of columns 2 j + second
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const unsigned w = pack<kType>(__uint_as_float(acc[q][2 * j]), __uint_as_float(acc[q][2 * j + 1]));
                two[j] = __byte_perm(w, __shfl_xor_sync(~0u, w, 2), which);
            }
            if (whole && n >= 16) {
                char *const to = keep + second * keep_step;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<unsigned *>(to + 2 * j * keep_near) = two[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (2 * j + second < n)
                        store(keep + (2 * j + second) * keep_step, two[j]);
            }
            keep += 16 * keep_step;
        }
        float h[8];                                      // of columns 2 i + odd
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float mine = __uint_as_float(odd ? acc[q][2 * i + 1] : acc[q][2 * i]);
            const float other = __shfl_xor_sync(~0u, __uint_as_float(odd ? acc[q][2 * i] : acc[q][2 * i + 1]), 1);
            h[i] = gnmr_act::activated<kAct>(odd ? other : mine) * (odd ? mine : other);
        }
        unsigned two[4];                                 // of columns 4 i + 2 second + odd
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned w = pack<kType>(h[2 * i], h[2 * i + 1]);
            two[i] = __byte_perm(w, __shfl_xor_sync(~0u, w, 2), which);
        }
        if (whole && n >= 16) {
            char *const to = out + (2 * second + odd) * out_step;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<unsigned *>(to + 4 * i * out_near) = two[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (4 * i + 2 * second + odd < n)
                    store(out + (4 * i + 2 * second + odd) * out_step, two[i]);
        }
        out += 16 * out_step;
    }
}

// The first piece's sums, or another's added to them.
template <bool kCodes>
__device__ __forceinline__ void begin_sum(uint32_t (&acc)[16])
{
    if (kCodes)
#pragma unroll
        for (int j = 0; j < 16; ++j)
            acc[j] = __float2int_rn(__uint_as_float(acc[j]));
}

template <bool kCodes>
__device__ __forceinline__ void add_to_sum(uint32_t (&acc)[16], const uint32_t (&v)[16])
{
#pragma unroll
    for (int j = 0; j < 16; ++j)
        acc[j] = kCodes ? acc[j] + __float2int_rn(__uint_as_float(v[j]))
                        : __float_as_uint(__uint_as_float(acc[j]) + __uint_as_float(v[j]));
}

// The barriers that the epilogue counts on, of `warps` warps a CTA.
template <int kCtas>
__device__ __forceinline__ void init_epilogue_barriers(Barriers &b, int warps)
{
    for (int h = 0; h < 2; ++h) {
        barrier_init(smem_addr(&b.done[h]), 1);
        barrier_init(smem_addr(&b.drained[h]), kCtas * warps);
    }
}

// The beginning of every kernel, after the barriers' initialisation: the other CTA's
// are initialised too by the time that join_pair returns.
__device__ __forceinline__ void greet_pair()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}

__device__ __forceinline__ void join_pair()
{
    fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    fence_after();
}

// The end of every kernel: both CTAs of a pair are through, and one with a role that gave up
// says so, and stays until the loads and multiplies that it left behind, microseconds' work, are over.
__device__ __forceinline__ void finish_pair(bool fine, int *gave_up)
{
    fence_before();
    if (__syncthreads_or(!fine)) {
        if (threadIdx.x == 0)
            *gave_up = 1;
        for (const uint64_t since = nanoseconds(); nanoseconds() - since < 1000000;)
            __nanosleep(1000);
    }
    cluster_sync();
    fence_after();
}

// A split tile: this warp's lanes and columns of this part go to memory, and the warp that
// gets here last takes the sum of all parts, in their order.  Warps do not wait for one
// another: whether this one has the sum.
template <int kPieces, bool kCodes>
__device__ __forceinline__ bool join_parts(const Product &p, const Cta &c, const Item &it, uint32_t (&acc)[kPieces][16],
                                           int cols, int col, int warp)
{
    const int lane = threadIdx.x & 31, split = c.split;
    uint32_t *part = reinterpret_cast<uint32_t *>(p.parts) + int64_t(it.tile) * split * kPartFloats +
                     c.rank * (kPartFloats / 2) + (warp & 3) * 32 + lane;
#pragma unroll
    for (int q = 0; q < kPieces; ++q)
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (q * 16 + j < cols)
                part[it.part * kPartFloats + (col + q * 16 + j) * 128] = acc[q][j];
    __threadfence();
    __syncwarp();
    unsigned before = 0;
    if (lane == 0) {
        unsigned *ticket = p.tickets + (2 * it.tile + c.rank) * kMostEpilogueWarps + warp - kFirstEpilogueWarp;
        before = atomicAdd(ticket, 1u);
        if (before + 1 == static_cast<unsigned>(split))
            *ticket = 0;                                 // for the next call
        __threadfence();
    }
    __syncwarp();                                        // the other lanes' loads come after that fence (a shuffle orders none)
    if (__shfl_sync(~0u, before, 0) + 1 != static_cast<unsigned>(split))
        return false;
#pragma unroll
    for (int q = 0; q < kPieces; ++q)
        if (q * 16 < cols) {
#pragma unroll 2
            for (int s = 0; s < split; ++s)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t v = q * 16 + j < cols ? __ldcg(part + s * kPartFloats + (col + q * 16 + j) * 128) : 0;
                    if (s == 0)
                        acc[q][j] = v;
                    else
                        acc[q][j] = kCodes ? acc[q][j] + v : __float_as_uint(__uint_as_float(acc[q][j]) + __uint_as_float(v));
                }
        }
    return true;
}

// The epilogue's warps, four (one to 32 lanes) for each of kSides shares of a tile's columns: its
// pieces added up and written.  kCtas: those that multiply as one.
template <int kColumns, int kSides, bool kCodes, int kStep, int kCtas, bool kGated = false>
__device__ __forceinline__ bool write_outputs(const Product &p, const Cta &c)
{
    constexpr int kPieces = kColumns / 16 / kSides;      // of 16 columns
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int quarter = warp & 3, side = (warp - kFirstEpilogueWarp) >> 2;
    const uint32_t done = smem_addr(&c.bars->done[0]), drained = in_cta(smem_addr(&c.bars->drained[0]), kCtas == 2 ? 0 : c.rank);
    int half = 0;
    uint32_t phase = 0;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const int span = parts_of(it.wide, 16 * kSides) * 16;               // columns of this warp, or fewer
        const int at = it.lane0 + c.rank * 128 + quarter * 32 + lane, col = side * span;
        if (p.add)
            fetch_outputs(p, c, it, warp - kFirstEpilogueWarp, 4 * kSides);
        uint32_t acc[kPieces][16];
        if (it.k0 == it.k1)
#pragma unroll
            for (int q = 0; q < kPieces; ++q)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    acc[q][j] = 0;
        for (int k = it.k0; k < it.k1; k += p.piece / kStep) {
            if (!wait<kCtas == 2>(done + half * 8, phase, p.most_ns))
                return false;
            fence_after();
            const uint32_t from = c.tmem + half * kColumns + (uint32_t(quarter * 32) << 16) + col;
            if (k == it.k0) {
#pragma unroll
                for (int q = 0; q < kPieces; ++q)
                    if (q * 16 < span)
                        load16(from + q * 16, acc[q]);
#pragma unroll
                for (int q = 0; q < kPieces; ++q) {
                    load_wait(acc[q]);
                    begin_sum<kCodes>(acc[q]);
                }
            } else {
#pragma unroll
                for (int q = 0; q < kPieces; ++q)
                    if (q * 16 < span) {
                        uint32_t v[16];
                        load16(from + q * 16, v);
                        load_wait(v);
                        add_to_sum<kCodes>(acc[q], v);
                    }
            }
            fence_before();
            __syncwarp();
            if (lane == 0)
                arrive(drained + half * 8);
            if (half ^= 1; half == 0)
                phase ^= 1;
        }
        if (c.split > 1 && !join_parts<kPieces, kCodes>(p, c, it, acc, min(span, it.cols - col), col, warp))
            continue;
        if (p.add && it.depth == 0)
            continue;                                    // nothing to add
        if (kGated) {
            if (p.bf16 && p.act == GNMR_ACT_SILU)
                finish_gated<kPieces, GNMR_DTYPE_BF16, GNMR_ACT_SILU>(p, it, acc, at, col, span);
            else if (p.bf16)
                finish_gated<kPieces, GNMR_DTYPE_BF16, GNMR_ACT_GELU>(p, it, acc, at, col, span);
            else if (p.act == GNMR_ACT_SILU)
                finish_gated<kPieces, GNMR_DTYPE_F16, GNMR_ACT_SILU>(p, it, acc, at, col, span);
            else
                finish_gated<kPieces, GNMR_DTYPE_F16, GNMR_ACT_GELU>(p, it, acc, at, col, span);
        } else if (p.out_type == GNMR_DTYPE_F32)
            finish<kPieces, kCodes, GNMR_DTYPE_F32>(p, it, acc, at, col, span);
        else if (p.out_type == GNMR_DTYPE_BF16)
            finish<kPieces, kCodes, GNMR_DTYPE_BF16>(p, it, acc, at, col, span);
        else
            finish<kPieces, kCodes, GNMR_DTYPE_F16>(p, it, acc, at, col, span);
    }
    return true;
}

}  // namespace gnmr_tiles
