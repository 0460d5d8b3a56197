// Expert products: the linear units of both paths, grouped by expert.  The 16-bit kernel
// and the calls; 8-bit codes have a file of their own.
//
// Every product is out[col][lane] = sum over c of A[lane][c] B[col][c]:
//   forward      A = W_g      [n_out lanes], c along its rows     B = x's rows    c < n_in
//   input grad   A = W_g^T    [n_in lanes], lanes along its rows  B = dy's rows   c < n_out
//   weight grad  A = x^T      [n_in lanes], lanes along its rows  B = dy^T        c < the group's rows
//   gated block  A = W_g's two halves, row by row in turn         B = x's rows    c < n_in
// so that the tensor cores' 128 lanes lie along the output's contiguous axis and a
// group's ragged rows are columns, of which a tile has any multiple of 32 up to 256.
// A gated block's two projections of one output are neighbouring lanes: its tiles of A are one load
// of a tensor map with a dimension for the halves of W_g before that for their rows.  So the epilogue has both in
// one warp, and the loop of loads and multiplies is the plain product's.
//
// A pair of CTAs computes 256 lanes by up to 256 columns (two SMs share an operand
// tile: 32 KB of operands an SM for 64 steps of the contraction, where one SM alone
// would need 48).  Per CTA: one warp has the TMA unit load tiles of 64 steps into a
// ring of stages, one (of the first CTA) issues the multiplies, eight or sixteen add up
// the finished pieces and write the outputs, and one clears what the last tile of a
// group's rows holds past their end (weight gradient).
//
// Measured (one GB300, 64 experts of 1408 x 2048, bf16): forward of 49,152 rows 190 to 200 us, 1.4 to 1.5 PFLOP/s,
// multiplies under way 79 % of the time at the 1.6 GHz that the power limit leaves; input gradient
// of 24,571 rows 102 us, weight gradient 123 us (bound by its outputs); forward of 282 rows 59 us, 6.3
// TB/s of weights.  Dense 4096^3 74 us, 1.85 PFLOP/s.
//
// A piece is at most 1,024 steps (512 for fp32 outputs).  The tensor cores cut
// sums that they hold rather than rounding them: 2,047 steps in one piece were
// 1.5e-6 of the result off, in fp32 arithmetic 3.9e-7.  Pieces are added in registers,
// rounded, while the next one is multiplied into the other half of tensor memory.
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
#include "gnmr_products.h"
#include "gnmr_tiles.cuh"

namespace {

using namespace gnmr_tiles;
using gnmr::Operand;
using gnmr::Operands;

constexpr int kGated = 4;                              // an op of this file: two projections, the activation, the product
constexpr int kStep = 64;                              // contraction steps of a stage: 128-byte rows of 16 bits
constexpr int kProducerWarp = 0, kMultiplyWarp = 1, kTailWarp = 2, kTablesWarp = 3;
constexpr int kAStage = 128 * 128;                     // bytes of A's tile in one CTA
constexpr int kBlock = 64 * 128;                       // bytes of a tile of 64 lanes or columns lying along rows

// The epilogue's warps and the registers that the warpgroups share out between them, out of what the
// block is launched with.  A weight gradient's contraction is short, so that it is bound by its
// epilogue: 16 warps of 64 columns each (12288 rows, 64 fp32 gradients of 1408 x 2048: 8 warps 156 us,
// 16 141).  So is a gated block of a short contraction, whose warps read two sums, take an exponential
// and store three numbers for each output (49152 rows, 64 x 1408 features, the projections kept: of 256 steps
// 189 us with 8 warps and 152 with 16, of 1024 235 and 217, of 2048, at the power limit, 355 to 413 and 356 to
// 403; 12000 rows, 24 x 1003, of 2048 steps 107 and 89; 3000 rows, 8 x 2048, of 4096 72 and 73.5).  The others have
// 8 warps of 128, with which 16 made no difference.  The 16 warps' 104 registers do not hold the 64 sums beside
// what addresses them: about 300 bytes a thread of a weight gradient are spilled, about 110 of a gated block.
template <int kOp> struct Roles {
    static constexpr int kSides = kOp == GNMR_PRODUCT_WEIGHT_GRAD || kOp == kGated ? 4 : 2;
    static constexpr int kThreads = 32 * (kFirstEpilogueWarp + 4 * kSides);
    static constexpr int kLaunchRegisters = kSides == 4 ? 96 : 168;
    static constexpr int kControlRegisters = kSides == 4 ? 64 : 72, kEpilogueRegisters = kSides == 4 ? 104 : 216;
    static_assert(128 * kControlRegisters + 128 * kSides * kEpilogueRegisters <= kThreads * kLaunchRegisters &&
                      kThreads * kLaunchRegisters <= 65536, "registers of the launch");
};

// kColumns columns at most; a CTA loads half of B's tile, as kBox rows in one load whatever
// there are (each load costs its issuing thread about 100 of the 512 cycles that a stage's
// multiplies take: with two for B, 8192^3 took 621 us).
template <int kColumns> struct Shape {
    static constexpr int kBox = kColumns / 2;
    static constexpr int kStage = kAStage + kBox * 128;
    static constexpr int kTmem = 2 * kColumns;
    static constexpr int kJoin = kColumns / 64;
};

// The stage with the tail is loaded first and multiplied fourth (or last): clearing it
// takes as long as multiplying a few others.  kTailTurn + 2 stages at least are in
// the ring, so that it is never waited for by a stage that waits for its place.
constexpr int kTailTurn = 3;

// ---- the kernel -------------------------------------------------------------------

// The contraction is a group's rows; lanes, or columns, lie along an operand's rows.
__host__ __device__ constexpr bool rows_deep(int op) { return op == GNMR_PRODUCT_WEIGHT_GRAD; }
__host__ __device__ constexpr bool a_along_lanes(int op)
{
    return op == GNMR_PRODUCT_WEIGHT_GRAD || op == GNMR_PRODUCT_INPUT_GRAD;
}
__host__ __device__ constexpr bool b_along_columns(int op) { return op == GNMR_PRODUCT_WEIGHT_GRAD; }

// The roles below are loops of whole warps, of which one lane issues: values that
// the compiler knows to be the same in all lanes stay in uniform registers, which
// these instructions take their operands from.

template <int kColumns, int kOp>
__device__ __forceinline__ bool load_stages(const CUtensorMap &map_a, const CUtensorMap &map_b, const Product &p, const Cta &c)
{
    using S = Shape<kColumns>;
    const uint32_t full = in_cta(smem_addr(&c.bars->full[0]), 0), empty = smem_addr(&c.bars->empty[0]);
    const uint32_t tail = smem_addr(&c.bars->tail[0]), base = smem_addr(c.stages);
    int stage = 0;
    uint32_t phase = 1;
    if (p.most_ns == 0)
        return false;                                    // no time at all: the others wait in vain
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const int half = it.wide / 2;                         // B's columns in this CTA
        const int a_lane = it.lane0 + c.rank * 128, b_col = it.col0 + c.rank * half + (rows_deep(kOp) ? 0 : it.row0);
        const int za = p.a_by_group ? it.g : 0;
        const bool two = b_along_columns(kOp) && (p.b_blocks || half > 64);        // blocks of B
        const uint32_t bytes = kAStage + (!b_along_columns(kOp) ? S::kBox * 128 : two ? 2 * kBlock : kBlock);
        for (int k = it.k0; k < it.k1; ++k) {
            if (!wait<true>(empty + stage * 8, phase, p.most_ns))
                return false;
            if (elected()) {
                int at = k * kStep;
                bool first_tail = false;
                if (rows_deep(kOp)) {
                    first_tail = it.tail && k == it.k0;
                    at = it.row0 + (!it.tail ? k : first_tail ? it.k1 - 1 : k - 1) * kStep;
                }
                const uint32_t bar = first_tail ? tail + stage * 8 : full + stage * 8;
                const uint32_t a = base + stage * S::kStage, b = a + kAStage;
                arrive_expect(first_tail ? in_cta(bar, c.rank) : bar, bytes);
                if (kOp == kGated) {
                    load_tile<2>(a, &map_a, at, 0, a_lane >> 1, za, bar);
                } else if (!a_along_lanes(kOp)) {
                    load_tile<2>(a, &map_a, at, a_lane, 0, za, bar);
                } else if (p.a_blocks) {
                    load_tile<2>(a, &map_a, 0, at, a_lane >> 6, za, bar);
                } else {
                    load_tile<2>(a, &map_a, a_lane, at, 0, za, bar);
                    load_tile<2>(a + kBlock, &map_a, a_lane + 64, at, 0, za, bar);
                }
                if (!b_along_columns(kOp)) {
                    load_tile<2>(b, &map_b, at, b_col, 0, 0, bar);
                } else if (p.b_blocks) {
                    load_tile<2>(b, &map_b, 0, at, b_col >> 6, 0, bar);
                } else {
                    load_tile<2>(b, &map_b, b_col, at, 0, 0, bar);
                    if (two)
                        load_tile<2>(b + kBlock, &map_b, b_col + 64, at, 0, 0, bar);
                }
            }
            __syncwarp();
            if (++stage == c.ring)
                stage = 0, phase ^= 1;
        }
    }
    return true;
}

template <int kColumns, int kOp>
__device__ __forceinline__ bool multiply_stages(const Product &p, const Cta &c)
{
    using S = Shape<kColumns>;
    constexpr uint32_t kALead = a_along_lanes(kOp) ? kBlock : 16, kANext = (a_along_lanes(kOp) ? 16 * 128 : 32) >> 4;
    constexpr uint32_t kBLead = b_along_columns(kOp) ? kBlock : 16, kBNext = (b_along_columns(kOp) ? 16 * 128 : 32) >> 4;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = smem_addr(&c.bars->empty[0]);
    const uint32_t done = smem_addr(&c.bars->done[0]), drained = smem_addr(&c.bars->drained[0]);
    const uint64_t first_a = operand(smem_addr(c.stages), kALead, 1024);
    const uint64_t first_b = operand(smem_addr(c.stages) + kAStage, kBLead, 1024);
    int stage = 0, half = 0;
    uint32_t phase = 0, free_phase = 1;                  // free_phase: of both halves, while half is 0
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const uint32_t idesc = shape<2>(p.bf16, a_along_lanes(kOp), b_along_columns(kOp), it.wide);
        const int count = it.k1 - it.k0, turn = it.tail ? min(kTailTurn, count - 1) : -1;
        const int first = stage;
        const uint32_t first_phase = phase;
        for (int k = 0; k < count;) {
            if (!wait<true>(drained + half * 8, free_phase, p.most_ns))
                return false;
            fence_after();
            const int stop = min(count, k + p.piece / kStep);
            const uint32_t sums = c.tmem + half * kColumns;
            for (bool add = false; k < stop; ++k, add = true) {
                int at = stage, left = it.depth - (it.k0 + k) * kStep;
                uint32_t its = phase;
                if (rows_deep(kOp)) {
                    left = kStep;
                    if (k < turn) {                      // the one after: the tail was loaded before all
                        if (++at == c.ring)
                            at = 0, its ^= 1;
                    } else if (k == turn) {
                        at = first, its = first_phase;
                        left = it.depth % kStep;
                    }
                }
                if (!wait<true>(full + at * 8, its, p.most_ns))
                    return false;
                fence_after();
                if (elected()) {
                    const uint64_t a = first_a + at * (S::kStage >> 4), b = first_b + at * (S::kStage >> 4);
                    multiply(sums, a, b, idesc, add);                    // steps of 16 wholly past the end are left out
                    if (left > 16)
                        multiply(sums, a + kANext, b + kBNext, idesc, true);
                    if (left > 32)
                        multiply(sums, a + 2 * kANext, b + 2 * kBNext, idesc, true);
                    if (left > 48)
                        multiply(sums, a + 3 * kANext, b + 3 * kBNext, idesc, true);
                    commit<2>(empty + at * 8);
                    if (k + 1 == stop)
                        commit<2>(done + half * 8);
                }
                __syncwarp();
                if (++stage == c.ring)
                    stage = 0, phase ^= 1;
            }
            if (half ^= 1; half == 0)
                free_phase ^= 1;
        }
    }
    return true;
}

// A group's last stage holds rows of the next group: cleared up to the
// next multiple of 16, beyond which nothing is multiplied.
template <int kColumns>
__device__ __forceinline__ bool clear_tails(const Product &p, const Cta &c)
{
    using S = Shape<kColumns>;
    const int lane = threadIdx.x & 31;
    const uint32_t full = in_cta(smem_addr(&c.bars->full[0]), 0);
    int stage = 0;
    uint32_t phase = 0;                                  // a bit for each stage
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        if (it.tail) {
            const int left = it.depth % kStep, at = stage;
            if (!wait<false>(smem_addr(&c.bars->tail[at]), (phase >> at) & 1, p.most_ns))
                return false;
            phase ^= 1u << at;
            const int blocks = 2 + parts_of(it.wide / 2, 64), stop = (left + 15) / 16 * 16;
            uint4 *to = reinterpret_cast<uint4 *>(c.stages + at * S::kStage);
            for (int q = 0; q < blocks; ++q)
                for (int v = left * 8 + lane; v < stop * 8; v += 32)
                    to[q * (kBlock / 16) + v] = make_uint4(0, 0, 0, 0);
            fence_async_proxy();
            __syncwarp();
            if (lane == 0)
                release_in_pair(full + at * 8);
        }
        stage = (stage + it.k1 - it.k0) % c.ring;
    }
    return true;
}

template <int kColumns, int kOp>
__global__ void __launch_bounds__(Roles<kOp>::kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Product p)
{
    using S = Shape<kColumns>;
    extern __shared__ __align__(1024) uint8_t dynamic[];
    Cta c = cta_of(p, dynamic, p.ring * S::kStage);
    Barriers &bars = *c.bars;

    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (warp == kProducerWarp && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < c.ring; ++s) {
            barrier_init(smem_addr(&bars.full[s]), 2);               // counts in the first CTA, from both
            barrier_init(smem_addr(&bars.empty[s]), 1);
            barrier_init(smem_addr(&bars.tail[s]), 1);
        }
        init_epilogue_barriers<2>(bars, 4 * Roles<kOp>::kSides);
        barrier_init_fence();
    }
    if (warp == kMultiplyWarp)
        tmem_alloc<2>(smem_addr(&bars.tmem), S::kTmem);
    __syncwarp();
    greet_pair();
    // Nothing above depends on the kernels before this one on the stream.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == kTablesWarp)
        fill_tables<kStep, S::kJoin>(p, c.tables, kColumns, c.lane_tiles, c.pairs);
    join_pair();
    c.tmem = bars.tmem;
    c.split = c.tables.each[p.groups];
    c.items = c.tables.first[p.groups] * c.split;

    bool fine = true;
    if (warp < kFirstEpilogueWarp) {
        fewer_registers<Roles<kOp>::kControlRegisters>();
        if (warp == kProducerWarp)
            fine = load_stages<kColumns, kOp>(map_a, map_b, p, c);
        else if (warp == kMultiplyWarp && c.rank == 0)
            fine = multiply_stages<kColumns, kOp>(p, c);
        else if (warp == kTailWarp && rows_deep(kOp))
            fine = clear_tails<kColumns>(p, c);
    } else {
        more_registers<Roles<kOp>::kEpilogueRegisters>();
        fine = write_outputs<kColumns, Roles<kOp>::kSides, false, kStep, 2, kOp == kGated>(p, c);
    }
    finish_pair(fine, p.gave_up);
    if (warp == kMultiplyWarp)
        tmem_free<2>(c.tmem, S::kTmem);
}

// ---- host -----------------------------------------------------------------------

gnmr_status fail(gnmr_status s, const char *why)
{
    gnmr::record_thread_error(why);
    return s;
}

bool sixteen(int32_t dtype) { return dtype == GNMR_DTYPE_BF16 || dtype == GNMR_DTYPE_F16; }

gnmr_status gave_up(const gnmr_products *h)
{
    if (*static_cast<volatile int *>(h->gave_up))
        return fail(GNMR_ERR_STATE, "products: a product of this handle gave up waiting inside the GPU");
    return GNMR_OK;
}

bool misaligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// How long a wait inside the kernel may take.  One warp's can span all the others' work (that for the
// last stage that rows end in, or past tiles that are only written), so it is many times the whole
// call's: padded multiplies at a ninth of the tensor cores' rate, padded outputs at a hundredth of memory's, and two
// seconds, in which all that memory holds is read thirty times.
int64_t most_ns(const gnmr_product *p, const Product &q, int64_t lane_tiles)
{
    const double lanes = double(lane_tiles) * kLanes, more = 256.0 * q.groups;
    const double cols = q.cols ? q.cols + 256.0 : double(p->rows) + more, depth = q.depth ? q.depth : double(p->rows) + more;
    const double outputs = lanes * cols * (q.cols ? q.groups : 1);
    return static_cast<int64_t>(std::min(2e9 + lanes * cols * depth / 1e5 + outputs / 10, 9e18));
}

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
    if ((x && p->x_stride > far) || (dy && p->dy_stride > far) || (w && (p->w_stride > far || p->w_group_stride > far)) ||
        p->out_stride > far || (wgrad && p->out_group_stride > far))
        return fail(GNMR_ERR_LAYOUT, "products: a stride above 2^36 elements");
    // a gradient's groups lie one after the other, or row by row beside each other
    const __int128 group = static_cast<__int128>(p->n_out - 1) * p->out_stride + p->n_in;
    const __int128 rows_of_all = static_cast<__int128>(p->groups - 1) * p->out_group_stride + p->n_in;
    const bool apart = p->out_group_stride >= group || (p->out_group_stride >= p->n_in && p->out_stride >= rows_of_all);
    if ((x && p->x_stride < p->n_in) || (dy && p->dy_stride < p->n_out) ||
        (w && (p->w_stride < p->n_in || p->w_group_stride < 0)) || p->out_stride < wide_out ||
        (wgrad && p->groups > 1 && !apart) || (p->d_mask && p->groups > 1 && p->mask_stride < 1))
        return fail(GNMR_ERR_LAYOUT, "products: a stride below what it strides over");
    // operands that could not be copied, whatever memory there is
    const __int128 most_rows = std::max<int64_t>(p->rows, w ? int64_t(p->groups) * p->n_out : 0);
    if (most_rows * std::max(p->n_out, p->n_in) > (int64_t(1) << 56))
        return fail(GNMR_ERR_LAYOUT, "products: operands too large");
    const size_t eb = codes ? 1 : 2, ob = p->out_dtype == GNMR_DTYPE_F32 ? 4 : 2;
    if ((x && misaligned(p->d_x, eb)) || (dy && misaligned(p->d_dy, eb)) || (w && misaligned(p->d_w, eb)) ||
        misaligned(p->d_out, ob) || misaligned(p->d_offsets, 8) ||
        (codes && (misaligned(p->d_x_scale, 4) || misaligned(p->d_w_scale, 4))))
        return fail(GNMR_ERR_LAYOUT, "products: an operand not aligned to its element size");
    return GNMR_OK;
}

// 8-bit codes: the rows are read in 8 bits too up to kFewestCodes to a group, and up to kFewCodes to a
// group, or any number of one group, while tiles are few; otherwise they are widened in memory first.
// Measured in 8 bits and widened, us: 5120 -> 13824, 16 rows 19.9 and 21.0, 32 rows 24.5 and 21.3; 64 experts of
// 2048 -> 1408, 282 rows 35 and 39, 1,024 rows 45 and 44, 31 rows each 57 and 45; one group, 4096 -> 1024, 100 rows
// (8 tiles) 11.6 and 20; 2048 -> 2048, 200 (32) 12.4 and 14.8; 7296 -> 4352, 200 (68) 56 and 27; 24 experts of
// 1371 -> 1003, 400 rows (28) 16 and 20.  Rows to a group are an average, the counts being on the device: 1,024 rows of
// one of 64 experts of 2048 -> 1408 27 and 19, 16 rows each 39 and 43.
constexpr int64_t kFewestCodes = 16, kFewCodes = 32, kFewCodeTiles = 48;
// 16-bit operands: tiles of 64 columns up to this many rows to a group, and for one group
// while they make one round at most.  5120 -> 13824, 16 rows: 26 us so, 28 in tiles of 256; 64: 27 and 29;
// 128: 39 and 30.  2048 -> 2048, 16 rows: 8 and 12; 200: 10 and 17.  64 experts of 1408 -> 2048, 1 row
// each: 39 and 42, 64 each: 66 and 65.  An average here too: 4,096 rows of one of 64 experts of 2048 -> 1408 34
// and 31, 2,796 of 4,056 rows one expert's 77 and 77.
constexpr int64_t kFewRows = 64;

Operands operands(const gnmr_product *p)
{
    const bool codes = p->op == GNMR_PRODUCT_FORWARD_I8;
    const int bytes = codes ? 1 : 2;
    const int64_t narrow = (int64_t(p->n_out) + kLanes - 1) / kLanes * ((p->rows + 63) / 64);
    const bool few = p->rows <= kFewestCodes * p->groups ||
                     ((p->groups == 1 || p->rows <= kFewCodes * p->groups) && narrow <= kFewCodeTiles);
    const Operand x{p->d_x, p->rows, p->n_in, p->x_stride, 0, 1, bytes, codes && few ? 1 : 2};
    const Operand dy{p->d_dy, p->rows, p->n_out, p->dy_stride, 0, 1, 2, 2};
    const bool shared = p->w_group_stride == 0;          // one weight for all groups
    const Operand w{p->d_w, p->n_out, p->n_in, p->w_stride, p->w_group_stride, shared ? 1 : p->groups, bytes, bytes};
    if (p->op == GNMR_PRODUCT_WEIGHT_GRAD)
        return {x, dy};
    return {w, p->op == GNMR_PRODUCT_INPUT_GRAD ? dy : x};
}

template <int kColumns, int kOp>
cudaError_t launch(const gnmr_products *h, const Operands &o, Product p, cudaStream_t st, bool *mapped)
{
    p.ring = ring_of(p.groups, Shape<kColumns>::kStage, 0);
    CUtensorMap a, b;
    const CUtensorMapDataType type = p.bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    *mapped = (kOp == kGated ? gnmr::halves_map(h, &a, o.a, type, 128)
                             : gnmr::tile_map(h, &a, o.a, type, a_along_lanes(kOp) ? kStep : 128, p.a_blocks ? 2 : 1)) &&
              gnmr::tile_map(h, &b, o.b, type, b_along_columns(kOp) ? kStep : Shape<kColumns>::kBox, p.b_blocks ? 2 : 1);
    if (!*mapped)
        return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * h->pairs);
    cfg.blockDim = dim3(Roles<kOp>::kThreads);
    cfg.dynamicSmemBytes = shared_bytes(p.groups, Shape<kColumns>::kStage, 0);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, product_kernel<kColumns, kOp>, a, b, p);
}

template <int kColumns, int kOp> cudaError_t allow_shared()
{
    return cudaFuncSetAttribute(product_kernel<kColumns, kOp>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
}

// The kernels, by op and whether a group has few rows.
using Launch = cudaError_t (*)(const gnmr_products *, const Operands &, Product, cudaStream_t, bool *);
constexpr Launch kLaunch[5][2] = {
    {launch<256, GNMR_PRODUCT_FORWARD>, launch<64, GNMR_PRODUCT_FORWARD>},
    {launch<256, GNMR_PRODUCT_INPUT_GRAD>, launch<64, GNMR_PRODUCT_INPUT_GRAD>},
    {launch<256, GNMR_PRODUCT_WEIGHT_GRAD>, launch<256, GNMR_PRODUCT_WEIGHT_GRAD>},
    {gnmr::launch_codes, gnmr::launch_codes},
    {launch<256, kGated>, launch<64, kGated>},
};

cudaError_t allow_all_shared()
{
    cudaError_t e = cudaSuccess;
    for (const cudaError_t r : {allow_shared<256, GNMR_PRODUCT_FORWARD>(), allow_shared<64, GNMR_PRODUCT_FORWARD>(),
                                allow_shared<256, GNMR_PRODUCT_INPUT_GRAD>(), allow_shared<64, GNMR_PRODUCT_INPUT_GRAD>(),
                                allow_shared<256, GNMR_PRODUCT_WEIGHT_GRAD>(), allow_shared<256, kGated>(), allow_shared<64, kGated>(),
                                gnmr::allow_codes_shared()})
        e = e == cudaSuccess ? r : e;
    return e;
}

}  // namespace

namespace gnmr {

static bool encode(const gnmr_products *h, CUtensorMap *map, CUtensorMapDataType type, const void *at, const cuuint64_t *dims,
                   const cuuint64_t *strides, const cuuint32_t *box)
{
    const cuuint32_t one[4] = {1, 1, 1, 1};
    const auto once = [&] {
        return h->encode(map, type, 4, const_cast<void *>(at), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    };
    CUresult r = once();
    if (r == CUDA_ERROR_INVALID_CONTEXT || r == CUDA_ERROR_NOT_INITIALIZED) {
        cudaSetDevice(h->device);                        // a host thread's first CUDA call: it has no context yet
        r = once();
    }
    return r == CUDA_SUCCESS;
}

bool tile_map(const gnmr_products *h, CUtensorMap *map, const Operand &o, CUtensorMapDataType type, int high, int blocks)
{
    if (o.rows == 0) {                                   // nothing will be loaded
        memset(map, 0, sizeof(*map));
        return true;
    }
    const int wide = 128 / o.read_bytes;
    const cuuint64_t row = static_cast<cuuint64_t>(o.stride) * o.read_bytes;
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(blocks > 1 ? wide : o.cols), static_cast<cuuint64_t>(o.rows),
                                static_cast<cuuint64_t>(blocks > 1 ? o.cols / wide : 1), static_cast<cuuint64_t>(o.groups)};
    const cuuint64_t strides[3] = {row, 128, o.groups > 1 ? static_cast<cuuint64_t>(o.group_stride) * o.read_bytes : row};
    const cuuint32_t box[4] = {static_cast<cuuint32_t>(wide), static_cast<cuuint32_t>(high), static_cast<cuuint32_t>(blocks), 1};
    return encode(h, map, type, o.at, dims, strides, box);
}

bool halves_map(const gnmr_products *h, CUtensorMap *map, const Operand &o, CUtensorMapDataType type, int high)
{
    const cuuint64_t row = static_cast<cuuint64_t>(o.stride) * o.read_bytes, half = static_cast<cuuint64_t>(o.rows / 2);
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(o.cols), 2, half, static_cast<cuuint64_t>(o.groups)};
    const cuuint64_t strides[3] = {half * row, row, o.groups > 1 ? static_cast<cuuint64_t>(o.group_stride) * o.read_bytes : row};
    const cuuint32_t box[4] = {static_cast<cuuint32_t>(128 / o.read_bytes), 2, static_cast<cuuint32_t>(high / 2), 1};
    return encode(h, map, type, o.at, dims, strides, box);
}

}  // namespace gnmr

namespace {

// A gated block as the forward product of both its projections.
gnmr_status check(const gnmr_gated *p, gnmr_product *both)
{
    if (!p)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    if (p->activation != GNMR_ACT_SILU && p->activation != GNMR_ACT_GELU)
        return fail(GNMR_ERR_INVALID_ARG, "products: unknown activation");
    if (p->n < 1 || p->n > INT32_MAX / 4)
        return fail(GNMR_ERR_INVALID_ARG, "products: n out of range");
    const int64_t wide = 2 * int64_t(p->n), far = int64_t(1) << 36;
    if (p->out_stride < p->n || (p->d_keep && p->keep_stride < wide))
        return fail(GNMR_ERR_LAYOUT, "products: a stride below what it strides over");
    if (p->out_stride > far || (p->d_keep && p->keep_stride > far))
        return fail(GNMR_ERR_LAYOUT, "products: a stride above 2^36 elements");
    if (misaligned(p->d_keep, 2))
        return fail(GNMR_ERR_LAYOUT, "products: an operand not aligned to its element size");
    *both = {};
    both->op = GNMR_PRODUCT_FORWARD;
    both->groups = p->groups;
    both->rows = p->rows;
    both->n_out = static_cast<int32_t>(wide);
    both->n_in = p->n_in;
    both->dtype = both->out_dtype = p->dtype;
    both->d_offsets = p->d_offsets;
    both->d_mask = p->d_mask;
    both->mask_stride = p->mask_stride;
    both->d_x = p->d_x;
    both->x_stride = p->x_stride;
    both->d_w = p->d_w;
    both->w_stride = p->w_stride;
    both->w_group_stride = p->w_group_stride;
    both->d_out = p->d_out;
    both->out_stride = wide;
    both->d_scratch = p->d_scratch;
    both->scratch_bytes = p->scratch_bytes;
    return check(both);
}

// One product, or, as the forward product of both projections, a gated block; checked.
gnmr_status run(gnmr_products *h, const gnmr_product *p, const gnmr_gated *gated, void *stream)
{
    if (const gnmr_status s = gave_up(h))
        return s;
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
    const int64_t lane_tiles = (int64_t(q.lanes) + kLanes - 1) / kLanes;
    q.lane_tiles_inverse = static_cast<unsigned>(((int64_t(1) << 32) + lane_tiles - 1) / lane_tiles);
    q.rows = static_cast<int>(p->rows);
    q.groups = p->groups;
    q.offsets = p->d_offsets;
    q.mask = p->d_mask;
    q.mask_stride = p->mask_stride;
    q.want = codes ? 0 : 1;
    q.a_by_group = o.a.groups > 1;
    q.a_blocks = (wgrad || back) && q.lanes % 64 == 0;
    q.b_blocks = wgrad && q.cols % 64 == 0;
    q.granule = q.b_blocks ? 128 : 32;
    q.bf16 = !codes && p->dtype == GNMR_DTYPE_BF16;
    q.piece = !codes && p->out_dtype == GNMR_DTYPE_F32 ? 512 : 1024;
    q.out = p->d_out;
    q.out_type = p->out_dtype;
    q.add = wgrad && p->add;
    q.out_col = p->out_stride;
    q.out_group = p->out_group_stride;
    q.pairs_aligned = !misaligned(p->d_out, 4) && p->out_stride % 2 == 0 && (!wgrad || p->groups == 1 || p->out_group_stride % 2 == 0);
    if (gated) {
        q.out_col = gated->out_stride;
        q.pairs_aligned = !misaligned(gated->d_out, 4) && gated->out_stride % 2 == 0;
        q.act = gated->activation;
        q.keep = gated->d_keep;
        q.keep_col = gated->keep_stride;
        q.keep_aligned = !misaligned(gated->d_keep, 4) && gated->keep_stride % 2 == 0 && gated->n % 2 == 0;
    }
    if (codes)
        q.lane_scale = p->d_w_scale, q.col_scale = p->d_x_scale;
    q.parts = h->parts;
    q.tickets = h->tickets;
    q.gave_up = h->gave_up;
    q.most_ns = h->wait_ns < 0 ? most_ns(p, q, lane_tiles) : h->wait_ns;

    int prev = h->device;
    cudaGetDevice(&prev);
    if (prev != h->device)
        cudaSetDevice(h->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    char *scratch = static_cast<char *>(p->d_scratch);
    for (Operand *m : {&o.a, &o.b})
        if (const int64_t n = m->copy_bytes(); n && e == cudaSuccess) {
            e = gnmr::copy_operand(*m, scratch, 2 * h->pairs, st);
            const bool widened = m->bytes != m->read_bytes;      // then the zeros after the last column count as columns
            *m = Operand{scratch, m->rows, widened ? m->held() : m->cols, m->held(), m->rows * m->held(), m->groups, m->read_bytes,
                         m->read_bytes};
            scratch += n;
        }
    const bool few = !wgrad && (p->rows <= kFewRows * p->groups || (p->groups == 1 && lane_tiles * ((p->rows + 63) / 64) <= h->pairs));
    bool mapped = true;
    if (e == cudaSuccess)
        e = kLaunch[gated ? kGated : p->op][few](h, o, q, st, &mapped);
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
    const size_t parts = size_t(kMaxParts) * kPartFloats * 4, tickets = size_t(kMaxParts) * 2 * kMostEpilogueWarps * 4;
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
        e = allow_all_shared();
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
    return run(h, p, nullptr, stream);
}

gnmr_status gnmr_gated_scratch_bytes(const gnmr_gated *p, int64_t *bytes)
{
    if (!bytes)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL argument");
    *bytes = 0;
    gnmr_product both;
    if (const gnmr_status s = check(p, &both))
        return s;
    const Operands o = operands(&both);
    *bytes = o.a.copy_bytes() + o.b.copy_bytes();
    return GNMR_OK;
}

gnmr_status gnmr_products_gated(gnmr_products *h, const gnmr_gated *p, void *stream)
{
    if (!h)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL handle");
    gnmr_product both;
    if (const gnmr_status s = check(p, &both))
        return s;
    return run(h, &both, p, stream);
}

gnmr_status gnmr_products_status(gnmr_products *h)
{
    if (!h)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL handle");
    return gave_up(h);
}

gnmr_status gnmr_products_set_wait_limit(gnmr_products *h, int64_t nanoseconds)
{
    if (!h)
        return fail(GNMR_ERR_INVALID_ARG, "products: NULL handle");
    h->wait_ns = nanoseconds;
    return GNMR_OK;
}

gnmr_status gnmr_products_destroy(gnmr_products *h)
{
    if (!h)
        return GNMR_OK;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaSetDevice(h->device);
    cudaError_t e = h->dmem ? cudaFree(h->dmem) : cudaSuccess;      // waits for the device
    gnmr_status status = GNMR_OK;
    if (h->gave_up) {
        status = gave_up(h);
        const cudaError_t f = cudaFreeHost(h->gave_up);
        e = e == cudaSuccess ? f : e;
    }
    cudaSetDevice(prev);
    delete h;
    return e == cudaSuccess ? status : GNMR_ERR_CUDA;
}

}  // extern "C"
