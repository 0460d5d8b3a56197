// Expert products on 8-bit codes.
//
// sm_103a's tensor cores take no 8-bit integers at their full rate, so codes are
// multiplied as fp16, which holds them exactly: products are below 2^14 and a piece of
// 1,024 of them sums to at most 2^24, exact in fp32; pieces are added as integers.
//
// Few rows to a group are bound by reading the weights, so these stay 8 bits wide up
// to the SM: eight warps widen A's tiles into tensor memory (from where the tensor cores
// take an operand as well, at no cost in shared-memory bandwidth), two more B's, a
// few columns, into shared memory.  Many rows are bound by the multiplies, and widening a
// tile again for every 256 columns would take the shared memory that the
// tensor cores read from: there both operands are widened in memory once, and the 16-bit
// kernel multiplies them.
#include <algorithm>
#include <cstring>

#include "gnmr_products.h"

namespace {

using namespace gnmr_tiles;
using gnmr::Operand;
using gnmr::Operands;

// Four codes as fp16 pairs: a code's bits with the sign bit turned are code + 128, the low
// byte of the fp16 number 1024 + (code + 128).
__device__ __forceinline__ uint2 widen4(uint32_t codes)
{
    const uint32_t w = codes ^ 0x80808080u;
    uint2 v;
    asm("{\n.reg .b32 lo, hi, k;\nmov.b32 k, 0xe480e480;\n"                  // -1152
        "prmt.b32 lo, %2, 0x64646464, 0x5140;\nprmt.b32 hi, %2, 0x64646464, 0x5342;\n"
        "add.rn.f16x2 %0, lo, k;\nadd.rn.f16x2 %1, hi, k;\n}"
        : "=r"(v.x), "=r"(v.y)
        : "r"(w));
    return v;
}

// ---- few rows to a group ------------------------------------------------------------

constexpr int kColumns = 64;                           // of a tile, at most
constexpr int kStep = 128;                             // contraction steps of a stage: 128-byte rows of codes
constexpr int kProducerWarp = 0, kMultiplyWarp = 1, kFirstBWarp = 2, kTablesWarp = 3;
constexpr int kFirstWidenWarp = kFirstEpilogueWarp + kEpilogueWarps, kWidenWarps = 8;
constexpr int kThreads = 32 * (kFirstWidenWarp + kWidenWarps);
constexpr int kAStage = 128 * kStep, kStage = kAStage + kColumns / 2 * kStep, kStages = 8;
// Widened: B in shared memory, as two tiles of 64 steps; A behind the sums in tensor
// memory, 64 columns of two steps each.
constexpr int kSlots = 4, kBTile = kColumns / 2 * 128, kSlot = 2 * kBTile;
constexpr int kFirstA = 256, kTmem = 512;
static_assert(2 * kColumns <= kFirstA && kFirstA + kSlots * kStep / 2 <= kTmem, "columns of tensor memory");
constexpr int kShared = kStages * kStage + kSlots * kSlot + static_cast<int>(sizeof(Tables)) + 1024;

__device__ __forceinline__ bool load_stages(const CUtensorMap &map_a, const CUtensorMap &map_b, const Product &p, const Cta &c)
{
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = smem_addr(&c.bars->empty[0]), base = smem_addr(c.stages);
    int stage = 0;
    uint32_t phase = 1;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, *c.tables, c.lane_tiles, i, g);
        const int half = (it.cols + 31) / 32 * 16;
        const int a_lane = it.lane0 + c.rank * 128, b_col = it.row0 + it.col0 + c.rank * half, za = p.a_by_group ? it.g : 0;
        for (int k = it.k0; k < it.k1; ++k) {
            if (!wait(empty + stage * 8, phase))
                return false;
            if (elected()) {
                const uint32_t bar = full + stage * 8, a = base + stage * kStage;
                arrive_expect(in_cta(bar, c.rank), kStage);
                load_tile(a, &map_a, k * kStep, a_lane, za, bar);
                load_tile(a + kAStage, &map_b, k * kStep, b_col, 0, bar);
            }
            __syncwarp();
            if (++stage == kStages)
                stage = 0, phase ^= 1;
        }
    }
    return true;
}

// A's tiles into tensor memory, by two teams of four warps that take the stages in turn.
__device__ __forceinline__ bool widen_a(const Product &p, const Cta &c)
{
    const int warp = threadIdx.x / 32 - kFirstWidenWarp, lane = threadIdx.x & 31, quarter = warp & 3, team = warp >> 2;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = in_cta(smem_addr(&c.bars->empty[0]), c.rank);
    const uint32_t used = smem_addr(&c.bars->used[0]), ready = in_cta(smem_addr(&c.bars->ready[0]), 0);
    const int row = quarter * 32 + lane;
    const uint8_t *raw = c.stages + row * 128;
    int n = 0;                                         // stages so far
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, *c.tables, c.lane_tiles, i, g);
        const int end = n + it.k1 - it.k0;
        for (n += (n ^ team) & 1; n < end; n += 2) {
            const int stage = n % kStages, slot = n % kSlots;
            if (!wait(full + stage * 8, (n / kStages) & 1) || !wait(used + slot * 8, (n / kSlots + 1) & 1))
                return false;
            fence_after();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t a[32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint4 codes = *reinterpret_cast<const uint4 *>(raw + stage * kStage + (((h * 4 + q) ^ (row & 7)) << 4));
                    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint2 v = widen4(w[j]);
                        a[8 * q + 2 * j] = v.x;
                        a[8 * q + 2 * j + 1] = v.y;
                    }
                }
                store32(c.tmem + kFirstA + slot * (kStep / 2) + h * 32 + (uint32_t(quarter * 32) << 16), a);
            }
            __syncwarp();
            if (lane == 0)
                arrive(empty + stage * 8);
            store_wait();
            fence_before();
            __syncwarp();
            if (lane == 0)
                arrive(ready + slot * 8);
        }
        n = end;
    }
    return true;
}

// B's tiles to shared memory, by two warps in turn.
__device__ __forceinline__ bool widen_b(const Product &p, const Cta &c)
{
    const int lane = threadIdx.x & 31, turn = threadIdx.x / 32 - kFirstBWarp, chunk = lane & 7;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = in_cta(smem_addr(&c.bars->empty[0]), c.rank);
    const uint32_t used = smem_addr(&c.bars->used[0]), ready = in_cta(smem_addr(&c.bars->ready[0]), 0);
    int n = 0;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, *c.tables, c.lane_tiles, i, g);
        const int end = n + it.k1 - it.k0, half = (it.cols + 31) / 32 * 16;
        for (n += (n ^ turn) & 1; n < end; n += 2) {
            const int stage = n % kStages, slot = n % kSlots;
            if (!wait(full + stage * 8, (n / kStages) & 1) || !wait(used + slot * 8, (n / kSlots + 1) & 1))
                return false;
            const uint8_t *raw = c.stages + stage * kStage + kAStage;
            uint8_t *to = c.stages + kStages * kStage + slot * kSlot + (chunk >> 2) * kBTile;
#pragma unroll 4
            for (int r = lane >> 3; r < half; r += 4) {
                const uint4 codes = *reinterpret_cast<const uint4 *>(raw + r * 128 + ((chunk ^ (r & 7)) << 4));
                const uint2 v0 = widen4(codes.x), v1 = widen4(codes.y), v2 = widen4(codes.z), v3 = widen4(codes.w);
                const int at = (chunk & 3) * 2, x = r & 7;
                *reinterpret_cast<uint4 *>(to + r * 128 + ((at ^ x) << 4)) = make_uint4(v0.x, v0.y, v1.x, v1.y);
                *reinterpret_cast<uint4 *>(to + r * 128 + (((at + 1) ^ x) << 4)) = make_uint4(v2.x, v2.y, v3.x, v3.y);
            }
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) {
                arrive(empty + stage * 8);
                arrive_release(ready + slot * 8);
            }
        }
        n = end;
    }
    return true;
}

__device__ __forceinline__ bool multiply_slots(const Product &p, const Cta &c)
{
    const uint32_t ready = smem_addr(&c.bars->ready[0]), used = smem_addr(&c.bars->used[0]);
    const uint32_t done = smem_addr(&c.bars->done[0]), drained = smem_addr(&c.bars->drained[0]);
    const uint64_t first_b = operand(smem_addr(c.stages) + kStages * kStage, 16, 1024);
    int slot = 0, half = 0;
    uint32_t phase = 0, free_phase = 1;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, *c.tables, c.lane_tiles, i, g);
        const uint32_t idesc = shape(false, false, false, (it.cols + 31) / 32 * 32);
        for (int k = it.k0; k < it.k1;) {
            if (!wait(drained + half * 8, free_phase))
                return false;
            fence_after();
            const int stop = min(it.k1, k + p.piece / kStep);
            const uint32_t sums = c.tmem + half * kColumns;
            for (bool add = false; k < stop; ++k, add = true) {
                if (!wait(ready + slot * 8, phase))
                    return false;
                fence_after();
                if (elected()) {
                    const uint32_t a = c.tmem + kFirstA + slot * (kStep / 2);
                    const uint64_t b = first_b + slot * (kSlot >> 4);
#pragma unroll
                    for (int q = 0; q < kStep / 16; ++q)
                        multiply(sums, a + q * 8, b + (q >> 2) * (kBTile >> 4) + (q & 3) * 2, idesc, q > 0 || add);
                    commit(used + slot * 8);
                    if (k + 1 == stop)
                        commit(done + half * 8);
                }
                __syncwarp();
                if (++slot == kSlots)
                    slot = 0, phase ^= 1;
            }
            if (half ^= 1; half == 0)
                free_phase ^= 1;
        }
    }
    return true;
}

__global__ void __launch_bounds__(kThreads, 1)
codes_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Product p)
{
    extern __shared__ uint8_t dynamic[];
    __shared__ Barriers bars;
    Cta c;
    c.stages = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(dynamic) + 1023) & ~uintptr_t(1023));
    Tables *tables = reinterpret_cast<Tables *>(c.stages + kStages * kStage + kSlots * kSlot);
    c.tables = tables;
    c.bars = &bars;
    c.rank = cta_rank();
    c.pair = blockIdx.x >> 1;
    c.pairs = gridDim.x >> 1;
    c.lane_tiles = parts_of(p.lanes, kLanes);

    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (warp == kProducerWarp && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < kStages; ++s) {
            barrier_init(smem_addr(&bars.full[s]), 1);
            barrier_init(smem_addr(&bars.empty[s]), kWidenWarps / 2 + 1);
        }
        for (int s = 0; s < kSlots; ++s) {
            barrier_init(smem_addr(&bars.ready[s]), 2 * (kWidenWarps / 2 + 1));    // counts in the first CTA, from both
            barrier_init(smem_addr(&bars.used[s]), 1);
        }
        init_epilogue_barriers(bars);
        barrier_init_fence();
    }
    if (warp == kMultiplyWarp)
        tmem_alloc(smem_addr(&bars.tmem), kTmem);
    // Nothing above depends on the kernels before this one on the stream.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == kTablesWarp)
        fill_tables<kStep>(p, *tables, kColumns, c.lane_tiles, c.pairs);
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    c.tmem = bars.tmem;
    c.items = tables->first[p.groups] * tables->split;

    bool fine = true;
    if (warp == kProducerWarp)
        fine = load_stages(map_a, map_b, p, c);
    else if (warp == kMultiplyWarp && c.rank == 0)
        fine = multiply_slots(p, c);
    else if (warp >= kFirstWidenWarp)
        fine = widen_a(p, c);
    else if (warp == kFirstBWarp || warp == kFirstBWarp + 1)
        fine = widen_b(p, c);
    else if (warp >= kFirstEpilogueWarp)
        fine = write_outputs<kColumns, true, kStep>(p, c);
    finish_pair(fine, p.gave_up);
    if (warp == kMultiplyWarp)
        tmem_free(c.tmem, kTmem);
}

// ---- copies of operands -------------------------------------------------------------
// [rows][cols] of every group to rows of `held` elements, a multiple of 16 bytes, what is past
// `cols` in each 0.  Bound by memory: 3 bytes a code, 4 a 16-bit number.
struct Copy {
    const void *from;
    void *to;
    int64_t rows, cols, stride, group_stride, held;
    const int64_t *offsets;                            // not NULL: groups without rows are left out
    const uint8_t *mask;                               // not NULL: and those that are not computed
    int64_t mask_stride;
    int want;
};

constexpr int kCopyThreads = 256;

// kFrom bytes an element to kTo; 16 codes or 8 numbers a thread and turn.  kWhole: rows that 16-byte loads can take.
template <int kFrom, int kTo, bool kWhole>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(Copy c)
{
    constexpr int kN = 16 / kFrom;
    const int g = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if ((c.offsets && c.offsets[g + 1] <= c.offsets[g]) || (c.mask && (c.mask[g * c.mask_stride] != 0) != (c.want != 0)))
        return;
    const char *from = static_cast<const char *>(c.from) + g * c.group_stride * kFrom;
    char *to = static_cast<char *>(c.to) + g * c.rows * c.held * kTo;
    const int64_t across = (c.held + kN - 1) / kN, total = c.rows * across;
    const bool flat = c.stride == c.held;              // then a row's last vector is whole too
    for (int64_t i = int64_t(blockIdx.x) * kCopyThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kCopyThreads) {
        int64_t at = i * kN, out = i * kN;
        int left = kN, room = kN;
        if (!flat || !kWhole) {
            const int64_t r = i / across, col = (i - r * across) * kN;
            at = r * c.stride + col;
            out = r * c.held + col;
            left = static_cast<int>(min(int64_t(kN), c.cols - col));
            room = static_cast<int>(min(int64_t(kN), c.held - col));
        }
        uint4 v;
        if (kWhole && left == kN) {
            v = __ldcs(reinterpret_cast<const uint4 *>(from + at * kFrom));
        } else {
            uint8_t e[16];
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                e[kFrom * j] = j < left ? from[(at + j) * kFrom] : 0;
                if (kFrom == 2)
                    e[2 * j + 1] = j < left ? from[(at + j) * kFrom + 1] : 0;
            }
            memcpy(&v, e, 16);
        }
        uint4 *w = reinterpret_cast<uint4 *>(to + out * kTo);
        if (kFrom == kTo) {
            *w = v;
        } else {
            const uint2 a = widen4(v.x), b = widen4(v.y), d = widen4(v.z), e = widen4(v.w);
            w[0] = make_uint4(a.x, a.y, b.x, b.y);
            if (room > 8)
                w[1] = make_uint4(d.x, d.y, e.x, e.y);
        }
    }
}

template <int kFrom, int kTo>
cudaError_t launch_copy(const Copy &c, int groups, bool whole, int sms, cudaStream_t st)
{
    const int64_t vectors = c.rows * ((c.held * kFrom + 15) / 16);
    const int64_t most = std::max<int64_t>(int64_t(sms) * 32 / groups, 1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(std::min((vectors + kCopyThreads - 1) / kCopyThreads, most)), groups);
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, whole ? copy_kernel<kFrom, kTo, true> : copy_kernel<kFrom, kTo, false>, c);
}

}  // namespace

namespace gnmr {

cudaError_t copy_operand(const Operand &o, void *to, const Product &p, bool by_group, int sms, cudaStream_t st)
{
    Copy c{o.at, to, o.rows, o.cols, o.stride, o.group_stride, o.held(), nullptr, nullptr, 0, 0};
    if (by_group) {
        c.offsets = p.offsets;
        c.mask = p.mask;
        c.mask_stride = p.mask_stride;
        c.want = p.want;
    }
    const int64_t steps = o.stride * o.bytes | (o.groups > 1 ? o.group_stride * o.bytes : 0);
    const bool whole = ((reinterpret_cast<uintptr_t>(o.at) | static_cast<uintptr_t>(steps)) & 15) == 0;
    if (o.bytes == 2)
        return launch_copy<2, 2>(c, o.groups, whole, sms, st);
    return o.read_bytes == 2 ? launch_copy<1, 2>(c, o.groups, whole, sms, st) : launch_copy<1, 1>(c, o.groups, whole, sms, st);
}

cudaError_t allow_codes_shared()
{
    return cudaFuncSetAttribute(codes_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared);
}

cudaError_t launch_codes(const gnmr_products *h, const Operands &o, const Product &p, cudaStream_t st, bool *mapped)
{
    CUtensorMap a, b;
    *mapped = tile_map(h, &a, o.a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 128) &&
              tile_map(h, &b, o.b, CU_TENSOR_MAP_DATA_TYPE_UINT8, kColumns / 2);
    if (!*mapped)
        return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * h->pairs);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kShared;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, codes_kernel, a, b, p);
}

}  // namespace gnmr
