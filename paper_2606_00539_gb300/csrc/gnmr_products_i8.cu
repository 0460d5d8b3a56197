// Expert products on 8-bit codes.
//
// sm_103a's tensor cores (tcgen05) take no 8-bit integers, so codes are multiplied as
// fp16, which holds them exactly: products are at most 2^14 and a piece of
// 1,024 of them sums to at most 2^24, exact in fp32; pieces are added as integers.
//
// The weights stay 8 bits wide up to the SM: eight warps widen A's tiles into tensor
// memory, from where the tensor cores take an operand as well, at no cost in
// shared-memory bandwidth (tiles of fp16 in shared memory, written and read again for each
// tile of columns, would take more of it than there is beside the multiplies).
//
// B, the rows, are widened by two more warps where they are few, and each CTA multiplies alone:
// what is widened in shared memory is then handed over within its CTA (between CTAs that takes
// 2,000 cycles a stage).  Else a kernel before this one widens them in memory, and CTAs multiply
// in pairs.  Widening the weights in memory too, for the 16-bit kernel, was slower at 4,001 rows
// to a group (5120 -> 13824: 380 us, this way 321 to 337).
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

// ---- weights in 8 bits --------------------------------------------------------------

constexpr int kStep = 128;                             // contraction steps of a stage: 128-byte rows of codes
constexpr int kProducerWarp = 0, kMultiplyWarp = 1, kFirstBWarp = 2, kTablesWarp = 3;
constexpr int kSides = 2, kFirstWidenWarp = kFirstEpilogueWarp + 4 * kSides, kWidenWarps = 8;
constexpr int kThreads = 32 * (kFirstWidenWarp + kWidenWarps);
// 96 registers a thread at launch, shared out anew: the epilogue holds the sums.
constexpr int kControlRegisters = 56, kEpilogueRegisters = 136, kWidenRegisters = 72;
static_assert(128 * kControlRegisters + 256 * kEpilogueRegisters + 256 * kWidenRegisters <= kThreads * 96, "registers of the launch");
constexpr int kAStage = 128 * kStep, kSlots = 4, kFirstA = 256, kTmem = 512;

// kWide: B comes in 16 bits, and a tile has up to 128 columns; else up to 32, widened here
// (up to 64 leave room for fewer stages: one token through 5120 -> 13824 23.9 us, 18.6 so).  Widened: A behind the sums in tensor memory, 64 columns of two steps each; B in
// shared memory, as two tiles of 64 steps.
template <bool kWide> struct Shape {
    static constexpr int kCtas = kWide ? 2 : 1;        // that multiply as one
    static constexpr int kColumns = kWide ? 128 : 32;
    static constexpr int kBRows = kColumns / kCtas, kBTile = kBRows * 128;
    static constexpr int kStage = kAStage + (kWide ? 2 : 1) * kBTile;
    static constexpr int kSlot = 2 * kBTile;           // B widened, before the stages
    static constexpr int kWidened = kWide ? 0 : kSlots * kSlot;
    static_assert(2 * kColumns <= kFirstA && kFirstA + kSlots * kStep / 2 <= kTmem, "columns of tensor memory");
};

template <bool kWide>
__device__ __forceinline__ bool load_stages(const CUtensorMap &map_a, const CUtensorMap &map_b, const Product &p, const Cta &c)
{
    using S = Shape<kWide>;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = smem_addr(&c.bars->empty[0]), base = smem_addr(c.stages) + S::kWidened;
    const uint32_t own = in_cta(full, c.rank), full_b = in_cta(smem_addr(&c.bars->tail[0]), 0);
    int stage = 0;
    uint32_t phase = 1;
    if (p.most_ns == 0)
        return false;                                    // no time at all: the others wait in vain
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const int a_lane = it.lane0 + c.rank * 128, za = p.a_by_group ? it.g : 0;
        const int b_col = it.row0 + it.col0 + (kWide ? c.rank * (it.wide / 2) : 0);
        for (int k = it.k0; k < it.k1; ++k) {
            if (!wait<kWide>(empty + stage * 8, phase, p.most_ns))
                return false;
            if (elected()) {
                const uint32_t bar = full + stage * 8, a = base + stage * S::kStage, b = a + kAStage;
                if (kWide) {
                    arrive_expect(own + stage * 8, kAStage);
                    arrive_expect(full_b + stage * 8, 2 * S::kBTile);
                    load_tile<S::kCtas>(a, &map_a, k * kStep, a_lane, 0, za, bar);
                    load_tile<S::kCtas>(b, &map_b, 0, b_col, 2 * k, 0, full_b + stage * 8);
                } else {
                    arrive_expect(own + stage * 8, S::kStage);
                    load_tile<S::kCtas>(a, &map_a, k * kStep, a_lane, 0, za, bar);
                    load_tile<S::kCtas>(b, &map_b, k * kStep, b_col, 0, 0, bar);
                }
            }
            __syncwarp();
            if (++stage == c.ring)
                stage = 0, phase ^= 1;
        }
    }
    return true;
}

// Two places on in a ring of n.
__device__ __forceinline__ void two_on(int &at, uint32_t &phase, int n)
{
    if ((at += 2) >= n)
        at -= n, phase ^= 1;
}

// A's tiles into tensor memory, by two teams of four warps that take the stages in turn.
template <bool kWide>
__device__ __forceinline__ bool widen_a(const Product &p, const Cta &c)
{
    constexpr int kStage = Shape<kWide>::kStage;
    const int warp = threadIdx.x / 32 - kFirstWidenWarp, lane = threadIdx.x & 31, quarter = warp & 3, team = warp >> 2;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = smem_addr(&c.bars->empty[0]);
    const uint32_t used = smem_addr(&c.bars->used[0]), ready = in_cta(smem_addr(&c.bars->ready[0]), kWide ? 0 : c.rank);
    const int row = quarter * 32 + lane;
    const uint8_t *raw = c.stages + Shape<kWide>::kWidened + row * 128;
    int stage = team, slot = team;                     // every other stage, from the team's first
    uint32_t phase = 0, slot_phase = 1;
    int skip = team;                                   // stages until then
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        int k = it.k0 + skip;
        for (; k < it.k1; k += 2) {
            if (!wait<false>(full + stage * 8, phase, p.most_ns) || !wait<kWide>(used + slot * 8, slot_phase, p.most_ns))
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
                release(empty + stage * 8);
            store_wait();
            fence_before();
            __syncwarp();
            if (lane == 0)
                arrive(ready + slot * 8);
            two_on(stage, phase, c.ring);
            two_on(slot, slot_phase, kSlots);
        }
        skip = k - it.k1;
    }
    return true;
}

// B's tiles to shared memory, by two warps in turn.
__device__ __forceinline__ bool widen_b(const Product &p, const Cta &c)
{
    using S = Shape<false>;
    constexpr int kStage = S::kStage, kSlot = S::kSlot, kBTile = S::kBTile;
    const int lane = threadIdx.x & 31, turn = threadIdx.x / 32 - kFirstBWarp, chunk = lane & 7;
    const uint32_t full = smem_addr(&c.bars->full[0]), empty = smem_addr(&c.bars->empty[0]);
    const uint32_t used = smem_addr(&c.bars->used[0]), ready = smem_addr(&c.bars->ready[0]);
    int stage = turn, slot = turn, skip = turn;
    uint32_t phase = 0, slot_phase = 1;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const int rows = it.cols;                      // those beyond are columns that nobody reads
        int k = it.k0 + skip;
        for (; k < it.k1; k += 2) {
            if (!wait<false>(full + stage * 8, phase, p.most_ns) || !wait<false>(used + slot * 8, slot_phase, p.most_ns))
                return false;
            const uint8_t *raw = c.stages + S::kWidened + stage * kStage + kAStage;
            uint8_t *to = c.stages + slot * kSlot + (chunk >> 2) * kBTile;
#pragma unroll 4
            for (int r = lane >> 3; r < rows; r += 4) {
                const uint4 codes = *reinterpret_cast<const uint4 *>(raw + r * 128 + ((chunk ^ (r & 7)) << 4));
                const uint2 v0 = widen4(codes.x), v1 = widen4(codes.y), v2 = widen4(codes.z), v3 = widen4(codes.w);
                const int at = (chunk & 3) * 2, x = r & 7;
                *reinterpret_cast<uint4 *>(to + r * 128 + ((at ^ x) << 4)) = make_uint4(v0.x, v0.y, v1.x, v1.y);
                *reinterpret_cast<uint4 *>(to + r * 128 + (((at + 1) ^ x) << 4)) = make_uint4(v2.x, v2.y, v3.x, v3.y);
            }
            fence_async_proxy();
            __syncwarp();
            if (lane == 0) {
                release(empty + stage * 8);
                release(ready + slot * 8);
            }
            two_on(stage, phase, c.ring);
            two_on(slot, slot_phase, kSlots);
        }
        skip = k - it.k1;
    }
    return true;
}

template <bool kWide>
__device__ __forceinline__ bool multiply_slots(const Product &p, const Cta &c)
{
    using S = Shape<kWide>;
    const uint32_t ready = smem_addr(&c.bars->ready[0]), used = smem_addr(&c.bars->used[0]);
    const uint32_t full_b = smem_addr(&c.bars->tail[0]), empty = smem_addr(&c.bars->empty[0]);
    const uint32_t done = smem_addr(&c.bars->done[0]), drained = smem_addr(&c.bars->drained[0]);
    const uint64_t first_b = operand(smem_addr(c.stages) + (kWide ? kAStage : 0), 16, 1024);
    int slot = 0, stage = 0, half = 0;
    uint32_t phase = 0, stage_phase = 0, free_phase = 1;
    for (int i = c.pair, g = 0; i < c.items; i += c.pairs) {
        const Item it = item_of<kStep>(p, c.tables, c.split, c.lane_tiles, i, g);
        const uint32_t idesc = shape<S::kCtas>(false, false, false, it.wide);
        for (int k = it.k0; k < it.k1;) {
            if (!wait<kWide>(drained + half * 8, free_phase, p.most_ns))
                return false;
            fence_after();
            const int stop = min(it.k1, k + p.piece / kStep);
            const uint32_t sums = c.tmem + half * S::kColumns;
            for (bool add = false; k < stop; ++k, add = true) {
                if ((kWide && !wait<true>(full_b + stage * 8, stage_phase, p.most_ns)) || !wait<kWide>(ready + slot * 8, phase, p.most_ns))
                    return false;
                fence_after();
                if (elected()) {
                    const uint32_t a = c.tmem + kFirstA + slot * (kStep / 2);
                    const uint64_t b = first_b + (kWide ? stage * (S::kStage >> 4) : slot * (S::kSlot >> 4));
#pragma unroll
                    for (int q = 0; q < kStep / 16; ++q)
                        multiply<S::kCtas>(sums, a + q * 8, b + (q >> 2) * (S::kBTile >> 4) + (q & 3) * 2, idesc, q > 0 || add);
                    commit<S::kCtas>(used + slot * 8);
                    if (kWide)
                        commit<S::kCtas>(empty + stage * 8);
                    if (k + 1 == stop)
                        commit<S::kCtas>(done + half * 8);
                }
                __syncwarp();
                if (++slot == kSlots)
                    slot = 0, phase ^= 1;
                if (++stage == c.ring)
                    stage = 0, stage_phase ^= 1;
            }
            if (half ^= 1; half == 0)
                free_phase ^= 1;
        }
    }
    return true;
}

template <bool kWide>
__global__ void __launch_bounds__(kThreads, 1)
codes_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Product p)
{
    using S = Shape<kWide>;
    extern __shared__ __align__(1024) uint8_t dynamic[];
    Cta c = cta_of(p, dynamic, p.ring * S::kStage + S::kWidened);
    Barriers &bars = *c.bars;

    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (warp == kProducerWarp && lane == 0) {
        prefetch_map(&map_a);
        prefetch_map(&map_b);
        for (int s = 0; s < c.ring; ++s) {
            barrier_init(smem_addr(&bars.full[s]), 1);
            barrier_init(smem_addr(&bars.empty[s]), kWidenWarps / 2 + 1);        // a team, and B's warp or multiplies
            barrier_init(smem_addr(&bars.tail[s]), 2);                           // B in 16 bits: in the first CTA, from both
        }
        for (int s = 0; s < kSlots; ++s) {
            barrier_init(smem_addr(&bars.ready[s]), kWide ? 2 * (kWidenWarps / 2) : kWidenWarps / 2 + 1);      // likewise; this CTA's
            barrier_init(smem_addr(&bars.used[s]), 1);
        }
        init_epilogue_barriers<S::kCtas>(bars, 4 * kSides);
        barrier_init_fence();
    }
    if (warp == kMultiplyWarp)
        tmem_alloc<S::kCtas>(smem_addr(&bars.tmem), kTmem);
    __syncwarp();
    greet_pair();
    // Nothing above depends on the kernels before this one on the stream.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (warp == kTablesWarp)
        fill_tables<kStep, kWide ? 2 : 1>(p, c.tables, S::kColumns, c.lane_tiles, c.pairs);
    join_pair();
    c.tmem = bars.tmem;
    c.split = c.tables.each[p.groups];
    c.items = c.tables.first[p.groups] * c.split;

    bool fine = true;
    if (warp < kFirstEpilogueWarp) {
        fewer_registers<kControlRegisters>();
        if (warp == kProducerWarp)
            fine = load_stages<kWide>(map_a, map_b, p, c);
        else if (warp == kMultiplyWarp && (c.rank == 0 || !kWide))
            fine = multiply_slots<kWide>(p, c);
        else if (!kWide && warp >= kFirstBWarp)
            fine = widen_b(p, c);
    } else if (warp < kFirstWidenWarp) {
        more_registers<kEpilogueRegisters>();
        fine = write_outputs<S::kColumns, kSides, true, kStep, S::kCtas>(p, c);
    } else {
        fewer_registers<kWidenRegisters>();
        fine = widen_a<kWide>(p, c);
    }
    finish_pair(fine, p.gave_up);
    if (warp == kMultiplyWarp)
        tmem_free<S::kCtas>(c.tmem, kTmem);
}

template <bool kWide>
cudaError_t launch(const gnmr_products *h, const Operands &o, Product p, cudaStream_t st, bool *mapped)
{
    using S = Shape<kWide>;
    p.ring = ring_of(p.groups, S::kStage, S::kWidened);
    CUtensorMap a, b;
    *mapped = gnmr::tile_map(h, &a, o.a, CU_TENSOR_MAP_DATA_TYPE_UINT8, 128, 1) &&
              (kWide ? gnmr::tile_map(h, &b, o.b, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, S::kBRows, 2)
                     : gnmr::tile_map(h, &b, o.b, CU_TENSOR_MAP_DATA_TYPE_UINT8, S::kBRows, 1));
    if (!*mapped)
        return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * h->pairs);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = shared_bytes(p.groups, S::kStage, S::kWidened);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, codes_kernel<kWide>, a, b, p);
}

// ---- copies of operands -------------------------------------------------------------
// [rows][cols] of every group to rows of `held` elements, a multiple of 16 bytes, what is past
// `cols` in each 0.  Bound by memory: 3 bytes a code, 4 a 16-bit number.
struct Copy {
    const void *from;
    void *to;
    int64_t rows, cols, stride, group_stride, held;
};

constexpr int kCopyThreads = 256;

// kFrom bytes an element to kTo; 16 codes or 8 numbers a thread and turn.  kWhole: rows that 16-byte loads can take,
// of codes to be widened (others of that kind are read in place).
template <int kFrom, int kTo, bool kWhole>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(Copy c)
{
    constexpr int kN = 16 / kFrom;
    static_assert(!kWhole || kFrom < kTo, "aligned operands that are not widened are not copied");
    const int g = blockIdx.y;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const char *from = static_cast<const char *>(c.from) + g * c.group_stride * kFrom;
    char *to = static_cast<char *>(c.to) + g * c.rows * c.held * kTo;
    const int64_t across = (c.held + kN - 1) / kN, total = c.rows * across;
    // then a row's last vector is whole too; with fewer columns than `held`, what follows the last
    // row's need not be the caller's
    const bool flat = c.stride == c.held && c.cols == c.held;
    for (int64_t i = int64_t(blockIdx.x) * kCopyThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kCopyThreads) {
        int64_t at = i * kN, out = i * kN;
        int left = kN;
        if (!flat || !kWhole) {
            const int64_t r = i / across, col = (i - r * across) * kN;
            at = r * c.stride + col;
            out = r * c.held + col;
            left = static_cast<int>(min(int64_t(kN), c.cols - col));
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
            w[1] = make_uint4(d.x, d.y, e.x, e.y);            // `held` is whole 128 bytes
        }
    }
}

template <int kFrom, int kTo, bool kWhole>
cudaError_t launch_copy(const Copy &c, int groups, int sms, cudaStream_t st)
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
    return cudaLaunchKernelEx(&cfg, copy_kernel<kFrom, kTo, kWhole>, c);
}

}  // namespace

namespace gnmr {

cudaError_t copy_operand(const Operand &o, void *to, int sms, cudaStream_t st)
{
    const Copy c{o.at, to, o.rows, o.cols, o.stride, o.group_stride, o.held()};
    const int64_t steps = o.stride * o.bytes | (o.groups > 1 ? o.group_stride * o.bytes : 0);
    const bool whole = ((reinterpret_cast<uintptr_t>(o.at) | static_cast<uintptr_t>(steps)) & 15) == 0;
    if (o.bytes == 2)
        return launch_copy<2, 2, false>(c, o.groups, sms, st);
    if (o.read_bytes == 1)
        return launch_copy<1, 1, false>(c, o.groups, sms, st);
    return whole ? launch_copy<1, 2, true>(c, o.groups, sms, st) : launch_copy<1, 2, false>(c, o.groups, sms, st);
}

cudaError_t allow_codes_shared()
{
    const cudaError_t e = cudaFuncSetAttribute(codes_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(codes_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost);
}

cudaError_t launch_codes(const gnmr_products *h, const Operands &o, Product p, cudaStream_t st, bool *mapped)
{
    return o.b.read_bytes == 2 ? launch<true>(h, o, p, st, mapped) : launch<false>(h, o, p, st, mapped);
}

}  // namespace gnmr
