// The expert products' handle and operands, and what their translation units
// call of each other.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdint>

#include "gnmr_tiles.cuh"

struct gnmr_products {
    int device = 0;
    int pairs = 1;
    float *parts = nullptr;            // [kMaxParts][kPartFloats]
    unsigned *tickets = nullptr;       // [kMaxParts][2][kMostEpilogueWarps], 0 between calls
    int *gave_up = nullptr;            // host memory that the kernels can write
    int64_t wait_ns = -1;              // limit of a wait; negative: by the call's sizes
    void *dmem = nullptr;
    CUresult (*encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                       const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                       CUtensorMapL2promotion, CUtensorMapFloatOOBfill) = nullptr;
};

namespace gnmr {

// A matrix operand of 1- or 2-byte elements, and the element size that its kernel
// reads; operands that are not read in place are copied to rows of `held` elements, zeros
// after the last column: whole 16 bytes, or whole blocks of 128 where they are widened.
struct Operand {
    const void *at;
    int64_t rows, cols, stride, group_stride;
    int groups;
    int bytes, read_bytes;
    int64_t held() const
    {
        const int64_t unit = (bytes == read_bytes ? 16 : 128) / read_bytes;
        return (cols + unit - 1) / unit * unit;
    }
    bool in_place() const
    {
        const int64_t steps = stride * bytes | (groups > 1 ? group_stride * bytes : 0);
        return bytes == read_bytes && ((reinterpret_cast<uintptr_t>(at) | static_cast<uintptr_t>(steps)) & 15) == 0;
    }
    int64_t copy_bytes() const
    {
        return in_place() || rows == 0 ? 0 : (groups * rows * held() * read_bytes + 255) / 256 * 256;
    }
};

struct Operands {
    Operand a, b;
};

// Tiles of `high` rows by `blocks` blocks of 128 bytes of an operand, a block after the other.
// Several blocks: the operand's columns are whole blocks.  Coordinates of a tile: its
// first column, or 0 where there are several blocks; row; block, or 0 where there is one; group.
bool tile_map(const gnmr_products *h, CUtensorMap *map, const Operand &o, CUtensorMapDataType type, int high, int blocks);

// Tiles of `high` rows by 128 bytes whose rows come from the operand's two halves in turn: row 2 i is row i, row
// 2 i + 1 is row rows / 2 + i.  Coordinates: first column; 0; row of a half; group.
bool halves_map(const gnmr_products *h, CUtensorMap *map, const Operand &o, CUtensorMapDataType type, int high);

// The copy of an operand in `to`.
cudaError_t copy_operand(const Operand &o, void *to, int sms, cudaStream_t st);

// The 8-bit product; b may be widened.
cudaError_t launch_codes(const gnmr_products *h, const Operands &o, gnmr_tiles::Product p, cudaStream_t st, bool *mapped);
cudaError_t allow_codes_shared();

}  // namespace gnmr
