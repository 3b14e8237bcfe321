// TMA copies of boxes of a row-major matrix: the tensor map, and the load of a
// box into 128- or 64-byte-swizzled shared memory.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <stddef.h>
#include <stdint.h>

namespace rola {

// A [rows][cols] matrix of `esz`-byte elements (cols * esz a multiple of 16),
// boxes of box_rows x box_cols.  Elements outside it read as zero.
bool encode_2d(CUtensorMap* m, CUtensorMapDataType type, int esz, const void* ptr, int64_t rows, int64_t cols,
               int box_cols, int box_rows, CUtensorMapSwizzle swizzle);

// [parts][rows][cols] fp32 (cols a multiple of 4), boxes of one part's 32 rows x 32 columns in 128-byte swizzle.
bool encode_parts(CUtensorMap* m, const float* ptr, int64_t parts, int64_t rows, int64_t cols);

namespace tc {

// x * element size must be a multiple of 16.
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* map, uint32_t bar, int x, int y)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n" ::"r"(
            dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}

// Stores of a box from shared memory (bulk-group completion); the coordinates lie inside the tensor, and what of the
// box does not is not written.
__device__ __forceinline__ void tma_store_2d(const void* map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n" ::"l"(map), "r"(src),
                 "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void tma_store_3d(const void* map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];\n" ::"l"(map), "r"(src),
                 "r"(x), "r"(y), "r"(z)
                 : "memory");
}

}  // namespace tc
}  // namespace rola
