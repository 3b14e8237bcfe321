// TMA copies of boxes of a row-major matrix: the tensor map, and the loads and
// stores of a box in 128- or 64-byte-swizzled shared memory.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <stddef.h>
#include <stdint.h>

namespace rola {

// A [rows][cols] matrix of `esz`-byte elements (cols * esz a multiple of 16),
// boxes of box_rows x box_cols.  Elements outside it read as zero and are not written.
bool encode_2d(CUtensorMap* m, CUtensorMapDataType type, int esz, const void* ptr, int64_t rows, int64_t cols,
               int box_cols, int box_rows, CUtensorMapSwizzle swizzle);

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
// Neither coordinate negative; what lies outside the matrix is not written.
__device__ __forceinline__ void tma_store_2d(const void* map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n" ::"l"(map), "r"(src),
                 "r"(x), "r"(y)
                 : "memory");
}
// Waits until at most one of this thread's committed bulk groups still reads shared memory.
__device__ __forceinline__ void bulk_wait_read_1() { asm volatile("cp.async.bulk.wait_group.read 1;\n" ::: "memory"); }

}  // namespace tc
}  // namespace rola
