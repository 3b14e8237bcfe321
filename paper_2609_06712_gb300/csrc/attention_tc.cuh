// Shared by the tensor-core attention kernels over a dense key set (forward
// and backward).
#pragma once

#include <cuda.h>

#include "block_ops.cuh"
#include "tcgen05.cuh"

namespace rola {

// A [heads][rows][128] bf16 tensor as (d, row, head), boxes of 64 d x box_rows
// rows in 128-byte swizzle: a d-chunk of a tile.  Rows past `rows` read as zero.
bool encode_rows(CUtensorMap* m, const void* ptr, int64_t rows, int64_t heads, int box_rows);

// dk and dv from D, in one launch (or their parts)
cudaError_t launch_attention_dkdv_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st);

// The item of a persistent CTA's turn: turns of gridDim.x items run forwards and backwards in turn, so that with
// items sorted by length (causal: the longest first) the CTAs' sums stay close; items or more when there is none.
// (4095 causal rows x 3 shared heads, 8 key heads: dk and dv 343 us in plain turns, 247 so; dq 138 and 123, the
// forward 140 and 99, with the rows in falling_tile's order.)
__device__ __forceinline__ int turn_item(int turn, int items)
{
    const int base = turn * (int)gridDim.x;
    if (base >= items) return items;
    return base + ((turn & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
}

// The j-th of `tiles` row tiles of a key head that `sharing` query heads share, by falling position: a head's rows
// follow the last head's, and each ends at its last position.  Where the heads do not fill whole tiles the order is
// off by less than a tile a head, which only the balance feels.
__device__ __forceinline__ int falling_tile(int j, int tiles, int sharing)
{
    const int per = tiles / sharing, rest = tiles - per * sharing;
    if (j < rest) return tiles - 1 - j;
    j -= rest;
    return (j % sharing + 1) * per - 1 - j / sharing;
}

namespace tc {

// True in one lane of the (converged) warp.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
    return p != 0;
}

// D[tmem] (+)= A[tmem] * B[smem]: A is M rows of K 16-bit values in TMEM,
// two per 32-bit column (the lower K index in the low half).
__device__ __forceinline__ void mma_ts_split(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi,
                                             uint32_t idesc, uint32_t accum)
{
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 db;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "mov.b64 db, {%2, %3};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}\n" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accum)
        : "memory");
}

// NC consecutive columns of this thread's TMEM lane
template <int NC>
__device__ __forceinline__ void row_load(uint32_t taddr, float (&v)[NC])
{
#pragma unroll
    for (int c = 0; c < NC / 16; ++c) tmem_ld16(taddr + c * 16, *reinterpret_cast<float(*)[16]>(&v[c * 16]));
    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&v[0]));
#pragma unroll
    for (int c = 1; c < NC / 16; ++c) reg_fence(*reinterpret_cast<float(*)[16]>(&v[c * 16]));
}
// 32 bytes at a 32-byte aligned address, one access
__device__ __forceinline__ void st_global32(void* p, const uint32_t (&y)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(p), "r"(y[0]), "r"(y[1]), "r"(y[2]),
                 "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                 : "memory");
}

// 16 bf16 at a 16-byte aligned address; `wide`: it is 32-byte aligned
__device__ __forceinline__ void store_row32(__nv_bfloat16* p, const uint32_t (&y)[8], bool wide)
{
    if (wide) {
        st_global32(p, y);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<uint4*>(p + 8) = make_uint4(y[4], y[5], y[6], y[7]);
    }
}

// (a, b) = (a * m + c, b * m + c), one packed f32x2 instruction (each element an IEEE fma)
__device__ __forceinline__ void ffma2(float& a, float& b, float m, float c)
{
    asm("{\n.reg .b64 ra, rm, rc;\nmov.b64 ra, {%0, %1};\nmov.b64 rm, {%2, %2};\nmov.b64 rc, {%3, %3};\n"
        "fma.rn.f32x2 ra, ra, rm, rc;\nmov.b64 {%0, %1}, ra;\n}\n"
        : "+f"(a), "+f"(b) : "f"(m), "f"(c));
}
// (a, b) = (a * m + c, b * m + d)
__device__ __forceinline__ void ffma2(float& a, float& b, float m, float c, float d)
{
    asm("{\n.reg .b64 ra, rm, rc;\nmov.b64 ra, {%0, %1};\nmov.b64 rm, {%2, %2};\nmov.b64 rc, {%3, %4};\n"
        "fma.rn.f32x2 ra, ra, rm, rc;\nmov.b64 {%0, %1}, ra;\n}\n"
        : "+f"(a), "+f"(b) : "f"(m), "f"(c), "f"(d));
}
// (a, b) = ((a + c) * p, (b + d) * q)
__device__ __forceinline__ void fadd_mul2(float& a, float& b, float c, float d, float p, float q)
{
    asm("{\n.reg .b64 ra, rc, rp;\nmov.b64 ra, {%0, %1};\nmov.b64 rc, {%2, %3};\nmov.b64 rp, {%4, %5};\n"
        "add.rn.f32x2 ra, ra, rc;\nmul.rn.f32x2 ra, ra, rp;\nmov.b64 {%0, %1}, ra;\n}\n"
        : "+f"(a), "+f"(b) : "f"(c), "f"(d), "f"(p), "f"(q));
}
__device__ __forceinline__ void fadd2(float& a, float& b, float p, float q)
{
    asm("{\n.reg .b64 ra, rp;\nmov.b64 ra, {%0, %1};\nmov.b64 rp, {%2, %3};\n"
        "add.rn.f32x2 ra, ra, rp;\nmov.b64 {%0, %1}, ra;\n}\n"
        : "+f"(a), "+f"(b) : "f"(p), "f"(q));
}

}  // namespace tc
}  // namespace rola
