// Shared by the norms: pieces of a row in registers, packed fp32 arithmetic on them, and sums over the threads that
// hold a row.
#pragma once

#include "block_ops.cuh"

namespace rola {

// A piece as loaded: 16 bytes (V elements), or one element (V = 1).
template <typename T, int V>
struct Piece {
    uint4 w;
};
template <typename T>
struct Piece<T, 1> {
    T w;
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p)
{
    Piece<T, V> x;
    x.w = *reinterpret_cast<const decltype(x.w)*>(p);
    return x;
}
template <typename T, int V>
__device__ __forceinline__ void unpack(const Piece<T, V>& x, float (&v)[V])
{
    if constexpr (V == 1) v[0] = to_float(x.w);
    else load16(reinterpret_cast<const T*>(&x.w), v);
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const float (&x)[V])
{
    if constexpr (V == 1) p[0] = from_float<T>(x[0]);
    else store16(p, x);
}

// Two elements an instruction (packed fp32, each element an IEEE operation): the rows of d = 1536 leave an SM
// 430 cycles a row, fewer than one instruction per element and operation would take.
__device__ __forceinline__ void fma2(float* d, const float* a, const float* b, const float* c)
{
    asm("{\n.reg .b64 ra, rb, rc;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmov.b64 rc, {%6, %7};\n"
        "fma.rn.f32x2 ra, ra, rb, rc;\nmov.b64 {%0, %1}, ra;\n}\n"
        : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]), "f"(c[0]), "f"(c[1]));
}
// d = a b + c of a piece; b and c may be one value for all elements
template <int V>
__device__ __forceinline__ void fma_piece(float (&d)[V], const float (&a)[V], const float (&b)[V], const float (&c)[V])
{
    if constexpr (V == 1) d[0] = fmaf(a[0], b[0], c[0]);
    else
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(d + e, a + e, b + e, c + e);
}
template <int V>
__device__ __forceinline__ void fma_piece(float (&d)[V], const float (&a)[V], float b, float c)
{
    const float bb[2] = {b, b}, cc[2] = {c, c};
    if constexpr (V == 1) d[0] = fmaf(a[0], b, c);
    else
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(d + e, a + e, bb, cc);
}
// s (two partial sums) += a b, or += a
template <int V>
__device__ __forceinline__ void dot_piece(float (&s)[2], const float (&a)[V], const float (&b)[V])
{
    if constexpr (V == 1) s[0] = fmaf(a[0], b[0], s[0]);
    else
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(s, a + e, b + e, s);
}
template <int V>
__device__ __forceinline__ void add_piece(float (&d)[V], const float (&a)[V])
{
    const float one[2] = {1.0f, 1.0f};
    if constexpr (V == 1) d[0] += a[0];
    else
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(d + e, a + e, one, d + e);
}
template <int V>
__device__ __forceinline__ void sum_piece(float (&s)[2], const float (&a)[V])
{
    const float one[2] = {1.0f, 1.0f};
    if constexpr (V == 1) s[0] += a[0];
    else
#pragma unroll
        for (int e = 0; e < V; e += 2) fma2(s, a + e, one, s);
}

// Sum of (a, b) over the threads of a group, the same bits in every thread.  A
// group of more than one warp is the whole CTA; `turn` alternates between two
// buffers, so that one barrier separates a sum's writes from its reads and the
// next sum's barrier its reads from the writes after that.
template <bool WARP>
__device__ __forceinline__ float2 group_sum(float a, float b, float2 (*red)[32], int& turn)
{
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, off);
        b += __shfl_xor_sync(0xffffffffu, b, off);
    }
    if constexpr (!WARP) {
        const int lane = threadIdx.x & 31;
        float2* buf = red[turn];
        turn ^= 1;
        if (lane == 0) buf[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        const int warps = blockDim.x >> 5;
        if (warps <= 4) {
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (w < warps) {
                    a += buf[w].x;
                    b += buf[w].y;
                }
        } else {
            const float2 t = lane < warps ? buf[lane] : make_float2(0.0f, 0.0f);
            a = t.x;
            b = t.y;
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, off);
                b += __shfl_xor_sync(0xffffffffu, b, off);
            }
        }
    }
    return make_float2(a, b);
}

}  // namespace rola
