// From the sums of a linear layer's product to its outputs: bias, Z, phi, residual, one rounding to bf16.
#pragma once

#include "attention_tc.cuh"

namespace rola {

struct LinearEnd {
    __nv_bfloat16* c;
    const __nv_bfloat16 *bias, *residual;        // or NULL
    float* Z;                                    // or NULL
    int act;
    int wide;                                    // rows of 32-byte sectors in c and in fp32 tensors of its shape
};

inline LinearEnd linear_end_of(void* c, const void* bias, const void* residual, float* Z, int N, int act)
{
    LinearEnd e;
    e.c = static_cast<__nv_bfloat16*>(c);
    e.bias = static_cast<const __nv_bfloat16*>(bias);
    e.residual = static_cast<const __nv_bfloat16*>(residual);
    e.Z = Z;
    e.act = act;
    e.wide = N % 16 == 0 && ((reinterpret_cast<uintptr_t>(c) | reinterpret_cast<uintptr_t>(Z)) & 31u) == 0;
    return e;
}

// 8 fp32 at a 16-byte aligned address; `wide`: it is 32-byte aligned
__device__ __forceinline__ void put8(float* p, const float* v, bool wide)
{
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
    if (wide) {
        tc::st_global32(p, w);
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(p + 4) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// W values of the row that starts at element `at`, from column f0 (a multiple of 8) of N on.
template <bool END, int W>
__device__ __forceinline__ void linear_end(const LinearEnd& p, size_t at, int f0, int N, float (&v)[W])
{
    if constexpr (END) {
        // the residual is on its way under what comes before it
        uint4 r[W / 8];
        if (p.residual)
#pragma unroll
            for (int e = 0; e < W; e += 8)
                if (f0 + e < N) r[e / 8] = *reinterpret_cast<const uint4*>(p.residual + at + f0 + e);
        if (p.bias)
#pragma unroll
            for (int e = 0; e < W; e += 8)
                if (f0 + e < N) {
                    float b[8];
                    load16(p.bias + f0 + e, b);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[e + j] += b[j];
                }
        if (p.Z)
#pragma unroll
            for (int e = 0; e < W; e += 8)
                if (f0 + e < N) put8(p.Z + at + f0 + e, v + e, p.wide);
        if (p.act != ROLA_LOWRANK_ACT_IDENTITY)
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] = act.phi(v[j]);
            });
        if (p.residual)
#pragma unroll
            for (int e = 0; e < W; e += 8)
                if (f0 + e < N) {
                    const uint32_t w[4] = {r[e / 8].x, r[e / 8].y, r[e / 8].z, r[e / 8].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 f = unpack_bf16(w[j]);
                        v[e + 2 * j] += f.x;
                        v[e + 2 * j + 1] += f.y;
                    }
                }
    }
#pragma unroll
    for (int e = 0; e < W; e += 16) {
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = e + 2 * j < W ? pack_bf16(v[e + 2 * j], v[e + 2 * j + 1]) : 0u;
        __nv_bfloat16* row = p.c + at + f0 + e;
        if (W >= 16 && f0 + e + 16 <= N) tc::store_row32(row, y, p.wide);
        else if (f0 + e < N) *reinterpret_cast<uint4*>(row) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

// The end of a product whose K axis was split: the parts [splits][M][N], added in order.
cudaError_t launch_linear_join(const LinearEnd& end, const float* part, int splits, int M, int N, cudaStream_t st);

}  // namespace rola
