// From the sums of a linear layer's product to its outputs: bias, Z, phi, residual, one rounding to bf16.
#pragma once

#include "block_ops.cuh"

namespace rola {

struct LinearEnd {
    __nv_bfloat16* c;
    const __nv_bfloat16 *bias, *residual;        // or NULL
    float* Z;                                    // or NULL
    int act;
};

inline LinearEnd linear_end_of(void* c, const void* bias, const void* residual, float* Z, int act)
{
    LinearEnd e;
    e.c = static_cast<__nv_bfloat16*>(c);
    e.bias = static_cast<const __nv_bfloat16*>(bias);
    e.residual = static_cast<const __nv_bfloat16*>(residual);
    e.Z = Z;
    e.act = act;
    return e;
}

// The end of a product whose K axis was split: the parts [splits][M][N], added in order.
cudaError_t launch_linear_join(const LinearEnd& end, const float* part, int splits, int M, int N, cudaStream_t st);

}  // namespace rola
