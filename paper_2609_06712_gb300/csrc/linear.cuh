// Linear layers with their epilogue: sizes and launches.
#pragma once

#include "block_ops.cuh"

namespace rola {

struct LinShape {
    int M, K, N, act;                // tokens, d_in, d_out
    uint64_t wait_limit_ns;
    int debug_flags;
};

// Z = X W^T + b, Y = R + phi(Z); b, R and Z may be NULL: fp32, bf16 (tensor cores)
cudaError_t launch_linear_simt(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                               float* Z, cudaStream_t st);
cudaError_t launch_linear_tc(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                             float* Z, DeviceStatus* status, cudaStream_t st);
// dX = dZ W and dW = dZ^T X, either NULL: fp32, bf16 (tensor cores)
cudaError_t launch_linear_backward_simt(const LinShape& s, const void* X, const void* W, const void* dZ, void* dX,
                                        void* dW, cudaStream_t st);
cudaError_t launch_linear_backward_tc(const LinShape& s, const void* X, const void* W, const void* dZ, void* dX,
                                      void* dW, DeviceStatus* status, cudaStream_t st);

// dZ = dY phi'(Z) (with Z), and db = its column sums (with db), in parts of rows that are joined in order
int linear_grad_parts(const LinShape& s);
cudaError_t launch_linear_grad(rola_dtype_t dt, const LinShape& s, const void* dY, const float* Z, void* dZ, float* db,
                               float* part, cudaStream_t st);

}  // namespace rola
