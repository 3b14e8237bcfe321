// Linear layers with their epilogue: sizes and launches.
#pragma once

#include "block_ops.cuh"

namespace rola {

struct LinShape {
    int M, K, N, act;                // tokens, d_in, d_out
    uint64_t wait_limit_ns;
    int debug_flags;
};

// Z = X W^T + b, Y = R + phi(Z); b, R and Z may be NULL
cudaError_t launch_linear_simt(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                               float* Z, cudaStream_t st);                                                 // fp32
// bf16, by tokens: weight rows against up to four, then weight tiles against few tokens, then 256-token tiles on tensor
// cores.  Each clears the status word.
bool linear_by_rows(const LinShape& s);
bool linear_few(const LinShape& s);
cudaError_t launch_linear_rows(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                               float* Z, DeviceStatus* status, cudaStream_t st);
cudaError_t launch_linear_few(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                              float* Z, DeviceStatus* status, cudaStream_t st);
cudaError_t launch_linear_tc(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                             float* Z, float* part, DeviceStatus* status, cudaStream_t st);

// dX = dZ W and dW = dZ^T X: fp32 (either NULL), bf16; `clear`: the status word is to be cleared
cudaError_t launch_linear_backward_simt(const LinShape& s, const void* X, const void* W, const void* dZ, void* dX,
                                        void* dW, cudaStream_t st);
cudaError_t launch_linear_few_dx(const LinShape& s, const void* W, const void* dZ, void* dX, bool clear,
                                 DeviceStatus* status, cudaStream_t st);
cudaError_t launch_linear_dx_tc(const LinShape& s, const void* W, const void* dZ, void* dX, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st);
cudaError_t launch_linear_dw_tc(const LinShape& s, const void* X, const void* dZ, void* dW, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st);

// Parts of the K axis of a product [M][N] over K on tensor cores.
int linear_splits(int64_t M, int64_t N, int64_t K);
inline size_t linear_part_bytes(int64_t M, int64_t N, int64_t K)
{
    const int splits = linear_splits(M, N, K);
    return splits > 1 ? 4 * (size_t)splits * M * N : 0;
}

// dZ = dY phi'(Z) (with Z), and db = its column sums (with db), in parts of rows that are joined in order; clears the
// status word
int linear_grad_parts(const LinShape& s);
cudaError_t launch_linear_grad(rola_dtype_t dt, const LinShape& s, const void* dY, const float* Z, void* dZ, float* db,
                               float* part, DeviceStatus* status, cudaStream_t st);

}  // namespace rola
