// The gated residual sum and its norms: sizes, tensors, the split of the rows, and the launches.
#pragma once

#include "block_ops.cuh"

namespace rola {

struct RnShape {
    int groups, rows, d;             // samples, rows of each, width
    int norm, branch;                // rola_norm_t of the sum and of the branch
    long long mod_stride, total;     // total: groups rows
    float eps;
    int debug_flags;
    uint64_t wait_limit_ns;          // of a row's copy
};

// Vectors that are not there are NULL.  Backward: part and moments are workspace.
struct RnArgs {
    const void *x, *h, *gate, *gamma_h, *gamma, *beta, *scale, *shift, *dout, *dy;
    void *out, *y, *dx, *dh;
    float* stats;                    // [total][4]: mean, rstd of the sum; mean, rstd of the branch
    float *dgate, *dgamma_h, *dgamma, *dbeta, *dscale, *dshift;
    float* part;                     // [parts + groups - 1][3][rn_padded(d)]: sums of dy v, dy and dx hh over the rows that a part and a sample share
    float* shared;                   // [rn_shares][3][rn_padded(d)]: of the vectors that all samples share
    float4* moments;                 // [total], rows too long for registers: the four means of the backward
    int parts;                       // of the rows
    const void* in[4];               // the matrices that a kernel streams, or NULL
    int norm_sums;                   // whether the norm's vectors have a gradient that is wanted
};

// Rows [rn_row(i), rn_row(i + 1)) are part i's; part i leaves the sums of sample s in slot i + s.  Parts and samples both
// ascend with the row, so that no two pairs (i, s) with rows in common have the same slot.
__host__ __device__ __forceinline__ long long rn_row(long long total, int parts, int i) { return total * i / parts; }
// The part of row r: the largest i with rn_row(i) <= r.
__host__ __device__ __forceinline__ int rn_part(long long total, int parts, long long r)
{
    return (int)(((r + 1) * parts - 1) / total);
}

__host__ __device__ __forceinline__ int rn_padded(int d) { return (d + 3) / 4 * 4; }
// Where a slot's sums start, in floats.  (Part and sample together may pass 31 bits, not 32.)
__host__ __device__ __forceinline__ size_t rn_slot(uint32_t part, uint32_t s, int d)
{
    return (size_t)(part + s) * 3 * rn_padded(d);
}

int rn_shares(const RnShape& s);                     // shares of the samples in the sums over them
int rn_parts(const RnShape& s);                      // most parts of the backward, for the workspace
bool rn_long(const RnShape& s);                      // whether the backward takes the rows from memory in several passes

cudaError_t launch_residual_norm(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st);
cudaError_t launch_residual_norm_backward(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st);

}  // namespace rola
