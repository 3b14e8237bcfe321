// The gradient of a linear layer's epilogue: dZ = dY phi'(Z), and the bias' gradient, the column sums of dZ.
//
// A pass over memory: dY and Z in (2 or 4, and 4 bytes an element), dZ out; with the identity dZ is dY and only the
// sums remain.  A CTA takes 256 neighbouring columns, eight a lane, and a part of the rows, one a warp at a time.  A
// lane sums its columns in registers, the warps meet in shared memory in warp order, the parts in a second kernel in
// part order: the same bits every time.  The sums are of dZ in fp32, before it is rounded.
//
// Measured: GELU at 8190 x 6144 69 us (402 MB, 5.8 TB/s; with erfcf and expf 143 us), the sums of 32760 x 1536 alone 16 us.
#include "linear.cuh"
#include "linear_finish.cuh"

namespace rola {
namespace {

constexpr int kWarps = 8, kColumns = 256;

__device__ __forceinline__ void load8(const float* p, float (&x)[8])
{
    const float4 a = load4(p), b = load4(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) { load16(p, x); }
__device__ __forceinline__ void store8(float* p, const float (&x)[8])
{
    store4(p, make_float4(x[0], x[1], x[2], x[3]));
    store4(p + 4, make_float4(x[4], x[5], x[6], x[7]));
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) { store16(p, x); }

// d *= phi'(z) of eight values.  bf16 layers take the fast forms of SiLU and GELU, whose errors (about 1e-6) are below
// what the sums over d_in leave in z.
template <typename T, int ACT>
__device__ __forceinline__ void times_slope(float (&d)[8], float (&z)[8])
{
    if constexpr (sizeof(T) == 2 && ACT == ROLA_LOWRANK_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) FastGelu::slope(*reinterpret_cast<float(*)[2]>(&z[e]));
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= z[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a, da;
            if constexpr (sizeof(T) == 2 && ACT == ROLA_LOWRANK_ACT_SILU) FastSilu::grad(z[e], a, da);
            else gate_act_grad(ACT, z[e], a, da);
            d[e] *= da;
        }
    }
}

// ACT: one of rola_lowrank_act_t, or -1 without Z.
template <typename T, int ACT>
__global__ void __launch_bounds__(32 * kWarps) linear_grad_kernel(int M, int N, const T* __restrict__ dY,
                                                                  const float* __restrict__ Z, T* __restrict__ dZ,
                                                                  float* __restrict__ part,
                                                                  DeviceStatus* __restrict__ status)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) status->code = status->where = 0;
    __shared__ float sum[kWarps][kColumns + 8];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * kColumns + lane * 8;
    const int r0 = (int)((long long)M * blockIdx.y / gridDim.y), r1 = (int)((long long)M * (blockIdx.y + 1) / gridDim.y);
    float s[8] = {};
    if (c < N) {                                             // N is a multiple of 8
#pragma unroll 2
        for (int r = r0 + w; r < r1; r += kWarps) {
            const size_t at = (size_t)r * N + c;
            float d[8];
            load8(dY + at, d);
            if constexpr (ACT >= 0) {
                float z[8];
                load8(Z + at, z);
                times_slope<T, ACT>(d, z);
                store8(dZ + at, d);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += d[e];
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[w][lane * 8 + e] = s[e];
    __syncthreads();
    const int col = blockIdx.x * kColumns + threadIdx.x;
    if (col >= N) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) t += sum[i][threadIdx.x];
    part[(size_t)blockIdx.y * N + col] = t;
}

// db = the sum of the parts [n][N]: 32 columns a CTA, whose warps add every 8th part and meet in warp order.
__global__ void __launch_bounds__(256) linear_bias_kernel(int n, int N, const float* __restrict__ part,
                                                          float* __restrict__ db)
{
    __shared__ float sum[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float t = 0.0f;
    if (c < N) {
#pragma unroll 4
        for (int i = w; i < n; i += 8) t += part[(size_t)i * N + c];
    }
    sum[w][lane] = t;
    __syncthreads();
    if (w || c >= N) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) t += sum[i][lane];
    db[c] = t;
}

// Eight outputs a thread from the parts of a split K axis.
__global__ void __launch_bounds__(256) linear_join_kernel(const LinearEnd end, const float* __restrict__ part, int splits, int M,
                                                          int N)
{
    const size_t all = (size_t)M * N, at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= all) return;
    float v[8];
    load8(part + at, v);
#pragma unroll 4
    for (int i = 1; i < splits; ++i) {
        float x[8];
        load8(part + i * all + at, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
    }
    if (end.bias) {
        float b[8];
        load8(end.bias + at % N, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += b[e];
    }
    if (end.Z) store8(end.Z + at, v);
    linear_phi(end.act, v);
    if (end.residual) {
        float r[8];
        load8(end.residual + at, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    store8(end.c + at, v);
}

template <typename T>
cudaError_t grad(const LinShape& s, const void* dY, const float* Z, void* dZ, float* db, float* part, DeviceStatus* status,
                 cudaStream_t st)
{
    const dim3 grid((s.N + kColumns - 1) / kColumns, linear_grad_parts(s));
    auto go = [&](auto kernel) {
        kernel<<<grid, 32 * kWarps, 0, st>>>(s.M, s.N, static_cast<const T*>(dY), Z, static_cast<T*>(dZ), db ? part : nullptr,
                                           status);
        return cudaGetLastError();
    };
    cudaError_t e;
    if (!Z) e = go(linear_grad_kernel<T, -1>);
    else if (s.act == ROLA_LOWRANK_ACT_SILU) e = go(linear_grad_kernel<T, ROLA_LOWRANK_ACT_SILU>);
    else if (s.act == ROLA_LOWRANK_ACT_TANH) e = go(linear_grad_kernel<T, ROLA_LOWRANK_ACT_TANH>);
    else if (s.act == ROLA_LOWRANK_ACT_RELU) e = go(linear_grad_kernel<T, ROLA_LOWRANK_ACT_RELU>);
    else e = go(linear_grad_kernel<T, ROLA_LOWRANK_ACT_GELU>);
    if (e != cudaSuccess || !db) return e;
    linear_bias_kernel<<<(s.N + 31) / 32, 256, 0, st>>>(grid.y, s.N, part, db);
    return cudaGetLastError();
}

}  // namespace

// Four CTAs on each of 152 SMs, each with a row a warp at least.
int linear_grad_parts(const LinShape& s)
{
    const int bands = (s.N + kColumns - 1) / kColumns, most = (s.M + kWarps - 1) / kWarps;
    const int want = (608 + bands - 1) / bands;
    return want < most ? want : most;
}

cudaError_t launch_linear_grad(rola_dtype_t dt, const LinShape& s, const void* dY, const float* Z, void* dZ, float* db,
                               float* part, DeviceStatus* status, cudaStream_t st)
{
    return dt == ROLA_BF16 ? grad<__nv_bfloat16>(s, dY, Z, dZ, db, part, status, st)
                           : grad<float>(s, dY, Z, dZ, db, part, status, st);
}

cudaError_t launch_linear_join(const LinearEnd& end, const float* part, int splits, int M, int N, cudaStream_t st)
{
    const size_t pieces = (size_t)M * N / 8;
    linear_join_kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(end, part, splits, M, N);
    return cudaGetLastError();
}

}  // namespace rola
