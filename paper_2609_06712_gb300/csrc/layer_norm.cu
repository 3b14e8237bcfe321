// Layer norm over the rows of x [rows][d], and its gradients.
//
//   y = (x - mu) rstd gamma + beta,   mu = mean x,   rstd = (mean (x - mu)^2 + eps)^(-1/2)
//   dx = rstd (a - mean a - xh mean(a xh)),   a = dy gamma,   xh = (x - mu) rstd
//   dgamma = sum_rows dy xh,   dbeta = sum_rows dy
//
// HBM-bound: x once in and y once out forward, x and dy in and dx out backward
// (a few fp32 operations per element against 4 or 6 bytes).  A row is held by
// a group of TPR threads in registers, NV pieces of V elements each, so that
// mean, centred sum of squares and output take one read of the row.  V is 16
// bytes where the row length and the pointers allow it, else one element.
// TPR = 32 (no barrier, one shuffle reduction) while the row needs at most
// kMaxWarpPieces pieces per lane, then 128 and 512 threads.
//
// Backward: every thread keeps the dgamma / dbeta sums of its own columns in
// registers over all the rows its group takes (row r of group g: g, g + G, ...),
// the groups of a CTA add theirs through shared memory in group order, and each
// CTA writes one partial row; a second kernel adds the partial rows in CTA
// order.  All sums are fp32.
#include "block_ops.cuh"

namespace rola {
namespace {

constexpr int kLnThreads = 128;          // of a CTA whose rows have a warp or 128 threads each


template <typename T, int V>
__device__ __forceinline__ void load_piece(const T* p, float (&x)[V])
{
    if constexpr (V == 1) x[0] = to_float(p[0]);
    else load16(p, x);
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const float (&x)[V])
{
    if constexpr (V == 1) p[0] = from_float<T>(x[0]);
    else store16(p, x);
}

// Sum of (a, b) over the TPR threads of a group, the same bits in every thread.
template <int TPR>
__device__ __forceinline__ float2 group_sum(float a, float b, float2* red)
{
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, off);
        b += __shfl_xor_sync(0xffffffffu, b, off);
    }
    if constexpr (TPR > 32) {
        __syncthreads();                               // the previous sum has been read
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) {
            a += red[w].x;
            b += red[w].y;
        }
    }
    return make_float2(a, b);
}

template <typename T, int V, int TPR, int NV>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR)
    ln_fwd_kernel(long long rows, int d, const T* x, const T* __restrict__ gamma,
                  const T* __restrict__ beta, float eps, T* y, float* __restrict__ mean, float* __restrict__ rstd)
{
    __shared__ float2 red[TPR / 32];
    constexpr int kGroups = TPR < kLnThreads ? kLnThreads / TPR : 1;
    const int gt = threadIdx.x % TPR;                  // thread of the group
    const int pieces = d / V;
    const float inv_d = 1.0f / (float)d;
    const long long stride = (long long)gridDim.x * kGroups;
    // with TPR > 32 the CTA is one group, so the barriers in group_sum are uniform
    for (long long r = (long long)blockIdx.x * kGroups + threadIdx.x / TPR; r < rows; r += stride) {
        const T* xr = x + r * d;
        float v[NV][V];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces) load_piece<T, V>(xr + (size_t)c * V, v[i]);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] = 0.0f;
#pragma unroll
            for (int e = 0; e < V; ++e) s += v[i][e];
        }
        const float mu = group_sum<TPR>(s, 0.0f, red).x * inv_d;
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (gt + i * TPR < pieces) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float t = v[i][e] - mu;
                    q = fmaf(t, t, q);
                }
            }
        const float rs = 1.0f / sqrtf(group_sum<TPR>(q, 0.0f, red).x * inv_d + eps);
        if (mean && gt == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        T* yr = y + r * d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces) {
                float g[V], b[V];
                if (gamma) load_piece<T, V>(gamma + (size_t)c * V, g);
                if (beta) load_piece<T, V>(beta + (size_t)c * V, b);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float t = (v[i][e] - mu) * rs;
                    if (gamma) t *= g[e];
                    if (beta) t += b[e];
                    v[i][e] = t;
                }
                store_piece<T, V>(yr + (size_t)c * V, v[i]);
            }
        }
    }
}

// Rows too long for registers: one CTA per row, three passes over it (L2).
template <typename T>
__global__ void __launch_bounds__(512) ln_fwd_long_kernel(long long rows, int d, const T* x, const T* __restrict__ gamma,
                                                          const T* __restrict__ beta, float eps, T* y,
                                                          float* __restrict__ mean, float* __restrict__ rstd)
{
    __shared__ float2 red[16];
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + r * d;
        float s = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) s += to_float(xr[c]);
        const float mu = group_sum<512>(s, 0.0f, red).x / (float)d;
        float q = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) {
            const float t = to_float(xr[c]) - mu;
            q = fmaf(t, t, q);
        }
        const float rs = 1.0f / sqrtf(group_sum<512>(q, 0.0f, red).x / (float)d + eps);
        if (mean && threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        for (int c = threadIdx.x; c < d; c += 512) {
            float t = (to_float(xr[c]) - mu) * rs;
            if (gamma) t *= to_float(gamma[c]);
            if (beta) t += to_float(beta[c]);
            y[r * d + c] = from_float<T>(t);
        }
    }
}

template <typename T, int V, int TPR, int NV>
__global__ void __launch_bounds__(TPR < kLnThreads ? kLnThreads : TPR)
    ln_bwd_kernel(long long rows, int d, const T* __restrict__ x, const T* __restrict__ gamma,
                  const float* __restrict__ mean, const float* __restrict__ rstd, const T* dy, T* dx,
                  float* __restrict__ part)
{
    extern __shared__ float cols[];                    // [d] of a CTA's column sums, twice; TPR = 32 only
    __shared__ float2 red[TPR / 32];
    constexpr int kGroups = TPR < kLnThreads ? kLnThreads / TPR : 1;
    const int gt = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int pieces = d / V;
    const float inv_d = 1.0f / (float)d;
    float dg[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) dg[i][e] = db[i][e] = 0.0f;
    const long long stride = (long long)gridDim.x * kGroups;
    for (long long r = (long long)blockIdx.x * kGroups + group; r < rows; r += stride) {
        const T *xr = x + r * d, *dyr = dy + r * d;
        float xh[NV][V], a[NV][V];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces) {
                load_piece<T, V>(xr + (size_t)c * V, xh[i]);
                load_piece<T, V>(dyr + (size_t)c * V, a[i]);
            }
        }
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces) {
                float g[V];
                if (gamma) load_piece<T, V>(gamma + (size_t)c * V, g);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    xh[i][e] = (xh[i][e] - mu) * rs;
                    dg[i][e] = fmaf(a[i][e], xh[i][e], dg[i][e]);
                    db[i][e] += a[i][e];
                    if (gamma) a[i][e] *= g[e];
                    s1 += a[i][e];
                    s2 = fmaf(a[i][e], xh[i][e], s2);
                }
            }
        }
        const float2 m = group_sum<TPR>(s1, s2, red);
        const float m1 = m.x * inv_d, m2 = m.y * inv_d;
        T* dxr = dx + r * d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces) {
#pragma unroll
                for (int e = 0; e < V; ++e) a[i][e] = rs * (a[i][e] - m1 - xh[i][e] * m2);
                store_piece<T, V>(dxr + (size_t)c * V, a[i]);
            }
        }
    }
    if (!part) return;
    float* pg = part + (size_t)blockIdx.x * 2 * d;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * TPR;
            if (c < pieces)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    pg[(size_t)c * V + e] = dg[i][e];
                    pg[d + (size_t)c * V + e] = db[i][e];
                }
        }
    } else {
        for (int g = 0; g < kGroups; ++g) {            // in group order: the same bits every time
            if (group == g) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = gt + i * TPR;
                    if (c < pieces)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            float *qg = cols + c * V + e, *qb = qg + d;
                            *qg = g == 0 ? dg[i][e] : *qg + dg[i][e];
                            *qb = g == 0 ? db[i][e] : *qb + db[i][e];
                        }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * d; c += kLnThreads) pg[c] = cols[c];
    }
}

// Rows too long for registers: dx, one CTA per row.
template <typename T>
__global__ void __launch_bounds__(512) ln_bwd_long_kernel(long long rows, int d, const T* __restrict__ x,
                                                          const T* __restrict__ gamma, const float* __restrict__ mean,
                                                          const float* __restrict__ rstd, const T* dy, T* dx)
{
    __shared__ float2 red[16];
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) {
            float a = to_float(dy[r * d + c]);
            if (gamma) a *= to_float(gamma[c]);
            s1 += a;
            s2 = fmaf(a, (to_float(x[r * d + c]) - mu) * rs, s2);
        }
        const float2 m = group_sum<512>(s1, s2, red);
        for (int c = threadIdx.x; c < d; c += 512) {
            float a = to_float(dy[r * d + c]);
            if (gamma) a *= to_float(gamma[c]);
            dx[r * d + c] = from_float<T>(rs * (a - m.x / (float)d - (to_float(x[r * d + c]) - mu) * rs * (m.y / (float)d)));
        }
    }
}
// ... and its column sums over the rows [g n / G, (g + 1) n / G) of grid row g; before dx, which may be dy.
template <typename T>
__global__ void __launch_bounds__(128) ln_bwd_long_cols_kernel(long long rows, int d, const T* __restrict__ x,
                                                               const float* __restrict__ mean,
                                                               const float* __restrict__ rstd, const T* __restrict__ dy,
                                                               float* __restrict__ part)
{
    const int c = blockIdx.x * 128 + threadIdx.x;
    if (c >= d) return;
    const long long r0 = rows * blockIdx.y / gridDim.y, r1 = rows * (blockIdx.y + 1) / gridDim.y;
    float dg = 0.0f, db = 0.0f;
    for (long long r = r0; r < r1; ++r) {
        const float a = to_float(dy[r * d + c]);
        dg = fmaf(a, (to_float(x[r * d + c]) - mean[r]) * rstd[r], dg);
        db += a;
    }
    part[(size_t)blockIdx.y * 2 * d + c] = dg;
    part[(size_t)blockIdx.y * 2 * d + d + c] = db;
}

// dgamma / dbeta = the sum of the n partial rows [n][2 d].  A CTA takes 32
// columns; its 8 warps add every eighth partial row, then the warps' sums meet
// in warp order.
__global__ void __launch_bounds__(256) ln_bwd_reduce_kernel(int n, int d, const float* __restrict__ part,
                                                            float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float a = 0.0f;
    if (c < 2 * d)
        for (int i = w; i < n; i += 8) a += part[(size_t)i * 2 * d + c];
    s[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < 2 * d) {
#pragma unroll
        for (int i = 1; i < 8; ++i) a += s[i][lane];
        if (c < d) dgamma[c] = a;
        else dbeta[c - d] = a;
    }
}

// ---------------------------------------------------------------- dispatch

constexpr int kFwdMax = 20;              // pieces a thread holds forward (x)
constexpr int kMaxPartials = 1216;       // partial rows of dgamma, dbeta: 8 CTAs on each of 152 SMs

bool wide(int d, int esz, const void* a, const void* b, const void* c, const void* e)
{
    const uintptr_t bits = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) |
                           reinterpret_cast<uintptr_t>(c) | reinterpret_cast<uintptr_t>(e);
    return (int64_t)d * esz % 16 == 0 && (bits & 15u) == 0;
}

cudaError_t sm_count(int* n)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
}

struct LnArgs {
    long long rows;
    int d;
    const void *x, *gamma, *beta, *dy;
    float eps;
    void* y;                 // dx of the backward
    float *mean, *rstd, *part;
    int nsm, grid;           // grid: CTAs of the backward, 0 forward
    cudaStream_t st;
};

template <typename T, int V, int TPR, int NV>
cudaError_t fwd_one(const LnArgs& a)
{
    constexpr int kThreads = TPR < kLnThreads ? kLnThreads : TPR, kGroups = kThreads / TPR;
    const long long want = (a.rows + kGroups - 1) / kGroups, cap = (long long)a.nsm * 16;
    ln_fwd_kernel<T, V, TPR, NV><<<(int)(want < cap ? want : cap), kThreads, 0, a.st>>>(
        a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma), static_cast<const T*>(a.beta), a.eps,
        static_cast<T*>(a.y), a.mean, a.rstd);
    return cudaGetLastError();
}
template <typename T, int V, int TPR, int NV>
cudaError_t bwd_one(const LnArgs& a)
{
    constexpr int kThreads = TPR < kLnThreads ? kLnThreads : TPR;
    const size_t smem = TPR < kLnThreads && a.part ? sizeof(float) * 2 * a.d : 0;
    ln_bwd_kernel<T, V, TPR, NV><<<a.grid, kThreads, smem, a.st>>>(
        a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma), a.mean, a.rstd,
        static_cast<const T*>(a.dy), static_cast<T*>(a.y), a.part);
    return cudaGetLastError();
}

// The instantiation whose TPR x NV pieces hold the row: NV is rounded up along this list.
template <typename T, int V, int TPR>
cudaError_t fwd_nv(const LnArgs& a, int nv)
{
    if (nv <= 1) return fwd_one<T, V, TPR, 1>(a);
    if (nv <= 2) return fwd_one<T, V, TPR, 2>(a);
    if (nv <= 4) return fwd_one<T, V, TPR, 4>(a);
    if (nv <= 6) return fwd_one<T, V, TPR, 6>(a);
    if (nv <= 10) return fwd_one<T, V, TPR, 10>(a);
    return fwd_one<T, V, TPR, kFwdMax>(a);
}
template <typename T, int V, int TPR, int MAX>
cudaError_t bwd_nv(const LnArgs& a, int nv)
{
    if (nv <= 1) return bwd_one<T, V, TPR, 1>(a);
    if (nv <= 2) return bwd_one<T, V, TPR, 2>(a);
    if (nv <= 4) return bwd_one<T, V, TPR, 4>(a);
    if constexpr (MAX > 6)
        if (nv > 6) return bwd_one<T, V, TPR, MAX>(a);
    return bwd_one<T, V, TPR, 6>(a);
}

template <typename T, int V>
cudaError_t fwd(const LnArgs& a)
{
    const int pieces = a.d / V;
    auto nv = [&](int tpr) { return (pieces + tpr - 1) / tpr; };
    if (nv(32) <= kFwdMax) return fwd_nv<T, V, 32>(a, nv(32));
    if (nv(128) <= kFwdMax) return fwd_nv<T, V, 128>(a, nv(128));
    if (nv(512) <= kFwdMax) return fwd_nv<T, V, 512>(a, nv(512));
    const long long cap = (long long)a.nsm * 4;
    ln_fwd_long_kernel<T><<<(int)(a.rows < cap ? a.rows : cap), 512, 0, a.st>>>(
        a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma), static_cast<const T*>(a.beta), a.eps,
        static_cast<T*>(a.y), a.mean, a.rstd);
    return cudaGetLastError();
}

template <int V>
constexpr int bwd_max()                  // pieces a thread holds backward (x, dy and two column sums)
{
    return V == 1 ? 16 : 6;
}
template <typename T, int V>
cudaError_t bwd(const LnArgs& a)
{
    constexpr int MAX = bwd_max<V>();
    const int pieces = a.d / V;
    auto nv = [&](int tpr) { return (pieces + tpr - 1) / tpr; };
    if (nv(32) <= MAX) return bwd_nv<T, V, 32, MAX>(a, nv(32));
    if (nv(128) <= MAX) return bwd_nv<T, V, 128, MAX>(a, nv(128));
    if (nv(512) <= MAX) return bwd_nv<T, V, 512, MAX>(a, nv(512));
    if (a.part) {
        const dim3 grid((a.d + 127) / 128, a.grid);
        ln_bwd_long_cols_kernel<T><<<grid, 128, 0, a.st>>>(a.rows, a.d, static_cast<const T*>(a.x), a.mean, a.rstd,
                                                           static_cast<const T*>(a.dy), a.part);
    }
    const long long cap = (long long)a.nsm * 4;
    ln_bwd_long_kernel<T><<<(int)(a.rows < cap ? a.rows : cap), 512, 0, a.st>>>(
        a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma), a.mean, a.rstd,
        static_cast<const T*>(a.dy), static_cast<T*>(a.y));
    return cudaGetLastError();
}

// CTAs of the backward: at most 8 on each SM, and no more than the rows fill with two rows per group,
// so that a partial row stands for several rows of the sum.
int bwd_grid(long long rows)
{
    const long long want = (rows + 7) / 8;
    return (int)(want < kMaxPartials ? want : kMaxPartials);
}

}  // namespace

size_t layer_norm_backward_scratch(long long rows, int d) { return sizeof(float) * 2 * (size_t)d * bwd_grid(rows); }

cudaError_t launch_layer_norm(rola_dtype_t dt, long long rows, int d, const void* x, const void* gamma,
                              const void* beta, float eps, void* y, float* mean, float* rstd, cudaStream_t st)
{
    LnArgs a{rows, d, x, gamma, beta, nullptr, eps, y, mean, rstd, nullptr, 0, 0, st};
    cudaError_t e = sm_count(&a.nsm);
    if (e != cudaSuccess) return e;
    if (dt == ROLA_BF16)
        return wide(d, 2, x, gamma, beta, y) ? fwd<__nv_bfloat16, 8>(a) : fwd<__nv_bfloat16, 1>(a);
    return wide(d, 4, x, gamma, beta, y) ? fwd<float, 4>(a) : fwd<float, 1>(a);
}

cudaError_t launch_layer_norm_backward(rola_dtype_t dt, long long rows, int d, const void* x, const void* gamma,
                                       const float* mean, const float* rstd, const void* dy, void* dx, float* dgamma,
                                       float* dbeta, float* part, cudaStream_t st)
{
    LnArgs a{rows, d, x, gamma, nullptr, dy, 0.0f, dx, const_cast<float*>(mean), const_cast<float*>(rstd),
             dgamma ? part : nullptr, 0, bwd_grid(rows), st};
    cudaError_t e = sm_count(&a.nsm);
    if (e != cudaSuccess) return e;
    if (dt == ROLA_BF16)
        e = wide(d, 2, x, gamma, dy, dx) ? bwd<__nv_bfloat16, 8>(a) : bwd<__nv_bfloat16, 1>(a);
    else
        e = wide(d, 4, x, gamma, dy, dx) ? bwd<float, 4>(a) : bwd<float, 1>(a);
    if (e != cudaSuccess || !dgamma) return e;
    ln_bwd_reduce_kernel<<<(2 * d + 31) / 32, 256, 0, st>>>(a.grid, d, part, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace rola
