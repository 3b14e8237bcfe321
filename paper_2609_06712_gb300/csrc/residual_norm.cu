// The gated residual sum of a block and its norms, and their gradients (formulas: include/rola.h).
//
//   hh = norm_b(h) or h,  u = x + gate gamma_h hh,  v = norm(u),  y = v g + c
//   with g = gamma (1 + scale), c = beta (1 + scale) + shift
//   a = dy g,  t = dout + rstd (a [- mean a] - v mean(a v)),  dx = t
//   e = t gate gamma_h,  dh = rstd_h (e [- mean e] - hh mean(e hh)) or e
//   column sums of each sample: A = sum dy v, B = sum dy, E = sum t hh; every vector's gradient is made of them.
#include "norm_rows.cuh"
#include "residual_norm.cuh"

namespace rola {
namespace {

// Element c of a vector of sample s, or `none`.
template <typename T>
__device__ __forceinline__ float vec(const void* p, size_t c, float none)
{
    return p ? to_float(static_cast<const T*>(p)[c]) : none;
}
// What the formulas above call g, c and gate gamma_h, of column c of sample s.
template <typename T>
__device__ __forceinline__ float gain_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return vec<T>(a.gamma, c, 1.0f) * (1.0f + vec<T>(a.scale, s * sh.mod_stride + c, 0.0f));
}
template <typename T>
__device__ __forceinline__ float shift_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return fmaf(vec<T>(a.beta, c, 0.0f), 1.0f + vec<T>(a.scale, s * sh.mod_stride + c, 0.0f),
                vec<T>(a.shift, s * sh.mod_stride + c, 0.0f));
}
template <typename T>
__device__ __forceinline__ float branch_gain_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return vec<T>(a.gate, s * sh.mod_stride + c, 1.0f) * vec<T>(a.gamma_h, c, 1.0f);
}

// ---------------------------------------------------------------- rows of any length, from memory

constexpr int kLongThreads = 512;

// Mean (0 for the RMS norm) and 1 / size of n values f(c), in two passes.
template <typename F>
__device__ __forceinline__ float2 row_stats(int kind, int d, float eps, float2 (*red)[32], int& turn, F f)
{
    float mu = 0.0f;
    if (kind == ROLA_NORM_LAYER) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < d; c += kLongThreads) s += f(c);
        mu = group_sum<false>(s, 0.0f, red, turn).x / (float)d;
    }
    float q = 0.0f;
    for (int c = threadIdx.x; c < d; c += kLongThreads) {
        const float t = f(c) - mu;
        q = fmaf(t, t, q);
    }
    return make_float2(mu, 1.0f / sqrtf(group_sum<false>(q, 0.0f, red, turn).x / (float)d + eps));
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_fwd_long_kernel(const RnShape sh, const RnArgs a)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const T *x = static_cast<const T*>(a.x) + r * sh.d, *h = a.h ? static_cast<const T*>(a.h) + r * sh.d : nullptr;
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float2 hs = make_float2(0.0f, 1.0f), us = make_float2(0.0f, 1.0f);
        if (h && sh.branch != ROLA_NORM_NONE) {
            hs = row_stats(sh.branch, sh.d, sh.eps, red, turn, [&](int c) { return to_float(h[c]); });
            st.z = hs.x;
            st.w = hs.y;
        }
        auto sum = [&](int c) {
            const float u = to_float(x[c]);
            return h ? fmaf(branch_gain_of<T>(sh, a, s, c), (to_float(h[c]) - hs.x) * hs.y, u) : u;
        };
        if (sh.norm != ROLA_NORM_NONE) {
            us = row_stats(sh.norm, sh.d, sh.eps, red, turn, sum);
            st.x = us.x;
            st.y = us.y;
        }
        for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
            const float u = sum(c);                       // read before the writes: out and y may be x or h
            if (a.out) static_cast<T*>(a.out)[r * sh.d + c] = from_float<T>(u);
            if (a.y)
                static_cast<T*>(a.y)[r * sh.d + c] =
                    from_float<T>(fmaf((u - us.x) * us.y, gain_of<T>(sh, a, s, c), shift_of<T>(sh, a, s, c)));
        }
        if (a.stats && threadIdx.x == 0) reinterpret_cast<float4*>(a.stats)[r] = st;
    }
}

// The values of one element of the backward: hh, v, and t given the row's means.
template <typename T>
struct Element {
    float hh, v, dy, t, gg;
    __device__ __forceinline__ Element(const RnShape& sh, const RnArgs& a, int s, long long r, int c, float4 st, float m1,
                                       float m2)
    {
        const size_t at = (size_t)(r * sh.d + c);
        hh = a.h ? to_float(static_cast<const T*>(a.h)[at]) : 0.0f;
        if (sh.branch != ROLA_NORM_NONE) hh = (hh - st.z) * st.w;
        gg = branch_gain_of<T>(sh, a, s, c);
        t = a.dout ? to_float(static_cast<const T*>(a.dout)[at]) : 0.0f;
        v = dy = 0.0f;
        if (sh.norm != ROLA_NORM_NONE) {
            v = (fmaf(gg, hh, to_float(static_cast<const T*>(a.x)[at])) - st.x) * st.y;
            dy = to_float(static_cast<const T*>(a.dy)[at]);
            t = fmaf(st.y, dy * gain_of<T>(sh, a, s, c) - m1 - v * m2, t);
        }
    }
};

// mean a, mean(a v), mean e and mean(e hh) of each row (the first and third 0 for the RMS norm).
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_moments_kernel(const RnShape sh, const RnArgs a)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    const float inv_d = 1.0f / (float)sh.d;
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const float4 st = reinterpret_cast<const float4*>(a.stats)[r];
        float4 m = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (sh.norm != ROLA_NORM_NONE) {
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
                const Element<T> e(sh, a, s, r, c, st, 0.0f, 0.0f);
                const float av = e.dy * gain_of<T>(sh, a, s, c);
                s1 += av;
                s2 = fmaf(av, e.v, s2);
            }
            const float2 q = group_sum<false>(s1, s2, red, turn);
            m.x = sh.norm == ROLA_NORM_LAYER ? q.x * inv_d : 0.0f;
            m.y = q.y * inv_d;
        }
        if (sh.branch != ROLA_NORM_NONE) {
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
                const Element<T> e(sh, a, s, r, c, st, m.x, m.y);
                s1 = fmaf(e.t, e.gg, s1);
                s2 = fmaf(e.t * e.gg, e.hh, s2);
            }
            const float2 q = group_sum<false>(s1, s2, red, turn);
            m.z = sh.branch == ROLA_NORM_LAYER ? q.x * inv_d : 0.0f;
            m.w = q.y * inv_d;
        }
        if (threadIdx.x == 0) a.moments[r] = m;
    }
}
// Column sums of part blockIdx.y; before dx and dh, which may take the place of dout and dy.
template <typename T>
__global__ void __launch_bounds__(128) rn_columns_kernel(const RnShape sh, const RnArgs a)
{
    const int c = blockIdx.x * 128 + threadIdx.x, part = blockIdx.y;
    if (c >= sh.d) return;
    const long long r1 = rn_row(sh.total, a.parts, part + 1);
    float A = 0.0f, B = 0.0f, E = 0.0f;
    for (long long r = rn_row(sh.total, a.parts, part); r < r1; ++r) {
        const int s = (int)(r / sh.rows);
        const float4 m = a.moments[r];
        const Element<T> e(sh, a, s, r, c, reinterpret_cast<const float4*>(a.stats)[r], m.x, m.y);
        A = fmaf(e.dy, e.v, A);
        B += e.dy;
        E = fmaf(e.t, e.hh, E);
        if (r + 1 == r1 || (r + 1) % sh.rows == 0) {
            float* out = a.part + (size_t)(part + s) * 3 * sh.d + c;
            out[0] = A;
            out[sh.d] = B;
            out[2 * (size_t)sh.d] = E;
            A = B = E = 0.0f;
        }
    }
}
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_bwd_long_kernel(const RnShape sh, const RnArgs a)
{
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const float4 st = reinterpret_cast<const float4*>(a.stats)[r], m = a.moments[r];
        for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
            const Element<T> e(sh, a, s, r, c, st, m.x, m.y);
            static_cast<T*>(a.dx)[r * sh.d + c] = from_float<T>(e.t);
            if (!a.dh) continue;
            float dh = e.t * e.gg;
            if (sh.branch != ROLA_NORM_NONE) dh = st.w * (dh - m.z - e.hh * m.w);
            static_cast<T*>(a.dh)[r * sh.d + c] = from_float<T>(dh);
        }
    }
}

// ---------------------------------------------------------------- column sums to gradients

// The vectors' gradients from the parts' sums.  A CTA takes 32 columns; its 32 warps share the samples, 32 / ways of
// them at a time, `ways` warps to a sample, which add every ways-th of its slots.  The warps' sums meet in warp order,
// the samples' in sample order within a warp, then in warp order: the same bits every time.
template <typename T>
__global__ void __launch_bounds__(1024) rn_reduce_kernel(const RnShape sh, const RnArgs a, int ways)
{
    __shared__ float sum[3][32][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    const int at_once = 32 / ways, way = w % ways;
    const bool in = c < sh.d;
    float dgamma = 0.0f, dbeta = 0.0f, dgamma_h = 0.0f;
    const float gamma = in ? vec<T>(a.gamma, c, 1.0f) : 0.0f, beta = in ? vec<T>(a.beta, c, 0.0f) : 0.0f;
    const float gamma_h = in ? vec<T>(a.gamma_h, c, 1.0f) : 0.0f;
    for (int s0 = 0; s0 < sh.groups; s0 += at_once) {
        const int s = s0 + w / ways;
        float A = 0.0f, B = 0.0f, E = 0.0f;
        if (s < sh.groups && in) {
            const int lo = rn_part(sh.total, a.parts, (long long)s * sh.rows);
            const int hi = rn_part(sh.total, a.parts, (long long)(s + 1) * sh.rows - 1);
#pragma unroll 4
            for (int i = lo + way; i <= hi; i += ways) {
                const float* p = a.part + (size_t)(i + s) * 3 * sh.d + c;
                A += p[0];
                B += p[sh.d];
                E += p[2 * (size_t)sh.d];
            }
        }
        if (ways > 1) {
            __syncthreads();                             // the last samples' sums have been read
            sum[0][w][lane] = A;
            sum[1][w][lane] = B;
            sum[2][w][lane] = E;
            __syncthreads();
            if (way == 0)
                for (int i = 1; i < ways; ++i) {
                    A += sum[0][w + i][lane];
                    B += sum[1][w + i][lane];
                    E += sum[2][w + i][lane];
                }
        }
        if (way == 0 && s < sh.groups && in) {
            const size_t at = (size_t)s * sh.d + c, mod = (size_t)(s * sh.mod_stride + c);
            if (a.dscale) a.dscale[at] = fmaf(gamma, A, beta * B);
            if (a.dshift) a.dshift[at] = B;
            if (a.dgate) a.dgate[at] = gamma_h * E;
            const float s1 = 1.0f + vec<T>(a.scale, mod, 0.0f);
            dgamma = fmaf(s1, A, dgamma);
            dbeta = fmaf(s1, B, dbeta);
            dgamma_h = fmaf(vec<T>(a.gate, mod, 1.0f), E, dgamma_h);
        }
    }
    if (!a.dgamma && !a.dbeta && !a.dgamma_h) return;
    __syncthreads();
    sum[0][w][lane] = dgamma;
    sum[1][w][lane] = dbeta;
    sum[2][w][lane] = dgamma_h;
    __syncthreads();
    if (w < 3 && in) {                                   // warps whose way is not 0 hold zeros
        float total = 0.0f;
        for (int i = 0; i < 32; i += ways) total += sum[w][i][lane];
        float* out = w == 0 ? a.dgamma : w == 1 ? a.dbeta : a.dgamma_h;
        if (out) out[c] = total;
    }
}

// ---------------------------------------------------------------- dispatch

int long_grid(long long rows) { return (int)(rows < 608 ? rows : 608); }     // four CTAs on each of 152 SMs

bool wants_sums(const RnArgs& a) { return a.dgate || a.dgamma_h || a.dgamma || a.dbeta || a.dscale || a.dshift; }

template <typename T>
cudaError_t backward(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    a.parts = rn_parts(s);
    rn_moments_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    if (wants_sums(a)) rn_columns_kernel<T><<<dim3((s.d + 127) / 128, a.parts), 128, 0, st>>>(s, a);
    rn_bwd_long_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    if (wants_sums(a)) {
        int ways = 32;
        while (ways > 1 && ways * s.groups > 32) ways /= 2;
        rn_reduce_kernel<T><<<(s.d + 31) / 32, 1024, 0, st>>>(s, a, ways);
    }
    return cudaGetLastError();
}

}  // namespace

int rn_parts(const RnShape& s)
{
    const long long want = (s.total + 1) / 2;
    return (int)(want < 1216 ? want : 1216);
}

bool rn_long(const RnShape&) { return true; }

cudaError_t launch_residual_norm(rola_dtype_t dt, const RnShape& s, const RnArgs& a, cudaStream_t st)
{
    const int grid = long_grid(s.total);
    if (dt == ROLA_BF16) rn_fwd_long_kernel<__nv_bfloat16><<<grid, kLongThreads, 0, st>>>(s, a);
    else rn_fwd_long_kernel<float><<<grid, kLongThreads, 0, st>>>(s, a);
    return cudaGetLastError();
}

cudaError_t launch_residual_norm_backward(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st)
{
    return dt == ROLA_BF16 ? backward<__nv_bfloat16>(s, a, st) : backward<float>(s, a, st);
}

}  // namespace rola
