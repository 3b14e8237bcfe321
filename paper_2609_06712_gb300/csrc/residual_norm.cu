// The gated residual sum of a block and its norms, and their gradients (formulas: include/rola.h).
//
//   hh = norm_b(h) or h,  u = x + gate gamma_h hh,  v = norm(u),  y = v g + c
//   with g = gamma (1 + scale), c = beta (1 + scale) + shift
//   a = dy g,  t = dout + rstd (a [- mean a] - v mean(a v)),  dx = t
//   e = t gate gamma_h,  dh = rstd_h (e [- mean e] - hh mean(e hh)) or e
//   column sums of each sample: A = sum dy v, B = sum dy, E = sum t hh; every vector's gradient is made of them.
#include "norm_rows.cuh"
#include "residual_norm.cuh"
#include "tcgen05.cuh"

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

// ---------------------------------------------------------------- rows in registers

constexpr int kWarpGroups = 4;                       // rows of a CTA whose rows have a warp each
constexpr int kMaxDepth = 16;                        // rows in a group's ring
constexpr size_t kRingBytes = 208 << 10;             // of the rings of an SM's CTAs
constexpr size_t kBarBytes = kWarpGroups * kMaxDepth * 8;
constexpr uint64_t kWaitLimitNs = 2000000000ull;     // bound of the wait for a row

// Bytes of a row's place in the ring: a row that starts anywhere is copied with the 16-byte words that it begins and
// ends in.
__host__ __device__ __forceinline__ uint32_t place_bytes(int d, int esz, bool wide)
{
    return wide ? (uint32_t)(d * esz) : (uint32_t)((d * esz + 15) / 16 * 16 + 16);
}

// A group's rows [next, end) of the matrices a.in (those that are not NULL), brought ahead into `depth` slots of shared
// memory by bulk copies, one per matrix, with an mbarrier a slot.  A slot is refilled after its row has been read into
// registers by the whole group.  V = 1: rows that start at any element; they are copied with the whole 16-byte words that
// they begin and end in, and where such a word is not all inside the matrix (its first and last row) element by element.
template <typename T, int V, int NV, int N>
struct Feed {
    long long next, end;
    int tpr, gt, depth, slot, phase;
    uint32_t ring, bars;

    static __device__ __forceinline__ uint32_t place(const RnShape& sh) { return place_bytes(sh.d, sizeof(T), V > 1); }
    static __device__ __forceinline__ int count(const RnArgs& a)
    {
        int k = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) k += a.in[n] != nullptr;
        return k;
    }
    // Bytes from a 16-byte word's begin to row r of matrix n.
    static __device__ __forceinline__ uint32_t offset(const RnShape& sh, const RnArgs& a, int n, long long r)
    {
        if constexpr (V > 1) return 0;
        else return (uint32_t)(reinterpret_cast<uintptr_t>(a.in[n]) + (unsigned long long)r * (sh.d * sizeof(T))) & 15u;
    }
    // Of the words that row r lies in, from its first, bytes [lo, hi) are copied: those of words inside the matrix.
    static __device__ __forceinline__ void span(const RnShape& sh, long long r, uint32_t from, uint32_t& lo, uint32_t& hi)
    {
        const uint32_t row = sh.d * (uint32_t)sizeof(T);
        lo = (unsigned long long)r * row < from ? 16u : 0u;
        hi = (from + row + 15u) & ~15u;
        if ((unsigned long long)(sh.total - r) * row < hi - from) hi -= 16u;
        if (hi < lo) hi = lo;
    }
    __device__ __forceinline__ void copy(const RnShape& sh, const RnArgs& a, int to)         // one thread
    {
        const uint32_t bar = bars + to * 8, step = place(sh);
        uint32_t at = ring + to * count(a) * step, bytes = count(a) * step;
        if constexpr (V == 1) {
            bytes = 0;
            uint32_t p = at;
#pragma unroll 1
            for (int n = 0; n < N; ++n)
                if (a.in[n]) {
                    const uint32_t from = offset(sh, a, n, next), row = sh.d * (uint32_t)sizeof(T);
                    uint32_t lo, hi;
                    span(sh, next, from, lo, hi);
                    bytes += hi - lo;
                    // elements outside [lo, hi): at most 15 bytes at each end
                    const T* src = static_cast<const T*>(a.in[n]) + next * sh.d;
                    for (uint32_t w = from; w < from + row; w += sizeof(T)) {
                        if (w >= lo && w < hi) {
                            w = hi - sizeof(T);          // on to the first element behind
                            continue;
                        }
                        const T x = src[(w - from) / sizeof(T)];
                        if constexpr (sizeof(T) == 4)
                            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(p + w), "f"(to_float(x)) : "memory");
                        else
                            asm volatile("st.shared.u16 [%0], %1;\n" ::"r"(p + w), "h"(*reinterpret_cast<const uint16_t*>(&x)) : "memory");
                    }
                    p += step;
                }
        }
        tc::mbar_expect_tx(bar, bytes);                  // arrives behind the elements stored above
#pragma unroll 1
        for (int n = 0; n < N; ++n)
            if (a.in[n]) {
                uint32_t from = 0, lo = 0, hi = step;
                if constexpr (V == 1) {
                    from = offset(sh, a, n, next);
                    span(sh, next, from, lo, hi);
                }
                if (hi > lo)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(
                                     at + lo),
                                 "l"(reinterpret_cast<uintptr_t>(static_cast<const T*>(a.in[n]) + next * sh.d) - from + lo),
                                 "r"(hi - lo), "r"(bar)
                                 : "memory");
                at += step;
            }
        ++next;
    }
    // rows [r0, end) of the group; smem: the groups' mbarriers, then their rings
    __device__ __forceinline__ void start(const RnShape& sh, const RnArgs& a, unsigned char* smem, int group, long long r0)
    {
        bars = smem_u32(smem) + group * kMaxDepth * 8;
        ring = smem_u32(smem) + (uint32_t)kBarBytes + (uint32_t)(group * depth * count(a)) * place(sh);
        next = r0;
        slot = phase = 0;
        if (gt == 0) {
            for (int i = 0; i < depth; ++i) tc::mbar_init(bars + i * 8, 1);
            tc::fence_mbar_init();
#pragma unroll 1
            for (int i = 0; i < depth && next < end; ++i) copy(sh, a, i);
        }
    }
    __device__ __forceinline__ bool wait() const
    {
        int never = 0;
        return tc::mbar_wait(bars + slot * 8, phase, &never, kWaitLimitNs);
    }
    // Row r of matrix n (k-th of those there) as fp32, zeros where there is none; NaN where its copy never arrived (the
    // call has no status word).
    __device__ __forceinline__ void read(const RnShape& sh, const RnArgs& a, int n, int k, long long r, bool ok,
                                         float (&v)[NV][V]) const
    {
        const int pieces = sh.d / V;
        const uint32_t at = ring + (uint32_t)(slot * count(a) + k) * place(sh) + offset(sh, a, n, r);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gt + i * tpr;
            if (a.in[n] && c < pieces) {
                if constexpr (V > 1) {
                    Piece<T, V> x;
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
                                 : "=r"(x.w.x), "=r"(x.w.y), "=r"(x.w.z), "=r"(x.w.w)
                                 : "r"(at + c * 16)
                                 : "memory");
                    unpack<T, V>(x, v[i]);
                } else if constexpr (sizeof(T) == 4) {
                    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v[i][0]) : "r"(at + c * 4) : "memory");
                } else {
                    uint16_t b;
                    asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(b) : "r"(at + c * 2) : "memory");
                    v[i][0] = __uint_as_float((uint32_t)b << 16);
                }
                if (!ok) v[i][0] = __int_as_float(0x7fc00000);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) v[i][e] = 0.0f;
            }
        }
    }
    __device__ __forceinline__ void refill(const RnShape& sh, const RnArgs& a)       // after every thread of the group has read
    {
        if (gt == 0 && next < end) copy(sh, a, slot);
        if (++slot == depth) {
            slot = 0;
            phase ^= 1;
        }
    }
};

template <bool WARP>
__device__ __forceinline__ void group_sync()
{
    if constexpr (WARP) __syncwarp();
    else __syncthreads();
}

// A piece of a vector, or `none` everywhere.
template <typename T, int V>
__device__ __forceinline__ void vec_piece(const void* p, size_t at, float none, float (&v)[V])
{
    if (p) {
        unpack<T, V>(load_piece<T, V>(static_cast<const T*>(p) + at), v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = none;
    }
}

// g, c and gate gamma_h of sample s for this thread's pieces.
template <typename T, int V, int NV, bool SHIFT>
__device__ __forceinline__ void load_vectors(const RnShape& sh, const RnArgs& a, int s, int gt, int tpr, int pieces,
                                             float (&g)[NV][V], float (&c)[NV][V], float (&b)[NV][V])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = gt + i * tpr;
        if (p >= pieces) {
#pragma unroll
            for (int e = 0; e < V; ++e) g[i][e] = c[i][e] = b[i][e] = 0.0f;
            continue;
        }
        const size_t at = (size_t)p * V, mod = (size_t)(s * sh.mod_stride) + at;
        float s1[V], w[V];
        vec_piece<T, V>(a.scale, mod, 0.0f, s1);
        vec_piece<T, V>(a.gamma, at, 1.0f, g[i]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s1[e] += 1.0f;
            g[i][e] *= s1[e];
        }
        if constexpr (SHIFT) {
            vec_piece<T, V>(a.beta, at, 0.0f, w);
            vec_piece<T, V>(a.shift, mod, 0.0f, c[i]);
#pragma unroll
            for (int e = 0; e < V; ++e) c[i][e] = fmaf(w[e], s1[e], c[i][e]);
        }
        vec_piece<T, V>(a.gate, mod, 1.0f, b[i]);
        vec_piece<T, V>(a.gamma_h, at, 1.0f, w);
#pragma unroll
        for (int e = 0; e < V; ++e) b[i][e] *= w[e];
    }
}

// v = normalised v; returns (mean, 1 / size).  `first` runs after the first barrier: every thread of the group has
// read its pieces.
template <bool WARP, int V, int NV, typename F>
__device__ __forceinline__ float2 normalise(int kind, int d, float eps, int gt, int tpr, int pieces, float (&v)[NV][V],
                                            float2 (*red)[32], int& turn, F first)
{
    float mu = 0.0f;
    if (kind == ROLA_NORM_LAYER) {
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) sum_piece<V>(s, v[i]);
        mu = group_sum<WARP>(s[0] + s[1], 0.0f, red, turn).x / (float)d;
        first();
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (gt + i * tpr < pieces) fma_piece<V>(v[i], v[i], 1.0f, -mu);
    }
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i) dot_piece<V>(q, v[i], v[i]);
    const float r = 1.0f / sqrtf(group_sum<WARP>(q[0] + q[1], 0.0f, red, turn).x / (float)d + eps);
    if (kind != ROLA_NORM_LAYER) first();
#pragma unroll
    for (int i = 0; i < NV; ++i) fma_piece<V>(v[i], v[i], r, 0.0f);
    return make_float2(mu, r);
}

template <typename T, int V, int EL, bool WARP, int TH, int MIN>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : TH, MIN)
    rn_fwd_kernel(const __grid_constant__ RnShape sh, const __grid_constant__ RnArgs a, int depth)
{
    constexpr int NV = EL / V;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float2 red[2][32];
    int turn = 0;
    const int group = WARP ? threadIdx.x >> 5 : 0, part = WARP ? blockIdx.x * kWarpGroups + group : blockIdx.x;
    if (part >= a.parts) return;                         // a whole warp: no barrier of the CTA follows
    Feed<T, V, NV, 2> q;
    q.tpr = WARP ? 32 : blockDim.x;
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.depth = depth;
    q.end = rn_row(sh.total, a.parts, part + 1);
    long long r = rn_row(sh.total, a.parts, part);
    const int pieces = sh.d / V;
    q.start(sh, a, smem, group, r);
    group_sync<WARP>();                                  // the mbarriers are there
#pragma unroll 1
    for (int s = (int)(r / sh.rows); r < q.end; ++s) {   // the part's samples, and their rows
        const long long stop = min(q.end, (long long)(s + 1) * sh.rows);
        float g[NV][V], c[NV][V], b[NV][V];
        load_vectors<T, V, NV, true>(sh, a, s, q.gt, q.tpr, pieces, g, c, b);
#pragma unroll 1
        for (; r < stop; ++r) {
            const bool ok = q.wait();
            float u[NV][V], hh[NV][V];
            q.read(sh, a, 0, 0, r, ok, u);
            q.read(sh, a, 1, 1, r, ok, hh);
            bool held = true;
            auto refill = [&]() {
                if (!held) return;
                held = false;
                if constexpr (WARP) __syncwarp();
                q.refill(sh, a);
            };
            float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (a.h) {
                if (sh.branch != ROLA_NORM_NONE) {
                    const float2 m = normalise<WARP, V, NV>(sh.branch, sh.d, sh.eps, q.gt, q.tpr, pieces, hh, red, turn, refill);
                    st.z = m.x;
                    st.w = m.y;
                }
                T* out = static_cast<T*>(a.out) + r * sh.d;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int p = q.gt + i * q.tpr;
                    if (p < pieces) {
                        fma_piece<V>(u[i], b[i], hh[i], u[i]);
                        store_piece<T, V>(out + (size_t)p * V, u[i]);
                    }
                }
            }
            if (sh.norm != ROLA_NORM_NONE) {
                const float2 m = normalise<WARP, V, NV>(sh.norm, sh.d, sh.eps, q.gt, q.tpr, pieces, u, red, turn, refill);
                st.x = m.x;
                st.y = m.y;
                T* y = static_cast<T*>(a.y) + r * sh.d;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int p = q.gt + i * q.tpr;
                    if (p < pieces) {
                        fma_piece<V>(u[i], u[i], g[i], c[i]);
                        store_piece<T, V>(y + (size_t)p * V, u[i]);
                    }
                }
            }
            if (held) {
                group_sync<WARP>();
                refill();
            }
            if (a.stats && q.gt == 0) reinterpret_cast<float4*>(a.stats)[r] = st;
        }
    }
}

template <typename T, int V, int EL, bool WARP, int TH, int MIN>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : TH, MIN)
    rn_bwd_kernel(const __grid_constant__ RnShape sh, const __grid_constant__ RnArgs a, int depth)
{
    constexpr int NV = EL / V;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float2 red[2][32];
    int turn = 0;
    const int group = WARP ? threadIdx.x >> 5 : 0, part = WARP ? blockIdx.x * kWarpGroups + group : blockIdx.x;
    if (part >= a.parts) return;
    const bool normed = sh.norm != ROLA_NORM_NONE;
    Feed<T, V, NV, 4> q;
    q.tpr = WARP ? 32 : blockDim.x;
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.depth = depth;
    q.end = rn_row(sh.total, a.parts, part + 1);
    long long r = rn_row(sh.total, a.parts, part);
    q.start(sh, a, smem, group, r);
    const int pieces = sh.d / V;
    const int k1 = a.in[0] != nullptr, k2 = k1 + (a.in[1] != nullptr), k3 = k2 + (a.in[2] != nullptr);
    const float inv_d = 1.0f / (float)sh.d;
    group_sync<WARP>();                                  // the mbarriers are there
    float4 st = reinterpret_cast<const float4*>(a.stats)[r];
#pragma unroll 1
    for (int s = (int)(r / sh.rows); r < q.end; ++s) {   // the part's samples, and their rows
        const long long stop = min(q.end, (long long)(s + 1) * sh.rows);
        float g[NV][V], b[NV][V], A[NV][V], B[NV][V], E[NV][V];
        load_vectors<T, V, NV, false>(sh, a, s, q.gt, q.tpr, pieces, g, A, b);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) A[i][e] = B[i][e] = E[i][e] = 0.0f;
#pragma unroll 1
        for (; r < stop; ++r) {
            const float4 now = st;
            if (r + 1 < q.end) st = reinterpret_cast<const float4*>(a.stats)[r + 1];
            const bool ok = q.wait();
            float v[NV][V], hh[NV][V], dy[NV][V], t[NV][V];
            q.read(sh, a, 0, 0, r, ok, v);
            q.read(sh, a, 1, k1, r, ok, hh);
            q.read(sh, a, 2, k2, r, ok, dy);
            q.read(sh, a, 3, k3, r, ok, t);
            bool held = true;
            auto refill = [&]() {
                if (!held) return;
                held = false;
                if constexpr (WARP) __syncwarp();
                q.refill(sh, a);
            };
            if (sh.branch != ROLA_NORM_NONE)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (q.gt + i * q.tpr < pieces) {
                        fma_piece<V>(hh[i], hh[i], 1.0f, -now.z);
                        fma_piece<V>(hh[i], hh[i], now.w, 0.0f);
                    }
            if (normed) {
                float s1[2] = {0.0f, 0.0f}, s2[2] = {0.0f, 0.0f}, zero[V] = {};
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (q.gt + i * q.tpr < pieces) {
                        fma_piece<V>(v[i], b[i], hh[i], v[i]);           // the forward's sum, to the bit
                        fma_piece<V>(v[i], v[i], 1.0f, -now.x);
                        fma_piece<V>(v[i], v[i], now.y, 0.0f);
                        fma_piece<V>(A[i], dy[i], v[i], A[i]);
                        add_piece<V>(B[i], dy[i]);
                        fma_piece<V>(dy[i], dy[i], g[i], zero);
                        sum_piece<V>(s1, dy[i]);
                        dot_piece<V>(s2, dy[i], v[i]);
                    }
                const float2 m = group_sum<WARP>(s1[0] + s1[1], s2[0] + s2[1], red, turn);
                refill();
                const float m1 = sh.norm == ROLA_NORM_LAYER ? m.x * inv_d : 0.0f, m2 = m.y * inv_d;
                const float size[2] = {now.y, now.y};
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    fma_piece<V>(v[i], v[i], -m2, -m1);
                    add_piece<V>(v[i], dy[i]);
                    if constexpr (V == 1) t[i][0] = fmaf(v[i][0], now.y, t[i][0]);
                    else
#pragma unroll
                        for (int e = 0; e < V; e += 2) fma2(&t[i][e], &v[i][e], size, &t[i][e]);
                }
            }
            T* dx = static_cast<T*>(a.dx) + r * sh.d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = q.gt + i * q.tpr;
                if (p < pieces) {
                    fma_piece<V>(E[i], t[i], hh[i], E[i]);
                    if (held) continue;                      // dx may be dout, of which the group has not read all yet
                    store_piece<T, V>(dx + (size_t)p * V, t[i]);
                }
            }
            if (held) {
                group_sync<WARP>();
                refill();
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int p = q.gt + i * q.tpr;
                    if (p < pieces) store_piece<T, V>(dx + (size_t)p * V, t[i]);
                }
            }
            if (a.dh) {
                float zero[V] = {};
                T* dh = static_cast<T*>(a.dh) + r * sh.d;
                float s1[2] = {0.0f, 0.0f}, s2[2] = {0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (q.gt + i * q.tpr < pieces) {
                        fma_piece<V>(t[i], t[i], b[i], zero);
                        sum_piece<V>(s1, t[i]);
                        dot_piece<V>(s2, t[i], hh[i]);
                    }
                if (sh.branch != ROLA_NORM_NONE) {
                    const float2 m = group_sum<WARP>(s1[0] + s1[1], s2[0] + s2[1], red, turn);
                    const float m1 = sh.branch == ROLA_NORM_LAYER ? m.x * inv_d : 0.0f, m2 = m.y * inv_d;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        fma_piece<V>(hh[i], hh[i], -m2, -m1);
                        add_piece<V>(t[i], hh[i]);
                        fma_piece<V>(t[i], t[i], now.w, 0.0f);
                    }
                }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int p = q.gt + i * q.tpr;
                    if (p < pieces) store_piece<T, V>(dh + (size_t)p * V, t[i]);
                }
            }
        }
        if (a.part) {
            float* out = a.part + (size_t)(part + s) * 3 * sh.d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int p = q.gt + i * q.tpr;
                if (p < pieces)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        out[(size_t)p * V + e] = A[i][e];
                        out[sh.d + (size_t)p * V + e] = B[i][e];
                        out[2 * (size_t)sh.d + (size_t)p * V + e] = E[i][e];
                    }
            }
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

constexpr int kMostParts = 4864, kMostCtas = 1216;       // of warps, of CTAs: 32 and 8 on each of 152 SMs
constexpr int kFwdRegisters = 16384, kBwdRegisters = 8192;       // longest rows that are held in registers

// Whether every row, and every vector, can be taken in 16-byte pieces.
bool wide(const RnShape& s, const RnArgs& a, int esz)
{
    uintptr_t bits = 0;
    for (const void* p : {a.x, a.h, a.gate, a.gamma_h, a.gamma, a.beta, a.scale, a.shift, a.dout, a.dy,
                          (const void*)a.out, (const void*)a.y, (const void*)a.dx, (const void*)a.dh})
        bits |= reinterpret_cast<uintptr_t>(p);
    return (int64_t)s.d * esz % 16 == 0 && s.mod_stride * esz % 16 == 0 && (bits & 15u) == 0;
}

cudaError_t sm_count(int* n)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
}

// Threads, parts, ring depth and shared memory of a launch: `ctas` of them fit an SM's registers.
struct Launch {
    int threads, grid, parts, depth;
    size_t smem;
};
template <typename K>
cudaError_t shape_of(K kernel, const RnShape& s, bool warp, int el, int registers, size_t row_bytes, long long most, Launch* l)
{
    int nsm = 0;
    cudaError_t e = sm_count(&nsm);
    if (e != cudaSuccess) return e;
    const int groups = warp ? kWarpGroups : 1;
    l->threads = warp ? 32 * kWarpGroups : ((s.d + el - 1) / el + 31) / 32 * 32;
    int ctas = 65536 / (registers * l->threads);
    ctas = ctas < 1 ? 1 : ctas > 8 ? 8 : ctas;
    while (ctas > 1 && groups * row_bytes * 2 * ctas > kRingBytes) --ctas;       // two rows a group at least, if they fit
    long long parts = (long long)nsm * ctas * groups;
    if (parts > s.total) parts = s.total;
    if (parts > most) parts = most;
    l->parts = (int)parts;
    l->grid = (int)((parts + groups - 1) / groups);
    const long long each = (s.total + parts - 1) / parts;
    long long n = (long long)(kRingBytes / (ctas * groups * row_bytes));
    if (n > each) n = each;
    if (n > kMaxDepth) n = kMaxDepth;
    l->depth = n < 1 ? 1 : (int)n;
    l->smem = kBarBytes + groups * l->depth * row_bytes;
    // The limit is the kernel's, not the call's: every call sets it to the same, since another thread may be about to launch.
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kRingBytes + kBarBytes));
}

template <typename T, int V, int EL, bool WARP, int TH, int MIN>
cudaError_t fwd_one(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    Launch l;
    auto kernel = rn_fwd_kernel<T, V, EL, WARP, TH, MIN>;
    const size_t row = (size_t)place_bytes(s.d, sizeof(T), V > 1) * (a.h ? 2 : 1);
    cudaError_t e = shape_of(kernel, s, WARP, EL, 65536 / (TH * MIN) / 8 * 8, row, 1ll << 30, &l);
    if (e != cudaSuccess) return e;
    a.in[0] = a.x;
    a.in[1] = a.h;
    a.parts = l.parts;
    kernel<<<l.grid, l.threads, l.smem, st>>>(s, a, l.depth);
    return cudaGetLastError();
}
template <typename T, int V, int EL, bool WARP, int TH, int MIN>
cudaError_t bwd_one(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    Launch l;
    auto kernel = rn_bwd_kernel<T, V, EL, WARP, TH, MIN>;
    const int matrices = (s.norm != ROLA_NORM_NONE ? 1 : 0) + (a.h ? 1 : 0) + (a.dy ? 1 : 0) + (a.dout ? 1 : 0);
    const size_t row = (size_t)place_bytes(s.d, sizeof(T), V > 1) * matrices;
    cudaError_t e = shape_of(kernel, s, WARP, EL, 65536 / (TH * MIN) / 8 * 8, row, rn_parts(s), &l);
    if (e != cudaSuccess) return e;
    a.in[0] = s.norm != ROLA_NORM_NONE ? a.x : nullptr;
    a.in[1] = a.h;
    a.in[2] = a.dy;
    a.in[3] = a.dout;
    a.parts = l.parts;
    kernel<<<l.grid, l.threads, l.smem, st>>>(s, a, l.depth);
    return cudaGetLastError();
}

// A warp a row up to 16 elements a lane, then a CTA a row of the least whole number of warps.
template <typename T, int V>
cudaError_t fwd(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (s.d <= 256) return fwd_one<T, V, 8, true, 128, 6>(s, a, st);
    if (s.d <= 512) return fwd_one<T, V, 16, true, 128, 4>(s, a, st);
    if (s.d <= 8 * 256) return fwd_one<T, V, 8, false, 256, 3>(s, a, st);
    if (s.d <= 16 * 320) return fwd_one<T, V, 16, false, 320, 2>(s, a, st);
    if (s.d <= 16 * 512) return fwd_one<T, V, 16, false, 512, 1>(s, a, st);
    if (s.d <= kFwdRegisters) return fwd_one<T, V, 32, false, 512, 1>(s, a, st);
    rn_fwd_long_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    return cudaGetLastError();
}

template <typename T, int V>
cudaError_t bwd(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (s.d <= 256) return bwd_one<T, V, 8, true, 128, 4>(s, a, st);
    if (s.d <= 512) return bwd_one<T, V, 16, true, 128, 2>(s, a, st);
    if (s.d <= 8 * 320) return bwd_one<T, V, 8, false, 320, 2>(s, a, st);
    if (s.d <= 8 * 640) return bwd_one<T, V, 8, false, 640, 1>(s, a, st);
    if (s.d <= kBwdRegisters) return bwd_one<T, V, 16, false, 512, 1>(s, a, st);
    a.parts = rn_parts(s);
    rn_moments_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    if (a.part) rn_columns_kernel<T><<<dim3((s.d + 127) / 128, a.parts), 128, 0, st>>>(s, a);
    rn_bwd_long_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    const bool sums = wants_sums(a);
    if (!sums) a.part = nullptr;
    cudaError_t e = wide(s, a, sizeof(T)) ? bwd<T, 16 / sizeof(T)>(s, a, st) : bwd<T, 1>(s, a, st);
    if (e != cudaSuccess || !sums) return e;
    int ways = 32;
    while (ways > 1 && ways * s.groups > 32) ways /= 2;
    rn_reduce_kernel<T><<<(s.d + 31) / 32, 1024, 0, st>>>(s, a, ways);
    return cudaGetLastError();
}

}  // namespace

int rn_parts(const RnShape& s)
{
    const long long want = (s.total + 1) / 2, most = s.d <= 512 ? kMostParts : kMostCtas;
    return (int)(want < most ? want : most);
}

bool rn_long(const RnShape& s) { return s.d > kBwdRegisters; }

cudaError_t launch_residual_norm(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (dt == ROLA_BF16) return wide(s, a, 2) ? fwd<__nv_bfloat16, 8>(s, a, st) : fwd<__nv_bfloat16, 1>(s, a, st);
    return wide(s, a, 4) ? fwd<float, 4>(s, a, st) : fwd<float, 1>(s, a, st);
}

cudaError_t launch_residual_norm_backward(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st)
{
    return dt == ROLA_BF16 ? backward<__nv_bfloat16>(s, a, st) : backward<float>(s, a, st);
}

}  // namespace rola
