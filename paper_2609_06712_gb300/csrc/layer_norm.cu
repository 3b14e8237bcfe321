// Layer norm over the rows of x [rows][d], and its gradients.
//
//   y = (x - mu) rstd gamma + beta,   mu = mean x,   rstd = (mean (x - mu)^2 + eps)^(-1/2)
//   dx = rstd (a - mean a - xh mean(a xh)),   a = dy gamma,   xh = (x - mu) rstd
//   dgamma = sum_rows dy xh,   dbeta = sum_rows dy
//
// HBM-bound: x once in and y once out forward, x and dy in and dx out backward
// (a few fp32 operations per element against 4 or 6 bytes).  A row is held in
// registers by the threads of a group, NV pieces each, so that mean, centred
// sum of squares and output take one read of the row; a piece is 16 bytes where
// the row length and the pointers allow it, else one element.  gamma and beta
// are converted once and stay in registers.  Short rows have a warp each (four
// in a CTA, no barrier), longer ones a CTA whose size is rounded up from the
// row's pieces, so that few threads idle.
//
// To keep HBM busy an SM needs some 60 KB of loads in flight (44 bytes per ns at
// over 1 us of latency); a row per CTA in registers is 10 KB at d = 5120.  So with
// 16-byte pieces the CTA's coming rows are copied ahead into a ring in shared
// memory (bulk asynchronous copies, one per row, each with its mbarrier).
// Rows of single elements, which need not start on 16 bytes, are fetched one
// ahead into registers instead.
//
// Backward: every thread keeps the dgamma / dbeta sums of its own columns in
// registers over all the rows its group takes (row r of group g: g, g + G, ...),
// the groups of a CTA add theirs through shared memory in group order, and each
// CTA writes one partial row; a second kernel adds the partial rows in a fixed
// order.  All sums are fp32.
//
// Measured, bf16: 75600 x 5120 forward 251 us (6.2 TB/s, 91 % of a copy), backward 390 us
// (6.0 TB/s); 32760 x 1536 39 and 63 us, where the ramp and the tail count.  Rows of 8200 to 16384 elements spill 360
// bytes a thread in the backward.
//
// The variance is taken about the rounded mean, so a common offset of the row does not cancel in it; the mean's own
// rounding, and with it a shift of x - mu of the order of 2^-24 |mu|, remains.
#include "norm_rows.cuh"
#include "tcgen05.cuh"

namespace rola {
namespace {

constexpr int kWarpGroups = 4;           // rows of a CTA whose rows have a warp each
constexpr int kMaxThreads = 512;         // of a CTA that has one row
constexpr size_t kStaticSmem = sizeof(float2[2][32]);    // of the row kernels: `red`

constexpr int kMaxDepth = 16;            // rows in a group's ring
constexpr size_t kRingBytes = 160 << 10;             // of the rings of an SM's CTAs
constexpr uint64_t kWaitLimitNs = 2000000000ull;     // bound of the wait for a row

// A group's rows r0, r0 + stride, ... of N matrices, brought ahead.  RING: into
// `depth` slots of N rows in shared memory, one bulk copy per matrix; a slot is
// refilled after its row has been read into registers (a barrier of the group lies
// between).  Otherwise one row ahead in registers.
template <typename T, int V, int NV, int N, bool WARP, bool RING>
struct Rows {
    const T* src[N];
    long long rows, stride, next;        // next: the row the next copy is of
    int d, tpr, gt, pieces, depth, slot, phase;
    uint32_t ring, bars;                 // shared memory: the slots, their mbarriers
    Piece<T, V> p[RING ? 1 : N][NV];

    __device__ __forceinline__ void copy(int to)         // one thread
    {
        const uint32_t bytes = (uint32_t)d * sizeof(T), bar = bars + to * 8;
        tc::mbar_expect_tx(bar, N * bytes);
#pragma unroll
        for (int n = 0; n < N; ++n)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(
                             ring + (uint32_t)(to * N + n) * bytes),
                         "l"(src[n] + next * d), "r"(bytes), "r"(bar)
                         : "memory");
        next += stride;
    }
    __device__ __forceinline__ void fetch(long long r)   // registers
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = gt + i * tpr;
                if (c < pieces) p[n][i] = load_piece<T, V>(src[n] + r * d + (size_t)c * V);
            }
    }
    __device__ __forceinline__ void start(long long r0)
    {
        if constexpr (RING) {
            next = r0;
            slot = phase = 0;
            if (gt == 0) {
                for (int i = 0; i < depth; ++i) tc::mbar_init(bars + i * 8, 1);
                tc::fence_mbar_init();
                for (int i = 0; i < depth && next < rows; ++i) copy(i);
            }
            if constexpr (WARP) __syncwarp();
            else __syncthreads();
        } else if (r0 < rows) {
            fetch(r0);
        }
    }
    // The present row's pieces as fp32.  In the ring its slot is then refilled by `refill`, after a barrier.
    __device__ __forceinline__ void read(float (&v)[N][NV][V])
    {
        // a copy that never arrives leaves NaN in the row's results (the call has no status word)
        bool ok = true;
        if constexpr (RING) {
            int never = 0;
            ok = tc::mbar_wait(bars + slot * 8, phase, &never, kWaitLimitNs);
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = gt + i * tpr;
                if (c < pieces) {
                    if constexpr (RING) {
                        Piece<T, V> x;
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
                                     : "=r"(x.w.x), "=r"(x.w.y), "=r"(x.w.z), "=r"(x.w.w)
                                     : "r"(ring + (uint32_t)(slot * N + n) * d * (uint32_t)sizeof(T) + c * 16)
                                     : "memory");
                        unpack<T, V>(x, v[n][i]);
                        if (!ok) v[n][i][0] = __int_as_float(0x7fc00000);
                    } else {
                        unpack<T, V>(p[n][i], v[n][i]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) v[n][i][e] = 0.0f;
                }
            }
    }
    __device__ __forceinline__ void ahead(long long r)   // registers: row r + stride
    {
        if constexpr (!RING)
            if (r + stride < rows) fetch(r + stride);
    }
    __device__ __forceinline__ void refill()             // ring: after every thread of the group has read
    {
        if constexpr (RING) {
            if (gt == 0 && next < rows) copy(slot);
            if (++slot == depth) {
                slot = 0;
                phase ^= 1;
            }
        }
    }
};

// Dynamic shared memory: the groups' mbarriers, then their rings (each a whole number of rows of 16-byte pieces).
template <typename R>
__device__ __forceinline__ void place(R& q, unsigned char* smem, int depth, int n, bool warp, int esz)
{
    const uint32_t group = warp ? threadIdx.x >> 5 : 0, groups = warp ? kWarpGroups : 1;
    q.depth = depth;
    q.bars = smem_u32(smem) + group * kMaxDepth * 8;
    q.ring = smem_u32(smem) + groups * kMaxDepth * 8 + group * (uint32_t)(depth * n * q.d * esz);
}

template <typename T, int V, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : kMaxThreads)
    ln_fwd_kernel(long long rows, int d, const T* x, const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                  T* y, float* __restrict__ mean, float* __restrict__ rstd, int depth)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float2 red[2][32];
    int turn = 0;
    Rows<T, V, NV, 1, WARP, (V > 1)> q;
    q.src[0] = x;
    q.rows = rows;
    q.d = d;
    q.tpr = WARP ? 32 : blockDim.x;
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.pieces = d / V;
    q.stride = (long long)gridDim.x * (WARP ? kWarpGroups : 1);
    place(q, smem, depth, 1, WARP, sizeof(T));
    const float inv_d = 1.0f / (float)d;
    long long r = WARP ? (long long)blockIdx.x * kWarpGroups + (threadIdx.x >> 5) : blockIdx.x;
    q.start(r);
    float g[NV][V], b[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = q.gt + i * q.tpr;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            g[i][e] = 1.0f;
            b[i][e] = 0.0f;
        }
        if (gamma && c < q.pieces) unpack<T, V>(load_piece<T, V>(gamma + (size_t)c * V), g[i]);
        if (beta && c < q.pieces) unpack<T, V>(load_piece<T, V>(beta + (size_t)c * V), b[i]);
    }
    for (; r < rows; r += q.stride) {    // uniform over a group
        float v[1][NV][V];
        q.read(v);
        q.ahead(r);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) sum_piece<V>(s, v[0][i]);
        const float mu = group_sum<WARP>(s[0] + s[1], 0.0f, red, turn).x * inv_d;
        q.refill();
        float sq[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (q.gt + i * q.tpr < q.pieces) {
                fma_piece<V>(v[0][i], v[0][i], 1.0f, -mu);
                dot_piece<V>(sq, v[0][i], v[0][i]);
            }
        const float rs = 1.0f / sqrtf(group_sum<WARP>(sq[0] + sq[1], 0.0f, red, turn).x * inv_d + eps);
        if (mean && q.gt == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        T* yr = y + r * d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = q.gt + i * q.tpr;
            if (c < q.pieces) {
                fma_piece<V>(v[0][i], v[0][i], rs, 0.0f);
                fma_piece<V>(v[0][i], v[0][i], g[i], b[i]);
                store_piece<T, V>(yr + (size_t)c * V, v[0][i]);
            }
        }
    }
}

template <typename T, int V, int NV, bool WARP, int TH = kMaxThreads, int MIN = 1>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : TH, MIN)
    ln_bwd_kernel(long long rows, int d, const T* __restrict__ x, const T* __restrict__ gamma,
                  const float* __restrict__ mean, const float* __restrict__ rstd, const T* dy, T* dx,
                  float* __restrict__ part, int depth)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float2 red[2][32];
    int turn = 0;
    Rows<T, V, NV, 2, WARP, (V > 1)> q;
    q.src[0] = x;
    q.src[1] = dy;
    q.rows = rows;
    q.d = d;
    q.tpr = WARP ? 32 : blockDim.x;
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.pieces = d / V;
    q.stride = (long long)gridDim.x * (WARP ? kWarpGroups : 1);
    place(q, smem, depth, 2, WARP, sizeof(T));
    const float inv_d = 1.0f / (float)d;
    long long r = WARP ? (long long)blockIdx.x * kWarpGroups + (threadIdx.x >> 5) : blockIdx.x;
    q.start(r);
    float g[NV][V], dg[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = q.gt + i * q.tpr;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            g[i][e] = 1.0f;
            dg[i][e] = db[i][e] = 0.0f;
        }
        if (gamma && c < q.pieces) unpack<T, V>(load_piece<T, V>(gamma + (size_t)c * V), g[i]);
    }
    float mu = r < rows ? mean[r] : 0.0f, rs = r < rows ? rstd[r] : 0.0f;
    for (; r < rows; r += q.stride) {
        float v[2][NV][V];               // xh, a
        q.read(v);
        q.ahead(r);
        float s1[2] = {0.0f, 0.0f}, s2[2] = {0.0f, 0.0f}, zero[V] = {};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (q.gt + i * q.tpr < q.pieces) {
                float (&xh)[V] = v[0][i], (&a)[V] = v[1][i];
                fma_piece<V>(xh, xh, 1.0f, -mu);         // centred first: mu may be far larger than x - mu
                fma_piece<V>(xh, xh, rs, 0.0f);
                fma_piece<V>(dg[i], a, xh, dg[i]);
                add_piece<V>(db[i], a);
                fma_piece<V>(a, a, g[i], zero);
                sum_piece<V>(s1, a);
                dot_piece<V>(s2, a, xh);
            }
        }
        const float rs0 = rs;
        if (r + q.stride < rows) {
            mu = mean[r + q.stride];
            rs = rstd[r + q.stride];
        }
        const float2 m = group_sum<WARP>(s1[0] + s1[1], s2[0] + s2[1], red, turn);
        q.refill();
        const float m1 = m.x * inv_d, m2 = m.y * inv_d;
        T* dxr = dx + r * d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = q.gt + i * q.tpr;
            if (c < q.pieces) {
                fma_piece<V>(v[0][i], v[0][i], -m2, -m1);        // rs (a - (m1 + xh m2))
                add_piece<V>(v[1][i], v[0][i]);
                fma_piece<V>(v[1][i], v[1][i], rs0, 0.0f);
                store_piece<T, V>(dxr + (size_t)c * V, v[1][i]);
            }
        }
    }
    if (!part) return;
    float* pg = part + (size_t)blockIdx.x * 2 * d;
    if constexpr (!WARP) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = q.gt + i * q.tpr;
            if (c < q.pieces)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    pg[(size_t)c * V + e] = dg[i][e];
                    pg[d + (size_t)c * V + e] = db[i][e];
                }
        }
    } else {
        // the CTA's sums [2 d] take the place of the rings, whose last rows have been read by then
        float* cols = reinterpret_cast<float*>(smem + kWarpGroups * kMaxDepth * 8);
        __syncthreads();
        for (int w = 0; w < kWarpGroups; ++w) {          // in group order: the same bits every time
            if ((int)(threadIdx.x >> 5) == w) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = q.gt + i * q.tpr;
                    if (c < q.pieces)
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            float *qg = cols + c * V + e, *qb = qg + d;
                            *qg = w == 0 ? dg[i][e] : *qg + dg[i][e];
                            *qb = w == 0 ? db[i][e] : *qb + db[i][e];
                        }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * d; c += 32 * kWarpGroups) pg[c] = cols[c];
    }
}

// Rows too long for registers: one CTA per row, passes over it from L2.
template <typename T>
__global__ void __launch_bounds__(512) ln_fwd_long_kernel(long long rows, int d, const T* x, const T* __restrict__ gamma,
                                                          const T* __restrict__ beta, float eps, T* y,
                                                          float* __restrict__ mean, float* __restrict__ rstd)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + r * d;
        float s = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) s += to_float(xr[c]);
        const float mu = group_sum<false>(s, 0.0f, red, turn).x / (float)d;
        float q = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) {
            const float t = to_float(xr[c]) - mu;
            q = fmaf(t, t, q);
        }
        const float rs = 1.0f / sqrtf(group_sum<false>(q, 0.0f, red, turn).x / (float)d + eps);
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

// Rows too long for registers: dx, one CTA per row.
template <typename T>
__global__ void __launch_bounds__(512) ln_bwd_long_kernel(long long rows, int d, const T* __restrict__ x,
                                                          const T* __restrict__ gamma, const float* __restrict__ mean,
                                                          const float* __restrict__ rstd, const T* dy, T* dx)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < d; c += 512) {
            float a = to_float(dy[r * d + c]);
            if (gamma) a *= to_float(gamma[c]);
            s1 += a;
            s2 = fmaf(a, (to_float(x[r * d + c]) - mu) * rs, s2);
        }
        const float2 m = group_sum<false>(s1, s2, red, turn);
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
// columns; its 32 warps add every 32nd partial row (four loads in flight each),
// then the warps' sums meet in warp order.
__global__ void __launch_bounds__(1024) ln_bwd_reduce_kernel(int n, int d, const float* __restrict__ part,
                                                             float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float a = 0.0f;
    if (c < 2 * d) {
#pragma unroll 4
        for (int i = w; i < n; i += 32) a += part[(size_t)i * 2 * d + c];
    }
    s[w][lane] = a;
    __syncthreads();
    if (w == 0 && c < 2 * d) {
#pragma unroll
        for (int i = 1; i < 32; ++i) a += s[i][lane];
        if (c < d) dgamma[c] = a;
        else dbeta[c - d] = a;
    }
}

// ---------------------------------------------------------------- dispatch

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
    int nsm, grid;           // grid: most CTAs of the backward (partial rows), set to those launched
    cudaStream_t st;
};

// CTA size, ring depth and grid of rows of `pieces` pieces, NV per thread: a warp per row, or a CTA of the
// least whole number of warps.  The rings of an SM's CTAs (as many as their registers allow, up to 1024
// threads) hold about 160 KB, and no more rows than a group has.  (Two rows at least: of 32 KB and two
// matrices at most, so a CTA's ring stays within 160 KB, and the warps' sums are far smaller.)
struct Launch {
    int threads, grid, depth;
    size_t smem;
};
template <typename K>
cudaError_t shape_of(K kernel, const LnArgs& a, bool warp, int pieces, int nv, int matrices, size_t row_bytes,
                     size_t sums, Launch* l)
{
    l->threads = warp ? 32 * kWarpGroups : ((pieces + nv - 1) / nv + 31) / 32 * 32;
    int ctas = 0;
    cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kernel, l->threads, 0);
    if (e != cudaSuccess) return e;
    if (ctas > 1024 / l->threads) ctas = 1024 / l->threads;
    const int groups = warp ? kWarpGroups : 1;
    const long long want = (a.rows + groups - 1) / groups;
    l->depth = 0;
    size_t ring = 0;
    if (row_bytes) {
        const long long each = (a.rows + (long long)a.nsm * ctas * groups - 1) / ((long long)a.nsm * ctas * groups);
        long long n = (long long)kRingBytes / (ctas * groups * matrices * (long long)row_bytes);
        if (n > each) n = each;
        if (n > kMaxDepth) n = kMaxDepth;
        l->depth = n < 2 ? 2 : (int)n;
        ring = (size_t)groups * matrices * l->depth * row_bytes;
    }
    l->smem = (size_t)groups * kMaxDepth * 8 + (ring > sums ? ring : sums);
    // 48 KB without asking are of static and dynamic shared memory together.  The limit is the kernel's, not the
    // call's: every call sets it to the same, the most that any needs, since another thread may be about to launch.
    if (l->smem + kStaticSmem > 48 << 10)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)(kRingBytes + kWarpGroups * kMaxDepth * 8));
    if (e != cudaSuccess) return e;
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, l->threads, l->smem);
    if (e != cudaSuccess) return e;
    const long long cap = (long long)a.nsm * (per_sm > 0 ? per_sm : 1);
    l->grid = (int)(want < cap ? want : cap);
    return cudaSuccess;
}

template <typename T, int V, int NV, bool WARP>
cudaError_t fwd_one(const LnArgs& a)
{
    Launch l;
    auto kernel = ln_fwd_kernel<T, V, NV, WARP>;
    cudaError_t e = shape_of(kernel, a, WARP, a.d / V, NV, 1, V > 1 ? sizeof(T) * a.d : 0, 0, &l);
    if (e != cudaSuccess) return e;
    kernel<<<l.grid, l.threads, l.smem, a.st>>>(a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma),
                                                static_cast<const T*>(a.beta), a.eps, static_cast<T*>(a.y), a.mean,
                                                a.rstd, l.depth);
    return cudaGetLastError();
}
template <typename T, int V, int NV, bool WARP, int TH = kMaxThreads, int MIN = 1>
cudaError_t bwd_one(LnArgs& a)
{
    Launch l;
    auto kernel = ln_bwd_kernel<T, V, NV, WARP, TH, MIN>;
    cudaError_t e = shape_of(kernel, a, WARP, a.d / V, NV, 2, V > 1 ? sizeof(T) * a.d : 0,
                             WARP && a.part ? sizeof(float) * 2 * a.d : 0, &l);
    if (e != cudaSuccess) return e;
    if (a.part && l.grid > a.grid) l.grid = a.grid;
    a.grid = l.grid;
    kernel<<<l.grid, l.threads, l.smem, a.st>>>(a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma),
                                                a.mean, a.rstd, static_cast<const T*>(a.dy), static_cast<T*>(a.y),
                                                a.part, l.depth);
    return cudaGetLastError();
}

// A warp per row up to two 16-byte pieces a lane (8 elements a lane element by element), then a CTA per
// row: the pieces a thread holds are bounded by its registers (forward x, gamma and beta as fp32,
// backward x, dy, gamma and two sums).
template <typename T, int V>
cudaError_t fwd(const LnArgs& a)
{
    const int pieces = a.d / V;
    if constexpr (V > 1) {
        if (pieces <= 32) return fwd_one<T, V, 1, true>(a);
        if (pieces <= 64) return fwd_one<T, V, 2, true>(a);
        if (pieces <= 2 * 128) return fwd_one<T, V, 2, false>(a);
        if (pieces <= 4 * kMaxThreads) return fwd_one<T, V, 4, false>(a);
    } else {
        if (pieces <= 4 * 32) return fwd_one<T, V, 4, true>(a);
        if (pieces <= 8 * 32) return fwd_one<T, V, 8, true>(a);
        if (pieces <= 4 * kMaxThreads) return fwd_one<T, V, 4, false>(a);
        if (pieces <= 16 * kMaxThreads) return fwd_one<T, V, 16, false>(a);
    }
    const long long cap = (long long)a.nsm * 4;
    ln_fwd_long_kernel<T><<<(int)(a.rows < cap ? a.rows : cap), 512, 0, a.st>>>(
        a.rows, a.d, static_cast<const T*>(a.x), static_cast<const T*>(a.gamma), static_cast<const T*>(a.beta), a.eps,
        static_cast<T*>(a.y), a.mean, a.rstd);
    return cudaGetLastError();
}

template <typename T, int V>
cudaError_t bwd(LnArgs& a)
{
    const int pieces = a.d / V;
    if constexpr (V > 1) {
        if (pieces <= 32) return bwd_one<T, V, 1, true>(a);
        if (pieces <= 64) return bwd_one<T, V, 2, true>(a);
        // up to 320 threads two CTAs an SM: with one, the barriers of a row (d = 5120) leave HBM idle
        if (pieces <= 2 * 320) return bwd_one<T, V, 2, false, 320, 2>(a);
        if (pieces <= 2 * kMaxThreads) return bwd_one<T, V, 2, false>(a);
        if (pieces <= 4 * kMaxThreads) return bwd_one<T, V, 4, false>(a);
    } else {
        if (pieces <= 4 * 32) return bwd_one<T, V, 4, true>(a);
        if (pieces <= 8 * 32) return bwd_one<T, V, 8, true>(a);
        if (pieces <= 4 * kMaxThreads) return bwd_one<T, V, 4, false>(a);
        if (pieces <= 16 * kMaxThreads) return bwd_one<T, V, 16, false>(a);
    }
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

// Most CTAs of the backward, each of which leaves a partial row: 8 on each of 152 SMs, and no more than
// leave four rows to a CTA.
int bwd_grid(long long rows)
{
    const long long want = (rows + 3) / 4;
    return (int)(want < 1216 ? want : 1216);
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
    ln_bwd_reduce_kernel<<<(2 * d + 31) / 32, 1024, 0, st>>>(a.grid, d, part, dgamma, dbeta);
    return cudaGetLastError();
}

}  // namespace rola
