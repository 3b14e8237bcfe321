// Dense softmax attention and its gradients in plain fp32 arithmetic (no
// tensor cores): the fp32 mode; and the small kernels both modes use (joining
// the parts of a split key axis, the row products dO . o).
//
//   o = softmax(scale q k^T) v over the keys a row sees; the gradients recompute
//   p = exp(scale q k^T - lse), dp = dO v^T, ds = scale p (dp - D), D = dO . o
//   dq = ds k,  dk = ds^T q,  dv = p^T dO
//
// Rows are the G Lq queries of the heads that share a key head, so dk and dv of
// a shared head are sums over rows like any other.  Tiles of 64 rows x 64 keys,
// 256 threads as 16 x 16 (thread (tx, ty) holds rows ty + 16 i, keys tx + 16 j),
// operands as fp32 rows of 132 words, so that the 16-byte reads of 8 rows touch
// all banks once.  Running maximum and sum per row in registers, shared by the
// 16 threads of the row through shuffles.  Bound by fp32 FMA issue.
#include "block_ops.cuh"

namespace rola {
namespace {

constexpr int kT = 64, kRow = 132, kPRow = 68;
constexpr int kTileF = kT * kRow, kPF = kT * kPRow;      // floats of an operand tile, of a 64 x 64 tile

// rows [r0, r0 + 64) of a [n][128] matrix, zeros past n
__device__ __forceinline__ void load_tile(float* s, const float* p, int r0, int n)
{
    for (int e = threadIdx.x; e < kT * 32; e += 256) {
        const int r = e / 32, c = (e % 32) * 4;
        const float4 x = r0 + r < n ? load4(p + (size_t)(r0 + r) * kDh + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        *reinterpret_cast<float4*>(s + r * kRow + c) = x;
    }
}

// acc[i][j] = A[ty + 16 i] . B[tx + 16 j] over 128
__device__ __forceinline__ void dot_tile(const float* A, const float* B, int tx, int ty, float (&acc)[4][4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
#pragma unroll 4
    for (int c = 0; c < kDh; c += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * kRow + c);
            b[i] = *reinterpret_cast<const float4*>(B + (tx + 16 * i) * kRow + c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc[i][j] = fmaf(a[i].x, b[j].x, acc[i][j]);
                acc[i][j] = fmaf(a[i].y, b[j].y, acc[i][j]);
                acc[i][j] = fmaf(a[i].z, b[j].z, acc[i][j]);
                acc[i][j] = fmaf(a[i].w, b[j].w, acc[i][j]);
            }
    }
}

// out[i][.] += sum_k W[ty + 16 i][k] X[k], k = 0..63, columns 4 tx .. and 64 + 4 tx ..
__device__ __forceinline__ void mix_tile(const float* W, const float* X, int tx, int ty, float (&out)[4][8])
{
#pragma unroll 2
    for (int k = 0; k < kT; k += 4) {
        float w[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            *reinterpret_cast<float4*>(w[i]) = *reinterpret_cast<const float4*>(W + (ty + 16 * i) * kPRow + k);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            float x[8];
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(X + (k + kk) * kRow + tx * 4);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(X + (k + kk) * kRow + 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) out[i][j] = fmaf(w[i][kk], x[j], out[i][j]);
        }
    }
}

__device__ __forceinline__ float row_max(float x)
{
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
    return x;
}
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

__device__ __forceinline__ void store_row(float* p, int tx, const float (&x)[8])
{
    store4(p + tx * 4, make_float4(x[0], x[1], x[2], x[3]));
    store4(p + 64 + tx * 4, make_float4(x[4], x[5], x[6], x[7]));
}

// grid (row tiles, heads, splits).  Part z of n parts takes the key tiles [z t / n, (z + 1) t / n) of the
// t that the row tile sees.
__global__ void __launch_bounds__(256) attention_simt_kernel(const AttnShape s, const AttnArgs a)
{
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *K = sm + kTileF, *V = K + kTileF, *P = V + kTileF;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int head = blockIdx.y, b = head / s.Hk, r0 = blockIdx.x * kT;
    const int len = attn_len(s, a.kv_len, b);
    const int last = min(r0 + kT, s.R) - 1;
    const int tiles = (attn_seen_most(s, len, r0, last) + kT - 1) / kT;
    const int t0 = (int)((long long)tiles * blockIdx.z / s.splits), t1 = (int)((long long)tiles * (blockIdx.z + 1) / s.splits);
    const float *q = static_cast<const float*>(a.q) + (size_t)head * s.R * kDh, *k = static_cast<const float*>(a.k) + (size_t)head * s.Lk * kDh,
            *v = static_cast<const float*>(a.v) + (size_t)head * s.Lk * kDh;
    load_tile(Q, q, r0, s.R);
    float m[4], l[4], o[4][8] = {};
    int seen[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.0f;
        const int r = r0 + ty + 16 * i;
        seen[i] = r < s.R ? attn_seen(s, len, r) : 0;
    }
    for (int t = t0; t < t1; ++t) {
        __syncthreads();
        load_tile(K, k, t * kT, len);
        load_tile(V, v, t * kT, len);
        __syncthreads();
        float x[4][4];
        dot_tile(Q, K, tx, ty, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float top = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[i][j] = t * kT + tx + 16 * j < seen[i] ? x[i][j] * s.scale : -INFINITY;
                top = fmaxf(top, x[i][j]);
            }
            top = row_max(top);
            const float base = top == -INFINITY ? 0.0f : top;      // a row that has seen nothing yet
            const float keep = expf(m[i] - base);
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[i][j] = expf(x[i][j] - base);
                sum += x[i][j];
                P[(ty + 16 * i) * kPRow + tx + 16 * j] = x[i][j];
            }
            l[i] = l[i] * keep + row_sum(sum);
            m[i] = top;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[i][j] *= keep;
        }
        __syncthreads();
        mix_tile(P, V, tx, ty, o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + ty + 16 * i;
        if (r >= s.R) continue;
        // l is 0 where nothing is seen, and over scores of -inf alone: then p is 0 / 0 (with parts the join says so)
        const float inv = l[i] == 0.0f ? (seen[i] > 0 && s.splits == 1 ? __int_as_float(0x7fc00000) : 0.0f) : 1.0f / l[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[i][j] *= inv;
        const size_t row = (size_t)head * s.R + r;
        const float lse = l[i] == 0.0f ? -INFINITY : m[i] + logf(l[i]);
        if (s.splits > 1) {
            const size_t at = (size_t)blockIdx.z * s.heads * s.R + row;
            store_row(a.part_o + at * kDh, tx, o[i]);
            if (tx == 0) a.part_lse[at] = lse;
        } else {
            store_row(static_cast<float*>(a.o) + row * kDh, tx, o[i]);
            if (a.lse && tx == 0) a.lse[row] = lse;
        }
    }
}

// o = sum_z w_z o_z with w_z = exp(lse_z - lse), the parts in order; NaN if a part is, or if the row sees keys but
// every score is -inf.  One warp per row.
template <typename T>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttnShape s, const AttnArgs a)
{
    const long long rows = (long long)s.heads * s.R;
    const int lane = threadIdx.x % 32;
    const long long row = (long long)blockIdx.x * 8 + threadIdx.x / 32;
    if (row >= rows) return;
    float top = -INFINITY;
    bool nan = false;
    for (int z = lane; z < s.splits; z += 32) {
        const float x = a.part_lse[z * rows + row];
        top = fmaxf(top, x);
        nan = nan || x != x;
    }
    nan = __any_sync(0xffffffffu, nan);
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.0f;
    if (top > -INFINITY || nan) {
        for (int z = 0; z < s.splits; ++z) {
            const float w = expf(a.part_lse[z * rows + row] - top);
            const float4 x = load4(a.part_o + (z * rows + row) * kDh + lane * 4);
            l += w;
            o.x = fmaf(w, x.x, o.x); o.y = fmaf(w, x.y, o.y); o.z = fmaf(w, x.z, o.z); o.w = fmaf(w, x.w, o.w);
        }
        const float inv = 1.0f / l;
        o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
    } else {
        const int head = (int)(row / s.R);
        if (attn_seen(s, attn_len(s, a.kv_len, head / s.Hk), (int)(row - (long long)head * s.R)) > 0)
            o.x = o.y = o.z = o.w = __int_as_float(0x7fc00000);
    }
    store4(static_cast<T*>(a.o) + row * kDh + lane * 4, o);
    if (a.lse && lane == 0) a.lse[row] = l == 0.0f ? -INFINITY : top + logf(l);
}

__device__ __forceinline__ void load8(const float* p, float (&x)[8])
{
    const float4 a = load4(p), b = load4(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8])
{
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {                        // a bf16 is the upper half of the fp32 of its value
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// D = rowsum(dO o), 16 lanes per row, 8 elements each (bf16: 16-byte loads), two rows on their way at once.
// Bound by HBM (196560 rows: 101 MB in 19 us; one row at a time 25).  It clears the status word for the kernels behind it
// (8 heads x 128 rows: the pass takes 18.2 us to 128 keys, where a memset does that, and 16.2 to 256 keys).
template <typename T>
__global__ void __launch_bounds__(256) attention_rowdot_kernel(long long rows, const T* __restrict__ dO,
                                                               const T* __restrict__ o, float* __restrict__ D,
                                                               DeviceStatus* status)
{
    static_assert(sizeof(DeviceStatus) == 64 * sizeof(int), "a word a thread");
    if (blockIdx.x == 0 && threadIdx.x < 64) reinterpret_cast<int*>(status)[threadIdx.x] = 0;
    constexpr int kEach = 2;
    const int lane = threadIdx.x % 16;
    const long long row0 = (long long)blockIdx.x * (16 * kEach) + threadIdx.x / 16;
    float x[kEach][8], y[kEach][8];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long row = row0 + 16 * i;
        if (row >= rows) continue;
        load8(dO + row * kDh + lane * 8, x[i]);
        load8(o + row * kDh + lane * 8, y[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long row = row0 + 16 * i;
        float d = 0.0f;
        if (row < rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d = fmaf(x[i][e], y[i][e], d);
        }
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
        if (lane == 0 && row < rows) D[row] = d;
    }
}

// p and ds of the tile at (rows r0 + .., keys k0 + ..) for this thread's 4 x 4 places; 0 where the row
// does not see the key.
struct Grad4 {
    float p[4][4], ds[4][4];
};
__device__ __forceinline__ void grad_tile(const AttnShape& s, const float* Q, const float* K, const float* dO,
                                          const float* V, const float (&lse)[4], const float (&D)[4],
                                          const int (&seen)[4], int k0, int tx, int ty, Grad4& g)
{
    float dp[4][4];
    dot_tile(Q, K, tx, ty, g.p);
    dot_tile(dO, V, tx, ty, dp);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = k0 + tx + 16 * j < seen[i];
            g.p[i][j] = in ? expf(g.p[i][j] * s.scale - lse[i]) : 0.0f;
            g.ds[i][j] = in ? g.p[i][j] * (dp[i][j] - D[i]) * s.scale : 0.0f;
        }
}

// grid (row tiles, heads)
__global__ void __launch_bounds__(256) attention_dq_simt_kernel(const AttnShape s, const AttnArgs a)
{
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *dO = Q + kTileF, *K = dO + kTileF, *V = K + kTileF, *S = V + kTileF;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int head = blockIdx.y, b = head / s.Hk, r0 = blockIdx.x * kT;
    const int len = attn_len(s, a.kv_len, b);
    const int tiles = (attn_seen_most(s, len, r0, min(r0 + kT, s.R) - 1) + kT - 1) / kT;
    const size_t qh = (size_t)head * s.R * kDh, kh = (size_t)head * s.Lk * kDh;
    load_tile(Q, static_cast<const float*>(a.q) + qh, r0, s.R);
    load_tile(dO, static_cast<const float*>(a.dO) + qh, r0, s.R);
    float lse[4], D[4], dq[4][8] = {};
    int seen[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + ty + 16 * i;
        const bool in = r < s.R;
        seen[i] = in ? attn_seen(s, len, r) : 0;
        lse[i] = in ? a.lse_in[(size_t)head * s.R + r] : 0.0f;
        D[i] = in ? a.D[(size_t)head * s.R + r] : 0.0f;
    }
    for (int t = 0; t < tiles; ++t) {
        __syncthreads();
        load_tile(K, static_cast<const float*>(a.k) + kh, t * kT, len);
        load_tile(V, static_cast<const float*>(a.v) + kh, t * kT, len);
        __syncthreads();
        Grad4 g;
        grad_tile(s, Q, K, dO, V, lse, D, seen, t * kT, tx, ty, g);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[(ty + 16 * i) * kPRow + tx + 16 * j] = g.ds[i][j];
        __syncthreads();
        mix_tile(S, K, tx, ty, dq);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + ty + 16 * i;
        if (r < s.R) store_row(static_cast<float*>(a.dq) + qh + (size_t)r * kDh, tx, dq[i]);
    }
}

// grid (key tiles, heads): dk and dv of 64 keys over all rows, in row order
__global__ void __launch_bounds__(256) attention_dkdv_simt_kernel(const AttnShape s, const AttnArgs a)
{
    extern __shared__ __align__(16) float sm[];
    float *K = sm, *V = K + kTileF, *Q = V + kTileF, *dO = Q + kTileF, *P = dO + kTileF, *S = P + kPF;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int head = blockIdx.y, b = head / s.Hk, k0 = blockIdx.x * kT;
    const int len = attn_len(s, a.kv_len, b);
    const size_t qh = (size_t)head * s.R * kDh, kh = (size_t)head * s.Lk * kDh;
    load_tile(K, static_cast<const float*>(a.k) + kh, k0, len);
    load_tile(V, static_cast<const float*>(a.v) + kh, k0, len);
    float dk[4][8] = {}, dv[4][8] = {};
    for (int r0 = 0; r0 < s.R && k0 < len; r0 += kT) {
        if (attn_seen_most(s, len, r0, min(r0 + kT, s.R) - 1) <= k0) continue;
        __syncthreads();
        load_tile(Q, static_cast<const float*>(a.q) + qh, r0, s.R);
        load_tile(dO, static_cast<const float*>(a.dO) + qh, r0, s.R);
        float lse[4], D[4];
        int seen[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + ty + 16 * i;
            const bool in = r < s.R;
            seen[i] = in ? attn_seen(s, len, r) : 0;
            lse[i] = in ? a.lse_in[(size_t)head * s.R + r] : 0.0f;
            D[i] = in ? a.D[(size_t)head * s.R + r] : 0.0f;
        }
        __syncthreads();
        Grad4 g;
        grad_tile(s, Q, K, dO, V, lse, D, seen, k0, tx, ty, g);
#pragma unroll
        for (int i = 0; i < 4; ++i)                    // transposed: row = key
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                P[(tx + 16 * j) * kPRow + ty + 16 * i] = g.p[i][j];
                S[(tx + 16 * j) * kPRow + ty + 16 * i] = g.ds[i][j];
            }
        __syncthreads();
        mix_tile(P, dO, tx, ty, dv);
        mix_tile(S, Q, tx, ty, dk);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = k0 + ty + 16 * i;
        if (j < s.Lk) {
            store_row(static_cast<float*>(a.dk) + kh + (size_t)j * kDh, tx, dk[i]);
            store_row(static_cast<float*>(a.dv) + kh + (size_t)j * kDh, tx, dv[i]);
        }
    }
}

template <typename K>
cudaError_t launch(K kernel, dim3 grid, size_t floats, const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    const size_t bytes = floats * sizeof(float);
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    kernel<<<grid, 256, bytes, st>>>(s, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_simt(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    return launch(attention_simt_kernel, dim3((s.R + kT - 1) / kT, s.heads, s.splits), 3 * kTileF + kPF, s, a, st);
}

template <typename T>
cudaError_t launch_attention_join(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    const long long rows = (long long)s.heads * s.R;
    attention_join_kernel<T><<<(unsigned)((rows + 7) / 8), 256, 0, st>>>(s, a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_attention_rowdot(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    const long long rows = (long long)s.heads * s.R;
    attention_rowdot_kernel<T><<<(unsigned)((rows + 31) / 32), 256, 0, st>>>(rows, static_cast<const T*>(a.dO),
                                                                           static_cast<const T*>(a.o_in), a.D, a.status);
    return cudaGetLastError();
}

cudaError_t launch_attention_backward_simt(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    cudaError_t e = launch(attention_dkdv_simt_kernel, dim3((s.Lk + kT - 1) / kT, s.heads), 4 * kTileF + 2 * kPF, s,
                           a, st);
    if (e != cudaSuccess) return e;
    return launch(attention_dq_simt_kernel, dim3((s.R + kT - 1) / kT, s.heads), 4 * kTileF + kPF, s, a, st);
}

#define ROLA_INSTANTIATE(T)                                                                                   \
    template cudaError_t launch_attention_join<T>(const AttnShape&, const AttnArgs&, cudaStream_t);           \
    template cudaError_t launch_attention_rowdot<T>(const AttnShape&, const AttnArgs&, cudaStream_t);
ROLA_INSTANTIATE(float)
ROLA_INSTANTIATE(__nv_bfloat16)
#undef ROLA_INSTANTIATE

}  // namespace rola
