// The gated feed-forward's and the linear layer's products in plain fp32 arithmetic (no tensor
// cores): the fp32 mode.
//
//   Y = R + phi(X W^T + b);  dX = dZ W,  dW = dZ^T X
//   H = phi(X Wg^T) * (X Wu^T),  Y = H Wd^T
//   dG, dU, H from dH = dY Wd;  dX = dG Wg + dU Wu;  dWg = dG^T X,  dWu = dU^T X,  dWd = dY^T H
//
// One kernel computes C(m, n) = sum_k A(m, k) B(n, k) for 128 x 128 tiles, 256
// threads with 8 x 8 outputs each (two groups of four rows and of four columns,
// so that shared memory is read in 16-byte words without conflicts: 4 words for
// 64 fused multiply-adds), K in steps of 16, the next step's words loaded into
// registers under the present step's arithmetic.  Each operand is contiguous
// along k or along m / n.  The B tile of the gate + up kernel is 64 rows of Wg
// and the same 64 rows of Wu, so that a thread holds g and u of the same
// features (columns tx*4 .. and 64 + tx*4 ..) and phi and the product need no
// exchange.  Bound by fp32 FMA issue.
//
// Where the tiles leave SMs idle (94 tokens at d_model 1360: 11 tiles for dX)
// the K axis of a tile is split over a cluster of up to 8 CTAs, whose parts meet in
// their shared memory and are added in rank order, each CTA a share of the rows.
//
// Up to 32 tokens that tile would be mostly empty rows, and the weights are what
// has to be read.  Then a warp takes whole weight rows against 8 tokens (up and
// down, whose weights lie along k), or a CTA 64 weight columns against 8 tokens, its 32
// warps sharing the K axis (dH and dX, whose weights lie across it); the parts
// meet in a fixed order.
#include "block_ops.cuh"
#include "cluster.cuh"
#include "linear.cuh"

namespace rola {
namespace {

constexpr int kTile = 128, kStep = 16, kPad = 132;

enum Epilogue { kStore, kGateUp, kGateGrad, kLinear };

// An operand: element (i, k) at p[i * ld + k] (k contiguous) or p[k * ld + i].
// ld and the contiguous extent are multiples of 8 elements, p is 16-byte aligned.
struct Operand {
    const float* p;
    int rows;                    // extent of i
    int ld;
};

struct Args {
    int M, N, K, sources, act;
    int ldc;
    const float *G_in, *U_in;        // kLinear: the bias and the residual, or NULL
    float *G, *U;                    // kLinear: Z in G, or NULL
    void *C, *C2, *C3;
};

// One output of a linear layer from its sum over k.
__device__ __forceinline__ float finish_linear(const Args& p, size_t at, int n, float z)
{
    if (p.G_in) z += p.G_in[n];
    if (p.G) p.G[at] = z;
    const float y = gate_act(p.act, z);
    return p.U_in ? y + p.U_in[at] : y;
}

// This thread's 8 elements of a 128 x 16 tile: along k, row t / 2 and k = 8 (t % 2); along i, k = t / 16 and
// rows 8 (t % 16).  Elements outside the operand are 0.
template <bool KC>
__device__ __forceinline__ void fetch(const Operand& o, int i0, int k0, int K, float (&x)[8])
{
    const int t = threadIdx.x;
    const int i = KC ? i0 + t / 2 : i0 + (t % 16) * 8, k = KC ? k0 + (t % 2) * 8 : k0 + t / 16;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    // the contiguous extent is a multiple of 8, so the 8 elements are all inside or all outside
    if (i < o.rows && k < K) {
        const float* p = KC ? o.p + (size_t)i * o.ld + k : o.p + (size_t)k * o.ld + i;
        const float4 a = load4(p), b = load4(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}
template <bool KC>
__device__ __forceinline__ void stage(float (*s)[kPad], const float (&x)[8])
{
    const int t = threadIdx.x;
    if constexpr (KC) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[(t % 2) * 8 + e][t / 2] = x[e];
    } else {
        *reinterpret_cast<float4*>(&s[t / 16][(t % 16) * 8]) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(&s[t / 16][(t % 16) * 8 + 4]) = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// The B tile of kGateUp: rows 0-63 from b0, 64-127 from b1, the same 64 features.
template <bool BK, int E>
__device__ __forceinline__ void fetch_b(const Operand& b0, const Operand& b1, int n0, int k0, int K, float (&x)[8])
{
    if constexpr (E == kGateUp) {
        static_assert(BK, "the weights are contiguous along k");
        const bool up = threadIdx.x >= 128;
        fetch<true>(up ? b1 : b0, up ? n0 - 64 : n0, k0, K, x);
    } else {
        fetch<BK>(b0, n0, k0, K, x);
    }
}

// Four sums of row m from column n on (kGateUp: of the gate in c, of the same features' up in u) to their outputs.
template <int E>
__device__ __forceinline__ void finish(const Args& p, int m, int n, float4 c, float4 u)
{
    if (m >= p.M || n >= p.N) return;                  // N is a multiple of 8
    const size_t at = (size_t)m * p.ldc + n;
    if constexpr (E == kGateUp) {
        store4(static_cast<float*>(p.C) + at,
               make_float4(gate_act(p.act, c.x) * u.x, gate_act(p.act, c.y) * u.y, gate_act(p.act, c.z) * u.z,
                           gate_act(p.act, c.w) * u.w));
        if (p.G) {
            store4(p.G + at, c);
            store4(p.U + at, u);
        }
    } else if constexpr (E == kStore) {
        store4(static_cast<float*>(p.C) + at, c);
    } else if constexpr (E == kLinear) {
        store4(static_cast<float*>(p.C) + at,
               make_float4(finish_linear(p, at, n, c.x), finish_linear(p, at + 1, n + 1, c.y),
                           finish_linear(p, at + 2, n + 2, c.z), finish_linear(p, at + 3, n + 3, c.w)));
    } else {
        const float4 g4 = load4(p.G_in + at), u4 = load4(p.U_in + at);
        const float cc[4] = {c.x, c.y, c.z, c.w}, g[4] = {g4.x, g4.y, g4.z, g4.w}, uu[4] = {u4.x, u4.y, u4.z, u4.w};
        float hh[4], dg[4], du[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float ph, dph;
            gate_act_grad(p.act, g[e], ph, dph);
            hh[e] = ph * uu[e];
            dg[e] = cc[e] * uu[e] * dph;
            du[e] = cc[e] * ph;
        }
        store4(static_cast<float*>(p.C) + at, make_float4(hh[0], hh[1], hh[2], hh[3]));
        store4(static_cast<float*>(p.C2) + at, make_float4(dg[0], dg[1], dg[2], dg[3]));
        store4(static_cast<float*>(p.C3) + at, make_float4(du[0], du[1], du[2], du[3]));
    }
}

// acc += a b for a pair of b, each an IEEE fma: one instruction of two leaves issue slots to the loads from
// shared memory (2048 tokens at widths 1536 x 4096: 1980 us with one fma an instruction, 1790 so, both in one part a tile).
__device__ __forceinline__ void fma_pair(unsigned long long& acc, float a, unsigned long long b)
{
    asm("{\n.reg .b64 aa;\nmov.b64 aa, {%1, %1};\nfma.rn.f32x2 %0, aa, %2, %0;\n}\n" : "+l"(acc) : "f"(a), "l"(b));
}

constexpr size_t kStageBytes = 2 * 2 * kStep * kPad * 4, kSumBytes = (size_t)kTile * kPad * 4;

// SPLIT: the grid's z axis is a cluster that shares the K axis of a tile; its shared memory holds kSumBytes.
template <bool AK, bool BK, int E, bool SPLIT>
__global__ void __launch_bounds__(256, 2) simt_gemm_kernel(Operand a0, Operand b0, Operand a1, Operand b1,
                                                           const Args p)
{
    extern __shared__ __align__(16) float sm[];
    using Stage = float[kStep][kPad];
    Stage* as = reinterpret_cast<Stage*>(sm);
    Stage* bs = as + 2;
    constexpr int kColumns = E == kGateUp ? 64 : kTile;
    const int m0 = blockIdx.y * kTile, n0 = blockIdx.x * kColumns;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    unsigned long long sum[8][4] = {};                 // pairs of neighbouring columns
    const int steps = (p.K + kStep - 1) / kStep;
    int begin = 0, end = steps * p.sources;
    if constexpr (SPLIT) {
        begin = (int)((long long)steps * p.sources * blockIdx.z / gridDim.z);
        end = (int)((long long)steps * p.sources * (blockIdx.z + 1) / gridDim.z);
    }
    float xa[8], xb[8];
    auto next = [&](int s) {
        const bool second = s >= steps;                // dX: the second product of the sum
        const int k0 = (second ? s - steps : s) * kStep;
        fetch<AK>(second ? a1 : a0, m0, k0, p.K, xa);
        if constexpr (E == kGateUp) fetch_b<BK, E>(b0, b1, n0, k0, p.K, xb);
        else fetch_b<BK, E>(second ? b1 : b0, b1, n0, k0, p.K, xb);
    };
    next(begin);
    stage<AK>(as[0], xa);
    stage<BK>(bs[0], xb);
    __syncthreads();
    for (int s = begin; s < end; ++s) {
        if (s + 1 < end) next(s + 1);
        const int cur = (s - begin) & 1;
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            float a[8];
            *reinterpret_cast<float4*>(a) = *reinterpret_cast<const float4*>(&as[cur][k][ty * 4]);
            *reinterpret_cast<float4*>(a + 4) = *reinterpret_cast<const float4*>(&as[cur][k][64 + ty * 4]);
            const ulonglong2 b0 = *reinterpret_cast<const ulonglong2*>(&bs[cur][k][tx * 4]);
            const ulonglong2 b1 = *reinterpret_cast<const ulonglong2*>(&bs[cur][k][64 + tx * 4]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                fma_pair(sum[i][0], a[i], b0.x);
                fma_pair(sum[i][1], a[i], b0.y);
                fma_pair(sum[i][2], a[i], b1.x);
                fma_pair(sum[i][3], a[i], b1.y);
            }
        }
        if (s + 1 < end) {
            stage<AK>(as[cur ^ 1], xa);                // last read before the previous barrier
            stage<BK>(bs[cur ^ 1], xb);
        }
        __syncthreads();
    }
    float acc[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm("mov.b64 {%0, %1}, %2;" : "=f"(acc[i][2 * j]), "=f"(acc[i][2 * j + 1]) : "l"(sum[i][j]));
    if constexpr (SPLIT) {
        // this CTA's part of the tile into shared memory, over the stages, which all have read
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float* row = sm + (i < 4 ? ty * 4 + i : 60 + ty * 4 + i) * kPad;
            *reinterpret_cast<float4*>(row + tx * 4) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
            *reinterpret_cast<float4*>(row + 64 + tx * 4) = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
        }
        cluster_sync();
        const int parts = gridDim.z, rank = blockIdx.z;
        const uint32_t base = (uint32_t)__cvta_generic_to_shared(sm);
        auto total = [&](int row, int column) {
            const uint32_t at = base + (uint32_t)(row * kPad + column) * 4;
            float4 c = ld_peer(peer(at, 0));
            for (int r = 1; r < parts; ++r) {
                const float4 x = ld_peer(peer(at, r));
                c.x += x.x; c.y += x.y; c.z += x.z; c.w += x.w;
            }
            return c;
        };
        constexpr int kLanes = kColumns / 4;           // threads of a row
        const int row1 = kTile * (rank + 1) / parts, column = (int)threadIdx.x % kLanes * 4;
        for (int row = kTile * rank / parts + (int)threadIdx.x / kLanes; row < row1; row += 256 / kLanes) {
            if (m0 + row >= p.M) break;
            const float4 c = total(row, column);
            finish<E>(p, m0 + row, n0 + column, c, E == kGateUp ? total(row, 64 + column) : c);
        }
        cluster_sync();                                // the peers' shared memory stays until all have read it
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = m0 + (i < 4 ? ty * 4 + i : 60 + ty * 4 + i);
            const float4 c = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
            const float4 d = make_float4(acc[i][4], acc[i][5], acc[i][6], acc[i][7]);
            finish<E>(p, m, n0 + tx * 4, c, d);
            if constexpr (E != kGateUp) finish<E>(p, m, n0 + 64 + tx * 4, d, d);
        }
    }
}

// ---------------------------------------------------------------- few tokens

constexpr int kFewTokens = 32, kChunk = 8;       // most tokens; of a CTA

// Outputs n .. n + R - 1 of a warp for the 8 tokens from 8 blockIdx.y on: sum_k a(m, k) b(n, k), both
// contiguous along k.  kGateUp: R / 2 features, W_gate rows first.
template <int R, int E>
__global__ void __launch_bounds__(256) few_rows_kernel(Operand a, Operand b0, Operand b1, const Args p)
{
    constexpr int FEATURES = E == kGateUp ? R / 2 : R;
    const int lane = threadIdx.x & 31;
    const int n0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * FEATURES, m0 = blockIdx.y * kChunk;
    if (n0 >= p.N) return;
    float acc[R][kChunk] = {};
    for (int k = lane * 4; k < p.K; k += 128) {
        float4 w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int n = min(n0 + r % FEATURES, p.N - 1);
            w[r] = load4((r < FEATURES ? b0.p : b1.p) + (size_t)n * b0.ld + k);
        }
#pragma unroll
        for (int m = 0; m < kChunk; ++m) {
            const float4 x = load4(a.p + (size_t)min(m0 + m, p.M - 1) * a.ld + k);
#pragma unroll
            for (int r = 0; r < R; ++r)
                acc[r][m] = fmaf(x.x, w[r].x, fmaf(x.y, w[r].y, fmaf(x.z, w[r].z, fmaf(x.w, w[r].w, acc[r][m]))));
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < kChunk; ++m)
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) acc[r][m] += __shfl_xor_sync(0xffffffffu, acc[r][m], off);
    // lane m writes token m
#pragma unroll
    for (int m = 0; m < kChunk; ++m) {
        if (lane != m || m0 + m >= p.M) continue;
#pragma unroll
        for (int f = 0; f < FEATURES; ++f) {
            if (n0 + f >= p.N) continue;
            const size_t at = (size_t)(m0 + m) * p.ldc + n0 + f;
            if constexpr (E == kGateUp) {
                const float g = acc[f][m], u = acc[f + FEATURES][m];
                static_cast<float*>(p.C)[at] = gate_act(p.act, g) * u;
                if (p.G) {
                    p.G[at] = g;
                    p.U[at] = u;
                }
            } else if constexpr (E == kLinear) {
                static_cast<float*>(p.C)[at] = finish_linear(p, at, n0 + f, acc[f][m]);
            } else {
                static_cast<float*>(p.C)[at] = acc[f][m];
            }
        }
    }
}

// Columns 64 blockIdx.x .. of 8 tokens: sum_k a(m, k) b(k, n), b contiguous along n; `sources` such products.
template <int E>
__global__ void __launch_bounds__(1024) few_columns_kernel(Operand a0, Operand b0, Operand a1, Operand b1, const Args p)
{
    constexpr int kPart = 512;                   // of the K axis staged at a time
    __shared__ __align__(16) float as[kChunk][kPart];
    __shared__ __align__(16) float part[32][64];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = blockIdx.x * 64 + (lane & 15) * 4, m0 = blockIdx.y * kChunk;
    const bool in = n < p.N;                     // N is a multiple of 8
    float acc[kChunk][4] = {};
    for (int s = 0; s < p.sources; ++s) {
        const Operand &a = s ? a1 : a0, &b = s ? b1 : b0;
        for (int k0 = 0; k0 < p.K; k0 += kPart) {
            __syncthreads();
            for (int e = threadIdx.x; e < kChunk * kPart; e += 1024) {
                const int m = e / kPart, k = k0 + e % kPart;
                as[m][e % kPart] = k < p.K && m0 + m < p.M ? a.p[(size_t)(m0 + m) * a.ld + k] : 0.0f;
            }
            __syncthreads();
            const int end = min(kPart, p.K - k0);
#pragma unroll 4
            for (int k = warp * 2 + (lane >> 4); k < end; k += 64) {
                const float4 w = in ? load4(b.p + (size_t)(k0 + k) * b.ld + n) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int m = 0; m < kChunk; ++m) {
                    const float x = as[m][k];
                    acc[m][0] = fmaf(x, w.x, acc[m][0]);
                    acc[m][1] = fmaf(x, w.y, acc[m][1]);
                    acc[m][2] = fmaf(x, w.z, acc[m][2]);
                    acc[m][3] = fmaf(x, w.w, acc[m][3]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kChunk; ++m) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[m][e] += __shfl_xor_sync(0xffffffffu, acc[m][e], 16);
        __syncthreads();
        if (lane < 16)
            *reinterpret_cast<float4*>(&part[warp][lane * 4]) = make_float4(acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
        __syncthreads();
        const int c = threadIdx.x, col = blockIdx.x * 64 + c;
        if (c < 64 && col < p.N && m0 + m < p.M) {
            float x = 0.0f;
#pragma unroll
            for (int w = 0; w < 32; ++w) x += part[w][c];
            const size_t at = (size_t)(m0 + m) * p.ldc + col;
            if constexpr (E == kStore) {
                static_cast<float*>(p.C)[at] = x;
            } else {
                float ph, dph;
                gate_act_grad(p.act, p.G_in[at], ph, dph);
                const float u = p.U_in[at];
                static_cast<float*>(p.C)[at] = ph * u;
                static_cast<float*>(p.C2)[at] = x * u * dph;
                static_cast<float*>(p.C3)[at] = x * ph;
            }
        }
    }
}

// Rows per warp: four (the tokens' words are read once for them) where that still leaves 8 warps for each SM.
template <int E>
cudaError_t few_rows(Operand a, Operand b0, Operand b1, const Args& p, cudaStream_t st)
{
    const int chunks = (p.M + kChunk - 1) / kChunk, per = E == kGateUp ? 2 : 1;      // rows of a feature
    auto go = [&](auto kernel, int rows) {
        const int features = 8 * rows / per;                                         // of a CTA
        kernel<<<dim3((p.N + features - 1) / features, chunks), 256, 0, st>>>(a, b0, b1, p);
        return cudaGetLastError();
    };
    return (int64_t)p.N * per * chunks / 4 >= 8 * 152 ? go(few_rows_kernel<4, E>, 4) : go(few_rows_kernel<per, E>, per);
}
template <int E>
cudaError_t few_columns(Operand a0, Operand b0, Operand a1, Operand b1, const Args& p, cudaStream_t st)
{
    few_columns_kernel<E><<<dim3((p.N + 63) / 64, (p.M + kChunk - 1) / kChunk), 1024, 0, st>>>(a0, b0, a1, b1, p);
    return cudaGetLastError();
}

// Parts of a tile's K axis of `total` steps, 1, 2, 4 or 8 (the sizes of cluster that fill the SMs best), each of three steps at
// least: those of least cost in steps.  The SM with the most CTAs has n of them, two at a time; one alone takes
// 0.65 of the time of two, and the exchange of the parts about two steps.  (Few tiles: 94 tokens at widths 1360 x 8120, training,
// 3889 us in one part, 805 so.  A last turn of few CTAs: 2048 tokens at 1536 x 4096, 1790 us in one part, 1540 so.)
int parts_of(int64_t tiles, int64_t total)
{
    auto cost = [&](int64_t parts) {
        const int64_t n = (tiles * parts + 151) / 152;
        return ((double)(n / 2) + (n % 2 ? 0.65 : 0.0)) * ((double)total / (double)parts + (parts > 1 ? 2.0 : 0.0));
    };
    int best = 1;
    for (int parts = 2; parts <= 8 && total >= 3 * parts; parts *= 2)
        if (cost(parts) < cost(best)) best = parts;
    return best;
}

template <bool AK, bool BK, int E>
cudaError_t gemm(Operand a0, Operand b0, Operand a1, Operand b1, const Args& p, cudaStream_t st)
{
    if (p.M <= kFewTokens && AK) {               // (a weight's gradient has its token along k)
        if constexpr (BK) return few_rows<E>(a0, b0, b1, p, st);
        else if constexpr (AK) return few_columns<E>(a0, b0, a1, b1, p, st);
    }
    const int nt = E == kGateUp ? 64 : kTile;
    const dim3 grid((p.N + nt - 1) / nt, (p.M + kTile - 1) / kTile);
    const int parts = parts_of((int64_t)grid.x * grid.y, (int64_t)((p.K + kStep - 1) / kStep) * p.sources);
    if (parts < 2) {
        simt_gemm_kernel<AK, BK, E, false><<<grid, 256, kStageBytes, st>>>(a0, b0, a1, b1, p);
        return cudaGetLastError();
    }
    auto kernel = simt_gemm_kernel<AK, BK, E, true>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSumBytes);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid.x, grid.y, parts);
    cfg.blockDim = dim3(256);
    cfg.dynamicSmemBytes = kSumBytes;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = parts;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a0, b0, a1, b1, p);
}

}  // namespace

cudaError_t launch_ffn_up_simt(const FfnShape& s, const void* X, const void* Wg, const void* Wu, void* H, float* G,
                               float* U, cudaStream_t st)
{
    Args p{};
    p.M = s.M; p.N = s.F; p.K = s.D; p.sources = 1; p.act = s.act; p.ldc = s.F;
    p.C = H; p.G = G; p.U = U;
    const Operand x{static_cast<const float*>(X), s.M, s.D};
    return gemm<true, true, kGateUp>(x, {static_cast<const float*>(Wg), s.F, s.D}, x,
                                        {static_cast<const float*>(Wu), s.F, s.D}, p, st);
}

cudaError_t launch_ffn_down_simt(const FfnShape& s, const void* H, const void* Wd, void* Y, cudaStream_t st)
{
    Args p{};
    p.M = s.M; p.N = s.D; p.K = s.F; p.sources = 1; p.ldc = s.D;
    p.C = Y;
    const Operand h{static_cast<const float*>(H), s.M, s.F}, w{static_cast<const float*>(Wd), s.D, s.F};
    return gemm<true, true, kStore>(h, w, h, w, p, st);
}

cudaError_t launch_ffn_backward_simt(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd,
                                     const float* G, const float* U, const void* dY, void* H, void* dG, void* dU,
                                     void* dX, void* dWg, void* dWu, void* dWd, cudaStream_t st)
{
    auto op = [](const void* p, int rows, int ld) { return Operand{static_cast<const float*>(p), rows, ld}; };
    Args p{};
    p.M = s.M; p.N = s.F; p.K = s.D; p.sources = 1; p.act = s.act; p.ldc = s.F;
    p.G_in = G; p.U_in = U; p.C = H; p.C2 = dG; p.C3 = dU;
    cudaError_t e = gemm<true, false, kGateGrad>(op(dY, s.M, s.D), op(Wd, s.F, s.F), op(dY, s.M, s.D),
                                                    op(Wd, s.F, s.F), p, st);
    if (e != cudaSuccess) return e;
    p = Args{};
    p.M = s.M; p.N = s.D; p.K = s.F; p.sources = 2; p.ldc = s.D; p.C = dX;
    e = gemm<true, false, kStore>(op(dG, s.M, s.F), op(Wg, s.D, s.D), op(dU, s.M, s.F), op(Wu, s.D, s.D), p, st);
    if (e != cudaSuccess) return e;
    // the weights' gradients: both operands contiguous along their output index, k = token
    const struct { const void *a, *b; int m, n; void* c; } w[3] = {
        {dG, X, s.F, s.D, dWg}, {dU, X, s.F, s.D, dWu}, {dY, H, s.D, s.F, dWd}};
    for (const auto& g : w) {
        p = Args{};
        p.M = g.m; p.N = g.n; p.K = s.M; p.sources = 1; p.ldc = g.n; p.C = g.c;
        e = gemm<false, false, kStore>(op(g.a, g.m, g.m), op(g.b, g.n, g.n), op(g.a, g.m, g.m), op(g.b, g.n, g.n),
                                          p, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_linear_simt(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                               float* Z, cudaStream_t st)
{
    Args p{};
    p.M = s.M; p.N = s.N; p.K = s.K; p.sources = 1; p.act = s.act; p.ldc = s.N;
    p.C = Y; p.G = Z; p.G_in = static_cast<const float*>(b); p.U_in = static_cast<const float*>(R);
    const Operand x{static_cast<const float*>(X), s.M, s.K}, w{static_cast<const float*>(W), s.N, s.K};
    return gemm<true, true, kLinear>(x, w, x, w, p, st);
}

cudaError_t launch_linear_backward_simt(const LinShape& s, const void* X, const void* W, const void* dZ, void* dX,
                                        void* dW, cudaStream_t st)
{
    auto op = [](const void* p, int rows, int ld) { return Operand{static_cast<const float*>(p), rows, ld}; };
    if (dX) {
        Args p{};
        p.M = s.M; p.N = s.K; p.K = s.N; p.sources = 1; p.ldc = s.K; p.C = dX;
        const Operand dz = op(dZ, s.M, s.N), w = op(W, s.K, s.K);
        cudaError_t e = gemm<true, false, kStore>(dz, w, dz, w, p, st);
        if (e != cudaSuccess) return e;
    }
    if (!dW) return cudaSuccess;
    Args p{};                                    // k = token
    p.M = s.N; p.N = s.K; p.K = s.M; p.sources = 1; p.ldc = s.K; p.C = dW;
    const Operand dz = op(dZ, s.N, s.N), x = op(X, s.K, s.K);
    return gemm<false, false, kStore>(dz, x, dz, x, p, st);
}

}  // namespace rola
