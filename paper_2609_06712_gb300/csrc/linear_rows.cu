// A linear layer for up to four tokens (bf16): every weight is read once for them, and nothing else counts.
//
//   Y = R + phi(X W^T + b)
//
// For weights of up to 32 MB, whose time is latency: of the loads, of the sums, of the call.  A warp takes R weight rows, 16
// bytes of each a lane and step, against all tokens, whose words it reads from L1; the products are added in fp32 in each
// lane and then over the lanes.  Plain loads: with no tensor maps, shared-memory limits or clusters to set up a call costs
// the host a launch, which is most of a small layer's time, and the weights need no more (a tile of the tensor cores would
// be 16 columns for one token).
//
// Where rows are few, or the axis long, `ways` warps of a CTA share a row's K axis and meet in shared memory in warp order.
#include "linear.cuh"

namespace rola {
namespace {

constexpr int kWarps = 8;

// f32x2: (a.x b.x + c.x, a.y b.y + c.y)
__device__ __forceinline__ void fma_pairs(float2& c, float2 a, float2 b)
{
    asm("{\n.reg .b64 ra, rb, rc;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmov.b64 rc, {%0, %1};\n"
        "fma.rn.f32x2 rc, ra, rb, rc;\nmov.b64 {%0, %1}, rc;\n}\n"
        : "+f"(c.x), "+f"(c.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
}

template <int M, int R>
__global__ void __launch_bounds__(32 * kWarps) linear_rows_kernel(int tokens, int K, int N, int act, int ways,
                                                                  const __nv_bfloat16* __restrict__ X,
                                                                  const __nv_bfloat16* __restrict__ W,
                                                                  const __nv_bfloat16* __restrict__ b,
                                                                  const __nv_bfloat16* residual, __nv_bfloat16* Y,
                                                                  float* __restrict__ Z, DeviceStatus* __restrict__ status)
{
    __shared__ float part[kWarps][R * M];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, way = warp % ways;
    if (blockIdx.x == 0 && threadIdx.x == 0) status->code = status->where = 0;
    const int n0 = (blockIdx.x * (kWarps / ways) + warp / ways) * R;
    float2 acc[R][M] = {};
    if (n0 < N) {
        const __nv_bfloat16* w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = W + (size_t)min(n0 + r, N - 1) * K;
#pragma unroll 4
        for (int k = (way * 32 + lane) * 8; k < K; k += ways * 256) {        // K is a multiple of 8
            uint4 x[M], y[R];
#pragma unroll
            for (int r = 0; r < R; ++r) y[r] = __ldcs(reinterpret_cast<const uint4*>(w[r] + k));
#pragma unroll
            for (int m = 0; m < M; ++m) x[m] = __ldg(reinterpret_cast<const uint4*>(X + (size_t)min(m, tokens - 1) * K + k));
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float2 f = unpack_bf16((&y[r].x)[e]);
#pragma unroll
                    for (int m = 0; m < M; ++m) fma_pairs(acc[r][m], f, unpack_bf16((&x[m].x)[e]));
                }
        }
    }
    float mine = 0.0f;                                       // lane i: output i of R M
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float s = acc[r][m].x + acc[r][m].y;
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (lane == r * M + m) mine = s;
        }
    if (ways > 1) {
        if (lane < R * M) part[warp][lane] = mine;
        __syncthreads();
        if (way) return;
        if (lane < R * M)
            for (int i = 1; i < ways; ++i) mine += part[warp + i][lane];
    }
    const int n = n0 + lane / M, m = lane % M;
    if (lane >= R * M || n >= N || m >= tokens) return;
    const size_t at = (size_t)m * N + n;
    float z = mine;
    if (b) z += __bfloat162float(b[n]);
    if (Z) Z[at] = z;
    float y = gate_act(act, z);
    if (residual) y += __bfloat162float(residual[at]);
    Y[at] = __float2bfloat16_rn(y);
}

template <int M>
cudaError_t rows_of(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y, float* Z,
                    DeviceStatus* status, cudaStream_t st)
{
    auto go = [&](auto kernel, int rows, int ways) {
        const int per_cta = kWarps / ways * rows;
        kernel<<<(s.N + per_cta - 1) / per_cta, 32 * kWarps, 0, st>>>(
            s.M, s.K, s.N, s.act, ways, static_cast<const __nv_bfloat16*>(X), static_cast<const __nv_bfloat16*>(W),
            static_cast<const __nv_bfloat16*>(b), static_cast<const __nv_bfloat16*>(R), static_cast<__nv_bfloat16*>(Y), Z,
            status);
        return cudaGetLastError();
    };
    // as many rows a warp as leave 16 warps to each of 152 SMs (the tokens' words are read once for them), then as many warps a
    // row as have 256 elements each
    constexpr int kWant = 16 * 152;
    if (s.N >= 4 * kWant) return go(linear_rows_kernel<M, 4>, 4, 1);
    if (s.N >= 2 * kWant) return go(linear_rows_kernel<M, 2>, 2, 1);
    int ways = 1;
    while (ways < kWarps && (int64_t)s.N * ways < kWant && s.K >= ways * 512) ways *= 2;
    return go(linear_rows_kernel<M, 1>, 1, ways);
}

}  // namespace

// Up to four tokens, and weights of up to 32 MB.  Us, this form / weight tiles (ffn_few.cu), weights from HBM, one token
// and four:  256 x 1536: 2.0, 2.4 / 4.6, 4.8;  1536 x 9216: 7.2, 9.3 / 10.0, 10.3;  8192 x 1024: 6.3, 8.5 / 11.6, 11.6;
// 4096 x 5120: 12.3, 16.1 / 11.5, 11.3;  5120 x 30720: 52, 94 / 51, 52.
bool linear_by_rows(const LinShape& s) { return s.M <= 4 && (int64_t)s.K * s.N <= 16000000; }

cudaError_t launch_linear_rows(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                               float* Z, DeviceStatus* status, cudaStream_t st)
{
    if (s.M == 1) return rows_of<1>(s, X, W, b, R, Y, Z, status, st);
    if (s.M == 2) return rows_of<2>(s, X, W, b, R, Y, Z, status, st);
    return rows_of<4>(s, X, W, b, R, Y, Z, status, st);
}

}  // namespace rola
