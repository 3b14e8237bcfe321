// A linear layer's products on the 5th-generation tensor cores (bf16 operands, fp32 accumulation in TMEM).
//
//   Y = R + phi(X W^T + b);  dX = dZ W,  dW = dZ^T X
//
// One persistent warp-specialised kernel computes C(m, n) = sum_k A(m, k) B(n, k) in tiles of 128 x 256, one CTA per
// SM: TMA brings A and B in steps of 64 k into a ring of four stages in 128-byte-swizzled shared memory, one thread
// issues the products, eight warps take the tile from TMEM (two buffers of 256 columns) under the next tile's products.
// An operand is contiguous along k (K-major) or along m / n (MN-major), so that none is transposed in memory; what lies
// past an edge is TMA's zero fill.
//
// Every mbarrier wait is bounded; a wait that gives up records ROLA_ERR_TIMEOUT in the status word, and the CTA stops
// issuing, lets what it issued complete and frees its TMEM.
#include <cudaTypedefs.h>

#include "attention_tc.cuh"
#include "linear.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kTileM = 128, kTileN = 256, kStepK = 64, kGroupM = 16;
constexpr int kThreads = 320, kEpiWarps = 8, kStages = 4;
constexpr uint32_t kABytes = kTileM * kStepK * 2, kBBytes = kTileN * kStepK * 2, kStageBytes = kABytes + kBBytes;
constexpr uint32_t kSmemTiles = kStages * kStageBytes;

enum Bar { FULL = 0, EMPTY = FULL + kStages, ACC_FULL = EMPTY + kStages, ACC_EMPTY = ACC_FULL + 2, DRAIN = ACC_EMPTY + 2, NUM_BARS };
struct Ctrl {
    uint64_t bar[NUM_BARS];
    uint32_t tmem_base;
    int abort;
};

struct Params {
    CUtensorMap a, b;
    __nv_bfloat16* c;
    const __nv_bfloat16 *bias, *residual;        // or NULL
    float* Z;                                    // or NULL
    int M, N, m_tiles, n_tiles, k_steps, act;
    int wide;                                    // the outputs' rows are 32-byte aligned
    int skip_first;                              // test hook: a CTA's first load is never issued
    DeviceStatus* status;
    uint64_t wait_limit_ns;
};

__device__ __forceinline__ void record_timeout(const Params& p, int where)
{
    if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 192 + where;
}

__device__ __forceinline__ void tile_of(const Params& p, int t, int& mt, int& nt)
{
    const int per_group = kGroupM * p.n_tiles, g = t / per_group;
    const int rows = min(kGroupM, p.m_tiles - g * kGroupM);
    t -= g * per_group;
    nt = t / rows;
    mt = g * kGroupM + t - nt * rows;
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32])
{
    tmem_ld16(taddr, *reinterpret_cast<float(*)[16]>(&v[0]));
    tmem_ld16(taddr + 16, *reinterpret_cast<float(*)[16]>(&v[16]));
    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&v[0]));
    reg_fence(*reinterpret_cast<float(*)[16]>(&v[16]));
}


// Y of 32 columns: v += bias, Z kept, phi, + residual, one rounding.
template <bool EPI>
__device__ __forceinline__ void finish(const Params& p, size_t at, int f0, float (&v)[32])
{
    if constexpr (EPI) {
        if (p.bias)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
                if (f0 + e < p.N) {
                    float b[8];
                    load16(p.bias + f0 + e, b);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[e + j] += b[j];
                }
        if (p.Z)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
                if (f0 + e < p.N) {
                    float* z = p.Z + at + f0 + e;
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[e + j]);
                    if (p.wide) {
                        st_global32(z, w);
                    } else {
                        *reinterpret_cast<uint4*>(z) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(z + 4) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                }
        if (p.act != ROLA_LOWRANK_ACT_IDENTITY)
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = act.phi(v[j]);
            });
        if (p.residual)
#pragma unroll
            for (int e = 0; e < 32; e += 8)
                if (f0 + e < p.N) {
                    float r[8];
                    load16(p.residual + at + f0 + e, r);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[e + j] += r[j];
                }
    }
#pragma unroll
    for (int e = 0; e < 32; e += 16) {
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(v[e + 2 * j], v[e + 2 * j + 1]);
        __nv_bfloat16* row = p.c + at + f0 + e;
        if (f0 + e + 16 <= p.N) store_row32(row, y, p.wide);
        else if (f0 + e < p.N) *reinterpret_cast<uint4*>(row) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

template <bool AMn, bool BMn, bool EPI>
__global__ void __launch_bounds__(kThreads, 1) linear_gemm_kernel(const __grid_constant__ Params p)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {     // the 128-byte swizzle atoms need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(&p.status->code, 0, (int)ROLA_ERR_UNSUPPORTED);
        return;
    }
    Ctrl& cb = *reinterpret_cast<Ctrl*>(smem_raw + kSmemTiles);
    const uint32_t sbase = smem_u32(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&cb.bar[i]); };
    if (tid == 0) {
        cb.abort = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(bar(FULL + i), 1);
            mbar_init(bar(EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(ACC_FULL + i), 1);
            mbar_init(bar(ACC_EMPTY + i), kEpiWarps);
        }
        mbar_init(bar(DRAIN), 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&cb.tmem_base), 2 * kTileN);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = cb.tmem_base;
    volatile int* abort = &cb.abort;
    const uint64_t limit = p.wait_limit_ns;
    const int tiles = p.m_tiles * p.n_tiles;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: a box per lane
        constexpr int kABoxes = AMn ? 2 : 1, kBBoxes = BMn ? kTileN / 64 : 1;
        bool ok = true;
        int g = 0;
        for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
            int mt, nt;
            tile_of(p, t, mt, nt);
            for (int ks = 0; ks < p.k_steps; ++ks, ++g) {
                const int s = g % kStages, k0 = ks * kStepK;
                if (g >= kStages) ok = mbar_wait(bar(EMPTY + s), ((g / kStages) - 1) & 1, abort, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                const bool skip = p.skip_first && g == 0;
                if (lane == 0 && !skip) mbar_expect_tx(bar(FULL + s), kStageBytes);
                __syncwarp();
                const uint32_t dst = sbase + s * kStageBytes;
                if (lane < kABoxes && !skip)
                    tma_load_2d(dst + lane * 8192, &p.a, bar(FULL + s), AMn ? mt * kTileM + lane * 64 : k0, AMn ? k0 : mt * kTileM);
                const int bl = lane - 2;
                if (bl >= 0 && bl < kBBoxes && !skip)
                    tma_load_2d(dst + kABytes + bl * 8192, &p.b, bar(FULL + s), BMn ? nt * kTileN + bl * 64 : k0,
                                BMn ? k0 : nt * kTileN);
            }
        }
        if (!ok && lane == 0) record_timeout(p, 1);
        // the copies still in flight land before the CTA exits
        if (lane == 0) {
            int never = 0;
            for (int u = g > kStages ? g - kStages : 0; u < g; ++u)
                mbar_wait(bar(FULL + u % kStages), (u / kStages) & 1, &never, limit);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ products
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16(kTileM, kTileN, AMn, BMn);
            const uint64_t da = smem_desc(sbase, AMn ? 8192 : 16, 1024), db = smem_desc(sbase + kABytes, BMn ? 8192 : 16, 1024);
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            constexpr uint32_t a_k = AMn ? 128 : 2, b_k = BMn ? 128 : 2;    // 16 k: 16 rows of 128 B, or 32 B of a row
            bool ok = true;
            int g = 0, it = 0;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++it) {
                const int ab = it & 1;
                if (it >= 2 && !(ok = mbar_wait(bar(ACC_EMPTY + ab), ((it >> 1) - 1) & 1, abort, limit))) break;
                fence_after_sync();
                for (int ks = 0; ks < p.k_steps; ++ks, ++g) {
                    const int s = g % kStages;
                    if (!(ok = mbar_wait(bar(FULL + s), (g / kStages) & 1, abort, limit))) break;
                    fence_after_sync();
                    const uint32_t off = s * (kStageBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kStepK / 16; ++kk)
                        mma_ss_split(tmem + ab * kTileN, a_lo + off + kk * a_k, a_hi, b_lo + off + kk * b_k, b_hi, idesc,
                                     (ks > 0 || kk > 0) ? 1u : 0u);
                    mma_commit(bar(EMPTY + s));
                }
                if (!ok) break;
                mma_commit(bar(ACC_FULL + ab));
            }
            if (!ok) record_timeout(p, 2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(DRAIN));
            mbar_wait(bar(DRAIN), 0, &never, limit);
        }
    } else {
        // ------------------------------------------------------------ epilogue: two warps for each quarter of the rows
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        constexpr int kChunks = kTileN / 2 / 32;
        bool ok = true;
        int it = 0;
        for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x, ++it) {
            int mt, nt;
            tile_of(p, t, mt, nt);
            const int ab = it & 1;
            if (!(ok = mbar_wait_warp(bar(ACC_FULL + ab), (it >> 1) & 1, abort, limit))) break;
            fence_after_sync();
            const int row = mt * kTileM + q * 32 + lane;
            for (int c = 0; c < kChunks; ++c) {
                const int col = half * (kTileN / 2) + c * 32;
                float v[32];
                tmem_ld32(tmem + lane_off + ab * kTileN + col, v);
                if (c == kChunks - 1) {          // in registers: the buffer is free for the tile after next
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(ACC_EMPTY + ab));
                }
                if (row < p.M) finish<EPI>(p, (size_t)row * p.N, nt * kTileN + col, v);
            }
        }
        if (!ok) record_timeout(p, 3);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, 2 * kTileN);
}

// ---------------------------------------------------------------- host side

// [rows][cols] row-major, the operand of a product whose K (kc) or whose output index lies along cols
bool operand_map(CUtensorMap* m, const void* p, int rows, int cols, bool kc, int box_rows)
{
    return encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, rows, cols, kStepK, kc ? box_rows : kStepK,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool AMn, bool BMn, bool EPI>
cudaError_t launch(const LinShape& s, Params& p, int M, int N, int K, DeviceStatus* status, cudaStream_t st)
{
    p.M = M; p.N = N;
    p.m_tiles = (M + kTileM - 1) / kTileM;
    p.n_tiles = (N + kTileN - 1) / kTileN;
    p.k_steps = (K + kStepK - 1) / kStepK;
    p.act = s.act;
    p.wide = N % 16 == 0 && ((reinterpret_cast<uintptr_t>(p.c) | reinterpret_cast<uintptr_t>(p.Z)) & 31u) == 0;
    p.status = status;
    p.wait_limit_ns = s.wait_limit_ns;
    p.skip_first = s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY ? 1 : 0;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = kSmemTiles + sizeof(Ctrl);
    auto kernel = linear_gemm_kernel<AMn, BMn, EPI>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int tiles = p.m_tiles * p.n_tiles;
    kernel<<<tiles < nsm ? tiles : nsm, kThreads, smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_linear_tc(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                             float* Z, DeviceStatus* status, cudaStream_t st)
{
    Params p{};
    if (!operand_map(&p.a, X, s.M, s.K, true, kTileM) || !operand_map(&p.b, W, s.N, s.K, true, kTileN))
        return cudaErrorInvalidValue;
    p.c = static_cast<__nv_bfloat16*>(Y);
    p.bias = static_cast<const __nv_bfloat16*>(b);
    p.residual = static_cast<const __nv_bfloat16*>(R);
    p.Z = Z;
    return launch<false, false, true>(s, p, s.M, s.N, s.K, status, st);
}

cudaError_t launch_linear_backward_tc(const LinShape& s, const void* X, const void* W, const void* dZ, void* dX,
                                      void* dW, DeviceStatus* status, cudaStream_t st)
{
    if (dX) {
        Params p{};
        if (!operand_map(&p.a, dZ, s.M, s.N, true, kTileM) || !operand_map(&p.b, W, s.N, s.K, false, 0))
            return cudaErrorInvalidValue;
        p.c = static_cast<__nv_bfloat16*>(dX);
        cudaError_t e = launch<false, true, false>(s, p, s.M, s.K, s.N, status, st);
        if (e != cudaSuccess) return e;
    }
    if (!dW) return cudaSuccess;
    Params p{};                                  // k = token
    if (!operand_map(&p.a, dZ, s.M, s.N, false, 0) || !operand_map(&p.b, X, s.M, s.K, false, 0)) return cudaErrorInvalidValue;
    p.c = static_cast<__nv_bfloat16*>(dW);
    return launch<true, true, false>(s, p, s.N, s.K, s.M, status, st);
}

}  // namespace rola
