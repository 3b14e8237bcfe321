// A linear layer's products on the 5th-generation tensor cores (bf16 operands, fp32 accumulation in TMEM).
//
//   Y = R + phi(X W^T + b);  dX = dZ W,  dW = dZ^T X
//
// One persistent warp-specialised kernel computes C(m, n) = sum_k A(m, k) B(n, k) with pairs of CTAs (clusters of two,
// one CTA an SM).  A pair has a tile of 256 x NT: CTA r holds rows 128 r .. of A and rows NT / 2 r .. of B in its shared
// memory, and the products of cta_group::2, which the pair's first CTA issues, read both CTAs' halves of B; its rows
// of the tile end up in each CTA's TMEM.  Against a CTA by itself the pair reads B from shared memory and L2 once instead
// of twice.  TMA brings both operands in steps of 64 k into 128-byte-swizzled rings; the copies of both CTAs arrive at
// the first one's mbarrier, the commits of its products at both.  The accumulator is double-buffered (2 x NT of 512
// columns), so that eight warps of each CTA take a tile from TMEM under the next tile's products.
//
// An operand is contiguous along k (K-major, boxes of 64 k) or along m / n (MN-major, boxes of 64 x 64 k); the tensor
// core reads either, so no operand is transposed in memory.  What lies past an edge is TMA's zero fill.
//
// Few tiles with a long K axis (the weights' gradients: K is the token) are split along K; the parts go to the
// workspace in fp32, and a second kernel adds them in order and finishes the outputs (launch_linear_join).
//
// Every mbarrier wait is bounded; a wait that gives up records ROLA_ERR_TIMEOUT in the status word, and the CTA stops
// issuing, lets what it issued complete, meets its pair and frees its TMEM.
#include <cudaTypedefs.h>

#include <type_traits>

#include "attention_tc.cuh"
#include "cluster.cuh"
#include "linear.cuh"
#include "linear_finish.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kHalfM = 128, kTileM = 2 * kHalfM, kStepK = 64, kGroupM = 8;
constexpr int kThreads = 320, kEpiWarps = 8;
constexpr uint32_t kABytes = kHalfM * kStepK * 2;
constexpr uint32_t kRingBytes = 192 * 1024;

template <int NT>
struct Cfg {
    static constexpr uint32_t kBBytes = NT / 2 * kStepK * 2, kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kRingBytes / kStageBytes;
    static constexpr int FULL = 0, EMPTY = FULL + kStages, ACC_FULL = EMPTY + kStages, ACC_EMPTY = ACC_FULL + 2,
                         DRAIN = ACC_EMPTY + 2, NUM_BARS = DRAIN + 1;
};
struct Ctrl {
    uint64_t bar[32];
    uint32_t tmem_base;
    int abort;
};
static_assert(Cfg<256>::NUM_BARS <= 32 && Cfg<128>::NUM_BARS <= 32, "mbarriers fit the control block");

struct Params {
    CUtensorMap a, b;
    LinearEnd end;                               // what becomes of the sums
    float* part;                                 // or, with splits, where they go: [splits][M][N]
    int M, N, m_tiles, n_tiles, k_steps, splits;
    int skip_first;                              // test hook: a CTA's first load is never issued
    int clear;                                   // the status word is this kernel's to clear
    DeviceStatus* status;
    uint64_t wait_limit_ns;
};

__device__ __forceinline__ void record_timeout(const Params& p, int where)
{
    if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 192 + where;
}

// Item i of the launch: (row tile, column tile) and K steps [k0, k1).  Splits outside, so that the pairs in flight share
// the same K range; row tiles in groups of kGroupM, column tiles outside, row tiles inside, so that they share a few
// column tiles of B and the group's rows of A in L2.
struct Item {
    int mt, nt, split, k0, k1;
};
__device__ __forceinline__ Item item_of(const Params& p, int i)
{
    Item t;
    const int tiles = p.m_tiles * p.n_tiles;
    t.split = i / tiles;
    i -= t.split * tiles;
    const int per_group = kGroupM * p.n_tiles, g = i / per_group;
    const int rows = min(kGroupM, p.m_tiles - g * kGroupM);
    i -= g * per_group;
    t.nt = i / rows;
    t.mt = g * kGroupM + i - t.nt * rows;
    t.k0 = (int)((long long)p.k_steps * t.split / p.splits);
    t.k1 = (int)((long long)p.k_steps * (t.split + 1) / p.splits);
    return t;
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32])
{
    tmem_ld16(taddr, *reinterpret_cast<float(*)[16]>(&v[0]));
    tmem_ld16(taddr + 16, *reinterpret_cast<float(*)[16]>(&v[16]));
    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&v[0]));
    reg_fence(*reinterpret_cast<float(*)[16]>(&v[16]));
}

// -- of a pair of CTAs

// A box into this CTA's shared memory, its bytes counted at an mbarrier of either CTA of the pair.
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const void* map, uint32_t bar, int x, int y)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n" ::"r"(
            dst),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                         uint32_t idesc, uint32_t accum)
{
    asm volatile(
        "{\n.reg .pred p;\n.reg .b64 da, db;\n"
        "setp.ne.b32 p, %6, 0;\n"
        "mov.b64 da, {%1, %2};\n"
        "mov.b64 db, {%3, %4};\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n}\n" ::"r"(d_tmem),
        "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accum)
        : "memory");
}
// Arrives on the mbarrier at this offset in both CTAs when every product issued so far is done.
__device__ __forceinline__ void pair_commit(uint32_t bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void remote_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t dst_smem, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(dst_smem), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(taddr), "r"(ncols) : "memory");
}

// END: the sums become outputs here (bias, phi, residual), PLAIN: rounded only, PART: kept in fp32 for a join.
enum Out { END, PLAIN, PART };

template <bool AMn, bool BMn, int OUT, int NT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) linear_gemm_kernel(const __grid_constant__ Params p)
{
    using C = Cfg<NT>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t sbase = smem_u32(smem_raw);           // 1024-byte aligned: there is no static shared memory
    Ctrl& cb = *reinterpret_cast<Ctrl*>(smem_raw + kRingBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    auto bar = [&](int i) { return smem_u32(&cb.bar[i]); };
    if (tid == 0) {
        cb.abort = 0;
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(bar(C::FULL + i), 1);
            mbar_init(bar(C::EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::ACC_FULL + i), 1);
            mbar_init(bar(C::ACC_EMPTY + i), 2 * kEpiWarps);
        }
        mbar_init(bar(C::DRAIN), 1);
        fence_mbar_init();
        // before any CTA can record a timeout, which takes 1 ms at least
        if (p.clear && blockIdx.x == 0) p.status->code = p.status->where = 0;
    }
    if (warp == 1) pair_tmem_alloc(smem_u32(&cb.tmem_base), 2 * NT);
    fence_before_sync();
    cluster_sync();
    fence_after_sync();
    const uint32_t tmem = cb.tmem_base;
    volatile int* abort = &cb.abort;
    const uint64_t limit = p.wait_limit_ns;
    const int items = p.m_tiles * p.n_tiles * p.splits;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer: a box per lane
        constexpr int kABoxes = AMn ? 2 : 1, kBBoxes = BMn ? NT / 128 : 1;
        constexpr uint32_t kBBox = BMn ? 8192 : C::kBBytes;
        bool ok = true;
        int g = 0;                                       // K steps issued by this CTA
        for (int i = pair; i < items && ok; i += pairs) {
            const Item t = item_of(p, i);
            const int m0 = t.mt * kTileM + rank * kHalfM, n0 = t.nt * NT + rank * (NT / 2);
            for (int ks = t.k0; ks < t.k1; ++ks, ++g) {
                const int s = g % C::kStages, k0 = ks * kStepK;
                if (g >= C::kStages) ok = mbar_wait(bar(C::EMPTY + s), ((g / C::kStages) - 1) & 1, abort, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                if (p.skip_first && g == 0) continue;
                if (lane == 0 && rank == 0) mbar_expect_tx(bar(C::FULL + s), 2 * C::kStageBytes);
                __syncwarp();
                const uint32_t dst = sbase + s * C::kStageBytes, full = peer(bar(C::FULL + s), 0);
                if (lane < kABoxes)
                    pair_load_2d(dst + lane * 8192, &p.a, full, AMn ? m0 + lane * 64 : k0, AMn ? k0 : m0);
                const int bl = lane - 2;
                if (bl >= 0 && bl < kBBoxes)
                    pair_load_2d(dst + kABytes + bl * kBBox, &p.b, full, BMn ? n0 + bl * 64 : k0, BMn ? k0 : n0);
            }
        }
        if (!ok && lane == 0) record_timeout(p, 1);
        // the pair's copies still in flight land, and the commits of its last products arrive, before either CTA goes on
        // to the last barrier and may leave
        if (lane == 0) {
            int never = 0;
            for (int u = g > C::kStages ? g - C::kStages : 0; u < g; ++u) {
                if (rank == 0) mbar_wait(bar(C::FULL + u % C::kStages), (u / C::kStages) & 1, &never, limit);
                if (!*abort && ok) ok = mbar_wait(bar(C::EMPTY + u % C::kStages), (u / C::kStages) & 1, abort, limit);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, issued by the first CTA
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = idesc_bf16(kTileM, NT, AMn, BMn);
            const uint64_t da = smem_desc(sbase, AMn ? 8192 : 16, 1024), db = smem_desc(sbase + kABytes, BMn ? 8192 : 16, 1024);
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            constexpr uint32_t a_k = AMn ? 128 : 2, b_k = BMn ? 128 : 2;    // 16 k: 16 rows of 128 B, or 32 B of a row
            bool ok = true;
            int g = 0, it = 0;
            for (int i = pair; i < items && ok; i += pairs, ++it) {
                const Item t = item_of(p, i);
                const int ab = it & 1;
                if (it >= 2 && !(ok = mbar_wait(bar(C::ACC_EMPTY + ab), ((it >> 1) - 1) & 1, abort, limit))) break;
                fence_after_sync();
                for (int ks = t.k0; ks < t.k1; ++ks, ++g) {
                    const int s = g % C::kStages;
                    if (!(ok = mbar_wait(bar(C::FULL + s), (g / C::kStages) & 1, abort, limit))) break;
                    fence_after_sync();
                    const uint32_t off = s * (C::kStageBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kStepK / 16; ++kk)
                        pair_mma(tmem + ab * NT, a_lo + off + kk * a_k, a_hi, b_lo + off + kk * b_k, b_hi, idesc,
                                 (ks > t.k0 || kk > 0) ? 1u : 0u);
                    pair_commit(bar(C::EMPTY + s));
                }
                if (!ok) break;
                pair_commit(bar(C::ACC_FULL + ab));
            }
            if (!ok) record_timeout(p, 2);
            pair_commit(bar(C::DRAIN));
        }
        // every product issued completes, and says so to both CTAs, before TMEM is released
        if (lane == 0) {
            int never = 0;
            mbar_wait(bar(C::DRAIN), 0, &never, 2 * limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue: two warps for each quarter of the rows
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        constexpr int kChunks = NT / 2 / 32;
        bool ok = true;
        int it = 0;
        for (int i = pair; i < items && ok; i += pairs, ++it) {
            const Item t = item_of(p, i);
            const int ab = it & 1;
            if (!(ok = mbar_wait_warp(bar(C::ACC_FULL + ab), (it >> 1) & 1, abort, limit))) break;
            fence_after_sync();
            const int row = t.mt * kTileM + rank * kHalfM + q * 32 + lane;
            for (int c = 0; c < kChunks; ++c) {
                const int col = half * (NT / 2) + c * 32, f0 = t.nt * NT + col;
                float v[32];
                tmem_ld32(tmem + lane_off + ab * NT + col, v);
                if (c == kChunks - 1) {          // in registers: the buffer is free for the tile after next
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) remote_arrive(peer(bar(C::ACC_EMPTY + ab), 0));
                }
                if (row >= p.M) continue;
                if constexpr (OUT == PART) {
                    float* to = p.part + ((size_t)t.split * p.M + row) * p.N + f0;
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (f0 + e < p.N) put8(to + e, v + e, p.end.wide);
                } else {
                    linear_end<OUT == END>(p.end, (size_t)row * p.N, f0, p.N, v);
                }
            }
        }
        if (!ok) record_timeout(p, 3);
    }
    fence_before_sync();
    cluster_sync();                                      // the pair's shared memory and TMEM stay until both are done
    fence_after_sync();
    if (warp == 1) pair_tmem_dealloc(tmem, 2 * NT);
}

// ---------------------------------------------------------------- host side

// [rows][cols] row-major, the operand of a product whose K (kc) or whose output index lies along cols
bool operand_map(CUtensorMap* m, const void* p, int rows, int cols, bool kc, int box_rows)
{
    return encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, rows, cols, kStepK, kc ? box_rows : kStepK,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool AMn, bool BMn, int OUT, int NT>
cudaError_t launch(const LinShape& s, Params& p, int pairs, cudaStream_t st)
{
    const size_t smem = kRingBytes + sizeof(Ctrl);
    auto kernel = linear_gemm_kernel<AMn, BMn, OUT, NT>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int items = p.m_tiles * p.n_tiles * p.splits;
    kernel<<<2 * (items < pairs ? items : pairs), kThreads, smem, st>>>(p);
    return cudaGetLastError();
}

// C [M][N] = sum over K of A B; OUT: END or PLAIN (without splits).
template <bool AMn, bool BMn, int OUT>
cudaError_t product(const LinShape& s, const void* A, const void* B, int M, int N, int K, const LinearEnd& end, float* part,
                    bool clear, DeviceStatus* status, cudaStream_t st)
{
    const LinearPlan plan = linear_plan(M, N, K);
    Params p{};
    p.M = M; p.N = N;
    p.m_tiles = (M + kTileM - 1) / kTileM;
    p.n_tiles = (N + plan.tile_n - 1) / plan.tile_n;
    p.k_steps = (K + kStepK - 1) / kStepK;
    p.splits = plan.splits;
    p.end = end;
    p.part = part;
    p.clear = clear;
    p.status = status;
    p.wait_limit_ns = s.wait_limit_ns;
    p.skip_first = s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY ? 1 : 0;
    if (!operand_map(&p.a, A, AMn ? K : M, AMn ? M : K, !AMn, kHalfM) ||
        !operand_map(&p.b, B, BMn ? K : N, BMn ? N : K, !BMn, plan.tile_n / 2))
        return cudaErrorInvalidValue;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const int pairs = nsm / 2;
    auto go = [&](auto out) {
        constexpr int O = decltype(out)::value;
        return plan.tile_n == 256 ? launch<AMn, BMn, O, 256>(s, p, pairs, st) : launch<AMn, BMn, O, 128>(s, p, pairs, st);
    };
    if (plan.splits == 1) return go(std::integral_constant<int, OUT>());
    e = go(std::integral_constant<int, PART>());
    return e == cudaSuccess ? launch_linear_join(end, part, plan.splits, M, N, st) : e;
}

}  // namespace

// Tile width and parts of K of least cost.  A pair takes 0.26 us a step of 64 k at 256 columns and 0.15 at 128, and some
// 2 us at its ends that no other tile covers; parts are written and read once more in fp32 at some 5 TB/s, and their
// join is a launch of 4 us.  76 pairs run at once.
LinearPlan linear_plan(int64_t M, int64_t N, int64_t K)
{
    const int64_t steps = (K + kStepK - 1) / kStepK;
    LinearPlan best{256, 1};
    double least = 1e30;
    for (int tile_n : {256, 128})
        for (int64_t splits = 1; splits <= 16 && splits * 4 <= steps + 3; ++splits) {
            const int64_t items = ((M + kTileM - 1) / kTileM) * ((N + tile_n - 1) / tile_n) * splits;
            const double turns = (double)((items + 75) / 76);
            const double us = turns * (double)((steps + splits - 1) / splits) * (tile_n == 256 ? 0.26 : 0.15) + 2.0 +
                              (splits > 1 ? 4.0 + 8.0 * (double)(splits * M * N) / 5e6 : 0.0);
            if (us < least * 0.999) {
                least = us;
                best = {tile_n, (int)splits};
            }
        }
    return best;
}

cudaError_t launch_linear_tc(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                             float* Z, float* part, DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(Y, b, R, Z, s.N, s.act);
    return product<false, false, END>(s, X, W, s.M, s.N, s.K, end, part, true, status, st);
}

cudaError_t launch_linear_dx_tc(const LinShape& s, const void* W, const void* dZ, void* dX, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(dX, nullptr, nullptr, nullptr, s.K, ROLA_LOWRANK_ACT_IDENTITY);
    return product<false, true, PLAIN>(s, dZ, W, s.M, s.K, s.N, end, part, clear, status, st);
}

cudaError_t launch_linear_dw_tc(const LinShape& s, const void* X, const void* dZ, void* dW, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(dW, nullptr, nullptr, nullptr, s.K, ROLA_LOWRANK_ACT_IDENTITY);
    return product<true, true, PLAIN>(s, dZ, X, s.N, s.K, s.M, end, part, clear, status, st);     // k = token
}

}  // namespace rola
