// A linear layer's products on the 5th-generation tensor cores (bf16 operands, fp32 accumulation in TMEM).
//
//   Y = R + phi(X W^T + b);  dX = dZ W,  dW = dZ^T X
//
// One persistent warp-specialised kernel computes C(m, n) = sum_k A(m, k) B(n, k) with pairs of CTAs (clusters of two,
// one CTA an SM).  A pair has a tile of 256 x 256: CTA r holds rows 128 r .. of A and rows 128 r .. of B in its shared
// memory, and the products of cta_group::2, which the pair's first CTA issues, read both CTAs' halves of B; its rows
// of the tile end up in each CTA's TMEM.  Against a CTA by itself the pair reads B from shared memory and L2 once instead
// of twice.  TMA brings both operands in steps of 64 k into 128-byte-swizzled rings; the copies of both CTAs arrive at
// the first one's mbarrier, the commits of its products at both.  The accumulator is double-buffered (2 x 256 of 512
// columns), so that eight warps of each CTA take a tile from TMEM under the next tile's products.
//
// An operand is contiguous along k (K-major, boxes of 64 k) or along m / n (MN-major, boxes of 64 x 64 k); the tensor
// core reads either, so no operand is transposed in memory.  What lies past an edge is TMA's zero fill.
//
// Epilogue: an epilogue warp has 32 rows and half of the columns.  It takes 32 columns at a time from TMEM, finishes them
// (bias, Z, phi, residual) and puts them into 4 KB of shared memory, from where a TMA store writes 32 x 64 of them; the
// residual comes into the same 4 KB by a TMA load that starts under the products.  (Rows stored by their lanes, 32 bytes
// each, kept the loads of the products waiting: 16380 x 5120 x 5120 with a residual 517 us, without any store 456.)
//
// Few tiles with a long K axis (the weights' gradients: K is the token) are split along K; the parts go to the
// workspace in fp32, and a second kernel adds them in order and finishes the outputs (launch_linear_join).
//
// Measured, bf16, between GPUs (whose power cap differs): 16380 x 5120 x 5120 with a residual 457 to 496 us (1732 to 1877
// TFLOP/s, 89 % of the tensor pipe), 32760 x 1536 x 4608 254 to 270 us (1717 to 1825), 8190 x 1536 x 6144 with GELU 101 us
// (1530), 514 x 4096 x 5120 with GELU 27 us.  What a large one lacks is the last turn of tiles; what a small one lacks are its
// ends (some 5 us) and pairs without a tile.
//
// Every mbarrier wait is bounded; a wait that gives up records ROLA_ERR_TIMEOUT in the status word, and the CTA stops
// issuing, lets what it issued complete, meets its pair and frees its TMEM.
#include <cudaTypedefs.h>

#include "attention_tc.cuh"
#include "cluster.cuh"
#include "linear.cuh"
#include "linear_finish.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kHalfM = 128, kTileM = 2 * kHalfM, kTileN = 256, kStepK = 64, kGroupM = 8;
constexpr int kThreads = 320, kEpiWarps = 8;
constexpr uint32_t kABytes = kHalfM * kStepK * 2, kBBytes = kTileN / 2 * kStepK * 2, kStageBytes = kABytes + kBBytes;
constexpr uint32_t kPieceBytes = 4096;                       // an epilogue warp's 32 rows of 128 bytes

// END: the sums become outputs here (bias, phi, residual); END_Z: and Z is kept; PLAIN: they are rounded only; PART: kept
// in fp32 for a join.
enum Out { END, END_Z, PLAIN, PART };

template <int OUT>
struct Cfg {
    static constexpr int kPieces = OUT == END_Z ? 2 : 1;     // of a warp: of Y and the residual, and of Z
    static constexpr int kStages = OUT == END_Z ? 5 : 6;
    static constexpr uint32_t kSmemEpi = kStages * kStageBytes, kSmemTiles = kSmemEpi + kEpiWarps * kPieces * kPieceBytes;
};
constexpr int kMaxStages = 6;
enum Bar { FULL = 0, EMPTY = FULL + kMaxStages, ACC_FULL = EMPTY + kMaxStages, ACC_EMPTY = ACC_FULL + 2,
           DRAIN = ACC_EMPTY + 2, RES = DRAIN + 1, NUM_BARS = RES + kEpiWarps };
struct Ctrl {
    uint64_t bar[NUM_BARS];
    alignas(16) __nv_bfloat16 bias[kEpiWarps][kTileN / 2];   // of an epilogue warp's columns of the present tile
    uint32_t tmem_base;
    int abort;
};
static_assert(Cfg<END_Z>::kSmemTiles + sizeof(Ctrl) <= 232448 && Cfg<END>::kSmemTiles + sizeof(Ctrl) <= 232448,
              "tiles and control block fit the 227 KB a CTA may have");

struct Params {
    CUtensorMap a, b;
    CUtensorMap c, residual, z;                  // outputs in pieces; PART: the parts, in c
    const __nv_bfloat16* bias;                   // or NULL
    int act, add;                                // add: there is a residual
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

// 16 bytes c of row `lane` of a piece (128-byte swizzle)
__device__ __forceinline__ uint32_t in_piece(uint32_t piece, int lane, int c) { return piece + lane * 128 + ((c ^ (lane & 7)) << 4); }
__device__ __forceinline__ void put16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 get16(uint32_t at)
{
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}

template <bool AMn, bool BMn, int OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1) linear_gemm_kernel(const __grid_constant__ Params p)
{
    using C = Cfg<OUT>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t sbase = smem_u32(smem_raw);           // 1024-byte aligned: there is no static shared memory
    Ctrl& cb = *reinterpret_cast<Ctrl*>(smem_raw + C::kSmemTiles);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    auto bar = [&](int i) { return smem_u32(&cb.bar[i]); };
    if (tid == 0) {
        cb.abort = 0;
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(bar(FULL + i), 1);
            mbar_init(bar(EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(ACC_FULL + i), 1);
            mbar_init(bar(ACC_EMPTY + i), 2 * kEpiWarps);
        }
        mbar_init(bar(DRAIN), 1);
        for (int i = 0; i < kEpiWarps; ++i) mbar_init(bar(RES + i), 1);
        fence_mbar_init();
        // before any CTA can record a timeout, which takes 1 ms at least
        if (p.clear && blockIdx.x == 0) p.status->code = p.status->where = 0;
        tma_prefetch_desc(&p.a);
        tma_prefetch_desc(&p.b);
        tma_prefetch_desc(&p.c);
    }
    if (warp == 1) pair_tmem_alloc(smem_u32(&cb.tmem_base), 2 * kTileN);
    fence_before_sync();
    cluster_sync();
    fence_after_sync();
    const uint32_t tmem = cb.tmem_base;
    volatile int* abort = &cb.abort;
    const uint64_t limit = p.wait_limit_ns;
    const int items = p.m_tiles * p.n_tiles * p.splits;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer, one lane: a step costs it a wait and the
        // copies.  (Lanes that share a step's copies meet once a step: 8192 x 5120 x 5120 268 us, so 252.)
        if (lane == 0) {
            constexpr int kABoxes = AMn ? 2 : 1, kBBoxes = BMn ? 2 : 1;
            const uint32_t full0 = peer(bar(FULL), 0);   // the first CTA's
            bool ok = true;
            int g = 0, s = 0, parity = 1;                // K steps issued; the present one's stage, and its last use
            for (int i = pair; i < items && ok; i += pairs) {
                const Item t = item_of(p, i);
                const int m0 = t.mt * kTileM + rank * kHalfM, n0 = t.nt * kTileN + rank * (kTileN / 2);
                for (int ks = t.k0; ks < t.k1; ++ks, ++g) {
                    if (g >= C::kStages && !(ok = mbar_wait(bar(EMPTY + s), parity, abort, limit))) break;
                    const uint32_t dst = sbase + s * kStageBytes, full = full0 + s * 8;
                    const int k0 = ks * kStepK;
                    if (!(p.skip_first && g == 0)) {
                        if (rank == 0) mbar_expect_tx(bar(FULL + s), 2 * kStageBytes);
#pragma unroll
                        for (int e = 0; e < kABoxes; ++e)
                            pair_load_2d(dst + e * 8192, &p.a, full, AMn ? m0 + e * 64 : k0, AMn ? k0 : m0);
#pragma unroll
                        for (int e = 0; e < kBBoxes; ++e)
                            pair_load_2d(dst + kABytes + e * 8192, &p.b, full, BMn ? n0 + e * 64 : k0, BMn ? k0 : n0);
                    }
                    if (++s == C::kStages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
            }
            if (!ok) record_timeout(p, 1);
            // the pair's copies still in flight land, and the commits of its last products arrive, before either CTA
            // goes on to the last barrier and may leave
            int never = 0;
            for (int u = g > C::kStages ? g - C::kStages : 0; u < g; ++u) {
                if (rank == 0) mbar_wait(bar(FULL + u % C::kStages), (u / C::kStages) & 1, &never, limit);
                if (!*abort && ok) ok = mbar_wait(bar(EMPTY + u % C::kStages), (u / C::kStages) & 1, abort, limit);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, issued by the first CTA
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = idesc_bf16(kTileM, kTileN, AMn, BMn);
            const uint64_t da = smem_desc(sbase, AMn ? 8192 : 16, 1024), db = smem_desc(sbase + kABytes, BMn ? 8192 : 16, 1024);
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            constexpr uint32_t a_k = AMn ? 128 : 2, b_k = BMn ? 128 : 2;    // 16 k: 16 rows of 128 B, or 32 B of a row
            bool ok = true;
            int s = 0, parity = 0, it = 0;
            for (int i = pair; i < items && ok; i += pairs, ++it) {
                const Item t = item_of(p, i);
                const int ab = it & 1;
                if (it >= 2 && !(ok = mbar_wait(bar(ACC_EMPTY + ab), ((it >> 1) - 1) & 1, abort, limit))) break;
                fence_after_sync();
                for (int ks = t.k0; ks < t.k1; ++ks) {
                    if (!(ok = mbar_wait(bar(FULL + s), parity, abort, limit))) break;
                    fence_after_sync();
                    const uint32_t off = s * (kStageBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kStepK / 16; ++kk)
                        pair_mma(tmem + ab * kTileN, a_lo + off + kk * a_k, a_hi, b_lo + off + kk * b_k, b_hi, idesc,
                                 (ks > t.k0 || kk > 0) ? 1u : 0u);
                    pair_commit(bar(EMPTY + s));
                    if (++s == C::kStages) {
                        s = 0;
                        parity ^= 1;
                    }
                }
                if (!ok) break;
                pair_commit(bar(ACC_FULL + ab));
            }
            if (!ok) record_timeout(p, 2);
            pair_commit(bar(DRAIN));
        }
        // every product issued completes, and says so to both CTAs, before TMEM is released
        if (lane == 0) {
            int never = 0;
            mbar_wait(bar(DRAIN), 0, &never, 2 * limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue: two warps for each quarter of the rows
        const int q = warp & 3, ew = warp - 2, half = ew >> 2;
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t piece = sbase + C::kSmemEpi + ew * C::kPieces * kPieceBytes, zpiece = piece + kPieceBytes;
        constexpr bool kEnd = OUT == END || OUT == END_Z;
        constexpr int kCols = OUT == PART ? 32 : 64, kChunks = kTileN / 2 / kCols;       // of a piece
        bool ok = true;
        int it = 0, asked = 0, got = 0;                  // residual pieces
        // the piece is free (its last store has read it, and every lane the last tile's bias), and the residual's part at (x, y) on its way into it
        auto begin = [&](int x, int y) {
            if (lane == 0) {
                bulk_wait_read_all();
                if (kEnd && p.add && x < p.N && y < p.M) {
                    mbar_expect_tx(bar(RES + ew), kPieceBytes);
                    tma_load_2d(piece, &p.residual, bar(RES + ew), x, y);
                }
            }
            if (kEnd && p.add && x < p.N && y < p.M) ++asked;
            __syncwarp();
        };
        for (int i = pair; i < items && ok; i += pairs, ++it) {
            const Item t = item_of(p, i);
            const int ab = it & 1, y = t.mt * kTileM + rank * kHalfM + q * 32, x0 = t.nt * kTileN + half * (kTileN / 2);
            begin(x0, y);
            if (kEnd && p.bias) {                        // four columns a lane; N is a multiple of 8
                const int x = min(x0 + lane * 4, p.N - 4);
                *reinterpret_cast<uint2*>(&cb.bias[ew][lane * 4]) = *reinterpret_cast<const uint2*>(p.bias + x);
                __syncwarp();
            }
            if (!(ok = mbar_wait_warp(bar(ACC_FULL + ab), (it >> 1) & 1, abort, limit))) break;
            fence_after_sync();
            for (int c = 0; c < kChunks && ok; ++c) {
                const int x = x0 + c * kCols;
                const bool in = x < p.N && y < p.M;      // of the warp: else nothing of the piece is inside
                if (c > 0) begin(x, y);
                if (got < asked) {
                    if (!(ok = mbar_wait_warp(bar(RES + ew), got & 1, abort, limit))) break;
                    ++got;
                }
#pragma unroll
                for (int h = 0; h < kCols / 32; ++h) {
                    float v[32];
                    tmem_ld32(tmem + lane_off + ab * kTileN + half * (kTileN / 2) + c * kCols + h * 32, v);
                    if (c == kChunks - 1 && h == kCols / 32 - 1) {       // in registers: the buffer is free for the tile after next
                        fence_before_sync();
                        __syncwarp();
                        if (lane == 0) remote_arrive(peer(bar(ACC_EMPTY + ab), 0));
                    }
                    if (!in) continue;
                    if constexpr (kEnd) {
                        if (p.bias)
#pragma unroll
                            for (int e = 0; e < 32; e += 8) {
                                float b[8];
                                load16(&cb.bias[ew][c * kCols + h * 32 + e], b);
#pragma unroll
                                for (int j = 0; j < 8; ++j) v[e + j] += b[j];
                            }
                        if constexpr (OUT == END_Z) {
                            if (lane == 0) bulk_wait_read_all();
                            __syncwarp();
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                put16(in_piece(zpiece, lane, e), __float_as_uint(v[4 * e]), __float_as_uint(v[4 * e + 1]),
                                      __float_as_uint(v[4 * e + 2]), __float_as_uint(v[4 * e + 3]));
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0 && x + h * 32 < p.N) {
                                tma_store_2d(&p.z, zpiece, x + h * 32, y);
                                bulk_commit();
                            }
                        }
                        linear_phi(p.act, v);
                        if (p.add)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint4 r = get16(in_piece(piece, lane, h * 4 + e));
                                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float2 f = unpack_bf16(w[j]);
                                    v[8 * e + 2 * j] += f.x;
                                    v[8 * e + 2 * j + 1] += f.y;
                                }
                            }
                    }
                    if constexpr (OUT == PART) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            put16(in_piece(piece, lane, e), __float_as_uint(v[4 * e]), __float_as_uint(v[4 * e + 1]),
                                  __float_as_uint(v[4 * e + 2]), __float_as_uint(v[4 * e + 3]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            put16(in_piece(piece, lane, h * 4 + e), pack_bf16(v[8 * e], v[8 * e + 1]),
                                  pack_bf16(v[8 * e + 2], v[8 * e + 3]), pack_bf16(v[8 * e + 4], v[8 * e + 5]),
                                  pack_bf16(v[8 * e + 6], v[8 * e + 7]));
                    }
                }
                if (!in) continue;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (OUT == PART) tma_store_3d(&p.c, piece, x, y, t.split);
                    else tma_store_2d(&p.c, piece, x, y);
                    bulk_commit();
                }
            }
        }
        if (!ok) record_timeout(p, 3);
        if (lane == 0) {                                 // what is in flight reads and writes this CTA's shared memory
            int never = 0;
            for (; got < asked; ++got) mbar_wait(bar(RES + ew), got & 1, &never, limit);
            bulk_wait_read_all();
        }
        __syncwarp();
    }
    fence_before_sync();
    cluster_sync();                                      // the pair's shared memory and TMEM stay until both are done
    fence_after_sync();
    if (warp == 1) pair_tmem_dealloc(tmem, 2 * kTileN);
}

// ---------------------------------------------------------------- host side

// [rows][cols] row-major, the operand of a product whose K (kc) or whose output index lies along cols
bool operand_map(CUtensorMap* m, const void* p, int rows, int cols, bool kc, int box_rows)
{
    return encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, rows, cols, kStepK, kc ? box_rows : kStepK,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool AMn, bool BMn, int OUT>
cudaError_t launch(const Params& p, cudaStream_t st)
{
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = Cfg<OUT>::kSmemTiles + sizeof(Ctrl);
    auto kernel = linear_gemm_kernel<AMn, BMn, OUT>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int items = p.m_tiles * p.n_tiles * p.splits, pairs = nsm / 2;
    kernel<<<2 * (items < pairs ? items : pairs), kThreads, smem, st>>>(p);
    return cudaGetLastError();
}

// C [M][N] = sum over K of A B, finished as `end` says (FINISH), or rounded only.
template <bool AMn, bool BMn, bool FINISH>
cudaError_t product(const LinShape& s, const void* A, const void* B, int M, int N, int K, const LinearEnd& end, float* part,
                    bool clear, DeviceStatus* status, cudaStream_t st)
{
    const auto bf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, f32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const auto swizzle = CU_TENSOR_MAP_SWIZZLE_128B;
    Params p{};
    p.M = M; p.N = N;
    p.m_tiles = (M + kTileM - 1) / kTileM;
    p.n_tiles = (N + kTileN - 1) / kTileN;
    p.k_steps = (K + kStepK - 1) / kStepK;
    p.splits = linear_splits(M, N, K);
    p.bias = end.bias;
    p.act = end.act;
    p.add = end.residual != nullptr;
    p.clear = clear;
    p.status = status;
    p.wait_limit_ns = s.wait_limit_ns;
    p.skip_first = s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY ? 1 : 0;
    if (!operand_map(&p.a, A, AMn ? K : M, AMn ? M : K, !AMn, kHalfM) ||
        !operand_map(&p.b, B, BMn ? K : N, BMn ? N : K, !BMn, kTileN / 2))
        return cudaErrorInvalidValue;
    if (p.splits > 1) {
        if (!encode_parts(&p.c, part, p.splits, M, N)) return cudaErrorInvalidValue;
        cudaError_t e = launch<AMn, BMn, PART>(p, st);
        return e == cudaSuccess ? launch_linear_join(end, part, p.splits, M, N, st) : e;
    }
    if (!encode_2d(&p.c, bf16, 2, end.c, M, N, 64, 32, swizzle) ||
        (p.add && !encode_2d(&p.residual, bf16, 2, end.residual, M, N, 64, 32, swizzle)) ||
        (end.Z && !encode_2d(&p.z, f32, 4, end.Z, M, N, 32, 32, swizzle)))
        return cudaErrorInvalidValue;
    if constexpr (FINISH) return end.Z ? launch<AMn, BMn, END_Z>(p, st) : launch<AMn, BMn, END>(p, st);
    else return launch<AMn, BMn, PLAIN>(p, st);
}

}  // namespace

// Parts of the K axis of least cost.  A pair takes 0.3 us a step of 64 k and some 3 us at its ends that no other tile
// covers; parts are written and read once more in fp32 at some 5 TB/s, and their join is a launch of 4 us.  76 pairs
// run at once.  (Tiles of 256 x 128 are no way to more items with steps of 64 k: a step of theirs takes as long, 0.3 us at
// 32760 x 1536 x 1536, most of it its wait, its announcement and its commit.  Deeper steps were not tried.)
int linear_splits(int64_t M, int64_t N, int64_t K)
{
    const int64_t steps = (K + kStepK - 1) / kStepK, tiles = ((M + kTileM - 1) / kTileM) * ((N + kTileN - 1) / kTileN);
    int best = 1;
    double least = 1e30;
    for (int64_t splits = 1; splits <= 16 && splits * 4 <= steps + 3; ++splits) {
        const double turns = (double)((tiles * splits + 75) / 76);
        const double us = turns * ((double)((steps + splits - 1) / splits) * 0.3 + 1.0) + 3.0 +
                          (splits > 1 ? 4.0 + 8.0 * (double)(splits * M * N) / 5e6 : 0.0);
        if (us < least * 0.999) {
            least = us;
            best = (int)splits;
        }
    }
    return best;
}

cudaError_t launch_linear_tc(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                             float* Z, float* part, DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(Y, b, R, Z, s.act);
    return product<false, false, true>(s, X, W, s.M, s.N, s.K, end, part, true, status, st);
}

cudaError_t launch_linear_dx_tc(const LinShape& s, const void* W, const void* dZ, void* dX, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(dX, nullptr, nullptr, nullptr, ROLA_LOWRANK_ACT_IDENTITY);
    return product<false, true, false>(s, dZ, W, s.M, s.K, s.N, end, part, clear, status, st);
}

cudaError_t launch_linear_dw_tc(const LinShape& s, const void* X, const void* dZ, void* dW, float* part, bool clear,
                                DeviceStatus* status, cudaStream_t st)
{
    const LinearEnd end = linear_end_of(dW, nullptr, nullptr, nullptr, ROLA_LOWRANK_ACT_IDENTITY);
    return product<true, true, false>(s, dZ, X, s.N, s.K, s.M, end, part, clear, status, st);     // k = token
}

}  // namespace rola
