// The gated feed-forward's products on the 5th-generation tensor cores (bf16
// operands, fp32 accumulation in TMEM).
//
//   H = phi(X Wg^T) * (X Wu^T),  Y = H Wd^T
//   dG, dU, H from dH = dY Wd;  dX = dG Wg + dU Wu;  dWg = dG^T X,  dWu = dU^T X,  dWd = dY^T H
//
// One persistent warp-specialised kernel computes C(m, n) = sum_k A(m, k) B(n, k)
// in tiles of 128 x 256, one CTA per SM.  Per K step of 64, A (16 KB) and B
// (32 KB) arrive by TMA in 128-byte-swizzled shared memory, four stages deep,
// and four tcgen05.mma M = 128, N = 256, K = 16 accumulate in TMEM.  The
// accumulator is double-buffered, so a tile's epilogue runs under the next
// tile's products.  An operand is contiguous along k (K-major, one box of 64 k)
// or along m / n (MN-major, boxes of 64 x 64 k); the tensor core reads either,
// so no operand is transposed in memory.  Ragged edges are TMA zero fill on
// loads (a zero adds nothing to the sum).
//
// Forms (Epilogue):
//   kStore     C rounded to bf16.  Y, the weights' gradients (three
//              products in one launch: 192 tiles each at widths 1536 x 4096
//              would be 1.3 waves of 152 SMs, 576 together are 3.8), and dX,
//              whose K axis is d_ff twice (dG Wg, then dU Wu, in one accumulator).
//   kGateUp    B = 128 rows of Wg and the same 128 rows of Wu: a thread
//              holds g and u of its row's features, so phi and the product
//              need no exchange.  H is stored once, G and U when training.
//   kGateGrad  dH stays in TMEM; G and U arrive by TMA beside it, a piece of 32
//              rows x 16 columns ahead of each epilogue warp.  (Tiles of 128 x 128 leave
//              room for larger pieces, but four stages of theirs cover 1000 cycles of
//              loads instead of 2000: 149 us against 121 at 8190 tokens x 1536 x 4096.)
//
// Tiles are taken in groups of kGroupM row tiles, column tiles outside, row
// tiles inside: the CTAs in flight share a few column tiles of B and the
// group's rows of A, which stay in L2 (129 MB), and B is read once per group.
//
// Epilogue: eight warps, two for each quarter of the TMEM lanes (32 rows), half
// of the columns each, 32 columns at a time; a lane stores whole 32-byte sectors of its
// row.  (Four warps that staged each piece in shared memory for TMA stores took
// 371 us for dH at 8190 tokens x 1536 x 4096 where the products need 55.)
//
// Measured at 8190 tokens x 1536 x 4096, training: up 172 us (G and U, 268 MB, written beside
// H; 125 without them), down 71, dH 120 (530 MB through HBM), dX 143, the weights 200; the plain products
// keep the tensor pipe 69 to 75 % busy (1440 to 1550 TFLOP/s), the last turn of tiles included.
//
// Warp roles (320 threads): warp 0 TMA producer, warp 1 MMA issuer and TMEM
// owner, warps 2-9 epilogue.  Every mbarrier wait is bounded; a wait that gives
// up records ROLA_ERR_TIMEOUT in the status word, and the CTA stops issuing, lets
// what it issued complete and frees its TMEM.
#include <cudaTypedefs.h>

#include "attention_tc.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

enum Epilogue { kStore, kGateUp, kGateGrad };

constexpr int kTileM = 128, kStepK = 64, kGroupM = 16;
constexpr uint32_t kABytes = kTileM * kStepK * 2;
constexpr int kThreads = 320, kEpiWarps = 8;
constexpr int NT = 256, kStages = 4;
constexpr uint32_t kBBytes = NT * kStepK * 2, kStageBytes = kABytes + kBBytes;
constexpr uint32_t kPieceBytes = 2048;                       // 32 rows x 16 columns, fp32

template <int E>
struct Cfg {
    static constexpr uint32_t kSmemEpi = kStages * kStageBytes;
    static constexpr uint32_t kEpiBytes = E == kGateGrad ? 2 * kPieceBytes : 0;      // a warp's piece of G and of U
    static constexpr uint32_t kSmemTiles = kSmemEpi + kEpiWarps * kEpiBytes;
    static constexpr int FULL = 0, EMPTY = FULL + kStages, ACC_FULL = EMPTY + kStages, ACC_EMPTY = ACC_FULL + 2,
                         DRAIN = ACC_EMPTY + 2, GU_FULL = DRAIN + 1, NUM_BARS = GU_FULL + kEpiWarps;
};

template <int E>
struct Ctrl {
    uint64_t bar[Cfg<E>::NUM_BARS];
    uint32_t tmem_base;
    int abort;
};
static_assert(Cfg<kStore>::kSmemTiles + sizeof(Ctrl<kStore>) <= 232448 &&
                  Cfg<kGateGrad>::kSmemTiles + sizeof(Ctrl<kGateGrad>) <= 232448,
              "tiles and control block fit the 227 KB a CTA may have");

// One product.  b[1] of kGateUp is W_up; a[1], b[1] with sources = 2 are the second product of the sum.
// c: C, or H; for kGateGrad dG and dU too.  Every output row is a multiple of 16 bytes long.
struct Problem {
    CUtensorMap a[2], b[2];
    __nv_bfloat16* c[3];
    int M, N;
    int wide;                        // the outputs' rows are 32-byte aligned
    int m_tiles, n_tiles, tile0;     // tiles [tile0, tile0 + m_tiles n_tiles) of the launch are this product's
    int k_steps, sources;            // K steps of 64 of one source
};

template <int E>
struct Params {
    Problem pr[E == kStore ? 3 : 1];
    CUtensorMap in[E == kGateGrad ? 2 : 1];      // kGateGrad: G and U
    float *G, *U;                    // kGateUp: out, or NULL
    int problems, tiles, act;
    int skip_first;                  // test hook: a CTA's first load is never issued
    DeviceStatus* status;
    uint64_t wait_limit_ns;
};

template <int E>
__device__ __forceinline__ void record_timeout(const Params<E>& p, int where)
{
    if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 64 + where;
}

// Tile t of the launch -> its product and (row tile, column tile).
template <int E>
__device__ __forceinline__ const Problem& tile_of(const Params<E>& p, int t, int& mt, int& nt)
{
    int i = 0;
    if constexpr (E == kStore)
        while (i + 1 < p.problems && t >= p.pr[i + 1].tile0) ++i;
    const Problem& r = p.pr[i];
    t -= r.tile0;
    const int per_group = kGroupM * r.n_tiles, g = t / per_group;
    const int rows = min(kGroupM, r.m_tiles - g * kGroupM);
    t -= g * per_group;
    nt = t / rows;
    mt = g * kGroupM + t - nt * rows;
    return r;
}

// W values of a row from column f0 of N (a multiple of 8) on: in bf16, and in fp32
template <int W>
__device__ __forceinline__ void store_row(__nv_bfloat16* row, int f0, int N, const float (&v)[W], bool wide)
{
#pragma unroll
    for (int e = 0; e < W; e += 16) {
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(v[e + 2 * j], v[e + 2 * j + 1]);
        if (f0 + e + 16 <= N) store_row32(row + f0 + e, y, wide);
        else if (f0 + e < N) *reinterpret_cast<uint4*>(row + f0 + e) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}
template <int W>
__device__ __forceinline__ void store_row(float* row, int f0, int N, const float (&v)[W], bool wide)
{
#pragma unroll
    for (int e = 0; e < W; e += 8) {
        if (f0 + e >= N) break;
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __float_as_uint(v[e + j]);
        if (wide) {
            st_global32(row + f0 + e, y);
        } else {
            *reinterpret_cast<uint4*>(row + f0 + e) = make_uint4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<uint4*>(row + f0 + e + 4) = make_uint4(y[4], y[5], y[6], y[7]);
        }
    }
}
// 16 fp32 of this lane's row of a piece, a row of 64 bytes (64-byte swizzle)
__device__ __forceinline__ void read_row(uint32_t buf, int lane, float (&v)[16])
{
#pragma unroll
    for (int c = 0; c < 4; ++c)
        asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];\n"
                     : "=f"(v[4 * c]), "=f"(v[4 * c + 1]), "=f"(v[4 * c + 2]), "=f"(v[4 * c + 3])
                     : "r"(buf + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4))
                     : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32])
{
    tmem_ld16(taddr, *reinterpret_cast<float(*)[16]>(&v[0]));
    tmem_ld16(taddr + 16, *reinterpret_cast<float(*)[16]>(&v[16]));
    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&v[0]));
    reg_fence(*reinterpret_cast<float(*)[16]>(&v[16]));
}

template <bool AMn, bool BMn, int E>
__global__ void __launch_bounds__(kThreads, 1) ffn_gemm_kernel(const __grid_constant__ Params<E> p)
{
    using C = Cfg<E>;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {     // the 128-byte swizzle atoms need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(&p.status->code, 0, (int)ROLA_ERR_UNSUPPORTED);
        return;
    }
    Ctrl<E>& cb = *reinterpret_cast<Ctrl<E>*>(smem_raw + C::kSmemTiles);
    const uint32_t sbase = smem_u32(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&cb.bar[i]); };

    if (tid == 0) {
        cb.abort = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(bar(C::FULL + i), 1);
            mbar_init(bar(C::EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::ACC_FULL + i), 1);
            mbar_init(bar(C::ACC_EMPTY + i), kEpiWarps);
        }
        mbar_init(bar(C::DRAIN), 1);
        for (int i = 0; i < kEpiWarps; ++i) mbar_init(bar(C::GU_FULL + i), 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&cb.tmem_base), 2 * NT);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = cb.tmem_base;
    volatile int* abort = &cb.abort;
    const uint64_t limit = p.wait_limit_ns;

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        // A box per lane: a lane's copies run one after another.  Lanes 0 (and 1): A; 2 ..: B.
        constexpr int kABoxes = AMn ? 2 : 1, kBBoxes = BMn ? NT / 64 : (E == kGateUp ? 2 : 1);
        bool ok = true;
        int g = 0;                                  // K steps issued by this CTA
        for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x) {
            int mt, nt;
            const Problem& r = tile_of(p, t, mt, nt);
            const int steps = r.k_steps * r.sources;
            for (int ks = 0; ks < steps; ++ks, ++g) {
                const int s = g % kStages;
                if (g >= kStages) ok = mbar_wait(bar(C::EMPTY + s), ((g / kStages) - 1) & 1, abort, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                const bool skip = p.skip_first && g == 0;
                if (lane == 0 && !skip) mbar_expect_tx(bar(C::FULL + s), kStageBytes);
                __syncwarp();
                const int src = ks >= r.k_steps ? 1 : 0, k0 = (ks - src * r.k_steps) * kStepK;
                const uint32_t dst = sbase + s * kStageBytes;
                if (lane < kABoxes && !skip) {
                    if constexpr (AMn)
                        tma_load_2d(dst + lane * 8192, &r.a[src], bar(C::FULL + s), mt * kTileM + lane * 64, k0);
                    else
                        tma_load_2d(dst, &r.a[src], bar(C::FULL + s), k0, mt * kTileM);
                }
                const int bl = lane - 2;
                if (bl >= 0 && bl < kBBoxes && !skip) {
                    if constexpr (BMn)
                        tma_load_2d(dst + kABytes + bl * 8192, &r.b[src], bar(C::FULL + s), nt * NT + bl * 64, k0);
                    else if constexpr (E == kGateUp)
                        tma_load_2d(dst + kABytes + bl * 16384, &r.b[bl], bar(C::FULL + s), k0, nt * 128);
                    else
                        tma_load_2d(dst + kABytes, &r.b[src], bar(C::FULL + s), k0, nt * NT);
                }
            }
        }
        if (!ok && lane == 0) record_timeout(p, 1);
        // the copies still in flight land before the CTA exits: wait for the last use of each stage
        if (lane == 0) {
            int never = 0;
            for (int u = g > kStages ? g - kStages : 0; u < g; ++u)
                mbar_wait(bar(C::FULL + u % kStages), (u / kStages) & 1, &never, limit);
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16(kTileM, NT, AMn, BMn);
            const uint64_t da = smem_desc(sbase, AMn ? 8192 : 16, 1024), db = smem_desc(sbase + kABytes, BMn ? 8192 : 16, 1024);
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32);
            const uint32_t b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            constexpr uint32_t a_k = AMn ? 128 : 2, b_k = BMn ? 128 : 2;    // 16 k: 16 rows of 128 B, or 32 B of a row
            bool ok = true;
            int g = 0, it = 0;
            for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x, ++it) {
                int mt, nt;
                const Problem& r = tile_of(p, t, mt, nt);
                const int steps = r.k_steps * r.sources, ab = it & 1;
                if (it >= 2 && !(ok = mbar_wait(bar(C::ACC_EMPTY + ab), ((it >> 1) - 1) & 1, abort, limit))) break;
                fence_after_sync();
                const uint32_t d = tmem + ab * NT;
                for (int ks = 0; ks < steps; ++ks, ++g) {
                    const int s = g % kStages;
                    if (!(ok = mbar_wait(bar(C::FULL + s), (g / kStages) & 1, abort, limit))) break;
                    fence_after_sync();
                    const uint32_t off = s * (kStageBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kStepK / 16; ++kk)
                        mma_ss_split(d, a_lo + off + kk * a_k, a_hi, b_lo + off + kk * b_k, b_hi, idesc,
                                     (ks > 0 || kk > 0) ? 1u : 0u);
                    mma_commit(bar(C::EMPTY + s));
                }
                if (!ok) break;
                mma_commit(bar(C::ACC_FULL + ab));
            }
            if (!ok) record_timeout(p, 2);
            // every MMA issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(C::DRAIN));
            mbar_wait(bar(C::DRAIN), 0, &never, limit);
        }
    } else {
        // ------------------------------------------------------------ epilogue
        const int q = warp & 3, ew = warp - 2;           // TMEM lane quarter: rows 32 q .. +31 of the tile
        const int half = ew >> 2;                        // of the columns
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t piece = sbase + C::kSmemEpi + ew * C::kEpiBytes;
        constexpr int kCols = E == kGateGrad ? 16 : 32;              // columns of a chunk
        constexpr int kHalf = (E == kGateUp ? 128 : NT) / 2, kChunks = kHalf / kCols;
        bool ok = true;
        int it = 0;
        // kGateGrad: G and U of chunk c of tile t
        int fetched = 0, used = 0;
        auto fetch = [&](int t, int c) {
            if (t >= p.tiles) return;
            int mt, nt;
            tile_of(p, t, mt, nt);
            if (lane == 0) {
                const uint32_t b = bar(C::GU_FULL + ew);
                const int x = nt * NT + half * kHalf + c * kCols, y = mt * kTileM + q * 32;
                mbar_expect_tx(b, 2 * kPieceBytes);
                tma_load_2d(piece, &p.in[0], b, x, y);
                tma_load_2d(piece + kPieceBytes, &p.in[E == kGateGrad ? 1 : 0], b, x, y);
            }
            ++fetched;
        };
        if constexpr (E == kGateGrad) fetch(blockIdx.x, 0);
        for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x, ++it) {
            int mt, nt;
            const Problem& r = tile_of(p, t, mt, nt);
            const int ab = it & 1;
            if (!(ok = mbar_wait_warp(bar(C::ACC_FULL + ab), (it >> 1) & 1, abort, limit))) break;
            fence_after_sync();
            const int row = mt * kTileM + q * 32 + lane;
            const bool in = row < r.M;
            const size_t at = (size_t)row * r.N;
            const uint32_t acc = tmem + lane_off + ab * NT;
            for (int c = 0; c < kChunks && ok; ++c) {
                // the last piece is in registers: the accumulator buffer is free for the tile after next
                auto release = [&]() {
                    if (c != kChunks - 1) return;
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::ACC_EMPTY + ab));
                };
                if constexpr (E == kStore) {
                    const int col = half * kHalf + c * kCols;
                    float v[32];
                    tmem_ld32(acc + col, v);
                    release();
                    if (in) store_row(r.c[0] + at, nt * NT + col, r.N, v, r.wide);
                } else if constexpr (E == kGateUp) {
                    const int col = half * kHalf + c * kCols, f0 = nt * 128 + col;
                    float gv[32], uv[32];
                    tmem_ld32(acc + col, gv);
                    tmem_ld32(acc + 128 + col, uv);
                    release();
                    if (in && p.G) {
                        store_row(p.G + at, f0, r.N, gv, r.wide);
                        store_row(p.U + at, f0, r.N, uv, r.wide);
                    }
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) gv[j] = act.phi(gv[j]) * uv[j];
                    });
                    if (in) store_row(r.c[0] + at, f0, r.N, gv, r.wide);
                } else {
                    const int col = half * kHalf + c * kCols, f0 = nt * NT + col;
                    float dh[16], gv[16], uv[16];
                    tmem_ld16(acc + col, dh);
                    tmem_ld_wait(dh);
                    release();
                    if (!(ok = mbar_wait_warp(bar(C::GU_FULL + ew), used & 1, abort, limit))) break;
                    ++used;
                    read_row(piece, lane, gv);
                    read_row(piece + kPieceBytes, lane, uv);
                    __syncwarp();                        // every lane has read its rows
                    // the next piece comes under this one's work
                    if (c + 1 < kChunks) fetch(t, c + 1);
                    else fetch(t + (int)gridDim.x, 0);
                    with_act(p.act, [&](auto act) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float a, da;
                            act.grad(gv[j], a, da);
                            const float d = dh[j], u = uv[j];
                            gv[j] = a * u;               // H
                            uv[j] = d * u * da;          // dG
                            dh[j] = d * a;               // dU
                        }
                    });
                    if (in) {
                        store_row(r.c[0] + at, f0, r.N, gv, r.wide);
                        store_row(r.c[1] + at, f0, r.N, uv, r.wide);
                        store_row(r.c[2] + at, f0, r.N, dh, r.wide);
                    }
                }
            }
        }
        if (!ok) record_timeout(p, 3);
        if constexpr (E == kGateGrad)                    // the pieces still in flight land before the CTA exits
            if (lane == 0) {
                int never = 0;
                for (; used < fetched; ++used) mbar_wait(bar(C::GU_FULL + ew), used & 1, &never, limit);
            }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, 2 * NT);
}

// ---------------------------------------------------------------- host side

// [rows][cols] row-major, the operand of a product whose K (kc) or whose output index lies along cols
bool operand_map(CUtensorMap* m, const void* p, int rows, int cols, bool kc, int box_rows)
{
    return encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, rows, cols, kStepK, kc ? box_rows : kStepK,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool AMn, bool BMn, int E>
cudaError_t launch(const FfnShape& s, Params<E>& p, DeviceStatus* status, cudaStream_t st)
{
    using C = Cfg<E>;
    p.act = s.act;
    p.status = status;
    p.wait_limit_ns = s.wait_limit_ns;
    p.skip_first = s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY ? 1 : 0;
    p.tiles = 0;
    for (int i = 0; i < p.problems; ++i) {
        Problem& r = p.pr[i];
        r.m_tiles = (r.M + kTileM - 1) / kTileM;
        r.n_tiles = (r.N + (E == kGateUp ? 127 : NT - 1)) / (E == kGateUp ? 128 : NT);
        r.wide = r.N % 16 == 0 && ((reinterpret_cast<uintptr_t>(p.G) | reinterpret_cast<uintptr_t>(p.U)) & 31u) == 0;
        for (const __nv_bfloat16* c : r.c) r.wide = r.wide && (reinterpret_cast<uintptr_t>(c) & 31u) == 0;
        r.tile0 = p.tiles;
        p.tiles += r.m_tiles * r.n_tiles;
    }
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = C::kSmemTiles + sizeof(Ctrl<E>);
    auto kernel = ffn_gemm_kernel<AMn, BMn, E>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<p.tiles < nsm ? p.tiles : nsm, kThreads, smem, st>>>(p);
    return cudaGetLastError();
}

int steps(int k) { return (k + kStepK - 1) / kStepK; }

// dH = dY Wd, and from it H, dG, dU
cudaError_t launch_dh(const FfnShape& s, const void* Wd, const float* G, const float* U, const void* dY, void* H,
                      void* dG, void* dU, DeviceStatus* status, cudaStream_t st)
{
    Params<kGateGrad> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    r.M = s.M; r.N = s.F; r.k_steps = steps(s.D); r.sources = 1;
    r.c[0] = static_cast<__nv_bfloat16*>(H);
    r.c[1] = static_cast<__nv_bfloat16*>(dG);
    r.c[2] = static_cast<__nv_bfloat16*>(dU);
    const auto f32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    if (!operand_map(&r.a[0], dY, s.M, s.D, true, kTileM) || !operand_map(&r.b[0], Wd, s.D, s.F, false, 0) ||
        !encode_2d(&p.in[0], f32, 4, G, s.M, s.F, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode_2d(&p.in[1], f32, 4, U, s.M, s.F, 16, 32, CU_TENSOR_MAP_SWIZZLE_64B))
        return cudaErrorInvalidValue;
    return launch<false, true, kGateGrad>(s, p, status, st);
}

// dX = dG Wg + dU Wu
cudaError_t launch_dx(const FfnShape& s, const void* Wg, const void* Wu, const void* dG, const void* dU, void* dX,
                      DeviceStatus* status, cudaStream_t st)
{
    Params<kStore> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    r.M = s.M; r.N = s.D; r.k_steps = steps(s.F); r.sources = 2;
    if (!operand_map(&r.a[0], dG, s.M, s.F, true, kTileM) || !operand_map(&r.a[1], dU, s.M, s.F, true, kTileM) ||
        !operand_map(&r.b[0], Wg, s.F, s.D, false, 0) || !operand_map(&r.b[1], Wu, s.F, s.D, false, 0))
        return cudaErrorInvalidValue;
    r.c[0] = static_cast<__nv_bfloat16*>(dX);
    return launch<false, true, kStore>(s, p, status, st);
}

}  // namespace

cudaError_t launch_ffn_up_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, void* H, float* G,
                             float* U, DeviceStatus* status, cudaStream_t st)
{
    Params<kGateUp> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    p.G = G;
    p.U = U;
    r.c[0] = static_cast<__nv_bfloat16*>(H);
    r.M = s.M; r.N = s.F; r.k_steps = steps(s.D); r.sources = 1;
    if (!operand_map(&r.a[0], X, s.M, s.D, true, kTileM) || !operand_map(&r.b[0], Wg, s.F, s.D, true, 128) ||
        !operand_map(&r.b[1], Wu, s.F, s.D, true, 128))
        return cudaErrorInvalidValue;
    return launch<false, false, kGateUp>(s, p, status, st);
}

cudaError_t launch_ffn_down_tc(const FfnShape& s, const void* H, const void* Wd, void* Y, DeviceStatus* status,
                               cudaStream_t st)
{
    Params<kStore> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    r.M = s.M; r.N = s.D; r.k_steps = steps(s.F); r.sources = 1;
    r.c[0] = static_cast<__nv_bfloat16*>(Y);
    if (!operand_map(&r.a[0], H, s.M, s.F, true, kTileM) || !operand_map(&r.b[0], Wd, s.D, s.F, true, 256))
        return cudaErrorInvalidValue;
    return launch<false, false, kStore>(s, p, status, st);
}

cudaError_t launch_ffn_backward_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd,
                                   const float* G, const float* U, const void* dY, void* H, void* dG, void* dU,
                                   void* dX, void* dWg, void* dWu, void* dWd, DeviceStatus* status, cudaStream_t st)
{
    if (s.M <= kFfnFewTokens) {
        cudaError_t e = launch_ffn_few_grad(s, Wg, Wu, Wd, G, U, dY, H, dG, dU, dX, status, st);
        if (e != cudaSuccess) return e;
    } else {
        cudaError_t e = launch_dh(s, Wd, G, U, dY, H, dG, dU, status, st);
        if (e == cudaSuccess) e = launch_dx(s, Wg, Wu, dG, dU, dX, status, st);
        if (e != cudaSuccess) return e;
    }
    // dWg = dG^T X, dWu = dU^T X, dWd = dY^T H: K is the token
    Params<kStore> p{};
    p.problems = 3;
    const struct { const void *a, *b; int m, n; void* c; } w[3] = {
        {dG, X, s.F, s.D, dWg}, {dU, X, s.F, s.D, dWu}, {dY, H, s.D, s.F, dWd}};
    for (int i = 0; i < 3; ++i) {
        Problem& r = p.pr[i];
        r.M = w[i].m; r.N = w[i].n; r.k_steps = steps(s.M); r.sources = 1;
        r.c[0] = static_cast<__nv_bfloat16*>(w[i].c);
        if (!operand_map(&r.a[0], w[i].a, s.M, w[i].m, false, 0) || !operand_map(&r.b[0], w[i].b, s.M, w[i].n, false, 0))
            return cudaErrorInvalidValue;
    }
    return launch<true, true, kStore>(s, p, status, st);
}

}  // namespace rola
