// The gated feed-forward's products on the 5th-generation tensor cores (bf16
// operands, fp32 accumulation in TMEM).
//
//   H = phi(X Wg^T) * (X Wu^T),  Y = H Wd^T
//   dG, dU, H from dH = dY Wd;  dX = dG Wg + dU Wu;  dWg = dG^T X,  dWu = dU^T X,  dWd = dY^T H
//
// One persistent warp-specialised kernel computes C(m, n) = sum_k A(m, k) B(n, k)
// in tiles of 128 x NT, one CTA per SM.  Per K step of 64, A (16 KB) and B
// (128 NT bytes) arrive by TMA in 128-byte-swizzled shared memory, four stages
// deep, and four tcgen05.mma M = 128, N = NT, K = 16 accumulate in TMEM.  The
// accumulator is double-buffered, so a tile's epilogue runs under the next
// tile's products.  An operand is contiguous along k (K-major, one box of 64 k)
// or along m / n (MN-major, boxes of 64 x 64 k); the tensor core reads either,
// so no operand is transposed in memory.  Ragged edges are TMA zero fill on
// loads (a zero adds nothing to the sum) and TMA clipping on stores.
//
// Forms (Epilogue):
//   kStore     NT = 256: C rounded to bf16.  Y, the weights' gradients (three
//              products in one launch: 192 tiles each at widths 1536 x 4096
//              would be 1.3 waves of 152 SMs, 576 together are 3.8), and dX,
//              whose K axis is d_ff twice (dG Wg, then dU Wu, in one accumulator).
//   kGateUp    NT = 256 = 128 rows of Wg and the same 128 rows of Wu: a thread
//              holds g and u of its row's features, so phi and the product
//              need no exchange.  H is stored once, G and U when training.
//   kGateGrad  NT = 128: dH stays in TMEM; G and U arrive by TMA in the
//              epilogue, dG, dU and H leave by TMA.  The narrower tile leaves
//              room for that traffic beside the four stages.
//
// Tiles are taken in groups of kGroupM row tiles, column tiles outside, row
// tiles inside: the CTAs in flight share a few column tiles of B and the
// group's rows of A, which stay in L2 (129 MB), and B is read once per group.
//
// Warp roles (192 threads): warp 0 TMA producer, warp 1 MMA issuer and TMEM
// owner, warps 2-5 epilogue (warp w reads TMEM lanes 32 (w mod 4) .. +31, its
// 32 rows).  Every mbarrier wait is bounded; a wait that gives up records
// ROLA_ERR_TIMEOUT in the status word, and the CTA stops issuing, lets what it
// issued complete and frees its TMEM.
#include <cudaTypedefs.h>

#include "block_ops.cuh"
#include "tcgen05.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

enum Epilogue { kStore, kGateUp, kGateGrad };

constexpr int kTileM = 128, kStepK = 64, kStages = 4, kGroupM = 16;
constexpr uint32_t kABytes = kTileM * kStepK * 2;
constexpr int kThreads = 192, kEpiWarps = 4;
constexpr uint32_t kStoreBytes = 4096;                       // 32 rows of 128 bytes

template <int E>
struct Cfg {
    static constexpr int NT = E == kGateGrad ? 128 : 256;
    static constexpr uint32_t kBBytes = NT * kStepK * 2;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr uint32_t kSmemEpi = kStages * kStageBytes;
    // an epilogue warp's shared memory: two store buffers; or two slots of G and U, and H, dG, dU
    // (32 features in bf16: 2 KB each)
    static constexpr uint32_t kEpiBytes = E == kGateGrad ? 4 * kStoreBytes + 3 * 2048 : 2 * kStoreBytes;
    static constexpr uint32_t kSmemTiles = kSmemEpi + kEpiWarps * kEpiBytes;
    static constexpr int FULL = 0, EMPTY = FULL + kStages, ACC_FULL = EMPTY + kStages, ACC_EMPTY = ACC_FULL + 2,
                         DRAIN = ACC_EMPTY + 2, GU_FULL = DRAIN + 1, NUM_BARS = GU_FULL + 2 * kEpiWarps;
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
// c: C, or H; c[1], c[2]: G and U (kGateUp, fp32) or dG and dU (kGateGrad); in: G and U of kGateGrad.
struct Problem {
    CUtensorMap a[2], b[2], c[3];
    int M, N;
    int m_tiles, n_tiles, tile0;     // tiles [tile0, tile0 + m_tiles n_tiles) of the launch are this product's
    int k_steps, sources;            // K steps of 64 of one source
};

template <int E>
struct Params {
    Problem pr[E == kStore ? 3 : 1];
    CUtensorMap in[E == kGateGrad ? 2 : 1];
    int problems, tiles, act, keep;  // keep: kGateUp writes G and U
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

// 32 bf16 of this lane's row into a 32 x 32 tile of 64-byte rows (64-byte swizzle)
__device__ __forceinline__ void stage_row32(uint32_t buf, int lane, const float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t w0 = pack_bf16(v[8 * c], v[8 * c + 1]), w1 = pack_bf16(v[8 * c + 2], v[8 * c + 3]);
        const uint32_t w2 = pack_bf16(v[8 * c + 4], v[8 * c + 5]), w3 = pack_bf16(v[8 * c + 6], v[8 * c + 7]);
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(buf + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)),
                     "r"(w0), "r"(w1), "r"(w2), "r"(w3)
                     : "memory");
    }
}
// the same 32 columns starting at 16-byte chunk c0 of a row of 128 bytes (128-byte swizzle)
__device__ __forceinline__ void stage_half_row64(uint32_t buf, int lane, int c0, const float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint32_t w0 = pack_bf16(v[8 * c], v[8 * c + 1]), w1 = pack_bf16(v[8 * c + 2], v[8 * c + 3]);
        const uint32_t w2 = pack_bf16(v[8 * c + 4], v[8 * c + 5]), w3 = pack_bf16(v[8 * c + 6], v[8 * c + 7]);
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(buf + lane * 128 + (((c0 + c) ^ (lane & 7)) << 4)),
                     "r"(w0), "r"(w1), "r"(w2), "r"(w3)
                     : "memory");
    }
}
// 32 fp32 of this lane's row, a row of 128 bytes (128-byte swizzle)
__device__ __forceinline__ void stage_row_f32(uint32_t buf, int lane, const float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 8; ++c)
        asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};\n" ::"r"(buf + lane * 128 + ((c ^ (lane & 7)) << 4)),
                     "f"(v[4 * c]), "f"(v[4 * c + 1]), "f"(v[4 * c + 2]), "f"(v[4 * c + 3])
                     : "memory");
}
__device__ __forceinline__ void read_row_f32(uint32_t buf, int lane, float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 8; ++c)
        asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];\n"
                     : "=f"(v[4 * c]), "=f"(v[4 * c + 1]), "=f"(v[4 * c + 2]), "=f"(v[4 * c + 3])
                     : "r"(buf + lane * 128 + ((c ^ (lane & 7)) << 4))
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
    constexpr int NT = C::NT;
    constexpr uint32_t kStageBytes = C::kStageBytes;
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
        for (int i = 0; i < 2 * kEpiWarps; ++i) mbar_init(bar(C::GU_FULL + i), 1);
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
        const int q = warp & 3;                          // TMEM lane quarter: rows 32 q .. +31 of the tile
        const uint32_t lane_off = (uint32_t)(q * 32) << 16;
        const uint32_t epi = sbase + C::kSmemEpi + (warp - 2) * C::kEpiBytes;
        bool ok = true;
        int it = 0, chunk = 0;
        // a store buffer is free once the store issued two chunks ago has read it
        auto next_buffer = [&]() {
            if (lane == 0 && chunk >= 2) bulk_wait_read_1();
            __syncwarp();
            return epi + (chunk++ & 1) * kStoreBytes;
        };
        auto send = [&](const CUtensorMap* map, uint32_t buf, int x, int y, bool in) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                if (in) tma_store_2d(map, buf, x, y);
                bulk_commit();                           // an empty group where nothing is stored
            }
        };
        // kGateGrad: the 32 x 32 pieces of G and U of chunk c of tile t, into slot `slot`
        auto fetch = [&](int t, int c, int slot) {
            int mt, nt;
            tile_of(p, t, mt, nt);
            if (lane == 0) {
                const uint32_t b = bar(C::GU_FULL + (warp - 2) * 2 + slot), dst = epi + slot * 2 * kStoreBytes;
                mbar_expect_tx(b, 2 * kStoreBytes);
                tma_load_2d(dst, &p.in[0], b, nt * NT + c * 32, mt * kTileM + q * 32);
                tma_load_2d(dst + kStoreBytes, &p.in[E == kGateGrad ? 1 : 0], b, nt * NT + c * 32, mt * kTileM + q * 32);
            }
        };
        int fetched = 0, used = 0;
        if constexpr (E == kGateGrad)
            if ((int)blockIdx.x < p.tiles) fetch(blockIdx.x, 0, fetched++ & 1);
        for (int t = blockIdx.x; t < p.tiles && ok; t += gridDim.x, ++it) {
            int mt, nt;
            const Problem& r = tile_of(p, t, mt, nt);
            const int ab = it & 1;
            if (!(ok = mbar_wait(bar(C::ACC_FULL + ab), (it >> 1) & 1, abort, limit))) break;
            fence_after_sync();
            const int row0 = mt * kTileM + q * 32;       // first row of this warp
            const uint32_t acc = tmem + lane_off + ab * NT;
            auto release = [&]() {                       // the accumulator buffer is free for the tile after next
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(C::ACC_EMPTY + ab));
            };
            if constexpr (E == kStore) {
                for (int c = 0; c < NT / 64; ++c) {
                    const int f0 = nt * NT + c * 64;
                    float v[64];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tmem_ld16(acc + c * 64 + j * 16, *reinterpret_cast<float(*)[16]>(&v[j * 16]));
                    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&v[0]));
#pragma unroll
                    for (int j = 1; j < 4; ++j) reg_fence(*reinterpret_cast<float(*)[16]>(&v[j * 16]));
                    if (c == NT / 64 - 1) release();
                    const uint32_t buf = next_buffer();
                    stage_half_row64(buf, lane, 0, *reinterpret_cast<float(*)[32]>(&v[0]));
                    stage_half_row64(buf, lane, 4, *reinterpret_cast<float(*)[32]>(&v[32]));
                    send(&r.c[0], buf, f0, row0, row0 < r.M && f0 < r.N);
                }
            } else if constexpr (E == kGateUp) {
                for (int c = 0; c < 2; ++c) {            // 64 of the tile's 128 features
                    const int f0 = nt * 128 + c * 64;
                    float h[64];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int col = c * 64 + half * 32, f = f0 + half * 32;
                        float gv[32], uv[32];
                        tmem_ld32(acc + col, gv);
                        tmem_ld32(acc + 128 + col, uv);
                        if (col == 96) release();
                        if (p.keep) {
                            const bool in = row0 < r.M && f < r.N;
                            uint32_t buf = next_buffer();
                            stage_row_f32(buf, lane, gv);
                            send(&r.c[1], buf, f, row0, in);
                            buf = next_buffer();
                            stage_row_f32(buf, lane, uv);
                            send(&r.c[2], buf, f, row0, in);
                        }
#pragma unroll
                        for (int j = 0; j < 32; ++j) h[half * 32 + j] = gate_act(p.act, gv[j]) * uv[j];
                    }
                    const uint32_t buf = next_buffer();
                    stage_half_row64(buf, lane, 0, *reinterpret_cast<float(*)[32]>(&h[0]));
                    stage_half_row64(buf, lane, 4, *reinterpret_cast<float(*)[32]>(&h[32]));
                    send(&r.c[0], buf, f0, row0, row0 < r.M && f0 < r.N);
                }
            } else {
                for (int c = 0; c < NT / 32; ++c, ++used) {
                    // the next piece is on its way while this one is used
                    const int tn = c + 1 < NT / 32 ? t : t + (int)gridDim.x;
                    __syncwarp();                        // its slot was read by every lane
                    if (tn < p.tiles) fetch(tn, c + 1 < NT / 32 ? c + 1 : 0, fetched++ & 1);
                    const int slot = used & 1;
                    if (!(ok = mbar_wait(bar(C::GU_FULL + (warp - 2) * 2 + slot), (used >> 1) & 1, abort, limit))) break;
                    float dh[32], gv[32], uv[32];
                    tmem_ld32(acc + c * 32, dh);
                    if (c == NT / 32 - 1) release();
                    read_row_f32(epi + slot * 2 * kStoreBytes, lane, gv);
                    read_row_f32(epi + slot * 2 * kStoreBytes + kStoreBytes, lane, uv);
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float a, da;
                        gate_act_grad(p.act, gv[j], a, da);
                        const float d = dh[j], u = uv[j];
                        gv[j] = a * u;                   // H
                        uv[j] = d * u * da;              // dG
                        dh[j] = d * a;                   // dU
                    }
                    const uint32_t buf = epi + 4 * kStoreBytes;
                    if (lane == 0) bulk_wait_read_all();
                    __syncwarp();
                    stage_row32(buf, lane, gv);
                    stage_row32(buf + 2048, lane, uv);
                    stage_row32(buf + 4096, lane, dh);
                    fence_proxy_async_smem();
                    __syncwarp();
                    const int f0 = nt * NT + c * 32;
                    if (lane == 0) {
                        if (row0 < r.M && f0 < r.N) {
                            tma_store_2d(&r.c[0], buf, f0, row0);
                            tma_store_2d(&r.c[1], buf + 2048, f0, row0);
                            tma_store_2d(&r.c[2], buf + 4096, f0, row0);
                        }
                        bulk_commit();
                    }
                }
            }
        }
        if (!ok) record_timeout(p, 3);
        if (lane == 0) {
            if constexpr (E == kGateGrad) {              // the pieces still in flight land before the CTA exits
                int never = 0;
                for (; used < fetched; ++used)
                    mbar_wait(bar(C::GU_FULL + (warp - 2) * 2 + (used & 1)), (used >> 1) & 1, &never, limit);
            }
            bulk_wait_all();                             // the stores have left shared memory
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
        r.n_tiles = (r.N + (E == kGateUp ? 127 : C::NT - 1)) / (E == kGateUp ? 128 : C::NT);
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

}  // namespace

cudaError_t launch_ffn_up_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, void* H, float* G,
                             float* U, DeviceStatus* status, cudaStream_t st)
{
    Params<kGateUp> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    p.keep = G != nullptr;
    r.M = s.M; r.N = s.F; r.k_steps = steps(s.D); r.sources = 1;
    bool ok = operand_map(&r.a[0], X, s.M, s.D, true, kTileM) && operand_map(&r.b[0], Wg, s.F, s.D, true, 128) &&
              operand_map(&r.b[1], Wu, s.F, s.D, true, 128) &&
              encode_2d(&r.c[0], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, H, s.M, s.F, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B);
    if (G)
        ok = ok && encode_2d(&r.c[1], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, G, s.M, s.F, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B) &&
             encode_2d(&r.c[2], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, U, s.M, s.F, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B);
    if (!ok) return cudaErrorInvalidValue;
    return launch<false, false, kGateUp>(s, p, status, st);
}

cudaError_t launch_ffn_down_tc(const FfnShape& s, const void* H, const void* Wd, void* Y, DeviceStatus* status,
                               cudaStream_t st)
{
    Params<kStore> p{};
    Problem& r = p.pr[0];
    p.problems = 1;
    r.M = s.M; r.N = s.D; r.k_steps = steps(s.F); r.sources = 1;
    if (!operand_map(&r.a[0], H, s.M, s.F, true, kTileM) || !operand_map(&r.b[0], Wd, s.D, s.F, true, 256) ||
        !encode_2d(&r.c[0], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, Y, s.M, s.D, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    return launch<false, false, kStore>(s, p, status, st);
}

cudaError_t launch_ffn_backward_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd,
                                   const float* G, const float* U, const void* dY, void* H, void* dG, void* dU,
                                   void* dX, void* dWg, void* dWu, void* dWd, DeviceStatus* status, cudaStream_t st)
{
    const auto bf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const auto f32 = CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
    const auto sw128 = CU_TENSOR_MAP_SWIZZLE_128B, sw64 = CU_TENSOR_MAP_SWIZZLE_64B;
    if (s.M <= kFfnFewTokens) {
        cudaError_t e = launch_ffn_few_grad(s, Wg, Wu, Wd, G, U, dY, H, dG, dU, dX, status, st);
        if (e != cudaSuccess) return e;
    } else {
    {   // dH = dY Wd, and from it H, dG, dU
        Params<kGateGrad> p{};
        Problem& r = p.pr[0];
        p.problems = 1;
        r.M = s.M; r.N = s.F; r.k_steps = steps(s.D); r.sources = 1;
        if (!operand_map(&r.a[0], dY, s.M, s.D, true, kTileM) || !operand_map(&r.b[0], Wd, s.D, s.F, false, 0) ||
            !encode_2d(&r.c[0], bf16, 2, H, s.M, s.F, 32, 32, sw64) || !encode_2d(&r.c[1], bf16, 2, dG, s.M, s.F, 32, 32, sw64) ||
            !encode_2d(&r.c[2], bf16, 2, dU, s.M, s.F, 32, 32, sw64) || !encode_2d(&p.in[0], f32, 4, G, s.M, s.F, 32, 32, sw128) ||
            !encode_2d(&p.in[1], f32, 4, U, s.M, s.F, 32, 32, sw128))
            return cudaErrorInvalidValue;
        cudaError_t e = launch<false, true, kGateGrad>(s, p, status, st);
        if (e != cudaSuccess) return e;
    }
    {   // dX = dG Wg + dU Wu
        Params<kStore> p{};
        Problem& r = p.pr[0];
        p.problems = 1;
        r.M = s.M; r.N = s.D; r.k_steps = steps(s.F); r.sources = 2;
        if (!operand_map(&r.a[0], dG, s.M, s.F, true, kTileM) || !operand_map(&r.a[1], dU, s.M, s.F, true, kTileM) ||
            !operand_map(&r.b[0], Wg, s.F, s.D, false, 0) || !operand_map(&r.b[1], Wu, s.F, s.D, false, 0) ||
            !encode_2d(&r.c[0], bf16, 2, dX, s.M, s.D, 64, 32, sw128))
            return cudaErrorInvalidValue;
        cudaError_t e = launch<false, true, kStore>(s, p, status, st);
        if (e != cudaSuccess) return e;
    }
    }
    // dWg = dG^T X, dWu = dU^T X, dWd = dY^T H: K is the token
    Params<kStore> p{};
    p.problems = 3;
    const struct { const void *a, *b; int m, n; void* c; } w[3] = {
        {dG, X, s.F, s.D, dWg}, {dU, X, s.F, s.D, dWu}, {dY, H, s.D, s.F, dWd}};
    for (int i = 0; i < 3; ++i) {
        Problem& r = p.pr[i];
        r.M = w[i].m; r.N = w[i].n; r.k_steps = steps(s.M); r.sources = 1;
        if (!operand_map(&r.a[0], w[i].a, s.M, w[i].m, false, 0) || !operand_map(&r.b[0], w[i].b, s.M, w[i].n, false, 0) ||
            !encode_2d(&r.c[0], bf16, 2, w[i].c, w[i].m, w[i].n, 64, 32, sw128))
            return cudaErrorInvalidValue;
    }
    return launch<true, true, kStore>(s, p, status, st);
}

}  // namespace rola
