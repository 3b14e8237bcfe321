// The gated feed-forward's and the linear layer's products for few tokens (bf16 operands, tcgen05):
// every weight is read once for all of them, and that is what bounds the work
// (one token at widths 5120 x 13824: 425 MB of weights, 63 us at the measured
// 6.8 TB/s, and 72 measured; its 0.4 GFLOP are nothing).  More than 96 tokens go in tiles of at most
// 96 side by side, which read the weights from L2 (ffn_few says up to where).
//
// The tokens are the N axis and 128 weight rows the M axis of the tensor core,
// so that a single token costs a tile of 16 columns instead of 128 rows:
//   kUp     g, u (128 features x tokens) = Wg X^T, Wu X^T;  H = phi(g) * u
//   kDown   Y^T  = Wd H^T
//   kGrad   dH^T = Wd^T dY^T  (Wd read MN-major);  H, dG, dU from it and G, U
//   kDX     dX^T = Wg^T dG^T + Wu^T dU^T  (MN-major; one sum over 2 d_ff); a linear layer's dX is one of them
//   kLinear Z^T  = W X^T + b;  Y = R + phi(Z)
// There are too few row tiles to occupy the GPU (12 of 128 rows at d_model
// 1536), so the K axis of a tile is split over a cluster of up to 8 CTAs.  Each
// streams its share through a TMA ring into its own TMEM accumulator, then the
// accumulators meet in the cluster's shared memory: CTA r of s adds the s parts
// of its share of the tokens, in rank order, and writes them.  No partial sum
// goes through global memory and the order of every sum is fixed.  About 110 KB
// of shared memory per CTA let two CTAs share an SM, so up to 304 CTAs stream
// at once (some 30 MB of loads in flight) and the last wave is never nearly empty.
//
// The second kernel of a pair is launched while the first still runs
// (programmatic dependent launch): it loads its first weights, which nothing
// before it writes, and waits for the first kernel only for the tokens.
//
// Warps (192 threads): 0 TMA, 1 products and TMEM, 2-5 epilogue.  Every mbarrier
// wait is bounded; all threads reach the cluster barriers whatever happens.
#include <algorithm>

#include "block_ops.cuh"
#include "cluster.cuh"
#include "linear.cuh"
#include "linear_finish.cuh"
#include "tcgen05.cuh"
#include "tma_2d.cuh"

namespace rola {
namespace {

using namespace tc;

enum Mode { kUp, kDown, kGrad, kDX, kLinear };

constexpr int kTileM = 128, kStepK = 64, kThreads = 192, kMaxStages = 8;
constexpr uint32_t kABytes = kTileM * kStepK * 2;
constexpr uint32_t kSmemBudget = 112 * 1024;                 // two CTAs of an SM's 227 KB
constexpr int kMaxCluster = 8;
constexpr int kMaxTokens = kFfnFewTokens;                    // of a tile: its two sums fit the 112 KB

enum Bar { FULL = 0, EMPTY = FULL + kMaxStages, ACC_FULL = EMPTY + kMaxStages, DRAIN, NUM_BARS };
struct Ctrl {
    uint64_t bar[NUM_BARS];
    uint32_t tmem_base;
    int abort;
};

constexpr size_t kSmemMost = kSmemBudget + sizeof(Ctrl);     // of a CTA, whatever the sizes

struct Params {
    CUtensorMap a[2], b[2];          // weights (kUp: gate and up; kDX: the two sources), tokens
    int M, rows;                     // tokens; weight rows of the output (d_ff or d_model)
    int nt;                          // tokens of a tile, a multiple of 16: the N of the products
    int k_steps, sources;            // K steps of 64 of one source
    int stages, act, skip_first;
    uint32_t stage_bytes, tiles_bytes;   // of a stage; of the tiles in front of the control block
    __nv_bfloat16 *c0, *c1, *c2;     // H / Y / dX; dG, dU
    float *G, *U;                    // kUp: out or NULL; kGrad: in; kLinear: Z in G, out or NULL
    const __nv_bfloat16 *bias, *residual;    // kLinear, or NULL
    int clear;                       // the status word is this kernel's to clear
    DeviceStatus* status;
    uint64_t wait_limit_ns;
};

template <int MODE>
__global__ void __launch_bounds__(kThreads, 2) ffn_few_kernel(const __grid_constant__ Params p)
{
    constexpr bool AMn = MODE == kGrad || MODE == kDX;
    constexpr int ACCS = MODE == kUp ? 2 : 1;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t sbase = smem_u32(smem_raw);
    Ctrl& cb = *reinterpret_cast<Ctrl*>(smem_raw + p.tiles_bytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&cb.bar[i]); };
    auto timeout = [&](int where) {
        if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 128 + where;
    };
    if (tid == 0) {
        // before any CTA can record a timeout, which takes 1 ms at least
        if (p.clear && blockIdx.x == 0 && blockIdx.y == 0) p.status->code = p.status->where = 0;
        cb.abort = 0;
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(bar(FULL + i), 1);
            mbar_init(bar(EMPTY + i), 1);
        }
        mbar_init(bar(ACC_FULL), 1);
        mbar_init(bar(DRAIN), 1);
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&cb.tmem_base), 128 * ACCS);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    // the next kernel of the stream may be launched now; it waits for this one where it has to
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const uint32_t tmem = cb.tmem_base;
    volatile int* abort = &cb.abort;
    const uint64_t limit = p.wait_limit_ns;
    const int s = (int)cluster_size(), rank = (int)cluster_rank();
    const int first_token = blockIdx.y * p.nt, tokens = min(p.M - first_token, p.nt);
    const int tile = blockIdx.x / s, total = p.k_steps * p.sources;
    const int k_begin = (int)((long long)total * rank / s), k_end = (int)((long long)total * (rank + 1) / s);
    const int steps = k_end - k_begin;
    const uint32_t b_off = ACCS * kABytes;               // the tokens' part of a stage

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        // a box per lane: weights on lanes 0, 1 (kUp: Wg and Wu; MN-major: 64 rows each), tokens on lane 2
        bool ok = true;
        auto coords = [&](int i, int& src, int& k0) {
            const int ks = k_begin + i;
            src = ks >= p.k_steps ? 1 : 0;
            k0 = (ks - src * p.k_steps) * kStepK;
        };
        auto load_weights = [&](int i) {
            int src, k0;
            coords(i, src, k0);
            const uint32_t dst = sbase + (i % p.stages) * p.stage_bytes, b = bar(FULL + i % p.stages);
            if (AMn) {
                if (lane < 2) tma_load_2d(dst + lane * 8192, &p.a[src], b, tile * kTileM + lane * 64, k0);
            } else if (lane < ACCS) {
                tma_load_2d(dst + lane * kABytes, &p.a[lane], b, k0, tile * kTileM);
            }
        };
        auto load_tokens = [&](int i) {
            int src, k0;
            coords(i, src, k0);
            if (lane == 2)
                tma_load_2d(sbase + (i % p.stages) * p.stage_bytes + b_off, &p.b[src], bar(FULL + i % p.stages), k0,
                            first_token);
        };
        // test hook: the first stage is never announced nor loaded, so the waits on it run out
        const int first = p.skip_first && steps > 0 ? 1 : 0, ahead = min(p.stages, steps);
        for (int i = first; i < ahead; ++i) {
            if (lane == 0) mbar_expect_tx(bar(FULL + i), p.stage_bytes);
            __syncwarp();
            load_weights(i);
        }
        asm volatile("griddepcontrol.wait;\n" ::: "memory");     // the tokens may be the previous kernel's output
        for (int i = first; i < ahead; ++i) load_tokens(i);
        int i = ahead;
        for (; i < steps; ++i) {
            const int st = i % p.stages;
            ok = __shfl_sync(0xffffffffu, mbar_wait(bar(EMPTY + st), ((i / p.stages) - 1) & 1, abort, limit), 0);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(bar(FULL + st), p.stage_bytes);
            __syncwarp();
            load_weights(i);
            load_tokens(i);
        }
        if (lane == 0) {
            if (!ok) timeout(1);
            // the copies still in flight land before the CTA exits
            int never = 0;
            for (int u = max(i - p.stages, first); u < i; ++u)
                mbar_wait(bar(FULL + u % p.stages), (u / p.stages) & 1, &never, limit);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products
        if (lane == 0) {
            const uint32_t idesc = idesc_bf16(kTileM, p.nt, AMn, false);
            const uint64_t da = smem_desc(sbase, AMn ? 8192 : 16, 1024), db = smem_desc(sbase + b_off, 16, 1024);
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            constexpr uint32_t a_k = AMn ? 128 : 2;
            bool ok = true;
            for (int i = 0; i < steps; ++i) {
                const int st = i % p.stages;
                if (!(ok = mbar_wait(bar(FULL + st), (i / p.stages) & 1, abort, limit))) break;
                fence_after_sync();
                const uint32_t off = st * (p.stage_bytes >> 4);
#pragma unroll
                for (int acc = 0; acc < ACCS; ++acc)
#pragma unroll
                    for (int kk = 0; kk < kStepK / 16; ++kk)
                        mma_ss_split(tmem + acc * 128, a_lo + off + acc * (kABytes >> 4) + kk * a_k, a_hi, b_lo + off + kk * 2,
                                     b_hi, idesc, (i > 0 || kk > 0) ? 1u : 0u);
                mma_commit(bar(EMPTY + st));
            }
            if (ok) mma_commit(bar(ACC_FULL));
            else timeout(2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(DRAIN));
            mbar_wait(bar(DRAIN), 0, &never, limit);
        }
        __syncwarp();
    } else {
        // this CTA's part of the sums into shared memory: [acc][token][128 rows] over the stages, which
        // every product has read
        const int q = warp & 3, row = q * 32 + lane;
        const bool ok = mbar_wait_warp(bar(ACC_FULL), 0, abort, limit);
        if (!ok) timeout(3);
        else {
            fence_after_sync();
            for (int acc = 0; acc < ACCS; ++acc)
                for (int c = 0; c < p.nt; c += 16) {
                    float v[16];
                    tmem_ld16(tmem + ((uint32_t)(q * 32) << 16) + acc * 128 + c, v);
                    tmem_ld_wait(v);
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        *reinterpret_cast<float*>(smem_raw + ((size_t)(acc * p.nt + c + e) * kTileM + row) * 4) = v[e];
                }
        }
    }
    fence_before_sync();
    cluster_sync();
    fence_after_sync();
    if (warp == 1) tmem_dealloc(tmem, 128 * ACCS);
    // a warp per token of this CTA's share, four neighbouring features a lane (d_model and d_ff are multiples of 8).
    // (A feature a lane and the tokens one after another on four warps, each a round trip to the peers:
    // their gradients of 77 tokens at widths 1536 x 4096 15.3 and 18.5 us, 10.1 and 13.8 so.)
    const int f = tile * kTileM + lane * 4, m1 = tokens * (rank + 1) / s;
    for (int m = tokens * rank / s + warp; m < m1 && f < p.rows; m += kThreads / 32) {
        // all parts are on their way before the first is added
        float4 part[ACCS][kMaxCluster];
#pragma unroll
        for (int acc = 0; acc < ACCS; ++acc)
#pragma unroll
            for (int r = 0; r < kMaxCluster; ++r)
                part[acc][r] = r < s ? ld_peer(peer(sbase + (uint32_t)((acc * p.nt + m) * kTileM + lane * 4) * 4, r))
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
        auto sum = [&](int acc, float (&x)[4]) {
            x[0] = part[acc][0].x; x[1] = part[acc][0].y; x[2] = part[acc][0].z; x[3] = part[acc][0].w;
#pragma unroll
            for (int r = 1; r < kMaxCluster; ++r) {
                x[0] += part[acc][r].x; x[1] += part[acc][r].y; x[2] += part[acc][r].z; x[3] += part[acc][r].w;
            }
        };
        float x[4];
        sum(0, x);
        const size_t at = (size_t)(first_token + m) * p.rows + f;
        if constexpr (MODE == kUp) {
            float u[4], h[4];
            sum(1, u);
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) h[e] = act.phi(x[e]) * u[e];
            });
            store4(p.c0 + at, make_float4(h[0], h[1], h[2], h[3]));
            if (p.G) {
                *reinterpret_cast<float4*>(p.G + at) = make_float4(x[0], x[1], x[2], x[3]);
                *reinterpret_cast<float4*>(p.U + at) = make_float4(u[0], u[1], u[2], u[3]);
            }
        } else if constexpr (MODE == kGrad) {
            const float4 gv = *reinterpret_cast<const float4*>(p.G + at), uv = *reinterpret_cast<const float4*>(p.U + at);
            const float g[4] = {gv.x, gv.y, gv.z, gv.w}, u[4] = {uv.x, uv.y, uv.z, uv.w};
            float h[4], dg[4], du[4];
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a = 0.0f, da = 0.0f;
                    act.grad(g[e], a, da);
                    h[e] = a * u[e];
                    dg[e] = x[e] * u[e] * da;
                    du[e] = x[e] * a;
                }
            });
            store4(p.c0 + at, make_float4(h[0], h[1], h[2], h[3]));
            store4(p.c1 + at, make_float4(dg[0], dg[1], dg[2], dg[3]));
            store4(p.c2 + at, make_float4(du[0], du[1], du[2], du[3]));
        } else if constexpr (MODE == kLinear) {
            if (p.bias) {
                const float4 b = load4(p.bias + f);
                x[0] += b.x; x[1] += b.y; x[2] += b.z; x[3] += b.w;
            }
            if (p.G) *reinterpret_cast<float4*>(p.G + at) = make_float4(x[0], x[1], x[2], x[3]);
            linear_phi(p.act, x);
            if (p.residual) {
                const float4 r = load4(p.residual + at);
                x[0] += r.x; x[1] += r.y; x[2] += r.z; x[3] += r.w;
            }
            store4(p.c0 + at, make_float4(x[0], x[1], x[2], x[3]));
        } else {
            store4(p.c0 + at, make_float4(x[0], x[1], x[2], x[3]));
        }
    }
    cluster_sync();                                      // the peers' shared memory stays until all have read it
}

// Stands for the kernels below where the occupancy is asked for: of one that allocates tensor memory the runtime
// counts one CTA an SM, however little it allocates.
__global__ void __launch_bounds__(kThreads, 2) like_ffn_few_kernel() {}

// ---------------------------------------------------------------- host side

bool map_of(CUtensorMap* m, const void* p, int rows, int cols, int box_rows)
{
    return encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, rows, cols, kStepK, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int MODE>
cudaError_t launch(const FfnShape& s, Params& p, bool dependent, DeviceStatus* status, cudaStream_t st)
{
    constexpr int ACCS = MODE == kUp ? 2 : 1;
    p.M = s.M;
    p.act = s.act;
    p.status = status;
    p.wait_limit_ns = s.wait_limit_ns;
    p.skip_first = s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY ? 1 : 0;
    const int tiles = (p.rows + kTileM - 1) / kTileM, total = p.k_steps * p.sources;
    const int token_tiles = (s.M + p.nt - 1) / p.nt;
    p.stage_bytes = ACCS * kABytes + p.nt * kStepK * 2;
    p.stages = (int)((kSmemBudget - sizeof(Ctrl)) / p.stage_bytes);
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    const uint32_t sums = (uint32_t)(ACCS * p.nt * kTileM * 4);
    p.tiles_bytes = p.stages * p.stage_bytes;
    if (p.tiles_bytes < sums) p.tiles_bytes = sums;
    p.tiles_bytes = (p.tiles_bytes + 1023) & ~1023u;
    const size_t smem = p.tiles_bytes + sizeof(Ctrl);
    auto kernel = ffn_few_kernel<MODE>;
    // the limit is the kernel's, not the call's: every call sets it to the same, since another thread may be about to launch
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
    if (e != cudaSuccess) return e;
    // As many CTAs as two per SM hold, each with two K steps at least, and with twice the weights of the sums that
    // it takes from its peers (77 tokens at widths 1536 x 4096: 24.7 us, 26.9 with 8 CTAs a tile in the up products).
    int cluster = 304 / (tiles * token_tiles);
    cluster = std::min(std::min(cluster, kMaxCluster), std::min(total / 2, total * 16 / p.nt));
    cluster = std::max(cluster, 1);
    cudaLaunchConfig_t cfg{};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    // A cluster's CTAs share a GPC, and not every size fills its SMs: 38 clusters of 7 are in flight at once, 46 of 6.
    // A few tiles left for a second wave cost a whole one (one token at 5120 x 13824, whose 40 down tiles
    // would take 7: 87 us, with 6 72).
    e = cudaFuncSetAttribute(like_ffn_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
    if (e != cudaSuccess) return e;
    for (;; --cluster) {
        at[0].val.clusterDim.x = cluster;
        cfg.gridDim = dim3(tiles * cluster, token_tiles);
        if (cluster == 1) break;
        int fit = 0;
        e = cudaOccupancyMaxActiveClusters(&fit, like_ffn_few_kernel, &cfg);
        if (e != cudaSuccess) return e;
        if (fit >= tiles * token_tiles) break;
    }
    cfg.numAttrs = dependent ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

int steps(int k) { return (k + kStepK - 1) / kStepK; }

Params params(const FfnShape& s)
{
    Params p{};
    const int tiles = (s.M + kMaxTokens - 1) / kMaxTokens;
    p.nt = ((s.M + tiles - 1) / tiles + 15) / 16 * 16;
    return p;
}

}  // namespace

// Up to 96 tokens, and beyond (up to seven tiles of 96) while the tiles of 128 x 256 would leave half of the 152 SMs
// idle in the down product and the weights, which every tile of tokens reads again from L2, stay below 3 x 1.5e8
// elements over all tiles.  Forward, us, this form / tiles of 128 x 256, the weights from HBM:
//   1536 x 4096: 130 tokens 27 / 45, 400 43 / 45, 600 51 / 54, 900 70 / 54, 1500 100 / 63
//   5120 x 13824: 130 tokens 120 / 158, 200 191 / 158, 300 261 / 183
//   512 x 8192: 130 tokens 31 / 63, 600 50 / 69, 1200 79 / 75, 4500 251 / 113
//   64 x 4096: 600 tokens 25 / 32, 1500 39 / 35, 9600 164 / 69;  256 x 1024: 130 tokens 21 / 19, 600 24 / 19
// (What decides is how often the weights are read against how long a tile's K axis is; these two numbers are within 1.4 %
// of the better form on average over 140 measured calls of nine widths, and within a third in the worst.)  The
// backward's products read their weights MN-major and gain nothing from tokens side by side (dX of 300 tokens at
// 1536 x 4096: 71 us against 46).
bool ffn_few(const FfnShape& s)
{
    const int64_t tiles = (s.M + kMaxTokens - 1) / kMaxTokens;
    return tiles == 1 || (tiles <= 7 && tiles * s.D * s.F <= 150000000 &&
                          (int64_t)((s.M + 127) / 128) * ((s.D + 255) / 256) < 76);
}

cudaError_t launch_ffn_few(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd, void* H,
                           float* G, float* U, void* Y, DeviceStatus* status, cudaStream_t st)
{
    Params p = params(s);
    p.rows = s.F; p.k_steps = steps(s.D); p.sources = 1;
    p.c0 = static_cast<__nv_bfloat16*>(H); p.G = G; p.U = U;
    if (!map_of(&p.a[0], Wg, s.F, s.D, kTileM) || !map_of(&p.a[1], Wu, s.F, s.D, kTileM) || !map_of(&p.b[0], X, s.M, s.D, p.nt))
        return cudaErrorInvalidValue;
    cudaError_t e = launch<kUp>(s, p, false, status, st);
    if (e != cudaSuccess) return e;
    p = params(s);
    p.rows = s.D; p.k_steps = steps(s.F); p.sources = 1;
    p.c0 = static_cast<__nv_bfloat16*>(Y);
    if (!map_of(&p.a[0], Wd, s.D, s.F, kTileM) || !map_of(&p.b[0], H, s.M, s.F, p.nt)) return cudaErrorInvalidValue;
    return launch<kDown>(s, p, true, status, st);
}

cudaError_t launch_ffn_few_grad(const FfnShape& s, const void* Wg, const void* Wu, const void* Wd, const float* G,
                                const float* U, const void* dY, void* H, void* dG, void* dU, void* dX,
                                DeviceStatus* status, cudaStream_t st)
{
    Params p = params(s);
    p.rows = s.F; p.k_steps = steps(s.D); p.sources = 1;
    p.c0 = static_cast<__nv_bfloat16*>(H); p.c1 = static_cast<__nv_bfloat16*>(dG); p.c2 = static_cast<__nv_bfloat16*>(dU);
    p.G = const_cast<float*>(G); p.U = const_cast<float*>(U);
    if (!map_of(&p.a[0], Wd, s.D, s.F, kStepK) || !map_of(&p.b[0], dY, s.M, s.D, p.nt)) return cudaErrorInvalidValue;
    cudaError_t e = launch<kGrad>(s, p, false, status, st);
    if (e != cudaSuccess) return e;
    p = params(s);
    p.rows = s.D; p.k_steps = steps(s.F); p.sources = 2;
    p.c0 = static_cast<__nv_bfloat16*>(dX);
    if (!map_of(&p.a[0], Wg, s.F, s.D, kStepK) || !map_of(&p.a[1], Wu, s.F, s.D, kStepK) ||
        !map_of(&p.b[0], dG, s.M, s.F, p.nt) || !map_of(&p.b[1], dU, s.M, s.F, p.nt))
        return cudaErrorInvalidValue;
    return launch<kDX>(s, p, true, status, st);
}

// One tile of up to 96 tokens, and up to seven while the weights that they all read stay below 3.2e7 elements.  Us, this
// form / tiles of CTA pairs, weights from HBM:
//   1536 x 1536: 128 tokens 7.5 / 11.4, 672 11.3 / 14.2;  1536 x 6144: 256 tokens 14.2 / 15.3, 384 22.1 / 15.7
//   8192 x 1024: 384 tokens 16.2 / 16.9, 514 20.6 / 18.2;  1536 x 9216: 192 tokens 14.9 / 15.7, 256 21.4 / 15.7
//   5120 x 5120: 96 tokens 16.1 / 19.3, 128 20.4 / 19.8;  5120 x 30720: 96 tokens 62 / 66, 128 101 / 66
bool linear_few(const LinShape& s)
{
    const int64_t tiles = (s.M + kMaxTokens - 1) / kMaxTokens;
    return tiles == 1 || (tiles <= 7 && tiles * s.K * s.N <= 32000000);
}

cudaError_t launch_linear_few(const LinShape& s, const void* X, const void* W, const void* b, const void* R, void* Y,
                              float* Z, DeviceStatus* status, cudaStream_t st)
{
    const FfnShape fs{s.M, s.K, s.N, s.act, s.wait_limit_ns, s.debug_flags};
    Params p = params(fs);
    p.rows = s.N; p.k_steps = steps(s.K); p.sources = 1;
    p.c0 = static_cast<__nv_bfloat16*>(Y);
    p.G = Z;
    p.bias = static_cast<const __nv_bfloat16*>(b);
    p.residual = static_cast<const __nv_bfloat16*>(R);
    p.clear = 1;
    if (!map_of(&p.a[0], W, s.N, s.K, kTileM) || !map_of(&p.b[0], X, s.M, s.K, p.nt)) return cudaErrorInvalidValue;
    return launch<kLinear>(fs, p, false, status, st);
}

cudaError_t launch_linear_few_dx(const LinShape& s, const void* W, const void* dZ, void* dX, bool clear,
                                 DeviceStatus* status, cudaStream_t st)
{
    const FfnShape fs{s.M, s.K, s.N, s.act, s.wait_limit_ns, s.debug_flags};
    Params p = params(fs);
    p.rows = s.K; p.k_steps = steps(s.N); p.sources = 1;
    p.c0 = static_cast<__nv_bfloat16*>(dX);
    p.clear = clear;
    if (!map_of(&p.a[0], W, s.N, s.K, kStepK) || !map_of(&p.b[0], dZ, s.M, s.N, p.nt)) return cudaErrorInvalidValue;
    return launch<kDX>(fs, p, false, status, st);
}

}  // namespace rola
