// Gradients of the dense softmax attention on the 5th-generation tensor cores
// (bf16 operands, fp32 accumulation in TMEM), recomputing the probabilities.
//
//   P = 2^(scale log2(e) q k^T - lse log2(e)),  dP = dO v^T,  dS = P (dP - D),  D = dO . o
//   dq = scale dS k        (attention_dq_tc_kernel,   an item is 128 rows,  its keys in stages of 64)
//   dv = P^T dO,  dk = scale dS^T q   (attention_dkdv_tc_kernel, an item is 128 keys, its rows in stages of 64)
//
// Two kernels instead of one: each accumulator then stays in TMEM over its whole
// sum, so nothing is added in memory and the order of every sum is fixed; the
// price is S and dP computed twice (7 products of 2 x 128 x 128 x 64 FLOP instead of 5).
//
// An item's 128 rows (or keys) are the TMEM lanes.  Stage n (64 keys or rows):
//   S_b  = A_0 B_0^T,  dP_b = A_1 B_1^T      b = n & 1, 128 x 64, A and B K-major in shared memory
//   dq:    A = (Q, dO), B = (K, V); dS overwrites the first half of S_b as bf16 and is the TMEM operand of
//          dQ += dS K          (K read MN-major from the same tile)
//   dk/dv: A = (K, V), B = (Q, dO): S and dP come out transposed, so P^T and dS^T are TMEM operands too:
//          dV += P^T dO,  dK += dS^T Q
// One thread issues all products, in the order  grad(n) SdP(n + 2) (at an item's
// end the next item's SdP as soon as its A has arrived): products of one thread execute in order, so SdP(n + 2) may overwrite what grad(n) reads.
// Two groups of four warps take the even and the odd stages, so the element-wise
// work of one stage runs under the products of the other.
//
// A key past the sequence's length has P = dS = 0 by selection whatever it
// holds, and in the dq kernel, where K is also the other operand of a sum over
// keys, its rows of K are zeroed in shared memory (0 x NaN would be NaN).
// If a row tile's keys fit one stage, D = sum_j P dP is taken from the stage
// itself instead of dO . o, whose o carries the output's bf16 rounding: over few
// keys that error is not small beside dP - D.
//
// Warps (320 threads, one persistent CTA per SM): 0-3 and 4-7 the two groups, 8
// TMA, 9 products.  Every mbarrier wait is bounded.
#include "attention_tc.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kM = 128, kN = 64;                          // lanes of an item, columns of a stage
constexpr int kTmaWarp = 8, kMmaWarp = 9, kThreads = 320;
constexpr uint32_t kABytes = kM * kDh * 2, kBBytes = kN * kDh * 2;   // [d-chunk][rows][64]
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemP = 128, kTmemAcc = 256;   // S_b at 64 b, dP_b at 128 + 64 b

template <bool DQ>
struct Cfg {
    static constexpr int AB = 1, NS = 5;
    static constexpr uint32_t kSmemA = 0, kSmemB = AB * 2 * kABytes, kSmemTiles = kSmemB + NS * 2 * kBBytes;
    static constexpr int A_FULL = 0, A_EMPTY = A_FULL + AB, B_FULL = A_EMPTY + AB, B_EMPTY = B_FULL + NS,
                         S_FULL = B_EMPTY + NS, DS_FULL = S_FULL + 2, O_FULL = DS_FULL + 2, O_EMPTY = O_FULL + 2,
                         DRAIN = O_EMPTY + 2, NUM_BARS = DRAIN + 1;
};

struct Cols {                                             // of a stage's 64 rows (dk/dv)
    alignas(16) float lse2[kN];
    alignas(16) float D[kN];
    alignas(16) int seen[kN];
};
template <bool DQ>
struct Ctrl {
    Cols cols[2];
    uint64_t bar[Cfg<DQ>::NUM_BARS];
    uint32_t tmem_base;
    int abort;
};
static_assert(Cfg<true>::kSmemTiles + sizeof(Ctrl<true>) <= 232448 &&
                  Cfg<false>::kSmemTiles + sizeof(Ctrl<false>) <= 232448,
              "tiles and control block fit the 227 KB a CTA may have");

struct Params {
    AttnShape s;
    const int32_t* kv_len;
    const float* lse;
    float* D;
    __nv_bfloat16 *out0, *out1;       // dq; or dv and dk
    DeviceStatus* status;
    int tiles, items;                 // item tiles of a head; tiles heads
};

// One item and the walk over its stages: t in [t0, end), those that `next` returns.
template <bool DQ>
struct Item {
    int head, x0, len;                // x0: first row (dq) or key (dk/dv)
    int end;                          // stages of the whole axis
    __device__ __forceinline__ Item() {}
    __device__ __forceinline__ Item(const Params& p, int i)
    {
        const AttnShape& s = p.s;
        int tile;
        if (s.causal) {               // the longest items of every head first: the last rows, the first keys
            tile = DQ ? p.tiles - 1 - i / s.heads : i / s.heads;
            head = i % s.heads;
        } else {
            head = i / p.tiles;
            tile = i - head * p.tiles;
        }
        x0 = tile * kM;
        len = attn_len(s, p.kv_len, head / s.Hk);
        if constexpr (DQ) end = (attn_seen_most(s, len, x0, min(x0 + kM, s.R) - 1) + kN - 1) / kN;
        else end = x0 < len ? (s.R + kN - 1) / kN : 0;
    }
    // the first stage >= t with something to do, or end
    __device__ __forceinline__ int next(const AttnShape& s, int t) const
    {
        if constexpr (!DQ) {
            while (s.causal && t < end) {
                const int r0 = t * kN, r1 = min(r0 + kN, s.R) - 1;
                if (attn_seen_most(s, len, r0, r1) > x0) break;
                // no row of the stage sees key x0: on to the stage of the head's first row that does
                t = max(t + 1, (r0 / s.Lq * s.Lq + min(max(x0 - len + s.Lq, 0), s.Lq - 1)) / kN);
            }
        }
        return min(t, end);
    }
};

template <bool DQ>
__global__ void __launch_bounds__(kThreads, 1) attention_bwd_tc_kernel(const __grid_constant__ CUtensorMap map_a0,
                                                                       const __grid_constant__ CUtensorMap map_a1,
                                                                       const __grid_constant__ CUtensorMap map_b0,
                                                                       const __grid_constant__ CUtensorMap map_b1,
                                                                       const Params p)
{
    using C = Cfg<DQ>;
    constexpr int AB = C::AB, NS = C::NS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {     // the 128-byte swizzle atoms need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(&p.status->code, 0, (int)ROLA_ERR_UNSUPPORTED);
        return;
    }
    Ctrl<DQ>& sm = *reinterpret_cast<Ctrl<DQ>*>(smem_raw + C::kSmemTiles);
    const uint32_t sbase = smem_u32(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&sm.bar[i]); };
    auto timeout = [&](int where) {
        if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = (DQ ? 96 : 112) + where;
    };
    const AttnShape& s = p.s;
    const uint64_t limit = s.wait_limit_ns;

    if (tid == 0) {
        sm.abort = 0;
        for (int i = 0; i < AB; ++i) {
            mbar_init(bar(C::A_FULL + i), 1);
            mbar_init(bar(C::A_EMPTY + i), 1);
        }
        for (int i = 0; i < NS; ++i) {
            mbar_init(bar(C::B_FULL + i), 1);
            mbar_init(bar(C::B_EMPTY + i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(C::S_FULL + i), 1);
            mbar_init(bar(C::DS_FULL + i), 4);
            mbar_init(bar(C::O_FULL + i), 1);
            mbar_init(bar(C::O_EMPTY + i), 8);
        }
        mbar_init(bar(C::DRAIN), 1);
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    volatile int* abort = &sm.abort;

    if (warp == kTmaWarp) {
        // ------------------------------------------------------------ TMA producer
        // lanes 0-3: d-chunk lane & 1 of operand lane >> 1, one box each (a lane's copies run one after another)
        const int chunk = lane & 1;
        const CUtensorMap *ma = lane & 2 ? &map_a1 : &map_a0, *mb = lane & 2 ? &map_b1 : &map_b0;
        bool ok = true;
        int na = 0, nb = 0;
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
            const Item<DQ> it(p, i);
            int t = it.next(s, 0);
            if (t >= it.end) continue;
            const int as = na % AB;
            if (na >= AB) ok = mbar_wait(bar(C::A_EMPTY + as), ((na / AB) - 1) & 1, abort, limit);
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(bar(C::A_FULL + as), 2 * kABytes);
            __syncwarp();
            if (lane < 4)
                tma_load_3d(sbase + C::kSmemA + (as * 2 + (lane >> 1)) * kABytes + chunk * (kABytes / 2), ma,
                            bar(C::A_FULL + as), chunk * 64, it.x0, it.head);
            ++na;
            for (; t < it.end; t = it.next(s, t + 1), ++nb) {
                const int st = nb % NS;
                if (nb >= NS) ok = mbar_wait(bar(C::B_EMPTY + st), ((nb / NS) - 1) & 1, abort, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                // test hook: the CTA's first stage is never loaded, so the waits on it run out
                const bool skip = (s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) && nb == 0;
                if (lane == 0 && !skip) mbar_expect_tx(bar(C::B_FULL + st), 2 * kBBytes);
                __syncwarp();
                if (lane < 4 && !skip)
                    tma_load_3d(sbase + C::kSmemB + (st * 2 + (lane >> 1)) * kBBytes + chunk * (kBBytes / 2), mb,
                                bar(C::B_FULL + st), chunk * 64, t * kN, it.head);
            }
        }
        if (!ok && lane == 0) timeout(1);
        // every copy this warp issued lands before the CTA exits (bounded by time only)
        if (lane == 0) {
            int never = 0;
            for (int u = na > AB ? na - AB : 0; u < na; ++u) mbar_wait(bar(C::A_FULL + u % AB), (u / AB) & 1, &never, limit);
            for (int u = nb > NS ? nb - NS : 0; u < nb; ++u) mbar_wait(bar(C::B_FULL + u % NS), (u / NS) & 1, &never, limit);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ products
        // The whole warp runs the loop (it zeroes rows of K together); lane 0 issues.
        const uint32_t id_s = idesc_bf16(kM, kN, false, false), id_g = idesc_bf16(kM, kDh, false, true);
        const uint64_t da = smem_desc(sbase + C::kSmemA, 16, 1024), db = smem_desc(sbase + C::kSmemB, 16, 1024);
        const uint64_t dg = smem_desc(sbase + C::kSmemB, kBBytes / 2, 1024);     // the same tiles read MN-major
        const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
        const uint32_t g_lo = (uint32_t)dg, g_hi = (uint32_t)(dg >> 32);
        bool ok = true;
        auto wait = [&](int b, int parity) {
            if (ok) ok = __shfl_sync(0xffffffffu, mbar_wait(bar(b), parity, abort, limit), 0);
            return ok;
        };
        // a position in the sequence of all stages of this CTA
        struct Walk {
            Item<DQ> it;
            int i, t, nt, item, stage;    // nt: the item's next stage; item, stage: running numbers
        };
        auto open = [&](Walk& w) {        // the first stage of item w.i or of the first after it that has one
            for (; w.i < p.items; w.i += gridDim.x) {
                w.it = Item<DQ>(p, w.i);
                w.t = w.it.next(s, 0);
                if (w.t < w.it.end) {
                    w.nt = w.it.next(s, w.t + 1);
                    return;
                }
            }
        };
        auto advance = [&](Walk& w) {
            ++w.stage;
            if (w.nt < w.it.end) {
                w.t = w.nt;
                w.nt = w.it.next(s, w.t + 1);
            } else {
                ++w.item;
                w.i += gridDim.x;
                open(w);
            }
        };
        // the first stage of an item is the one no earlier stage of it precedes
        int opened = -1;                  // items whose A has been waited for
        auto sdp = [&](Walk& w) {
            const int as = w.item % AB, st = w.stage % NS, b = w.stage & 1;
            if (opened != w.item) {
                if (!wait(C::A_FULL + as, (w.item / AB) & 1)) return;
                opened = w.item;
            }
            if (!wait(C::B_FULL + st, (w.stage / NS) & 1)) return;
            if constexpr (DQ) {
                const int valid = w.it.len - w.t * kN;
                if (valid < kN) {         // rows of K past the length (a row: 128 bytes in each d-chunk)
                    const uint32_t k = sbase + C::kSmemB + st * 2 * kBBytes;
                    for (int e = lane; e < (kN - valid) * 16; e += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};\n" ::"r"(
                                         k + ((e & 8) ? kBBytes / 2 : 0) + (valid + (e >> 4)) * 128 + (e & 7) * 16),
                                     "r"(0)
                                     : "memory");
                    fence_proxy_async_smem();
                    __syncwarp();
                }
            }
            fence_after_sync();
            if (lane == 0) {
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const uint32_t a = a_lo + (as * 2 + o) * (kABytes >> 4), bb = b_lo + (st * 2 + o) * (kBBytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        mma_ss_split(tmem + (o ? kTmemP : kTmemS) + b * 64, a + (kk >> 2) * (kABytes >> 5) + (kk & 3) * 2,
                                     a_hi, bb + (kk >> 2) * (kBBytes >> 5) + (kk & 3) * 2, b_hi, id_s, kk > 0 ? 1u : 0u);
                }
                mma_commit(bar(C::S_FULL + b));
                if (w.nt >= w.it.end) mma_commit(bar(C::A_EMPTY + as));
            }
            __syncwarp();
            advance(w);
        };
        Walk w{}, v{};
        w.i = v.i = blockIdx.x;
        open(w);
        open(v);
        bool fresh = true;                // v is at its item's first stage
        while (ok && v.i < p.items) {
            // up to two stages ahead; the next item's first only once its A is there, unless nothing else is left to do
            while (ok && w.i < p.items && w.stage - v.stage < 2) {
                if (opened != w.item && w.stage != v.stage &&
                    !__shfl_sync(0xffffffffu, mbar_try_wait(bar(C::A_FULL + w.item % AB), (w.item / AB) & 1), 0))
                    break;
                sdp(w);
            }
            if (!ok) break;
            const int st = v.stage % NS, b = v.stage & 1, ob = DQ ? v.item & 1 : 0;
            const bool last = v.nt >= v.it.end;
            if (!wait(C::DS_FULL + b, (v.stage >> 1) & 1)) break;
            if (fresh) {                  // the accumulators of two items (dq) or one item ago have been read
                const int ago = DQ ? 2 : 1;
                if (v.item >= ago && !wait(C::O_EMPTY + ob, (v.item / ago - 1) & 1)) break;
            }
            fence_after_sync();
            if (lane == 0) {
                // 16 columns of the stage: 8 TMEM columns of the operand, 2 KB of the tile
                if constexpr (DQ) {
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_ts_split(tmem + kTmemAcc + ob * 128, tmem + kTmemS + b * 64 + kk * 8,
                                     g_lo + st * 2 * (kBBytes >> 4) + kk * 128, g_hi, id_g, (!fresh || kk > 0) ? 1u : 0u);
                } else {
#pragma unroll
                    for (int o = 0; o < 2; ++o)          // dV += P^T dO, dK += dS^T Q
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_ts_split(tmem + kTmemAcc + o * 128, tmem + (o ? kTmemP : kTmemS) + b * 64 + kk * 8,
                                         g_lo + (st * 2 + 1 - o) * (kBBytes >> 4) + kk * 128, g_hi, id_g,
                                         (!fresh || kk > 0) ? 1u : 0u);
                }
                mma_commit(bar(C::B_EMPTY + st));
                if (last) mma_commit(bar(C::O_FULL + ob));
            }
            __syncwarp();
            fresh = last;
            advance(v);
        }
        if (lane == 0) {
            if (!ok) timeout(2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(C::DRAIN));
            mbar_wait(bar(C::DRAIN), 0, &never, limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ element-wise work + epilogue
        const int g = warp >> 2, gt = tid & 127;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const float c_log2 = s.scale_log2, log2e = 1.4426950408889634f;
        bool ok = true;
        int stage = 0, items = 0;
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
            const Item<DQ> it(p, i);
            const int x = it.x0 + gt;                     // this thread's row (dq) or key (dk/dv)
            int t = it.next(s, 0);
            const bool any = t < it.end;
            const size_t rows = (size_t)it.head * s.R;
            if constexpr (DQ) {
                const bool in = x < s.R;
                const int seen = in ? attn_seen(s, it.len, x) : 0;
                const int least = any ? attn_seen_least(s, it.len, it.x0, min(it.x0 + kM, s.R) - 1) : 0;
                const bool own_D = it.end == 1;
                const float neg_lse = in ? -p.lse[rows + x] * log2e : 0.0f;
                float D = in && any && !own_D ? p.D[rows + x] : 0.0f;
                for (; t < it.end; ++t, ++stage) {
                    const int b = stage & 1;
                    if (b != g) continue;
                    if (!(ok = mbar_wait(bar(C::S_FULL + b), (stage >> 1) & 1, abort, limit))) break;
                    fence_after_sync();
                    float pr[64], dp[64];
                    row_load<64>(tmem + lane_off + kTmemS + b * 64, pr);
                    row_load<64>(tmem + lane_off + kTmemP + b * 64, dp);
                    const int m = t * kN + kN > least || it.x0 + kM > s.R ? seen - t * kN : kN;
#pragma unroll
                    for (int j = 0; j < 64; j += 2) {
                        ffma2(pr[j], pr[j + 1], c_log2, neg_lse);
                        pr[j] = fast_exp2(pr[j]);
                        pr[j + 1] = fast_exp2(pr[j + 1]);
                    }
                    if (m < kN) {
#pragma unroll
                        for (int j = 0; j < 64; ++j)
                            if (j >= m) pr[j] = dp[j] = 0.0f;
                    }
                    if (own_D) {
                        float d0 = 0.0f, d1 = 0.0f;
#pragma unroll
                        for (int j = 0; j < 64; j += 2) {
                            d0 = fmaf(pr[j], dp[j], d0);
                            d1 = fmaf(pr[j + 1], dp[j + 1], d1);
                        }
                        D = d0 + d1;
                        if (in) p.D[rows + x] = D;
                    }
                    uint32_t pk[32];
#pragma unroll
                    for (int j = 0; j < 64; j += 2) pk[j >> 1] = pack_bf16(pr[j] * (dp[j] - D), pr[j + 1] * (dp[j + 1] - D));
                    tmem_st16(tmem + lane_off + kTmemS + b * 64, *reinterpret_cast<const float(*)[16]>(&pk[0]));
                    tmem_st16(tmem + lane_off + kTmemS + b * 64 + 16, *reinterpret_cast<const float(*)[16]>(&pk[16]));
                    tmem_st_wait();
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::DS_FULL + b));
                }
            } else {
                Cols& cols = sm.cols[g];
                // this thread's share of a stage's row values: threads 0-63 lse and the row's limit, 64-127 D
                float val = 0.0f;
                int lim = 0;
                auto fetch = [&](int tt) {
                    const int r = tt * kN + (gt & 63);
                    const bool in = r < s.R;
                    lim = in ? attn_seen(s, it.len, r) : 0;
                    // a row past the end: p = 2^(-inf) = 0
                    val = gt < 64 ? (in ? -p.lse[rows + r] * log2e : -INFINITY) : (in ? p.D[rows + r] : 0.0f);
                };
                int mine = -1;                            // the stage whose values `val` holds
                while (t < it.end) {
                    const int b = stage & 1, nt = it.next(s, t + 1);
                    if (b == g) {
                        if (mine != t) fetch(t);
                        bar_sync(1 + g, 128);             // the previous stage's values have been read
                        if (gt < 64) {
                            cols.lse2[gt] = val;
                            cols.seen[gt] = lim;
                        } else {
                            cols.D[gt - 64] = val;
                        }
                        bar_sync(1 + g, 128);
                        // the group's next stage: its values come while this one is worked on
                        mine = nt < it.end ? it.next(s, nt + 1) : it.end;
                        if (mine < it.end) fetch(mine);
                        const int r0 = t * kN, r1 = min(r0 + kN, s.R) - 1;
                        const bool whole = it.x0 + kM <= attn_seen_least(s, it.len, r0, r1);
                        if (!(ok = mbar_wait(bar(C::S_FULL + b), (stage >> 1) & 1, abort, limit))) break;
                        fence_after_sync();
                        // two halves of 32 rows, so that half of the stage is in registers
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float pr[32], dp[32];
                            row_load<32>(tmem + lane_off + kTmemS + b * 64 + h * 32, pr);
                            row_load<32>(tmem + lane_off + kTmemP + b * 64 + h * 32, dp);
                            uint32_t pp[16], pd[16];
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(&cols.lse2[h * 32 + j]);
                                const float4 D = *reinterpret_cast<const float4*>(&cols.D[h * 32 + j]);
                                float q0 = fast_exp2(fmaf(pr[j], c_log2, l.x)), q1 = fast_exp2(fmaf(pr[j + 1], c_log2, l.y));
                                float q2 = fast_exp2(fmaf(pr[j + 2], c_log2, l.z)), q3 = fast_exp2(fmaf(pr[j + 3], c_log2, l.w));
                                float e0 = dp[j], e1 = dp[j + 1], e2 = dp[j + 2], e3 = dp[j + 3];
                                if (!whole) {
                                    const int4 n = *reinterpret_cast<const int4*>(&cols.seen[h * 32 + j]);
                                    if (x >= n.x) q0 = e0 = 0.0f;
                                    if (x >= n.y) q1 = e1 = 0.0f;
                                    if (x >= n.z) q2 = e2 = 0.0f;
                                    if (x >= n.w) q3 = e3 = 0.0f;
                                }
                                pp[j >> 1] = pack_bf16(q0, q1);
                                pp[(j >> 1) + 1] = pack_bf16(q2, q3);
                                pd[j >> 1] = pack_bf16(q0 * (e0 - D.x), q1 * (e1 - D.y));
                                pd[(j >> 1) + 1] = pack_bf16(q2 * (e2 - D.z), q3 * (e3 - D.w));
                            }
                            // the halves of P^T and dS^T go where the first half of S and dP was: read already
                            tmem_st16(tmem + lane_off + kTmemS + b * 64 + h * 16, *reinterpret_cast<const float(*)[16]>(pp));
                            tmem_st16(tmem + lane_off + kTmemP + b * 64 + h * 16, *reinterpret_cast<const float(*)[16]>(pd));
                        }
                        tmem_st_wait();
                        fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(C::DS_FULL + b));
                    }
                    t = nt;
                    ++stage;
                }
            }
            if (!ok) break;
            // ---- epilogue.  dq: group g writes d 64 g .. +63 of dq; dk/dv: group 0 dv, group 1 dk.
            const int ob = DQ ? items & 1 : 0;
            if (any) {
                if (!(ok = mbar_wait(bar(C::O_FULL + ob), (DQ ? items >> 1 : items) & 1, abort, limit))) break;
                fence_after_sync();
                ++items;
            }
            const float mul = DQ || g == 1 ? s.scale : 1.0f;
            const int width = DQ ? 64 : 128, rows_end = DQ ? s.R : s.Lk;
            const uint32_t acc = tmem + lane_off + kTmemAcc + (DQ ? ob * 128 + g * 64 : g * 128);
            __nv_bfloat16* out = (DQ || g == 0 ? p.out0 : p.out1) + ((size_t)it.head * rows_end + x) * kDh + (DQ ? g * 64 : 0);
            // a key past the length holds zeros or its own garbage: its gradient is 0
            const bool live = DQ || x < it.len;
#pragma unroll
            for (int c = 0; c < width / 32; ++c) {
                float v[32];
                if (any) row_load<32>(acc + c * 32, v);
                if (any && c == width / 32 - 1) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(C::O_EMPTY + ob));
                }
                if (x >= rows_end) continue;
                uint4* dst = reinterpret_cast<uint4*>(out + c * 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = any && live ? v[8 * e + j] * mul : 0.0f;
                    dst[e] = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                }
            }
        }
        if (!ok) timeout(3);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

template <bool DQ>
cudaError_t launch(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    using C = Cfg<DQ>;
    CUtensorMap a0, a1, b0, b1;
    const int rows = DQ ? kM : kN, keys = DQ ? kN : kM;
    if (!encode_rows(DQ ? &a0 : &b0, a.q, s.R, s.heads, rows) || !encode_rows(DQ ? &a1 : &b1, a.dO, s.R, s.heads, rows) ||
        !encode_rows(DQ ? &b0 : &a0, a.k, s.Lk, s.heads, keys) || !encode_rows(DQ ? &b1 : &a1, a.v, s.Lk, s.heads, keys))
        return cudaErrorInvalidValue;
    Params p{};
    p.s = s;
    p.kv_len = a.kv_len;
    p.lse = a.lse_in;
    p.D = a.D;
    p.out0 = static_cast<__nv_bfloat16*>(DQ ? a.dq : a.dv);
    p.out1 = static_cast<__nv_bfloat16*>(a.dk);
    p.status = a.status;
    p.tiles = ((DQ ? s.R : s.Lk) + kM - 1) / kM;
    p.items = p.tiles * s.heads;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = C::kSmemTiles + sizeof(Ctrl<DQ>);
    auto kernel = attention_bwd_tc_kernel<DQ>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kernel<<<p.items < nsm ? p.items : nsm, kThreads, smem, st>>>(a0, a1, b0, b1, p);
    return cudaGetLastError();
}

}  // namespace

// dq first: it leaves in D the row values that the dk / dv kernel reads.
cudaError_t launch_attention_backward_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    cudaError_t e = launch<true>(s, a, st);
    return e != cudaSuccess ? e : launch<false>(s, a, st);
}

}  // namespace rola
