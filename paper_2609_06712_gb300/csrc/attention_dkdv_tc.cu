// Gradients of the dense softmax attention's keys and values on the
// 5th-generation tensor cores (bf16 operands, fp32 accumulation in TMEM),
// recomputing the probabilities.
//
//   P = 2^(scale log2(e) q k^T - lse log2(e)),  dP = dO v^T,  dS = P (dP - D)
//   dv = P^T dO,  dk = scale dS^T q
//
// An item is 128 keys of a head, the TMEM lanes; the rows that see them come in
// stages of 64.  Stage n is of group g = n & 1 (four warps, a key a thread):
//   S_g^T = K Q^T,  dP_g^T = V dO^T     128 x 64, K-major operands in shared memory
//   dV += P^T dO,   dK += dS^T Q        P^T over S_g, dS^T over dP_g (bf16 in TMEM), dO and Q read MN-major
// TMEM (512 columns): S_0, S_1, dP_0, dP_1 (64 each), dV, dK (128 each).  Both
// accumulators stay there over all rows, so nothing is added in memory and the order
// of every sum is fixed.
// A group's S and dP are issued by a thread of its own as soon as the products
// that read P and dS of its last stage are done; a third thread issues dV and dK of
// all stages in order.  So each group goes through scores, P, dP, dS at its own
// pace, under the other's products.  (With stages of 128 rows in which both groups
// work side by side the four steps form one chain of 4100 cycles, 2048 of them products:
// 814 us at 12 heads x 8190 x 8190, 672 us so, 1230 TFLOP/s.  The tensor pipe is then 63 % busy, its
// 128 x 64 products taking 48 cycles each where half a 128 x 128 one would take 32; the rest are waits within
// the groups' chains.  64 bytes a thread are spilled.)
//
// A key past the sequence's length has P = dS = 0 by selection whatever it holds.
// Few items: their rows are split over several (AttnShape::splits_dkv); the parts
// are written in fp32 and added in order by a second kernel.
//
// Warps (384 threads, one persistent CTA per SM): 0-3 and 4-7 the groups, 8 TMA,
// 9 and 10 S and dP of group 0 and 1, 11 gradients.  Every mbarrier wait is bounded.
#include "attention_tc.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kM = 128, kN = 64;                          // keys of an item, rows of a stage
constexpr int kTmaWarp = 8, kSWarp = 9, kGradWarp = 11, kThreads = 384, kSlots = 8;
constexpr uint32_t kABytes = kM * kDh * 2, kBBytes = kN * kDh * 2;        // [d-chunk][rows][64]
constexpr uint32_t kSmemA = 0, kSmemB = 2 * kABytes, kSmemTiles = kSmemB + kSlots * kBBytes;
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemP = 128, kTmemV = 256, kTmemK = 384;

// B: a ring of tiles, Q of stage n in use 2n, dO in 2n + 1.  S_FULL .. K_DONE, COLS: + g.  COLS: a stage's row values
// are in shared memory (a group's warps meet at no barrier of the CTA, whose wait would have no limit).
enum Bar { A_FULL = 0, A_EMPTY, B_FULL, B_EMPTY = B_FULL + kSlots, S_FULL = B_EMPTY + kSlots, DP_FULL = S_FULL + 2,
           P_FULL = DP_FULL + 2, DS_FULL = P_FULL + 2, V_DONE = DS_FULL + 2, K_DONE = V_DONE + 2, O_FULL = K_DONE + 2,
           O_EMPTY, COLS, DRAIN = COLS + 2, NUM_BARS = DRAIN + 3 };

struct Cols {                                             // of a stage's rows
    alignas(16) float lse2[kN];
    alignas(16) float neg_D[kN];
    alignas(16) short seen[kN];                           // keys of the item that the row sees: 0 .. 128
};
struct Ctrl {
    Cols cols[2][2];                                      // [stage / 2 & 1][group]
    uint64_t bar[NUM_BARS];
    uint32_t tmem_base;
    int abort;
};
static_assert(kSmemTiles + sizeof(Ctrl) <= 232448, "tiles and control block fit the 227 KB a CTA may have");

template <bool V>
struct Flag {
    static constexpr bool value = V;
};

struct Params {
    AttnShape s;
    const int32_t* kv_len;
    const float *lse, *D;
    __nv_bfloat16 *dv, *dk;
    float *part_dv, *part_dk;         // with splits: their parts, [splits][heads][keys][128]
    DeviceStatus* status;
    int splits, tiles, items;         // 128-key tiles of a head; tiles heads splits
    bool wide;                        // dv and dk are 32-byte aligned
};

// One item and the walk over its stages: from begin to end, those that `next` returns.
struct Item {
    int head, x0, len, part;          // x0: first key
    int begin, end;                   // stages of this part
    __device__ __forceinline__ Item(const Params& p, int i)
    {
        const AttnShape& s = p.s;
        part = 0;
        if (p.splits > 1) {
            part = i % p.splits;
            i /= p.splits;
        }
        int tile;
        if (s.causal) {               // the longest items of every head first: the first keys
            tile = i / s.heads;
            head = i % s.heads;
        } else {
            head = i / p.tiles;
            tile = i - head * p.tiles;
        }
        x0 = tile * kM;
        len = attn_len(s, p.kv_len, head / s.Hk);
        const int all = x0 < len ? (s.R + kN - 1) / kN : 0;
        begin = 0;
        end = all;
        if (p.splits > 1) {
            begin = (int)((long long)all * part / p.splits);
            end = (int)((long long)all * (part + 1) / p.splits);
        }
        begin = next(s, begin);
    }
    // the first stage >= t with something to do, or end
    __device__ __forceinline__ int next(const AttnShape& s, int t) const
    {
        while (s.causal && t < end) {
            const int r0 = t * kN, r1 = min(r0 + kN, s.R) - 1;
            if (attn_seen_most(s, len, r0, r1) > x0) break;
            // no row of the stage sees key x0: on to the stage of the head's first row that does
            t = max(t + 1, (r0 / s.Lq * s.Lq + min(max(x0 - len + s.Lq, 0), s.Lq - 1)) / kN);
        }
        return min(t, end);
    }
};

// D (128 x 64) = A B^T over 128 d, both K-major in shared memory
__device__ __forceinline__ void product(uint32_t d, uint32_t a, uint32_t a_hi, uint32_t b, uint32_t b_hi, uint32_t idesc)
{
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
        mma_ss_split(d, a + (kk >> 2) * (kABytes >> 5) + (kk & 3) * 2, a_hi, b + (kk >> 2) * (kBBytes >> 5) + (kk & 3) * 2,
                     b_hi, idesc, kk > 0 ? 1u : 0u);
}
// acc (+)= X B: X 128 x 64 bf16 in TMEM, B a tile read MN-major
__device__ __forceinline__ void gradient(uint32_t acc, uint32_t x, uint32_t b, uint32_t b_hi, uint32_t idesc, bool first)
{
    mma_ts_split(acc, x, b, b_hi, idesc, first ? 0u : 1u);
#pragma unroll
    for (int kk = 1; kk < 4; ++kk)          // 16 rows: 8 columns, 2 KB of the tile
        mma_ts_split(acc, x + kk * 8, b + kk * 128, b_hi, idesc, 1u);
}

__global__ void __launch_bounds__(kThreads, 1) attention_dkdv_tc_kernel(const __grid_constant__ CUtensorMap map_k,
                                                                        const __grid_constant__ CUtensorMap map_v,
                                                                        const __grid_constant__ CUtensorMap map_q,
                                                                        const __grid_constant__ CUtensorMap map_o,
                                                                        const Params p)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    if (smem_u32(smem_raw) & 1023u) {     // the 128-byte swizzle atoms need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(&p.status->code, 0, (int)ROLA_ERR_UNSUPPORTED);
        return;
    }
    Ctrl& sm = *reinterpret_cast<Ctrl*>(smem_raw + kSmemTiles);
    const uint32_t sbase = smem_u32(smem_raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto bar = [&](int i) { return smem_u32(&sm.bar[i]); };
    auto timeout = [&](int where) {
        if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 112 + where;
    };
    const AttnShape& s = p.s;
    const uint64_t limit = s.wait_limit_ns;

    if (tid == 0) {
        sm.abort = 0;
        for (int i = 0; i < NUM_BARS; ++i) {
            int count = 1;
            if (i == A_EMPTY || (i >= B_EMPTY && i < B_EMPTY + kSlots)) count = 2;      // two issuing threads
            if ((i >= P_FULL && i < V_DONE) || (i >= COLS && i < DRAIN)) count = 4;     // a group's warps
            if (i == O_EMPTY) count = 8;
            mbar_init(bar(i), count);
        }
        fence_mbar_init();
    }
    if (warp == kSWarp) {
        tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    volatile int* abort = &sm.abort;
    bool ok = true;
    auto wait = [&](int b, int parity) {
        if (ok) ok = mbar_wait(bar(b), parity & 1, abort, limit);
        return ok;
    };

    if (warp == kTmaWarp) {
        // ------------------------------------------------------------ TMA producer
        // d-chunk lane & 1 of a tile, one box a lane (a lane's copies run one after another): K and Q on lanes
        // 0, 1, V and dO on 2, 3
        int na = 0, c = 0;
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it(p, i);
            if (it.begin >= it.end) continue;
            if (na >= 1) wait(A_EMPTY, na - 1);
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(bar(A_FULL), 2 * kABytes);
            __syncwarp();
            if (lane < 4)
                tma_load_3d(sbase + kSmemA + (lane >> 1) * kABytes + (lane & 1) * (kABytes / 2), lane & 2 ? &map_v : &map_k,
                            bar(A_FULL), (lane & 1) * 64, it.x0, it.head);
            ++na;
            for (int t = it.begin; t < it.end && ok; t = it.next(s, t + 1)) {
                for (int o = 0; o < 2; ++o, ++c) {
                    const int slot = c % kSlots;
                    if (c >= kSlots) wait(B_EMPTY + slot, c / kSlots - 1);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (!ok) break;
                    // test hook: the CTA's first tile is never loaded, so the waits on it run out
                    const bool skip = (s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) && c == 0;
                    if (lane == 0 && !skip) mbar_expect_tx(bar(B_FULL + slot), kBBytes);
                    __syncwarp();
                    if ((lane >> 1) == o && !skip)
                        tma_load_3d(sbase + kSmemB + slot * kBBytes + (lane & 1) * (kBBytes / 2), o ? &map_o : &map_q,
                                    bar(B_FULL + slot), (lane & 1) * 64, t * kN, it.head);
                }
            }
        }
        if (lane == 0) {
            if (!ok) timeout(1);
            // every copy this warp issued lands before the CTA exits (bounded by time only)
            int never = 0;
            if (na > 0) mbar_wait(bar(A_FULL), (na - 1) & 1, &never, limit);
            for (int u = c > kSlots ? c - kSlots : 0; u < c; ++u)
                mbar_wait(bar(B_FULL + u % kSlots), (u / kSlots) & 1, &never, limit);
        }
        __syncwarp();
    } else if (warp >= kSWarp) {
        // ------------------------------------------------------------ products
        if (elect_one()) {
            const uint64_t da = smem_desc(sbase + kSmemA, 16, 1024), db = smem_desc(sbase + kSmemB, 16, 1024);
            const uint64_t dg = smem_desc(sbase + kSmemB, kBBytes / 2, 1024);        // the same tiles read MN-major
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            const uint32_t g_lo = (uint32_t)dg, g_hi = (uint32_t)(dg >> 32);
            const uint32_t id_s = idesc_bf16(kM, kN, false, false), id_g = idesc_bf16(kM, kDh, false, true);
            auto tile = [&](int use) { return (uint32_t)(use % kSlots) * (kBBytes >> 4); };
            const int mine = warp - kSWarp;                   // group of an S thread
            int n = 0, items = 0;
            for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
                const Item it(p, i);
                if (it.begin >= it.end) continue;
                if (warp != kGradWarp) wait(A_FULL, items);
                bool used = false;
                for (int t = it.begin; t < it.end && ok; t = it.next(s, t + 1), ++n) {
                    const int u0 = 2 * n, u1 = 2 * n + 1, g = n & 1, k = n >> 1;      // k: the group's stage
                    if (warp != kGradWarp) {
                        if (g != mine) continue;
                        wait(B_FULL + u0 % kSlots, u0 / kSlots);
                        if (k >= 1) wait(V_DONE + g, k - 1);
                        if (!ok) break;
                        fence_after_sync();
                        product(tmem + kTmemS + g * 64, a_lo, a_hi, b_lo + tile(u0), b_hi, id_s);
                        mma_commit(bar(S_FULL + g));
                        mma_commit(bar(B_EMPTY + u0 % kSlots));
                        wait(B_FULL + u1 % kSlots, u1 / kSlots);
                        if (k >= 1) wait(K_DONE + g, k - 1);
                        if (!ok) break;
                        fence_after_sync();
                        product(tmem + kTmemP + g * 64, a_lo + (kABytes >> 4), a_hi, b_lo + tile(u1), b_hi, id_s);
                        mma_commit(bar(DP_FULL + g));
                        mma_commit(bar(B_EMPTY + u1 % kSlots));
                        used = true;
                    } else {
                        const bool first = t == it.begin;
                        wait(P_FULL + g, k);
                        // P says that Q is there, by way of S; dO, of which it knows nothing, may still be on its way
                        wait(B_FULL + u1 % kSlots, u1 / kSlots);
                        if (first && items >= 1) wait(O_EMPTY, items - 1);
                        if (!ok) break;
                        fence_after_sync();
                        gradient(tmem + kTmemV, tmem + kTmemS + g * 64, g_lo + tile(u1), g_hi, id_g, first);
                        mma_commit(bar(V_DONE + g));
                        mma_commit(bar(B_EMPTY + u1 % kSlots));
                        if (!wait(DS_FULL + g, k)) break;
                        fence_after_sync();
                        gradient(tmem + kTmemK, tmem + kTmemP + g * 64, g_lo + tile(u0), g_hi, id_g, first);
                        mma_commit(bar(K_DONE + g));
                        mma_commit(bar(B_EMPTY + u0 % kSlots));
                    }
                }
                if (!ok) break;
                if (warp == kGradWarp) mma_commit(bar(O_FULL));
                else if (used) mma_commit(bar(A_EMPTY));
                else mbar_arrive(bar(A_EMPTY));
                ++items;
            }
            if (!ok) timeout(warp == kGradWarp ? 5 : 2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(DRAIN + mine));
            mbar_wait(bar(DRAIN + mine), 0, &never, limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ element-wise work + epilogue
        const int g = warp >> 2, gt = tid & 127;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + lane_off + kTmemS + g * 64, p_addr = tmem + lane_off + kTmemP + g * 64;
        const float c_log2 = s.scale_log2, log2e = 1.4426950408889634f;
        auto warp_wait = [&](int b, int parity) {
            if (ok) ok = mbar_wait_warp(bar(b), parity & 1, abort, limit);
            return ok;
        };
        auto arrive = [&](int b) {
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(b));
        };
        int n = 0, items = 0;
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it(p, i);
            const int x = it.x0 + gt;                     // this thread's key
            const bool any = it.begin < it.end;
            const size_t rows = (size_t)it.head * s.R;
            // this thread's share of a stage's row values: threads 0-63 lse and the row's limit, 64-127 D
            float val = 0.0f;
            int lim = 0, have = -1;                       // have: the stage they are of
            auto fetch = [&](int t) {
                have = t;
                if (t >= it.end) return;
                const int r = t * kN + (gt & 63);
                const bool in = r < s.R;
                lim = in && gt < 64 ? min(max(attn_seen(s, it.len, r) - it.x0, 0), kM) : 0;
                // a row past the end: p = 2^(-inf) = 0
                val = gt < 64 ? (in ? -p.lse[rows + r] * log2e : -INFINITY) : (in ? -p.D[rows + r] : 0.0f);
            };
            for (int t = it.begin; t < it.end; ++n) {
                const int nt = it.next(s, t + 1), k = n >> 1;
                if ((n & 1) != g) {
                    if (have != nt) fetch(nt);
                    t = nt;
                    continue;
                }
                if (have != t) fetch(t);
                Cols& cols = sm.cols[k & 1][g];
                if (gt < 64) {
                    cols.lse2[gt] = val;
                    cols.seen[gt] = (short)lim;
                } else {
                    cols.neg_D[gt - 64] = val;
                }
                // a buffer is written again two stages on, past the next stage's COLS, for which every warp has read this one
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(COLS + g));
                fetch(it.next(s, nt + 1));                // on their way under this stage's work
                const int r0 = t * kN, r1 = min(r0 + kN, s.R) - 1;
                const bool whole = it.x0 + kM <= attn_seen_least(s, it.len, r0, r1);
                if (!warp_wait(S_FULL + g, k) || !warp_wait(COLS + g, k)) break;
                fence_after_sync();
                float pr[64];
                // p of 32 rows from their scores; `masked`: some row does not see all of the item's keys
                auto scores = [&](int h, auto masked) {
                    float (&q)[32] = *reinterpret_cast<float(*)[32]>(&pr[h * 32]);
                    row_load<32>(s_addr + h * 32, q);
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 l = *reinterpret_cast<const float4*>(&cols.lse2[h * 32 + j]);
                        ffma2(q[j], q[j + 1], c_log2, l.x, l.y);
                        ffma2(q[j + 2], q[j + 3], c_log2, l.z, l.w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[j + e] = fast_exp2(q[j + e]);
                        if constexpr (masked.value) {
                            const short4 m = *reinterpret_cast<const short4*>(&cols.seen[h * 32 + j]);
                            if (gt >= m.x) q[j] = 0.0f;
                            if (gt >= m.y) q[j + 1] = 0.0f;
                            if (gt >= m.z) q[j + 2] = 0.0f;
                            if (gt >= m.w) q[j + 3] = 0.0f;
                        }
                        pk[j >> 1] = pack_bf16(q[j], q[j + 1]);
                        pk[(j >> 1) + 1] = pack_bf16(q[j + 2], q[j + 3]);
                    }
                    // over the scores of the first half, which are in registers
                    tmem_st16(s_addr + h * 16, *reinterpret_cast<const float(*)[16]>(pk));
                };
                auto grads = [&](int h, auto masked) {
                    float dp[32];
                    row_load<32>(p_addr + h * 32, dp);
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 D = *reinterpret_cast<const float4*>(&cols.neg_D[h * 32 + j]);
                        const float* q = &pr[h * 32 + j];
                        fadd_mul2(dp[j], dp[j + 1], D.x, D.y, q[0], q[1]);
                        fadd_mul2(dp[j + 2], dp[j + 3], D.z, D.w, q[2], q[3]);
                        if constexpr (masked.value) {     // where p is 0 by selection dp may be anything
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (q[e] == 0.0f) dp[j + e] = 0.0f;
                        }
                        pk[j >> 1] = pack_bf16(dp[j], dp[j + 1]);
                        pk[(j >> 1) + 1] = pack_bf16(dp[j + 2], dp[j + 3]);
                    }
                    tmem_st16(p_addr + h * 16, *reinterpret_cast<const float(*)[16]>(pk));
                };
                if (whole) {
                    scores(0, Flag<false>());
                    scores(1, Flag<false>());
                } else {
                    scores(0, Flag<true>());
                    scores(1, Flag<true>());
                }
                tmem_st_wait();
                arrive(P_FULL + g);
                if (!warp_wait(DP_FULL + g, k)) break;
                fence_after_sync();
                if (whole) {
                    grads(0, Flag<false>());
                    grads(1, Flag<false>());
                } else {
                    grads(0, Flag<true>());
                    grads(1, Flag<true>());
                }
                tmem_st_wait();
                arrive(DS_FULL + g);
                t = nt;
            }
            if (!ok) break;
            // ---- epilogue: group 0 writes dv, group 1 dk
            if (any) {
                if (!warp_wait(O_FULL, items)) break;
                fence_after_sync();
                ++items;
            }
            const uint32_t acc = tmem + lane_off + (g ? kTmemK : kTmemV);
            const float mul = g ? s.scale : 1.0f;
            const size_t row = ((size_t)it.head * s.Lk + x) * kDh;
            __nv_bfloat16* out = (g ? p.dk : p.dv) + row;
            float* part = (g ? p.part_dk : p.part_dv) + (size_t)it.part * s.heads * s.Lk * kDh + row;
            // a key past the length holds zeros or its own garbage: its gradient is 0
            const bool live = any && x < it.len;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float v[32];
                if (any) row_load<32>(acc + c * 32, v);
                if (any && c == 3) arrive(O_EMPTY);
                if (x >= s.Lk) continue;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = live ? v[j] * mul : 0.0f;
                if (p.splits > 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = __float_as_uint(v[e + j]);
                        st_global32(part + c * 32 + e, y);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 16) {
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(v[e + 2 * j], v[e + 2 * j + 1]);
                        store_row32(out + c * 32 + e, y, p.wide);
                    }
                }
            }
        }
        if (!ok) timeout(3);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kSWarp) tmem_dealloc(tmem, kTmemCols);
}

}  // namespace

cudaError_t launch_attention_dkdv_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    CUtensorMap mk, mv, mq, mo;
    if (!encode_rows(&mk, a.k, s.Lk, s.heads, kM) || !encode_rows(&mv, a.v, s.Lk, s.heads, kM) ||
        !encode_rows(&mq, a.q, s.R, s.heads, kN) || !encode_rows(&mo, a.dO, s.R, s.heads, kN))
        return cudaErrorInvalidValue;
    Params p{};
    p.s = s;
    p.kv_len = a.kv_len;
    p.lse = a.lse_in;
    p.D = a.D;
    p.dv = static_cast<__nv_bfloat16*>(a.dv);
    p.dk = static_cast<__nv_bfloat16*>(a.dk);
    p.part_dv = a.part_dv;
    p.part_dk = a.part_dk;
    p.status = a.status;
    p.splits = s.splits_dkv;
    p.tiles = (s.Lk + kM - 1) / kM;
    p.items = p.tiles * s.heads * p.splits;
    p.wide = ((reinterpret_cast<uintptr_t>(p.dv) | reinterpret_cast<uintptr_t>(p.dk)) & 31u) == 0;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = kSmemTiles + sizeof(Ctrl);
    e = cudaFuncSetAttribute(attention_dkdv_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attention_dkdv_tc_kernel<<<p.items < nsm ? p.items : nsm, kThreads, smem, st>>>(mk, mv, mq, mo, p);
    return cudaGetLastError();
}

}  // namespace rola
