// Gradients of the dense softmax attention's queries on the 5th-generation
// tensor cores (bf16 operands, fp32 accumulation in TMEM), recomputing the
// probabilities; and the backward pass's launches.
//
//   P = 2^(scale log2(e) q k^T - lse log2(e)),  dP = dO v^T,  dS = P (dP - D),  D = dO . o,  dq = scale dS k
//
// dq and dk / dv (attention_dkdv_tc.cu) are two kernels: each accumulator then
// stays in TMEM over its whole sum, so nothing is added in memory and the order of
// every sum is fixed; the price is S and dP computed twice (7 products instead of 5).
//
// An item is 128 rows of a head, the TMEM lanes; their keys come in stages of 128.  Stage n:
//   S_b = Q K^T,  dP = dO V^T      128 x 128, K-major operands in shared memory, b = n & 1
//   dQ += dS K                     dS over half of S_b as bf16, K read MN-major from the same tile
// TMEM (512 columns): S_0, S_1, dP, dQ.  One thread issues S and dP: S(n) once
// dQ(n - 2) has read its buffer, dP(n) as soon as dP(n - 1) is in registers;
// another issues dQ.  Two groups of four warps work on a stage, 64 of its columns
// each, under the products of the stages beside it.  (One issuing thread and stages
// of 64 took 1.7 times as long: a 128 x 64 product takes 48 cycles instead of 32, and
// one thread's waits, products and commits, 150, 17 and 50 to 150 cycles each, were the bound.
// 430 us at 12 heads x 8190 x 8190, 1440 TFLOP/s.)
//
// A key past the sequence's length has P = dS = 0 by selection whatever it
// holds, and since K is also the other operand of a sum over keys, its rows of K
// are zeroed in shared memory (0 x NaN would be NaN).
// If a row tile's keys fit one stage, D = sum_j P dP is taken from the stage
// itself instead of dO . o, whose o carries the output's bf16 rounding: over few
// keys that error is not small beside dP - D.
//
// Few items: their stages are split over several (AttnShape::splits_dq); the parts
// are written in fp32 and added in order by a second kernel.
//
// Warps (384 threads, one persistent CTA per SM): 0-3 and 4-7 the two groups, 8
// TMA, 9 S and dP, 10 dQ, 11 the zeroing of K's rows.  Every mbarrier wait is bounded.
#include "attention_tc.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kM = 128;                                   // lanes of an item, columns of a stage
constexpr int kTmaWarp = 8, kSWarp = 9, kGradWarp = 10, kCutWarp = 11, kThreads = 384, kSlots = 5;
constexpr uint32_t kTileBytes = kM * kDh * 2;             // [d-chunk][128 rows][64]
constexpr uint32_t kSmemA = 0, kSmemB = 2 * kTileBytes, kSmemTiles = kSmemB + kSlots * kTileBytes;
constexpr uint32_t kTmemCols = 512;

constexpr uint32_t kTmemS = 0, kTmemP = 256, kTmemAcc = 384;      // S_b at 128 b

// B: a ring of tiles, K of stage n in use 2n, V in 2n + 1.  READ: dP is in registers; S_FULL, DS_FULL, DONE: + b, since dS of
// stage n + 1 may be there before the dQ thread has looked for that of stage n; D_FULL: the
// groups' parts of D are in shared memory (the warps meet at no barrier of the CTA, whose wait would have no limit).
enum Bar { A_FULL = 0, A_EMPTY, B_FULL, B_EMPTY = B_FULL + kSlots, S_FULL = B_EMPTY + kSlots, DP_FULL = S_FULL + 2, READ,
           DS_FULL, DONE = DS_FULL + 2, O_FULL = DONE + 2, O_EMPTY, D_FULL, CUT, DRAIN = CUT + 4, NUM_BARS = DRAIN + 2 };

struct Ctrl {
    float D[2][2][kM];                                    // the groups' parts of D, [single-stage item & 1][group]
    uint64_t bar[NUM_BARS];
    uint32_t tmem_base;
    int abort;
};
static_assert(kSmemTiles + sizeof(Ctrl) <= 232448, "tiles and control block fit the 227 KB a CTA may have");

struct Params {
    AttnShape s;
    const int32_t* kv_len;
    const float* lse;
    float* D;
    __nv_bfloat16* dq;
    float* part;                      // with splits: its parts, [splits][heads][rows][128]
    DeviceStatus* status;
    int splits, tiles, items;         // 128-row tiles of a head; tiles heads splits
    bool wide;                        // dq is 32-byte aligned
};

// One item: its stages from begin to end.
struct Item {
    int head, x0, len, part;          // x0: first row
    int begin, end, all;              // stages of this part; of the whole axis
    __device__ __forceinline__ Item(const Params& p, int i)
    {
        const AttnShape& s = p.s;
        part = 0;
        if (p.splits > 1) {
            part = i % p.splits;
            i /= p.splits;
        }
        int tile;
        if (s.causal) {               // the longest items of every head first: the last rows
            tile = falling_tile(i / s.heads, p.tiles, s.H / s.Hk);
            head = i % s.heads;
        } else {
            head = i / p.tiles;
            tile = i - head * p.tiles;
        }
        x0 = tile * kM;
        len = attn_len(s, p.kv_len, head / s.Hk);
        all = (attn_seen_most(s, len, x0, min(x0 + kM, s.R) - 1) + kM - 1) / kM;
        begin = 0;
        end = all;
        if (p.splits > 1) {           // stages x parts stays below 2^31: at most 2^23 stages and 152 parts
            begin = all * part / p.splits;
            end = all * (part + 1) / p.splits;
        }
    }
    // stage t's keys end past the sequence's length, where the memory holds other keys (past Lk the copy writes zeros)
    __device__ __forceinline__ bool cut(const AttnShape& s, int t) const
    {
        return (t + 1) * kM > len && len < s.Lk;
    }
};

// D = A B^T over 128 d of two tiles in shared memory, K-major
__device__ __forceinline__ void product(uint32_t d, uint32_t a, uint32_t a_hi, uint32_t b, uint32_t b_hi, uint32_t idesc)
{
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
        const uint32_t o = (kk >> 2) * (kTileBytes >> 5) + (kk & 3) * 2;
        mma_ss_split(d, a + o, a_hi, b + o, b_hi, idesc, kk > 0 ? 1u : 0u);
    }
}
// acc (+)= X B: X 128 x 128 bf16 in TMEM, columns 0-31 (the first 64 values) and 64-95; B a tile read MN-major
__device__ __forceinline__ void gradient(uint32_t acc, uint32_t x, uint32_t b, uint32_t b_hi, uint32_t idesc, bool first)
{
    mma_ts_split(acc, x, b, b_hi, idesc, first ? 0u : 1u);
#pragma unroll
    for (int kk = 1; kk < 8; ++kk)          // 16 values: 8 columns, 2 KB of the tile
        mma_ts_split(acc, x + (kk >> 2) * 64 + (kk & 3) * 8, b + kk * 128, b_hi, idesc, 1u);
}

__global__ void __launch_bounds__(kThreads, 1) attention_dq_tc_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                      const __grid_constant__ CUtensorMap map_o,
                                                                      const __grid_constant__ CUtensorMap map_k,
                                                                      const __grid_constant__ CUtensorMap map_v,
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
        if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 96 + where;
    };
    const AttnShape& s = p.s;
    const uint64_t limit = s.wait_limit_ns;

    if (tid == 0) {
        sm.abort = 0;
        for (int i = 0; i < NUM_BARS; ++i) {
            const bool groups = i == READ || (i >= DS_FULL && i < DONE) || i == O_EMPTY || i == D_FULL;
            // a tile is followed by the zeroing warp too where there is work for it
            const bool two = i >= B_EMPTY && i < B_EMPTY + kSlots && p.kv_len;
            mbar_init(bar(i), groups ? 8 : (two ? 2 : 1));
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
        // d-chunk lane & 1 of a tile, one box a lane (a lane's copies run one after another): A_0 on lanes 0, 1
        // and A_1 on 2, 3; the tiles of the ring on 0, 1 and 2, 3 in turn
        int na = 0, c = 0;
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it(p, i);
            if (it.begin >= it.end) continue;
            if (na >= 1) wait(A_EMPTY, na - 1);
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(bar(A_FULL), 2 * kTileBytes);
            __syncwarp();
            if (lane < 4)
                tma_load_3d(sbase + kSmemA + (lane >> 1) * kTileBytes + (lane & 1) * (kTileBytes / 2),
                            lane & 2 ? &map_o : &map_q, bar(A_FULL), (lane & 1) * 64, it.x0, it.head);
            ++na;
            for (int t = it.begin; t < it.end && ok; ++t) {
                for (int o = 0; o < 2; ++o, ++c) {
                    const int slot = c % kSlots;
                    if (c >= kSlots) wait(B_EMPTY + slot, c / kSlots - 1);
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    if (!ok) break;
                    // test hook: the CTA's first tile is never loaded, so the waits on it run out
                    const bool skip = (s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) && c == 0;
                    if (lane == 0 && !skip) mbar_expect_tx(bar(B_FULL + slot), kTileBytes);
                    __syncwarp();
                    if ((lane >> 1) == o && !skip)
                        tma_load_3d(sbase + kSmemB + slot * kTileBytes + (lane & 1) * (kTileBytes / 2), o ? &map_v : &map_k,
                                    bar(B_FULL + slot), (lane & 1) * 64, t * kM, it.head);
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
    } else if (warp == kSWarp || warp == kGradWarp) {
        // ------------------------------------------------------------ products
        if (elect_one()) {
            const uint64_t da = smem_desc(sbase + kSmemA, 16, 1024), db = smem_desc(sbase + kSmemB, 16, 1024);
            const uint64_t dg = smem_desc(sbase + kSmemB, kTileBytes / 2, 1024);     // the same tiles read MN-major
            const uint32_t a_lo = (uint32_t)da, a_hi = (uint32_t)(da >> 32), b_lo = (uint32_t)db, b_hi = (uint32_t)(db >> 32);
            const uint32_t g_lo = (uint32_t)dg, g_hi = (uint32_t)(dg >> 32);
            int n = 0, items = 0, ncut = 0;
            auto tile = [&](int use) { return (uint32_t)(use % kSlots) * (kTileBytes >> 4); };
            for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
                const Item it(p, i);
                for (int t = it.begin; t < it.end && ok; ++t, ++n) {
                    const bool last = t + 1 == it.end;
                    const int u0 = 2 * n, u1 = 2 * n + 1;
                    if (warp == kSWarp) {
                        const uint32_t id = idesc_bf16(kM, kM, false, false);
                        if (t == it.begin) wait(A_FULL, items);
                        wait(B_FULL + u0 % kSlots, u0 / kSlots);
                        if (n >= 2) wait(DONE + (n & 1), (n >> 1) - 1);
                        if (!ok) break;
                        fence_after_sync();
                        product(tmem + kTmemS + (n & 1) * 128, a_lo, a_hi, b_lo + tile(u0), b_hi, id);
                        mma_commit(bar(S_FULL + (n & 1)));
                        wait(B_FULL + u1 % kSlots, u1 / kSlots);
                        if (n >= 1) wait(READ, n - 1);
                        if (!ok) break;
                        fence_after_sync();
                        product(tmem + kTmemP, a_lo + (kTileBytes >> 4), a_hi, b_lo + tile(u1), b_hi, id);
                        mma_commit(bar(DP_FULL));
                        mma_commit(bar(B_EMPTY + u1 % kSlots));
                        if (last) mma_commit(bar(A_EMPTY));
                    } else {
                        const uint32_t id = idesc_bf16(kM, kDh, false, true);
                        const bool first = t == it.begin;
                        if (it.cut(s, t)) {
                            wait(CUT + (ncut & 3), ncut >> 2);
                            ++ncut;
                        }
                        wait(DS_FULL + (n & 1), n >> 1);
                        if (first && items >= 1) wait(O_EMPTY, items - 1);
                        if (!ok) break;
                        fence_after_sync();
                        gradient(tmem + kTmemAcc, tmem + kTmemS + (n & 1) * 128, g_lo + tile(u0), g_hi, id, first);
                        mma_commit(bar(DONE + (n & 1)));
                        mma_commit(bar(B_EMPTY + u0 % kSlots));
                        if (last) mma_commit(bar(O_FULL));
                    }
                }
                if (it.begin < it.end) ++items;
            }
            if (!ok) timeout(warp == kSWarp ? 2 : 5);
            // every product issued completes before TMEM is released
            int never = 0;
            const uint32_t drain = bar(DRAIN + (warp == kSWarp ? 0 : 1));
            mma_commit(drain);
            mbar_wait(drain, 0, &never, limit);
        }
        __syncwarp();
    } else if (warp == kCutWarp) {
        // ------------------------------------------------------------ K past a sequence's length
        // The warp follows every tile, so that it knows each slot's turn; CUT has four barriers because the
        // gradients' thread may be up to two K tiles of the ring behind it.
        int c = 0, ncut = 0;
        auto next = [&]() {
            wait(B_FULL + c % kSlots, c / kSlots);
            ok = __all_sync(0xffffffffu, ok);
            return ok;
        };
        auto done = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_EMPTY + c % kSlots));
            ++c;
        };
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok && p.kv_len; ++turn) {
            const Item it(p, i);
            for (int t = it.begin; t < it.end; ++t) {
                if (!next()) break;                   // K
                if (it.cut(s, t)) {
                    const int slot = c % kSlots, valid = it.len - t * kM;
                    // row r of d-chunk h: 128 bytes at h 16 KB + r 128; the swizzle stays within a row
                    for (int e = lane; e < (kM - valid) * 16; e += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};\n" ::"r"(
                                         sbase + kSmemB + slot * kTileBytes + ((e & 8) ? kTileBytes / 2 : 0) +
                                         (valid + (e >> 4)) * 128 + (e & 7) * 16),
                                     "r"(0)
                                     : "memory");
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(CUT + (ncut & 3)));
                    ++ncut;
                }
                done();
                if (!next()) break;                   // V
                done();
            }
        }
        if (!ok && lane == 0) timeout(4);
    } else {
        // ------------------------------------------------------------ element-wise work + epilogue
        const int g = warp >> 2, gt = tid & 127;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + lane_off + g * 64, p_addr = tmem + lane_off + kTmemP + g * 64;   // this group's columns
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
        int n = 0, items = 0, singles = 0;                // singles: items of one stage
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it(p, i);
            const int x = it.x0 + gt;                     // this thread's row
            const bool any = it.begin < it.end;
            const size_t rows = (size_t)it.head * s.R;
            const bool in = x < s.R;
            const int seen = in ? attn_seen(s, it.len, x) : 0;
            const int least = any && it.x0 + kM <= s.R ? attn_seen_least(s, it.len, it.x0, it.x0 + kM - 1) : 0;
            const float neg_lse = in ? -p.lse[rows + x] * log2e : 0.0f;
            // (a row that sees nothing: its dO may be anything, and 0 x infinity in D would show in dq)
            float D = seen > 0 && any && it.all > 1 ? p.D[rows + x] : 0.0f;
            for (int t = it.begin; t < it.end; ++t, ++n) {
                const int b = n & 1;
                if (!warp_wait(S_FULL + b, n >> 1)) break;
                fence_after_sync();
                float pr[64];
                row_load<64>(s_addr + b * 128, pr);
#pragma unroll
                for (int j = 0; j < 64; j += 2) {
                    ffma2(pr[j], pr[j + 1], c_log2, neg_lse);
                    pr[j] = fast_exp2(pr[j]);
                    pr[j + 1] = fast_exp2(pr[j + 1]);
                }
                const bool whole = t * kM + kM <= least;
                if (!whole) {                         // some row does not see all of the stage's keys
                    const int m = seen - t * kM - g * 64;
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if (j >= m) pr[j] = 0.0f;
                }
                if (!warp_wait(DP_FULL, n)) break;
                fence_after_sync();
                if (it.all == 1) {                    // D from this stage, the only one
                    float d0 = 0.0f, d1 = 0.0f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float dp[32];
                        row_load<32>(p_addr + h * 32, dp);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float q0 = pr[h * 32 + j], q1 = pr[h * 32 + j + 1];
                            if (q0 != 0.0f) d0 = fmaf(q0, dp[j], d0);
                            if (q1 != 0.0f) d1 = fmaf(q1, dp[j + 1], d1);
                        }
                    }
                    // a buffer is written again two such items on, past the next one's D_FULL, for which every
                    // warp has read this one
                    float (&part)[2][kM] = sm.D[singles & 1];
                    part[g][gt] = d0 + d1;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(D_FULL));
                    if (!warp_wait(D_FULL, singles)) break;
                    ++singles;
                    D = part[0][gt] + part[1][gt];
                    if (in && g == 0) p.D[rows + x] = D;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float dp[32];
                    row_load<32>(p_addr + h * 32, dp);
                    if (h == 1) arrive(READ);
                    if (!whole) {                     // where p is 0 by selection dp may be anything
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (pr[h * 32 + j] == 0.0f) dp[j] = D;
                    }
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        fadd_mul2(dp[j], dp[j + 1], -D, -D, pr[h * 32 + j], pr[h * 32 + j + 1]);
                        pk[j >> 1] = pack_bf16(dp[j], dp[j + 1]);
                    }
                    tmem_st16(s_addr + b * 128 + h * 16, *reinterpret_cast<const float(*)[16]>(pk));
                }
                tmem_st_wait();
                arrive(DS_FULL + b);
            }
            if (!ok) break;
            // ---- epilogue: group g writes d 64 g .. +63
            if (any) {
                if (!warp_wait(O_FULL, items)) break;
                fence_after_sync();
                ++items;
            }
            const uint32_t acc = tmem + lane_off + kTmemAcc + g * 64;
            const size_t row = (rows + x) * kDh + g * 64;
            float* part = p.part + (size_t)it.part * s.heads * s.R * kDh + row;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float v[32];
                if (any) row_load<32>(acc + c * 32, v);
                if (any && c == 1) arrive(O_EMPTY);
                if (!in) continue;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = any ? v[j] * s.scale : 0.0f;
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
                        store_row32(p.dq + row + c * 32 + e, y, p.wide);
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

cudaError_t launch_dq(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mo, mk, mv;
    if (!encode_rows(&mq, a.q, s.R, s.heads, kM) || !encode_rows(&mo, a.dO, s.R, s.heads, kM) ||
        !encode_rows(&mk, a.k, s.Lk, s.heads, kM) || !encode_rows(&mv, a.v, s.Lk, s.heads, kM))
        return cudaErrorInvalidValue;
    Params p{};
    p.s = s;
    p.kv_len = a.kv_len;
    p.lse = a.lse_in;
    p.D = a.D;
    p.dq = static_cast<__nv_bfloat16*>(a.dq);
    p.part = a.part_dq;
    p.status = a.status;
    p.splits = s.splits_dq;
    p.tiles = (s.R + kM - 1) / kM;
    p.items = p.tiles * s.heads * p.splits;
    p.wide = (reinterpret_cast<uintptr_t>(p.dq) & 31u) == 0;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = kSmemTiles + sizeof(Ctrl);
    e = cudaFuncSetAttribute(attention_dq_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attention_dq_tc_kernel<<<p.items < nsm ? p.items : nsm, kThreads, smem, st>>>(mq, mo, mk, mv, p);
    return cudaGetLastError();
}

// out = the sum of n parts, in order; eight values a thread
__global__ void __launch_bounds__(256) add_parts_kernel(long long count, int n, const float* __restrict__ part,
                                                        __nv_bfloat16* __restrict__ out)
{
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= count) return;
    float v[8] = {};
    for (int z = 0; z < n; ++z) {
        const float4 a = load4(part + z * count + i), b = load4(part + z * count + i + 4);
        v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
        v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
    }
    store16(out + i, v);
}
cudaError_t add_parts(long long rows, int n, const float* part, void* out, cudaStream_t st)
{
    const long long count = rows * kDh;
    add_parts_kernel<<<(unsigned)((count + 2047) / 2048), 256, 0, st>>>(count, n, part, static_cast<__nv_bfloat16*>(out));
    return cudaGetLastError();
}

}  // namespace

// dq first: it leaves in D the row values that the dk / dv kernel reads.
cudaError_t launch_attention_backward_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    cudaError_t e = launch_dq(s, a, st);
    if (e == cudaSuccess) e = launch_attention_dkdv_tc(s, a, st);
    const long long rows = (long long)s.heads * s.R, keys = (long long)s.heads * s.Lk;
    if (e == cudaSuccess && s.splits_dq > 1) e = add_parts(rows, s.splits_dq, a.part_dq, a.dq, st);
    if (e == cudaSuccess && s.splits_dkv > 1) e = add_parts(keys, s.splits_dkv, a.part_dv, a.dv, st);
    if (e == cudaSuccess && s.splits_dkv > 1) e = add_parts(keys, s.splits_dkv, a.part_dk, a.dk, st);
    return e;
}

}  // namespace rola
