// Softmax attention over a dense key set on the 5th-generation tensor cores
// (bf16 operands, fp32 accumulation in TMEM).
//
//   o_r = sum_j softmax_j(scale q_r . k_j) v_j   over the keys row r sees
//
// Rows are the G Lq queries of the heads that share a key head (contiguous in
// q), so a shared key head is read once for all of them.  An item is 256 rows of
// a head (two groups of 128) over a range of its key tiles of 128 keys:
//   S_g  = Q_g (128 rows x 128 d, smem, K-major)  x  K^T (128 keys, smem, K-major)
//   O_g += P_g (128 rows x 128 keys, TMEM, bf16)  x  V   (128 keys x 128 d, smem, MN-major)
// TMEM (512 columns): S_0, S_1, O_0, O_1, 128 columns each; P_g overwrites the
// first 64 columns of S_g.  One thread issues all products in the order
// PV_0(t) QK_0(t+1) PV_1(t) QK_1(t+1): products of one thread execute in order,
// so QK_g(t+1) may overwrite S_g / P_g, and S_g(t+1) being complete implies
// that O_g holds PV_g(t).  While a group's softmax runs, the tensor core does
// the other group's products; at an item's end the next item's first QK is
// issued the same way, so items follow one another without a gap.
//
// Softmax (base 2, one thread per row, the whole row of S in registers): each
// row keeps -m and its sum l in fp32.  With t = s scale log2(e) - m, m is raised
// only when the tile's largest t exceeds 2^3 (or on the item's first tile); O
// and l are then scaled by 2^(m_old - m_new).  p = 2^t enters l in fp32 and the
// product rounded to bf16 (the operand type of the tensor core).  A row sees a
// prefix of the keys (its length, or its causal limit), so a row that sees
// nothing in the item's first tile sees nothing in the item: its p stay 0, l = 0.
// Keys past the length: their scores are replaced by -inf whatever they are, and
// their rows of V are zeroed in shared memory (0 x NaN would be NaN).
//
// Warps (320 threads, one persistent CTA per SM): 0-3 softmax and epilogue of
// group 0, 4-7 of group 1, 8 TMA (Q of both groups, and K, V tiles in one ring of
// five 32 KB slots), 9 products.  Shared memory 64 + 160 KB.  Every mbarrier wait
// is bounded; a wait that gives up records ROLA_ERR_TIMEOUT and the CTA drains
// what it issued and frees its TMEM.
#include "attention_tc.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kRows = 128, kKeys = 128, kSlots = 5;
constexpr int kTmaWarp = 8, kMmaWarp = 9, kThreads = 320;
constexpr uint32_t kTileBytes = 128 * 128 * 2;               // [d-chunk][128 rows][64]
constexpr uint32_t kSmemQ = 0, kSmemKV = 2 * kTileBytes, kSmemTiles = kSmemKV + kSlots * kTileBytes;
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemO = 256;   // S_g at 128 g, O_g at 256 + 128 g
constexpr float kRescaleThreshold = 8.0f;                    // log2 units

enum Bar { Q_FULL = 0, Q_EMPTY = 2, S_FULL = 4, P_FULL = 6, O_FULL = 8, O_EMPTY = 10, KV_FULL = 12,
           KV_EMPTY = KV_FULL + kSlots, DRAIN = KV_EMPTY + kSlots, NUM_BARS = DRAIN + 1 };

struct Ctrl {
    uint64_t bar[NUM_BARS];
    uint32_t tmem_base;
    int abort;
};
static_assert(kSmemTiles + sizeof(Ctrl) <= 232448, "tiles and control block fit the 227 KB a CTA may have");

struct Params {
    AttnShape s;
    const int32_t* kv_len;
    __nv_bfloat16* o;
    float *lse, *part_o, *part_lse;
    DeviceStatus* status;
    int q_tiles;                 // 256-row tiles of a head
    int items;                   // q_tiles heads splits
};

__device__ __forceinline__ void record_timeout(const Params& p, int where)
{
    if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 80 + where;
}

// One item: rows r0 .. of `head`, key tiles first .. first + T[g] of group g (T[g] 0: the group has no
// rows, or its rows see nothing there).
struct Item {
    int head, r0, len, part, first;
    int T0, T1, T;               // per group, and the larger
    bool has1;
};
__device__ __forceinline__ Item item_of(const Params& p, int i)
{
    const AttnShape& s = p.s;
    Item it;
    it.part = i % s.splits;
    i /= s.splits;
    int qt;
    if (s.causal) {              // the longest rows of every head first
        qt = p.q_tiles - 1 - i / s.heads;
        it.head = i % s.heads;
    } else {                     // head by head: the CTAs in flight share few heads' keys
        it.head = i / p.q_tiles;
        qt = i - it.head * p.q_tiles;
    }
    it.r0 = qt * 2 * kRows;
    it.len = attn_len(s, p.kv_len, it.head / s.Hk);
    it.has1 = it.r0 + kRows < s.R;
    const int last0 = min(it.r0 + kRows, s.R) - 1, last1 = min(it.r0 + 2 * kRows, s.R) - 1;
    const int n0 = attn_seen_most(s, it.len, it.r0, last0);
    const int n1 = it.has1 ? attn_seen_most(s, it.len, it.r0 + kRows, last1) : 0;
    const int t0 = (n0 + kKeys - 1) / kKeys, t1 = (n1 + kKeys - 1) / kKeys, t = max(t0, t1);
    it.first = (int)((long long)t * it.part / s.splits);
    const int end = (int)((long long)t * (it.part + 1) / s.splits);
    it.T0 = max(min(t0, end) - it.first, 0);
    it.T1 = max(min(t1, end) - it.first, 0);
    it.T = max(it.T0, it.T1);
    return it;
}

__global__ void __launch_bounds__(kThreads, 1) attention_tc_kernel(const __grid_constant__ CUtensorMap map_q,
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
    const AttnShape& s = p.s;
    const uint64_t limit = s.wait_limit_ns;

    if (tid == 0) {
        sm.abort = 0;
        for (int g = 0; g < 2; ++g) {
            mbar_init(bar(Q_FULL + g), 1);
            mbar_init(bar(Q_EMPTY + g), 1);
            mbar_init(bar(S_FULL + g), 1);
            mbar_init(bar(P_FULL + g), 4);
            mbar_init(bar(O_FULL + g), 1);
            mbar_init(bar(O_EMPTY + g), 4);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(bar(KV_FULL + i), 1);
            mbar_init(bar(KV_EMPTY + i), 1);
        }
        mbar_init(bar(DRAIN), 1);
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
        tmem_relinquish();
    }
    if (warp == kTmaWarp && lane == 0) {
        tma_prefetch_desc(&map_q);
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = sm.tmem_base;
    volatile int* abort = &sm.abort;

    if (warp == kTmaWarp) {
        // ------------------------------------------------------------ TMA producer
        // A d-chunk (64 columns) of a tile is one box of 128 rows; lanes 0 and 1 load one each (a
        // lane's copies run one after another).
        bool ok = true;
        int nq[2] = {0, 0}, c = 0;                       // Q tiles per group, ring slots used
        auto ring = [&](const CUtensorMap* map, int key0, int head, bool skip) {
            const int slot = c % kSlots;
            if (c >= kSlots) ok = mbar_wait(bar(KV_EMPTY + slot), ((c / kSlots) - 1) & 1, abort, limit);
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) return;
            if (lane == 0 && !skip) mbar_expect_tx(bar(KV_FULL + slot), kTileBytes);
            __syncwarp();
            if (lane < 2 && !skip)
                tma_load_3d(sbase + kSmemKV + slot * kTileBytes + lane * (kTileBytes / 2), map, bar(KV_FULL + slot),
                            lane * 64, key0, head);
            ++c;
        };
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
            const Item it = item_of(p, i);
            if (it.T == 0) continue;
            for (int g = 0; g < 2 && ok; ++g) {
                if ((g ? it.T1 : it.T0) == 0) continue;
                if (nq[g] >= 1) ok = mbar_wait(bar(Q_EMPTY + g), (nq[g] - 1) & 1, abort, limit);
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(bar(Q_FULL + g), kTileBytes);
                __syncwarp();
                if (lane < 2)
                    tma_load_3d(sbase + kSmemQ + g * kTileBytes + lane * (kTileBytes / 2), &map_q, bar(Q_FULL + g),
                                lane * 64, it.r0 + g * kRows, it.head);
                ++nq[g];
            }
            for (int t = 0; t < it.T && ok; ++t) {
                const int key0 = (it.first + t) * kKeys;
                // test hook: the CTA's first K tile is never loaded, so the waits on it run out
                ring(&map_k, key0, it.head, (s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) && c == 0);
                if (ok) ring(&map_v, key0, it.head, false);
            }
        }
        if (!ok && lane == 0) record_timeout(p, 1);
        // every copy this warp issued lands before the CTA exits (bounded by time only)
        if (lane == 0) {
            int never = 0;
            for (int g = 0; g < 2; ++g)
                if (nq[g]) mbar_wait(bar(Q_FULL + g), (nq[g] - 1) & 1, &never, limit);
            for (int u = c > kSlots ? c - kSlots : 0; u < c; ++u)
                mbar_wait(bar(KV_FULL + u % kSlots), (u / kSlots) & 1, &never, limit);
        }
    } else if (warp == kMmaWarp) {
        // ------------------------------------------------------------ products
        // The whole warp runs the loop (it zeroes rows of V together); lane 0 issues.
        const uint32_t id_qk = idesc_bf16(kRows, kKeys, false, false), id_pv = idesc_bf16(kRows, kDh, false, true);
        const uint64_t dq = smem_desc(sbase + kSmemQ, 16, 1024);                      // A of QK (K-major)
        const uint64_t dk = smem_desc(sbase + kSmemKV, 16, 1024);                     // B of QK (K-major)
        const uint64_t dv = smem_desc(sbase + kSmemKV, kTileBytes / 2, 1024);         // B of PV (MN-major)
        const uint32_t q_lo = (uint32_t)dq, q_hi = (uint32_t)(dq >> 32), k_lo = (uint32_t)dk, k_hi = (uint32_t)(dk >> 32);
        const uint32_t v_lo = (uint32_t)dv, v_hi = (uint32_t)(dv >> 32);
        bool ok = true;
        int u = 0;                                       // tiles whose V was used; K of tile u in slot 2u, V in 2u + 1
        int np[2] = {0, 0}, nq[2] = {0, 0}, no[2] = {0, 0};   // per group: P tiles, Q tiles, items with O
        auto wait = [&](int b, int parity) {
            if (ok) ok = __shfl_sync(0xffffffffu, mbar_wait(bar(b), parity, abort, limit), 0);
            return ok;
        };
        // S_g = Q_g K^T of ring slot ck; `first`: of an item (its Q has to have arrived), `last`: Q is free after it
        auto qk = [&](int g, int ck, bool first, bool last) {
            if (first && !wait(Q_FULL + g, nq[g]++ & 1)) return;
            if (!wait(KV_FULL + ck % kSlots, (ck / kSlots) & 1)) return;
            fence_after_sync();
            if (lane == 0) {
                const uint32_t a = q_lo + g * (kTileBytes >> 4), b = k_lo + (ck % kSlots) * (kTileBytes >> 4);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t o = (kk >> 2) * (kTileBytes >> 5) + (kk & 3) * 2;
                    mma_ss_split(tmem + kTmemS + g * 128, a + o, q_hi, b + o, k_hi, id_qk, kk > 0 ? 1u : 0u);
                }
                mma_commit(bar(S_FULL + g));
                if (last) mma_commit(bar(Q_EMPTY + g));
            }
            __syncwarp();
        };
        auto free_slot = [&](int c) {
            if (lane == 0) mma_commit(bar(KV_EMPTY + c % kSlots));
            __syncwarp();
        };
        // the next item that has tiles
        auto next_item = [&](int i, Item& it) {
            for (; i < p.items; i += gridDim.x) {
                it = item_of(p, i);
                if (it.T) return i;
            }
            return i;
        };
        Item it{}, nx{};
        int i = next_item(blockIdx.x, it);
        if (i < p.items) {
            if (it.T0) qk(0, 0, true, it.T0 == 1);
            if (ok && it.T1) qk(1, 0, true, it.T1 == 1);
            if (ok) free_slot(0);
        }
        while (i < p.items && ok) {
            const int ni = next_item(i + gridDim.x, nx);
            for (int t = 0; t < it.T && ok; ++t, ++u) {
                const bool end = t == it.T - 1, more = !end || ni < p.items;
                const int cv = 2 * u + 1, ck = 2 * u + 2, vs = cv % kSlots;
                const int valid = it.len - (it.first + t) * kKeys;      // keys of the tile that exist
                for (int g = 0; g < 2 && ok; ++g) {
                    const int Tg = g ? it.T1 : it.T0;
                    if (t < Tg) {
                        if (!wait(P_FULL + g, np[g]++ & 1)) break;
                        if (!wait(KV_FULL + vs, (cv / kSlots) & 1)) break;
                        if (t == 0 && no[g] > 0 && !wait(O_EMPTY + g, (no[g] - 1) & 1)) break;
                        if (valid < kKeys && (g == 0 || t >= it.T0)) {
                            // rows of V past the length take no part whatever they hold; the first group to use the tile
                            // clears them (row r of chunk h: 128 bytes at h 16 KB + r 128; the swizzle stays within a row)
                            const uint32_t v = sbase + kSmemKV + vs * kTileBytes;
                            for (int e = lane; e < (kKeys - valid) * 16; e += 32)
                                asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};\n" ::"r"(
                                                 v + ((e & 8) ? kTileBytes / 2 : 0) + (valid + (e >> 4)) * 128 + (e & 7) * 16),
                                             "r"(0)
                                             : "memory");
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                        fence_after_sync();
                        if (lane == 0) {
                            const uint32_t a = tmem + kTmemS + g * 128, b = v_lo + vs * (kTileBytes >> 4);
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)          // 16 keys: 8 columns of P, 2 KB of V
                                mma_ts_split(tmem + kTmemO + g * 128, a + kk * 8, b + kk * 128, v_hi, id_pv,
                                             (t > 0 || kk > 0) ? 1u : 0u);
                            if (t == Tg - 1) mma_commit(bar(O_FULL + g));
                        }
                        if (t == Tg - 1) ++no[g];
                        __syncwarp();
                    }
                    const int Tn = end ? (ni < p.items ? (g ? nx.T1 : nx.T0) : 0) : Tg;
                    const int tn = end ? 0 : t + 1;
                    if (tn < Tn) qk(g, ck, tn == 0, tn == Tn - 1);
                }
                if (ok) free_slot(cv);
                if (ok && more) free_slot(ck);
            }
            it = nx;
            i = ni;
        }
        if (lane == 0) {
            if (!ok) record_timeout(p, 2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(DRAIN));
            mbar_wait(bar(DRAIN), 0, &never, limit);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax + epilogue
        const int g = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + lane_off + kTmemS + g * 128, o_addr = tmem + lane_off + kTmemO + g * 128;
        const float c_log2 = s.scale_log2;
        bool ok = true;
        int n = 0, items = 0;                            // tiles and items of this group
        for (int i = blockIdx.x; i < p.items && ok; i += gridDim.x) {
            const Item it = item_of(p, i);
            if (g == 1 && !it.has1) continue;
            const int r0 = it.r0 + g * kRows, r = r0 + (tid & 127);
            const int T = g ? it.T1 : it.T0;
            const int seen = r < s.R ? attn_seen(s, it.len, r) : it.len;
            const int least = T ? attn_seen_least(s, it.len, r0, min(r0 + kRows, s.R) - 1) : 0;
            float neg_m = 0.0f, l0 = 0.0f, l1 = 0.0f, l2 = 0.0f, l3 = 0.0f;
            for (int t = 0; t < T; ++t, ++n) {
                const int key0 = (it.first + t) * kKeys;
                if (!(ok = mbar_wait(bar(S_FULL + g), n & 1, abort, limit))) break;
                fence_after_sync();
                float x[128];
                row_load128(s_addr, x);
                if (key0 + kKeys > least) {              // some row of the tile does not see all of its keys
                    const int m = seen - key0;
#pragma unroll
                    for (int j = 0; j < 128; ++j) x[j] = j < m ? x[j] : -INFINITY;
                }
                float mx[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) mx[j] = x[j];
#pragma unroll
                for (int j = 8; j < 128; ++j) mx[j & 7] = fmaxf(mx[j & 7], x[j]);
                const float top = fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])),
                                        fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
                const bool need = t == 0 || fmaf(top, c_log2, neg_m) > kRescaleThreshold;
                if (__any_sync(0xffffffffu, need)) {
                    const float neg_m_new = need ? (top == -INFINITY ? 0.0f : -top * c_log2) : neg_m;
                    if (t > 0) {
                        // O holds PV(t - 1): S(t) was issued after it and is complete
                        const float alpha = fast_exp2(neg_m_new - neg_m);
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            float ov[16];
                            tmem_ld16(o_addr + c * 16, ov);
                            tmem_ld_wait(ov);
#pragma unroll
                            for (int e = 0; e < 16; ++e) ov[e] *= alpha;
                            tmem_st16(o_addr + c * 16, ov);
                        }
                        l0 *= alpha; l1 *= alpha; l2 *= alpha; l3 *= alpha;
                    }
                    neg_m = neg_m_new;
                }
                // p = 2^t: row sum in fp32, P packed to bf16 pairs (the lower key in the low half)
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        float* y = &x[h * 32 + j];
                        ffma2(y[0], y[1], c_log2, neg_m);
                        ffma2(y[2], y[3], c_log2, neg_m);
                        const float p0 = fast_exp2(y[0]), p1 = fast_exp2(y[1]);
                        const float p2 = fast_exp2(y[2]), p3 = fast_exp2(y[3]);
                        fadd2(l0, l1, p0, p1);
                        fadd2(l2, l3, p2, p3);
                        pk[j >> 1] = pack_bf16(p0, p1);
                        pk[(j >> 1) + 1] = pack_bf16(p2, p3);
                    }
                    tmem_st16(s_addr + h * 16, *reinterpret_cast<const float(*)[16]>(pk));
                }
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL + g));
            }
            if (!ok) break;
            const float l = (l0 + l1) + (l2 + l3);
            const size_t row = (size_t)it.head * s.R + r;
            const size_t at = s.splits > 1 ? (size_t)it.part * s.heads * s.R + row : row;
            const float inv = l > 0.0f ? 1.0f / l : 0.0f;
            if (r < s.R) {
                const float lse = l > 0.0f ? (log2f(l) - neg_m) * 0.6931471805599453f : -INFINITY;
                if (s.splits > 1) p.part_lse[at] = lse;
                else if (p.lse) p.lse[at] = lse;
            }
            if (T) {
                if (!(ok = mbar_wait(bar(O_FULL + g), items & 1, abort, limit))) break;
                ++items;
                fence_after_sync();
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {                // 32 d at a time
                float ov[32];
                if (T) {
                    tmem_ld16(o_addr + c * 32, *reinterpret_cast<float(*)[16]>(&ov[0]));
                    tmem_ld16(o_addr + c * 32 + 16, *reinterpret_cast<float(*)[16]>(&ov[16]));
                    tmem_ld_wait(*reinterpret_cast<float(*)[16]>(&ov[0]));
                    reg_fence(*reinterpret_cast<float(*)[16]>(&ov[16]));
#pragma unroll
                    for (int e = 0; e < 32; ++e) ov[e] *= inv;
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) ov[e] = 0.0f;
                }
                if (c == 3 && T) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(O_EMPTY + g));
                }
                if (r >= s.R) continue;
                if (s.splits > 1) {
                    float* dst = p.part_o + at * kDh + c * 32;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<float4*>(dst + e) = make_float4(ov[e], ov[e + 1], ov[e + 2], ov[e + 3]);
                } else {
                    uint4* dst = reinterpret_cast<uint4*>(p.o + at * kDh + c * 32);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        dst[e] = make_uint4(pack_bf16(ov[8 * e], ov[8 * e + 1]), pack_bf16(ov[8 * e + 2], ov[8 * e + 3]),
                                            pack_bf16(ov[8 * e + 4], ov[8 * e + 5]), pack_bf16(ov[8 * e + 6], ov[8 * e + 7]));
                }
            }
        }
        if (!ok) record_timeout(p, 3);
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

}  // namespace

cudaError_t launch_attention_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st)
{
    CUtensorMap mq, mk, mv;
    if (!encode_rows(&mq, a.q, s.R, s.heads, kRows) || !encode_rows(&mk, a.k, s.Lk, s.heads, kKeys) ||
        !encode_rows(&mv, a.v, s.Lk, s.heads, kKeys))
        return cudaErrorInvalidValue;
    Params p{};
    p.s = s;
    p.kv_len = a.kv_len;
    p.o = static_cast<__nv_bfloat16*>(a.o);
    p.lse = a.lse; p.part_o = a.part_o; p.part_lse = a.part_lse;
    p.status = a.status;
    p.q_tiles = (s.R + 2 * kRows - 1) / (2 * kRows);
    p.items = p.q_tiles * s.heads * s.splits;
    int dev = 0, nsm = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    e = cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const size_t smem = kSmemTiles + sizeof(Ctrl);
    e = cudaFuncSetAttribute(attention_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attention_tc_kernel<<<p.items < nsm ? p.items : nsm, kThreads, smem, st>>>(mq, mk, mv, p);
    return cudaGetLastError();
}

}  // namespace rola
