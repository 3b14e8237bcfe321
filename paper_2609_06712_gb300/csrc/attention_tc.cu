// Softmax attention over a dense key set on the 5th-generation tensor cores
// (bf16 operands, fp32 accumulation in TMEM).
//
//   o_r = sum_j softmax_j(scale q_r . k_j) v_j   over the keys row r sees
//
// Rows are the G Lq queries of the heads that share a key head (contiguous in
// q), so a shared key head is read once for all of them.  An item is 256 rows of
// a head (two groups of 128) over a range of its keys, which come in tiles of 128
// and are worked on in steps of 64:
//   S_g  = Q_g (128 rows x 128 d, smem, K-major)  x  K^T (64 keys x 128 d, smem, K-major)
//   O_g += P_g (128 rows x 64 keys, TMEM, bf16)   x  V   (64 keys x 128 d, smem, MN-major)
// TMEM (512 columns): per group two S buffers of 64 columns and O, 128 columns;
// P overwrites the first half of its S buffer.  One thread issues a group's
// products: after PV_g(n) comes QK_g(n + 2) into the same buffer (products of one
// thread execute in order), so a group's softmax has its next scores ready when it is
// done with the present ones, and the two groups' softmax runs under each other's
// products.  Steps run on across items, so items follow one another without a gap.
// With steps of 128 TMEM would hold one S buffer per group, and QK(n + 1) would
// wait for PV(n), and that for the softmax of step n.
//
// Softmax (base 2, one thread per row, the whole row of S in registers): each
// row keeps -m and its sum l in fp32.  With t = s scale log2(e) - m, m is raised
// only when the step's largest t exceeds 2^3 (or on the item's first step); O
// and l are then scaled by 2^(m_old - m_new).  p = 2^t enters l in fp32 and the
// product rounded to bf16 (the operand type of the tensor core).  A row sees a
// prefix of the keys (its length, or its causal limit), so a row that sees
// nothing in the item's first step sees nothing in the item: its p stay 0, l = 0.  Where the first
// scores are -inf (infinite keys) m starts at the lowest number and is raised by the first finite one.
// Keys past the length: their scores are replaced by -inf whatever they are, and
// their rows of V are zeroed in shared memory (0 x NaN would be NaN).
//
// Measured: 40 heads of 75600 rows to 512 keys 680 us (1170 TFLOP/s), of 4725 rows to 8192 keys 530 us (1500 TFLOP/s), 12
// heads of 8190 rows to 8190 keys 315 us (1310 TFLOP/s); one token, 4 x 40 heads on 8, 32760 keys 94 us (5.7 TB/s).  A
// single token is bound by HBM.  Else the tensor pipe is 69 % busy (8190 keys), its QK products of 128 x 64 at 3/4 of
// the full rate; the rest are waits along the chain scores, softmax, PV of each group.  Over 512 keys an
// item takes 8.7 us: products 5.0, its ends 1.6, and 2.1 that no measurement has placed yet.
//
// Warps (384 threads, one persistent CTA per SM): 0-3 softmax and epilogue of
// group 0, 4-7 of group 1, 8 TMA (Q of both groups, and K, V tiles in one ring of
// five 32 KB slots), 9 and 10 products, 11 the zeroing of V's rows.  Shared memory 64 + 160 KB.  Every mbarrier wait
// is bounded; a wait that gives up records ROLA_ERR_TIMEOUT and the CTA drains
// what it issued and frees its TMEM.
#include <float.h>

#include "attention_tc.cuh"

namespace rola {
namespace {

using namespace tc;

constexpr int kRows = 128, kKeys = 128, kStep = 64, kSlots = 5;    // rows of a group, keys of a tile and of a step
constexpr int kTmaWarp = 8, kMmaWarp = 9, kCutWarp = 11, kThreads = 384;
constexpr uint32_t kTileBytes = 128 * 128 * 2;               // [d-chunk][128 rows][64]
constexpr uint32_t kSmemQ = 0, kSmemKV = 2 * kTileBytes, kSmemTiles = kSmemKV + kSlots * kTileBytes;
constexpr uint32_t kTmemCols = 512, kTmemS = 0, kTmemO = 256;   // S_g,b at 128 g + 64 b, O_g at 256 + 128 g
constexpr float kRescaleThreshold = 8.0f;                    // log2 units

// S_FULL, P_FULL: 2 g + b; the others g, or a slot
enum Bar { Q_FULL = 0, Q_EMPTY = 2, S_FULL = 4, P_FULL = 8, PV_DONE = 12, O_FULL = 14, O_EMPTY = 16, KV_FULL = 18,
           KV_EMPTY = KV_FULL + kSlots, V_CUT = KV_EMPTY + kSlots, DRAIN = V_CUT + 4, NUM_BARS = DRAIN + 2 };

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
    bool wide;                   // o is 32-byte aligned
    int q_tiles;                 // 256-row tiles of a head
    int items;                   // q_tiles heads splits
};

__device__ __forceinline__ void record_timeout(const Params& p, int where)
{
    if (atomicCAS(&p.status->code, 0, (int)ROLA_ERR_TIMEOUT) == 0) p.status->where = 80 + where;
}

// One item: rows r0 .. of `head`, key tiles from `first`, H0 and H1 steps of the two groups from
// there (0: the group has no rows, or its rows see nothing there).
struct Item {
    int head, r0, len, part, first;
    int H0, H1, H;               // per group, and the larger
    bool has1;
};
__device__ __forceinline__ Item item_of(const Params& p, int i)
{
    const AttnShape& s = p.s;
    Item it;
    it.part = 0;
    if (s.splits > 1) {
        it.part = i % s.splits;
        i /= s.splits;
    }
    int qt;
    if (s.causal) {              // the longest rows of every head first
        qt = falling_tile(i / s.heads, p.q_tiles, s.H / s.Hk);
        it.head = i % s.heads;
    } else {                     // head by head: the CTAs in flight share few heads' keys
        it.head = i / p.q_tiles;
        qt = i - it.head * p.q_tiles;
    }
    it.r0 = qt * 2 * kRows;
    it.len = attn_len(s, p.kv_len, it.head / s.Hk);
    it.has1 = it.r0 + kRows < s.R;
    const int n0 = attn_seen_most(s, it.len, it.r0, min(it.r0 + kRows, s.R) - 1);
    const int n1 = it.has1 ? attn_seen_most(s, it.len, it.r0 + kRows, min(it.r0 + 2 * kRows, s.R) - 1) : 0;
    const int t = (max(n0, n1) + kKeys - 1) / kKeys;
    int end = t;
    it.first = 0;
    if (s.splits > 1) {          // tiles x parts stays below 2^31: at most 2^23 tiles and 152 parts
        it.first = t * it.part / s.splits;
        end = t * (it.part + 1) / s.splits;
    }
    const int from = it.first * 2;
    it.H0 = max(min((n0 + kStep - 1) / kStep, end * 2) - from, 0);
    it.H1 = max(min((n1 + kStep - 1) / kStep, end * 2) - from, 0);
    it.H = max(it.H0, it.H1);
    return it;
}

// Tile t of the item ends past the sequence's length, where the memory holds other keys (past Lk the copy
// writes zeros).
__device__ __forceinline__ bool cut_tile(const AttnShape& s, const Item& it, int t)
{
    return (it.first + t + 1) * kKeys > it.len && it.len < s.Lk;
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
            for (int b = 0; b < 2; ++b) {
                mbar_init(bar(S_FULL + 2 * g + b), 1);
                mbar_init(bar(P_FULL + 2 * g + b), 4);
            }
            mbar_init(bar(PV_DONE + g), 1);
            mbar_init(bar(DRAIN + g), 1);
            mbar_init(bar(O_FULL + g), 1);
            mbar_init(bar(O_EMPTY + g), 4);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(bar(KV_FULL + i), 1);
            mbar_init(bar(KV_EMPTY + i), p.kv_len ? 3 : 2);      // both groups, and the zeroing warp
        }
        for (int i = 0; i < 4; ++i) mbar_init(bar(V_CUT + i), 1);
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
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it = item_of(p, i);
            if (it.H == 0) continue;
            for (int t = 0; t < (it.H + 1) / 2 && ok; ++t) {
                const int key0 = (it.first + t) * kKeys;
                // test hook: the CTA's first K tile is never loaded, so the waits on it run out
                ring(&map_k, key0, it.head, (s.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) && c == 0);
                if (ok) ring(&map_v, key0, it.head, false);
                if (t) continue;
                // Q, whose buffers are free only after the last item's QK, behind the first tiles, whose slots are
                // free before (75600 rows to 512 keys: 705 us the other way round, 684 so)
                for (int g = 0; g < 2 && ok; ++g) {
                    if ((g ? it.H1 : it.H0) == 0) continue;
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
    } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
        // ------------------------------------------------------------ products of group g
        // One elected thread per group.  A wait that is over costs it some 150 cycles, 8 products 140, a commit 50
        // to 150: one thread for both groups took 2000 cycles a step where the tensor core needs 1280.
        const int g = warp - kMmaWarp;
        if (elect_one()) {
            const uint32_t id_qk = idesc_bf16(kRows, kStep, false, false), id_pv = idesc_bf16(kRows, kDh, false, true);
            const uint64_t dq = smem_desc(sbase + kSmemQ + g * kTileBytes, 16, 1024);     // A of QK (K-major)
            const uint64_t dk = smem_desc(sbase + kSmemKV, 16, 1024);                     // B of QK (K-major)
            const uint64_t dv = smem_desc(sbase + kSmemKV, kTileBytes / 2, 1024);         // B of PV (MN-major)
            const uint32_t q_lo = (uint32_t)dq, q_hi = (uint32_t)(dq >> 32), k_lo = (uint32_t)dk, k_hi = (uint32_t)(dk >> 32);
            const uint32_t v_lo = (uint32_t)dv, v_hi = (uint32_t)(dv >> 32);
            const uint32_t t_s = tmem + kTmemS + g * 128, t_o = tmem + kTmemO + g * 128;
            bool ok = true;
            auto wait = [&](int b, int parity) {
                if (ok) ok = mbar_wait(bar(b), parity, abort, limit);
                return ok;
            };
            int nqk = 0, npv = 0, nq = 0, no = 0, ncut = 0;      // steps, Q tiles, items with O, cut tiles
            // This group is done with the slot of ring use c: after its products, or, where it had none, once the
            // tile is there (the slot's uses stay in step that way).
            auto release = [&](int slot, bool used) {
                if (!ok) return;
                if (used) mma_commit(bar(KV_EMPTY + slot));
                else mbar_arrive(bar(KV_EMPTY + slot));
            };
            // S = Q K^T of step h of an item that starts at the CTA's `tile`-th tile; Hg: the group's steps
            auto qk = [&](const Item& it, int Hg, int tile, int h) {
                const int c = 2 * (tile + (h >> 1)), slot = c % kSlots;
                if ((h & 1) == 0) wait(KV_FULL + slot, (c / kSlots) & 1);
                const bool mine = h < Hg;
                if (h == 0 && mine) wait(Q_FULL + g, nq++ & 1);
                if (mine && ok) {
                    const int b = nqk++ & 1;
                    const uint32_t k = k_lo + slot * (kTileBytes >> 4) + (h & 1) * 512;       // 64 rows of 128 bytes
                    fence_after_sync();
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        const uint32_t o = (kk >> 2) * (kTileBytes >> 5) + (kk & 3) * 2;
                        mma_ss_split(t_s + b * 64, q_lo + o, q_hi, k + o, k_hi, id_qk, kk > 0 ? 1u : 0u);
                    }
                    mma_commit(bar(S_FULL + 2 * g + b));
                    if (h == Hg - 1) mma_commit(bar(Q_EMPTY + g));
                }
                if ((h & 1) || h == it.H - 1) release(slot, (h & ~1) < Hg);
            };
            // the next item that has steps, from the turn on
            auto next_item = [&](int& turn, Item& it) {
                int i;
                for (; (i = turn_item(turn, p.items)) < p.items; ++turn) {
                    it = item_of(p, i);
                    if (it.H) break;
                }
                return i < p.items;
            };
            Item it{}, nx{};
            int turn = 0, tile = 0, done = 0;      // done: QK steps of `it` issued already
            bool have = next_item(turn, it);
            while (have && ok) {
                ++turn;
                const bool more = next_item(turn, nx);
                const int ntile = tile + (it.H + 1) / 2;
                const int Hg = g ? it.H1 : it.H0, Hn = more ? (g ? nx.H1 : nx.H0) : 0;
                const int nsteps = more ? min(nx.H, 2) : 0;
                int ndone = 0;
                for (; done < min(it.H, 2) && ok; ++done) qk(it, Hg, tile, done);
                for (int h = 0; h < it.H && ok; ++h) {
                    const int c = 2 * (tile + (h >> 1)) + 1, slot = c % kSlots;
                    if ((h & 1) == 0) {
                        wait(KV_FULL + slot, (c / kSlots) & 1);
                        if (cut_tile(s, it, h >> 1)) {
                            wait(V_CUT + (ncut & 3), (ncut >> 2) & 1);
                            ++ncut;
                        }
                    }
                    if (h < Hg) {
                        const int b = npv & 1;
                        wait(P_FULL + 2 * g + b, (npv++ >> 1) & 1);
                        if (h == 0 && no > 0) wait(O_EMPTY + g, (no - 1) & 1);
                        if (!ok) break;
                        const uint32_t v = v_lo + slot * (kTileBytes >> 4) + (h & 1) * 512;
                        fence_after_sync();
                        mma_ts_split(t_o, t_s + b * 64, v, v_hi, id_pv, h > 0 ? 1u : 0u);
#pragma unroll
                        for (int kk = 1; kk < 4; ++kk)              // 16 keys: 8 columns of P, 2 KB of V
                            mma_ts_split(t_o, t_s + b * 64 + kk * 8, v + kk * 128, v_hi, id_pv, 1u);
                        if (h == Hg - 2) mma_commit(bar(PV_DONE + g));
                        if (h == Hg - 1) {
                            ++no;
                            mma_commit(bar(O_FULL + g));
                        }
                    }
                    if ((h & 1) || h == it.H - 1) release(slot, (h & ~1) < Hg);
                    if (h + 2 < it.H) {
                        qk(it, Hg, tile, h + 2);
                    } else if (ndone < nsteps && (ndone > 0 || Hn == 0 || mbar_try_wait(bar(Q_FULL + g), nq & 1))) {
                        qk(nx, Hn, ntile, ndone);      // the next item's first steps, once its Q is there
                        ++ndone;
                    }
                }
                it = nx;
                have = more;
                tile = ntile;
                done = ndone;
            }
            if (!ok) record_timeout(p, 2);
            // every product issued completes before TMEM is released
            int never = 0;
            mma_commit(bar(DRAIN + g));
            mbar_wait(bar(DRAIN + g), 0, &never, limit);
        }
        __syncwarp();
    } else if (warp == kCutWarp) {
        // ------------------------------------------------------------ V past a sequence's length
        // Those rows take no part whatever they hold: they are cleared in shared memory before the product
        // reads them (row r of chunk h: 128 bytes at h 16 KB + r 128; the swizzle stays within a row).  The warp
        // follows every tile, so that it knows each slot's turn; V_CUT has four barriers because a group may be up to
        // two V tiles of the ring behind it.
        bool ok = true;
        int c = 0, ncut = 0;
        auto next = [&]() {
            ok = __all_sync(0xffffffffu, mbar_wait(bar(KV_FULL + c % kSlots), (c / kSlots) & 1, abort, limit));
            return ok;
        };
        auto done = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(KV_EMPTY + c % kSlots));
            ++c;
        };
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok && p.kv_len; ++turn) {
            const Item it = item_of(p, i);
            for (int t = 0; t < (it.H + 1) / 2; ++t) {
                if (!next()) break;                      // K
                done();
                if (!next()) break;                      // V
                if (cut_tile(s, it, t)) {
                    const int slot = c % kSlots, valid = it.len - (it.first + t) * kKeys;
                    for (int e = lane; e < (kKeys - valid) * 16; e += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};\n" ::"r"(
                                         sbase + kSmemKV + slot * kTileBytes + ((e & 8) ? kTileBytes / 2 : 0) +
                                         (valid + (e >> 4)) * 128 + (e & 7) * 16),
                                     "r"(0)
                                     : "memory");
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(V_CUT + (ncut & 3)));
                    ++ncut;
                }
                done();
            }
        }
        if (!ok && lane == 0) record_timeout(p, 4);
    } else {
        // ------------------------------------------------------------ softmax + epilogue
        const int g = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_base = tmem + lane_off + kTmemS + g * 128, o_addr = tmem + lane_off + kTmemO + g * 128;
        const float c_log2 = s.scale_log2;
        bool ok = true;
        int n = 0, items = 0, pairs = 0;                 // steps and items of this group, items of two steps or more
        for (int turn = 0, i; (i = turn_item(turn, p.items)) < p.items && ok; ++turn) {
            const Item it = item_of(p, i);
            if (g == 1 && !it.has1) continue;
            const int r0 = it.r0 + g * kRows, r = r0 + (tid & 127);
            const int H = g ? it.H1 : it.H0;
            const int seen = r < s.R ? attn_seen(s, it.len, r) : it.len;
            const int least = H ? attn_seen_least(s, it.len, r0, min(r0 + kRows, s.R) - 1) : 0;
            float neg_m = 0.0f, l0 = 0.0f, l1 = 0.0f, l2 = 0.0f, l3 = 0.0f;
            for (int h = 0; h < H; ++h, ++n) {
                const int key0 = it.first * kKeys + h * kStep, b = n & 1;
                const uint32_t s_addr = s_base + b * 64;
                if (!(ok = mbar_wait_warp(bar(S_FULL + 2 * g + b), (n >> 1) & 1, abort, limit))) break;
                fence_after_sync();
                float x[64];
                row_load<64>(s_addr, x);
                if (key0 + kStep > least) {              // some row of the group does not see all of the step's keys
                    const int m = seen - key0;
#pragma unroll
                    for (int j = 0; j < 64; ++j) x[j] = j < m ? x[j] : -INFINITY;
                }
                float mx[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) mx[j] = x[j];
#pragma unroll
                for (int j = 8; j < 64; ++j) mx[j & 7] = fmaxf(mx[j & 7], x[j]);
                const float top = fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])),
                                        fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7])));
                const bool need = h == 0 || fmaf(top, c_log2, neg_m) > kRescaleThreshold;
                if (__any_sync(0xffffffffu, need)) {
                    // over scores of -inf alone m is the lowest number, which any finite score to come exceeds
                    const float neg_m_new = need ? fminf(-top * c_log2, FLT_MAX) : neg_m;
                    if (h > 0) {
                        // O has to hold PV(n - 1) before it is scaled: S(n + 1) was issued after it; on the
                        // item's last step there may be no S(n + 1) yet, and PV(n - 1) has a barrier of its own
                        ok = h < H - 1 ? mbar_wait_warp(bar(S_FULL + 2 * g + (b ^ 1)), ((n + 1) >> 1) & 1, abort, limit)
                                       : mbar_wait_warp(bar(PV_DONE + g), pairs & 1, abort, limit);
                        if (!ok) break;
                        fence_after_sync();
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
                for (int q = 0; q < 2; ++q) {
                    uint32_t pk[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        float* y = &x[q * 32 + j];
                        ffma2(y[0], y[1], c_log2, neg_m);
                        ffma2(y[2], y[3], c_log2, neg_m);
                        const float p0 = fast_exp2(y[0]), p1 = fast_exp2(y[1]);
                        const float p2 = fast_exp2(y[2]), p3 = fast_exp2(y[3]);
                        fadd2(l0, l1, p0, p1);
                        fadd2(l2, l3, p2, p3);
                        pk[j >> 1] = pack_bf16(p0, p1);
                        pk[(j >> 1) + 1] = pack_bf16(p2, p3);
                    }
                    tmem_st16(s_addr + q * 16, *reinterpret_cast<const float(*)[16]>(pk));
                }
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(P_FULL + 2 * g + b));
            }
            if (!ok) break;
            const float l = (l0 + l1) + (l2 + l3);
            const size_t row = (size_t)it.head * s.R + r;
            const size_t at = s.splits > 1 ? (size_t)it.part * s.heads * s.R + row : row;
            // l is 0 where nothing is seen, and over scores of -inf alone: then p is 0 / 0 (with parts the join says
            // so); a NaN sum stays one
            const float inv = l == 0.0f ? (seen > 0 && s.splits == 1 ? __int_as_float(0x7fc00000) : 0.0f) : 1.0f / l;
            if (r < s.R) {
                const float lse = l == 0.0f ? -INFINITY : (log2f(l) - neg_m) * 0.6931471805599453f;
                if (s.splits > 1) p.part_lse[at] = lse;
                else if (p.lse) p.lse[at] = lse;
            }
            if (H) {
                if (!(ok = mbar_wait_warp(bar(O_FULL + g), items & 1, abort, limit))) break;
                ++items;
                if (H > 1) ++pairs;
                fence_after_sync();
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {                // 32 d at a time
                float ov[32];
                if (H) {
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
                if (c == 3 && H) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(O_EMPTY + g));
                }
                if (r >= s.R) continue;
                if (s.splits > 1) {
                    float* dst = p.part_o + at * kDh + c * 32;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = __float_as_uint(ov[e + j]);
                        st_global32(dst + e, y);
                    }
                } else {
                    // 32 bytes (a whole sector) of the lane's row at a time
                    __nv_bfloat16* dst = p.o + at * kDh + c * 32;
#pragma unroll
                    for (int e = 0; e < 32; e += 16) {
                        uint32_t y[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) y[j] = pack_bf16(ov[e + 2 * j], ov[e + 2 * j + 1]);
                        store_row32(dst + e, y, p.wide);
                    }
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
    p.wide = (reinterpret_cast<uintptr_t>(a.o) & 31u) == 0;
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
