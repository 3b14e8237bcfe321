// The gated residual sum of a block and its norms, and their gradients (formulas: include/rola.h).
//
//   hh = norm_b(h) or h,  u = x + gate gamma_h hh,  v = norm(u),  y = v g + c
//   with g = gamma (1 + scale), c = beta (1 + scale) + shift
//   a = dy g,  t = dout + rstd (a [- mean a] - v mean(a v)),  dx = t
//   e = t gate gamma_h,  dh = rstd_h (e [- mean e] - hh mean(e hh)) or e
//   column sums of each sample: A = sum dy v, B = sum dy, E = sum t hh; every vector's gradient is made of them.
//
// HBM-bound: x and h in, the sum and y out forward; x, h, dy and dout in, dx and dh out backward (the sum is formed again from
// x and h, as many bytes as reading it would take, so that nothing is lost to its rounding), with some 20 and 40 fp32
// operations an element.  What has to be kept up with is 44 bytes per ns and SM, 580 cycles for a row of 1536 forward:
//   - a row is held in registers by the threads of a group (a warp, or a CTA), 16 elements a thread, so that the norm's
//     two passes, the sums and the outputs read it once; a group's coming rows are copied ahead into a ring in shared
//     memory (Feed), 200 KB an SM in flight, whatever they are aligned to;
//   - a row's sums are one step of shuffles, shared memory and a barrier for up to eight values (sum_group); backward, the
//     sums of both norms are taken apart so that they all are one step;
//   - arithmetic is two elements an instruction, and where a row fills its threads nothing is masked (FULL).
// A group takes neighbouring rows, and its column sums stay in registers until a sample or its rows end; then it leaves them
// in a slot of its own, and a second kernel, launched ahead, adds the slots in a fixed order.  All statistics and sums
// are fp32.  Rows too long for registers, or of a length that no form takes, go through memory in several passes.
//
// Measured, bf16, with gate, scale and shift: 75600 x 5120 forward 514 us (6.0 TB/s, 89 % of a copy), backward 750 us (6.2);
// 2 x 16380 x 1536 forward 76, backward 112 us (5.3, 5.4; the ramp and the tail count); with a norm behind the branch too,
// 3 x 4095 x 2560 46 and 83 us.  Backward, rows of 5121 to 8192 elements spill 270 bytes a thread (20000 x 8192: 3.8 TB/s).
//
// The variance is taken about the rounded mean, as in the layer norm.
#include <type_traits>

#include "norm_rows.cuh"
#include "residual_norm.cuh"
#include "tcgen05.cuh"

namespace rola {
namespace {

// Element c of a vector of sample s, or `none`.
template <typename T>
__device__ __forceinline__ float vec(const void* p, size_t c, float none)
{
    return p ? to_float(static_cast<const T*>(p)[c]) : none;
}
// What the formulas above call g, c and gate gamma_h, of column c of sample s.
template <typename T>
__device__ __forceinline__ float gain_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return vec<T>(a.gamma, c, 1.0f) * (1.0f + vec<T>(a.scale, s * sh.mod_stride + c, 0.0f));
}
template <typename T>
__device__ __forceinline__ float shift_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return fmaf(vec<T>(a.beta, c, 0.0f), 1.0f + vec<T>(a.scale, s * sh.mod_stride + c, 0.0f),
                vec<T>(a.shift, s * sh.mod_stride + c, 0.0f));
}
template <typename T>
__device__ __forceinline__ float branch_gain_of(const RnShape& sh, const RnArgs& a, int s, int c)
{
    return vec<T>(a.gate, s * sh.mod_stride + c, 1.0f) * vec<T>(a.gamma_h, c, 1.0f);
}

// ---------------------------------------------------------------- rows of any length, from memory

constexpr int kLongThreads = 512;

// Mean (0 for the RMS norm) and 1 / size of n values f(c), in two passes.
template <typename F>
__device__ __forceinline__ float2 row_stats(int kind, int d, float eps, float2 (*red)[32], int& turn, F f)
{
    float mu = 0.0f;
    if (kind == ROLA_NORM_LAYER) {
        float s = 0.0f;
        for (int c = threadIdx.x; c < d; c += kLongThreads) s += f(c);
        mu = group_sum<false>(s, 0.0f, red, turn).x / (float)d;
    }
    float q = 0.0f;
    for (int c = threadIdx.x; c < d; c += kLongThreads) {
        const float t = f(c) - mu;
        q = fmaf(t, t, q);
    }
    return make_float2(mu, 1.0f / sqrtf(group_sum<false>(q, 0.0f, red, turn).x / (float)d + eps));
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_fwd_long_kernel(const RnShape sh, const RnArgs a)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const T *x = static_cast<const T*>(a.x) + r * sh.d, *h = a.h ? static_cast<const T*>(a.h) + r * sh.d : nullptr;
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float2 hs = make_float2(0.0f, 1.0f), us = make_float2(0.0f, 1.0f);
        if (h && sh.branch != ROLA_NORM_NONE) {
            hs = row_stats(sh.branch, sh.d, sh.eps, red, turn, [&](int c) { return to_float(h[c]); });
            st.z = hs.x;
            st.w = hs.y;
        }
        auto sum = [&](int c) {
            const float u = to_float(x[c]);
            return h ? fmaf(branch_gain_of<T>(sh, a, s, c), (to_float(h[c]) - hs.x) * hs.y, u) : u;
        };
        if (sh.norm != ROLA_NORM_NONE) {
            us = row_stats(sh.norm, sh.d, sh.eps, red, turn, sum);
            st.x = us.x;
            st.y = us.y;
        }
        for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
            const float u = sum(c);                       // read before the writes: out and y may be x or h
            if (a.out) static_cast<T*>(a.out)[r * sh.d + c] = from_float<T>(u);
            if (a.y)
                static_cast<T*>(a.y)[r * sh.d + c] =
                    from_float<T>(fmaf((u - us.x) * us.y, gain_of<T>(sh, a, s, c), shift_of<T>(sh, a, s, c)));
        }
        if (a.stats && threadIdx.x == 0) reinterpret_cast<float4*>(a.stats)[r] = st;
    }
}

// The values of one element of the backward: hh, v, and t given the row's means.
template <typename T>
struct Element {
    float hh, v, dy, t, gg;
    __device__ __forceinline__ Element(const RnShape& sh, const RnArgs& a, int s, long long r, int c, float4 st, float m1,
                                       float m2)
    {
        const size_t at = (size_t)(r * sh.d + c);
        hh = a.h ? to_float(static_cast<const T*>(a.h)[at]) : 0.0f;
        if (sh.branch != ROLA_NORM_NONE) hh = (hh - st.z) * st.w;
        gg = branch_gain_of<T>(sh, a, s, c);
        t = a.dout ? to_float(static_cast<const T*>(a.dout)[at]) : 0.0f;
        v = dy = 0.0f;
        if (sh.norm != ROLA_NORM_NONE) {
            v = (fmaf(gg, hh, to_float(static_cast<const T*>(a.x)[at])) - st.x) * st.y;
            dy = to_float(static_cast<const T*>(a.dy)[at]);
            t = fmaf(st.y, dy * gain_of<T>(sh, a, s, c) - m1 - v * m2, t);
        }
    }
};

// mean a, mean(a v), mean e and mean(e hh) of each row (the first and third 0 for the RMS norm).
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_moments_kernel(const RnShape sh, const RnArgs a)
{
    __shared__ float2 red[2][32];
    int turn = 0;
    const float inv_d = 1.0f / (float)sh.d;
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const float4 st = reinterpret_cast<const float4*>(a.stats)[r];
        float4 m = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (sh.norm != ROLA_NORM_NONE) {
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
                const Element<T> e(sh, a, s, r, c, st, 0.0f, 0.0f);
                const float av = e.dy * gain_of<T>(sh, a, s, c);
                s1 += av;
                s2 = fmaf(av, e.v, s2);
            }
            const float2 q = group_sum<false>(s1, s2, red, turn);
            m.x = sh.norm == ROLA_NORM_LAYER ? q.x * inv_d : 0.0f;
            m.y = q.y * inv_d;
        }
        if (sh.branch != ROLA_NORM_NONE) {
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
                const Element<T> e(sh, a, s, r, c, st, m.x, m.y);
                s1 = fmaf(e.t, e.gg, s1);
                s2 = fmaf(e.t * e.gg, e.hh, s2);
            }
            const float2 q = group_sum<false>(s1, s2, red, turn);
            m.z = sh.branch == ROLA_NORM_LAYER ? q.x * inv_d : 0.0f;
            m.w = q.y * inv_d;
        }
        if (threadIdx.x == 0) a.moments[r] = m;
    }
}
// Column sums of part blockIdx.y; before dx and dh, which may take the place of dout and dy.
template <typename T>
__global__ void __launch_bounds__(128) rn_columns_kernel(const RnShape sh, const RnArgs a)
{
    const int c = blockIdx.x * 128 + threadIdx.x, part = blockIdx.y;
    if (c >= sh.d) return;
    const long long r1 = rn_row(sh.total, a.parts, part + 1);
    float A = 0.0f, B = 0.0f, E = 0.0f;
    for (long long r = rn_row(sh.total, a.parts, part); r < r1; ++r) {
        const int s = (int)(r / sh.rows);
        const float4 m = a.moments[r];
        const Element<T> e(sh, a, s, r, c, reinterpret_cast<const float4*>(a.stats)[r], m.x, m.y);
        A = fmaf(e.dy, e.v, A);
        B += e.dy;
        E = fmaf(e.t, e.hh, E);
        if (r + 1 == r1 || (r + 1) % sh.rows == 0) {
            const int dp = rn_padded(sh.d);
            float* out = a.part + rn_slot(part, s, sh.d) + c;
            out[0] = A;
            out[dp] = B;
            out[2 * (size_t)dp] = E;
            A = B = E = 0.0f;
        }
    }
}
template <typename T>
__global__ void __launch_bounds__(kLongThreads) rn_bwd_long_kernel(const RnShape sh, const RnArgs a)
{
    for (long long r = blockIdx.x; r < sh.total; r += gridDim.x) {
        const int s = (int)(r / sh.rows);
        const float4 st = reinterpret_cast<const float4*>(a.stats)[r], m = a.moments[r];
        for (int c = threadIdx.x; c < sh.d; c += kLongThreads) {
            const Element<T> e(sh, a, s, r, c, st, m.x, m.y);
            static_cast<T*>(a.dx)[r * sh.d + c] = from_float<T>(e.t);
            if (!a.dh) continue;
            float dh = e.t * e.gg;
            if (sh.branch != ROLA_NORM_NONE) dh = st.w * (dh - m.z - e.hh * m.w);
            static_cast<T*>(a.dh)[r * sh.d + c] = from_float<T>(dh);
        }
    }
}

// ---------------------------------------------------------------- rows in registers

constexpr int kWarpGroups = 4;                       // rows of a CTA whose rows have a warp each
constexpr int kMaxDepth = 16;                        // rows in a group's ring
constexpr size_t kRingBytes = 208 << 10;             // of the rings of an SM's CTAs
constexpr size_t kBarBytes = kWarpGroups * kMaxDepth * 8;

// The elements of piece i of a thread's EL.
template <int V, int EL>
__device__ __forceinline__ float (&slice(float (&v)[EL], int i))[V] { return reinterpret_cast<float(&)[V]>(v[i * V]); }

// v = 0 past the row's end.
template <int V, bool FULL, int EL>
__device__ __forceinline__ void clear_rest(int gt, int tpr, int pieces, float (&v)[EL])
{
    if constexpr (!FULL)
#pragma unroll
        for (int i = 0; i < EL / V; ++i) {
            const bool in = gt + i * tpr < pieces;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = in ? v[i * V + e] : 0.0f;
        }
}

// Pieces are 16 bytes where every row starts at a multiple of them, else one element, or two of bf16 where the width
// and the pointers allow 4 bytes.
template <typename T, int V>
constexpr bool kWide = V * sizeof(T) == 16;

// Bytes of a row's place in the ring: a row that starts anywhere is copied with the 16-byte words that it begins and
// ends in.
__host__ __device__ __forceinline__ uint32_t place_bytes(int d, int esz, bool wide)
{
    return wide ? (uint32_t)(d * esz) : (uint32_t)((d * esz + 15) / 16 * 16 + 16);
}

// A group's rows [next, end) of the matrices a.in (those that are not NULL), brought ahead into `depth` slots of shared
// memory by bulk copies, one per matrix, with an mbarrier a slot.  A slot is refilled after its row has been read into
// registers by the whole group.  A row that does not arrive is lost: it becomes NaN (the call has no status word).  A thread
// that has waited in vain sees what is under way land, so long as it does within the limit once more, then waits no more, and
// if it is the copying one issues no more copies: the group's rows behind those are lost too.
// Pieces of less than 16 bytes: rows that start at any element; they are copied with the whole 16-byte words that they begin
// and end in, and where such a word is not all inside the matrix (its first and last row) element by element.
template <typename T, int V, int EL, int N, bool FULL>
struct Feed {
    long long next, end;
    int tpr, gt, depth, slot, phase;
    bool lost;                           // this thread has waited in vain
    uint32_t ring, bars, here, step;     // here: the present slot; step: bytes of a slot

    static __device__ __forceinline__ uint32_t place(const RnShape& sh) { return place_bytes(sh.d, sizeof(T), kWide<T, V>); }
    static __device__ __forceinline__ int count(const RnArgs& a)
    {
        int k = 0;
#pragma unroll
        for (int n = 0; n < N; ++n) k += a.in[n] != nullptr;
        return k;
    }
    // Bytes from a 16-byte word's begin to row r of matrix n.
    static __device__ __forceinline__ uint32_t offset(const RnShape& sh, const RnArgs& a, int n, long long r)
    {
        if constexpr (kWide<T, V>) return 0;
        else return (uint32_t)(reinterpret_cast<uintptr_t>(a.in[n]) + (unsigned long long)r * (sh.d * sizeof(T))) & 15u;
    }
    // Of the words that row r lies in, from its first, bytes [lo, hi) are copied: those of words inside the matrix.
    static __device__ __forceinline__ void span(const RnShape& sh, long long r, uint32_t from, uint32_t& lo, uint32_t& hi)
    {
        const uint32_t row = sh.d * (uint32_t)sizeof(T);
        lo = (unsigned long long)r * row < from ? 16u : 0u;
        hi = (from + row + 15u) & ~15u;
        if ((unsigned long long)(sh.total - r) * row < hi - from) hi -= 16u;
        if (hi < lo) hi = lo;
    }
    __device__ __forceinline__ void copy(const RnShape& sh, const RnArgs& a, int to)         // one thread
    {
        const uint32_t bar = bars + to * 8, step = place(sh);
        uint32_t at = ring + to * this->step, bytes = this->step;
        if constexpr (!kWide<T, V>) {
            bytes = 0;
            uint32_t p = at;
#pragma unroll 1
            for (int n = 0; n < N; ++n)
                if (a.in[n]) {
                    const uint32_t from = offset(sh, a, n, next), row = sh.d * (uint32_t)sizeof(T);
                    uint32_t lo, hi;
                    span(sh, next, from, lo, hi);
                    bytes += hi - lo;
                    // elements outside [lo, hi): at most 15 bytes at each end
                    const T* src = static_cast<const T*>(a.in[n]) + next * sh.d;
                    for (uint32_t w = from; w < from + row; w += sizeof(T)) {
                        if (w >= lo && w < hi) {
                            w = hi - sizeof(T);          // on to the first element behind
                            continue;
                        }
                        const T x = src[(w - from) / sizeof(T)];
                        if constexpr (sizeof(T) == 4)
                            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(p + w), "f"(to_float(x)) : "memory");
                        else
                            asm volatile("st.shared.u16 [%0], %1;\n" ::"r"(p + w), "h"(*reinterpret_cast<const uint16_t*>(&x)) : "memory");
                    }
                    p += step;
                }
        }
        tc::mbar_expect_tx(bar, bytes);                  // arrives behind the elements stored above
#pragma unroll 1
        for (int n = 0; n < N; ++n)
            if (a.in[n]) {
                uint32_t from = 0, lo = 0, hi = step;
                if constexpr (!kWide<T, V>) {
                    from = offset(sh, a, n, next);
                    span(sh, next, from, lo, hi);
                }
                if (hi > lo)
                    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(
                                     at + lo),
                                 "l"(reinterpret_cast<uintptr_t>(static_cast<const T*>(a.in[n]) + next * sh.d) - from + lo),
                                 "r"(hi - lo), "r"(bar)
                                 : "memory");
                at += step;
            }
        ++next;
    }
    // rows [r0, end) of the group; smem: the groups' mbarriers, then their rings
    __device__ __forceinline__ void start(const RnShape& sh, const RnArgs& a, unsigned char* smem, int group, long long r0)
    {
        bars = smem_u32(smem) + group * kMaxDepth * 8;
        ring = smem_u32(smem) + (uint32_t)kBarBytes + (uint32_t)(group * depth * count(a)) * place(sh);
        step = count(a) * place(sh);
        here = ring;
        next = r0;
        slot = phase = 0;
        lost = false;
        if (gt == 0) {
            for (int i = 0; i < depth; ++i) tc::mbar_init(bars + i * 8, 1);
            tc::fence_mbar_init();
            int i = 0;
            if (sh.debug_flags & ROLA_DEBUG_SKIP_FIRST_K_COPY) {     // test hook: the first row is never announced nor copied
                ++next;
                ++i;
            }
#pragma unroll 1
            for (; i < depth && next < end; ++i) copy(sh, a, i);
        }
    }
    // Until row r is in its slot, or NaN.
    __device__ __forceinline__ void wait(const RnShape& sh, const RnArgs& a, long long r)
    {
        if (!tc::mbar_try_wait(bars + slot * 8, phase)) wait_longer(sh, a, r);
    }
    __device__ __forceinline__ void wait_longer(const RnShape& sh, const RnArgs& a, long long r)
    {
        if (!lost) {
            int gave_up = 0;
            if (tc::mbar_wait(bars + slot * 8, phase, &gave_up, sh.wait_limit_ns)) return;
            lost = true;
            next = end;
            int to = slot, parity = phase;
#pragma unroll 1
            for (int i = 0; i < depth; ++i) {
                gave_up = 0;
                tc::mbar_wait(bars + to * 8, parity, &gave_up, sh.wait_limit_ns / kMaxDepth);
                if (++to == depth) {
                    to = 0;
                    parity ^= 1;
                }
            }
        }
        uint32_t row = here;                             // NaN in all that this thread reads of it
#pragma unroll 1
        for (int n = 0; n < N; ++n) {
            if (!a.in[n]) continue;
            const uint32_t at = row + offset(sh, a, n, r);
#pragma unroll 1
            for (int c = gt; c < sh.d / V; c += tpr) {
                if constexpr (kWide<T, V>)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};\n" ::"r"(at + c * 16), "r"(0xffffffffu) : "memory");
                else if constexpr (V * sizeof(T) == 4)
                    asm volatile("st.shared.b32 [%0], %1;\n" ::"r"(at + c * 4), "r"(0xffffffffu) : "memory");
                else
                    asm volatile("st.shared.b16 [%0], %1;\n" ::"r"(at + c * 2), "h"((uint16_t)0xffff) : "memory");
            }
            row += place(sh);
        }
    }
    // Row r of matrix n (`skip` bytes into a slot) as fp32, zeros where there is none.
    __device__ __forceinline__ void read(const RnShape& sh, const RnArgs& a, int n, uint32_t skip, long long r,
                                         float (&v)[EL]) const
    {
        const int pieces = sh.d / V;
        const uint32_t at = here + skip + offset(sh, a, n, r);
        if (!a.in[n]) {
#pragma unroll
            for (int e = 0; e < EL; ++e) v[e] = 0.0f;
            return;
        }
#pragma unroll
        for (int i = 0; i < EL / V; ++i) {
            // past the row's end its last piece is read and cleared: no branch
            const int c = gt + i * tpr, k = FULL ? c : min(c, pieces - 1);
            if constexpr (V * sizeof(T) == 16) {
                Piece<T, V> x;
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];\n"
                             : "=r"(x.w.x), "=r"(x.w.y), "=r"(x.w.z), "=r"(x.w.w)
                             : "r"(at + k * 16)
                             : "memory");
                unpack<T, V>(x, slice<V>(v, i));
            } else if constexpr (sizeof(T) == 4) {
                asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v[i]) : "r"(at + k * 4) : "memory");
            } else if constexpr (V == 2) {
                uint32_t x;
                asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(x) : "r"(at + k * 4) : "memory");
                v[2 * i] = __uint_as_float(x << 16);
                v[2 * i + 1] = __uint_as_float(x & 0xffff0000u);
            } else {
                uint16_t x;
                asm volatile("ld.shared.u16 %0, [%1];\n" : "=h"(x) : "r"(at + k * 2) : "memory");
                v[i] = __uint_as_float((uint32_t)x << 16);
            }
        }
        clear_rest<V, FULL>(gt, tpr, pieces, v);
    }
    __device__ __forceinline__ void refill(const RnShape& sh, const RnArgs& a)       // after every thread of the group has read
    {
        if (gt == 0 && next < end) copy(sh, a, slot);
        here += step;
        if (++slot == depth) {
            slot = 0;
            here = ring;
            phase ^= 1;
        }
    }
};

template <bool WARP>
__device__ __forceinline__ void group_sync()
{
    if constexpr (WARP) __syncwarp();
    else __syncthreads();
}

// Piece `at` / V of a vector, or `none` everywhere.
template <typename T, int V>
__device__ __forceinline__ void vec_piece(const void* p, size_t at, float none, float (&v)[V])
{
    if (!p) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = none;
    } else if constexpr (sizeof(T) == 2 && V == 2) {
        const float2 x = unpack_bf16(*reinterpret_cast<const uint32_t*>(static_cast<const T*>(p) + at));
        v[0] = x.x;
        v[1] = x.y;
    } else {
        unpack<T, V>(load_piece<T, V>(static_cast<const T*>(p) + at), v);
    }
}
template <typename T, int V>
__device__ __forceinline__ void put_piece(T* p, const float (&v)[V])
{
    if constexpr (sizeof(T) == 2 && V == 2) *reinterpret_cast<uint32_t*>(p) = pack_bf16(v[0], v[1]);
    else store_piece<T, V>(p, v);
}

// Sums of N = 1, 2, 4 or 8 values over the threads of a group, the same bits in every thread.  While a lane holds more
// than one value a step hands half of them to the lane across and takes the others' (8 values take 9 shuffles, not
// 40).  The warps' sums meet in shared memory, [two buffers][value][warp], zero where there is no warp; `turn`
// alternates between the buffers, so that a sum's barrier separates its reads from the writes of the sum after the next.
struct Sums {
    float buf[2][8][32];
};
template <bool WARP, int N>
__device__ __forceinline__ void sum_group(float (&v)[N], Sums& red, int& turn)
{
    constexpr unsigned kAll = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    int off = 16;
#pragma unroll
    for (int n = N / 2; n >= 1; n >>= 1, off >>= 1) {
        const bool upper = lane & off;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float mine = upper ? v[i + n] : v[i], other = upper ? v[i] : v[i + n];
            v[i] = mine + __shfl_xor_sync(kAll, other, off);
        }
    }
    float x = v[0];                                  // of value lane / (32 / N)
#pragma unroll
    for (; off >= 1; off >>= 1) x += __shfl_xor_sync(kAll, x, off);
    constexpr int kLanes = 32 / N;
    if constexpr (!WARP) {
        float(&buf)[8][32] = red.buf[turn];
        turn ^= 1;
        if (lane % kLanes == 0) buf[lane / kLanes][threadIdx.x >> 5] = x;
        __syncthreads();
        const int warps = blockDim.x >> 5;
        if constexpr (N <= 2) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                v[n] = 0.0f;
#pragma unroll
                for (int w = 0; w < 20; w += 4)
                    if (w < warps) {
                        const float4 t = *reinterpret_cast<const float4*>(&buf[n][w]);
                        v[n] += (t.x + t.y) + (t.z + t.w);
                    }
            }
            return;
        }
        x = 0.0f;
        for (int w = lane % kLanes; w < warps; w += kLanes) x += buf[lane / kLanes][w];
#pragma unroll
        for (off = kLanes / 2; off >= 1; off >>= 1) x += __shfl_xor_sync(kAll, x, off);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = __shfl_sync(kAll, x, n * kLanes);
}
template <bool WARP>
__device__ __forceinline__ float sum_group(float a, Sums& red, int& turn)
{
    float v[1] = {a};
    sum_group<WARP, 1>(v, red, turn);
    return v[0];
}

// g, c and gate gamma_h of sample s for this thread's pieces.
template <typename T, int V, int EL, bool SHIFT, bool FULL>
__device__ __forceinline__ void load_vectors(const RnShape& sh, const RnArgs& a, int s, int gt, int tpr, int pieces,
                                             float (&g)[EL], float (&c)[EL], float (&b)[EL])
{
#pragma unroll
    for (int i = 0; i < EL / V; ++i) {
        const int p = gt + i * tpr;
        float(&gp)[V] = slice<V>(g, i), (&cp)[V] = slice<V>(c, i), (&bp)[V] = slice<V>(b, i);
        if (!FULL && p >= pieces) {
#pragma unroll
            for (int e = 0; e < V; ++e) gp[e] = cp[e] = bp[e] = 0.0f;
            continue;
        }
        const size_t at = (size_t)p * V, mod = (size_t)(s * sh.mod_stride) + at;
        float s1[V], w[V];
        vec_piece<T, V>(a.scale, mod, 0.0f, s1);
        vec_piece<T, V>(a.gamma, at, 1.0f, gp);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s1[e] += 1.0f;
            gp[e] *= s1[e];
        }
        if constexpr (SHIFT) {
            vec_piece<T, V>(a.beta, at, 0.0f, w);
            vec_piece<T, V>(a.shift, mod, 0.0f, cp);
#pragma unroll
            for (int e = 0; e < V; ++e) cp[e] = fmaf(w[e], s1[e], cp[e]);
        }
        vec_piece<T, V>(a.gate, mod, 1.0f, bp);
        vec_piece<T, V>(a.gamma_h, at, 1.0f, w);
#pragma unroll
        for (int e = 0; e < V; ++e) bp[e] *= w[e];
    }
}

// t += k v
template <int EL>
__device__ __forceinline__ void scaled_add(float (&t)[EL], const float (&v)[EL], float k)
{
    const float kk[2] = {k, k};
#pragma unroll
    for (int e = 0; e < EL; e += 2) fma2(&t[e], &v[e], kk, &t[e]);
}

// This thread's pieces of a row into `row`.
template <typename T, int V, bool FULL, int EL>
__device__ __forceinline__ void put_row(T* row, int gt, int tpr, int pieces, float (&v)[EL])
{
#pragma unroll
    for (int i = 0; i < EL / V; ++i) {
        const int p = gt + i * tpr;
        if (FULL || p < pieces) put_piece<T, V>(row + (size_t)p * V, slice<V>(v, i));
    }
}

// x / d for 1 / d rounded: the quotient's remainder once more (of a row of one value the mean is that value, as with the
// division, which takes some twenty instructions in each thread).
__device__ __forceinline__ float quotient(float x, int d, float inv_d)
{
    const float q = x * inv_d;
    return fmaf(fmaf(-q, (float)d, x), inv_d, q);
}

// v = normalised v; returns (mean, 1 / size).  `first` runs after the first barrier: every thread of the group has
// read its pieces.
template <bool WARP, int V, bool FULL, int EL, typename F>
__device__ __forceinline__ float2 normalise(int kind, int d, float inv_d, float eps, int gt, int tpr, int pieces,
                                            float (&v)[EL], Sums& red, int& turn, F first)
{
    float mu = 0.0f;
    if (kind == ROLA_NORM_LAYER) {
        float s[2] = {0.0f, 0.0f};
        sum_piece<EL>(s, v);
        mu = quotient(sum_group<WARP>(s[0] + s[1], red, turn), d, inv_d);
        first();
        fma_piece<EL>(v, v, 1.0f, -mu);
        clear_rest<V, FULL>(gt, tpr, pieces, v);
    }
    float q[2] = {0.0f, 0.0f};
    dot_piece<EL>(q, v, v);
    const float r = rsqrtf(fmaf(sum_group<WARP>(q[0] + q[1], red, turn), inv_d, eps));
    if (kind != ROLA_NORM_LAYER) first();
    fma_piece<EL>(v, v, r, 0.0f);
    return make_float2(mu, r);
}

template <typename T, int V, int EL, bool WARP, bool FULL, int TH, int MIN>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : TH, MIN)
    rn_fwd_kernel(const __grid_constant__ RnShape sh, const __grid_constant__ RnArgs a, int depth)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) Sums red;
    int turn = 0;
    if constexpr (!WARP)                                 // (the barrier in front of the rows follows)
        for (int i = threadIdx.x; i < 512; i += blockDim.x) (&red.buf[0][0][0])[i] = 0.0f;
    const int group = WARP ? threadIdx.x >> 5 : 0, part = WARP ? blockIdx.x * kWarpGroups + group : blockIdx.x;
    if (part >= a.parts) return;                         // a whole warp: no barrier of the CTA follows
    Feed<T, V, EL, 2, FULL> q;
    q.tpr = WARP ? 32 : kWide<T, V> ? (int)blockDim.x : TH;     // (small pieces: addresses are then known to the compiler)
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.depth = depth;
    q.end = rn_row(sh.total, a.parts, part + 1);
    long long r = rn_row(sh.total, a.parts, part);
    const int pieces = sh.d / V;
    const uint32_t place = q.place(sh);
    q.start(sh, a, smem, group, r);
    const float inv_d = 1.0f / (float)sh.d;
    size_t at = (size_t)r * sh.d;                        // the row's first element
    group_sync<WARP>();                                  // the mbarriers are there
#pragma unroll 1
    for (int s = (int)(r / sh.rows); r < q.end; ++s) {   // the part's samples, and their rows
        const long long stop = min(q.end, (long long)(s + 1) * sh.rows);
        float g[EL], c[EL], b[EL];
        load_vectors<T, V, EL, true, FULL>(sh, a, s, q.gt, q.tpr, pieces, g, c, b);
#pragma unroll 1
        for (; r < stop; ++r, at += sh.d) {
            q.wait(sh, a, r);
            float u[EL], hh[EL];
            q.read(sh, a, 0, 0, r, u);
            q.read(sh, a, 1, place, r, hh);
            bool held = true;
            auto refill = [&]() {
                if (!held) return;
                held = false;
                if constexpr (WARP) __syncwarp();
                q.refill(sh, a);
            };
            float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (a.h) {
                if (sh.branch != ROLA_NORM_NONE) {
                    const float2 m = normalise<WARP, V, FULL>(sh.branch, sh.d, inv_d, sh.eps, q.gt, q.tpr, pieces, hh, red, turn, refill);
                    st.z = m.x;
                    st.w = m.y;
                }
                fma_piece<EL>(u, b, hh, u);
                put_row<T, V, FULL>(static_cast<T*>(a.out) + at, q.gt, q.tpr, pieces, u);
            }
            if (sh.norm != ROLA_NORM_NONE) {
                const float2 m = normalise<WARP, V, FULL>(sh.norm, sh.d, inv_d, sh.eps, q.gt, q.tpr, pieces, u, red, turn, refill);
                st.x = m.x;
                st.y = m.y;
                fma_piece<EL>(u, u, g, c);
                put_row<T, V, FULL>(static_cast<T*>(a.y) + at, q.gt, q.tpr, pieces, u);
            }
            if (held) {
                group_sync<WARP>();
                refill();
            }
            if (a.stats && q.gt == 0) reinterpret_cast<float4*>(a.stats)[r] = st;
        }
    }
}

template <typename T, int V, int EL, bool WARP, bool FULL, int TH, int MIN>
__global__ void __launch_bounds__(WARP ? 32 * kWarpGroups : TH, MIN)
    rn_bwd_kernel(const __grid_constant__ RnShape sh, const __grid_constant__ RnArgs a, int depth)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) Sums red;
    int turn = 0;
    if constexpr (!WARP)                                 // (the barrier in front of the rows follows)
        for (int i = threadIdx.x; i < 512; i += blockDim.x) (&red.buf[0][0][0])[i] = 0.0f;
    const int group = WARP ? threadIdx.x >> 5 : 0, part = WARP ? blockIdx.x * kWarpGroups + group : blockIdx.x;
    if (part >= a.parts) return;
    const bool normed = sh.norm != ROLA_NORM_NONE;
    Feed<T, V, EL, 4, FULL> q;
    q.tpr = WARP ? 32 : kWide<T, V> ? (int)blockDim.x : TH;     // (small pieces: addresses are then known to the compiler)
    q.gt = WARP ? threadIdx.x & 31 : threadIdx.x;
    q.depth = depth;
    q.end = rn_row(sh.total, a.parts, part + 1);
    long long r = rn_row(sh.total, a.parts, part);
    q.start(sh, a, smem, group, r);
    const int pieces = sh.d / V;
    const uint32_t place = q.place(sh), k1 = a.in[0] ? place : 0, k2 = k1 + (a.in[1] ? place : 0), k3 = k2 + (a.in[2] ? place : 0);
    const float inv_d = 1.0f / (float)sh.d;
    size_t at = (size_t)r * sh.d;                        // the row's first element
    group_sync<WARP>();                                  // the mbarriers are there
    float4 st = reinterpret_cast<const float4*>(a.stats)[r];
    if (a.part) asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");       // the sums' kernel, which waits
#pragma unroll 1
    for (int s = (int)(r / sh.rows); r < q.end; ++s) {   // the part's samples, and their rows
        const long long stop = min(q.end, (long long)(s + 1) * sh.rows);
        float g[EL], b[EL], A[EL], B[EL], E[EL];
        load_vectors<T, V, EL, false, FULL>(sh, a, s, q.gt, q.tpr, pieces, g, A, b);
#pragma unroll
        for (int e = 0; e < EL; ++e) A[e] = B[e] = E[e] = 0.0f;
#pragma unroll 1
        for (; r < stop; ++r, at += sh.d) {
            const float4 now = st;
            if (r + 1 < q.end) st = reinterpret_cast<const float4*>(a.stats)[r + 1];
            q.wait(sh, a, r);
            float v[EL], hh[EL], dy[EL], t[EL];
            q.read(sh, a, 0, 0, r, v);
            q.read(sh, a, 1, k1, r, hh);
            q.read(sh, a, 2, k2, r, dy);
            q.read(sh, a, 3, k3, r, t);
            bool held = true;
            auto refill = [&]() {
                if (!held) return;
                held = false;
                if constexpr (WARP) __syncwarp();
                q.refill(sh, a);
            };
            if (sh.branch != ROLA_NORM_NONE) {
                fma_piece<EL>(hh, hh, 1.0f, -now.z);
                fma_piece<EL>(hh, hh, now.w, 0.0f);
                clear_rest<V, FULL>(q.gt, q.tpr, pieces, hh);
            }
            // With a norm behind the branch its two sums are of e = b t, t = t0 + k1 + k2 v with t0 = dout + rstd a and
            // k1, k2 known only after the sums of a and a v.  They are taken apart instead, and all sums are one step:
            //   sum e = sum b t0 + k1 sum b + k2 sum b v,  sum e hh = sum b hh t0 + k1 sum b hh + k2 sum b hh v
            float n1 = 0.0f, n2 = 0.0f;                      // mean e (layer norm), mean e hh
            if (normed) {
                float zero[EL] = {};
                fma_piece<EL>(v, b, hh, v);                  // the forward's sum, to the bit
                fma_piece<EL>(v, v, 1.0f, -now.x);
                fma_piece<EL>(v, v, now.y, 0.0f);
                clear_rest<V, FULL>(q.gt, q.tpr, pieces, v);
                fma_piece<EL>(A, dy, v, A);
                add_piece<EL>(B, dy);
                fma_piece<EL>(dy, dy, g, zero);
                scaled_add(t, dy, now.y);
                float sa[2] = {0.0f, 0.0f}, sav[2] = {0.0f, 0.0f};
                sum_piece<EL>(sa, dy);
                dot_piece<EL>(sav, dy, v);
                const bool centred = sh.norm == ROLA_NORM_LAYER, branch_centred = sh.branch == ROLA_NORM_LAYER;
                float k1, k2;
                if (sh.branch == ROLA_NORM_NONE) {
                    float sum[2] = {sa[0] + sa[1], sav[0] + sav[1]};
                    sum_group<WARP, 2>(sum, red, turn);
                    k1 = centred ? -now.y * (sum[0] * inv_d) : 0.0f;
                    k2 = -now.y * (sum[1] * inv_d);
                } else {
                    float c[2] = {0.0f, 0.0f}, cv[2] = {0.0f, 0.0f}, w[EL];      // sum b hh t0, sum b hh v
                    fma_piece<EL>(w, b, hh, zero);
                    dot_piece<EL>(c, w, t);
                    dot_piece<EL>(cv, w, v);
                    if (!centred && !branch_centred) {
                        float sum[4] = {sav[0] + sav[1], c[0] + c[1], cv[0] + cv[1], 0.0f};
                        sum_group<WARP, 4>(sum, red, turn);
                        k1 = 0.0f;
                        k2 = -now.y * (sum[0] * inv_d);
                        n2 = fmaf(k2, sum[2], sum[1]) * inv_d;
                    } else {
                        float sb[2] = {0.0f, 0.0f}, sbv[2] = {0.0f, 0.0f}, sbt[2] = {0.0f, 0.0f}, sw[2] = {0.0f, 0.0f};
                        sum_piece<EL>(sb, b);
                        dot_piece<EL>(sbv, b, v);
                        dot_piece<EL>(sbt, b, t);
                        sum_piece<EL>(sw, w);
                        float sum[8] = {sa[0] + sa[1],   sav[0] + sav[1], sbt[0] + sbt[1], sb[0] + sb[1],
                                        sbv[0] + sbv[1], c[0] + c[1],     sw[0] + sw[1],   cv[0] + cv[1]};
                        sum_group<WARP, 8>(sum, red, turn);
                        k1 = centred ? -now.y * (sum[0] * inv_d) : 0.0f;
                        k2 = -now.y * (sum[1] * inv_d);
                        n1 = branch_centred ? fmaf(k2, sum[4], fmaf(k1, sum[3], sum[2])) * inv_d : 0.0f;
                        n2 = fmaf(k2, sum[7], fmaf(k1, sum[6], sum[5])) * inv_d;
                    }
                }
                refill();
                fma_piece<EL>(v, v, k2, k1);
                add_piece<EL>(t, v);                         // k1 past the row's end, where b is 0
            } else if (sh.branch != ROLA_NORM_NONE) {
                float zero[EL] = {}, w[EL], se[2] = {0.0f, 0.0f}, seh[2] = {0.0f, 0.0f};
                fma_piece<EL>(w, b, t, zero);
                sum_piece<EL>(se, w);
                dot_piece<EL>(seh, w, hh);
                float sum[2] = {se[0] + se[1], seh[0] + seh[1]};
                sum_group<WARP, 2>(sum, red, turn);
                refill();
                n1 = sh.branch == ROLA_NORM_LAYER ? sum[0] * inv_d : 0.0f;
                n2 = sum[1] * inv_d;
            }
            if (held) {                                      // dx may be dout, of which the group has not read all yet
                group_sync<WARP>();
                refill();
            }
            fma_piece<EL>(E, t, hh, E);
            put_row<T, V, FULL>(static_cast<T*>(a.dx) + at, q.gt, q.tpr, pieces, t);
            if (a.dh) {
                float zero[EL] = {};
                fma_piece<EL>(t, t, b, zero);
                if (sh.branch != ROLA_NORM_NONE) {
                    fma_piece<EL>(hh, hh, -n2, -n1);
                    add_piece<EL>(t, hh);
                    fma_piece<EL>(t, t, now.w, 0.0f);
                }
                put_row<T, V, FULL>(static_cast<T*>(a.dh) + at, q.gt, q.tpr, pieces, t);
            }
        }
        if (a.part) {
            const int dp = rn_padded(sh.d);
            float* out = a.part + rn_slot(part, s, sh.d);
#pragma unroll
            for (int i = 0; i < EL / V; ++i) {
                const int p = (q.gt + i * q.tpr) * V;
                if (!FULL && p >= sh.d) continue;
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    const float(&x)[V] = slice<V>(n == 0 ? A : n == 1 ? B : E, i);
                    float* to = out + n * dp + p;
                    if constexpr (V >= 4) {
#pragma unroll
                        for (int e = 0; e < V; e += 4) store4(to + e, make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]));
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) to[e] = x[e];
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------- column sums to gradients

constexpr int kReduceWarps = 16;

__device__ __forceinline__ float4 operator+(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 shuffled(float4 a, int off)
{
    constexpr unsigned kAll = 0xffffffffu;
    return make_float4(__shfl_xor_sync(kAll, a.x, off), __shfl_xor_sync(kAll, a.y, off), __shfl_xor_sync(kAll, a.z, off),
                       __shfl_xor_sync(kAll, a.w, off));
}

// The vectors' gradients from the parts' sums.  A CTA takes 32 columns, four a lane, and of grid y = 0 the sums A and B, of
// 1 the sums E; grid z shares the samples out.  A warp's four groups of eight lanes and `ways` warps share the slots of a
// sample, 16 / ways samples at a time.  They meet in a fixed order, as do the samples: the same bits every time.  What
// is summed over the samples goes to `shared` [z][3][dp] where there is more than one z.
// It is launched while the rows' kernel runs and waits for it (programmatic dependent launch).
template <typename T>
__global__ void __launch_bounds__(32 * kReduceWarps) rn_reduce_kernel(const __grid_constant__ RnShape sh,
                                                                      const __grid_constant__ RnArgs a, int ways)
{
    __shared__ float4 sum[2][kReduceWarps][8];
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, quad = lane & 7;
    const int c = blockIdx.x * 32 + quad * 4, dp = rn_padded(sh.d), at_once = kReduceWarps / ways, way = w % ways;
    const bool branch = blockIdx.y + (a.norm_sums ? 0 : 1) == 1;
    const uint32_t s_begin = (uint32_t)((long long)sh.groups * blockIdx.z / gridDim.z);
    const uint32_t s_end = (uint32_t)((long long)sh.groups * (blockIdx.z + 1) / gridDim.z);
    float4 total[2] = {};                                // over the samples: of (1 + scale) A and (1 + scale) B, or of gate E
    for (uint32_t s0 = s_begin; s0 < s_end; s0 += at_once) {     // (unsigned: s may pass s_end, and with it 31 bits)
        const uint32_t s = s0 + w / ways;
        float4 x[2] = {};
        if (s < s_end && c < sh.d) {
            const int lo = rn_part(sh.total, a.parts, (long long)s * sh.rows);
            const int hi = rn_part(sh.total, a.parts, (long long)(s + 1) * sh.rows - 1);
#pragma unroll 4
            for (int i = lo + way * 4 + (lane >> 3); i <= hi; i += ways * 4) {
                const float* p = a.part + rn_slot(i, s, sh.d) + c;
                x[0] = x[0] + *reinterpret_cast<const float4*>(p + (branch ? 2 * dp : 0));
                if (!branch) x[1] = x[1] + *reinterpret_cast<const float4*>(p + dp);
            }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            x[n] = x[n] + shuffled(x[n], 8);
            x[n] = x[n] + shuffled(x[n], 16);
        }
        if (ways > 1) {
            __syncthreads();                             // the last samples' sums have been read
            if (lane < 8)
#pragma unroll
                for (int n = 0; n < 2; ++n) sum[n][w][quad] = x[n];
            __syncthreads();
            if (way == 0)
                for (int i = 1; i < ways; ++i)
#pragma unroll
                    for (int n = 0; n < 2; ++n) x[n] = x[n] + sum[n][w + i][quad];
        }
        if (way == 0 && s < s_end && lane < 8) {
            const float A[4] = {x[0].x, x[0].y, x[0].z, x[0].w}, B[4] = {x[1].x, x[1].y, x[1].z, x[1].w};
            float tA[4] = {total[0].x, total[0].y, total[0].z, total[0].w}, tB[4] = {total[1].x, total[1].y, total[1].z, total[1].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c + e >= sh.d) break;
                const size_t at = (size_t)s * sh.d + c + e, mod = (size_t)(s * sh.mod_stride + c + e);
                if (branch) {
                    if (a.dgate) a.dgate[at] = vec<T>(a.gamma_h, c + e, 1.0f) * A[e];
                    tA[e] = fmaf(vec<T>(a.gate, mod, 1.0f), A[e], tA[e]);
                } else {
                    if (a.dscale) a.dscale[at] = fmaf(vec<T>(a.gamma, c + e, 1.0f), A[e], vec<T>(a.beta, c + e, 0.0f) * B[e]);
                    if (a.dshift) a.dshift[at] = B[e];
                    const float s1 = 1.0f + vec<T>(a.scale, mod, 0.0f);
                    tA[e] = fmaf(s1, A[e], tA[e]);
                    tB[e] = fmaf(s1, B[e], tB[e]);
                }
            }
            total[0] = make_float4(tA[0], tA[1], tA[2], tA[3]);
            total[1] = make_float4(tB[0], tB[1], tB[2], tB[3]);
        }
    }
    if (!a.dgamma && !a.dbeta && !a.dgamma_h) return;
    __syncthreads();
    if (lane < 8)
#pragma unroll
        for (int n = 0; n < 2; ++n) sum[n][w][quad] = total[n];      // warps whose way is not 0 hold zeros
    __syncthreads();
    const int n = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    if (n >= (branch ? 1 : 2) || col >= sh.d) return;
    float t = 0.0f;
    for (int i = 0; i < kReduceWarps; i += ways) t += reinterpret_cast<const float*>(&sum[n][i][0])[lane];
    float* out = branch ? a.dgamma_h : n ? a.dbeta : a.dgamma;
    if (gridDim.z > 1) a.shared[((size_t)blockIdx.z * 3 + (branch ? 2 : n)) * dp + col] = t;
    else if (out) out[col] = t;
}

// dgamma, dbeta, dgamma_h from the sums over each z's samples.
__global__ void __launch_bounds__(128) rn_shared_kernel(const __grid_constant__ RnShape sh, const __grid_constant__ RnArgs a, int z)
{
    const int c = blockIdx.x * 128 + threadIdx.x, n = blockIdx.y, dp = rn_padded(sh.d);
    float* out = n == 0 ? a.dgamma : n == 1 ? a.dbeta : a.dgamma_h;
    if (c >= sh.d || !out) return;
    float t = 0.0f;
#pragma unroll 4
    for (int i = 0; i < z; ++i) t += a.shared[((size_t)i * 3 + n) * dp + c];
    out[c] = t;
}

// ---------------------------------------------------------------- dispatch

int long_grid(long long rows) { return (int)(rows < 608 ? rows : 608); }     // four CTAs on each of 152 SMs

bool wants_sums(const RnArgs& a) { return a.dgate || a.dgamma_h || a.dgamma || a.dbeta || a.dscale || a.dshift; }

constexpr int kMostParts = 4864, kMostCtas = 1216;       // of warps, of CTAs: 32 and 8 on each of 152 SMs
constexpr int kFwdRegisters = 16384, kBwdRegisters = 8192;       // longest rows held in registers (forward, single elements: 8192)

constexpr int kFewRows = 456, kFewRowsBwd = 1216;        // 3 and 8 for each of 152 SMs

// Whether every row and every vector starts at a multiple of `to` bytes.
bool starts_at(int to, const RnShape& s, const RnArgs& a, int esz)
{
    uintptr_t bits = 0;
    for (const void* p : {a.x, a.h, a.gate, a.gamma_h, a.gamma, a.beta, a.scale, a.shift, a.dout, a.dy,
                          (const void*)a.out, (const void*)a.y, (const void*)a.dx, (const void*)a.dh})
        bits |= reinterpret_cast<uintptr_t>(p);
    return (int64_t)s.d * esz % to == 0 && s.mod_stride * esz % to == 0 && (bits & (to - 1)) == 0;
}

cudaError_t sm_count(int* n)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    return cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
}

// Registers of a thread that let `ctas` CTAs of `threads` onto an SM: its four sub-partitions hold 512 of a warp's each.
constexpr int registers_of(int threads, int ctas) { return 512 / ((threads / 32 * ctas + 3) / 4) / 8 * 8; }

// Threads, parts, ring depth and shared memory of a launch.
struct Launch {
    int threads, grid, parts, depth;
    size_t smem;
};
template <typename K>
cudaError_t shape_of(K kernel, const RnShape& s, bool warp, int el, int fixed, int registers, size_t row_bytes, long long most, Launch* l)
{
    int nsm = 0;
    cudaError_t e = sm_count(&nsm);
    if (e != cudaSuccess) return e;
    const int groups = warp ? kWarpGroups : 1;
    l->threads = warp ? 32 * kWarpGroups : fixed ? fixed : ((s.d + el - 1) / el + 31) / 32 * 32;
    int ctas = 512 / registers * 4 / (l->threads / 32);
    ctas = ctas < 1 ? 1 : ctas > 8 ? 8 : ctas;
    while (ctas > 1 && groups * row_bytes * 2 * ctas > kRingBytes) --ctas;       // two rows a group at least, if they fit
    long long parts = (long long)nsm * ctas * groups;
    if (parts > s.total) parts = s.total;
    if (parts > most) parts = most;
    l->parts = (int)parts;
    l->grid = (int)((parts + groups - 1) / groups);
    const long long each = (s.total + parts - 1) / parts;
    long long n = (long long)(kRingBytes / (ctas * groups * row_bytes));
    if (n > each) n = each;
    if (n > kMaxDepth) n = kMaxDepth;
    l->depth = n < 1 ? 1 : (int)n;
    l->smem = kBarBytes + groups * l->depth * row_bytes;
    // 48 KB without asking are of static and dynamic shared memory together.  The limit is the kernel's, not the call's:
    // every call sets it to the same, since another thread may be about to launch.
    if (l->smem + sizeof(Sums) <= 48 << 10) return cudaSuccess;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kRingBytes + kBarBytes));
}

template <typename T, int V, int EL, bool WARP, int TH, int MIN, bool FULL = false>
cudaError_t fwd_one(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if constexpr (kWide<T, V> && !WARP && !FULL)
        if (s.d % (32 * EL) == 0) return fwd_one<T, V, EL, WARP, TH, MIN, true>(s, a, st);
    Launch l;
    auto kernel = rn_fwd_kernel<T, V, EL, WARP, FULL, TH, MIN>;
    const size_t row = (size_t)place_bytes(s.d, sizeof(T), kWide<T, V>) * (a.h ? 2 : 1);
    cudaError_t e = shape_of(kernel, s, WARP, EL, kWide<T, V> ? 0 : TH, registers_of(TH, MIN), row, 1ll << 30, &l);
    if (e != cudaSuccess) return e;
    a.in[0] = a.x;
    a.in[1] = a.h;
    a.parts = l.parts;
    kernel<<<l.grid, l.threads, l.smem, st>>>(s, a, l.depth);
    return cudaGetLastError();
}
template <typename T, int V, int EL, bool WARP, int TH, int MIN, bool FULL = false>
cudaError_t bwd_one(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if constexpr (kWide<T, V> && !WARP && !FULL)
        if (s.d % (32 * EL) == 0) return bwd_one<T, V, EL, WARP, TH, MIN, true>(s, a, st);
    Launch l;
    auto kernel = rn_bwd_kernel<T, V, EL, WARP, FULL, TH, MIN>;
    const int matrices = (s.norm != ROLA_NORM_NONE ? 1 : 0) + (a.h ? 1 : 0) + (a.dy ? 1 : 0) + (a.dout ? 1 : 0);
    const size_t row = (size_t)place_bytes(s.d, sizeof(T), kWide<T, V>) * matrices;
    cudaError_t e = shape_of(kernel, s, WARP, EL, kWide<T, V> ? 0 : TH, registers_of(TH, MIN), row, rn_parts(s), &l);
    if (e != cudaSuccess) return e;
    a.in[0] = s.norm != ROLA_NORM_NONE ? a.x : nullptr;
    a.in[1] = a.h;
    a.in[2] = a.dy;
    a.in[3] = a.dout;
    a.parts = l.parts;
    kernel<<<l.grid, l.threads, l.smem, st>>>(s, a, l.depth);
    return cudaGetLastError();
}

// A warp a row up to 16 elements a lane, then a CTA a row of the least whole number of warps, 16 elements a thread: with
// 8 the work that a warp does once a row counts twice (2 x 16380 x 1536: backward 133 us with 8, 118 with 16; forward
// 76 either way, 1024 wide 68 and 54).  The register limit is that of 16 warps an SM forward (12 or 10 backward).
template <typename T, int V>
cudaError_t fwd(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (s.d <= 256) return fwd_one<T, V, 8, true, 128, 6>(s, a, st);
    if (s.d <= 512) return fwd_one<T, V, 16, true, 128, 4>(s, a, st);
    if constexpr (!kWide<T, V>) {
        // Where an SM has a few rows only, it is one row's time that counts: 300 x 777 5.8 us, 8.8 with 16 elements a thread
        // (600 rows 8.8 and 9.1, in fp32 7.9 and 6.8; rows of 16-byte pieces gain nothing: 600 x 2048 5.7 and 4.5)
        if (s.total <= kFewRows && s.d <= 8 * 256) return fwd_one<T, V, 8, false, 256, 3>(s, a, st);
        // CTAs of a fixed size: 32760 x 1537 153 us, with the least number of warps 276
        if (s.d <= 16 * 64) return fwd_one<T, V, 16, false, 64, 6>(s, a, st);
        if (s.d <= 16 * 128) return fwd_one<T, V, 16, false, 128, 3>(s, a, st);
        if (s.d <= 16 * 160) return fwd_one<T, V, 16, false, 160, 2>(s, a, st);
        if (s.d <= 16 * 224) return fwd_one<T, V, 16, false, 224, 1>(s, a, st);
        if (s.d <= 16 * 320) return fwd_one<T, V, 16, false, 320, 1>(s, a, st);
    } else {
        if (s.d <= 16 * 160) return fwd_one<T, V, 16, false, 160, 3>(s, a, st);
        if (s.d <= 16 * 320) return fwd_one<T, V, 16, false, 320, 2>(s, a, st);
    }
    if (s.d <= 16 * 512) return fwd_one<T, V, 16, false, 512, 1>(s, a, st);
    if constexpr (kWide<T, V>)
        if (s.d <= kFwdRegisters) return fwd_one<T, V, 32, false, 512, 1>(s, a, st);
    rn_fwd_long_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    return cudaGetLastError();
}

template <typename T, int V>
cudaError_t bwd(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (s.d <= 256) return bwd_one<T, V, 8, true, 128, 4>(s, a, st);
    if (s.d <= 512) return bwd_one<T, V, 16, true, 128, 2>(s, a, st);
    // the same: 300 x 777 12.2 us, 14.7 with 16 elements a thread; 1200 x 1536 14.6 and 15.6 (600 and fewer alike)
    if (s.total <= kFewRowsBwd && s.d <= 8 * 256) return bwd_one<T, V, 8, false, 256, 2>(s, a, st);
    if constexpr (!kWide<T, V>) {
        if (s.d <= 16 * 64) return bwd_one<T, V, 16, false, 64, 6>(s, a, st);
        if (s.d <= 16 * 128) return bwd_one<T, V, 16, false, 128, 3>(s, a, st);
        if (s.d <= 16 * 160) return bwd_one<T, V, 16, false, 160, 2>(s, a, st);
        if (s.d <= 16 * 224) return bwd_one<T, V, 16, false, 224, 1>(s, a, st);
    }
    if (s.d <= 16 * 320) return bwd_one<T, V, 16, false, 320, 1>(s, a, st);
    if (s.d <= kBwdRegisters) return bwd_one<T, V, 16, false, 512, 1>(s, a, st);
    a.parts = rn_parts(s);
    rn_moments_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    if (a.part) rn_columns_kernel<T><<<dim3((s.d + 127) / 128, a.parts), 128, 0, st>>>(s, a);
    rn_bwd_long_kernel<T><<<long_grid(s.total), kLongThreads, 0, st>>>(s, a);
    return cudaGetLastError();
}

// f of the largest piece that every row and every vector can be taken in.
template <typename T, typename F>
cudaError_t by_piece(const RnShape& s, const RnArgs& a, F f)
{
    if (starts_at(16, s, a, sizeof(T))) return f(std::integral_constant<int, 16 / sizeof(T)>());
    if constexpr (sizeof(T) == 2)
        if (starts_at(4, s, a, 2)) return f(std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 1>());
}

template <typename T>
cudaError_t backward(const RnShape& s, RnArgs& a, cudaStream_t st)
{
    const bool sums = wants_sums(a);
    if (!sums) a.part = nullptr;
    cudaError_t e = by_piece<T>(s, a, [&](auto v) { return bwd<T, decltype(v)::value>(s, a, st); });
    if (e != cudaSuccess || !sums) return e;
    a.norm_sums = a.dgamma || a.dbeta || a.dscale || a.dshift;
    const bool branch_sums = a.dgate || a.dgamma_h, shared = a.dgamma || a.dbeta || a.dgamma_h;
    int ways = kReduceWarps;
    while (ways > 1 && (int64_t)ways * s.groups > kReduceWarps) ways /= 2;
    const int z = rn_shares(s), columns = (s.d + 31) / 32;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(columns, a.norm_sums && branch_sums ? 2 : 1, z);
    cfg.blockDim = dim3(32 * kReduceWarps);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, rn_reduce_kernel<T>, s, static_cast<const RnArgs&>(a), ways);
    if (e != cudaSuccess || z == 1 || !shared) return e;
    rn_shared_kernel<<<dim3((s.d + 127) / 128, 3), 128, 0, st>>>(s, a, z);
    return cudaGetLastError();
}

}  // namespace

int rn_parts(const RnShape& s)
{
    const long long want = (s.total + 1) / 2, most = s.d <= 512 ? kMostParts : kMostCtas;
    return (int)(want < most ? want : most);
}

int rn_shares(const RnShape& s)
{
    // 32 samples a share at least, and some 4000 CTAs at most
    const int64_t columns = (s.d + 31) / 32, most = (4096 + columns - 1) / columns, want = ((int64_t)s.groups + 31) / 32;
    return (int)(want < most ? want : most);
}

bool rn_long(const RnShape& s) { return s.d > kBwdRegisters; }

cudaError_t launch_residual_norm(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st)
{
    if (dt == ROLA_BF16)
        return by_piece<__nv_bfloat16>(s, a, [&](auto v) { return fwd<__nv_bfloat16, decltype(v)::value>(s, a, st); });
    return by_piece<float>(s, a, [&](auto v) { return fwd<float, decltype(v)::value>(s, a, st); });
}

cudaError_t launch_residual_norm_backward(rola_dtype_t dt, const RnShape& s, RnArgs& a, cudaStream_t st)
{
    return dt == ROLA_BF16 ? backward<__nv_bfloat16>(s, a, st) : backward<float>(s, a, st);
}

}  // namespace rola
