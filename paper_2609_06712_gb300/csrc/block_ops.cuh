// Shared by the block operators around the module: layer norm, gated
// feed-forward and dense attention.
#pragma once

#include "common.cuh"

namespace rola {

// ---------------------------------------------------------------- element types

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x)
{
    if constexpr (sizeof(T) == 4) return x;
    else return __float2bfloat16_rn(x);
}

// 16 bytes at a 16-byte aligned address <-> fp32 values
__device__ __forceinline__ void load16(const float* p, float (&x)[4])
{
    const float4 u = *reinterpret_cast<const float4*>(p);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
}
__device__ __forceinline__ void load16(const __nv_bfloat16* p, float (&x)[8])
{
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack_bf16(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void store16(float* p, const float (&x)[4])
{
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&x)[8])
{
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
// four values at p (16-byte aligned for fp32, 8-byte for bf16)
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p)
{
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    const float2 a = unpack_bf16(u.x), b = unpack_bf16(u.y);
    return make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void store4(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 x)
{
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}

// ---------------------------------------------------------------- feature maps

// phi(g) and phi'(g) of the gate, from CUDA's expf / tanhf / erfcf (gelu is g Phi(g) with
// Phi(g) = erfc(-g / sqrt 2) / 2, which keeps its digits for negative g).  For
// silu, s = sigmoid(g): phi = g s, phi' = s (1 + g (1 - s)); g s is 0, not NaN, where s underflows.
__device__ __forceinline__ float gate_act(int kind, float g)
{
    switch (kind) {
        case ROLA_LOWRANK_ACT_SILU: return g / (1.0f + expf(-g));
        case ROLA_LOWRANK_ACT_IDENTITY: return g;
        case ROLA_LOWRANK_ACT_TANH: return tanhf(g);
        case ROLA_LOWRANK_ACT_RELU: return g <= 0.0f ? 0.0f : g;         // (fmaxf would make a NaN 0)
        default: return 0.5f * g * erfcf(g * -0.7071067811865476f);
    }
}
__device__ __forceinline__ void gate_act_grad(int kind, float g, float& a, float& da)
{
    switch (kind) {
        case ROLA_LOWRANK_ACT_SILU: {
            const float s = 1.0f / (1.0f + expf(-g));
            a = g * s;
            da = fmaf(a, 1.0f - s, s);
            return;
        }
        case ROLA_LOWRANK_ACT_IDENTITY: a = g; da = 1.0f; return;
        case ROLA_LOWRANK_ACT_TANH: a = tanhf(g); da = fmaf(-a, a, 1.0f); return;
        case ROLA_LOWRANK_ACT_RELU:
            a = g <= 0.0f ? 0.0f : g;
            da = g > 0.0f ? 1.0f : a;                                    // 0, or NaN
            return;
        default: {
            const float cdf = 0.5f * erfcf(g * -0.7071067811865476f);
            a = g * cdf;
            da = fmaf(g * 0.3989422804014327f, expf(-0.5f * g * g), cdf);
            return;
        }
    }
}

// The same for results that are rounded to bf16, one type per map, so that the choice is made once for a
// whole loop and not once per element.  The fast exponential is documented within 2 + 1.173 |g| units in the last
// place and the quotient within 2, so silu is within (4 + 1.2 |g|) 2^-23 of its value: 2^-19 up to |g| = 10,
// 2^-16 at 80, where bf16's rounding is 2^-9.
struct FastSilu {
    static __device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }
    static __device__ __forceinline__ float phi(float g) { return g * sigmoid(g); }
    static __device__ __forceinline__ void grad(float g, float& a, float& da)
    {
        const float s = sigmoid(g);
        a = g * s;
        da = fmaf(a, 1.0f - s, s);
    }
};
template <int KIND>
struct PlainAct {
    static __device__ __forceinline__ float phi(float g) { return gate_act(KIND, g); }
    static __device__ __forceinline__ void grad(float g, float& a, float& da) { gate_act_grad(KIND, g, a, da); }
};
template <typename F>
__device__ __forceinline__ void with_act(int kind, F f)
{
    switch (kind) {
        case ROLA_LOWRANK_ACT_SILU: f(FastSilu()); break;
        case ROLA_LOWRANK_ACT_IDENTITY: f(PlainAct<ROLA_LOWRANK_ACT_IDENTITY>()); break;
        case ROLA_LOWRANK_ACT_TANH: f(PlainAct<ROLA_LOWRANK_ACT_TANH>()); break;
        case ROLA_LOWRANK_ACT_RELU: f(PlainAct<ROLA_LOWRANK_ACT_RELU>()); break;
        default: f(PlainAct<ROLA_LOWRANK_ACT_GELU>()); break;
    }
}

// ---------------------------------------------------------------- feed-forward

struct FfnShape {
    int M, D, F, act;            // tokens, d_model, d_ff
    uint64_t wait_limit_ns;
    int debug_flags;
};

// ---------------------------------------------------------------- attention

// One key head of one batch element is a head here: the G = H / H_kv query
// heads that read it are G Lq consecutive rows of q, and row r is query r mod Lq.
struct AttnShape {
    int B, H, Hk, Lq, Lk, R;     // R = (H / Hk) Lq rows per key head
    int heads;                   // B Hk
    int causal;
    float scale, scale_log2;     // of the scores, and times log2 e
    int splits;                  // parts of the key axis forward (1: none)
    int splits_dq, splits_dkv;   // bf16 backward: of the key axis for dq, of the row axis for dk and dv
    uint64_t wait_limit_ns;
    int debug_flags;
};

// Keys of batch element b.
__device__ __forceinline__ int attn_len(const AttnShape& s, const int32_t* __restrict__ kv_len, int b)
{
    return kv_len ? min(max(__ldg(kv_len + b), 0), s.Lk) : s.Lk;
}
// Keys that row r sees, out of len.
__device__ __forceinline__ int attn_seen(const AttnShape& s, int len, int r)
{
    if (!s.causal) return len;
    return min(max(r % s.Lq + len - s.Lq + 1, 0), len);
}
// The most and the fewest keys that the rows r0 .. r1 see (r0 <= r1 < R).
__device__ __forceinline__ int attn_seen_most(const AttnShape& s, int len, int r0, int r1)
{
    if (!s.causal || r0 / s.Lq != r1 / s.Lq) return len;      // a range that wraps holds some last query
    return attn_seen(s, len, r1);
}
__device__ __forceinline__ int attn_seen_least(const AttnShape& s, int len, int r0, int r1)
{
    if (!s.causal) return len;
    return r0 / s.Lq != r1 / s.Lq ? attn_seen(s, len, 0) : attn_seen(s, len, r0);
}

// Tensors of one attention call.  Forward writes o and lse, or with splits the
// parts: part_o [splits][heads R][128] (each part's own softmax average) and
// part_lse [splits][heads R].
struct AttnArgs {
    const void *q, *k, *v, *dO, *o_in;
    const int32_t* kv_len;
    void *o, *dq, *dk, *dv;
    float *lse, *part_o, *part_lse;
    float *part_dq, *part_dk, *part_dv;      // backward with splits: [splits][heads][rows or keys][128]
    const float* lse_in;
    float* D;                    // rowsum(dO o), [heads R]
    DeviceStatus* status;
};

// ---------------------------------------------------------------- host side

size_t layer_norm_backward_scratch(long long rows, int d);     // bytes
cudaError_t launch_layer_norm(rola_dtype_t dt, long long rows, int d, const void* x, const void* gamma,
                              const void* beta, float eps, void* y, float* mean, float* rstd, cudaStream_t st);
cudaError_t launch_layer_norm_backward(rola_dtype_t dt, long long rows, int d, const void* x, const void* gamma,
                                       const float* mean, const float* rstd, const void* dy, void* dx, float* dgamma,
                                       float* dbeta, float* part, cudaStream_t st);

// H = phi(X Wg^T) * (X Wu^T), G and U kept where given (both or neither): fp32, bf16 (tensor cores)
cudaError_t launch_ffn_up_simt(const FfnShape& s, const void* X, const void* Wg, const void* Wu, void* H, float* G,
                               float* U, cudaStream_t st);
cudaError_t launch_ffn_up_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, void* H, float* G,
                             float* U, DeviceStatus* status, cudaStream_t st);
// Y = H Wd^T
cudaError_t launch_ffn_down_simt(const FfnShape& s, const void* H, const void* Wd, void* Y, cudaStream_t st);
cudaError_t launch_ffn_down_tc(const FfnShape& s, const void* H, const void* Wd, void* Y, DeviceStatus* status,
                               cudaStream_t st);
// Few tokens: both products of the forward (and G, U where given); H, dG, dU and dX of the backward.
constexpr int kFfnFewTokens = 96;    // of one tile; the backward's form up to there
bool ffn_few(const FfnShape& s);     // whether it is the forward's form for these sizes
cudaError_t launch_ffn_few(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd, void* H,
                           float* G, float* U, void* Y, DeviceStatus* status, cudaStream_t st);
cudaError_t launch_ffn_few_grad(const FfnShape& s, const void* Wg, const void* Wu, const void* Wd, const float* G,
                                const float* U, const void* dY, void* H, void* dG, void* dU, void* dX,
                                DeviceStatus* status, cudaStream_t st);
// dG, dU, H from dY Wd, G and U; then the four gradients
cudaError_t launch_ffn_backward_simt(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd,
                                     const float* G, const float* U, const void* dY, void* H, void* dG, void* dU,
                                     void* dX, void* dWg, void* dWu, void* dWd, cudaStream_t st);
cudaError_t launch_ffn_backward_tc(const FfnShape& s, const void* X, const void* Wg, const void* Wu, const void* Wd,
                                   const float* G, const float* U, const void* dY, void* H, void* dG, void* dU,
                                   void* dX, void* dWg, void* dWu, void* dWd, DeviceStatus* status, cudaStream_t st);

// o and lse, or the parts of a split key axis: fp32, bf16 (tensor cores)
cudaError_t launch_attention_simt(const AttnShape& s, const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attention_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st);
// o and lse from the parts
template <typename T>
cudaError_t launch_attention_join(const AttnShape& s, const AttnArgs& a, cudaStream_t st);
// D = rowsum(dO o)
template <typename T>
cudaError_t launch_attention_rowdot(const AttnShape& s, const AttnArgs& a, cudaStream_t st);
// dq, dk, dv from D
cudaError_t launch_attention_backward_simt(const AttnShape& s, const AttnArgs& a, cudaStream_t st);
cudaError_t launch_attention_backward_tc(const AttnShape& s, const AttnArgs& a, cudaStream_t st);

}  // namespace rola
