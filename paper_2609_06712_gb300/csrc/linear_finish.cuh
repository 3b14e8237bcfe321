// From the sums of a linear layer's product to its outputs: bias, Z, phi, residual, one rounding to bf16.
#pragma once

#include "block_ops.cuh"

namespace rola {

struct LinearEnd {
    __nv_bfloat16* c;
    const __nv_bfloat16 *bias, *residual;        // or NULL
    float* Z;                                    // or NULL
    int act;
};

inline LinearEnd linear_end_of(void* c, const void* bias, const void* residual, float* Z, int act)
{
    LinearEnd e;
    e.c = static_cast<__nv_bfloat16*>(c);
    e.bias = static_cast<const __nv_bfloat16*>(bias);
    e.residual = static_cast<const __nv_bfloat16*>(residual);
    e.Z = Z;
    e.act = act;
    return e;
}

// GELU of bf16 layers, two values at a time.  With u = |z|, x = u / sqrt 2 and erfcx(x) = e^(x^2) erfc(x):
//   tail = Phi(-u) = erfcx(x) e^(-z^2 / 2) / 2,  gelu(z) = max(z, 0) - u tail,  gelu'(z) = Phi(z) + z e^(-z^2 / 2) / sqrt(2 pi)
// u is held at 16, past which the tail underflows.  max(z, 0) is z / 2 + |z / 2| (exact but in odd subnormals), so that
// z = -inf gives NaN in every form of the layer, as the definition z Phi(z) = -inf * 0 does (and gelu' at both infinities).
// erfcx is t P(t), t = 1 / (1 + 0.44 x): P of degree 7 fitted here to the least relative error over 0 <= x <= 10 (2e-7, with
// fp32's roundings 5e-7), beyond which the tail is 0 beside any z.  One exponential serves both; its argument's rounding adds
// 2^-23 z^2 relative to the tail.  About 11 instructions a value, where erfcf takes some 45: of the feed-forward's
// first layer at 8190 x 1536 x 6144 the epilogue took longer than its tile's products.
struct FastGelu {
    static __device__ __forceinline__ void fma2(float (&d)[2], const float (&a)[2], const float (&b)[2], const float (&c)[2])
    {
        asm("{\n.reg .b64 ra, rb, rc;\nmov.b64 ra, {%2, %3};\nmov.b64 rb, {%4, %5};\nmov.b64 rc, {%6, %7};\n"
            "fma.rn.f32x2 ra, ra, rb, rc;\nmov.b64 {%0, %1}, ra;\n}\n"
            : "=f"(d[0]), "=f"(d[1]) : "f"(a[0]), "f"(a[1]), "f"(b[0]), "f"(b[1]), "f"(c[0]), "f"(c[1]));
    }
    static __device__ __forceinline__ void fma2(float (&d)[2], const float (&a)[2], const float (&b)[2], float c)
    {
        const float cc[2] = {c, c};
        fma2(d, a, b, cc);
    }
    // u = min(|z|, 16), tail = Phi(-u) and e = e^(-z^2 / 2) of two values
    static __device__ __forceinline__ void parts(const float (&z)[2], float (&u)[2], float (&tail)[2], float (&e)[2])
    {
        float t[2], s[2], r[2];
        const float p[2] = {0.44f * 0.70710678f, 0.44f * 0.70710678f}, c[2] = {-0.72134752f, -0.72134752f};
#pragma unroll
        for (int i = 0; i < 2; ++i) u[i] = fminf(fabsf(z[i]), 16.0f);
        fma2(t, u, p, 1.0f);
        fma2(s, u, c, 0.0f);
        fma2(s, s, u, 0.0f);                             // -z^2 log2(e) / 2
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t[i]) : "f"(t[i]));
            asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e[i]) : "f"(s[i]));
        }
        // P / 2
        r[0] = r[1] = 0.5f * 0.07122340798377991f;
        fma2(r, r, t, 0.5f * -0.2779477834701538f);
        fma2(r, r, t, 0.5f * 0.29668712615966797f);
        fma2(r, r, t, 0.5f * -0.02018037997186184f);
        fma2(r, r, t, 0.5f * 0.2158121019601822f);
        fma2(r, r, t, 0.5f * 0.21731358766555786f);
        fma2(r, r, t, 0.5f * 0.24887117743492126f);
        fma2(r, r, t, 0.5f * 0.24822095036506653f);
        fma2(r, r, t, 0.0f);
        fma2(tail, r, e, 0.0f);
    }
    static __device__ __forceinline__ void phi(float (&z)[2])
    {
        float u[2], tail[2], e[2], top[2];
        const float half[2] = {0.5f, 0.5f};
        parts(z, u, tail, e);
        fma2(top, z, half, 0.0f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] += fabsf(top[i]);
            u[i] = -u[i];
        }
        fma2(z, u, tail, top);
    }
    // z = gelu'(z)
    static __device__ __forceinline__ void slope(float (&z)[2])
    {
        float u[2], tail[2], e[2], cdf[2];
        parts(z, u, tail, e);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            cdf[i] = z[i] < 0.0f ? tail[i] : 1.0f - tail[i];
            e[i] *= 0.3989422804014327f;
        }
        fma2(z, z, e, cdf);
    }
};

// v = phi(v) of a bf16 layer
template <int W>
__device__ __forceinline__ void linear_phi(int kind, float (&v)[W])
{
    if (kind == ROLA_LOWRANK_ACT_IDENTITY) return;
    if (kind == ROLA_LOWRANK_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < W; j += 2) FastGelu::phi(*reinterpret_cast<float(*)[2]>(&v[j]));
        return;
    }
    with_act(kind, [&](auto act) {
#pragma unroll
        for (int j = 0; j < W; ++j) v[j] = act.phi(v[j]);
    });
}

// The end of a product whose K axis was split: the parts [splits][M][N], added in order.
cudaError_t launch_linear_join(const LinearEnd& end, const float* part, int splits, int M, int N, cudaStream_t st);

}  // namespace rola
