// C ABI entry points of the block operators in include/rola.h (layer norm,
// gated feed-forward, linear layer, dense attention, residual norm): validation,
// workspace layout, launches.
#include <limits.h>
#include <math.h>
#include <string.h>

#include "block_ops.cuh"
#include "linear.cuh"
#include "residual_norm.cuh"

using namespace rola;

namespace {

constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

template <typename... P>
bool aligned(size_t to, P... p)
{
    return (((reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0) && ...);
}

template <typename T>
T* at(void* ws, size_t off) { return reinterpret_cast<T*>(static_cast<uint8_t*>(ws) + off); }

size_t elem(rola_dtype_t dt) { return dt == ROLA_BF16 ? 2 : 4; }

rola_status_t check_ws(const void* ws, size_t have, size_t need)
{
    return !ws || !aligned(kAlign, ws) || have < need ? ROLA_ERR_WORKSPACE : ROLA_OK;
}

#define ROLA_TRY(expr)                                  \
    do {                                                \
        cudaError_t e_ = (expr);                        \
        if (e_ != cudaSuccess) return ROLA_ERR_CUDA;    \
    } while (0)

#define ROLA_CHECK(expr)                                \
    do {                                                \
        rola_status_t st_ = (expr);                     \
        if (st_ != ROLA_OK) return st_;                 \
    } while (0)

uint64_t wait_limit_ns(int32_t ms) { return (uint64_t)(ms > 0 ? ms : 2000) * 1000000ull; }

// ---------------------------------------------------------------- layer norm

rola_status_t validate_norm(int64_t rows, int32_t d, rola_dtype_t dt)
{
    if (rows < 1 || d < 1 || (dt != ROLA_BF16 && dt != ROLA_FP32)) return ROLA_ERR_INVALID_ARG;
    if (d > (1 << 20) || rows > ((int64_t)1 << 40) / d) return ROLA_ERR_UNSUPPORTED;
    return ROLA_OK;
}

// ---------------------------------------------------------------- feed-forward

rola_status_t validate(const rola_ffn_config_t* c)
{
    if (!c || c->tokens < 1 || c->d_model < 8 || c->d_ff < 8 || c->d_model % 8 || c->d_ff % 8)
        return ROLA_ERR_INVALID_ARG;
    if (c->dtype != ROLA_BF16 && c->dtype != ROLA_FP32) return ROLA_ERR_INVALID_ARG;
    if (c->act < ROLA_LOWRANK_ACT_SILU || c->act > ROLA_LOWRANK_ACT_GELU) return ROLA_ERR_INVALID_ARG;
    if (c->wait_limit_ms < 0 || c->wait_limit_ms > 60000) return ROLA_ERR_INVALID_ARG;
    if (c->debug_flags & ~ROLA_DEBUG_SKIP_FIRST_K_COPY) return ROLA_ERR_INVALID_ARG;
    // grid limits of the kernels (65535 tiles of 128 tokens)
    if (c->tokens > (1 << 22) || c->d_model > (1 << 20) || c->d_ff > (1 << 20)) return ROLA_ERR_UNSUPPORTED;
    return ROLA_OK;
}

FfnShape make_shape(const rola_ffn_config_t& c)
{
    return {c.tokens, c.d_model, c.d_ff, c.act, wait_limit_ns(c.wait_limit_ms), c.debug_flags};
}

struct FfnWorkspace {
    size_t status, H, dG, dU, total;
};
FfnWorkspace ffn_layout(const rola_ffn_config_t& c, bool backward)
{
    const size_t act = elem(c.dtype) * (size_t)c.tokens * c.d_ff;
    FfnWorkspace w;
    size_t off = 0;
    w.status = off; off = align_up(off + sizeof(DeviceStatus));
    w.H = off; off = align_up(off + act);
    w.dG = off; off = align_up(off + (backward ? act : 0));
    w.dU = off; off = align_up(off + (backward ? act : 0));
    w.total = off;
    return w;
}

rola_status_t ffn_forward(const rola_ffn_config_t* cfg, const void* X, const void* Wg, const void* Wu, const void* Wd,
                          void* Y, float* G, float* U, void* ws, size_t ws_bytes, void* stream)
{
    if (!X || !Wg || !Wu || !Wd || !Y || !aligned(16, X, Wg, Wu, Wd, Y, G, U)) return ROLA_ERR_INVALID_ARG;
    const FfnWorkspace w = ffn_layout(*cfg, false);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const FfnShape s = make_shape(*cfg);
    void* H = at<void>(ws, w.H);
    ROLA_TRY(cudaMemsetAsync(at<uint8_t>(ws, w.status), 0, sizeof(DeviceStatus), st));
    if (cfg->dtype == ROLA_BF16 && ffn_few(s)) {
        ROLA_TRY(launch_ffn_few(s, X, Wg, Wu, Wd, H, G, U, Y, at<DeviceStatus>(ws, w.status), st));
    } else if (cfg->dtype == ROLA_BF16) {
        ROLA_TRY(launch_ffn_up_tc(s, X, Wg, Wu, H, G, U, at<DeviceStatus>(ws, w.status), st));
        ROLA_TRY(launch_ffn_down_tc(s, H, Wd, Y, at<DeviceStatus>(ws, w.status), st));
    } else {
        ROLA_TRY(launch_ffn_up_simt(s, X, Wg, Wu, H, G, U, st));
        ROLA_TRY(launch_ffn_down_simt(s, H, Wd, Y, st));
    }
    return ROLA_OK;
}

// ---------------------------------------------------------------- linear

rola_status_t validate(const rola_linear_config_t* c)
{
    if (!c || c->tokens < 1 || c->d_in < 8 || c->d_out < 8 || c->d_in % 8 || c->d_out % 8) return ROLA_ERR_INVALID_ARG;
    if (c->dtype != ROLA_BF16 && c->dtype != ROLA_FP32) return ROLA_ERR_INVALID_ARG;
    if (c->act < ROLA_LOWRANK_ACT_SILU || c->act > ROLA_LOWRANK_ACT_GELU) return ROLA_ERR_INVALID_ARG;
    if (c->wait_limit_ms < 0 || c->wait_limit_ms > 60000) return ROLA_ERR_INVALID_ARG;
    if (c->debug_flags & ~ROLA_DEBUG_SKIP_FIRST_K_COPY) return ROLA_ERR_INVALID_ARG;
    if (c->tokens > (1 << 22) || c->d_in > (1 << 20) || c->d_out > (1 << 20)) return ROLA_ERR_UNSUPPORTED;
    return ROLA_OK;
}

LinShape make_shape(const rola_linear_config_t& c)
{
    return {c.tokens, c.d_in, c.d_out, c.act, wait_limit_ns(c.wait_limit_ms), c.debug_flags};
}

// The form of a bf16 layer's forward pass, and of its dX.
enum LinearForm { kLinearByRows, kLinearFew, kLinearTiles };
LinearForm linear_form(const LinShape& s)
{
    return linear_by_rows(s) ? kLinearByRows : linear_few(s) ? kLinearFew : kLinearTiles;
}
LinearForm linear_dx_form(const LinShape& s) { return s.M <= kFfnFewTokens ? kLinearFew : kLinearTiles; }

struct LinWorkspace {
    size_t status, dZ, sums, part, total;
};
LinWorkspace linear_layout(const rola_linear_config_t& c, bool backward)
{
    const LinShape s = make_shape(c);
    const bool dz = backward && c.act != ROLA_LOWRANK_ACT_IDENTITY;      // else dZ is dY
    size_t part = 0;                             // of a split K axis, of one product at a time
    if (c.dtype == ROLA_BF16 && !backward && linear_form(s) == kLinearTiles) part = linear_part_bytes(s.M, s.N, s.K);
    if (c.dtype == ROLA_BF16 && backward) {
        const size_t dx = linear_dx_form(s) == kLinearTiles ? linear_part_bytes(s.M, s.K, s.N) : 0;
        const size_t dw = linear_part_bytes(s.N, s.K, s.M);
        part = dx > dw ? dx : dw;
    }
    LinWorkspace w;
    size_t off = 0;
    w.status = off; off = align_up(off + sizeof(DeviceStatus));
    w.dZ = off; off = align_up(off + (dz ? elem(c.dtype) * (size_t)s.M * s.N : 0));
    w.sums = off; off = align_up(off + (backward ? 4 * (size_t)linear_grad_parts(s) * s.N : 0));
    w.part = off; off = align_up(off + part);
    w.total = off;
    return w;
}

// Whether the output p starts where one of the others does.  (A CTA would read there what another has written.)
template <typename... Q>
bool same_start(const void* p, Q... others)
{
    return p && ((p == static_cast<const void*>(others)) || ...);
}

rola_status_t linear_forward(const rola_linear_config_t* cfg, const void* X, const void* W, const void* b, const void* R,
                             void* Y, float* Z, void* ws, size_t ws_bytes, void* stream)
{
    if (!X || !W || !Y || !aligned(16, X, W, b, R, Y, Z)) return ROLA_ERR_INVALID_ARG;
    const LinWorkspace w = linear_layout(*cfg, false);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    if (same_start(Y, X, W, b, Z, ws) || same_start(Z, X, W, b, R, ws)) return ROLA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    DeviceStatus* status = at<DeviceStatus>(ws, w.status);
    const LinShape s = make_shape(*cfg);
    if (cfg->dtype == ROLA_FP32) {
        ROLA_TRY(cudaMemsetAsync(status, 0, sizeof(DeviceStatus), st));
        ROLA_TRY(launch_linear_simt(s, X, W, b, R, Y, Z, st));
        return ROLA_OK;
    }
    switch (linear_form(s)) {
        case kLinearByRows: ROLA_TRY(launch_linear_rows(s, X, W, b, R, Y, Z, status, st)); break;
        case kLinearFew: ROLA_TRY(launch_linear_few(s, X, W, b, R, Y, Z, status, st)); break;
        default: ROLA_TRY(launch_linear_tc(s, X, W, b, R, Y, Z, at<float>(ws, w.part), status, st));
    }
    return ROLA_OK;
}

// ---------------------------------------------------------------- attention

rola_status_t validate(const rola_attention_config_t* c)
{
    if (!c || c->B < 1 || c->H < 1 || c->H_kv < 1 || c->Lq < 1 || c->Lk < 1 || c->H % c->H_kv)
        return ROLA_ERR_INVALID_ARG;
    if (c->d_h != kDh) return c->d_h > 0 ? ROLA_ERR_UNSUPPORTED : ROLA_ERR_INVALID_ARG;
    if (c->causal != 0 && c->causal != 1) return ROLA_ERR_INVALID_ARG;
    if (!isfinite(c->scale) || c->scale < 0.0f) return ROLA_ERR_INVALID_ARG;
    if (c->dtype != ROLA_BF16 && c->dtype != ROLA_FP32) return ROLA_ERR_INVALID_ARG;
    if (c->wait_limit_ms < 0 || c->wait_limit_ms > 60000) return ROLA_ERR_INVALID_ARG;
    if (c->debug_flags & ~ROLA_DEBUG_SKIP_FIRST_K_COPY) return ROLA_ERR_INVALID_ARG;
    // grid and index limits of the kernels: heads on a grid axis, rows and keys of a head in 30 bits, all
    // (head, row tile) and (head, key tile) items in 31
    const int64_t heads = (int64_t)c->B * c->H_kv, R = (int64_t)(c->H / c->H_kv) * c->Lq;
    if (heads > 65535 || R > (1 << 30) || c->Lk > (1 << 30)) return ROLA_ERR_UNSUPPORTED;
    if (heads * ((R + 63) / 64 + 1) > (1 << 28) || heads * (((int64_t)c->Lk + 63) / 64) > (1 << 28))
        return ROLA_ERR_UNSUPPORTED;
    return ROLA_OK;
}

// Parts of an axis of `tiles` tiles, for `items` items without splitting.  One
// CTA runs on each of 152 SMs, so `items` items in n parts take
// ceil(items n / 152) turns of tiles / n steps; with parts, their `bytes` (of fp32
// output, each) are written and read once more at some 5 TB/s, and the second
// kernel costs 4 us.  step_us: a step's measured time.  The n of least cost is
// taken, among those whose parts keep two tiles at least.
int attn_splits(int64_t items, int64_t tiles, double step_us, double bytes)
{
    constexpr int64_t kSMs = 152;
    auto cost = [&](int64_t n) {
        const double turns = (double)((items * n + kSMs - 1) / kSMs);
        return turns * (double)tiles / (double)n * step_us + (n > 1 ? (double)n * 2.0 * bytes / 5e6 + 4.0 : 0.0);
    };
    int64_t best = 1;
    for (int64_t n = 2; n <= tiles / 2 && n <= kSMs; ++n)
        if (cost(n) < cost(best)) best = n;
    return (int)best;
}

AttnShape make_shape(const rola_attention_config_t& c)
{
    AttnShape s;
    s.B = c.B; s.H = c.H; s.Hk = c.H_kv; s.Lq = c.Lq; s.Lk = c.Lk;
    s.R = c.H / c.H_kv * c.Lq;
    s.heads = c.B * c.H_kv;
    s.causal = c.causal;
    const double scale = c.scale > 0.0f ? (double)c.scale : 1.0 / sqrt((double)kDh);
    s.scale = (float)scale;
    s.scale_log2 = (float)(scale * 1.4426950408889634);
    auto tiles = [](int64_t n, int of) { return (n + of - 1) / of; };
    const double rows = 4.0 * kDh * s.heads * s.R, keys = 4.0 * kDh * s.heads * s.Lk;
    const double part = s.causal ? 0.5 : 1.0;    // of the tiles that a row sees
    if (c.dtype == ROLA_BF16) {          // items of 256 rows forward, of 128 rows or keys backward; tiles of 128
        s.splits = attn_splits(s.heads * tiles(s.R, 256), tiles(s.Lk, 128), 1.7 * part, rows);
        s.splits_dq = attn_splits(s.heads * tiles(s.R, 128), tiles(s.Lk, 128), 1.0 * part, rows);
        s.splits_dkv = attn_splits(s.heads * tiles(s.Lk, 128), tiles(s.R, 128), 1.3 * part, 2.0 * keys);
    } else {
        s.splits = attn_splits(s.heads * tiles(s.R, 64), tiles(s.Lk, 64), 8.0 * part, rows);
        s.splits_dq = s.splits_dkv = 1;
    }
    s.wait_limit_ns = wait_limit_ns(c.wait_limit_ms);
    s.debug_flags = c.debug_flags;
    return s;
}

struct AttnWorkspace {
    size_t status, part_o, part_lse, D, part_dq, part_dk, part_dv, total;
};
AttnWorkspace attn_layout(const AttnShape& s, bool backward)
{
    const size_t rows = (size_t)s.heads * s.R, parts = !backward && s.splits > 1 ? s.splits : 0;
    AttnWorkspace w;
    size_t off = 0;
    w.status = off; off = align_up(off + sizeof(DeviceStatus));
    w.part_o = off; off = align_up(off + 4 * parts * rows * kDh);
    w.part_lse = off; off = align_up(off + 4 * parts * rows);
    w.D = off; off = align_up(off + (backward ? 4 * rows : 0));
    const size_t dq = backward && s.splits_dq > 1 ? 4 * s.splits_dq * rows * kDh : 0;
    const size_t dkv = backward && s.splits_dkv > 1 ? 4 * (size_t)s.splits_dkv * s.heads * s.Lk * kDh : 0;
    w.part_dq = off; off = align_up(off + dq);
    w.part_dk = off; off = align_up(off + dkv);
    w.part_dv = off; off = align_up(off + dkv);
    w.total = off;
    return w;
}

// ---------------------------------------------------------------- residual norm

bool norm_kind(int n) { return n == ROLA_NORM_NONE || n == ROLA_NORM_LAYER || n == ROLA_NORM_RMS; }

rola_status_t validate(const rola_residual_norm_config_t* c)
{
    if (!c || c->groups < 1 || c->rows < 1 || c->d < 1 || !norm_kind(c->norm) || !norm_kind(c->branch_norm))
        return ROLA_ERR_INVALID_ARG;
    if (c->mod_stride != 0 && c->mod_stride < c->d) return ROLA_ERR_INVALID_ARG;
    if (!(c->eps >= 0.0f) || !isfinite(c->eps) || (c->dtype != ROLA_BF16 && c->dtype != ROLA_FP32))
        return ROLA_ERR_INVALID_ARG;
    if (c->wait_limit_ms < 0 || c->wait_limit_ms > 60000) return ROLA_ERR_INVALID_ARG;
    if (c->debug_flags & ~ROLA_DEBUG_SKIP_FIRST_K_COPY) return ROLA_ERR_INVALID_ARG;
    if (c->d > (1 << 20) || (int64_t)c->groups * c->rows > ((int64_t)1 << 40) / c->d) return ROLA_ERR_UNSUPPORTED;
    return ROLA_OK;
}

RnShape make_shape(const rola_residual_norm_config_t& c)
{
    RnShape s;
    s.groups = c.groups; s.rows = c.rows; s.d = c.d;
    s.norm = c.norm; s.branch = c.branch_norm;
    s.mod_stride = c.mod_stride ? c.mod_stride : c.d;
    s.total = (int64_t)c.groups * c.rows;
    s.eps = c.eps;
    s.wait_limit_ns = wait_limit_ns(c.wait_limit_ms);
    s.debug_flags = c.debug_flags;
    return s;
}

struct RnWorkspace {
    size_t part, shared, moments, total;
};
RnWorkspace rn_layout(const RnShape& s)
{
    RnWorkspace w;
    size_t off = 0;
    const size_t slot = sizeof(float) * 3 * (size_t)rn_padded(s.d);
    w.part = off; off = align_up(off + slot * ((size_t)rn_parts(s) + s.groups - 1));
    w.shared = off; off = align_up(off + slot * rn_shares(s));
    w.moments = off; off = align_up(off + (rn_long(s) ? sizeof(float4) * (size_t)s.total : 0));
    w.total = off;
    return w;
}

// The vectors that a residual norm's sizes allow: those of the branch with h, those of the norm with a norm.
bool rn_vectors(const rola_residual_norm_config_t& c, const void* h, const void* gate, const void* gamma_h,
                const void* gamma, const void* beta, const void* scale, const void* shift)
{
    if (!h && (gate || gamma_h || c.branch_norm != ROLA_NORM_NONE || c.norm == ROLA_NORM_NONE)) return false;
    if (gamma_h && c.branch_norm == ROLA_NORM_NONE) return false;
    return c.norm != ROLA_NORM_NONE || (!gamma && !beta && !scale && !shift);
}

}  // namespace

extern "C" {

rola_status_t rola_layer_norm(int64_t rows, int32_t d, rola_dtype_t dtype, const void* x, const void* gamma,
                              const void* beta, float eps, void* y, float* mean, float* rstd, void* stream)
{
    ROLA_CHECK(validate_norm(rows, d, dtype));
    if (!x || !y || !mean != !rstd || !(eps >= 0.0f) || !isfinite(eps)) return ROLA_ERR_INVALID_ARG;
    if (!aligned(elem(dtype), x, gamma, beta, y) || !aligned(4, mean, rstd)) return ROLA_ERR_INVALID_ARG;
    ROLA_TRY(launch_layer_norm(dtype, rows, d, x, gamma, beta, eps, y, mean, rstd, static_cast<cudaStream_t>(stream)));
    return ROLA_OK;
}

size_t rola_layer_norm_backward_workspace_bytes(int64_t rows, int32_t d, rola_dtype_t dtype)
{
    if (validate_norm(rows, d, dtype) != ROLA_OK) return 0;
    return align_up(layer_norm_backward_scratch(rows, d));
}

rola_status_t rola_layer_norm_backward(int64_t rows, int32_t d, rola_dtype_t dtype, const void* x, const void* gamma,
                                       const float* mean, const float* rstd, const void* dy, void* dx, float* dgamma,
                                       float* dbeta, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate_norm(rows, d, dtype));
    if (!x || !mean || !rstd || !dy || !dx || !dgamma != !dbeta) return ROLA_ERR_INVALID_ARG;
    if (!aligned(elem(dtype), x, gamma, dy, dx) || !aligned(4, mean, rstd, dgamma, dbeta)) return ROLA_ERR_INVALID_ARG;
    ROLA_CHECK(check_ws(ws, ws_bytes, layer_norm_backward_scratch(rows, d)));
    ROLA_TRY(launch_layer_norm_backward(dtype, rows, d, x, gamma, mean, rstd, dy, dx, dgamma, dbeta,
                                        static_cast<float*>(ws), static_cast<cudaStream_t>(stream)));
    return ROLA_OK;
}

rola_status_t rola_residual_norm_config_init(rola_residual_norm_config_t* cfg)
{
    if (!cfg) return ROLA_ERR_INVALID_ARG;
    memset(cfg, 0, sizeof(*cfg));
    cfg->norm = ROLA_NORM_LAYER;
    cfg->branch_norm = ROLA_NORM_NONE;
    cfg->eps = 1e-6f;
    cfg->dtype = ROLA_BF16;
    return ROLA_OK;
}

rola_status_t rola_residual_norm(const rola_residual_norm_config_t* cfg, const void* x, const void* h, const void* gate,
                                 const void* gamma_h, const void* gamma, const void* beta, const void* scale,
                                 const void* shift, void* out, void* y, float* stats, void* stream)
{
    ROLA_CHECK(validate(cfg));
    if (!x || !h != !out || (cfg->norm == ROLA_NORM_NONE) != !y || (out && out == y)) return ROLA_ERR_INVALID_ARG;
    if (!rn_vectors(*cfg, h, gate, gamma_h, gamma, beta, scale, shift)) return ROLA_ERR_INVALID_ARG;
    if (!aligned(elem(cfg->dtype), x, h, gate, gamma_h, gamma, beta, scale, shift, out, y) || !aligned(16, stats))
        return ROLA_ERR_INVALID_ARG;
    RnArgs a{};
    a.x = x; a.h = h; a.gate = gate; a.gamma_h = gamma_h; a.gamma = gamma; a.beta = beta; a.scale = scale; a.shift = shift;
    a.out = out; a.y = y; a.stats = stats;
    ROLA_TRY(launch_residual_norm(cfg->dtype, make_shape(*cfg), a, static_cast<cudaStream_t>(stream)));
    return ROLA_OK;
}

size_t rola_residual_norm_backward_workspace_bytes(const rola_residual_norm_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? rn_layout(make_shape(*cfg)).total : 0;
}

rola_status_t rola_residual_norm_backward(const rola_residual_norm_config_t* cfg, const void* x, const void* h,
                                          const void* gate, const void* gamma_h, const void* gamma, const void* beta,
                                          const void* scale, const float* stats, const void* dout, const void* dy,
                                          void* dx, void* dh, float* dgate, float* dgamma_h, float* dgamma,
                                          float* dbeta, float* dscale, float* dshift, void* ws, size_t ws_bytes,
                                          void* stream)
{
    ROLA_CHECK(validate(cfg));
    if (!x || !stats || !dx || !h != !dh || dx == dh || (!dout && !dy) || (cfg->norm == ROLA_NORM_NONE) != !dy)
        return ROLA_ERR_INVALID_ARG;
    if (!rn_vectors(*cfg, h, gate, gamma_h, gamma, beta, scale, dshift)) return ROLA_ERR_INVALID_ARG;
    if ((dgate && !gate) || (dgamma_h && !gamma_h) || (dgamma && !gamma) || (dbeta && !beta) || (dscale && !scale))
        return ROLA_ERR_INVALID_ARG;
    if (!aligned(elem(cfg->dtype), x, h, gate, gamma_h, gamma, beta, scale, dout, dy, dx, dh) || !aligned(16, stats) ||
        !aligned(4, dgate, dgamma_h, dgamma, dbeta, dscale, dshift))
        return ROLA_ERR_INVALID_ARG;
    const RnShape s = make_shape(*cfg);
    const RnWorkspace w = rn_layout(s);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    RnArgs a{};
    a.x = x; a.h = h; a.gate = gate; a.gamma_h = gamma_h; a.gamma = gamma; a.beta = beta; a.scale = scale;
    a.stats = const_cast<float*>(stats); a.dout = dout; a.dy = dy; a.dx = dx; a.dh = dh;
    a.dgate = dgate; a.dgamma_h = dgamma_h; a.dgamma = dgamma; a.dbeta = dbeta; a.dscale = dscale; a.dshift = dshift;
    a.part = at<float>(ws, w.part);
    a.shared = at<float>(ws, w.shared);
    a.moments = at<float4>(ws, w.moments);
    ROLA_TRY(launch_residual_norm_backward(cfg->dtype, s, a, static_cast<cudaStream_t>(stream)));
    return ROLA_OK;
}

rola_status_t rola_ffn_config_init(rola_ffn_config_t* cfg)
{
    if (!cfg) return ROLA_ERR_INVALID_ARG;
    memset(cfg, 0, sizeof(*cfg));
    cfg->act = ROLA_LOWRANK_ACT_SILU;
    cfg->dtype = ROLA_BF16;
    return ROLA_OK;
}

size_t rola_ffn_workspace_bytes(const rola_ffn_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? ffn_layout(*cfg, false).total : 0;
}

size_t rola_ffn_backward_workspace_bytes(const rola_ffn_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? ffn_layout(*cfg, true).total : 0;
}

rola_status_t rola_ffn(const rola_ffn_config_t* cfg, const void* X, const void* W_gate, const void* W_up,
                       const void* W_down, void* Y, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    return ffn_forward(cfg, X, W_gate, W_up, W_down, Y, nullptr, nullptr, ws, ws_bytes, stream);
}

rola_status_t rola_ffn_train(const rola_ffn_config_t* cfg, const void* X, const void* W_gate, const void* W_up,
                             const void* W_down, void* Y, float* G, float* U, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    if (!G || !U) return ROLA_ERR_INVALID_ARG;
    return ffn_forward(cfg, X, W_gate, W_up, W_down, Y, G, U, ws, ws_bytes, stream);
}

rola_status_t rola_ffn_backward(const rola_ffn_config_t* cfg, const void* X, const void* W_gate, const void* W_up,
                                const void* W_down, const float* G, const float* U, const void* dY, void* dX,
                                void* dW_gate, void* dW_up, void* dW_down, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    const void* need[] = {X, W_gate, W_up, W_down, G, U, dY, dX, dW_gate, dW_up, dW_down};
    for (const void* p : need)
        if (!p || !aligned(16, p)) return ROLA_ERR_INVALID_ARG;
    const FfnWorkspace w = ffn_layout(*cfg, true);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const FfnShape s = make_shape(*cfg);
    void *H = at<void>(ws, w.H), *dG = at<void>(ws, w.dG), *dU = at<void>(ws, w.dU);
    ROLA_TRY(cudaMemsetAsync(at<uint8_t>(ws, w.status), 0, sizeof(DeviceStatus), st));
    if (cfg->dtype == ROLA_BF16)
        ROLA_TRY(launch_ffn_backward_tc(s, X, W_gate, W_up, W_down, G, U, dY, H, dG, dU, dX, dW_gate, dW_up, dW_down,
                                        at<DeviceStatus>(ws, w.status), st));
    else
        ROLA_TRY(launch_ffn_backward_simt(s, X, W_gate, W_up, W_down, G, U, dY, H, dG, dU, dX, dW_gate, dW_up, dW_down,
                                          st));
    return ROLA_OK;
}

rola_status_t rola_linear_config_init(rola_linear_config_t* cfg)
{
    if (!cfg) return ROLA_ERR_INVALID_ARG;
    memset(cfg, 0, sizeof(*cfg));
    cfg->act = ROLA_LOWRANK_ACT_IDENTITY;
    cfg->dtype = ROLA_BF16;
    return ROLA_OK;
}

size_t rola_linear_workspace_bytes(const rola_linear_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? linear_layout(*cfg, false).total : 0;
}

size_t rola_linear_backward_workspace_bytes(const rola_linear_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? linear_layout(*cfg, true).total : 0;
}

rola_status_t rola_linear(const rola_linear_config_t* cfg, const void* X, const void* W, const void* b,
                          const void* residual, void* Y, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    return linear_forward(cfg, X, W, b, residual, Y, nullptr, ws, ws_bytes, stream);
}

rola_status_t rola_linear_train(const rola_linear_config_t* cfg, const void* X, const void* W, const void* b,
                                const void* residual, void* Y, float* Z, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    if (!Z && cfg->act != ROLA_LOWRANK_ACT_IDENTITY) return ROLA_ERR_INVALID_ARG;
    return linear_forward(cfg, X, W, b, residual, Y, Z, ws, ws_bytes, stream);
}

rola_status_t rola_linear_backward(const rola_linear_config_t* cfg, const void* X, const void* W, const float* Z,
                                   const void* dY, void* dX, void* dW, float* db, void* ws, size_t ws_bytes,
                                   void* stream)
{
    ROLA_CHECK(validate(cfg));
    const bool identity = cfg->act == ROLA_LOWRANK_ACT_IDENTITY;
    if (!X || !W || !dY || (!Z && !identity) || (!dX && !dW && !db)) return ROLA_ERR_INVALID_ARG;
    if (!aligned(16, X, W, Z, dY, dX, dW, db)) return ROLA_ERR_INVALID_ARG;
    const LinWorkspace w = linear_layout(*cfg, true);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    if (same_start(dX, X, W, Z, dY, dW, db, ws) || same_start(dW, X, W, Z, dY, db, ws) || same_start(db, X, W, Z, dY, ws))
        return ROLA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const LinShape s = make_shape(*cfg);
    DeviceStatus* status = at<DeviceStatus>(ws, w.status);
    const void* dZ = identity ? dY : at<void>(ws, w.dZ);
    bool clear = true;                           // whether the next kernel clears the status word
    if (!identity || db) {
        ROLA_TRY(launch_linear_grad(cfg->dtype, s, dY, identity ? nullptr : Z, at<void>(ws, w.dZ), db, at<float>(ws, w.sums),
                                    status, st));
        clear = false;
    }
    if (cfg->dtype == ROLA_FP32) {
        if (clear) ROLA_TRY(cudaMemsetAsync(status, 0, sizeof(DeviceStatus), st));
        ROLA_TRY(launch_linear_backward_simt(s, X, W, dZ, dX, dW, st));
        return ROLA_OK;
    }
    if (dX) {
        if (linear_dx_form(s) == kLinearFew) ROLA_TRY(launch_linear_few_dx(s, W, dZ, dX, clear, status, st));
        else ROLA_TRY(launch_linear_dx_tc(s, W, dZ, dX, at<float>(ws, w.part), clear, status, st));
    }
    if (dW) ROLA_TRY(launch_linear_dw_tc(s, X, dZ, dW, at<float>(ws, w.part), clear && !dX, status, st));
    return ROLA_OK;
}

rola_status_t rola_attention_config_init(rola_attention_config_t* cfg)
{
    if (!cfg) return ROLA_ERR_INVALID_ARG;
    memset(cfg, 0, sizeof(*cfg));
    cfg->d_h = kDh;
    cfg->dtype = ROLA_BF16;
    return ROLA_OK;
}

size_t rola_attention_workspace_bytes(const rola_attention_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? attn_layout(make_shape(*cfg), false).total : 0;
}

size_t rola_attention_backward_workspace_bytes(const rola_attention_config_t* cfg)
{
    return validate(cfg) == ROLA_OK ? attn_layout(make_shape(*cfg), true).total : 0;
}

rola_status_t rola_attention(const rola_attention_config_t* cfg, const void* q, const void* k, const void* v,
                             const int32_t* kv_len, void* o, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    if (!q || !k || !v || !o || !aligned(16, q, k, v, o) || !aligned(4, kv_len, lse)) return ROLA_ERR_INVALID_ARG;
    const AttnShape s = make_shape(*cfg);
    const AttnWorkspace w = attn_layout(s, false);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    AttnArgs a{};
    a.q = q; a.k = k; a.v = v; a.kv_len = kv_len; a.o = o; a.lse = lse;
    a.part_o = at<float>(ws, w.part_o); a.part_lse = at<float>(ws, w.part_lse);
    a.status = at<DeviceStatus>(ws, w.status);
    ROLA_TRY(cudaMemsetAsync(a.status, 0, sizeof(DeviceStatus), st));
    const bool bf16 = cfg->dtype == ROLA_BF16;
    ROLA_TRY(bf16 ? launch_attention_tc(s, a, st) : launch_attention_simt(s, a, st));
    if (s.splits > 1)
        ROLA_TRY(bf16 ? launch_attention_join<__nv_bfloat16>(s, a, st) : launch_attention_join<float>(s, a, st));
    return ROLA_OK;
}

rola_status_t rola_attention_backward(const rola_attention_config_t* cfg, const void* q, const void* k, const void* v,
                                      const int32_t* kv_len, const void* o, const float* lse, const void* dO, void* dq,
                                      void* dk, void* dv, void* ws, size_t ws_bytes, void* stream)
{
    ROLA_CHECK(validate(cfg));
    const void* need[] = {q, k, v, o, dO, dq, dk, dv};
    for (const void* p : need)
        if (!p || !aligned(16, p)) return ROLA_ERR_INVALID_ARG;
    if (!lse || !aligned(4, lse, kv_len)) return ROLA_ERR_INVALID_ARG;
    const AttnShape s = make_shape(*cfg);
    const AttnWorkspace w = attn_layout(s, true);
    ROLA_CHECK(check_ws(ws, ws_bytes, w.total));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    AttnArgs a{};
    a.q = q; a.k = k; a.v = v; a.kv_len = kv_len; a.o_in = o; a.lse_in = lse; a.dO = dO;
    a.dq = dq; a.dk = dk; a.dv = dv;
    a.D = at<float>(ws, w.D);
    a.part_dq = at<float>(ws, w.part_dq); a.part_dk = at<float>(ws, w.part_dk); a.part_dv = at<float>(ws, w.part_dv);
    a.status = at<DeviceStatus>(ws, w.status);
    if (cfg->dtype == ROLA_BF16) {
        // the row sums' kernel clears the status too; over one stage of keys the dq kernel forms D itself
        if (s.Lk > 128) ROLA_TRY(launch_attention_rowdot<__nv_bfloat16>(s, a, st));
        else ROLA_TRY(cudaMemsetAsync(a.status, 0, sizeof(DeviceStatus), st));
        ROLA_TRY(launch_attention_backward_tc(s, a, st));
    } else {
        ROLA_TRY(launch_attention_rowdot<float>(s, a, st));
        ROLA_TRY(launch_attention_backward_simt(s, a, st));
    }
    return ROLA_OK;
}

}  // extern "C"
