// C ABI of libadama: context, argument checks, host-side constants, launches.
#include <float.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "adama_internal.h"

struct adama_ctx {
    adama_config cfg;
    int64_t t;    // step counter of Algorithm 2
    int n_micro;  // N of the current mini-batch (0 before the first)
    adama::FoldConstants fold_c;
    int sm_count;
    unsigned *status_dev;      // 256-byte device status block
    cudaStream_t copy_stream;  // host-buffer variants: H2D copies overlap the folds
    cudaStream_t d2h_stream;   // ADAMA_ASYNC_COPYBACK: weights go back to the host here
    cudaEvent_t ev_applied, ev_d2h_done;
    bool d2h_pending;          // a copy-back that no stream has been made to wait for yet
    cudaEvent_t ev_copied[2], ev_folded[2], ev_entry;
    int64_t launches;
    double weight_decay;  // decoupled (AdamW) decay; 0 = the paper's plain update
    adama::WgradVariant variant;  // adama_debug_set_wgrad_variant; all 0 = automatic
    char err[256];
};

namespace adama {

FoldConstants make_fold_constants(double beta1, double beta2, int n_micro, unsigned flags) {
    double N = (flags & ADAMA_GRADS_PRESCALED) ? 1.0 : (double)n_micro;
    FoldConstants c;
    c.a = (float)((1.0 - beta1) / N);
    c.b = (float)((1.0 - beta2) / (N * N));
    return c;
}

void split_hi_lo(double x, float *hi, float *lo) {
    *hi = (float)x;
    *lo = (float)(x - (double)*hi);
}

ApplyConstants make_apply_constants(double beta1, double beta2, double eps, int64_t t, double lr,
                                    int world, bool sharded, double weight_decay) {
    ApplyConstants c;
    const double R = (double)world;
    double bc1 = 1.0 - pow(beta1, (double)t);
    double bc2 = 1.0 - pow(beta2, (double)t);
    // m_t = m/R, v_t = v/R^2 (Eqs. 6-7); w -= lr * (m_t/bc1) / (sqrt(v_t/bc2) + eps)
    c.step = (float)(lr / bc1 / R);
    c.inv_bc2 = (float)(1.0 / bc2 / (R * R));
    c.eps = (float)eps;
    c.w_keep = (float)(1.0 - lr * weight_decay);
    // stored for the next mini-batch: beta1*m_t = (beta1/R)*m and R*beta2*v_t = (beta2/R)*v
    // (sharded: the owner keeps R*beta1*m_t = beta1*m and R^2*beta2*v_t = beta2*v)
    split_hi_lo(sharded ? beta1 : beta1 / R, &c.beta1_hi, &c.beta1_lo);
    split_hi_lo(sharded ? beta2 : beta2 / R, &c.beta2_hi, &c.beta2_lo);
    return c;
}

}  // namespace adama

namespace {

adama_status fail(adama_ctx *ctx, adama_status st, const char *msg) {
    if (ctx) snprintf(ctx->err, sizeof(ctx->err), "%s", msg);
    return st;
}

adama_status cuda_fail(adama_ctx *ctx, const char *what, cudaError_t e) {
    if (ctx) snprintf(ctx->err, sizeof(ctx->err), "%s: %s", what, cudaGetErrorString(e));
    return ADAMA_ERR_CUDA;
}

bool aligned_to(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Makes ctx's device current for the duration of a call and restores the caller's.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) ok = (cudaSetDevice(dev) == cudaSuccess);
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

size_t dtype_size(adama_dtype d) { return d == ADAMA_F32 ? 4 : 2; }

// ADAMA_ASYNC_COPYBACK: before `stream` may overwrite weights, it waits for the copy-back that
// is still reading them.
cudaError_t join_copyback(adama_ctx *ctx, cudaStream_t stream) {
    if (!ctx->d2h_pending) return cudaSuccess;
    ctx->d2h_pending = false;
    return cudaStreamWaitEvent(stream, ctx->ev_d2h_done, 0);
}

bool config_ok(const adama_config *cfg) {
    return cfg && cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0 &&
           cfg->eps >= 0.0 && isfinite(cfg->eps) && cfg->device >= 0 &&
           (cfg->flags & ~(ADAMA_GRADS_PRESCALED | ADAMA_ASYNC_COPYBACK | ADAMA_INPUTS_SETTLED)) == 0;
}

adama_status check_fold_args(adama_ctx *ctx, const void *grad, adama_dtype gdt, float *m, float *v,
                             size_t n) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (gdt != ADAMA_F32 && gdt != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold: unknown gradient dtype");
    if (n > 0 && (!grad || !m || !v)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold: null pointer");
    if (ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "fold: adama_begin_minibatch has not been called");
    if (!aligned_to(grad, dtype_size(gdt)) || !aligned_to(m, 4) || !aligned_to(v, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "fold: pointer not aligned to its element size");
    return ADAMA_OK;
}

adama_status check_wgrad_args(adama_ctx *ctx, const void *X, const void *dY, int tokens, int d_in,
                              int d_out, int64_t ldx, int64_t ldy, float *m, float *v,
                              int64_t ldmv) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (tokens < 0 || d_in < 1 || d_out < 1)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold: bad shape");
    if (!m || !v || (tokens > 0 && (!X || !dY)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold: null pointer");
    if (ldx < d_in || ldy < d_out || ldmv < d_out)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold: row pitch smaller than the row");
    if (ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "wgrad_fold: adama_begin_minibatch has not been called");
    if (!aligned_to(X, 16) || !aligned_to(dY, 16) || !aligned_to(m, 16) || !aligned_to(v, 16))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "wgrad_fold: X, dY, m, v must be 16-byte aligned");
    if (ldx % 8 || ldy % 8 || ldmv % 4)
        return fail(ctx, ADAMA_ERR_MISALIGNED,
                    "wgrad_fold: ldx, ldy must be multiples of 8 and ldmv of 4");
    // tensor-map strides are limited to 2^40 bytes
    if (ldx * 2 >= (1ll << 40) || ldy * 2 >= (1ll << 40) || ldmv * 4 >= (1ll << 40))
        return fail(ctx, ADAMA_ERR_UNSUPPORTED, "wgrad_fold: row pitch too large for a tensor map");
    return ADAMA_OK;
}

adama_status check_apply_args(adama_ctx *ctx, float *w, float *m, float *v, size_t n, double lr) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (n > 0 && (!w || !m || !v)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply: null pointer");
    if (!isfinite(lr)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply: lr is not finite");
    if (ctx->t < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "apply: no mini-batch has been started (t == 0)");
    if (!aligned_to(w, 4) || !aligned_to(m, 4) || !aligned_to(v, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "apply: pointer not aligned to 4 bytes");
    return ADAMA_OK;
}

// Walks a list in ranges of at most `most` tensors: launch(first, count) for each.
template <typename Launch>
adama_status for_ranges(adama_ctx *ctx, int count, int most, const char *what, Launch launch) {
    for (int first = 0; first < count; first += most) {
        const int k = count - first < most ? count - first : most;
        cudaError_t e = launch(first, k);
        if (e != cudaSuccess) return cuda_fail(ctx, what, e);
    }
    return ADAMA_OK;
}

}  // namespace

extern "C" {

const char *adama_version(void) { return "0.1.0"; }

adama_status adama_init(adama_ctx **out, const adama_config *cfg) {
    if (!out) return ADAMA_ERR_INVALID_ARG;
    *out = nullptr;
    if (!config_ok(cfg)) return ADAMA_ERR_INVALID_ARG;
    int count = 0;
    if (cudaGetDeviceCount(&count) != cudaSuccess || cfg->device >= count) return ADAMA_ERR_CUDA;
    // the two attributes alone: a whole cudaDeviceProp takes milliseconds to fill
    int major = 0, sm_count = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, cfg->device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, cfg->device) != cudaSuccess)
        return ADAMA_ERR_CUDA;
    if (major != 10) return ADAMA_ERR_UNSUPPORTED;  // kernels are built for sm_100a only

    adama_ctx *ctx = new (std::nothrow) adama_ctx();
    if (!ctx) return ADAMA_ERR_CUDA;
    memset(ctx, 0, sizeof(*ctx));
    ctx->cfg = *cfg;
    ctx->sm_count = sm_count;

    DeviceGuard guard(cfg->device);
    const char *msg = "";
    cudaError_t e = guard.ok ? cudaSuccess : cudaErrorInvalidDevice;
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&ctx->status_dev), 256);
    if (e == cudaSuccess) e = cudaMemset(ctx->status_dev, 0, 256);
    if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&ctx->copy_stream, cudaStreamNonBlocking);
    for (int i = 0; i < 2 && e == cudaSuccess; ++i) {
        e = cudaEventCreateWithFlags(&ctx->ev_copied[i], cudaEventDisableTiming);
        if (e == cudaSuccess)
            e = cudaEventCreateWithFlags(&ctx->ev_folded[i], cudaEventDisableTiming);
    }
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->ev_entry, cudaEventDisableTiming);
    if (e == cudaSuccess && (cfg->flags & ADAMA_ASYNC_COPYBACK)) {
        e = cudaStreamCreateWithFlags(&ctx->d2h_stream, cudaStreamNonBlocking);
        if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->ev_applied, cudaEventDisableTiming);
        if (e == cudaSuccess) e = cudaEventCreateWithFlags(&ctx->ev_d2h_done, cudaEventDisableTiming);
    }
    if (e == cudaSuccess) e = adama::wgrad_fold_setup(&msg);
    if (e != cudaSuccess) {
        adama_destroy(ctx);
        return ADAMA_ERR_CUDA;
    }
    *out = ctx;
    return ADAMA_OK;
}

adama_status adama_destroy(adama_ctx *ctx) {
    if (!ctx) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    if (ctx->status_dev) cudaFree(ctx->status_dev);
    if (ctx->copy_stream) cudaStreamDestroy(ctx->copy_stream);
    if (ctx->d2h_stream) {
        cudaStreamSynchronize(ctx->d2h_stream);  // a copy-back may still be writing host memory
        cudaStreamDestroy(ctx->d2h_stream);
    }
    if (ctx->ev_applied) cudaEventDestroy(ctx->ev_applied);
    if (ctx->ev_d2h_done) cudaEventDestroy(ctx->ev_d2h_done);
    for (int i = 0; i < 2; ++i) {
        if (ctx->ev_copied[i]) cudaEventDestroy(ctx->ev_copied[i]);
        if (ctx->ev_folded[i]) cudaEventDestroy(ctx->ev_folded[i]);
    }
    if (ctx->ev_entry) cudaEventDestroy(ctx->ev_entry);
    delete ctx;
    return ADAMA_OK;
}

adama_status adama_begin_minibatch(adama_ctx *ctx, int n_micro) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (n_micro < 1) return fail(ctx, ADAMA_ERR_INVALID_ARG, "begin_minibatch: n_micro must be >= 1");
    ctx->t += 1;
    ctx->n_micro = n_micro;
    ctx->fold_c = adama::make_fold_constants(ctx->cfg.beta1, ctx->cfg.beta2, n_micro, ctx->cfg.flags);
    return ADAMA_OK;
}

adama_status adama_fold(adama_ctx *ctx, const void *grad, adama_dtype gdt, float *m, float *v,
                        size_t n, void *cuda_stream) {
    adama_status st = check_fold_args(ctx, grad, gdt, m, v, n);
    if (st != ADAMA_OK) return st;
    if (n == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    cudaError_t e = adama::launch_fold(grad, gdt, m, v, n, ctx->fold_c, ctx->sm_count,
                                       static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "fold launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

static adama_status wgrad_impl(adama_ctx *ctx, const void *X, const void *dY, int tokens, int d_in,
                               int d_out, int64_t ldx, int64_t ldy, float *m, float *v,
                               int64_t ldmv, float *bias_m, float *bias_v, void *cuda_stream,
                               unsigned long long wait_limit_ns = 0, int withhold_last_load = 0) {
    adama_status st = check_wgrad_args(ctx, X, dY, tokens, d_in, d_out, ldx, ldy, m, v, ldmv);
    if (st != ADAMA_OK) return st;
    if (tokens == 0) return ADAMA_OK;  // empty sum: G = 0, nothing to add
    DeviceGuard guard(ctx->cfg.device);
    adama::WgradArgs a;
    a.X = X;
    a.dY = dY;
    a.tokens = tokens;
    a.d_in = d_in;
    a.d_out = d_out;
    a.ldx = ldx;
    a.ldy = ldy;
    a.ldmv = ldmv;
    a.m = m;
    a.v = v;
    a.c = ctx->fold_c;
    a.status = ctx->status_dev;
    a.sm_count = ctx->sm_count;
    a.stream = static_cast<cudaStream_t>(cuda_stream);
    a.bias_m = bias_m;
    a.bias_v = bias_v;
    a.variant = ctx->variant;
    a.wait_limit_ns = wait_limit_ns;
    a.withhold_last_load = withhold_last_load;
    a.inputs_settled = (ctx->cfg.flags & ADAMA_INPUTS_SETTLED) ? 1 : 0;
    const char *msg = "wgrad_fold";
    cudaError_t e = adama::launch_wgrad_fold(a, &msg);
    if (e != cudaSuccess) return cuda_fail(ctx, msg, e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_linear_wgrad_fold(adama_ctx *ctx, const void *X, const void *dY, int tokens,
                                     int d_in, int d_out, int64_t ldx, int64_t ldy, float *m,
                                     float *v, int64_t ldmv, void *cuda_stream) {
    return wgrad_impl(ctx, X, dY, tokens, d_in, d_out, ldx, ldy, m, v, ldmv, nullptr, nullptr,
                      cuda_stream);
}

adama_status adama_linear_wgrad_bias_fold(adama_ctx *ctx, const void *X, const void *dY, int tokens,
                                          int d_in, int d_out, int64_t ldx, int64_t ldy, float *m,
                                          float *v, int64_t ldmv, float *m_bias, float *v_bias,
                                          void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!m_bias || !v_bias)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_bias_fold: null bias moments");
    if (!aligned_to(m_bias, 4) || !aligned_to(v_bias, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "wgrad_bias_fold: bias moments not aligned to 4 bytes");
    return wgrad_impl(ctx, X, dY, tokens, d_in, d_out, ldx, ldy, m, v, ldmv, m_bias, v_bias,
                      cuda_stream);
}

adama_status adama_linear_wgrad_fold_multi(adama_ctx *ctx, const adama_linear_item *items, int count,
                                           void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && !items))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold_multi: null list or negative count");
    for (int i = 0; i < count; ++i) {
        const adama_linear_item &it = items[i];
        adama_status st = check_wgrad_args(ctx, it.X, it.dY, it.tokens, it.d_in, it.d_out, it.ldx,
                                           it.ldy, it.m, it.v, it.ldmv);
        if (st != ADAMA_OK) return st;
        if ((it.m_bias == nullptr) != (it.v_bias == nullptr))
            return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold_multi: m_bias and v_bias go together");
        if (!aligned_to(it.m_bias, 4) || !aligned_to(it.v_bias, 4))
            return fail(ctx, ADAMA_ERR_MISALIGNED, "wgrad_fold_multi: bias moments not aligned to 4 bytes");
    }
    DeviceGuard guard(ctx->cfg.device);
    adama::WgradArgs batch[adama::kMaxWgradLayers];
    int k = 0;
    bool first_launch = true;
    for (int i = 0; i <= count; ++i) {
        if ((i == count || k == adama::kMaxWgradLayers) && k > 0) {
            // From the call's second launch on, the kernel just before is this call's own previous
            // launch, which writes only m, v and bias moments: the operand loads need not wait for it.
            if (!first_launch) batch[0].inputs_settled = 1;
            const char *msg = "wgrad_fold_multi";
            cudaError_t e = adama::launch_wgrad_fold_multi(batch, k, &msg);
            if (e != cudaSuccess) return cuda_fail(ctx, msg, e);
            ctx->launches += 1;
            first_launch = false;
            k = 0;
        }
        if (i == count) break;
        const adama_linear_item &it = items[i];
        if (it.tokens == 0) continue;  // empty sum: nothing to add
        adama::WgradArgs &a = batch[k++];
        a = adama::WgradArgs();
        a.X = it.X;
        a.dY = it.dY;
        a.tokens = it.tokens;
        a.d_in = it.d_in;
        a.d_out = it.d_out;
        a.ldx = it.ldx;
        a.ldy = it.ldy;
        a.ldmv = it.ldmv;
        a.m = it.m;
        a.v = it.v;
        a.c = ctx->fold_c;
        a.status = ctx->status_dev;
        a.sm_count = ctx->sm_count;
        a.stream = static_cast<cudaStream_t>(cuda_stream);
        a.bias_m = it.m_bias;
        a.bias_v = it.v_bias;
        a.variant = ctx->variant;
        a.inputs_settled = (ctx->cfg.flags & ADAMA_INPUTS_SETTLED) ? 1 : 0;
    }
    return ADAMA_OK;
}

static adama_status apply_impl(adama_ctx *ctx, float *w, float *m, float *v, size_t n, double lr,
                               int world, bool sharded, void *cuda_stream,
                               void *w_bf16_out = nullptr) {
    adama_status st = check_apply_args(ctx, w, m, v, n, lr);
    if (st != ADAMA_OK) return st;
    if (world < 1) return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply: world_size must be >= 1");
    if (n == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    adama::ApplyConstants c = adama::make_apply_constants(ctx->cfg.beta1, ctx->cfg.beta2,
                                                          ctx->cfg.eps, ctx->t, lr, world, sharded,
                                                          ctx->weight_decay);
    cudaError_t e = join_copyback(ctx, static_cast<cudaStream_t>(cuda_stream));
    if (e == cudaSuccess)
        e = adama::launch_apply(w, m, v, n, c, ctx->sm_count,
                                static_cast<cudaStream_t>(cuda_stream), w_bf16_out);
    if (e != cudaSuccess) return cuda_fail(ctx, "apply launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_apply_bf16_copy(adama_ctx *ctx, float *w, float *m, float *v, void *w_bf16_out,
                                   size_t n, double lr, void *cuda_stream) {
    if (ctx && n > 0 && !w_bf16_out)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_bf16_copy: null bf16 output");
    if (ctx && !aligned_to(w_bf16_out, 2))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "apply_bf16_copy: bf16 output not 2-byte aligned");
    return apply_impl(ctx, w, m, v, n, lr, 1, false, cuda_stream, w_bf16_out);
}

adama_status adama_apply(adama_ctx *ctx, float *w, float *m, float *v, size_t n, double lr,
                         void *cuda_stream) {
    return apply_impl(ctx, w, m, v, n, lr, 1, false, cuda_stream);
}

adama_status adama_apply_allreduced(adama_ctx *ctx, float *w, float *m, float *v, size_t n,
                                    double lr, int world_size, void *cuda_stream) {
    return apply_impl(ctx, w, m, v, n, lr, world_size, false, cuda_stream);
}

adama_status adama_apply_sharded(adama_ctx *ctx, float *w, float *m, float *v, size_t n, double lr,
                                 int world_size, void *cuda_stream) {
    return apply_impl(ctx, w, m, v, n, lr, world_size, true, cuda_stream);
}

adama_status adama_apply_sharded_peers(adama_ctx *ctx, float *const *w_peers, float *const *m_peers,
                                       float *const *v_peers, int world_size, int rank, size_t n,
                                       double lr, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (world_size < 1 || rank < 0 || rank >= world_size || !w_peers || !m_peers || !v_peers)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_sharded_peers: bad world size, rank or list");
    if (world_size > adama::kMaxPeers)
        return fail(ctx, ADAMA_ERR_UNSUPPORTED, "apply_sharded_peers: more than 16 peers");
    if (!isfinite(lr)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_sharded_peers: lr is not finite");
    if (ctx->t < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "apply_sharded_peers: no mini-batch has been started");
    if (n % (4 * (size_t)world_size))
        return fail(ctx, ADAMA_ERR_UNSUPPORTED,
                    "apply_sharded_peers: n must be a multiple of 4*world_size (pad the buffers)");
    for (int q = 0; q < world_size; ++q) {
        if (n > 0 && (!w_peers[q] || !m_peers[q] || !v_peers[q]))
            return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_sharded_peers: null peer pointer");
        if (!aligned_to(w_peers[q], 16) || !aligned_to(m_peers[q], 16) || !aligned_to(v_peers[q], 16))
            return fail(ctx, ADAMA_ERR_MISALIGNED, "apply_sharded_peers: buffers must be 16-byte aligned");
    }
    if (n == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    const adama::ApplyConstants c =
        adama::make_apply_constants(ctx->cfg.beta1, ctx->cfg.beta2, ctx->cfg.eps, ctx->t, lr,
                                    world_size, true, ctx->weight_decay);
    cudaError_t e = join_copyback(ctx, static_cast<cudaStream_t>(cuda_stream));
    if (e == cudaSuccess)
        e = adama::launch_apply_sharded_peers(w_peers, m_peers, v_peers, world_size, rank, n, c,
                                              ctx->sm_count, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "apply_sharded_peers launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_bias_grad_fold(adama_ctx *ctx, const void *dY, int tokens, int d_out,
                                  int64_t ldy, float *m, float *v, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (tokens < 0 || d_out < 1 || !m || !v || (tokens > 0 && !dY) || ldy < d_out)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "bias_grad_fold: bad shape, null pointer or pitch");
    if (ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "bias_grad_fold: adama_begin_minibatch has not been called");
    if (!aligned_to(dY, 16) || ldy % 8 || !aligned_to(m, 4) || !aligned_to(v, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED,
                    "bias_grad_fold: dY must be 16-byte aligned with ldy a multiple of 8");
    if (tokens == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    cudaError_t e = adama::launch_bias_grad_fold(dY, tokens, d_out, ldy, m, v, ctx->fold_c,
                                                 static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "bias_grad_fold launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

// ---- multi-tensor forms ---------------------------------------------------------------------

// Tensors at least this long go to the single-tensor kernels (they saturate the GPU alone).
static const size_t kMultiLargeThreshold = (size_t)1 << 22;

adama_status adama_fold_multi(adama_ctx *ctx, const void *const *grads, adama_dtype gdt,
                              float *const *m, float *const *v, const size_t *n, int count,
                              void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && (!grads || !m || !v || !n)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_multi: null list or negative count");
    for (int i = 0; i < count; ++i) {
        adama_status st = check_fold_args(ctx, grads[i], gdt, m[i], v[i], n[i]);
        if (st != ADAMA_OK) return st;
    }
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const void *g_[adama::kMultiMax];
    float *m_[adama::kMultiMax], *v_[adama::kMultiMax];
    size_t n_[adama::kMultiMax];
    int k = 0;
    cudaError_t e = cudaSuccess;
    for (int i = 0; i <= count && e == cudaSuccess; ++i) {
        const bool flush = (i == count) || k == adama::kMultiMax;
        if (flush && k > 0) {
            e = adama::launch_fold_multi(g_, gdt, m_, v_, n_, k, ctx->fold_c, ctx->sm_count, stream);
            ctx->launches += 1;
            k = 0;
        }
        if (i == count || e != cudaSuccess) break;
        if (n[i] == 0) continue;
        if (n[i] >= kMultiLargeThreshold) {
            e = adama::launch_fold(grads[i], gdt, m[i], v[i], n[i], ctx->fold_c, ctx->sm_count, stream);
            ctx->launches += 1;
            continue;
        }
        g_[k] = grads[i];
        m_[k] = m[i];
        v_[k] = v[i];
        n_[k] = n[i];
        ++k;
    }
    if (e != cudaSuccess) return cuda_fail(ctx, "fold_multi launch", e);
    return ADAMA_OK;
}

adama_status adama_apply_multi(adama_ctx *ctx, float *const *w, float *const *m, float *const *v,
                               const size_t *n, int count, double lr, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && (!w || !m || !v || !n)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_multi: null list or negative count");
    for (int i = 0; i < count; ++i) {
        adama_status st = check_apply_args(ctx, w[i], m[i], v[i], n[i], lr);
        if (st != ADAMA_OK) return st;
    }
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const adama::ApplyConstants c = adama::make_apply_constants(
        ctx->cfg.beta1, ctx->cfg.beta2, ctx->cfg.eps, ctx->t, lr, 1, false, ctx->weight_decay);
    float *w_[adama::kMultiMax], *m_[adama::kMultiMax], *v_[adama::kMultiMax];
    size_t n_[adama::kMultiMax];
    int k = 0;
    cudaError_t e = join_copyback(ctx, stream);
    for (int i = 0; i <= count && e == cudaSuccess; ++i) {
        const bool flush = (i == count) || k == adama::kMultiMax;
        if (flush && k > 0) {
            e = adama::launch_apply_multi(w_, m_, v_, n_, k, c, ctx->sm_count, stream);
            ctx->launches += 1;
            k = 0;
        }
        if (i == count || e != cudaSuccess) break;
        if (n[i] == 0) continue;
        if (n[i] >= kMultiLargeThreshold) {
            e = adama::launch_apply(w[i], m[i], v[i], n[i], c, ctx->sm_count, stream);
            ctx->launches += 1;
            continue;
        }
        w_[k] = w[i];
        m_[k] = m[i];
        v_[k] = v[i];
        n_[k] = n[i];
        ++k;
    }
    if (e != cudaSuccess) return cuda_fail(ctx, "apply_multi launch", e);
    return ADAMA_OK;
}

// ---- the end of a fine-tuning step ------------------------------------------------------------

static bool any_element(const size_t *n, int first, int count) {
    for (int i = first; i < first + count; ++i)
        if (n[i] > 0) return true;
    return false;
}

static adama_status check_state8(adama_ctx *ctx, const adama_state8 &s, size_t n) {
    if (n > 0 && (!s.m_codes || !s.m_scale || !s.v_codes || !s.v_scale))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "state8: null pointer");
    if (!aligned_to(s.m_scale, 4) || !aligned_to(s.v_scale, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "state8: scales not aligned to 4 bytes");
    return ADAMA_OK;
}

static adama_status fold_apply_impl(adama_ctx *ctx, const void *const *grads, adama_dtype gdt,
                                    float *const *w, float *const *m, float *const *v,
                                    const adama_state8 *states, void *const *w_bf16, const size_t *n,
                                    int count, double lr, const float *grad_factor, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    const bool packed = states != nullptr;
    if (count < 0 || (count > 0 && (!grads || !w || !n || (!packed && (!m || !v)))))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_apply: null list or negative count");
    if (gdt != ADAMA_F32 && gdt != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_apply: unknown gradient dtype");
    if (!isfinite(lr)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_apply: lr is not finite");
    if (ctx->n_micro < 1 || ctx->t < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "fold_apply: adama_begin_minibatch has not been called");
    if (!aligned_to(grad_factor, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "fold_apply: grad_factor not aligned to 4 bytes");
    for (int i = 0; i < count; ++i) {
        if (n[i] > 0 && (!grads[i] || !w[i] || (!packed && (!m[i] || !v[i]))))
            return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_apply: null pointer");
        if (!aligned_to(grads[i], dtype_size(gdt)) || !aligned_to(w[i], 4) ||
            (!packed && (!aligned_to(m[i], 4) || !aligned_to(v[i], 4))) ||
            (w_bf16 && !aligned_to(w_bf16[i], 2)))
            return fail(ctx, ADAMA_ERR_MISALIGNED, "fold_apply: pointer not aligned to its element size");
        if (packed) {
            adama_status st = check_state8(ctx, states[i], n[i]);
            if (st != ADAMA_OK) return st;
        }
    }
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const adama::ApplyConstants c = adama::make_apply_constants(
        ctx->cfg.beta1, ctx->cfg.beta2, ctx->cfg.eps, ctx->t, lr, 1, false, ctx->weight_decay);
    cudaError_t e = join_copyback(ctx, stream);
    if (e != cudaSuccess) return cuda_fail(ctx, "fold_apply", e);
    adama::StepList list;
    list.g = grads;
    list.w = w;
    list.m = m;
    list.v = v;
    list.s8 = states;
    list.copy = w_bf16;
    list.n = n;
    return for_ranges(ctx, count, packed ? adama::kStep8Max : adama::kStepMax, "fold_apply launch",
                      [&](int first, int k) {
        if (!any_element(n, first, k)) return cudaSuccess;
        ctx->launches += 1;
        return packed ? adama::launch_fold_apply8_multi(list, gdt, first, k, ctx->fold_c, c, grad_factor,
                                                        ctx->status_dev, ctx->sm_count, stream)
                      : adama::launch_fold_apply_multi(list, gdt, first, k, ctx->fold_c, c, grad_factor,
                                                       ctx->status_dev, ctx->sm_count, stream);
    });
}

adama_status adama_fold_apply_multi(adama_ctx *ctx, const void *const *grads, adama_dtype gdt,
                                    float *const *w, float *const *m, float *const *v,
                                    void *const *w_bf16, const size_t *n, int count, double lr,
                                    const float *grad_factor, void *cuda_stream) {
    return fold_apply_impl(ctx, grads, gdt, w, m, v, nullptr, w_bf16, n, count, lr, grad_factor, cuda_stream);
}

adama_status adama_fold_apply8_multi(adama_ctx *ctx, const void *const *grads, adama_dtype gdt,
                                     float *const *w, const adama_state8 *states, void *const *w_bf16,
                                     const size_t *n, int count, double lr, const float *grad_factor,
                                     void *cuda_stream) {
    static const adama_state8 none = {nullptr, nullptr, nullptr, nullptr};
    if (ctx && count > 0 && !states)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_apply8: null list of states");
    return fold_apply_impl(ctx, grads, gdt, w, nullptr, nullptr, states ? states : &none, w_bf16, n, count, lr,
                           grad_factor, cuda_stream);
}

static adama_status state8_convert(adama_ctx *ctx, bool pack, float *const *m, float *const *v,
                                   const adama_state8 *states, const size_t *n, int count,
                                   void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && (!m || !v || !states || !n)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "state8: null list or negative count");
    for (int i = 0; i < count; ++i) {
        if (n[i] > 0 && (!m[i] || !v[i])) return fail(ctx, ADAMA_ERR_INVALID_ARG, "state8: null pointer");
        if (!aligned_to(m[i], 4) || !aligned_to(v[i], 4))
            return fail(ctx, ADAMA_ERR_MISALIGNED, "state8: moments not aligned to 4 bytes");
        adama_status st = check_state8(ctx, states[i], n[i]);
        if (st != ADAMA_OK) return st;
    }
    DeviceGuard guard(ctx->cfg.device);
    adama::StepList list;
    list.m = m;
    list.v = v;
    list.s8 = states;
    list.n = n;
    return for_ranges(ctx, count, adama::kStep8Max, "state8 launch", [&](int first, int k) {
        if (!any_element(n, first, k)) return cudaSuccess;
        ctx->launches += 1;
        return adama::launch_state8_convert(list, pack, first, k, ctx->sm_count,
                                            static_cast<cudaStream_t>(cuda_stream));
    });
}

adama_status adama_state8_pack_multi(adama_ctx *ctx, const float *const *m, const float *const *v,
                                     const adama_state8 *states, const size_t *n, int count,
                                     void *cuda_stream) {
    // the kernel only reads m and v in this direction
    return state8_convert(ctx, true, const_cast<float *const *>(m), const_cast<float *const *>(v), states, n,
                          count, cuda_stream);
}

adama_status adama_state8_unpack_multi(adama_ctx *ctx, const adama_state8 *states, float *const *m,
                                       float *const *v, const size_t *n, int count, void *cuda_stream) {
    return state8_convert(ctx, false, m, v, states, n, count, cuda_stream);
}

adama_status adama_grad_norm_multi(adama_ctx *ctx, const void *const *grads, adama_dtype gdt,
                                   const size_t *n, int count, double max_norm, int accumulate,
                                   adama_grad_norm *out, void *workspace, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (count < 0 || (count > 0 && (!grads || !n)) || !out || !workspace)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "grad_norm: null pointer or negative count");
    if (gdt != ADAMA_F32 && gdt != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "grad_norm: unknown gradient dtype");
    if (!(max_norm > 0.0)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "grad_norm: max_norm must be > 0");
    if (!aligned_to(out, 8) || !aligned_to(workspace, 16))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "grad_norm: out needs 8-byte, workspace 16-byte alignment");
    for (int i = 0; i < count; ++i) {
        if (n[i] > 0 && !grads[i]) return fail(ctx, ADAMA_ERR_INVALID_ARG, "grad_norm: null pointer");
        if (!aligned_to(grads[i], dtype_size(gdt)))
            return fail(ctx, ADAMA_ERR_MISALIGNED, "grad_norm: pointer not aligned to its element size");
    }
    DeviceGuard guard(ctx->cfg.device);
    auto launch = [&](int first, int k) {
        ctx->launches += 1;
        return adama::launch_grad_norm(grads + first, gdt, n + first, k, (float)max_norm,
                                       accumulate || first > 0, out, workspace, ctx->sm_count,
                                       static_cast<cudaStream_t>(cuda_stream));
    };
    if (count == 0) {  // still writes the result of the empty sum
        static const void *const no_grads[1] = {nullptr};
        static const size_t no_n[1] = {0};
        grads = no_grads;
        n = no_n;
        count = 1;
    }
    return for_ranges(ctx, count, adama::kNormMax, "grad_norm launch", launch);
}

static adama_status check_logits(adama_ctx *ctx, const void *logits, adama_dtype dt, int64_t rows,
                                 int64_t vocab, int64_t ld, const int64_t *targets, double logit_scale) {
    if (rows < 0 || vocab < 1 || vocab > INT32_MAX || ld < vocab)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "logits: bad shape or a row pitch smaller than the row");
    if (rows > INT32_MAX) return fail(ctx, ADAMA_ERR_UNSUPPORTED, "logits: more than 2^31-1 rows");
    if (dt != ADAMA_F32 && dt != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "logits: unknown dtype");
    if (rows > 0 && (!logits || !targets)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "logits: null pointer");
    // the exponentials are taken to base 2: their factor, logit_scale*log2(e), has to be an fp32 number
    if (!(logit_scale > 0.0) || !(logit_scale * 1.4426950408889634 <= FLT_MAX))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "logits: logit_scale must be > 0 and at most 2.3e38");
    if (!aligned_to(logits, dtype_size(dt)) || !aligned_to(targets, 8))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "logits: pointer not aligned to its element size");
    return ADAMA_OK;
}

adama_status adama_token_logprobs(adama_ctx *ctx, const void *logits, adama_dtype dt, int64_t rows,
                                  int64_t vocab, int64_t ld, const int64_t *targets, double logit_scale,
                                  float *logp, float *lse, float *entropy, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    adama_status st = check_logits(ctx, logits, dt, rows, vocab, ld, targets, logit_scale);
    if (st != ADAMA_OK) return st;
    if (rows > 0 && !logp) return fail(ctx, ADAMA_ERR_INVALID_ARG, "token_logprobs: null output");
    if (!aligned_to(logp, 4) || !aligned_to(lse, 4) || !aligned_to(entropy, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "token_logprobs: output not aligned to 4 bytes");
    if (rows == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    adama::LogprobArgs a;
    a.logits = logits;
    a.dtype = dt;
    a.rows = rows;
    a.vocab = vocab;
    a.ld = ld;
    a.targets = targets;
    a.scale = logit_scale;
    a.logp = logp;
    a.lse = lse;
    a.entropy = entropy;
    a.status = ctx->status_dev;
    cudaError_t e = adama::launch_token_logprobs(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "token_logprobs launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_policy_loss(adama_ctx *ctx, const adama_policy_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: null arguments");
    adama_status st = check_logits(ctx, p->logits, p->logits_dtype, p->rows, p->vocab, p->ld_logits,
                                   p->targets, p->logit_scale);
    if (st != ADAMA_OK) return st;
    if (p->dlogits_dtype != ADAMA_F32 && p->dlogits_dtype != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: unknown gradient dtype");
    if (!p->stats || !p->workspace ||
        (p->rows > 0 && (!p->old_logp || !p->advantages || !p->weights)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: null pointer");
    if (p->dlogits && p->ld_dlogits < p->vocab)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: row pitch of dlogits smaller than the row");
    if (p->dlogits == p->logits && p->rows > 0 &&
        (p->dlogits_dtype != p->logits_dtype || p->ld_dlogits != p->ld_logits))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: in place needs one dtype and one pitch");
    if (!(p->clip_low >= 0.0) || !(p->clip_low <= 1.0) || !(p->clip_high >= 0.0) || !isfinite(p->kl_coef))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "policy_loss: clip range or kl_coef out of range");
    if (!aligned_to(p->dlogits, dtype_size(p->dlogits_dtype)) || !aligned_to(p->old_logp, 4) ||
        !aligned_to(p->ref_logp, 4) || !aligned_to(p->advantages, 4) || !aligned_to(p->weights, 4) ||
        !aligned_to(p->logp, 4) || !aligned_to(p->stats, 4) || !aligned_to(p->workspace, 16))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "policy_loss: pointer not aligned");
    DeviceGuard guard(ctx->cfg.device);
    adama::PolicyArgs a;
    a.logits = p->logits;
    a.dlogits = p->dlogits;
    a.logits_dtype = p->logits_dtype;
    a.dlogits_dtype = p->dlogits_dtype;
    a.rows = p->rows;
    a.vocab = p->vocab;
    a.ld_logits = p->ld_logits;
    a.ld_dlogits = p->ld_dlogits;
    a.targets = p->targets;
    a.old_logp = p->old_logp;
    a.ref_logp = p->ref_logp;
    a.advantages = p->advantages;
    a.weights = p->weights;
    a.scale_exact = p->logit_scale;
    a.scale = (float)p->logit_scale;
    a.ratio_min = (float)(1.0 - p->clip_low);
    a.ratio_max = (float)(1.0 + p->clip_high);
    a.kl_coef = (float)p->kl_coef;
    a.logp = p->logp;
    a.stats = p->stats;
    a.workspace = p->workspace;
    a.status = ctx->status_dev;
    cudaError_t e = adama::launch_policy_loss(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "policy_loss launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_distill_loss(adama_ctx *ctx, const adama_distill_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: null arguments");
    // (the entries' indices stand where the targets of the other calls do)
    adama_status st = check_logits(ctx, p->logits, p->logits_dtype, p->rows, p->vocab, p->ld_logits, p->ids, p->logit_scale);
    if (st != ADAMA_OK) return st;
    if ((p->dlogits_dtype != ADAMA_F32 && p->dlogits_dtype != ADAMA_BF16) ||
        (p->teacher_dtype != ADAMA_F32 && p->teacher_dtype != ADAMA_BF16))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: unknown dtype");
    if (!p->stats || !p->workspace || (p->rows > 0 && (!p->teacher_logits || !p->weights || !p->scratch)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: null pointer");
    if (p->top < 1) return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: a row needs an entry");
    if (p->top > ADAMA_DISTILL_TOP) return fail(ctx, ADAMA_ERR_UNSUPPORTED, "distill_loss: more than 128 entries in a row");
    if (p->ld_teacher < p->top || p->ld_ids < p->top || (p->dlogits && p->ld_dlogits < p->vocab))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: a row pitch smaller than the row");
    if (p->dlogits == p->logits && p->rows > 0 &&
        (p->dlogits_dtype != p->logits_dtype || p->ld_dlogits != p->ld_logits))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "distill_loss: in place needs one dtype and one pitch");
    if (!aligned_to(p->dlogits, dtype_size(p->dlogits_dtype)) || !aligned_to(p->teacher_logits, dtype_size(p->teacher_dtype)) ||
        !aligned_to(p->teacher_lse, 4) || !aligned_to(p->weights, 4) || !aligned_to(p->loss, 4) || !aligned_to(p->stats, 4) ||
        !aligned_to(p->workspace, 16) || !aligned_to(p->scratch, 16))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "distill_loss: pointer not aligned");
    DeviceGuard guard(ctx->cfg.device);
    adama::DistillArgs a = {};
    a.logits = p->logits;
    a.dlogits = p->dlogits;
    a.logits_dtype = p->logits_dtype;
    a.dlogits_dtype = p->dlogits_dtype;
    a.teacher_dtype = p->teacher_dtype;
    a.top = p->top;
    a.rows = p->rows;
    a.vocab = p->vocab;
    a.ld_logits = p->ld_logits;
    a.ld_dlogits = p->ld_dlogits;
    a.ld_teacher = p->ld_teacher;
    a.ld_ids = p->ld_ids;
    a.teacher = p->teacher_logits;
    a.ids = p->ids;
    a.teacher_lse = p->teacher_lse;
    a.weights = p->weights;
    a.scale_exact = p->logit_scale;
    a.scale = (float)p->logit_scale;
    a.loss = p->loss;
    a.stats = p->stats;
    a.workspace = p->workspace;
    a.status = ctx->status_dev;
    int launches = 0;
    cudaError_t e = adama::launch_distill_loss(a, p->scratch, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream), &launches);
    ctx->launches += launches;
    return e == cudaSuccess ? ADAMA_OK : cuda_fail(ctx, "distill_loss launch", e);
}

size_t adama_distill_scratch(const adama_ctx *ctx, int64_t rows, int64_t top) {
    if (!ctx || rows < 0 || rows > INT32_MAX || top < 1 || top > ADAMA_DISTILL_TOP) return 0;
    return adama::distill_scratch_bytes(rows, (int)top);
}

// ---- norms and embeddings ---------------------------------------------------------------------

// A [rows, cols] matrix of a call: what is wrong with it, or OK.
static adama_status check_matrix(adama_ctx *ctx, const char *call, const char *name, const void *p, adama_dtype dt,
                                 int64_t rows, int64_t cols, int64_t ld) {
    char msg[160];
    adama_status st = ADAMA_OK;
    const char *what = "";
    if (dt != ADAMA_F32 && dt != ADAMA_BF16) {
        st = ADAMA_ERR_INVALID_ARG;
        what = "has an unknown dtype";
    } else if (rows > 0 && !p) {
        st = ADAMA_ERR_INVALID_ARG;
        what = "is a null pointer";
    } else if (ld < cols) {
        st = ADAMA_ERR_INVALID_ARG;
        what = "has a row pitch smaller than the row";
    } else if (rows > 0 && ld > INT64_MAX / 8 / rows) {
        st = ADAMA_ERR_UNSUPPORTED;
        what = "is larger than the address space";
    } else if (!aligned_to(p, dtype_size(dt))) {
        st = ADAMA_ERR_MISALIGNED;
        what = "is not aligned to its element size";
    }
    if (st == ADAMA_OK) return st;
    snprintf(msg, sizeof(msg), "%s: %s %s", call, name, what);
    return fail(ctx, st, msg);
}

static adama_status check_rows(adama_ctx *ctx, const char *call, int64_t rows, int64_t dim) {
    char msg[96];
    const bool large = rows > INT32_MAX || dim > INT32_MAX / 2;
    if (rows >= 0 && dim >= 1 && !large) return ADAMA_OK;
    snprintf(msg, sizeof(msg), large ? "%s: 2^31 rows or 2^30 columns or more" : "%s: bad shape", call);
    return fail(ctx, large ? ADAMA_ERR_UNSUPPORTED : ADAMA_ERR_INVALID_ARG, msg);
}

adama_status adama_layer_norm(adama_ctx *ctx, const adama_layer_norm_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm: null arguments");
    adama_status st = check_rows(ctx, "layer_norm", p->rows, p->dim);
    if (st == ADAMA_OK) st = check_matrix(ctx, "layer_norm", "x", p->x, p->x_dtype, p->rows, p->dim, p->ld_x);
    if (st == ADAMA_OK) st = check_matrix(ctx, "layer_norm", "y", p->y, p->y_dtype, p->rows, p->dim, p->ld_y);
    if (st != ADAMA_OK) return st;
    if (!p->weight) return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm: null weight");
    if (!(p->eps >= 0.0) || !(p->eps <= FLT_MAX)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm: eps must be finite and >= 0");
    if (p->y == p->x && p->rows > 0 && (p->y_dtype != p->x_dtype || p->ld_y != p->ld_x))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm: in place needs one dtype and one pitch");
    if (!aligned_to(p->weight, 4) || !aligned_to(p->bias, 4) || !aligned_to(p->mean, 4) || !aligned_to(p->rstd, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "layer_norm: pointer not aligned to 4 bytes");
    if (p->rows == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    adama::NormArgs a;
    a.x = p->x;
    a.y = p->y;
    a.x_dtype = p->x_dtype;
    a.y_dtype = p->y_dtype;
    a.rows = p->rows;
    a.ld_x = p->ld_x;
    a.ld_y = p->ld_y;
    a.dim = (int)p->dim;
    a.weight = p->weight;
    a.bias = p->bias;
    a.eps = (float)p->eps;
    a.inv_dim = (float)(1.0 / (double)p->dim);
    a.mean = p->mean;
    a.rstd = p->rstd;
    cudaError_t e = adama::launch_layer_norm(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "layer_norm launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

size_t adama_layer_norm_workspace(const adama_ctx *ctx, int64_t rows, int64_t dim) {
    if (!ctx || rows < 0 || rows > INT32_MAX || dim < 1 || dim > INT32_MAX / 2) return 0;
    return adama::norm_workspace_bytes(rows, (int)dim, ctx->sm_count);
}

adama_status adama_layer_norm_backward(adama_ctx *ctx, const adama_layer_norm_backward_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm_backward: null arguments");
    const char *const call = "layer_norm_backward";
    adama_status st = check_rows(ctx, call, p->rows, p->dim);
    if (st == ADAMA_OK) st = check_matrix(ctx, call, "dy", p->dy, p->dy_dtype, p->rows, p->dim, p->ld_dy);
    if (st == ADAMA_OK) st = check_matrix(ctx, call, "x", p->x, p->x_dtype, p->rows, p->dim, p->ld_x);
    if (st == ADAMA_OK && p->dx) st = check_matrix(ctx, call, "dx", p->dx, p->x_dtype, p->rows, p->dim, p->ld_dx);
    if (st != ADAMA_OK) return st;
    if (!p->weight || (p->rows > 0 && (!p->mean || !p->rstd)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm_backward: null weight, mean or rstd");
    if ((p->m_weight == nullptr) != (p->v_weight == nullptr) || (p->m_bias == nullptr) != (p->v_bias == nullptr))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm_backward: moments are given in pairs");
    const bool fold = p->m_weight || p->m_bias, params = fold || p->dweight || p->dbias;
    if (fold && ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "layer_norm_backward: adama_begin_minibatch has not been called");
    if (p->rows > 0 && p->dx &&
        ((p->dx == p->x && p->ld_dx != p->ld_x) || (p->dx == p->dy && (p->dy_dtype != p->x_dtype || p->ld_dx != p->ld_dy))))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm_backward: in place needs one dtype and one pitch");
    const void *const singles[] = {p->weight, p->mean, p->rstd, p->dweight, p->dbias, p->m_weight, p->v_weight, p->m_bias, p->v_bias};
    for (const void *q : singles)
        if (!aligned_to(q, 4)) return fail(ctx, ADAMA_ERR_MISALIGNED, "layer_norm_backward: pointer not aligned to 4 bytes");
    if (!aligned_to(p->workspace, 16)) return fail(ctx, ADAMA_ERR_MISALIGNED, "layer_norm_backward: workspace needs 16-byte alignment");
    if (!p->workspace && (params || p->dim > 8192))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "layer_norm_backward: null workspace");
    if (!params && (!p->dx || p->rows == 0)) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    adama::NormBackArgs a;
    a.dy = p->dy;
    a.x = p->x;
    a.dx = p->dx;
    a.dy_dtype = p->dy_dtype;
    a.x_dtype = p->x_dtype;
    a.rows = p->rows;
    a.ld_dy = p->ld_dy;
    a.ld_x = p->ld_x;
    a.ld_dx = p->ld_dx;
    a.dim = (int)p->dim;
    a.weight = p->weight;
    a.mean = p->mean;
    a.rstd = p->rstd;
    a.inv_dim = (float)(1.0 / (double)p->dim);
    a.dweight = p->dweight;
    a.dbias = p->dbias;
    a.m_weight = p->m_weight;
    a.v_weight = p->v_weight;
    a.m_bias = p->m_bias;
    a.v_bias = p->v_bias;
    a.fold = ctx->fold_c;
    a.workspace = p->workspace;
    a.parts = params ? static_cast<float *>(p->workspace) : nullptr;
    int launches = 0;
    cudaError_t e = adama::launch_layer_norm_backward(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream), &launches);
    ctx->launches += launches;
    return e == cudaSuccess ? ADAMA_OK : cuda_fail(ctx, "layer_norm_backward launch", e);
}

adama_status adama_embedding(adama_ctx *ctx, const adama_embedding_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding: null arguments");
    adama_status st = check_rows(ctx, "embedding", p->tokens, p->dim);
    if (st == ADAMA_OK && (p->vocab < 1 || p->vocab >= INT32_MAX))
        st = fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding: vocab must be from 1 to 2^31-2");
    if (st == ADAMA_OK) st = check_matrix(ctx, "embedding", "table", p->table, p->table_dtype, p->vocab, p->dim, p->ld_table);
    if (st == ADAMA_OK) st = check_matrix(ctx, "embedding", "out", p->out, p->out_dtype, p->tokens, p->dim, p->ld_out);
    if (st != ADAMA_OK) return st;
    if (p->tokens > 0 && !p->ids) return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding: null ids");
    if (!aligned_to(p->ids, 8)) return fail(ctx, ADAMA_ERR_MISALIGNED, "embedding: ids not aligned to 8 bytes");
    if (!isfinite(p->scale) || !(fabs(p->scale) <= FLT_MAX))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding: scale must be a finite 32-bit number");
    if (p->tokens == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    adama::EmbeddingArgs a;
    a.ids = p->ids;
    a.table = p->table;
    a.out = p->out;
    a.table_dtype = p->table_dtype;
    a.out_dtype = p->out_dtype;
    a.tokens = p->tokens;
    a.vocab = p->vocab;
    a.ld_table = p->ld_table;
    a.ld_out = p->ld_out;
    a.dim = (int)p->dim;
    a.scale = (float)p->scale;
    a.status = ctx->status_dev;
    cudaError_t e = adama::launch_embedding(a, static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "embedding launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

constexpr int64_t kEmbeddingDim = 1 << 23;  // of the gradient: its sums are joined in a grid with a row for 256 columns

size_t adama_embedding_workspace(const adama_ctx *ctx, int64_t tokens, int64_t dim) {
    if (!ctx || tokens < 0 || tokens > INT32_MAX || dim < 1 || dim > kEmbeddingDim) return 0;
    return adama::embedding_workspace_bytes(tokens, (int)dim, ctx->sm_count);
}

adama_status adama_embedding_grad(adama_ctx *ctx, const adama_embedding_grad_args *p, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!p) return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding_grad: null arguments");
    const char *const call = "embedding_grad";
    adama_status st = check_rows(ctx, call, p->tokens, p->dim);
    if (st == ADAMA_OK && p->dim > kEmbeddingDim) st = fail(ctx, ADAMA_ERR_UNSUPPORTED, "embedding_grad: more than 2^23 columns");
    if (st == ADAMA_OK && (p->vocab < 1 || p->vocab >= INT32_MAX))
        st = fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding_grad: vocab must be from 1 to 2^31-2");
    if (st == ADAMA_OK) st = check_matrix(ctx, call, "dy", p->dy, p->dy_dtype, p->tokens, p->dim, p->ld_dy);
    if (st != ADAMA_OK) return st;
    const bool fold = p->m || p->v;
    if (fold ? !p->m || !p->v || p->grad || p->accumulate : !p->grad)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding_grad: either grad or both moments are given");
    const adama_dtype dt = fold ? ADAMA_F32 : p->grad_dtype;
    st = check_matrix(ctx, call, fold ? "m" : "grad", fold ? p->m : p->grad, dt, p->vocab, p->dim, p->ld_grad);
    if (st == ADAMA_OK && fold) st = check_matrix(ctx, call, "v", p->v, dt, p->vocab, p->dim, p->ld_grad);
    if (st != ADAMA_OK) return st;
    if (fold && ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "embedding_grad: adama_begin_minibatch has not been called");
    if (p->tokens > 0 && (!p->ids || !p->workspace)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding_grad: null ids or workspace");
    if (!aligned_to(p->ids, 8) || !aligned_to(p->workspace, 16))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "embedding_grad: ids need 8-byte, workspace 16-byte alignment");
    if (!isfinite(p->scale) || !(fabs(p->scale) <= FLT_MAX))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "embedding_grad: scale must be a finite 32-bit number");
    DeviceGuard guard(ctx->cfg.device);
    adama::EmbeddingGradArgs a = {};
    a.ids = p->ids;
    a.dy = p->dy;
    a.dy_dtype = p->dy_dtype;
    a.grad_dtype = dt;
    a.tokens = p->tokens;
    a.vocab = p->vocab;
    a.ld_dy = p->ld_dy;
    a.ld_grad = p->ld_grad;
    a.dim = (int)p->dim;
    a.scale = (float)p->scale;
    a.accumulate = p->accumulate != 0;
    a.grad = p->grad;
    a.m = p->m;
    a.v = p->v;
    a.fold = ctx->fold_c;
    a.workspace = p->workspace;
    a.status = ctx->status_dev;
    int launches = 0;
    cudaError_t e = adama::launch_embedding_grad(a, ctx->sm_count, static_cast<cudaStream_t>(cuda_stream), &launches);
    ctx->launches += launches;
    return e == cudaSuccess ? ADAMA_OK : cuda_fail(ctx, "embedding_grad launch", e);
}

// ---- host-buffer variants -------------------------------------------------------------------

adama_status adama_fold_host(adama_ctx *ctx, const void *grad_host, adama_dtype gdt, float *m,
                             float *v, size_t n, void *staging, size_t staging_bytes,
                             void *cuda_stream) {
    adama_status st = check_fold_args(ctx, grad_host, gdt, m, v, n);
    if (st != ADAMA_OK) return st;
    if (n == 0) return ADAMA_OK;
    if (!staging || staging_bytes < (2u << 20))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "fold_host: staging buffer smaller than 2 MiB");
    if (!aligned_to(staging, 256))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "fold_host: staging must be 256-byte aligned");
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const size_t esz = dtype_size(gdt);
    // two halves, each a multiple of 256 bytes, so every chunk keeps m, v and grad 16-byte aligned
    const size_t half_bytes = (staging_bytes / 2) & ~(size_t)255;
    const size_t chunk = half_bytes / esz;
    char *half[2] = {static_cast<char *>(staging), static_cast<char *>(staging) + half_bytes};
    const char *src = static_cast<const char *>(grad_host);

    // the staging buffer may still be in use by earlier work on `stream`
    cudaError_t e = cudaEventRecord(ctx->ev_entry, stream);
    if (e == cudaSuccess) e = cudaStreamWaitEvent(ctx->copy_stream, ctx->ev_entry, 0);
    size_t done = 0;
    for (int it = 0; done < n && e == cudaSuccess; ++it) {
        const int h = it & 1;
        const size_t cnt = (n - done < chunk) ? (n - done) : chunk;
        if (it >= 2) e = cudaStreamWaitEvent(ctx->copy_stream, ctx->ev_folded[h], 0);
        if (e == cudaSuccess)
            e = cudaMemcpyAsync(half[h], src + done * esz, cnt * esz, cudaMemcpyHostToDevice,
                                ctx->copy_stream);
        if (e == cudaSuccess) e = cudaEventRecord(ctx->ev_copied[h], ctx->copy_stream);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(stream, ctx->ev_copied[h], 0);
        if (e == cudaSuccess) {
            e = adama::launch_fold(half[h], gdt, m + done, v + done, cnt, ctx->fold_c,
                                   ctx->sm_count, stream);
            ctx->launches += 1;
        }
        if (e == cudaSuccess) e = cudaEventRecord(ctx->ev_folded[h], stream);
        done += cnt;
    }
    if (e != cudaSuccess) return cuda_fail(ctx, "fold_host", e);
    return ADAMA_OK;
}

adama_status adama_linear_wgrad_fold_host(adama_ctx *ctx, const void *X_host, const void *dY_host,
                                          int tokens, int d_in, int d_out, float *m, float *v,
                                          int64_t ldmv, void *staging, size_t staging_bytes,
                                          void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (tokens < 0 || d_in < 1 || d_out < 1)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold_host: bad shape");
    if (d_in % 8 || d_out % 8)
        return fail(ctx, ADAMA_ERR_MISALIGNED,
                    "wgrad_fold_host: dense rows need d_in, d_out multiples of 8");
    const size_t x_bytes = (size_t)tokens * d_in * 2, y_bytes = (size_t)tokens * d_out * 2;
    const size_t y_off = (x_bytes + 255) & ~(size_t)255;
    if (!staging || staging_bytes < y_off + y_bytes)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold_host: staging buffer too small");
    if (!aligned_to(staging, 256))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "wgrad_fold_host: staging must be 256-byte aligned");
    char *Xd = static_cast<char *>(staging), *Yd = Xd + y_off;
    adama_status st = check_wgrad_args(ctx, Xd, Yd, tokens, d_in, d_out, d_in, d_out, m, v, ldmv);
    if (st != ADAMA_OK) return st;
    if (tokens == 0) return ADAMA_OK;
    if (!X_host || !dY_host) return fail(ctx, ADAMA_ERR_INVALID_ARG, "wgrad_fold_host: null pointer");
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = cudaMemcpyAsync(Xd, X_host, x_bytes, cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaMemcpyAsync(Yd, dY_host, y_bytes, cudaMemcpyHostToDevice, stream);
    if (e != cudaSuccess) return cuda_fail(ctx, "wgrad_fold_host copy", e);
    return adama_linear_wgrad_fold(ctx, Xd, Yd, tokens, d_in, d_out, d_in, d_out, m, v, ldmv,
                                   cuda_stream);
}

adama_status adama_apply_to_host(adama_ctx *ctx, float *w, float *m, float *v, size_t n, double lr,
                                 float *w_host, void *cuda_stream) {
    if (ctx && n > 0 && !w_host)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "apply_to_host: null host pointer");
    adama_status st = adama_apply(ctx, w, m, v, n, lr, cuda_stream);
    if (st != ADAMA_OK || n == 0) return st;
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (ctx->cfg.flags & ADAMA_ASYNC_COPYBACK) {
        e = cudaEventRecord(ctx->ev_applied, stream);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(ctx->d2h_stream, ctx->ev_applied, 0);
        if (e == cudaSuccess)
            e = cudaMemcpyAsync(w_host, w, n * sizeof(float), cudaMemcpyDeviceToHost, ctx->d2h_stream);
        if (e == cudaSuccess) e = cudaEventRecord(ctx->ev_d2h_done, ctx->d2h_stream);
        if (e == cudaSuccess) ctx->d2h_pending = true;
    } else {
        e = cudaMemcpyAsync(w_host, w, n * sizeof(float), cudaMemcpyDeviceToHost, stream);
    }
    if (e != cudaSuccess) return cuda_fail(ctx, "apply_to_host copy", e);
    return ADAMA_OK;
}

// ---- SGD with momentum on the same pipeline; coefficient statistics ----------------------------

adama_status adama_sgdm_fold(adama_ctx *ctx, const void *grad, adama_dtype gdt, float *buf, size_t n,
                             void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (gdt != ADAMA_F32 && gdt != ADAMA_BF16)
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "sgdm_fold: unknown gradient dtype");
    if (n > 0 && (!grad || !buf)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "sgdm_fold: null pointer");
    if (ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "sgdm_fold: adama_begin_minibatch has not been called");
    if (!aligned_to(grad, dtype_size(gdt)) || !aligned_to(buf, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "sgdm_fold: pointer not aligned to its element size");
    if (n == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    const double N = (ctx->cfg.flags & ADAMA_GRADS_PRESCALED) ? 1.0 : (double)ctx->n_micro;
    cudaError_t e = adama::launch_sgdm_fold(grad, gdt, buf, n, (float)(1.0 / N), ctx->sm_count,
                                            static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "sgdm_fold launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_sgdm_apply(adama_ctx *ctx, float *w, float *buf, size_t n, double lr,
                              double momentum, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (n > 0 && (!w || !buf)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "sgdm_apply: null pointer");
    if (!isfinite(lr)) return fail(ctx, ADAMA_ERR_INVALID_ARG, "sgdm_apply: lr is not finite");
    if (!(momentum >= 0.0) || !(momentum < 1.0))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "sgdm_apply: momentum must be in [0, 1)");
    if (ctx->t < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE, "sgdm_apply: no mini-batch has been started (t == 0)");
    if (!aligned_to(w, 4) || !aligned_to(buf, 4))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "sgdm_apply: pointer not aligned to 4 bytes");
    if (n == 0) return ADAMA_OK;
    DeviceGuard guard(ctx->cfg.device);
    float mu_hi, mu_lo;
    adama::split_hi_lo(momentum, &mu_hi, &mu_lo);
    cudaError_t e = join_copyback(ctx, static_cast<cudaStream_t>(cuda_stream));
    if (e == cudaSuccess)
        e = adama::launch_sgdm_apply(w, buf, n, (float)lr, mu_hi, mu_lo, ctx->sm_count,
                                     static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "sgdm_apply launch", e);
    ctx->launches += 1;
    return ADAMA_OK;
}

adama_status adama_coefficient_stats(adama_ctx *ctx, const float *m, const float *m_begin,
                                     const float *v, float *v_adam, size_t n, double *stats_dev,
                                     void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!stats_dev || (n > 0 && (!m || !v || !v_adam)))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "coefficient_stats: null pointer");
    if (ctx->n_micro < 1)
        return fail(ctx, ADAMA_ERR_BAD_STATE,
                    "coefficient_stats: adama_begin_minibatch has not been called");
    if (!(ctx->cfg.beta1 < 1.0))
        return fail(ctx, ADAMA_ERR_UNSUPPORTED, "coefficient_stats: needs beta1 < 1");
    if (!aligned_to(m, 4) || !aligned_to(v, 4) || !aligned_to(v_adam, 4) ||
        (m_begin && !aligned_to(m_begin, 4)) || !aligned_to(stats_dev, 8))
        return fail(ctx, ADAMA_ERR_MISALIGNED, "coefficient_stats: pointer not aligned");
    DeviceGuard guard(ctx->cfg.device);
    adama::CoefConstants c;
    const double om1 = 1.0 - ctx->cfg.beta1;
    c.k = (float)((1.0 - ctx->cfg.beta2) / (om1 * om1));
    adama::split_hi_lo(ctx->cfg.beta2, &c.beta2_hi, &c.beta2_lo);
    cudaError_t e = adama::launch_coefficient_stats(m, m_begin, v, v_adam, n, c, stats_dev,
                                                    ctx->sm_count,
                                                    static_cast<cudaStream_t>(cuda_stream));
    if (e != cudaSuccess) return cuda_fail(ctx, "coefficient_stats launch", e);
    ctx->launches += (n > 0 ? 2 : 1);
    return ADAMA_OK;
}

// ---- state and diagnostics ------------------------------------------------------------------

int64_t adama_get_step(const adama_ctx *ctx) { return ctx ? ctx->t : -1; }

adama_status adama_set_step(adama_ctx *ctx, int64_t t) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (t < 0) return fail(ctx, ADAMA_ERR_INVALID_ARG, "set_step: t must be >= 0");
    ctx->t = t;
    return ADAMA_OK;
}

int adama_get_n_micro(const adama_ctx *ctx) { return ctx ? ctx->n_micro : -1; }

adama_status adama_set_weight_decay(adama_ctx *ctx, double weight_decay) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (!(weight_decay >= 0.0) || !isfinite(weight_decay))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "set_weight_decay: must be finite and >= 0");
    ctx->weight_decay = weight_decay;
    return ADAMA_OK;
}

adama_status adama_sync_status(adama_ctx *ctx, void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    unsigned host[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    cudaError_t e = join_copyback(ctx, stream);
    if (e == cudaSuccess)
        e = cudaMemcpyAsync(host, ctx->status_dev, sizeof(host), cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return cuda_fail(ctx, "sync_status", e);
    // One report a call, an expired wait first; what is not reported yet stays for the next call.
    const auto clear = [&](int first) {
        cudaError_t c = cudaMemsetAsync(ctx->status_dev + first, 0, 4 * sizeof(unsigned), stream);
        if (c == cudaSuccess) c = cudaStreamSynchronize(stream);
        return c;
    };
    if (host[0] != adama::kDevOk) {
        e = clear(0);
        if (e != cudaSuccess) return cuda_fail(ctx, "sync_status", e);
        snprintf(ctx->err, sizeof(ctx->err),
                 "device-side wait expired in the %s kernel (code %u, wait %u, tile %u)",
                 host[1] == adama::kWaitPolicyRing   ? "policy-loss or distillation"
                 : host[1] == adama::kWaitState8Ring ? "8-bit update"
                 : host[1] == adama::kWaitStepRing   ? "update"
                                                     : "fused weight-gradient",
                 host[0], host[1], host[2]);
        return ADAMA_ERR_TIMEOUT;
    }
    const unsigned *target = host + adama::kStatusTarget;
    if (target[0] != 0) {
        e = clear(adama::kStatusTarget);
        if (e != cudaSuccess) return cuda_fail(ctx, "sync_status", e);
        snprintf(ctx->err, sizeof(ctx->err), "a target, an id or an index lies outside the vocabulary (row %llu of its call)",
                 (unsigned long long)target[2] << 32 | target[1]);
        return ADAMA_ERR_INVALID_ARG;
    }
    return ADAMA_OK;
}

adama_status adama_debug_set_status(adama_ctx *ctx, unsigned code, unsigned wait, unsigned tile,
                                    void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    DeviceGuard guard(ctx->cfg.device);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const unsigned words[4] = {code, wait, tile, 0};
    cudaError_t e = cudaMemcpyAsync(ctx->status_dev, words, sizeof(words), cudaMemcpyHostToDevice, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);  // `words` lives on this stack frame
    if (e != cudaSuccess) return cuda_fail(ctx, "debug_set_status", e);
    return ADAMA_OK;
}

adama_status adama_debug_wgrad_expire_wait(adama_ctx *ctx, const void *X, const void *dY,
                                           int tokens, int d_in, int d_out, int64_t ldx, int64_t ldy,
                                           float *m, float *v, int64_t ldmv, uint64_t wait_limit_ns,
                                           void *cuda_stream) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (wait_limit_ns < 1000 || wait_limit_ns > 1000000000ull || tokens == 0)
        return fail(ctx, ADAMA_ERR_INVALID_ARG,
                    "debug_wgrad_expire_wait: limit must be 1 us .. 1 s and tokens > 0");
    return wgrad_impl(ctx, X, dY, tokens, d_in, d_out, ldx, ldy, m, v, ldmv, nullptr, nullptr,
                      cuda_stream, wait_limit_ns, 1);
}

adama_status adama_debug_set_wgrad_variant(adama_ctx *ctx, int epilogue, int epi_warps,
                                           int box_loads, int no_pdl) {
    if (!ctx) return ADAMA_ERR_INVALID_ARG;
    if (epilogue < 0 || epilogue > 2 || (epi_warps != 0 && epi_warps != 4 && epi_warps != 8) ||
        (box_loads != 0 && box_loads != 1) || (no_pdl != 0 && no_pdl != 1))
        return fail(ctx, ADAMA_ERR_INVALID_ARG, "debug_set_wgrad_variant: value out of range");
    ctx->variant.epilogue = epilogue;
    ctx->variant.epi_warps = epi_warps;
    ctx->variant.box_loads = box_loads;
    ctx->variant.no_pdl = no_pdl;
    return ADAMA_OK;
}

int adama_debug_setup_state(int device) { return adama::wgrad_setup_state(device); }

const char *adama_last_error(const adama_ctx *ctx) { return ctx ? ctx->err : ""; }

uint64_t adama_stream_capture_id(void *cuda_stream) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    unsigned long long id = 0;
    if (cudaStreamGetCaptureInfo(static_cast<cudaStream_t>(cuda_stream), &status, &id) != cudaSuccess) {
        cudaGetLastError();  // e.g. the legacy stream while another one captures: it is not captured itself
        return 0;
    }
    return status == cudaStreamCaptureStatusActive ? id : 0;
}

int64_t adama_launch_count(const adama_ctx *ctx) { return ctx ? ctx->launches : -1; }

adama_status adama_host_constants(const adama_config *cfg, int n_micro, int64_t t, double lr,
                                  float out[9]) {
    return adama_host_constants_allreduced(cfg, n_micro, t, lr, 1, out);
}

adama_status adama_host_constants_sharded(const adama_config *cfg, int n_micro, int64_t t, double lr,
                                          int world_size, float out[9]) {
    adama_status st = adama_host_constants_allreduced(cfg, n_micro, t, lr, world_size, out);
    if (st != ADAMA_OK) return st;
    adama::ApplyConstants c =
        adama::make_apply_constants(cfg->beta1, cfg->beta2, cfg->eps, t, lr, world_size, true);
    out[5] = c.beta1_hi;
    out[6] = c.beta1_lo;
    out[7] = c.beta2_hi;
    out[8] = c.beta2_lo;
    return ADAMA_OK;
}

adama_status adama_host_constants_allreduced(const adama_config *cfg, int n_micro, int64_t t,
                                             double lr, int world_size, float out[9]) {
    if (!config_ok(cfg) || !out || n_micro < 1 || t < 1 || world_size < 1)
        return ADAMA_ERR_INVALID_ARG;
    adama::FoldConstants f = adama::make_fold_constants(cfg->beta1, cfg->beta2, n_micro, cfg->flags);
    adama::ApplyConstants c =
        adama::make_apply_constants(cfg->beta1, cfg->beta2, cfg->eps, t, lr, world_size);
    out[0] = f.a;
    out[1] = f.b;
    out[2] = c.step;
    out[3] = c.inv_bc2;
    out[4] = c.eps;
    out[5] = c.beta1_hi;
    out[6] = c.beta1_lo;
    out[7] = c.beta2_hi;
    out[8] = c.beta2_lo;
    return ADAMA_OK;
}

}  // extern "C"
