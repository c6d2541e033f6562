// Token log-probabilities and the clipped policy loss with its gradient, from rows of logits.
// With z = s*x (s = logit_scale) a row's lse = log sum_j exp(z_j), p_j = exp(z_j - lse),
// logp = z_target - lse, entropy = lse - sum_j p_j z_j.  For a row with weight w:
//     r = exp(logp - old),  pg = -min(r*A, clamp(r, 1-cl, 1+ch)*A),  d = ref - logp,
//     kl = exp(d) - d - 1,  loss += w*(pg + beta*kl)
//     dlogits_j = w*s*c*([j = target] - p_j),  c = -(r*A while r*A <= the clamped product) + beta*(1 - exp(d))
#include <math_constants.h>

#include "adama_device.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

// Softmax statistics of a set of logits, with k = s*log2(e): the largest one, the sum of
// 2^(k*(x - top)) and that of the same times k*(x - top).  The difference is formed first: a common
// offset of the logits, or the lowest value of their type as a mask, then costs neither precision
// nor range.  An empty set, or one of -inf alone, has top = -inf and sums of zero.
struct Stats {
    float top, sum, wsum;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Statistics of a union: both brought to the larger top.
__device__ __forceinline__ Stats join(const Stats &a, const Stats &b, float k) {
    Stats r;
    r.top = fmaxf(a.top, b.top);
    const float da = a.top == r.top ? 0.f : k * (a.top - r.top), db = b.top == r.top ? 0.f : k * (b.top - r.top);
    const float ea = exp2_fast(da), eb = exp2_fast(db);
    r.sum = a.sum * ea + b.sum * eb;
    // an empty side has weight 0 and distance -inf: its product is left out
    r.wsum = (ea > 0.f ? ea * (a.wsum + a.sum * da) : 0.f) + (eb > 0.f ? eb * (b.wsum + b.sum * db) : 0.f);
    return r;
}

template <int N>
__device__ __forceinline__ void add(Stats &s, const float (&x)[N], float k) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    if (top > s.top) {
        const float d = s.top == -CUDART_INF_F ? 0.f : k * (s.top - top), e = exp2_fast(d);
        s.wsum = e > 0.f ? e * (s.wsum + s.sum * d) : 0.f;
        s.sum *= e;
        s.top = top;
    }
    const float ref = s.top == -CUDART_INF_F ? 0.f : s.top;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = k * (x[i] - ref), e = exp2_fast(d);
        s.sum += e;
        s.wsum += e * fmaxf(d, -1e30f);  // -inf has e = 0
    }
}

// eight consecutive logits, widened exactly; the pointer is 16-byte aligned.  Not a read-only load:
// the gradient may be written over the logits.
__device__ __forceinline__ void load_row8(const float *p, float (&x)[8]) {
    const float4 a = ld_stream(reinterpret_cast<const float4 *>(p)), b = ld_stream(reinterpret_cast<const float4 *>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load_row8(const __nv_bfloat16 *p, float (&x)[8]) {
    const float4 t = ld_stream(reinterpret_cast<const float4 *>(p));
    const unsigned u[4] = {__float_as_uint(t.x), __float_as_uint(t.y), __float_as_uint(t.z), __float_as_uint(t.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // bf16 -> fp32 is a 16-bit left shift
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ Stats shfl_join(Stats s, float k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Stats b;
        b.top = __shfl_xor_sync(0xffffffffu, s.top, o);
        b.sum = __shfl_xor_sync(0xffffffffu, s.sum, o);
        b.wsum = __shfl_xor_sync(0xffffffffu, s.wsum, o);
        s = join(s, b, k);
    }
    return s;
}

template <typename T>
__device__ __forceinline__ int head_of_row(const T *x, int64_t vocab) {
    const int mis = (int)((reinterpret_cast<uintptr_t>(x) % 16) / sizeof(T));
    const int64_t head = mis ? 16 / sizeof(T) - mis : 0;
    return (int)(head < vocab ? head : vocab);
}

// Statistics of a whole row by the CTA; every thread gets them.
template <typename T>
__device__ __forceinline__ Stats row_stats(const T *x, int64_t vocab, float k, Stats *shared) {
    Stats s = {-CUDART_INF_F, 0.f, 0.f};
    const int head = head_of_row(x, vocab);
    const int64_t body = (vocab - head) / 8;
    for (int64_t i = threadIdx.x; i < body; i += kThreads) {
        float v[8];
        load_row8(x + head + 8 * i, v);
        add(s, v, k);
    }
    const int64_t tail0 = head + 8 * body;
    for (int64_t i = threadIdx.x; i < head + (vocab - tail0); i += kThreads) {
        const float v[1] = {widen(x[i < head ? i : tail0 + (i - head)])};
        add(s, v, k);
    }
    s = shfl_join(s, k);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = s;
    __syncthreads();
    s = shared[0];
    for (int i = 1; i < kWarps; ++i) s = join(s, shared[i], k);
    __syncthreads();
    return s;
}

__device__ __forceinline__ void record_bad_target(unsigned *status, int64_t row) {
    if (atomicCAS(status, (unsigned)kDevOk, (unsigned)kDevBadTarget) == (unsigned)kDevOk) {
        status[1] = (unsigned)row;
        status[2] = (unsigned)(row >> 32);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
token_logprobs_kernel(const LogprobArgs a, float k) {
    __shared__ Stats shared[kWarps];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t target = a.targets[row];
        const T *x = static_cast<const T *>(a.logits) + row * a.ld;
        float logp = 0.f, lse = 0.f, entropy = 0.f;
        if (target >= 0) {
            const Stats s = row_stats(x, a.vocab, k, shared);
            const float log2sum = log2f(s.sum);
            lse = fmaf(s.top, (float)a.scale, CUDART_LN2_F * log2sum);
            logp = target < a.vocab ? CUDART_LN2_F * (k * (widen(x[target]) - s.top) - log2sum) : CUDART_NAN_F;
            entropy = CUDART_LN2_F * (log2sum - s.wsum / s.sum);
            if (target >= a.vocab && threadIdx.x == 0) record_bad_target(a.status, row);
        }
        if (threadIdx.x == 0) {
            a.logp[row] = logp;
            if (a.lse) a.lse[row] = lse;
            if (a.entropy) a.entropy[row] = entropy;
        }
    }
}

// Loss terms of one row and its slope dloss/dlogp (without weight and scale).
struct Terms {
    float pg, kl, cut, slope;
};
__device__ __forceinline__ Terms loss_terms(float logp, float old, float adv, const float *ref, int64_t row,
                                            const PolicyArgs &a) {
    Terms t;
    const float r = expf(logp - old), plain = r * adv;
    const float clipped = fminf(fmaxf(r, a.ratio_min), a.ratio_max) * adv;
    const bool cut = plain > clipped;
    t.pg = -(cut ? clipped : plain);
    t.cut = cut ? 1.f : 0.f;
    t.slope = cut ? 0.f : -plain;
    t.kl = 0.f;
    if (ref) {
        const float d = ref[row] - logp, e = expf(d);
        t.kl = e - d - 1.f;
        t.slope += a.kl_coef * (1.f - e);
    }
    if (r != r) t.pg = t.slope = r;  // a NaN log-probability stays visible
    return t;
}

template <typename T>
__device__ __forceinline__ void store_out8(T *p, const float (&y)[8]);
template <>
__device__ __forceinline__ void store_out8(float *p, const float (&y)[8]) {
    st_stream(reinterpret_cast<float4 *>(p), make_float4(y[0], y[1], y[2], y[3]));
    st_stream(reinterpret_cast<float4 *>(p) + 1, make_float4(y[4], y[5], y[6], y[7]));
}
template <>
__device__ __forceinline__ void store_out8(__nv_bfloat16 *p, const float (&y)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2_bf16(y[0], y[1]), pack2_bf16(y[2], y[3]),
                                               pack2_bf16(y[4], y[5]), pack2_bf16(y[6], y[7]));
}
__device__ __forceinline__ void store1(float *p, float y) { *p = y; }
__device__ __forceinline__ void store1(__nv_bfloat16 *p, float y) { *p = __float2bfloat16_rn(y); }

template <typename T, typename O>
__global__ void __launch_bounds__(kThreads)
policy_loss_kernel(const PolicyArgs a, float k) {
    __shared__ Stats shared[kWarps];
    __shared__ double sums[4][kWarps];
    __shared__ bool last;
    Workspace *ws = static_cast<Workspace *>(a.workspace);
    double acc[4] = {0.0, 0.0, 0.0, 0.0};  // thread 0's
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t target = a.targets[row];
        const float weight = a.weights[row];
        const T *x = static_cast<const T *>(a.logits) + row * a.ld_logits;
        O *y = a.dlogits ? static_cast<O *>(a.dlogits) + row * a.ld_dlogits : nullptr;
        float logp = 0.f, unit = 0.f, top = 0.f, per_e = 0.f;  // gradient: unit*one-hot + per_e*2^(k*(x - top))
        const bool live = weight != 0.f && target >= 0;
        if (live) {
            const Stats s = row_stats(x, a.vocab, k, shared);
            const float log2sum = log2f(s.sum);
            logp = target < a.vocab ? CUDART_LN2_F * (k * (widen(x[target]) - s.top) - log2sum) : CUDART_NAN_F;
            top = s.top;
            const Terms t = loss_terms(logp, a.old_logp[row], a.advantages[row], a.ref_logp, row, a);
            unit = weight * t.slope * a.scale;
            per_e = -unit / s.sum;
            if (threadIdx.x == 0) {
                acc[0] += (double)weight * (t.pg + (a.ref_logp ? a.kl_coef * t.kl : 0.f));
                acc[1] += (double)weight * t.pg;
                acc[2] += (double)weight * t.kl;
                acc[3] += (double)weight * t.cut;
                if (target >= a.vocab) record_bad_target(a.status, row);
            }
        }
        if (threadIdx.x == 0 && a.logp) a.logp[row] = logp;
        if (!y) continue;
        const int head = head_of_row(x, a.vocab);
        const int64_t body = (a.vocab - head) / 8, tail0 = head + 8 * body;
        const bool wide = reinterpret_cast<uintptr_t>(y + head) % 16 == 0;
        __syncthreads();  // in place: every thread has read the target's logit
        for (int64_t i = threadIdx.x; i < body; i += kThreads) {
            const int64_t j = head + 8 * i;
            float v[8];
            if (live) {
                load_row8(x + j, v);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    v[q] = per_e * exp2_fast(k * (v[q] - top));
                    if (j + q == target) v[q] += unit;
                }
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = 0.f;
            }
            if (wide) {
                store_out8(y + j, v);
            } else {
#pragma unroll
                for (int q = 0; q < 8; ++q) store1(y + j + q, v[q]);
            }
        }
        for (int64_t i = threadIdx.x; i < head + (a.vocab - tail0); i += kThreads) {
            const int64_t j = i < head ? i : tail0 + (i - head);
            float v = live ? per_e * exp2_fast(k * (widen(x[j]) - top)) : 0.f;
            if (live && j == target) v += unit;
            store1(y + j, v);
        }
    }
    // the CTAs' sums, added in their order by the last CTA to finish
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) ws->part[4 * blockIdx.x + i] = acc[i];
        __threadfence();
        last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double all[4] = {0.0, 0.0, 0.0, 0.0};
    for (unsigned b = threadIdx.x; b < gridDim.x; b += kThreads)
        for (int i = 0; i < 4; ++i) all[i] += __ldcg(&ws->part[4 * b + i]);
    for (int i = 0; i < 4; ++i) {
        for (int o = 16; o > 0; o >>= 1) all[i] += __shfl_down_sync(0xffffffffu, all[i], o);
        if (threadIdx.x % 32 == 0) sums[i][threadIdx.x / 32] = all[i];
    }
    __syncthreads();
    if (threadIdx.x < 4) {
        double s = 0.0;
        for (int i = 0; i < kWarps; ++i) s += sums[threadIdx.x][i];
        a.stats[threadIdx.x] = (float)s;
    }
    if (threadIdx.x == 0) ws->ticket = 0;
}

unsigned row_grid(int64_t rows, int sm_count, int per_sm) {
    int64_t cap = (int64_t)sm_count * per_sm;
    if (cap > kWorkspaceParts / 4) cap = kWorkspaceParts / 4;
    return (unsigned)(rows < 1 ? 1 : rows < cap ? rows : cap);
}

constexpr double kLog2e = 1.4426950408889634074;

}  // namespace

cudaError_t launch_token_logprobs(const LogprobArgs &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale * kLog2e);
    const unsigned grid = row_grid(a.rows, sm_count, 4);
    if (a.dtype == ADAMA_F32)
        token_logprobs_kernel<float><<<grid, kThreads, 0, stream>>>(a, k);
    else
        token_logprobs_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(a, k);
    return cudaGetLastError();
}

cudaError_t launch_policy_loss(const PolicyArgs &a, int sm_count, cudaStream_t stream) {
    const float k = (float)(a.scale_exact * kLog2e);
    const unsigned grid = row_grid(a.rows, sm_count, 4);
    if (a.logits_dtype == ADAMA_F32 && a.dlogits_dtype == ADAMA_F32)
        policy_loss_kernel<float, float><<<grid, kThreads, 0, stream>>>(a, k);
    else if (a.logits_dtype == ADAMA_F32)
        policy_loss_kernel<float, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(a, k);
    else if (a.dlogits_dtype == ADAMA_F32)
        policy_loss_kernel<__nv_bfloat16, float><<<grid, kThreads, 0, stream>>>(a, k);
    else
        policy_loss_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(a, k);
    return cudaGetLastError();
}

}  // namespace adama
