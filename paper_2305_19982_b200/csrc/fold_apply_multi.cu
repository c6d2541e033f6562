// The mini-batch's last fold and its update in ONE pass over many tensors (Algorithm 2: the inner
// loop body for the last micro-batch, "Update", and the decay of the next mini-batch):
//     m += a*g,  v += b*g^2,  w -= step*m/(sqrt(v*inv_bc2) + eps),  m *= beta1,  v *= beta2
// with g times an optional factor (gradient clipping) that lies in device memory.  With one
// micro-batch a mini-batch this is a whole AdamW step: 26 B/param (bf16 gradient) instead of the
// 18 + 24 of a fold and an apply.  Same arithmetic as those two, bit for bit.
// Bound by HBM: 369 M parameters in 144 tensors (bf16 gradients, 9.6 GB) take 1478-1504 us = 6.38-6.49 TB/s, 99 to
// 100 % of a copy's rate; 30.7 M with the bf16 copy 135.5 us (97 %).  A list too short to stream is one launch's
// latency: 64 tensors of 1600 to 6400 elements 2.9 us.
#include "adama_device.cuh"
#include "bulk_copy.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kChunk / (4 * kThreads);  // float4 groups of one thread in a chunk
constexpr unsigned char kScalar = 255;            // no common alignment: element by element

template <int CAP>
struct StepTable {
    const void *g[CAP];
    float *w[CAP];
    float *m[CAP];
    float *v[CAP];
    __nv_bfloat16 *copy[CAP];  // entries may be null
    unsigned long long n[CAP];
    unsigned chunk_start[CAP + 1];
    unsigned char head[CAP];  // elements before the vector accesses begin (0..7), or kScalar
    unsigned char bulk[CAP];  // 1: the gradient is 16-byte aligned there too
    int count;
};
static_assert(sizeof(StepTable<kStepMax>) <= 32000, "table must fit the kernel parameter space");

struct Group {
    Grad4 g;
    float4 w, m, v;
};

__device__ __forceinline__ void step1(float g, float &w, float &m, float &v, const FoldConstants &f,
                                      const ApplyConstants &c) {
    fold1(g, m, v, f.a, f.b);
    apply1(w, m, v, c);
}

template <typename G>
__device__ __forceinline__ void scalar_element(const G *g, float *w, float *m, float *v,
                                               __nv_bfloat16 *copy, size_t i, float factor,
                                               const FoldConstants &f, const ApplyConstants &c) {
    float wi = w[i], mi = m[i], vi = v[i];
    step1(widen(g[i]) * factor, wi, mi, vi, f, c);
    w[i] = wi;
    m[i] = mi;
    v[i] = vi;
    if (copy) copy[i] = __float2bfloat16_rn(wi);
}

// Elements [i, end) at a distance of `stride`, four of them on their way at a time.
template <typename G>
__device__ __forceinline__ void scalar_run(const G *g, float *w, float *m, float *v, __nv_bfloat16 *copy, size_t i, size_t end,
                                           size_t stride, float factor, const FoldConstants &f, const ApplyConstants &c) {
    for (; i < end; i += 4 * stride) {
        float gg[4], ww[4], mm[4], vv[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const size_t j = i + q * stride;
            if (j < end) {
                gg[q] = widen(g[j]);
                ww[q] = w[j];
                mm[q] = m[j];
                vv[q] = v[j];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const size_t j = i + q * stride;
            if (j < end) {
                step1(gg[q] * factor, ww[q], mm[q], vv[q], f, c);
                w[j] = ww[q];
                m[j] = mm[q];
                v[j] = vv[q];
                if (copy) copy[j] = __float2bfloat16_rn(ww[q]);
            }
        }
    }
}

__device__ __forceinline__ void step4(const Grad4 &g, float factor, float4 &x, float4 &y, float4 &z, const FoldConstants &f,
                                      const ApplyConstants &c) {
    step1(g.x * factor, x.x, y.x, z.x, f, c);
    step1(g.y * factor, x.y, y.y, z.y, f, c);
    step1(g.z * factor, x.z, y.z, z.z, f, c);
    step1(g.w * factor, x.w, y.w, z.w, f, c);
}
__device__ __forceinline__ void store4(float *w, float *m, float *v, __nv_bfloat16 *copy, size_t i, const float4 &x,
                                       const float4 &y, const float4 &z) {
    st_stream(reinterpret_cast<float4 *>(w + i), x);
    st_stream(reinterpret_cast<float4 *>(m + i), y);
    st_stream(reinterpret_cast<float4 *>(v + i), z);
    if (copy) *reinterpret_cast<uint2 *>(copy + i) = make_uint2(pack2_bf16(x.x, x.y), pack2_bf16(x.z, x.w));
}

// Short lists: straight from global memory, all loads of a chunk first.
template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
fold_apply_multi_kernel(const __grid_constant__ StepTable<CAP> tab, FoldConstants f, ApplyConstants c,
                        const float *__restrict__ factor_ptr) {
    const float factor = factor_ptr ? *factor_ptr : 1.f;
    if (factor != factor) return;  // a NaN factor (non-finite gradient norm) skips the step
    const unsigned total = tab.chunk_start[tab.count];
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t k = chunk - tab.chunk_start[t], n = (size_t)tab.n[t];
        const G *g = static_cast<const G *>(tab.g[t]);
        float *w = tab.w[t], *m = tab.m[t], *v = tab.v[t];
        __nv_bfloat16 *copy = tab.copy[t];
        const unsigned char head = tab.head[t];
        if (head == kScalar) {
            const size_t end = (k + 1) * kChunk < n ? (k + 1) * kChunk : n;
            scalar_run(g, w, m, v, copy, k * kChunk + threadIdx.x, end, kThreads, factor, f, c);
            continue;
        }
        if (k == 0 && threadIdx.x < head && threadIdx.x < n) scalar_element(g, w, m, v, copy, threadIdx.x, factor, f, c);
        const size_t base = head + k * kChunk + 4 * threadIdx.x;
        Group r[kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const size_t i = base + (size_t)u * 4 * kThreads;
            if (i + 4 <= n) {
                r[u].g = load_grad4(g + i, 0);
                r[u].w = ld_stream(reinterpret_cast<float4 *>(w + i));
                r[u].m = ld_stream(reinterpret_cast<float4 *>(m + i));
                r[u].v = ld_stream(reinterpret_cast<float4 *>(v + i));
            }
        }
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
            const size_t i = base + (size_t)u * 4 * kThreads;
            if (i + 4 <= n) {
                step4(r[u].g, factor, r[u].w, r[u].m, r[u].v, f, c);
                store4(w, m, v, copy, i, r[u].w, r[u].m, r[u].v);
            } else {
                for (size_t j = i; j < n && j < i + 4; ++j) scalar_element(g, w, m, v, copy, j, factor, f, c);
            }
        }
    }
}

// Long lists: a producer warp keeps the next chunks' gradients, weights and moments on their way to
// shared memory by bulk copies; each of the other threads takes four elements of a chunk.
// Three stages, 84-96 KB on their way per SM, is where DRAM is fullest: 12 GPT-2-XL-shaped blocks
// (369 M parameters, bf16 gradients) take 1630 us with 2 stages, 1495 with 3, 1588 with 4, 1648 with 7
// (more reads in flight crowd out the writes); chunks of 1024 1642 at best, of 4096 1513 (2 stages).
constexpr int kRingChunk = 2048;
constexpr int kRingStages = 3;
constexpr int kRingWork = kRingChunk / 4;
constexpr int kRingThreads = kRingWork + 32;

template <typename G>
struct StepStage {
    alignas(16) float w[kRingChunk], m[kRingChunk], v[kRingChunk];
    alignas(16) G g[kRingChunk];
};
template <typename G>
struct StepRing {
    StepStage<G> stage[kRingStages];
    unsigned long long full[kRingStages], empty[kRingStages];
    int tensor[kRingStages], loaded[kRingStages];  // the chunk's tensor; its elements that the copies brought
    int give_up;
};

template <typename G, int CAP>
__global__ void __launch_bounds__(kRingThreads, 1)
fold_apply_ring_kernel(const __grid_constant__ StepTable<CAP> tab, FoldConstants f, ApplyConstants c,
                       const float *__restrict__ factor_ptr, unsigned *status) {
    extern __shared__ unsigned char raw[];
    StepRing<G> &sh = *reinterpret_cast<StepRing<G> *>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    constexpr int kStages = kRingStages;
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const float factor = factor_ptr ? *factor_ptr : 1.f;
    if (factor != factor) return;  // a NaN factor (non-finite gradient norm) skips the step
    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            barrier_init(shared_addr(&sh.full[i]), 1);
            barrier_init(shared_addr(&sh.empty[i]), kRingWork / 32);
        }
        sh.give_up = 0;
        barrier_init_fence();
    }
    __syncthreads();
    const unsigned total = tab.chunk_start[tab.count];
    int slot = 0;
    uint32_t parity = 0;
    const auto advance = [&]() {
        if (++slot == kStages) {
            slot = 0;
            parity ^= 1;
        }
    };
    if (warp == kRingWork / 32) {
        if (lane != 0) return;
        int issued = 0, t = tensor_of_chunk(tab.chunk_start, tab.count, blockIdx.x);
        for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x, advance()) {
            t = tensor_from(tab.chunk_start, t, chunk);
            const size_t n = (size_t)tab.n[t];
            const unsigned char head = tab.head[t];
            const size_t base = (size_t)(chunk - tab.chunk_start[t]) * kRingChunk + (head == kScalar ? 0 : head);
            const G *g = static_cast<const G *>(tab.g[t]) + base;
            const size_t left = n > base ? n - base : 0;
            // whole units of eight elements of an aligned tensor; the threads fetch the rest themselves
            const uint32_t k = tab.bulk[t] ? (uint32_t)(left < kRingChunk ? left : kRingChunk) & ~7u : 0;
            if (issued == kStages && !barrier_wait(shared_addr(&sh.empty[slot]), parity ^ 1, &sh.give_up)) break;
            const uint32_t full = shared_addr(&sh.full[slot]);
            sh.tensor[slot] = t;
            sh.loaded[slot] = (int)k;
            barrier_expect(full, k * (12 + (uint32_t)sizeof(G)));
            if (k) {
                StepStage<G> &st = sh.stage[slot];
                bulk_load(shared_addr(st.g), g, k * (uint32_t)sizeof(G), full);
                bulk_load(shared_addr(st.w), tab.w[t] + base, 4 * k, full);
                bulk_load(shared_addr(st.m), tab.m[t] + base, 4 * k, full);
                bulk_load(shared_addr(st.v), tab.v[t] + base, 4 * k, full);
            }
            if (issued < kStages) ++issued;
        }
        if (*(volatile int *)&sh.give_up) {  // copies in flight end before the CTA does
            int none = 0;
            for (int i = 0; i < issued; ++i) {
                if (slot == 0) parity ^= 1;
                slot = slot ? slot - 1 : kStages - 1;
                barrier_wait(shared_addr(&sh.full[slot]), parity, &none);
            }
        }
        report_expired_wait(&sh.give_up, status, kWaitStepRing);
        return;
    }
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x, advance()) {
        if (!barrier_wait(shared_addr(&sh.full[slot]), parity, &sh.give_up)) break;  // nothing of this chunk is written
        const int t = sh.tensor[slot], loaded = sh.loaded[slot];
        const size_t n = (size_t)tab.n[t], k = chunk - tab.chunk_start[t];
        const unsigned char head = tab.head[t];
        const size_t base = k * kRingChunk + (head == kScalar ? 0 : head);
        const G *g = static_cast<const G *>(tab.g[t]);
        float *w = tab.w[t], *m = tab.m[t], *v = tab.v[t];
        __nv_bfloat16 *copy = tab.copy[t];
        const bool mine = 4 * tid < loaded;
        Group r;
        if (mine) {
            const StepStage<G> &st = sh.stage[slot];
            r.g = shared_grad4(st.g + 4 * tid);
            r.w = *reinterpret_cast<const float4 *>(st.w + 4 * tid);
            r.m = *reinterpret_cast<const float4 *>(st.m + 4 * tid);
            r.v = *reinterpret_cast<const float4 *>(st.v + 4 * tid);
        }
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_addr(&sh.empty[slot]));
        if (mine) {
            step4(r.g, factor, r.w, r.m, r.v, f, c);
            store4(w, m, v, copy, base + 4 * tid, r.w, r.m, r.v);
        }
        if (loaded == kRingChunk && (k > 0 || head == 0)) continue;
        // before the first boundary, behind the last whole unit, or all of an unaligned tensor's chunk
        if (k == 0 && head != kScalar && tid < head && (size_t)tid < n) scalar_element(g, w, m, v, copy, tid, factor, f, c);
        const size_t end = base + kRingChunk < n ? base + kRingChunk : n;
        if (!tab.bulk[t] && head != kScalar && end >= base + 4 * tid + 4) {  // aligned, but not for bulk copies
            const size_t i = base + 4 * tid;
            r.g = load_grad4(g + i, 0);
            r.w = ld_stream(reinterpret_cast<float4 *>(w + i));
            r.m = ld_stream(reinterpret_cast<float4 *>(m + i));
            r.v = ld_stream(reinterpret_cast<float4 *>(v + i));
            step4(r.g, factor, r.w, r.m, r.v, f, c);
            store4(w, m, v, copy, i, r.w, r.m, r.v);
        }
        const size_t done = tab.bulk[t] ? base + loaded : head == kScalar ? base : end > base ? base + (end - base) / 4 * 4 : end;
        scalar_run(g, w, m, v, copy, done + tid, end, kRingWork, factor, f, c);
    }
    if (lane == 0) report_expired_wait(&sh.give_up, status, kWaitStepRing);
}

// Elements before w, m, v are at a 16-byte boundary, the gradient at one too (bulk copies need it) or
// at least at its own 4-element boundary, and the copy at 8 bytes; kScalar where there is no such place.
void place_of(const void *g, adama_dtype gdt, const float *w, const float *m, const float *v, const void *copy,
              unsigned char &head, unsigned char &bulk) {
    const uintptr_t gs = gdt == ADAMA_F32 ? 4 : 2;
    const auto at = [](const void *p, uintptr_t bytes, uintptr_t align) {
        return (reinterpret_cast<uintptr_t>(p) + bytes) % align == 0;
    };
    for (int whole = 1; whole >= 0; --whole) {
        for (uintptr_t h = 0; h < 8; ++h) {
            if (!at(w, 4 * h, 16) || !at(m, 4 * h, 16) || !at(v, 4 * h, 16) || !at(g, gs * h, whole ? 16 : 4 * gs)) continue;
            if (copy && !at(copy, 2 * h, 8)) continue;
            head = (unsigned char)h;
            bulk = (unsigned char)whole;
            return;
        }
    }
    head = kScalar;
    bulk = 0;
}

constexpr unsigned kRingFrom = 4;  // chunks of the ring per SM from which it is used

template <typename G, int CAP>
cudaError_t launch_kernels(StepTable<CAP> &tab, const size_t *n, int count, FoldConstants f, ApplyConstants c,
                           const float *factor, unsigned *status, int sm_count, cudaStream_t stream) {
    unsigned chunks = fill_chunks(tab.n, tab.chunk_start, n, count, kRingChunk);
    if (chunks < kRingFrom * (unsigned)sm_count) {
        chunks = fill_chunks(tab.n, tab.chunk_start, n, count);
        if (chunks == 0) return cudaSuccess;
        const unsigned cap = (unsigned)sm_count * 3u;
        fold_apply_multi_kernel<G, CAP><<<chunks < cap ? chunks : cap, kThreads, 0, stream>>>(tab, f, c, factor);
        return cudaGetLastError();
    }
    constexpr int bytes = (int)sizeof(StepRing<G>) + 128;
    static std::atomic<unsigned long long> ready{0};
    cudaError_t e = allow_shared(fold_apply_ring_kernel<G, CAP>, bytes, ready);
    if (e != cudaSuccess) return e;
    fold_apply_ring_kernel<G, CAP><<<(unsigned)sm_count, kRingThreads, bytes, stream>>>(tab, f, c, factor, status);
    return cudaGetLastError();
}

template <int CAP>
cudaError_t launch(const StepList &s, adama_dtype gdt, int first, int count, FoldConstants f,
                   ApplyConstants c, const float *factor, unsigned *status, int sm_count, cudaStream_t stream) {
    StepTable<CAP> tab;
    for (int i = 0; i < count; ++i) {
        tab.g[i] = s.g[first + i];
        tab.w[i] = s.w[first + i];
        tab.m[i] = s.m[first + i];
        tab.v[i] = s.v[first + i];
        tab.copy[i] = s.copy ? static_cast<__nv_bfloat16 *>(s.copy[first + i]) : nullptr;
        place_of(tab.g[i], gdt, tab.w[i], tab.m[i], tab.v[i], tab.copy[i], tab.head[i], tab.bulk[i]);
    }
    tab.count = count;
    return gdt == ADAMA_F32
               ? launch_kernels<float>(tab, s.n + first, count, f, c, factor, status, sm_count, stream)
               : launch_kernels<__nv_bfloat16>(tab, s.n + first, count, f, c, factor, status, sm_count, stream);
}

}  // namespace

cudaError_t launch_fold_apply_multi(const StepList &s, adama_dtype gdt, int first, int count,
                                    FoldConstants f, ApplyConstants c, const float *factor,
                                    unsigned *status, int sm_count, cudaStream_t stream) {
    if (count <= kStepSmall) return launch<kStepSmall>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
    if (count <= kStepMid) return launch<kStepMid>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
    return launch<kStepMax>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
}

}  // namespace adama
