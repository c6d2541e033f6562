// Global 2-norm of a list of gradients, and the clip factor that follows from it, left on the
// device for the step that multiplies by it.  One pass, 2 or 4 B/element; each CTA's sum goes to
// the workspace as a double, the last CTA to finish adds them in the CTAs' order, so that the
// result does not depend on scheduling.  Bound by HBM: 369 M bf16 gradients take 107.4 us = 6.87 TB/s
// (reads alone run above a copy's rate); 16 M 9.4 us, twice their floor: launch, first loads and two
// dependent reductions are not yet hidden by so few bytes; 150 short tensors 5.0-5.5 us, nothing but these.
#include "softmax_rows.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
// 4 CTAs per SM with 8 units of each thread in flight: 369 M bf16 gradients take 107.7 us (6.85 TB/s);
// 4 x 4 109.3, 8 x 4 111.6, 2 x 8 109.4, 2 x 16 106.3 but 8.4 instead of 5.7 us for short lists.  Lists of
// 16 M elements (50 MB and less) want the bytes in flight most: 10.7 us with 8 units, 14.1 with 2.
constexpr int kCtasPerSm = 4;
constexpr int kUnits = 8;

template <int CAP>
struct NormTable {
    const void *g[CAP];
    unsigned long long n[CAP];
    unsigned chunk_start[CAP + 1];
    int count;
};
static_assert(sizeof(NormTable<kNormMax>) <= 32000, "table must fit the kernel parameter space");

__device__ __forceinline__ double block_sum(double x, double *shared) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_down_sync(0xffffffffu, x, o);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = x;
    __syncthreads();
    double sum = 0.0;
    for (int i = 0; i < kThreads / 32; ++i) sum += shared[i];
    __syncthreads();
    return sum;
}

// A chunk is kUnits 16-byte units of each thread, all loaded before the first is used.
template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const __grid_constant__ NormTable<CAP> tab, float max_norm, int accumulate,
                 adama_grad_norm *out, Workspace *ws) {
    constexpr int kVec = 16 / sizeof(G), kNormChunk = kUnits * kThreads * kVec;
    __shared__ double shared[kThreads / 32];
    __shared__ bool last;
    const unsigned total = tab.chunk_start[tab.count];
    double sum = 0.0;
    int t = tensor_of_chunk(tab.chunk_start, tab.count, blockIdx.x);
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        t = tensor_from(tab.chunk_start, t, chunk);
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kNormChunk;
        const G *g = static_cast<const G *>(tab.g[t]);
        const size_t mis = (reinterpret_cast<uintptr_t>(g) % 16) / sizeof(G);
        const size_t head = mis ? kVec - mis : 0;  // chunk c covers [head + c*kNormChunk, ...), the first one the head too
        const size_t base = head + first + (size_t)threadIdx.x * kVec;
        float part = 0.f;
        uint4 u[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            u[i] = make_uint4(0, 0, 0, 0);
            if (base + (size_t)i * kThreads * kVec + kVec <= n)
                u[i] = ld_unit_ro(reinterpret_cast<const uint4 *>(g + base + (size_t)i * kThreads * kVec));
        }
        if (first == 0 && threadIdx.x < head && threadIdx.x < n) {
            const float x = widen(g[threadIdx.x]);
            part = fmaf(x, x, part);
        }
        if (first + kNormChunk >= n && n > head) {  // the tensor's last chunk: what its end cuts off a unit
            const size_t j = head + (n - head) / kVec * kVec + threadIdx.x;
            if (j < n) {
                const float x = widen(g[j]);
                part = fmaf(x, x, part);
            }
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            Pair p = 0;
#pragma unroll
            for (int q = 0; q < kVec / 2; ++q) {
                const Pair x = unit_pair<G>(u[i], q);
                p = fma2(x, x, p);
            }
            float lo, hi;
            split(p, lo, hi);
            part += lo + hi;
        }
        sum += (double)part;
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        ws->part[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
        if (last) __threadfence();  // the loads behind the barrier see what came before the other CTAs' tickets
    }
    __syncthreads();
    if (!last) return;
    double all = 0.0;
    for (unsigned i = threadIdx.x; i < gridDim.x; i += kThreads) all += __ldcg(&ws->part[i]);
    all = block_sum(all, shared);
    if (threadIdx.x == 0) {
        if (accumulate) all += out->sumsq;
        const float norm = (float)sqrt(all);
        out->sumsq = all;
        out->norm = norm;
        out->factor = !isfinite(norm) ? NAN : norm > max_norm ? max_norm / norm : 1.f;
        ws->ticket = 0;
    }
}

template <typename G, int CAP>
cudaError_t launch(const void *const *g, const size_t *n, int count, float max_norm, int accumulate,
                   adama_grad_norm *out, Workspace *ws, int sm_count, cudaStream_t stream) {
    NormTable<CAP> tab;
    for (int i = 0; i < count; ++i) tab.g[i] = g[i];
    tab.count = count;
    const unsigned chunks = fill_chunks(tab.n, tab.chunk_start, n, count, kUnits * kThreads * 16 / sizeof(G));
    unsigned cap = (unsigned)(sm_count * kCtasPerSm);
    if (cap > kWorkspaceParts) cap = kWorkspaceParts;
    const unsigned grid = chunks == 0 ? 1 : chunks < cap ? chunks : cap;
    grad_norm_kernel<G, CAP><<<grid, kThreads, 0, stream>>>(tab, max_norm, accumulate, out, ws);
    return cudaGetLastError();
}

template <typename G>
cudaError_t launch(const void *const *g, const size_t *n, int count, float max_norm, int accumulate,
                   adama_grad_norm *out, Workspace *ws, int sm_count, cudaStream_t stream) {
    // the table is copied with every launch: 20 KB of it cost 2 us more than 1
    if (count <= kStepSmall) return launch<G, kStepSmall>(g, n, count, max_norm, accumulate, out, ws, sm_count, stream);
    if (count <= kNormMid) return launch<G, kNormMid>(g, n, count, max_norm, accumulate, out, ws, sm_count, stream);
    return launch<G, kNormMax>(g, n, count, max_norm, accumulate, out, ws, sm_count, stream);
}

}  // namespace

cudaError_t launch_grad_norm(const void *const *g, adama_dtype gdt, const size_t *n, int count,
                             float max_norm, int accumulate, adama_grad_norm *out, void *workspace,
                             int sm_count, cudaStream_t stream) {
    Workspace *ws = static_cast<Workspace *>(workspace);
    return gdt == ADAMA_F32
               ? launch<float>(g, n, count, max_norm, accumulate, out, ws, sm_count, stream)
               : launch<__nv_bfloat16>(g, n, count, max_norm, accumulate, out, ws, sm_count, stream);
}

}  // namespace adama
