// Global 2-norm of a list of gradients, and the clip factor that follows from it, left on the
// device for the step that multiplies by it.  One pass, 2 or 4 B/element; each CTA's sum goes to
// the workspace as a double, the last CTA to finish adds them in the CTAs' order, so that the
// result does not depend on scheduling.
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
constexpr int kCtasPerSm = 4;

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

template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
grad_norm_kernel(const __grid_constant__ NormTable<CAP> tab, float max_norm, int accumulate,
                 adama_grad_norm *out, Workspace *ws) {
    constexpr int kVec = 16 / sizeof(G);
    __shared__ double shared[kThreads / 32];
    __shared__ bool last;
    const unsigned total = tab.chunk_start[tab.count];
    double sum = 0.0;
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kChunk;
        const G *g = static_cast<const G *>(tab.g[t]);
        const size_t mis = (reinterpret_cast<uintptr_t>(g) % 16) / sizeof(G);
        const size_t head = mis ? kVec - mis : 0;  // chunk c covers [head + c*kChunk, ...), the first one the head too
        float part = 0.f;
        if (first == 0 && threadIdx.x < head && threadIdx.x < n) {
            const float x = widen(g[threadIdx.x]);
            part = fmaf(x, x, part);
        }
#pragma unroll
        for (int u = 0; u < kChunk / (kVec * kThreads); ++u) {
            const size_t i = head + first + (size_t)(u * kThreads + threadIdx.x) * kVec;
            if (i + kVec <= n) {
                if (sizeof(G) == 2) {
                    float x[8];
                    load_grad8(g + i, x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) part = fmaf(x[j], x[j], part);
                } else {
                    const Grad4 x = load_grad4(g + i, 0);
                    part = fmaf(x.x, x.x, fmaf(x.y, x.y, fmaf(x.z, x.z, fmaf(x.w, x.w, part))));
                }
            } else {
                for (size_t j = i; j < n && j < i + kVec; ++j) {
                    const float x = widen(g[j]);
                    part = fmaf(x, x, part);
                }
            }
        }
        sum += (double)part;
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) {
        ws->part[blockIdx.x] = sum;
        __threadfence();
        last = atomicAdd(&ws->ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
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

template <int CAP>
cudaError_t launch(const void *const *g, adama_dtype gdt, const size_t *n, int count, float max_norm,
                   int accumulate, adama_grad_norm *out, Workspace *ws, int sm_count, cudaStream_t stream) {
    NormTable<CAP> tab;
    for (int i = 0; i < count; ++i) tab.g[i] = g[i];
    tab.count = count;
    const unsigned chunks = fill_chunks(tab.n, tab.chunk_start, n, count);
    unsigned cap = (unsigned)(sm_count * kCtasPerSm);
    if (cap > kWorkspaceParts) cap = kWorkspaceParts;
    const unsigned grid = chunks == 0 ? 1 : chunks < cap ? chunks : cap;
    if (gdt == ADAMA_F32)
        grad_norm_kernel<float, CAP><<<grid, kThreads, 0, stream>>>(tab, max_norm, accumulate, out, ws);
    else
        grad_norm_kernel<__nv_bfloat16, CAP><<<grid, kThreads, 0, stream>>>(tab, max_norm, accumulate, out, ws);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_grad_norm(const void *const *g, adama_dtype gdt, const size_t *n, int count,
                             float max_norm, int accumulate, adama_grad_norm *out, void *workspace,
                             int sm_count, cudaStream_t stream) {
    Workspace *ws = static_cast<Workspace *>(workspace);
    return count <= kStepSmall
               ? launch<kStepSmall>(g, gdt, n, count, max_norm, accumulate, out, ws, sm_count, stream)
               : launch<kNormMax>(g, gdt, n, count, max_norm, accumulate, out, ws, sm_count, stream);
}

}  // namespace adama
