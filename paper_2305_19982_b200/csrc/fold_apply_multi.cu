// The mini-batch's last fold and its update in ONE pass over many tensors (Algorithm 2: the inner
// loop body for the last micro-batch, "Update", and the decay of the next mini-batch):
//     m += a*g,  v += b*g^2,  w -= step*m/(sqrt(v*inv_bc2) + eps),  m *= beta1,  v *= beta2
// with g times an optional factor (gradient clipping) that lies in device memory.  With one
// micro-batch a mini-batch this is a whole AdamW step: 26 B/param (bf16 gradient) instead of the
// 18 + 24 of a fold and an apply.  Same arithmetic as those two, bit for bit.
#include "adama_device.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kChunk / (4 * kThreads);  // float4 groups of one thread in a chunk
constexpr unsigned char kScalar = 255;            // no common 16-byte alignment: element by element

template <int CAP>
struct StepTable {
    const void *g[CAP];
    float *w[CAP];
    float *m[CAP];
    float *v[CAP];
    __nv_bfloat16 *copy[CAP];  // entries may be null
    unsigned long long n[CAP];
    unsigned chunk_start[CAP + 1];
    unsigned char head[CAP];  // elements before the first 16-byte boundary of w, m, v; or kScalar
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
            for (size_t i = k * kChunk + threadIdx.x; i < end; i += kThreads)
                scalar_element(g, w, m, v, copy, i, factor, f, c);
            continue;
        }
        if (k == 0 && threadIdx.x < head) scalar_element(g, w, m, v, copy, threadIdx.x, factor, f, c);
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
                float4 &x = r[u].w, &y = r[u].m, &z = r[u].v;
                step1(r[u].g.x * factor, x.x, y.x, z.x, f, c);
                step1(r[u].g.y * factor, x.y, y.y, z.y, f, c);
                step1(r[u].g.z * factor, x.z, y.z, z.z, f, c);
                step1(r[u].g.w * factor, x.w, y.w, z.w, f, c);
                st_stream(reinterpret_cast<float4 *>(w + i), x);
                st_stream(reinterpret_cast<float4 *>(m + i), y);
                st_stream(reinterpret_cast<float4 *>(v + i), z);
                if (copy)
                    *reinterpret_cast<uint2 *>(copy + i) = make_uint2(pack2_bf16(x.x, x.y), pack2_bf16(x.z, x.w));
            } else {
                for (size_t j = i; j < n && j < i + 4; ++j) scalar_element(g, w, m, v, copy, j, factor, f, c);
            }
        }
    }
}

// Elements up to the first 16-byte boundary when w, m, v reach it together and the gradient (and
// the copy) reach their own 4-element boundary there too; kScalar otherwise.
unsigned char head_of(const void *g, adama_dtype gdt, const float *w, const float *m, const float *v,
                      const void *copy) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(w) & 15;
    const uintptr_t head = at ? (16 - at) / 4 : 0;
    const uintptr_t gs = gdt == ADAMA_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(m) & 15) != at || (reinterpret_cast<uintptr_t>(v) & 15) != at ||
        (reinterpret_cast<uintptr_t>(g) + head * gs) % (4 * gs) != 0 ||
        (copy && (reinterpret_cast<uintptr_t>(copy) + head * 2) % 8 != 0))
        return kScalar;
    return (unsigned char)head;
}

template <int CAP>
cudaError_t launch(const StepList &s, adama_dtype gdt, int first, int count, FoldConstants f,
                   ApplyConstants c, const float *factor, int sm_count, cudaStream_t stream) {
    StepTable<CAP> tab;
    for (int i = 0; i < count; ++i) {
        tab.g[i] = s.g[first + i];
        tab.w[i] = s.w[first + i];
        tab.m[i] = s.m[first + i];
        tab.v[i] = s.v[first + i];
        tab.copy[i] = s.copy ? static_cast<__nv_bfloat16 *>(s.copy[first + i]) : nullptr;
        tab.head[i] = head_of(tab.g[i], gdt, tab.w[i], tab.m[i], tab.v[i], tab.copy[i]);
    }
    tab.count = count;
    const unsigned chunks = fill_chunks(tab.n, tab.chunk_start, s.n + first, count);
    if (chunks == 0) return cudaSuccess;
    const unsigned cap = (unsigned)sm_count * 3u, grid = chunks < cap ? chunks : cap;
    if (gdt == ADAMA_F32)
        fold_apply_multi_kernel<float, CAP><<<grid, kThreads, 0, stream>>>(tab, f, c, factor);
    else
        fold_apply_multi_kernel<__nv_bfloat16, CAP><<<grid, kThreads, 0, stream>>>(tab, f, c, factor);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_fold_apply_multi(const StepList &s, adama_dtype gdt, int first, int count,
                                    FoldConstants f, ApplyConstants c, const float *factor,
                                    int sm_count, cudaStream_t stream) {
    return count <= kStepSmall ? launch<kStepSmall>(s, gdt, first, count, f, c, factor, sm_count, stream)
                               : launch<kStepMax>(s, gdt, first, count, f, c, factor, sm_count, stream);
}

}  // namespace adama
