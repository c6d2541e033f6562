// Lists of tensors in a kernel's parameter space: the work of one launch is the list's chunks (of
// kChunk elements, or what the kernel states), numbered through all tensors; a CTA finds the tensor
// of a chunk by bisection.
#pragma once

#include <cuda_bf16.h>

#include <atomic>

#include "adama_internal.h"
#include "stream_access.cuh"

namespace adama {

constexpr int kChunk = 4096;  // elements of one chunk

// chunk_start[i] = number of chunks before tensor i; returns the tensor that holds chunk `c`
__device__ __forceinline__ int tensor_of_chunk(const unsigned *chunk_start, int count, unsigned c) {
    int lo = 0, hi = count;  // chunk_start[lo] <= c < chunk_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (chunk_start[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The same for a chunk behind one that lies in tensor t: steps forward from there (a loop over chunks
// passes few tensor borders at a time; bisecting anew for each chunk cost the producers of the rings
// more than the copies that they issue).
__device__ __forceinline__ int tensor_from(const unsigned *chunk_start, int t, unsigned c) {
    while (chunk_start[t + 1] <= c) ++t;
    return t;
}

// Fills n and chunk_start for `count` tensors; returns the number of chunks.
inline unsigned fill_chunks(unsigned long long *n_out, unsigned *chunk_start, const size_t *n, int count,
                            size_t chunk = kChunk) {
    unsigned acc = 0;
    for (int i = 0; i < count; ++i) {
        n_out[i] = (unsigned long long)n[i];
        chunk_start[i] = acc;
        acc += (unsigned)((n[i] + chunk - 1) / chunk);
    }
    chunk_start[count] = acc;
    return acc;
}

// eight consecutive gradient values, widened exactly; the pointer is 16-byte aligned
__device__ __forceinline__ void load_grad8(const float *g, float (&x)[8]) {
    const float4 a = ld_stream_ro(reinterpret_cast<const float4 *>(g));
    const float4 b = ld_stream_ro(reinterpret_cast<const float4 *>(g) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void load_grad8(const __nv_bfloat16 *g, float (&x)[8]) {
    const float4 t = ld_stream_ro(reinterpret_cast<const float4 *>(g));
    const unsigned u[4] = {__float_as_uint(t.x), __float_as_uint(t.y), __float_as_uint(t.z), __float_as_uint(t.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // bf16 -> fp32 is a 16-bit left shift
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}

// four gradient values from shared memory, widened exactly
__device__ __forceinline__ Grad4 shared_grad4(const float *p) {
    const float4 t = *reinterpret_cast<const float4 *>(p);
    return {t.x, t.y, t.z, t.w};
}
__device__ __forceinline__ Grad4 shared_grad4(const __nv_bfloat16 *p) {
    const uint2 t = *reinterpret_cast<const uint2 *>(p);
    return {__uint_as_float(t.x << 16), __uint_as_float(t.x & 0xffff0000u),
            __uint_as_float(t.y << 16), __uint_as_float(t.y & 0xffff0000u)};
}

// Sets a kernel's limit of dynamic shared memory once per device (`ready`: one bit per device).
template <typename Kernel>
inline cudaError_t allow_shared(Kernel kernel, int bytes, std::atomic<unsigned long long> &ready) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = device < 64 ? 1ull << device : 0;
    if (ready.load() & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) ready.fetch_or(bit);
    return e;
}

// two fp32 -> packed bf16x2, round to nearest even (the weight copy a bf16 forward pass reads)
__device__ __forceinline__ unsigned pack2_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned *>(&p);
}

}  // namespace adama
