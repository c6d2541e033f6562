// Adam moments in 8 bits.  Blocks of kStateBlock consecutive elements share one fp32 scale each:
//     m = M * sm   M: e4m3 (sign, 4 exponent bits, 3 mantissa bits), largest 448
//     v = V * sv   V: unsigned, 5 exponent bits, 3 mantissa bits, (1 + c%8/8) * 2^(c/8 - 31), largest 1.875
// Adam divides m by sqrt(v), element by element, so both need relative, not absolute, precision:
// 1/16 at most for m; for sqrt(v) half of v's 1/16, over the 31 binades of v that a block spans.
// A v that is not zero never becomes code 0 (it would divide m by eps alone): the smallest code
// stands in.  The decay of Algorithm 2 multiplies the block's scale and leaves the codes alone:
// 0.999 of a code value would round back to it for ever.
#include <cuda_fp8.h>
#include <float.h>

#include "adama_device.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerLane = kStateBlock / 32;                      // elements of a block that one lane holds
constexpr int kBlocksPerWarp = kChunk / (kStateBlock * kWarps); // blocks of a chunk that one warp takes
static_assert(kPerLane == 8, "one 64-bit access per lane moves its codes");

constexpr float kMTop = 448.f, kVTop = 1.875f;
constexpr float kMTopInv = (float)(1.0 / 448.0), kVTopInv = (float)(1.0 / 1.875);

template <int CAP>
struct Table8 {
    const void *g[CAP];
    float *w[CAP];
    __nv_bfloat16 *copy[CAP];  // entries may be null
    adama_state8 s[CAP];
    unsigned long long n[CAP];
    unsigned chunk_start[CAP + 1];
    unsigned char vec[CAP];  // 1: every pointer allows the widest access
    int count;
};
static_assert(sizeof(Table8<kStep8Max>) <= 32000, "table must fit the kernel parameter space");

__device__ __forceinline__ float decode_v(unsigned code) {
    return code ? __uint_as_float((code << 20) + (96u << 23)) : 0.f;
}
// y = v/top*1.875: round to 3 mantissa bits, ties to even
__device__ __forceinline__ unsigned encode_v(float v, float inv) {
    const int bits = __float_as_int(__fmul_rn(v, inv));
    int code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - (96 << 3);
    code = code < 1 ? 1 : code > 255 ? 255 : code;
    return v > 0.f ? (unsigned)code : 0u;
}
__device__ __forceinline__ float2 decode_m2(unsigned codes) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}
__device__ __forceinline__ unsigned encode_m2(float a, float b, float inv) {
    return __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(a, inv), __fmul_rn(b, inv)), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float code_factor(float top, float code_top) {
    return fminf(__fmul_rn(__frcp_rn(top), code_top), FLT_MAX);  // top == 0 and subnormal tops stay finite
}
// The block's largest magnitude, on the bits: the order of non-negative floats, NaN above all.
__device__ __forceinline__ float warp_top(float x) {
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
}

// What one lane holds of a block.
struct Lane {
    float m[kPerLane], v[kPerLane];

    __device__ __forceinline__ void decode(uint2 mc, uint2 vc, float sm, float sv) {
        const unsigned mw[2] = {mc.x, mc.y}, vw[2] = {vc.x, vc.y};
#pragma unroll
        for (int i = 0; i < kPerLane; i += 2) {
            const float2 p = decode_m2((mw[i / 4] >> (8 * (i % 4))) & 0xffffu);
            m[i] = __fmul_rn(p.x, sm);
            m[i + 1] = __fmul_rn(p.y, sm);
            v[i] = __fmul_rn(decode_v((vw[i / 4] >> (8 * (i % 4))) & 0xffu), sv);
            v[i + 1] = __fmul_rn(decode_v((vw[i / 4] >> (8 * (i % 4) + 8)) & 0xffu), sv);
        }
    }
    // all 32 lanes of the warp; returns the block's largest |m| and v
    __device__ __forceinline__ float2 encode(uint2 &mc, uint2 &vc) const {
        float mt = 0.f, vt = 0.f;
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            mt = __uint_as_float(max(__float_as_uint(mt), __float_as_uint(fabsf(m[i]))));
            vt = __uint_as_float(max(__float_as_uint(vt), __float_as_uint(fabsf(v[i]))));
        }
        mt = warp_top(mt);
        vt = warp_top(vt);
        const float mi = code_factor(mt, kMTop), vi = code_factor(vt, kVTop);
        unsigned mw[2] = {0, 0}, vw[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < kPerLane; i += 2) {
            mw[i / 4] |= encode_m2(m[i], m[i + 1], mi) << (8 * (i % 4));
            vw[i / 4] |= (encode_v(v[i], vi) | encode_v(v[i + 1], vi) << 8) << (8 * (i % 4));
        }
        mc = make_uint2(mw[0], mw[1]);
        vc = make_uint2(vw[0], vw[1]);
        return make_float2(mt, vt);
    }
};

// One update with separately rounded products and sums (the codes that come out are then those of
// the formula evaluated in fp32, operation by operation); the decay is left to the scales.
__device__ __forceinline__ void step8_1(float g, float &w, float &m, float &v, const FoldConstants &f,
                                        const ApplyConstants &c) {
    m = __fadd_rn(m, __fmul_rn(g, f.a));
    v = __fadd_rn(v, __fmul_rn(__fmul_rn(g, f.b), g));
    const float denom = sqrt_fast(v * c.inv_bc2) + c.eps;
    w = fmaf(-c.step, m * rcp_fast(denom), w * c.w_keep);
}

// Byte i of a lane's eight codes lies at element 8*lane + i (vector form) or lane + 32*i.
__device__ __forceinline__ uint2 gather_codes(const uint8_t *p, size_t at, size_t n, int lane) {
    unsigned x[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
        if (at + lane + 32 * i < n) x[i / 4] |= (unsigned)p[at + lane + 32 * i] << (8 * (i % 4));
    return make_uint2(x[0], x[1]);
}
__device__ __forceinline__ void scatter_codes(uint8_t *p, size_t at, size_t n, int lane, uint2 c) {
    const unsigned x[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
        if (at + lane + 32 * i < n) p[at + lane + 32 * i] = (uint8_t)(x[i / 4] >> (8 * (i % 4)));
}
__device__ __forceinline__ uint2 load_codes(const uint8_t *p) { return *reinterpret_cast<const uint2 *>(p); }
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 c) { *reinterpret_cast<uint2 *>(p) = c; }

__device__ __forceinline__ void load8(const float *p, float (&x)[kPerLane]) {
    const float4 a = ld_stream(reinterpret_cast<const float4 *>(p));
    const float4 b = ld_stream(reinterpret_cast<const float4 *>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[kPerLane]) {
    st_stream(reinterpret_cast<float4 *>(p), make_float4(x[0], x[1], x[2], x[3]));
    st_stream(reinterpret_cast<float4 *>(p) + 1, make_float4(x[4], x[5], x[6], x[7]));
}

template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
fold_apply8_kernel(const __grid_constant__ Table8<CAP> tab, FoldConstants f, ApplyConstants c,
                   const float *__restrict__ factor_ptr) {
    const float factor = factor_ptr ? *factor_ptr : 1.f;
    if (factor != factor) return;  // a NaN factor (non-finite gradient norm) skips the step
    const unsigned total = tab.chunk_start[tab.count];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kChunk;
        const adama_state8 s = tab.s[t];
        const G *g = static_cast<const G *>(tab.g[t]);
        float *w = tab.w[t];
        __nv_bfloat16 *copy = tab.copy[t];
        for (int b = 0; b < kBlocksPerWarp; ++b) {
            const size_t at = first + (size_t)(warp + b * kWarps) * kStateBlock;
            if (at >= n) break;
            const size_t blk = at / kStateBlock;
            const float sm = s.m_scale[blk], sv = s.v_scale[blk];
            Lane x;
            uint2 mc, vc;
            float gg[kPerLane], ww[kPerLane];
            const bool wide = tab.vec[t] && at + kStateBlock <= n;
            const size_t i0 = at + lane * kPerLane;
            if (wide) {
                load_grad8(g + i0, gg);
                load8(w + i0, ww);
                mc = load_codes(s.m_codes + i0);
                vc = load_codes(s.v_codes + i0);
            } else {
                mc = gather_codes(s.m_codes, at, n, lane);
                vc = gather_codes(s.v_codes, at, n, lane);
#pragma unroll
                for (int i = 0; i < kPerLane; ++i) {
                    const size_t j = at + lane + 32 * i;
                    gg[i] = j < n ? widen(g[j]) : 0.f;
                    ww[i] = j < n ? w[j] : 0.f;
                }
            }
            x.decode(mc, vc, sm, sv);
#pragma unroll
            for (int i = 0; i < kPerLane; ++i) step8_1(__fmul_rn(gg[i], factor), ww[i], x.m[i], x.v[i], f, c);
            const float2 top = x.encode(mc, vc);
            if (wide) {
                store8(w + i0, ww);
                store_codes(s.m_codes + i0, mc);
                store_codes(s.v_codes + i0, vc);
                if (copy)
                    *reinterpret_cast<uint4 *>(copy + i0) =
                        make_uint4(pack2_bf16(ww[0], ww[1]), pack2_bf16(ww[2], ww[3]),
                                   pack2_bf16(ww[4], ww[5]), pack2_bf16(ww[6], ww[7]));
            } else {
                scatter_codes(s.m_codes, at, n, lane, mc);
                scatter_codes(s.v_codes, at, n, lane, vc);
#pragma unroll
                for (int i = 0; i < kPerLane; ++i) {
                    const size_t j = at + lane + 32 * i;
                    if (j < n) {
                        w[j] = ww[i];
                        if (copy) copy[j] = __float2bfloat16_rn(ww[i]);
                    }
                }
            }
            if (lane == 0) {
                s.m_scale[blk] = __fmul_rn(__fmul_rn(top.x, kMTopInv), c.beta1_hi);
                s.v_scale[blk] = __fmul_rn(__fmul_rn(top.y, kVTopInv), c.beta2_hi);
            }
        }
    }
}

template <int CAP>
struct ConvertTable {
    float *m[CAP];
    float *v[CAP];
    adama_state8 s[CAP];
    unsigned long long n[CAP];
    unsigned chunk_start[CAP + 1];
    unsigned char vec[CAP];
    int count;
};
static_assert(sizeof(ConvertTable<kStep8Max>) <= 32000, "table must fit the kernel parameter space");

// PACK: fp32 moments -> codes and scales; otherwise codes and scales -> the values they stand for.
template <bool PACK, int CAP>
__global__ void __launch_bounds__(kThreads)
state8_convert_kernel(const __grid_constant__ ConvertTable<CAP> tab) {
    const unsigned total = tab.chunk_start[tab.count];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kChunk;
        const adama_state8 s = tab.s[t];
        float *m = tab.m[t], *v = tab.v[t];
        for (int b = 0; b < kBlocksPerWarp; ++b) {
            const size_t at = first + (size_t)(warp + b * kWarps) * kStateBlock;
            if (at >= n) break;
            const size_t blk = at / kStateBlock, i0 = at + lane * kPerLane;
            const bool wide = tab.vec[t] && at + kStateBlock <= n;
            Lane x;
            uint2 mc, vc;
            if (PACK) {
                if (wide) {
                    load8(m + i0, x.m);
                    load8(v + i0, x.v);
                } else {
#pragma unroll
                    for (int i = 0; i < kPerLane; ++i) {
                        const size_t j = at + lane + 32 * i;
                        x.m[i] = j < n ? m[j] : 0.f;
                        x.v[i] = j < n ? v[j] : 0.f;
                    }
                }
                const float2 top = x.encode(mc, vc);
                if (wide) {
                    store_codes(s.m_codes + i0, mc);
                    store_codes(s.v_codes + i0, vc);
                } else {
                    scatter_codes(s.m_codes, at, n, lane, mc);
                    scatter_codes(s.v_codes, at, n, lane, vc);
                }
                if (lane == 0) {
                    s.m_scale[blk] = __fmul_rn(top.x, kMTopInv);
                    s.v_scale[blk] = __fmul_rn(top.y, kVTopInv);
                }
            } else {
                mc = wide ? load_codes(s.m_codes + i0) : gather_codes(s.m_codes, at, n, lane);
                vc = wide ? load_codes(s.v_codes + i0) : gather_codes(s.v_codes, at, n, lane);
                x.decode(mc, vc, s.m_scale[blk], s.v_scale[blk]);
                if (wide) {
                    store8(m + i0, x.m);
                    store8(v + i0, x.v);
                } else {
#pragma unroll
                    for (int i = 0; i < kPerLane; ++i) {
                        const size_t j = at + lane + 32 * i;
                        if (j < n) {
                            m[j] = x.m[i];
                            v[j] = x.v[i];
                        }
                    }
                }
            }
        }
    }
}

bool state_wide(const adama_state8 &s) { return aligned(s.m_codes, 8) && aligned(s.v_codes, 8); }

unsigned grid_of(unsigned chunks, int sm_count, int per_sm) {
    const unsigned cap = (unsigned)(sm_count * per_sm);
    return chunks < cap ? chunks : cap;
}

template <int CAP>
cudaError_t launch_step(const StepList &s, adama_dtype gdt, int first, int count, FoldConstants f,
                        ApplyConstants c, const float *factor, int sm_count, cudaStream_t stream) {
    Table8<CAP> tab;
    for (int i = 0; i < count; ++i) {
        tab.g[i] = s.g[first + i];
        tab.w[i] = s.w[first + i];
        tab.copy[i] = s.copy ? static_cast<__nv_bfloat16 *>(s.copy[first + i]) : nullptr;
        tab.s[i] = s.s8[first + i];
        tab.vec[i] = aligned(tab.g[i], 16) && aligned(tab.w[i], 16) && aligned(tab.copy[i], 16) && state_wide(tab.s[i]);
    }
    tab.count = count;
    const unsigned chunks = fill_chunks(tab.n, tab.chunk_start, s.n + first, count);
    if (chunks == 0) return cudaSuccess;
    const unsigned grid = grid_of(chunks, sm_count, 4);
    if (gdt == ADAMA_F32)
        fold_apply8_kernel<float, CAP><<<grid, kThreads, 0, stream>>>(tab, f, c, factor);
    else
        fold_apply8_kernel<__nv_bfloat16, CAP><<<grid, kThreads, 0, stream>>>(tab, f, c, factor);
    return cudaGetLastError();
}

template <bool PACK, int CAP>
cudaError_t launch_convert(const StepList &s, int first, int count, int sm_count, cudaStream_t stream) {
    ConvertTable<CAP> tab;
    for (int i = 0; i < count; ++i) {
        tab.m[i] = s.m[first + i];
        tab.v[i] = s.v[first + i];
        tab.s[i] = s.s8[first + i];
        tab.vec[i] = aligned(tab.m[i], 16) && aligned(tab.v[i], 16) && state_wide(tab.s[i]);
    }
    tab.count = count;
    const unsigned chunks = fill_chunks(tab.n, tab.chunk_start, s.n + first, count);
    if (chunks == 0) return cudaSuccess;
    state8_convert_kernel<PACK, CAP><<<grid_of(chunks, sm_count, 8), kThreads, 0, stream>>>(tab);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_fold_apply8_multi(const StepList &s, adama_dtype gdt, int first, int count,
                                     FoldConstants f, ApplyConstants c, const float *factor,
                                     int sm_count, cudaStream_t stream) {
    return count <= kStepSmall ? launch_step<kStepSmall>(s, gdt, first, count, f, c, factor, sm_count, stream)
                               : launch_step<kStep8Max>(s, gdt, first, count, f, c, factor, sm_count, stream);
}

cudaError_t launch_state8_convert(const StepList &s, bool pack, int first, int count, int sm_count,
                                  cudaStream_t stream) {
    if (pack)
        return count <= kStepSmall ? launch_convert<true, kStepSmall>(s, first, count, sm_count, stream)
                                   : launch_convert<true, kStep8Max>(s, first, count, sm_count, stream);
    return count <= kStepSmall ? launch_convert<false, kStepSmall>(s, first, count, sm_count, stream)
                               : launch_convert<false, kStep8Max>(s, first, count, sm_count, stream);
}

}  // namespace adama
