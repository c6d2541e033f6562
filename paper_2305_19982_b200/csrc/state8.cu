// Adam moments in 8 bits.  Blocks of kStateBlock consecutive elements share one fp32 scale each:
//     m = M * sm   M: e4m3 (sign, 4 exponent bits, 3 mantissa bits), largest 448
//     v = V * sv   V: unsigned, 5 exponent bits, 3 mantissa bits, (1 + c%8/8) * 2^(c/8 - 31), largest 1.875
// Adam divides m by sqrt(v), element by element, so both need relative, not absolute, precision:
// 1/16 at most for an m of 1/28672 of its block's largest or more (e4m3's normal numbers, 15 binades); below,
// e4m3's subnormals lose precision, and an m under 1/458752 of the largest becomes 0.  For sqrt(v) half of v's
// 1/16, over the 31 binades of v that a block spans.
// A v that is not zero never becomes code 0 (it would divide m by eps alone): the smallest code
// stands in.  The decay of Algorithm 2 multiplies the block's scale and leaves the codes alone:
// 0.999 of a code value would round back to it for ever.
// The update moves 14.06 B/param (bf16 gradients) and is bound by HBM, with the issue slots 70 % busy:
// 405 M parameters take 838 us (6.8 TB/s, just above a copy's rate), 30.7 M with the bf16 copy 80 us
// (6.2 TB/s).
#include <cuda_fp8.h>
#include <float.h>

#include "adama_device.cuh"
#include "bulk_copy.cuh"
#include "tensor_table.cuh"

namespace adama {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPerLane = kStateBlock / 32;                      // elements of a block that one lane holds
constexpr int kBlocks = kChunk / kStateBlock;                   // blocks of a chunk
// A lane holds elements 4*lane .. 4*lane+3 of the block's first half and of its second half: every
// access of a warp is then contiguous (512 bytes of fp32, 256 of bf16, 128 of codes).
constexpr int kHalf = kStateBlock / 2;
static_assert(kPerLane == 8, "two groups of four");
static_assert(kBlocks == 16, "one lane of the producer warp to each of a chunk's scales");

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

// What a lane moves: eight values of four arrays; group h of it lies kHalf*h further on.  In the
// element form value i lies at element lane + 32*i and elements from n on are left alone.
__device__ __forceinline__ uint2 load_codes(const uint8_t *p) {
    return make_uint2(*reinterpret_cast<const unsigned *>(p), *reinterpret_cast<const unsigned *>(p + kHalf));
}
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 c) {
    *reinterpret_cast<unsigned *>(p) = c.x;
    *reinterpret_cast<unsigned *>(p + kHalf) = c.y;
}
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
__device__ __forceinline__ void put4(float (&x)[kPerLane], int h, float4 a) {
    x[4 * h] = a.x;
    x[4 * h + 1] = a.y;
    x[4 * h + 2] = a.z;
    x[4 * h + 3] = a.w;
}
__device__ __forceinline__ void load8(const float *p, float (&x)[kPerLane]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) put4(x, h, ld_stream(reinterpret_cast<const float4 *>(p + kHalf * h)));
}
template <typename G>
__device__ __forceinline__ void load_grads(const G *p, float (&x)[kPerLane]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const Grad4 a = load_grad4(p + kHalf * h, 0);
        put4(x, h, make_float4(a.x, a.y, a.z, a.w));
    }
}
__device__ __forceinline__ void store8(float *p, const float (&x)[kPerLane]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        st_stream(reinterpret_cast<float4 *>(p + kHalf * h), make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]));
}
__device__ __forceinline__ void store_copy(__nv_bfloat16 *p, const float (&x)[kPerLane]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        *reinterpret_cast<uint2 *>(p + kHalf * h) =
            make_uint2(pack2_bf16(x[4 * h], x[4 * h + 1]), pack2_bf16(x[4 * h + 2], x[4 * h + 3]));
}

// One block by one warp: the update of what has been loaded, and the stores.
struct Block8 {
    float g[kPerLane], w[kPerLane];
    uint2 mc, vc;
    float sm, sv;

    __device__ __forceinline__ float2 update(float factor, const FoldConstants &f, const ApplyConstants &c) {
        Lane x;
        x.decode(mc, vc, sm, sv);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) step8_1(__fmul_rn(g[i], factor), w[i], x.m[i], x.v[i], f, c);
        return x.encode(mc, vc);
    }
    __device__ __forceinline__ static void store_scales(const adama_state8 &s, size_t blk, float2 top, int lane,
                                                        const ApplyConstants &c) {
        if (lane == 0) {
            s.m_scale[blk] = __fmul_rn(__fmul_rn(top.x, kMTopInv), c.beta1_hi);
            s.v_scale[blk] = __fmul_rn(__fmul_rn(top.y, kVTopInv), c.beta2_hi);
        }
    }
    // element i0 = the block's first + 4*lane
    __device__ __forceinline__ void store_wide(const adama_state8 &s, float *w_out, __nv_bfloat16 *copy, size_t i0) const {
        store8(w_out + i0, w);
        store_codes(s.m_codes + i0, mc);
        store_codes(s.v_codes + i0, vc);
        if (copy) store_copy(copy + i0, w);
    }
};

// A block straight from global memory, of any length and alignment.
template <typename G>
__device__ __forceinline__ void block_direct(const G *g, float *w, __nv_bfloat16 *copy, const adama_state8 &s, size_t at,
                                             size_t n, bool wide, int lane, float factor, const FoldConstants &f,
                                             const ApplyConstants &c) {
    const size_t blk = at / kStateBlock, i0 = at + 4 * lane;
    Block8 x;
    x.sm = s.m_scale[blk];
    x.sv = s.v_scale[blk];
    if (wide) {
        load_grads(g + i0, x.g);
        load8(w + i0, x.w);
        x.mc = load_codes(s.m_codes + i0);
        x.vc = load_codes(s.v_codes + i0);
    } else {
        x.mc = gather_codes(s.m_codes, at, n, lane);
        x.vc = gather_codes(s.v_codes, at, n, lane);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const size_t j = at + lane + 32 * i;
            x.g[i] = j < n ? widen(g[j]) : 0.f;
            x.w[i] = j < n ? w[j] : 0.f;
        }
    }
    const float2 top = x.update(factor, f, c);
    if (wide) {
        x.store_wide(s, w, copy, i0);
    } else {
        scatter_codes(s.m_codes, at, n, lane, x.mc);
        scatter_codes(s.v_codes, at, n, lane, x.vc);
#pragma unroll
        for (int i = 0; i < kPerLane; ++i) {
            const size_t j = at + lane + 32 * i;
            if (j < n) {
                w[j] = x.w[i];
                if (copy) copy[j] = __float2bfloat16_rn(x.w[i]);
            }
        }
    }
    Block8::store_scales(s, blk, top, lane, c);
}

// Short lists: one warp to a block, straight from global memory.
template <typename G, int CAP>
__global__ void __launch_bounds__(kThreads)
fold_apply8_kernel(const __grid_constant__ Table8<CAP> tab, FoldConstants f, ApplyConstants c,
                   const float *__restrict__ factor_ptr) {
    const float factor = factor_ptr ? *factor_ptr : 1.f;
    if (factor != factor) return;  // a NaN factor (non-finite gradient norm) skips the step
    const unsigned total = tab.chunk_start[tab.count];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (unsigned i = blockIdx.x; i < total * (kBlocks / kWarps); i += gridDim.x) {
        const unsigned chunk = i / (kBlocks / kWarps);
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t n = (size_t)tab.n[t];
        const size_t at = (size_t)(chunk - tab.chunk_start[t]) * kChunk +
                          (size_t)(i % (kBlocks / kWarps) * kWarps + warp) * kStateBlock;
        if (at < n)
            block_direct(static_cast<const G *>(tab.g[t]), tab.w[t], tab.copy[t], tab.s[t], at, n,
                         tab.vec[t] && at + kStateBlock <= n, lane, factor, f, c);
    }
}

// Long lists: a producer warp keeps several chunks' gradients, weights, codes and scales on their way
// to shared memory by bulk copies; each of the other warps takes one block of a chunk.
// Three stages: two Llama-7B-shaped blocks (405 M parameters, bf16 gradients) take 922 us with 2, 839
// with 3, 855 with 4, 870 with 6 (more reads in flight crowd out the writes).
constexpr int kRingStages = 3;
constexpr int kRingWarps = kBlocks;
constexpr int kRingThreads = 32 * (kRingWarps + 1);

template <typename G>
struct Stage8 {
    alignas(16) float w[kChunk];
    alignas(16) G g[kChunk];
    alignas(16) uint8_t m[kChunk], v[kChunk];
    alignas(16) float sm[kBlocks], sv[kBlocks];
};
template <typename G>
struct Ring8 {
    Stage8<G> stage[kRingStages];
    unsigned long long full[kRingStages], empty[kRingStages];
    int tensor[kRingStages];
    int give_up;
};

template <typename G, int CAP>
__global__ void __launch_bounds__(kRingThreads, 1)
fold_apply8_ring_kernel(const __grid_constant__ Table8<CAP> tab, FoldConstants f, ApplyConstants c,
                        const float *__restrict__ factor_ptr, unsigned *status) {
    extern __shared__ unsigned char raw[];
    Ring8<G> &sh = *reinterpret_cast<Ring8<G> *>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    constexpr int kStages = kRingStages;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const float factor = factor_ptr ? *factor_ptr : 1.f;
    if (factor != factor) return;  // a NaN factor (non-finite gradient norm) skips the step
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            barrier_init(shared_addr(&sh.full[i]), 1 + 32);  // the bulk copies, and each lane's scales
            barrier_init(shared_addr(&sh.empty[i]), kRingWarps);
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
    if (warp == kRingWarps) {
        int issued = 0, t = tensor_of_chunk(tab.chunk_start, tab.count, blockIdx.x);
        for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x, advance()) {
            t = tensor_from(tab.chunk_start, t, chunk);
            const size_t first = (size_t)(chunk - tab.chunk_start[t]) * kChunk, left = (size_t)tab.n[t] - first;
            const adama_state8 &s = tab.s[t];
            Stage8<G> &st = sh.stage[slot];
            const uint32_t full = shared_addr(&sh.full[slot]);
            if (issued == kStages && !barrier_wait(shared_addr(&sh.empty[slot]), parity ^ 1, &sh.give_up)) break;
            __syncwarp();
            if (lane == 0) {
                sh.tensor[slot] = t;
                // whole blocks of an aligned tensor; the warps fetch the rest themselves
                const uint32_t blocks = tab.vec[t] ? (uint32_t)(left < kChunk ? left / kStateBlock : kBlocks) : 0;
                const uint32_t k = blocks * kStateBlock;
                barrier_expect(full, k * (6 + (uint32_t)sizeof(G)));
                if (k) {
                    bulk_load(shared_addr(st.w), tab.w[t] + first, 4 * k, full);
                    bulk_load(shared_addr(st.g), static_cast<const G *>(tab.g[t]) + first, k * (uint32_t)sizeof(G), full);
                    bulk_load(shared_addr(st.m), s.m_codes + first, k, full);
                    bulk_load(shared_addr(st.v), s.v_codes + first, k, full);
                }
            }
            const int b = lane % kBlocks;
            if ((size_t)b * kStateBlock < left) {
                if (lane < kBlocks) small_load(shared_addr(st.sm + b), s.m_scale + first / kStateBlock + b);
                else small_load(shared_addr(st.sv + b), s.v_scale + first / kStateBlock + b);
            }
            small_loads_arrive(full);
            if (issued < kStages) ++issued;
        }
        if (*(volatile int *)&sh.give_up) {  // copies in flight end before the CTA does
            small_loads_wait();
            int none = 0;
            for (int i = 0; i < issued; ++i) {
                if (slot == 0) parity ^= 1;
                slot = slot ? slot - 1 : kStages - 1;
                barrier_wait(shared_addr(&sh.full[slot]), parity, &none);
            }
        }
        if (lane == 0) report_expired_wait(&sh.give_up, status, kWaitState8Ring);
        return;
    }
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x, advance()) {
        if (!barrier_wait(shared_addr(&sh.full[slot]), parity, &sh.give_up)) break;  // nothing of this chunk is written
        const int t = sh.tensor[slot];
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kChunk;
        const size_t at = first + (size_t)warp * kStateBlock;
        const adama_state8 s = tab.s[t];
        if (tab.vec[t] && at + kStateBlock <= n) {
            const Stage8<G> &st = sh.stage[slot];
            const int o = warp * kStateBlock + 4 * lane;
            const size_t blk = at / kStateBlock;
            Block8 x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                put4(x.w, h, *reinterpret_cast<const float4 *>(st.w + o + kHalf * h));
                const Grad4 q = shared_grad4(st.g + o + kHalf * h);
                put4(x.g, h, make_float4(q.x, q.y, q.z, q.w));
            }
            x.mc = load_codes(st.m + o);
            x.vc = load_codes(st.v + o);
            x.sm = st.sm[warp];
            x.sv = st.sv[warp];
            // The stage is given back when it has been read, not when its loads have been issued (one that is still on its way
            // when the arrival is seen would find the stage filled anew): at an address that depends on a vote of all lanes
            // (one arrives for its warp, and lanes may run apart) on their weights and on the blocks' largest moments, which
            // gradients, codes and scales have gone into.  The zero is not known to the compiler.
            const unsigned weights = __float_as_uint(x.w[0]) ^ __float_as_uint(x.w[4]), zero = (unsigned)(n >> 63);
            const float2 top = x.update(factor, f, c);
            const unsigned nothing = __any_sync(0xffffffffu, ((weights ^ __float_as_uint(top.x) ^ __float_as_uint(top.y)) & zero) != 0u);
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_addr(&sh.empty[slot]) + nothing);
            x.store_wide(s, tab.w[t], tab.copy[t], at + 4 * lane);
            Block8::store_scales(s, blk, top, lane, c);
        } else {
            __syncwarp();  // every lane is past the wait and has read tensor[slot] before the slot is given back
            if (lane == 0) barrier_arrive(shared_addr(&sh.empty[slot]));
            if (at < n)
                block_direct(static_cast<const G *>(tab.g[t]), tab.w[t], tab.copy[t], s, at, n, false, lane, factor, f, c);
        }
    }
    if (lane == 0) report_expired_wait(&sh.give_up, status, kWaitState8Ring);
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

// fp32 moments -> codes and scales; one warp to a block.
template <int CAP>
__global__ void __launch_bounds__(kThreads)
state8_pack_kernel(const __grid_constant__ ConvertTable<CAP> tab) {
    const unsigned total = tab.chunk_start[tab.count];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (unsigned chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
        const int t = tensor_of_chunk(tab.chunk_start, tab.count, chunk);
        const size_t n = (size_t)tab.n[t], first = (size_t)(chunk - tab.chunk_start[t]) * kChunk;
        const adama_state8 s = tab.s[t];
        const float *m = tab.m[t], *v = tab.v[t];
        for (int b = 0; b < kBlocks / kWarps; ++b) {
            const size_t at = first + (size_t)(warp + b * kWarps) * kStateBlock;
            if (at >= n) break;
            const size_t blk = at / kStateBlock, i0 = at + 4 * lane;
            const bool wide = tab.vec[t] && at + kStateBlock <= n;
            Lane x;
            uint2 mc, vc;
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
        }
    }
}

// Codes and scales -> the values they stand for; one warp to kUnpackBlocks consecutive blocks of a
// chunk.  The next chunk's codes are on their way while this one's values are written.
constexpr int kUnpackBlocks = kBlocks / kWarps;
// 405 M parameters take 651 us (4/5 of it writes) with 3 CTAs per SM, 725 with 2, 713 with 4, 712 with 6,
// 684 without the look-ahead at 8, 690 with the codes streamed through shared memory.
constexpr int kUnpackCtas = 3;

struct UnpackBlocks {
    size_t first, n;  // of the warp's elements; n: where the tensor ends (0: no chunk)
    int t;
    uint2 mc[kUnpackBlocks], vc[kUnpackBlocks];
    float sm[kUnpackBlocks], sv[kUnpackBlocks];

    template <int CAP>
    __device__ __forceinline__ void load(const ConvertTable<CAP> &tab, unsigned chunk, int from, int warp, int lane) {
        t = tensor_from(tab.chunk_start, from, chunk);
        n = (size_t)tab.n[t];
        first = (size_t)(chunk - tab.chunk_start[t]) * kChunk + (size_t)warp * kUnpackBlocks * kStateBlock;
        const adama_state8 &s = tab.s[t];
#pragma unroll
        for (int b = 0; b < kUnpackBlocks; ++b) {
            const size_t at = first + b * kStateBlock, blk = at / kStateBlock;
            if (at < n) {
                const bool wide = tab.vec[t] && at + kStateBlock <= n;
                mc[b] = wide ? load_codes(s.m_codes + at + 4 * lane) : gather_codes(s.m_codes, at, n, lane);
                vc[b] = wide ? load_codes(s.v_codes + at + 4 * lane) : gather_codes(s.v_codes, at, n, lane);
                sm[b] = s.m_scale[blk];
                sv[b] = s.v_scale[blk];
            }
        }
    }
    template <int CAP>
    __device__ __forceinline__ void store(const ConvertTable<CAP> &tab, int lane) const {
        float *m = tab.m[t], *v = tab.v[t];
#pragma unroll
        for (int b = 0; b < kUnpackBlocks; ++b) {
            const size_t at = first + b * kStateBlock;
            if (at >= n) continue;
            Lane x;
            x.decode(mc[b], vc[b], sm[b], sv[b]);
            if (tab.vec[t] && at + kStateBlock <= n) {
                store8(m + at + 4 * lane, x.m);
                store8(v + at + 4 * lane, x.v);
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
};

template <int CAP>
__global__ void __launch_bounds__(kThreads)
state8_unpack_kernel(const __grid_constant__ ConvertTable<CAP> tab) {
    const unsigned total = tab.chunk_start[tab.count];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    unsigned chunk = blockIdx.x;
    if (chunk >= total) return;
    UnpackBlocks a, b;
    a.load(tab, chunk, tensor_of_chunk(tab.chunk_start, tab.count, chunk), warp, lane);
    for (;;) {
        chunk += gridDim.x;
        if (chunk < total) b.load(tab, chunk, a.t, warp, lane);
        a.store(tab, lane);
        if (chunk >= total) return;
        chunk += gridDim.x;
        if (chunk < total) a.load(tab, chunk, b.t, warp, lane);
        b.store(tab, lane);
        if (chunk >= total) return;
    }
}

bool state_wide(const adama_state8 &s) { return aligned(s.m_codes, 16) && aligned(s.v_codes, 16); }

constexpr unsigned kRingFrom = 2;  // chunks per SM from which the ring is used

unsigned grid_of(unsigned chunks, int sm_count, int per_sm) {
    const unsigned cap = (unsigned)(sm_count * per_sm);
    return chunks < cap ? chunks : cap;
}

template <typename G, int CAP>
cudaError_t launch_kernels(const Table8<CAP> &tab, unsigned chunks, FoldConstants f, ApplyConstants c, const float *factor,
                           unsigned *status, int sm_count, cudaStream_t stream) {
    if (chunks < kRingFrom * (unsigned)sm_count) {
        const unsigned ctas = chunks * (kBlocks / kWarps);
        fold_apply8_kernel<G, CAP><<<grid_of(ctas, sm_count, 4), kThreads, 0, stream>>>(tab, f, c, factor);
        return cudaGetLastError();
    }
    constexpr int bytes = (int)sizeof(Ring8<G>) + 128;
    static std::atomic<unsigned long long> ready{0};
    cudaError_t e = allow_shared(fold_apply8_ring_kernel<G, CAP>, bytes, ready);
    if (e != cudaSuccess) return e;
    fold_apply8_ring_kernel<G, CAP><<<grid_of(chunks, sm_count, 1), kRingThreads, bytes, stream>>>(tab, f, c, factor, status);
    return cudaGetLastError();
}

template <int CAP>
cudaError_t launch_step(const StepList &s, adama_dtype gdt, int first, int count, FoldConstants f,
                        ApplyConstants c, const float *factor, unsigned *status, int sm_count,
                        cudaStream_t stream) {
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
    return gdt == ADAMA_F32 ? launch_kernels<float>(tab, chunks, f, c, factor, status, sm_count, stream)
                            : launch_kernels<__nv_bfloat16>(tab, chunks, f, c, factor, status, sm_count, stream);
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
    if (PACK) state8_pack_kernel<CAP><<<grid_of(chunks, sm_count, 8), kThreads, 0, stream>>>(tab);
    else state8_unpack_kernel<CAP><<<grid_of(chunks, sm_count, kUnpackCtas), kThreads, 0, stream>>>(tab);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_fold_apply8_multi(const StepList &s, adama_dtype gdt, int first, int count,
                                     FoldConstants f, ApplyConstants c, const float *factor,
                                     unsigned *status, int sm_count, cudaStream_t stream) {
    if (count <= kStepSmall) return launch_step<kStepSmall>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
    if (count <= kStepMid) return launch_step<kStepMid>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
    return launch_step<kStep8Max>(s, gdt, first, count, f, c, factor, status, sm_count, stream);
}

template <bool PACK>
static cudaError_t convert(const StepList &s, int first, int count, int sm_count, cudaStream_t stream) {
    if (count <= kStepSmall) return launch_convert<PACK, kStepSmall>(s, first, count, sm_count, stream);
    if (count <= kStepMid) return launch_convert<PACK, kStepMid>(s, first, count, sm_count, stream);
    return launch_convert<PACK, kStep8Max>(s, first, count, sm_count, stream);
}

cudaError_t launch_state8_convert(const StepList &s, bool pack, int first, int count, int sm_count,
                                  cudaStream_t stream) {
    return pack ? convert<true>(s, first, count, sm_count, stream) : convert<false>(s, first, count, sm_count, stream);
}

}  // namespace adama
